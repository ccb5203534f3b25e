// Attention of new tokens over the paged key-value cache (sph_attention).
//
// For one kv head, row r = t * group + h is new token t under query head h of the head's group. A workgroup
// takes 16 or 32 rows and a stretch of keys; its waves take tiles of 32 keys in turn, each with a running
// maximum m and sum l per row (o and l scale by exp(m_old - m_new) when m grows), and meet in LDS at the
// end. A long sequence is cut into stretches for several workgroups, whose partial (o, m, l) a second kernel joins in order.
//
// Products are v_mfma_f32_16x16x32_f16. S^T = K Q^T has a row per key and a column per query row: of the tile's two
// products of 16 keys, a lane keeps keys 4 (lane / 16) .. + 3 of each for one row. In O^T = V^T P^T the order of the 32 keys
// is free as long as both operands share it, so the lane's eight weights go into that product where they are, and
// V^T's operand takes the same keys from rows staged in LDS by two transposing reads of four keys each.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "sph_attn.h"

namespace {

constexpr int kTile = 32;                 // keys of a wave's step
constexpr int kEvenBatch = 512;           // sequences that are cut into equal shares

template <int DIM, int BITS>
struct Lay {
  static constexpr int kRowBytes = DIM * BITS / 8;
  // bytes of a key row that one of its four lanes loads at once
  static constexpr int kPiece = kRowBytes % 64 == 0 ? 16 : kRowBytes % 32 == 0 ? 8 : 4;
  static constexpr int kLoads = kRowBytes / (4 * kPiece);
  static constexpr int kPieceCh = kPiece * 8 / BITS;
  static constexpr int kSteps = DIM / 32;
  static constexpr int kBlocks = kPieceCh / 8;              // products of a piece
  // a value row's pieces: eight fp16 channels or 16 codes (eight where 16 rows of pieces would not be whole loads), loaded
  // by half tiles of 16 rows
  static constexpr int kVCh = BITS == 16 || DIM % 64 == 32 ? 8 : 16;
  static constexpr int kVPiece = kVCh * BITS / 8;
  static constexpr int kVPer = DIM / kVCh;
  static constexpr int kVLoads = 16 * kVPer / 64;
  static_assert(16 * kVPer % 64 == 0, "whole loads");
  __device__ static __forceinline__ int v_row(int lane, int i) {
    return 64 % kVPer ? (lane + 64 * i) / kVPer : lane / kVPer + i * (64 / kVPer);
  }
  __device__ static __forceinline__ int v_piece(int lane, int i) { return 64 % kVPer ? (lane + 64 * i) % kVPer : lane % kVPer; }
  static constexpr int kVStride = DIM * 2 + 32;             // bytes between rows in LDS: four rows' transposed read hits all banks
};

// A wave's loads of one tile of keys, as they come from memory.
template <int DIM, int BITS>
struct Tile {
  typedef Lay<DIM, BITS> L;
  uint32_t k[2][L::kLoads][L::kPiece / 4], v[2 * L::kVLoads][L::kVPiece / 4];
  uint32_t k_par[2][L::kLoads], v_par[2 * L::kVLoads];
};

// Where a tile's rows are. Pages of 16 tokens and more (UNI): each half of the tile lies in one page, so a scalar buffer
// descriptor holds its address, and a lane's 32-bit offset into it stays the same from tile to tile. Smaller pages: lane l % 32 holds
// the offsets of key l % 32, and the lanes that load a part of its row fetch them by a shuffle.
template <bool UNI>
struct Rows {
  int64_t off[2], par_off[2];
  // page: lane l holds the page of key kt + l % 32
  __device__ __forceinline__ void set(const Pages& pg, int page, int kt, int lane, bool par) {
    if constexpr (UNI) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int p = __builtin_amdgcn_readlane(page, 16 * h), in_page = (kt + 16 * h) & pg.mask;
        off[h] = p * pg.stride + (uint32_t)(in_page * pg.token);
        if (par) par_off[h] = p * pg.par_stride + (uint32_t)(in_page * pg.par_token);
      }
    } else {
      const int in_page = (kt + (lane & 31)) & pg.mask;
      off[0] = page * pg.stride + (uint32_t)(in_page * pg.token);
      if (par) par_off[0] = page * pg.par_stride + (uint32_t)(in_page * pg.par_token);
    }
  }
  __device__ __forceinline__ static int64_t shuffled(int64_t v, int from) {
    return (int64_t)(uint32_t)__shfl((int)(uint32_t)v, from) | (int64_t)__shfl((int)(v >> 32), from) << 32;
  }
};

// Words of rows of one half of a tile: of row `row`, which is `lane_row` + a constant, from byte `byte` on. STREAM: not to be kept in caches.
template <int BYTES, bool UNI, bool STREAM = false>
__device__ __forceinline__ void load_row(const char* base, const int64_t* off, int token, int half, int lane_row, int row, int byte, uint32_t* w) {
  if constexpr (UNI) {
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void*)(base + off[half]), 0, 16 * token, 0x00020000);
    constexpr int kAux = STREAM ? 2 : 0;
    const int voff = lane_row * token + byte, soff = (row - lane_row) * token;
    if constexpr (BYTES == 16) {
      const u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(r, voff, soff, kAux);
      w[0] = v[0], w[1] = v[1], w[2] = v[2], w[3] = v[3];
    } else if constexpr (BYTES == 8) {
      const u32x2 v = __builtin_amdgcn_raw_buffer_load_b64(r, voff, soff, kAux);
      w[0] = v[0], w[1] = v[1];
    } else {
      w[0] = __builtin_amdgcn_raw_buffer_load_b32(r, voff, soff, kAux);
    }
  } else {
    load_words<BYTES, STREAM>(base + Rows<false>::shuffled(off[0], 16 * half + row) + byte, w);
  }
}

template <int DIM, int BITS, bool UNI>
__device__ __forceinline__ void load_keys(Tile<DIM, BITS>& t, const Pages& pg, const Rows<UNI>& rows, int lane) {
  typedef Lay<DIM, BITS> L;
  const int col = lane & 15, g4 = lane >> 4;
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int i = 0; i < L::kLoads; ++i) {
      load_row<L::kPiece, UNI>(pg.k, rows.off, pg.token, u, col, col, (4 * i + g4) * L::kPiece, t.k[u][i]);
      if constexpr (BITS < 16)
        load_row<4, UNI>(pg.k_par, rows.par_off, pg.par_token, u, col, col, g4 * L::kPieceCh / 32 * 4 + i * L::kPieceCh / 8 * 4, &t.k_par[u][i]);
    }
}

// A load of values takes whole lines, which nobody reads again in this call; the keys' take halves of lines.
template <int DIM, int BITS, bool UNI, bool STREAM>
__device__ __forceinline__ void load_values(Tile<DIM, BITS>& t, const Pages& pg, const Rows<UNI>& rows, int lane) {
  typedef Lay<DIM, BITS> L;
#pragma unroll
  for (int i = 0; i < 2 * L::kVLoads; ++i) {
    const int half = i / L::kVLoads, row = L::v_row(lane, i % L::kVLoads), piece = L::v_piece(lane, i % L::kVLoads);
    const int lane_row = 64 % L::kVPer ? row : lane / L::kVPer;
    load_row<L::kVPiece, UNI, STREAM>(pg.v, rows.off, pg.token, half, lane_row, row, piece * L::kVPiece, t.v[i]);
    if constexpr (BITS < 16)
      load_row<4, UNI>(pg.v_par, rows.par_off, pg.par_token, half, lane_row, row, piece * L::kVCh / 32 * 4, &t.v_par[i]);
  }
}

// Inclusive sum over the lanes of a wave: within rows of 16 by shifts, then the rows' last lanes to the rows behind.
__device__ __forceinline__ int wave_scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);
  return v;
}

// Tiles c_lo .. c_hi - 1 of sequence b, as seen from the first that its rows see, under one kv head: its rows' outputs, or their part
// `slot`.
//
// What bounds it: HBM reads of the pages, for short sequences the latency of the steps of a wave one after the other. Each wave keeps one
// tile of keys and values in flight in registers while it works on the one before; the 16 rows that a product has cost the same
// whether one query head or 16 share the kv head. The page numbers of a tile are loaded two tiles ahead.
// 32 query heads over 8 kv heads of 128 channels: one sequence of 131072 tokens in fp16 87 us (6.2 TB/s), 64 of up to 8192 at 8 bits
// 78 us (5.2 TB/s), 16 of 32768 under 40 query heads at 4 bits 124 us (5.4 TB/s: the vector ALU, which decodes, is 54% busy beside the reads); one
// of 517 tokens 11.3 us (512 tokens 9.4, one 5.8).
template <int DIM, int BITS, int NB, bool UNI>
__device__ __forceinline__ void attend(const AttnArgs& a, char* lds, float2 (*ml_s)[16 * NB], int kvh, int b, int c_lo, int c_hi, int slot) {
  typedef Lay<DIM, BITS> L;
  constexpr int kRows = 16 * NB, kVBytes = kTile * L::kVStride, kOStride = DIM + 4;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, g4 = lane >> 4;
  Seq s;
  s.load(a, b);
  if (s.bad) {
    write_bad(a, s, kvh);
    return;
  }
  if (s.n == 0) return;
  const int nrow = s.n * a.group;
  const int first = s.len - s.n;                            // position of the first new token
  const int p_lo = first, p_hi = s.len - 1;                 // positions of the rows
  const int lo = a.window ? max(0, p_lo - a.window + 1) : 0, hi = s.len;
  const int k_lo = max(lo, (lo & ~(kTile - 1)) + c_lo * kTile), k_hi = min(hi, (lo & ~(kTile - 1)) + c_hi * kTile);
  const Span span = {k_lo, k_hi, p_lo, p_hi, a.window, kTile};
  const int32_t* pages = a.pages + b * a.pages_stride;
  Pages pg;
  pg.set(a.c, kvh);

  int pos[NB];
  bool odd = false;
  f32x4 o[NB][DIM / 16] = {};
  Ref ref[NB];
  float l[NB];
#pragma unroll
  for (int n = 0; n < NB; ++n) ref[n] = {-INFINITY, 0.0f}, l[n] = 0.0f;
  const int t0 = (k_lo & ~(kTile - 1)) + kTile * wave;
  if (t0 < k_hi) {
    f16x8 q[NB][L::kSteps];
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      const int r = min(16 * n + col, nrow - 1), t = r / a.group, h = kvh * a.group + r % a.group;
      pos[n] = first + t;
      const char* qr = a.q + (s.start + t) * a.qt + h * a.qh;
#pragma unroll
      for (int i = 0; i < L::kLoads; ++i)
#pragma unroll
        for (int j = 0; j < L::kBlocks; ++j)
          q[n][i * L::kBlocks + j] = *(const f16x8*)(qr + 2 * ((4 * i + g4) * L::kPieceCh + 8 * j));
    }
    const int e_lo = k_lo >> pg.shift, e_hi = (k_hi - 1) >> pg.shift;
    // keys outside the stretch take a page inside it: their rows are read and not used
    auto page_of = [&](int kt) { return pages[min(max((kt + (lane & 31)) >> pg.shift, e_lo), e_hi)]; };
    char* vs = lds + wave * kVBytes;

    Tile<DIM, BITS> T;
    int kt = t0, nt = t0 + kTile * kWaves < k_hi ? t0 + kTile * kWaves : t0;
    int page = page_of(kt), next = page_of(nt);
    uint64_t gone = __ballot(!pg.there(page));
    page = pg.there(page) ? page : 0;
    Rows<UNI> at;
    at.set(pg, page, kt, lane, BITS < 16);
    load_keys<DIM, BITS, UNI>(T, pg, at, lane);
    auto load_v = [&]() {
      if (a.stream)
        load_values<DIM, BITS, UNI, true>(T, pg, at, lane);
      else
        load_values<DIM, BITS, UNI, false>(T, pg, at, lane);
    };
    load_v();
    while (true) {
      const bool last = kt + kTile * kWaves >= k_hi;
      // every row sees the whole tile
      const bool whole = span.whole(kt) && !gone;
      const uint64_t next_gone = __ballot(!pg.there(next));
      page = pg.there(next) ? next : 0;
      at.set(pg, page, nt, lane, BITS < 16);
      // scores
      f32x4 st[NB][2] = {};
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < L::kLoads; ++i)
#pragma unroll
          for (int j = 0; j < L::kBlocks; ++j) {
            f16x8 kv;
            if constexpr (BITS == 16)
              kv = __builtin_bit_cast(f16x8, make_uint4(T.k[u][i][0], T.k[u][i][1], T.k[u][i][2], T.k[u][i][3]));
            else if constexpr (BITS == 8)
              kv = decode8w<8>(T.k[u][i][2 * j], T.k[u][i][2 * j + 1], T.k_par[u][i]);
            else
              kv = decode8w<4>(T.k[u][i][j], 0, T.k_par[u][i]);
#pragma unroll
            for (int n = 0; n < NB; ++n) st[n][u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kv, q[n][i * L::kBlocks + j], st[n][u], 0, 0, 0);
          }
      // not above the products: the loads would take registers of their own beside those that they refill
      __builtin_amdgcn_sched_barrier(0);
      load_keys<DIM, BITS, UNI>(T, pg, at, lane);
      __builtin_amdgcn_sched_barrier(0);
      // values into LDS
#pragma unroll
      for (int i = 0; i < 2 * L::kVLoads; ++i) {
        const int kk = i / L::kVLoads * 16 + L::v_row(lane, i % L::kVLoads), piece = L::v_piece(lane, i % L::kVLoads);
        f16x8 v[L::kVCh / 8];
#pragma unroll
        for (int j = 0; j < L::kVCh / 8; ++j) {
          if constexpr (BITS == 16)
            v[j] = __builtin_bit_cast(f16x8, make_uint4(T.v[i][0], T.v[i][1], T.v[i][2], T.v[i][3]));
          else if constexpr (BITS == 8)
            v[j] = decode8w<8>(T.v[i][2 * j], T.v[i][2 * j + 1], T.v_par[i]);
          else
            v[j] = decode8w<4>(T.v[i][j], 0, T.v_par[i]);
        }
#pragma unroll
        for (int j = 0; j < L::kVCh / 8; ++j) *(f16x8*)(vs + kk * L::kVStride + (piece * L::kVCh + 8 * j) * 2) = v[j];
      }
      __builtin_amdgcn_sched_barrier(0);
      load_v();
      __builtin_amdgcn_sched_barrier(0);
      const int nnt = nt + kTile * kWaves < k_hi ? nt + kTile * kWaves : nt;
      next = page_of(nnt);
      f16x8 p[NB];
      bool rise = false;
      float x[NB][8], top[NB];
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        top[n] = -INFINITY;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[n][i] = st[n][i >> 2][i & 3] * a.scale;
        if (!whole) {
          // (opaque here: a branch stays, and what its tests compare with is not kept in registers around the loop)
          int at_pos = pos[n], key = kt + 4 * g4;
          uint32_t lost = (uint32_t)gone >> (4 * g4);
          asm volatile("" : "+v"(at_pos), "+v"(key), "+v"(lost));
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int kk = 16 * (i >> 2) + (i & 3);
            x[n][i] = !span.seen(key + kk, at_pos) ? -INFINITY : (lost >> kk & 1) ? __builtin_nanf("") : x[n][i];
          }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) top[n] = fmaxf(top[n], x[n][i]);
        rise |= top[n] > ref[n].top;
      }
      if (__any(rise)) {
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          float mn = top[n];
          mn = fmaxf(mn, __shfl_xor(mn, 16));
          mn = fmaxf(mn, __shfl_xor(mn, 32));
          float keep;
          if (!ref[n].raise(mn, keep)) continue;
          l[n] *= keep;
#pragma unroll
          for (int i = 0; i < DIM / 16; ++i) o[n][i] *= keep;
        }
      }
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          // of the rounded score, as the reference was: not fused with its product
#pragma clang fp contract(off)
          x[n][i] = __builtin_amdgcn_exp2f(x[n][i] - ref[n].base);
          l[n] += x[n][i];
          p[n][i] = (_Float16)x[n][i];
        }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      if (!whole) {
        // A weight of 0 does not hide an infinity or a NaN in a value that its row does not see: values that no row sees
        // become zeros here, and so do infinities and NaN, which the rows that see them get at the end.
#pragma unroll 2
        for (int i = lane; i < kTile * (DIM / 8); i += 64) {
          const int kk = i / (DIM / 8);
          odd |= clean_piece(vs + kk * L::kVStride + i % (DIM / 8) * 16, kt + kk < k_lo || kt + kk >= k_hi || (gone >> kk & 1));
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
      }
#pragma unroll
      for (int i = 0; i < DIM / 16; ++i) {
        f16x8 vt;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const s16x4 w = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (__attribute__((address_space(3))) s16x4*)(vs + (16 * j + 4 * g4 + (col >> 2)) * L::kVStride + 32 * i + 8 * (col & 3)));
          const f16x4 f = __builtin_bit_cast(f16x4, w);
#pragma unroll
          for (int e = 0; e < 4; ++e) vt[4 * j + e] = f[e];
        }
#pragma unroll
        for (int n = 0; n < NB; ++n) o[n][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vt, p[n], o[n][i], 0, 0, 0);
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      if (last) break;
      kt = nt;
      nt = nnt;
      gone = next_gone;
    }
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      l[n] += __shfl_xor(l[n], 16);
      l[n] += __shfl_xor(l[n], 32);
    }
  }

  // the waves' parts meet
  const bool any_odd = __syncthreads_or(odd);
  float* os = (float*)lds + wave * kRows * kOStride;
#pragma unroll
  for (int n = 0; n < NB; ++n) {
    if (g4 == 0) ml_s[wave][16 * n + col] = make_float2(ref[n].log(), l[n]);
#pragma unroll
    for (int i = 0; i < DIM / 16; ++i) *(f32x4*)(os + (16 * n + col) * kOStride + 16 * i + 4 * g4) = o[n][i];
  }
  __syncthreads();
  for (int i = threadIdx.x; i < nrow * (DIM / 4); i += kThreads) {
    const int row = i / (DIM / 4), ch = i % (DIM / 4) * 4;
    float mm = ml_s[0][row].x;
#pragma unroll
    for (int w = 1; w < kWaves; ++w) mm = fmaxf(mm, ml_s[w][row].x);
    const float ref = mm == -INFINITY ? 0.0f : mm;
    f32x4 acc = {};
    float ll = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float f = __builtin_amdgcn_exp2f(ml_s[w][row].x - ref);
      ll += f * ml_s[w][row].y;
      acc += f * *(const f32x4*)((float*)lds + (w * kRows + row) * kOStride + ch);
    }
    if (any_odd) acc += odd_values<DIM, BITS>(span, pg, pages, first + row / a.group, ch);
    if (slot < 0)
      write_out(a, s.start + row / a.group, kvh * a.group + row % a.group, ch, acc, mm, ll);
    else
      write_part(a, slot, kvh, row, ch, acc, mm, ll);
  }
}

// Inclusive sums over all sequences' counts: before[b + 1] = counts of 0 .. b. Returns their total.
__device__ __forceinline__ int scan_counts(const int* counts, int rounds, int* before, int* sums) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int mine[kEvenBatch / kThreads] = {};
#pragma unroll
  for (int i = 0; i < kEvenBatch / kThreads; ++i) {
    if (i < rounds) {
      mine[i] = wave_scan(counts[i]);
      if (lane == 63) sums[i * kWaves + wave] = mine[i];
    }
  }
  if (threadIdx.x == 0) before[0] = 0;
  __syncthreads();
  int total = 0;
#pragma unroll
  for (int i = 0; i < kEvenBatch / kThreads; ++i) {
    if (i < rounds) {
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        if (w == wave) before[threadIdx.x + i * kThreads + 1] = total + mine[i];
        total += sums[i * kWaves + w];
      }
    }
  }
  __syncthreads();
  return __builtin_amdgcn_readfirstlane(total);
}

// The sequence whose counts hold place `at`.
__device__ __forceinline__ int find_count(int at, int rounds, const int* before, int* sums) {
  for (int i = 0; i < rounds; ++i) {
    const int b = threadIdx.x + i * kThreads;
    if (before[b] <= at && at < before[b + 1]) sums[0] = b;
  }
  __syncthreads();
  return __builtin_amdgcn_readfirstlane(sums[0]);
}

template <int DIM, int BITS, int NB, bool UNI>
__global__ __launch_bounds__(kThreads, (DIM * NB <= 64 ? 3 : DIM * NB <= 128 ? (BITS == 4 ? 3 : 2) : 1)) void k_attn(AttnArgs) {
  // read where they are used: kept for the whole kernel, the arguments would push the loop's scalars out of their registers
  const AttnArgs& a = *(const AttnArgs*)__builtin_amdgcn_kernarg_segment_ptr();
  constexpr int kRows = 16 * NB, kVBytes = kTile * Lay<DIM, BITS>::kVStride, kOBytes = kRows * (DIM + 4) * 4;
  __shared__ __attribute__((aligned(16))) char lds[kWaves * (kVBytes > kOBytes ? kVBytes : kOBytes)];
  __shared__ float2 ml_s[kWaves][kRows];
  __shared__ int before[kEvenBatch + 1], sums[kEvenBatch / 32];
  const int kvh = blockIdx.x % a.c.kv_heads, share = blockIdx.x / a.c.kv_heads;
  int b = share, c_lo = 0, c_hi = (1 << 30) / kTile, slot = -1;
  int at = 0, end = 0, per = 0;
  if (a.shares) {
    const int rounds = (a.batch + kThreads - 1) / kThreads;
    int tiles[kEvenBatch / kThreads] = {};
#pragma unroll
    for (int i = 0; i < kEvenBatch / kThreads; ++i) {
      const int bb = threadIdx.x + i * kThreads;
      if (bb < a.batch) {
        Seq s;
        s.load(a, bb);
        tiles[i] = s.tiles(a.window);
      }
    }
    const int total = scan_counts(tiles, rounds, before, sums);
    if (a.shares >= 2 * a.batch) {
      // Shares to spare: each is a stretch of one sequence, ceil(tiles / per) stretches a sequence. This many tiles always suffice:
      per = max(kWaves, (total + a.shares - a.batch - 1) / (a.shares - a.batch));
      // Where that is a wave's step above the mean or more, the least of four smaller numbers that does, too (16 sequences of 32768 tokens at 4 bits
      // under 40 query heads 130 us, without 139; one, two or three long sequences within 1%).
      if ((int64_t)total * a.batch > (int64_t)kWaves * a.shares * (a.shares - a.batch)) {
        constexpr int kTry[4] = {8, 9, 10, 12};              // eighths of the mean
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const int each = (int)(((int64_t)total * kTry[t] + 8 * a.shares - 1) / (8 * a.shares));
          int need = 0;
#pragma unroll
          for (int i = 0; i < kEvenBatch / kThreads; ++i) need += (tiles[i] + each - 1) / each;
          need = wave_scan(need);
          if ((threadIdx.x & 63) == 63) sums[t * kWaves + (threadIdx.x >> 6)] = need;
        }
        static_assert(4 * kWaves <= kEvenBatch / 32, "sums");
        __syncthreads();
#pragma unroll
        for (int t = 3; t >= 0; --t) {
          int need = 0;
#pragma unroll
          for (int w = 0; w < kWaves; ++w) need += sums[t * kWaves + w];
          if (__builtin_amdgcn_readfirstlane(need) <= a.shares) per = min(per, (int)(((int64_t)total * kTry[t] + 8 * a.shares - 1) / (8 * a.shares)));
        }
        __syncthreads();
      }
#pragma unroll
      for (int i = 0; i < kEvenBatch / kThreads; ++i) tiles[i] = (tiles[i] + per - 1) / per;
      if (share >= scan_counts(tiles, rounds, before, sums)) return;
      b = find_count(share, rounds, before, sums);
      const int lo = __builtin_amdgcn_readfirstlane(before[b]), n = __builtin_amdgcn_readfirstlane(before[b + 1]) - lo;
      Seq s;
      s.load(a, b);
      const int64_t all = s.tiles(a.window);
      c_lo = (int)((share - lo) * all / n), c_hi = (int)((share - lo + 1) * all / n);
      if (n > 1) slot = share;
      if (share == lo && kvh == 0 && threadIdx.x == 0) a.where[b] = make_int2(lo, n);
    } else {
      // The tiles of all sequences in a row, cut into equal shares, which may hold the end of one sequence and the start of the next.
      per = max(kWaves, (total + a.shares - 1) / a.shares);
      at = share * per, end = min(total, at + per);
      if (at >= total) return;
      b = find_count(at, rounds, before, sums);
    }
  }
  while (true) {
    if (at < end) {
      int lo, hi;
      while ((lo = __builtin_amdgcn_readfirstlane(before[b])) == (hi = __builtin_amdgcn_readfirstlane(before[b + 1]))) ++b;  // no queries
      c_lo = at - lo, c_hi = min(end, hi) - lo;
      at = lo + c_hi;
      const int s_lo = lo / per, s_hi = (hi - 1) / per;
      slot = s_lo == s_hi ? -1 : share + b;
      if (c_lo == 0 && kvh == 0 && threadIdx.x == 0) a.where[b] = make_int2(s_lo + b, s_hi - s_lo + 1);
    }
    attend<DIM, BITS, NB, UNI>(a, lds, ml_s, kvh, b, c_lo, c_hi, slot);
    if (at >= end) return;
    ++b;
    __syncthreads();
  }
}

constexpr int kMaxSplits = 512, kJoinCh = 32, kFewParts = 8;

// Joins the parts of a row. Where a row may have many, a wave takes 32 channels of it: each group of eight lanes adds every eighth part
// in order, and the groups' sums are added. Where rows are many and have few parts (FEW), a wave takes a whole row. (One way for
// both cost: 96 parts of 32 rows 5 us against 11 by whole rows; 2 parts of 32000 rows 14 us against 58 by 32 channels.)
// A part without a seen key has l = 0.
template <bool FEW>
__global__ __launch_bounds__(kThreads) void k_attn_join(AttnArgs a) {
  const int lane = threadIdx.x & 63;
  const uint32_t per = FEW ? a.c.dim / 4 : kJoinCh / 4, groups = 64 / per, chunks = FEW ? 1 : a.c.dim / kJoinCh, rows = a.max_q * a.group;
  uint32_t id = blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (id >= chunks * a.c.kv_heads * rows * a.batch) return;
  const uint32_t group = lane / per, ch = id % chunks * kJoinCh + lane % per * 4;
  id /= chunks;
  const int kvh = id % a.c.kv_heads;
  id /= a.c.kv_heads;
  const int row = id % rows, b = id / rows;
  Seq s;
  s.load(a, b);
  if (s.bad || row >= s.n * a.group) return;
  // k_attn's parts follow each other, k_attn_wide's are `batch` apart
  int slot = b, apart = a.batch, parts = a.splits;
  if (a.shares) {
    const int2 w = a.where[b];
    slot = w.x, apart = 1, parts = w.y;
    if (parts == 1) return;                                  // written already
  }
  const int64_t first = part_at(a, slot, kvh, row), step = part_at(a, slot + apart, kvh, row) - first;
  float mm = -INFINITY;
  for (int p = lane; p < parts; p += 64) mm = fmaxf(mm, a.ml[first + p * step].x);
#pragma unroll
  for (int d = 32; d; d >>= 1) mm = fmaxf(mm, __shfl_xor(mm, d));
  const float ref = mm == -INFINITY ? 0.0f : mm;
  f32x4 acc = {};
  float l = 0.0f;
  if (group < groups) {
#pragma unroll 4
    for (int p = group; p < parts; p += groups) {
      const int64_t at = first + p * step;
      const float2 ml = a.ml[at];
      const f32x4 part = *(const f32x4*)(a.part + at * a.c.dim + ch);
      const float f = __builtin_amdgcn_exp2f(ml.x - ref);
      l += f * ml.y;
      acc += f * part;
    }
  }
  // the groups' sums, in order, to the first
  for (uint32_t g = 1; g < groups; ++g) {
    const float more = __shfl(l, (int)(g * per + lane % per));
    l += group ? 0.0f : more;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float x = __shfl(acc[i], (int)(g * per + lane % per));
      acc[i] += group ? 0.0f : x;
    }
  }
  if (group == 0) write_out(a, s.start + row / a.group, kvh * a.group + row % a.group, ch, acc, mm, l);
}

// ------------------------------------------------------------------ host side

struct Plan {
  int wide, nb, splits, chunk, shares, fold, window;
  int64_t tiles;                           // (up to 2^33 before the launch is refused)
  int64_t grid, joins;                     // workgroups; waves of the join
  bool few;                                // k_attn_join's form
  size_t parts;                            // rows of partial sums
  size_t bytes;
};

// k_attn: a workgroup a sequence and kv head where sequences are short (a few tiles a wave; joining would cost as much) or so many
// that they fill the chip; otherwise as many workgroups as are resident at once, with equal shares of all keys.
// k_attn_wide: stretches of at least four tiles where the rows alone would leave the chip idle.
constexpr int kCus = 256;

// Pools that the last cache before memory cannot hold are read past it (values: see load_values). One sequence of 131072 tokens in fp16 86 us
// instead of 95, 64 of up to 8192 at 8 bits 78 instead of 82; a pool of 41 MB that stays in that cache from call to call 26 instead of 24.
constexpr int64_t kLastCache = 256 << 20;

// Workgroups of k_attn on a CU: as many as keep about 64 KiB of pages on their way to it, a tile a wave. More lengthen the queue that every
// dependent load waits in, or wait for registers: 64 ragged sequences of up to 8192 tokens at 8 bits take 98, 78 and 95 us with one, two and three
// workgroups a CU; 16 of 32768 tokens at 4 bits 195, 135 and 123; one of 131072 tokens in fp16 86, 88 and 90, and its join 4.7, 5.9 and 6.9.
int workgroups_per_cu(const sph_kv_cache* c) {
  const int tile = kTile * 2 * c->head_dim * c->bits / 8;
  return std::max(1, std::min(3, (64 << 10) / (kWaves * tile)));
}

Plan plan_of(const sph_kv_cache* c, int64_t batch, int q_heads, int64_t max_q, int64_t max_len, int64_t window) {
  Plan p{};
  // one that hides nothing is none (and positions minus a window stay inside 32 bits)
  p.window = window > max_len ? 0 : (int)window;
  window = p.window;
  const int group = q_heads / c->kv_heads;
  const int64_t rows = max_q * group;
  // two blocks of rows of wider heads do not fit the registers
  p.nb = rows <= 16 || c->head_dim > 128 ? 1 : 2;
  p.wide = rows > 16 * p.nb;
  p.splits = 1;
  int64_t slots = 0;
  if (!p.wide) {
    p.tiles = 1;
    const int64_t span = window > 0 ? std::min<int64_t>(max_len, window + max_q + kTile) : max_len;
    // Short: up to 6 tiles of 128 channels a wave, or 16 where sequences and heads give half the CUs a workgroup, since the counting
    // of shares and their join cost about 8 us and such calls gain little from a few more workgroups. 8 kv heads, fp16, direct against
    // shares and join: one sequence of 512 keys 9.4 and 12.2 us, 768 11.9 and 11.9, 1024 14.5 and 12.3; 16 ragged ones of up to 1024
    // 16.0 and 17.6, 2048 24.5 and 23.5; 64 of up to 2048 52.8 and 54.4. 64 channels: one of 1536 12.2 and 11.8; 256: one of 384 14.4 and 15.4.
    const int64_t steps = (2 * batch * c->kv_heads >= kCus ? 16 : 6) * 128;
    const int64_t rounds = steps / c->head_dim;
    if (batch <= kEvenBatch && span > kTile * kWaves * rounds && batch * (span / kTile + 2) < (1 << 30)) {
      p.shares = (int)std::min<int64_t>(kMaxSplits - 1, std::max<int64_t>(1, kCus * workgroups_per_cu(c) / c->kv_heads));
      p.shares = (int)std::min<int64_t>(p.shares, batch * ((span + kTile * kWaves - 1) / (kTile * kWaves) + 1));
      slots = p.shares + batch;
    }
  } else {
    p.tiles = (rows + kWideRows - 1) / kWideRows;
    const int64_t tile = sph_attn_wide_tile(c->head_dim), step = 4 * tile;
    const int64_t span = window > 0 ? std::min<int64_t>(max_len, window + kWideRows / group + 1 + tile) : max_len;
    // None where the rows alone give half the CUs a workgroup: two parts save less than their join costs (900 rows of one prompt 35 us,
    // in two parts 33 + 17). Otherwise two a CU, and four where sequences are several, since ragged ones leave many with little
    // to do (8 of up to 8000 tokens, 40 of each new: 67 + 6 us with two, 40 + 7 with four).
    const int64_t units = c->kv_heads * batch * p.tiles, per_cu = batch > 1 ? 4 : 2;
    const int64_t want = 2 * units > kCus ? 1 : std::min<int64_t>(kMaxSplits, per_cu * kCus / units);
    p.chunk = (int)std::max<int64_t>(step, ((span + want - 1) / want + step - 1) / step * step);
    p.splits = (int)std::max<int64_t>(1, (span + p.chunk - 1) / p.chunk);
    if (p.splits > 1) slots = p.splits * batch;
    // All workgroups resident at once, two on some CUs (the i-th and the (i + 256)-th; of 64 channels a CU takes more, of 192 one): long
    // rows share theirs with short ones. 8 kv heads of 128 channels, so and with the longest first, fp16: prompts of 2048 tokens 62.0 and 65.0 us,
    // 1536 46.3 and 47.9, four of 512 26.8 and 30.1, 1300 behind 6700 others 236 and 243; four of 500 at 8 bits 30.7 and 35.6; 2048 of 96
    // channels 51.1 and 52.6, of 64 43.2 and 43.3.
    if (c->head_dim > 64 && c->head_dim <= 128 && p.splits == 1 && kCus % c->kv_heads == 0 && units > kCus && units <= 2 * kCus)
      p.fold = kCus / c->kv_heads;
  }
  p.parts = (size_t)slots * c->kv_heads * rows;
  if (slots) p.bytes = p.parts * (c->head_dim + 2) * sizeof(float) + (size_t)batch * sizeof(int2);
  const int64_t heads = c->kv_heads, all = heads * batch * rows;
  p.grid = p.wide ? heads * batch * p.tiles * p.splits : heads * (p.shares ? p.shares : batch);
  // k_attn_wide's parts are few, and k_attn's where sequences share a workgroup rather than the other way round
  p.few = p.wide ? p.splits <= kFewParts : 2 * batch > p.shares && p.shares <= kFewParts * batch;
  p.joins = p.few ? all : all * (c->head_dim / kJoinCh);
  return p;
}

// Whether launches take it (and rows of a sequence fit 32 bits).
bool launchable(const Plan& p) { return p.grid < (1 << 24) && (!p.bytes || p.joins < (1 << 26)); }

sph_status check_sizes(const sph_kv_cache* c, int64_t batch, int64_t tokens, int32_t q_heads, int64_t max_q, int64_t max_len,
                       int64_t window) {
  if (!c) return SPH_ERR_NULL;
  if (const int st = sph_cache_check(c)) return (sph_status)st;
  if (batch < 0 || batch > 65536 || tokens < 0 || tokens > (1 << 26) || q_heads < 1 || q_heads > 65535 || q_heads % c->kv_heads ||
      max_q < 1 || max_q > (1 << 24) || max_len < 0 || max_len > (1 << 30) || window < 0)
    return SPH_ERR_SHAPE;
  return SPH_OK;
}

template <int BITS, int NB, bool UNI>
const void* kernel_for(int dim) {
  if (dim == 64) return (const void*)k_attn<64, BITS, NB, UNI>;
  if (dim == 96) return (const void*)k_attn<96, BITS, NB, UNI>;
  if (dim == 128) return (const void*)k_attn<128, BITS, NB, UNI>;
  if constexpr (NB == 1) return dim == 192 ? (const void*)k_attn<192, BITS, 1, UNI> : (const void*)k_attn<256, BITS, 1, UNI>;
  return nullptr;
}

template <int NB, bool UNI>
const void* kernel_for(int bits, int dim) {
  return bits == 16 ? kernel_for<16, NB, UNI>(dim) : bits == 8 ? kernel_for<8, NB, UNI>(dim) : kernel_for<4, NB, UNI>(dim);
}

bool launch_ok(const void* fn, dim3 grid, hipStream_t s, AttnArgs& a) {
  void* kargs[] = {(void*)&a};
  return hipLaunchKernel(fn, grid, dim3(kThreads), kargs, 0, s) == hipSuccess && hipGetLastError() == hipSuccess;
}

}  // namespace

extern "C" {

sph_status sph_attention_workspace_bytes(const sph_kv_cache* cache, int64_t batch, int64_t tokens, int32_t q_heads,
                                         int64_t max_q, int64_t max_len, int64_t window, size_t* bytes) {
  if (!bytes) return SPH_ERR_NULL;
  if (const sph_status st = check_sizes(cache, batch, tokens, q_heads, max_q, max_len, window)) return st;
  *bytes = 0;
  if (!batch || !tokens) return SPH_OK;
  const Plan p = plan_of(cache, batch, q_heads, max_q, max_len, window);
  if (!launchable(p)) return SPH_ERR_SHAPE;
  *bytes = p.bytes;
  return SPH_OK;
}

sph_status sph_attention(const sph_kv_cache* cache, int64_t batch, int64_t tokens, int32_t q_heads, const void* d_q,
                         int64_t q_token_stride, int64_t q_head_stride, const int32_t* d_q_start, int64_t max_q,
                         const int32_t* d_pages, int64_t pages_stride, const int32_t* d_seq_lens, int64_t max_len,
                         int64_t window, float scale, void* d_o, int64_t o_token_stride, int64_t o_head_stride,
                         float* d_lse, void* d_ws, size_t ws_bytes, void* stream) {
  if (const sph_status st = check_sizes(cache, batch, tokens, q_heads, max_q, max_len, window)) return st;
  if (!std::isfinite(scale)) return SPH_ERR_BAD_VALUE;
  if (!d_q_start && (max_q != 1 || tokens != batch)) return SPH_ERR_SHAPE;
  const int64_t pages_needed = (max_len + cache->page_size - 1) / cache->page_size;
  if (pages_stride < pages_needed || pages_stride > INT32_MAX) return SPH_ERR_SHAPE;
  if (!batch || !tokens) return SPH_OK;
  if (!d_q || !d_o || !d_seq_lens || (!d_pages && max_len > 0)) return SPH_ERR_NULL;
  const int64_t lim = int64_t(1) << 40;
  for (int64_t s : {q_token_stride, q_head_stride, o_token_stride, o_head_stride})
    if (s < 0 || s >= lim || s % 8) return SPH_ERR_SHAPE;
  if ((uintptr_t)d_q % 16 || (uintptr_t)d_o % 16 || (uintptr_t)d_q_start % 4 || (uintptr_t)d_pages % 4 || (uintptr_t)d_seq_lens % 4 ||
      (uintptr_t)d_lse % 4 || (uintptr_t)d_ws % 256)
    return SPH_ERR_SHAPE;
  if ((tokens > 1 && o_token_stride == 0) || (q_heads > 1 && o_head_stride == 0)) return SPH_ERR_SHAPE;  // rows written twice
  const Plan p = plan_of(cache, batch, q_heads, max_q, max_len, window);
  if (!launchable(p)) return SPH_ERR_SHAPE;
  if (p.bytes && !d_ws) return SPH_ERR_NULL;
  if (ws_bytes < p.bytes) return SPH_ERR_BUFFER_TOO_SMALL;
  const int bits = cache->bits, dim = cache->head_dim;
  AttnArgs a{};
  a.c = sph_cache_view(cache);
  a.q = (const char*)d_q, a.o = (char*)d_o;
  a.qt = 2 * q_token_stride, a.qh = 2 * q_head_stride, a.ot = 2 * o_token_stride, a.oh = 2 * o_head_stride;
  a.q_start = d_q_start, a.pages = d_pages, a.pages_stride = pages_stride, a.lens = d_seq_lens, a.lse = d_lse;
  a.tokens = tokens, a.batch = (int)batch, a.q_heads = q_heads, a.group = q_heads / cache->kv_heads;
  a.max_q = (int)max_q, a.max_len = (int)max_len, a.window = p.window;
  a.tiles = (int)p.tiles, a.splits = p.splits, a.chunk = p.chunk, a.shares = p.shares, a.fold = p.fold;
  a.scale = scale * kLog2e;
  a.stream = cache->n_pages * cache->page_size * cache->kv_heads * (int64_t)dim * bits / 4 > kLastCache;
  if (p.bytes) {
    a.part = (float*)d_ws;
    a.ml = (float2*)(a.part + p.parts * cache->head_dim);
    a.where = (int2*)(a.ml + p.parts);
  }
  const void* fn = p.wide ? sph_attn_wide_kernel(bits, dim)
                   : cache->page_size >= 16 ? (p.nb == 1 ? kernel_for<1, true>(bits, dim) : kernel_for<2, true>(bits, dim))
                                          : (p.nb == 1 ? kernel_for<1, false>(bits, dim) : kernel_for<2, false>(bits, dim));
  if (!launch_ok(fn, dim3((unsigned)p.grid), (hipStream_t)stream, a)) return SPH_ERR_HIP;
  if (p.bytes && !launch_ok(p.few ? (const void*)k_attn_join<true> : (const void*)k_attn_join<false>, dim3((unsigned)((p.joins + kWaves - 1) / kWaves)),
                            (hipStream_t)stream, a))
    return SPH_ERR_HIP;
  return SPH_OK;
}

}  // extern "C"
