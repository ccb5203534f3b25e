// The attention of up to 32 rows of a kv head, as sph_attn.hip describes it: tiles of one sequence, and what shares sequences out.
#pragma once
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
//
// ALONE: a wave by itself, beside others that have other sequences. It writes its part, without waiting for anyone.
template <int DIM, int BITS, int NB, bool UNI, bool ALONE, typename A>
__device__ __forceinline__ void attend(const A& a, char* lds, float2 (*ml_s)[16 * NB], int kvh, int b, int c_lo, int c_hi, int slot) {
  typedef Lay<DIM, BITS> L;
  constexpr int kRows = 16 * NB, kVBytes = kTile * L::kVStride, kOStride = DIM + 4, kStep = kTile * (ALONE ? 1 : kWaves);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, g4 = lane >> 4;
  Seq s;
  s.load(a, b);
  if (s.bad) {
    if constexpr (!A::kParts) write_bad(a, s, kvh);
    return;
  }
  if (s.n == 0) return;
  const int nrow = s.n * a.group;
  const int first = A::kFlat ? s.len - 1 : s.len - s.n;     // position of the first new token
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
  const int t0 = (k_lo & ~(kTile - 1)) + (ALONE ? 0 : kTile * wave);
  if (t0 < k_hi) {
    f16x8 q[NB][L::kSteps];
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      const int r = min(16 * n + col, nrow - 1), t = r / a.group, h = kvh * a.group + r % a.group;
      pos[n] = A::kFlat ? first : first + t;
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
    int kt = t0, nt = t0 + kStep < k_hi ? t0 + kStep : t0;
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
      const bool last = kt + kStep >= k_hi;
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
      const int nnt = nt + kStep < k_hi ? nt + kStep : nt;
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

  if constexpr (ALONE) {
    const bool some_odd = __any(odd);
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      const int row = 16 * n + col;
      if (row >= nrow) continue;
      const int64_t part = part_at(a, slot, kvh, row);
#pragma unroll
      for (int i = 0; i < DIM / 16; ++i) {
        f32x4 acc = o[n][i];
        if (some_odd) acc += odd_values<DIM, BITS>(span, pg, pages, A::kFlat ? first : first + row / a.group, 16 * i + 4 * g4);
        write_part(a, part, 16 * i + 4 * g4, acc, ref[n].log(), l[n]);
      }
    }
    return;
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
    if (any_odd) acc += odd_values<DIM, BITS>(span, pg, pages, A::kFlat ? first : first + row / a.group, ch);
    if (!A::kParts && slot < 0)
      write_out(a, s.start + row / a.group, kvh * a.group + row % a.group, ch, acc, mm, ll);
    else
      write_part(a, part_at(a, slot, kvh, row), ch, acc, mm, ll);
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

}  // namespace
