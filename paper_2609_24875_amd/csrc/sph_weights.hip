// How much attention every cached token got (sph_attention_weights): for key j the sum over the rows r that see it of
// 2^(scale log2(e) q_r.k_j - log2(e) lse_r), on top of what it got before. The softmax's sums are at hand (lse), so one pass over the keys does, and
// values are not read.
//
// For one kv head, row r = t * group + h is new token t under query head h of the head's group, as in the attention. S = Q K^T is computed
// with a row per query row and a column per key, so a lane keeps some rows' scores of one key, and a key's sum stays with it: no key is
// shared, no atomics, and keys are read once, whatever the number of rows. Queries and keys are fp16 (keys of codes as sph_kv_read gives them), products are
// exact, and everything from the score on is fp32: beside 64 bits sums are off by 3e-8 (single tokens) to 2e-7 (2048 rows) of the largest.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "sph_attn_few.h"

namespace {

struct WeightArgs {
  static constexpr bool kFlat = false;
  CacheView c;
  const char* q;
  int64_t qt, qh;          // strides in bytes
  const int32_t* q_start;
  const int32_t* pages;
  int64_t pages_stride;
  const int32_t* lens;
  const float* lse;        // [tokens][q_heads]
  const float* before;
  float* out;
  int64_t bs, bh, os, oh;  // strides in elements
  float* part;             // [batch][kv_heads][splits][max_len]: sums of some rows, to be joined
  int64_t tokens;
  int batch, q_heads, group, max_q, max_len, window, heads, tiles, splits;
  float scale;             // times log2 e
};

// A wave's keys as the products take them: lane l has pieces of key l % 32 of each 32. The order of a product's channels is
// free as long as both operands share it, so a lane loads 16 bytes at once whatever the number of bits.
template <int DIM, int BITS>
struct Keys {
  static constexpr int kSteps = DIM / 16;
  static constexpr int kBlocks = DIM <= 128 ? 2 : 1, kKeys = 32 * kBlocks;
  static constexpr int kPiece = DIM * BITS / 8 % 32 == 0 ? 16 : 8;      // bytes
  static constexpr int kPieceCh = kPiece * 8 / BITS, kPer = kPieceCh / 8, kLoads = kSteps / kPer;
  static_assert(kSteps % kPer == 0, "whole pieces");
  f16x8 k[kBlocks][kSteps];
  bool gone[kBlocks];                                        // the lane's key is in a page outside the pool
  // the piece of eight channels that step `i` of a product takes from lanes of half h
  __device__ static __forceinline__ int piece(int i, int h) { return (2 * (i / kPer) + h) * kPer + i % kPer; }
  // Keys kt .. kt + kKeys - 1 of a sequence; those outside lo .. hi - 1 (not empty) take a page inside, and are read and not used.
  __device__ __forceinline__ void load(const Pages& pg, const int32_t* pages, int kt, int lo, int hi, int lane) {
    const int e_lo = lo >> pg.shift, e_hi = (hi - 1) >> pg.shift, h = lane >> 5;
    uint32_t w[kBlocks][kLoads][kPiece / 4], par[kBlocks][kLoads];
    int page[kBlocks];
#pragma unroll
    for (int u = 0; u < kBlocks; ++u) page[u] = pages[min(max((kt + 32 * u + (lane & 31)) >> pg.shift, e_lo), e_hi)];
#pragma unroll
    for (int u = 0; u < kBlocks; ++u) {
      const int key = kt + 32 * u + (lane & 31);
      gone[u] = !pg.there(page[u]);
      const int p = gone[u] ? 0 : page[u];
      const char* row = pg.row(pg.k, pg.stride, pg.token, p, key);
#pragma unroll
      for (int i = 0; i < kLoads; ++i) load_words<kPiece>(row + (2 * i + h) * kPiece, w[u][i]);
      if constexpr (BITS < 16) {
        const char* pr = pg.row(pg.k_par, pg.par_stride, pg.par_token, p, key);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) par[u][i] = *(const uint32_t*)(pr + (2 * i + h) * kPieceCh / 32 * 4);
      }
    }
#pragma unroll
    for (int u = 0; u < kBlocks; ++u)
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
          if constexpr (BITS == 16)
            k[u][i] = __builtin_bit_cast(f16x8, make_uint4(w[u][i][0], w[u][i][1], w[u][i][2], w[u][i][3]));
          else if constexpr (BITS == 8)
            k[u][i * kPer + e] = decode8w<8>(w[u][i][2 * e], w[u][i][2 * e + 1], par[u][i]);
          else
            k[u][i * kPer + e] = decode8w<4>(w[u][i][e], 0, par[u][i]);
        }
  }
};

// Base-2 logarithm of a row's softmax sum; a row without one (it sees nothing, or only scores of -inf) gives no weight.
__device__ __forceinline__ float log2_sum(float lse) { return lse == -INFINITY ? INFINITY : lse * kLog2e; }

// The weights that rows 8 j + 4 h .. + 3 of 32 give to the lane's key: scores st, logarithms l of these rows.
__device__ __forceinline__ float weigh(const f32x16& st, int j, const f32x4& l, float scale) {
  float x[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = __builtin_amdgcn_exp2f(fmaf(st[4 * j + i], scale, -l[i]));
  return (x[0] + x[1]) + (x[2] + x[3]);
}

// Those of all 32 where not every row sees the key: those whose position pos_s hides it give nothing.
__device__ __forceinline__ float weigh_seen(const f32x16& st, const float* lse_s, const int* pos_s, float scale, int key, int window, bool gone, int h) {
  float sum = 0.0f;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const f32x4 l = *(const f32x4*)(lse_s + 8 * j + 4 * h);
    const int4 p = *(const int4*)(pos_s + 8 * j + 4 * h);
    const int pos[4] = {p.x, p.y, p.z, p.w};
    float x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = __builtin_amdgcn_exp2f(fmaf(st[4 * j + i], scale, -l[i]));
      // (a select, not a branch around the exponential)
      asm("" : "+v"(x[i]));
      x[i] = key > pos[i] || (window && key <= pos[i] - window) ? 0.0f : gone ? __builtin_nanf("") : x[i];
    }
    sum += (x[0] + x[1]) + (x[2] + x[3]);
  }
  return sum;
}

// A key's new sum, 0 behind the sequence's last token.
__device__ __forceinline__ void write_sum(const WeightArgs& a, int b, int head, int key, int len, float sum) {
  if (key >= a.max_len) return;
  float x = 0.0f;
  if (key < len) x = sum + (a.before ? a.before[b * a.bs + head * a.bh + key] : 0.0f);
  a.out[b * a.os + head * a.oh + key] = x;
}

// A wave's step of up to 32 rows: kBlocks times 16 keys in registers as they are stored, 8 KiB of 128 channels. Products are
// v_mfma_f32_16x16x32_f16 with a column per key, whose 16 rows' scores lie in four lanes.
//
// UNI: pages of 16 tokens and more, each block of keys in one, so that scalars hold its address; smaller ones: each lane has its own key's.
template <int DIM, int BITS, bool UNI>
struct Step {
  typedef Lay<DIM, BITS> L;
  static constexpr int kWords = DIM * BITS / 128;            // a lane's registers of 16 keys
  static constexpr int kBlocks = kWords >= 32 ? 1 : kWords >= 16 ? 2 : 4, kKeys = 16 * kBlocks;
  uint32_t k[kBlocks][L::kLoads][L::kPiece / 4], par[kBlocks][L::kLoads];
  // Keys from kt on, lane l with those at 16 u + l % 16 in pages page[u] (those outside the pool: any, their rows are not used).
  __device__ __forceinline__ void load(const Pages& pg, const int* page, int kt, int lane) {
    const int col = lane & 15, g4 = lane >> 4;
#pragma unroll
    for (int u = 0; u < kBlocks; ++u) {
      const int p = pg.there(page[u]) ? page[u] : 0, key = kt + 16 * u + col;
      if constexpr (UNI) {
        const int in_page = (kt + 16 * u) & pg.mask;
        const int64_t off = p * pg.stride + (uint32_t)(in_page * pg.token), par_off = p * pg.par_stride + (uint32_t)(in_page * pg.par_token);
#pragma unroll
        for (int i = 0; i < L::kLoads; ++i) {
          load_row<L::kPiece, true>(pg.k, &off, pg.token, 0, col, col, (4 * i + g4) * L::kPiece, k[u][i]);
          if constexpr (BITS < 16)
            load_row<4, true>(pg.k_par, &par_off, pg.par_token, 0, col, col, g4 * L::kPieceCh / 32 * 4 + i * L::kPieceCh / 8 * 4, &par[u][i]);
        }
      } else {
        const char* row = pg.row(pg.k, pg.stride, pg.token, p, key) + g4 * L::kPiece;
        const char* pr = pg.row(pg.k_par, pg.par_stride, pg.par_token, p, key) + g4 * L::kPieceCh / 32 * 4;
#pragma unroll
        for (int i = 0; i < L::kLoads; ++i) {
          load_words<L::kPiece>(row + 4 * i * L::kPiece, k[u][i]);
          if constexpr (BITS < 16) par[u][i] = *(const uint32_t*)(pr + i * L::kPieceCh / 8 * 4);
        }
      }
    }
  }
  __device__ __forceinline__ f16x8 piece(int u, int i, int j) const {
    if constexpr (BITS == 16)
      return __builtin_bit_cast(f16x8, make_uint4(k[u][i][0], k[u][i][1], k[u][i][2], k[u][i][3]));
    else if constexpr (BITS == 8)
      return decode8w<8>(k[u][i][2 * j], k[u][i][2 * j + 1], par[u][i]);
    else
      return decode8w<4>(k[u][i][j], 0, par[u][i]);
  }
};

// Up to 32 rows a kv head (single tokens, short drafts): each wave goes through keys of its own, kRun steps of them, the next step's loads issued
// when one's products are done; with one sum for all heads the workgroup's waves take the heads in turn and meet in LDS.
//
// Bound by memory: 64 sequences of all lengths up to 8192, 8 kv heads of 128 channels at 8 bits 57 us, 4.0 TB/s of keys, parameters and sums. Waves are many and
// short since a ragged batch leaves no one else to even them out: with 1, 2, 3, 4 and 6 steps a wave 69, 60, 60, 63 and 63 us, and 57 with four
// waves a SIMD (which keys as they are stored, not decoded, leave the registers for), where 32x32x16 products and keys decoded at once had 78 and two.
constexpr int kRun = 2;

template <int DIM, int BITS, int NB, bool UNI>
__global__ __launch_bounds__(kThreads, NB == 1 && DIM <= 128 && (UNI || BITS != 8) ? 4 : 2) void k_weights_few(WeightArgs) {
  const WeightArgs& a = *(const WeightArgs*)__builtin_amdgcn_kernarg_segment_ptr();
  typedef Step<DIM, BITS, UNI> K;
  typedef Lay<DIM, BITS> L;
  __shared__ float sum_s[kWaves][K::kKeys];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, g4 = lane >> 4;
  uint32_t id = blockIdx.x;
  const int head = id % a.heads;
  id /= a.heads;
  const bool each = a.heads > 1 || a.c.kv_heads == 1;
  // (turned by the sequence's number: otherwise the first tiles, which all sequences have, come to the same part of the chip)
  const int b = id / a.tiles, tile = (id + b) % a.tiles;
  const int t0 = (each ? tile * kWaves + wave : tile) * (each ? kRun : 1) * K::kKeys;
  if (t0 >= a.max_len) return;                               // (with one sum for all heads for all waves alike)
  Seq s;
  s.load(a, b);
  const int nrow = s.n * a.group, first = s.len - s.n;
  const int lo = a.window ? max(0, first - a.window + 1) : 0;
  const int t1 = min(a.max_len, t0 + (each ? kRun : 1) * K::kKeys), len = s.bad ? a.max_len : s.len;
  // the steps of keys that a row may see: k_lo .. k_hi
  const bool none = s.bad || nrow == 0;
  const int k_lo = none ? t1 : min(t1, max(t0, lo / K::kKeys * K::kKeys)), k_hi = none ? t1 : min(t1, s.len);
  const float nothing = s.bad ? __builtin_nanf("") : 0.0f;
  if (each)
    for (int kt = t0; kt < t1; kt += K::kKeys)
      if ((kt < k_lo || kt >= k_hi) && lane < K::kKeys) write_sum(a, b, head, kt + lane, len, nothing);
  float sum[K::kBlocks];
#pragma unroll
  for (int u = 0; u < K::kBlocks; ++u) sum[u] = nothing;
  int kvh = each ? head : wave;
  if (k_lo < k_hi && kvh < a.c.kv_heads) {
    Pages pg;
    pg.set(a.c, kvh);
    const int32_t* pages = a.pages + b * a.pages_stride;
    const int e_lo = lo >> pg.shift, e_hi = (s.len - 1) >> pg.shift;
    // keys outside those that are seen take a page inside: they are read and not used
    auto pages_of = [&](int kt, int* page) __attribute__((always_inline)) {
#pragma unroll
      for (int u = 0; u < K::kBlocks; ++u) page[u] = pages[min(max((kt + 16 * u + (UNI ? 0 : col)) >> pg.shift, e_lo), e_hi)];
    };
    f16x8 q[NB][L::kSteps];
    float lse[NB][4];
    int pos[NB][4];
    // (asked for before the next step's keys, which would hold up what is loaded behind them)
    auto old_sum = [&](int k) { return each && a.before && lane < K::kKeys && k + lane < min(s.len, a.max_len) ? a.before[b * a.bs + head * a.bh + k + lane] : 0.0f; };
    auto load_rows = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        const int r = min(16 * n + col, nrow - 1);
        const char* qr = a.q + (int64_t)(s.start + r / a.group) * a.qt + (kvh * a.group + r % a.group) * a.qh;
#pragma unroll
        for (int i = 0; i < L::kLoads; ++i)
#pragma unroll
          for (int j = 0; j < L::kBlocks; ++j) q[n][i * L::kBlocks + j] = *(const f16x8*)(qr + 2 * ((4 * i + g4) * L::kPieceCh + 8 * j));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          // rows behind the last give nothing
          const int row = 16 * n + 4 * g4 + i, rr = min(row, nrow - 1), t = rr / a.group;
          const float x = log2_sum(a.lse[(int64_t)(s.start + t) * a.q_heads + kvh * a.group + rr % a.group]);
          lse[n][i] = row < nrow ? x : INFINITY;
          pos[n][i] = row < nrow ? first + t : -1;
        }
      }
    };
    K T;
    int kt = k_lo, page[K::kBlocks], next[K::kBlocks];
    pages_of(kt, page);
    float old = old_sum(kt);
    T.load(pg, page, kt, lane);
    load_rows();
    while (true) {
      // the next step: of this head, or with one sum for all heads the same keys of the wave's next one
      const int to = each ? kt + K::kKeys : kt, to_head = each ? kvh : kvh + kWaves;
      const bool more = each ? to < k_hi : to_head < a.c.kv_heads;
      pages_of(more ? to : kt, next);
      f32x4 st[K::kBlocks][NB] = {};
#pragma unroll
      for (int u = 0; u < K::kBlocks; ++u)
#pragma unroll
        for (int i = 0; i < L::kLoads; ++i)
#pragma unroll
          for (int j = 0; j < L::kBlocks; ++j) {
            const f16x8 kf = T.piece(u, i, j);
#pragma unroll
            for (int n = 0; n < NB; ++n) st[u][n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(q[n][i * L::kBlocks + j], kf, st[u][n], 0, 0, 0);
            // (decoded when they are needed: keys of all blocks at once would cost a wave a SIMD)
            if (j == L::kBlocks - 1) __builtin_amdgcn_sched_barrier(0);
          }
      // not above the products: the loads would take registers of their own beside those that they refill
      __builtin_amdgcn_sched_barrier(0);
      const float old_now = old;
      if (more) {
        if (!each) pg.set(a.c, to_head);
        old = old_sum(to);
        T.load(pg, next, to, lane);
      }
      __builtin_amdgcn_sched_barrier(0);
      const bool whole = kt >= lo && kt + K::kKeys - 1 <= first && (!a.window || kt > s.len - 1 - a.window);
#pragma unroll
      for (int u = 0; u < K::kBlocks; ++u) {
        const int key = kt + 16 * u + col;
        const bool gone = !pg.there(page[u]), plain = whole && !__any(gone);
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          float x[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) x[i] = __builtin_amdgcn_exp2f(fmaf(st[u][n][i], a.scale, -lse[n][i]));
          if (!plain) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const bool seen = key <= pos[n][i] && (!a.window || key > pos[n][i] - a.window);
              x[i] = !seen ? 0.0f : gone ? __builtin_nanf("") : x[i];
            }
          }
          sum[u] += (x[0] + x[1]) + (x[2] + x[3]);
        }
        page[u] = next[u];
      }
      if (each) {
        // lane 16 u + l has key 16 u + l
        float mine = 0.0f;
#pragma unroll
        for (int u = 0; u < K::kBlocks; ++u) {
          sum[u] += __shfl_xor(sum[u], 16);
          sum[u] += __shfl_xor(sum[u], 32);
          mine = g4 == u ? sum[u] : mine;
          sum[u] = 0.0f;
        }
        if (lane < K::kKeys && kt + lane < a.max_len) a.out[b * a.os + head * a.oh + kt + lane] = kt + lane < len ? old_now + mine : 0.0f;
      }
      if (!more) break;
      kt = to;
      if (!each) {
        kvh = to_head;
        load_rows();
      }
    }
  }
  if (each) return;
#pragma unroll
  for (int u = 0; u < K::kBlocks; ++u) {
    sum[u] += __shfl_xor(sum[u], 16);
    sum[u] += __shfl_xor(sum[u], 32);
    if (g4 == 0) sum_s[wave][16 * u + col] = sum[u];
  }
  __syncthreads();
  if (wave || lane >= K::kKeys) return;
  float x = sum_s[0][lane];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) x += sum_s[w][lane];
  write_sum(a, b, head, t0 + lane, len, x);
}


// Rows of a step, so that two workgroups fit a CU's LDS.
constexpr int many_rows(int dim) { return dim <= 128 ? 128 : 64; }

// More rows (prompts, long drafts): a workgroup's waves have keys of their own in registers, and go together through the rows that see any of
// them, which come 128 (64) at a time through LDS, the next ones on their way meanwhile. Products are v_mfma_f32_32x32x16_f16: a lane has rows
// 8 j + 4 (lane / 32) + i of key lane % 32. Keys, not rows, stay in registers since their sums do, too.
//
// Bound by the exponentials beside the products: of a block of 32 rows and 64 keys a wave's 16 products take 512 cycles and its 32 exponentials 256, beside which
// a multiplication and an addition each. 2048 rows of a prompt of 16384 tokens under 32 query heads 290 us (0.89 PFLOP/s of what is seen); without the products 178, without the
// exponentials 238. Scores kept for a block longer, so that weights run beside the next block's products, 366 -> 290 us; products and weights in groups by scheduling
// hints 337, and neither more workgroups of fewer rows nor other occupancies gain.
template <int DIM, int BITS>
__global__ __launch_bounds__(kThreads, 2) void k_weights_many(WeightArgs) {
  const WeightArgs& a = *(const WeightArgs*)__builtin_amdgcn_kernarg_segment_ptr();
  typedef Keys<DIM, BITS> K;
  typedef RowPlaces<DIM> L;
  constexpr int kManyRows = many_rows(DIM), kBytes = kManyRows * L::kRow, kShare = kManyRows * L::kPer / kThreads;
  static_assert(kManyRows * L::kPer % kThreads == 0, "whole shares");
  // two arrays, not one of two: loads on their way into one do not hold up reads of the other
  __shared__ __attribute__((aligned(16))) char rows_a[kBytes], rows_b[kBytes];
  // of the step before, this one, the next one, whose rows are on their way, and the one after it: rows' logarithms, positions and places
  __shared__ __attribute__((aligned(16))) float lse_s[4][kManyRows];
  __shared__ __attribute__((aligned(16))) int pos_s[4][kManyRows];
  __shared__ int64_t off_s[4][kManyRows];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, h = lane >> 5;
  // the first keys are seen by most rows, so they come first
  uint32_t id = blockIdx.x;
  const int kvh = id % a.c.kv_heads;
  id /= a.c.kv_heads;
  const int split = id % a.splits;
  id /= a.splits;
  const int b = id % a.batch, k0 = id / a.batch * (kWaves * K::kKeys), kt = k0 + wave * K::kKeys;
  Seq s;
  s.load(a, b);
  const bool direct = a.splits == 1 && (a.heads > 1 || a.c.kv_heads == 1);
  float acc[K::kBlocks] = {};
  const int first = s.len - s.n;
  const int k1 = min(k0 + kWaves * K::kKeys, s.len);         // the workgroup's keys: k0 .. k1 - 1
  if (!s.bad && k0 < k1) {
    // tokens that see one of them, and this split's rows of theirs
    const int t_lo = max(0, k0 - first), t_hi = a.window ? (int)min((int64_t)s.n, max((int64_t)0, (int64_t)k1 - 1 + a.window - first)) : s.n;
    const int all = max(0, t_hi - t_lo) * a.group, steps = (all + kManyRows - 1) / kManyRows;
    const int r_lo = t_lo * a.group + (int)((int64_t)steps * split / a.splits) * kManyRows;
    const int r_hi = min(t_lo * a.group + all, t_lo * a.group + (int)((int64_t)steps * (split + 1) / a.splits) * kManyRows);
    if (r_lo < r_hi) {
      Pages pg;
      pg.set(a.c, kvh);
      K keys;
      keys.load(pg, a.pages + b * a.pages_stride, kt, k0, k1, lane);
      bool any_gone = false;
#pragma unroll
      for (int u = 0; u < K::kBlocks; ++u) any_gone |= keys.gone[u];
      any_gone = __any(any_gone);
      auto load_rows = [&](int slot, char* to) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < kShare; ++i) {
          const int idx = threadIdx.x + kThreads * i, row = idx / L::kPer, place = idx % L::kPer;
          const char* from = a.q + off_s[slot][row] + ((place ^ L::turn(row)) << 4);
          __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from,
                                           (__attribute__((address_space(3))) void*)(to + (kThreads * i + 64 * wave) * 16), 16, 0, 0);
        }
      };
      // Row `threadIdx.x` of a step, worked out once for all lanes that load or weigh it: those behind the last are read as it is and see nothing.
      float lse = 0.0f;
      int pos = 0;
      int64_t off = 0;
      auto find_row = [&](int r0) __attribute__((always_inline)) {
        const uint32_t r = min(r0 + (int)threadIdx.x, r_hi - 1), t = r / (uint32_t)a.group, hq = kvh * a.group + r % (uint32_t)a.group;
        lse = log2_sum(a.lse[(int64_t)(s.start + t) * a.q_heads + hq]);
        pos = r0 + (int)threadIdx.x < r_hi ? first + (int)t : -1;
        off = (int64_t)(s.start + t) * a.qt + hq * a.qh;
      };
      auto keep_row = [&](int slot) __attribute__((always_inline)) { lse_s[slot][threadIdx.x] = lse, pos_s[slot][threadIdx.x] = pos, off_s[slot][threadIdx.x] = off; };
      const bool finds = threadIdx.x < kManyRows;
      if (finds) {
        find_row(r_lo);
        keep_row(0);
        if (r_lo + kManyRows < r_hi) {
          find_row(r_lo + kManyRows);
          keep_row(1);
        }
      }
      __syncthreads();
      load_rows(0, rows_a);
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
      int at = 0;                                            // the step's place of four
      f32x16 st[2][K::kBlocks];
      bool left = false;                                     // the weights of the last step's last block are still to be added: its scores are in st[1]
      auto logs_of = [&](f32x4* l, int slot, int rb) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < 4; ++j) l[j] = *(const f32x4*)(lse_s[slot] + 32 * rb + 8 * j + 4 * h);
      };
      auto weigh_piece = [&](const f32x16* of, const f32x4* l, int p) __attribute__((always_inline)) {
        acc[p % K::kBlocks] += weigh(of[p % K::kBlocks], p / K::kBlocks, l[p / K::kBlocks], a.scale);
      };
      constexpr int kPieces = 4 * K::kBlocks;
      auto add_left = [&]() __attribute__((always_inline)) {
        f32x4 l[4];
        logs_of(l, (at + 3) & 3, kManyRows / 32 - 1);
#pragma unroll
        for (int p = 0; p < kPieces; ++p) weigh_piece(st[1], l, p);
      };
      auto step = [&](int r0, const char* from, char* to) __attribute__((always_inline)) {
        const bool more = r0 + 2 * kManyRows < r_hi;
        const int next = (at + 1) & 3, after = (at + 2) & 3;
        if (r0 + kManyRows < r_hi) load_rows(next, to);
        if (more && finds) find_row(r0 + 2 * kManyRows);
        const int p_lo = first + r0 / a.group, p_hi = first + (min(r0 + kManyRows, r_hi) - 1) / a.group;
        const bool whole = r0 + kManyRows <= r_hi && kt + K::kKeys - 1 <= p_lo && (!a.window || kt > p_hi - a.window) && !any_gone;
        const bool work = kt <= p_hi && (!a.window || kt + K::kKeys > p_lo - a.window + 1);
        constexpr int kRowBlocks = kManyRows / 32;
        auto read = [&](f16x8* q, int rb) __attribute__((always_inline)) {
#pragma unroll
          for (int i = 0; i < K::kSteps; ++i) q[i] = *(const f16x8*)(from + L::at(32 * rb + col, K::piece(i, h)));
        };
        auto products = [&](f32x16* st, const f16x8* q) __attribute__((always_inline)) {
#pragma unroll
          for (int u = 0; u < K::kBlocks; ++u) st[u] = f32x16{};
#pragma unroll
          for (int i = 0; i < K::kSteps; ++i)
#pragma unroll
            for (int u = 0; u < K::kBlocks; ++u) st[u] = __builtin_amdgcn_mfma_f32_32x32x16_f16(q[i], keys.k[u][i], st[u], 0, 0, 0);
        };
        if (work && whole) {
          // A block's products run beside the weights of the one before, a few of them behind each step of products (left to itself, the compiler puts
          // all of one kind behind the other), the first block's beside those of the last step's last. A step's rows are read for the next block
          // when its products are under way.
          static_assert(kRowBlocks % 2 == 0, "the last block's scores are in st[1]");
          // (a ring of kAhead steps of rows: of 256 channels, all steps of a block would not fit the registers)
          constexpr int kAhead = K::kSteps == 16 ? 8 : K::kSteps;
          f16x8 q[kAhead];
          auto read_step = [&](int rb, int i) __attribute__((always_inline)) { q[i % kAhead] = *(const f16x8*)(from + L::at(32 * rb + col, K::piece(i, h))); };
#pragma unroll
          for (int i = 0; i < kAhead; ++i) read_step(0, i);
#pragma unroll
          for (int rb = 0; rb < kRowBlocks; ++rb) {
            f32x4 l[4];
            logs_of(l, rb ? at : (at + 3) & 3, rb ? rb - 1 : kRowBlocks - 1);
            f32x16* now = st[rb & 1];
            const f32x16* last = st[(rb + 1) & 1];
#pragma unroll
            for (int u = 0; u < K::kBlocks; ++u) now[u] = f32x16{};
#pragma unroll
            for (int i = 0; i < K::kSteps; ++i) {
#pragma unroll
              for (int u = 0; u < K::kBlocks; ++u) now[u] = __builtin_amdgcn_mfma_f32_32x32x16_f16(q[i % kAhead], keys.k[u][i], now[u], 0, 0, 0);
              if (i + kAhead < K::kSteps)
                read_step(rb, i + kAhead);
              else if (rb + 1 < kRowBlocks)
                read_step(rb + 1, i + kAhead - K::kSteps);
              if (rb > 0 || left)
#pragma unroll
                for (int p = i * kPieces / K::kSteps; p < (i + 1) * kPieces / K::kSteps; ++p) weigh_piece(last, l, p);
              __builtin_amdgcn_sched_barrier(0);
            }
          }
          left = true;
        } else {
          if (left) add_left();
          left = false;
#pragma unroll 1
          for (int rb = work ? 0 : kRowBlocks; rb < kRowBlocks; ++rb) {
            f16x8 q[K::kSteps];
            read(q, rb);
            products(st[0], q);
#pragma unroll
            for (int u = 0; u < K::kBlocks; ++u)
              acc[u] += weigh_seen(st[0][u], lse_s[at] + 32 * rb, pos_s[at] + 32 * rb, a.scale, kt + 32 * u + col, a.window, keys.gone[u], h);
          }
        }
        if (more && finds) keep_row(after);
        at = next;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
      };
      for (int r0 = r_lo; r0 < r_hi; r0 += 2 * kManyRows) {
        step(r0, rows_a, rows_b);
        if (r0 + kManyRows >= r_hi) break;
        step(r0 + kManyRows, rows_b, rows_a);
      }
      if (left) add_left();
    }
  }
#pragma unroll
  for (int u = 0; u < K::kBlocks; ++u) acc[u] += __shfl_xor(acc[u], 32);
  const float sum = s.bad ? __builtin_nanf("") : K::kBlocks == 2 && h ? acc[K::kBlocks - 1] : acc[0];
  if (lane >= K::kKeys) return;
  if (direct)
    write_sum(a, b, a.heads > 1 ? kvh : 0, kt + lane, s.bad ? a.max_len : s.len, sum);
  else if (kt + lane < a.max_len)
    a.part[(((int64_t)b * a.c.kv_heads + kvh) * a.splits + split) * a.max_len + kt + lane] = sum;
}

// Adds up k_weights_many's parts, in order: 4 us for the 8 heads' sums of 16384 keys, the latency of a launch and of its loads.
__global__ __launch_bounds__(kThreads) void k_weights_join(WeightArgs a) {
  const uint32_t per = ((uint32_t)a.max_len + kThreads - 1) / kThreads;
  uint32_t id = blockIdx.x;
  const int key = id % per * kThreads + threadIdx.x;
  id /= per;
  const int head = id % a.heads, b = id / a.heads;
  if (key >= a.max_len) return;
  Seq s;
  s.load(a, b);
  const int parts = a.heads > 1 || a.c.kv_heads == 1 ? a.splits : a.splits * a.c.kv_heads;
  const float* p = a.part + ((int64_t)b * a.c.kv_heads + head) * a.splits * a.max_len + key;
  float sum = s.bad ? __builtin_nanf("") : 0.0f;
  if (!s.bad && key < s.len)
#pragma unroll 8
    for (int i = 0; i < parts; ++i) sum += p[(int64_t)i * a.max_len];
  write_sum(a, b, head, key, s.bad ? a.max_len : s.len, sum);
}

// ------------------------------------------------------------------ host side

constexpr int kFewRows = 32, kCus = 256;

struct Plan {
  bool few, join;
  int nb, tiles, splits, window;
  int64_t grid, joins;
  size_t bytes;
};

Plan plan_of(const sph_kv_cache* c, int64_t batch, int q_heads, int heads, int64_t max_q, int64_t max_len, int64_t window) {
  Plan p{};
  // one that hides nothing is none (and positions minus a window stay inside 32 bits)
  p.window = window > max_len ? 0 : (int)window;
  const int64_t rows = max_q * (q_heads / c->kv_heads);
  const bool each = heads > 1 || c->kv_heads == 1;
  p.few = rows <= kFewRows;
  p.nb = rows <= 16 ? 1 : 2;
  p.splits = 1;
  if (p.few) {
    const int64_t words = c->head_dim * c->bits / 128, keys = (words >= 32 ? 16 : words >= 16 ? 32 : 64) * (each ? kRun * kWaves : 1);   // (as Step has them)
    p.tiles = (int)((max_len + keys - 1) / keys);
    p.grid = batch * heads * p.tiles;
    return p;
  }
  const int64_t keys = c->head_dim <= 128 ? 64 : 32;
  p.tiles = (int)((max_len + keys * kWaves - 1) / (keys * kWaves));
  const int64_t units = batch * c->kv_heads * std::max(1, p.tiles);
  // rows are split where keys alone leave the chip idle, in parts of 256 at least
  p.splits = (int)std::max<int64_t>(1, std::min<int64_t>((2 * kCus + units - 1) / units, rows / 256));
  p.join = !each || p.splits > 1;
  p.grid = units * p.splits;
  p.joins = batch * heads * ((max_len + kThreads - 1) / kThreads);
  if (p.join) p.bytes = (size_t)batch * c->kv_heads * p.splits * max_len * sizeof(float);
  return p;
}

bool launchable(const Plan& p) { return p.grid < (1 << 24) && p.joins < (1 << 24); }

sph_status check_sizes(const sph_kv_cache* c, int64_t batch, int64_t tokens, int32_t q_heads, int32_t heads, int64_t max_q, int64_t max_len,
                       int64_t window) {
  if (!c) return SPH_ERR_NULL;
  if (const int st = sph_cache_check(c)) return (sph_status)st;
  if (batch < 0 || batch > 65536 || tokens < 0 || tokens > (1 << 26) || q_heads < 1 || q_heads > 65535 || q_heads % c->kv_heads ||
      (heads != 1 && heads != c->kv_heads) || max_q < 1 || max_q > (1 << 24) || max_len < 0 || max_len > (1 << 30) || window < 0 ||
      max_q * (q_heads / c->kv_heads) > (1 << 30))
    return SPH_ERR_SHAPE;
  return SPH_OK;
}

template <int DIM, int BITS, int NB>
const void* few_for(bool uni) {
  return uni ? (const void*)k_weights_few<DIM, BITS, NB, true> : (const void*)k_weights_few<DIM, BITS, NB, false>;
}

template <int DIM, int BITS>
const void* kernel_for(const Plan& p, bool uni) {
  return !p.few ? (const void*)k_weights_many<DIM, BITS> : p.nb == 1 ? few_for<DIM, BITS, 1>(uni) : few_for<DIM, BITS, 2>(uni);
}

template <int BITS>
const void* kernel_for(const Plan& p, int dim, bool uni) {
  switch (dim) {
    case 64: return kernel_for<64, BITS>(p, uni);
    case 96: return kernel_for<96, BITS>(p, uni);
    case 128: return kernel_for<128, BITS>(p, uni);
    case 192: return kernel_for<192, BITS>(p, uni);
    default: return kernel_for<256, BITS>(p, uni);
  }
}

bool launch_ok(const void* fn, int64_t blocks, hipStream_t s, WeightArgs& a) {
  void* kargs[] = {(void*)&a};
  return hipLaunchKernel(fn, dim3((unsigned)blocks), dim3(kThreads), kargs, 0, s) == hipSuccess && hipGetLastError() == hipSuccess;
}

}  // namespace

extern "C" {

sph_status sph_attention_weights_workspace_bytes(const sph_kv_cache* cache, int64_t batch, int64_t tokens, int32_t q_heads, int32_t heads,
                                                 int64_t max_q, int64_t max_len, int64_t window, size_t* bytes) {
  if (!bytes) return SPH_ERR_NULL;
  if (const sph_status st = check_sizes(cache, batch, tokens, q_heads, heads, max_q, max_len, window)) return st;
  *bytes = 0;
  if (!batch || !max_len) return SPH_OK;
  const Plan p = plan_of(cache, batch, q_heads, heads, max_q, max_len, window);
  if (!launchable(p)) return SPH_ERR_SHAPE;
  *bytes = p.bytes;
  return SPH_OK;
}

sph_status sph_attention_weights(const sph_kv_cache* cache, int64_t batch, int64_t tokens, int32_t q_heads, const void* d_q,
                                 int64_t q_token_stride, int64_t q_head_stride, const int32_t* d_q_start, int64_t max_q,
                                 const int32_t* d_pages, int64_t pages_stride, const int32_t* d_seq_lens, int64_t max_len, int64_t window,
                                 float scale, const float* d_lse, int32_t heads, const float* d_before, int64_t before_seq_stride,
                                 int64_t before_head_stride, float* d_sums, int64_t sums_seq_stride, int64_t sums_head_stride, void* d_ws,
                                 size_t ws_bytes, void* stream) {
  if (const sph_status st = check_sizes(cache, batch, tokens, q_heads, heads, max_q, max_len, window)) return st;
  if (!std::isfinite(scale)) return SPH_ERR_BAD_VALUE;
  if (!d_q_start && (max_q != 1 || tokens != batch)) return SPH_ERR_SHAPE;
  const int64_t pages_needed = (max_len + cache->page_size - 1) / cache->page_size;
  if (pages_stride < pages_needed || pages_stride > INT32_MAX) return SPH_ERR_SHAPE;
  const int64_t lim = int64_t(1) << 40;
  for (int64_t s : {q_token_stride, q_head_stride})
    if (s < 0 || s >= lim || s % 8) return SPH_ERR_SHAPE;
  for (int64_t s : {before_seq_stride, before_head_stride, sums_seq_stride, sums_head_stride})
    if (s < 0 || s >= lim) return SPH_ERR_SHAPE;
  // rows that are written must not overlap
  if ((batch > 1 && sums_seq_stride < max_len) || (heads > 1 && sums_head_stride < max_len)) return SPH_ERR_SHAPE;
  if (batch > 1 && heads > 1 && sums_seq_stride < (heads - 1) * sums_head_stride + max_len &&
      sums_head_stride < (batch - 1) * sums_seq_stride + max_len)
    return SPH_ERR_SHAPE;
  if (!batch || !max_len) return SPH_OK;
  if (!d_seq_lens || !d_pages || !d_sums || (tokens > 0 && (!d_q || !d_lse))) return SPH_ERR_NULL;
  if ((uintptr_t)d_q % 16 || (uintptr_t)d_q_start % 4 || (uintptr_t)d_pages % 4 || (uintptr_t)d_seq_lens % 4 || (uintptr_t)d_lse % 4 ||
      (uintptr_t)d_before % 4 || (uintptr_t)d_sums % 4 || (uintptr_t)d_ws % 256)
    return SPH_ERR_SHAPE;
  // sums added to in place have to be so row by row
  if (d_sums == d_before && ((batch > 1 && sums_seq_stride != before_seq_stride) || (heads > 1 && sums_head_stride != before_head_stride)))
    return SPH_ERR_SHAPE;
  const Plan p = plan_of(cache, batch, q_heads, heads, max_q, max_len, window);
  if (!launchable(p)) return SPH_ERR_SHAPE;
  if (p.bytes && !d_ws) return SPH_ERR_NULL;
  if (ws_bytes < p.bytes) return SPH_ERR_BUFFER_TOO_SMALL;
  WeightArgs a{};
  a.c = sph_cache_view(cache);
  a.q = (const char*)d_q, a.qt = 2 * q_token_stride, a.qh = 2 * q_head_stride;
  a.q_start = d_q_start, a.pages = d_pages, a.pages_stride = pages_stride, a.lens = d_seq_lens, a.lse = d_lse;
  a.before = d_before, a.out = d_sums;
  a.bs = before_seq_stride, a.bh = before_head_stride, a.os = sums_seq_stride, a.oh = sums_head_stride;
  a.part = (float*)d_ws;
  a.tokens = tokens, a.batch = (int)batch, a.q_heads = q_heads, a.group = q_heads / cache->kv_heads;
  a.max_q = (int)max_q, a.max_len = (int)max_len, a.window = p.window, a.heads = heads, a.tiles = p.tiles, a.splits = p.splits;
  a.scale = scale * kLog2e;
  const int bits = cache->bits, dim = cache->head_dim;
  const bool uni = cache->page_size >= 16;
  const void* fn = bits == 16 ? kernel_for<16>(p, dim, uni) : bits == 8 ? kernel_for<8>(p, dim, uni) : kernel_for<4>(p, dim, uni);
  if (!launch_ok(fn, p.grid, (hipStream_t)stream, a)) return SPH_ERR_HIP;
  if (p.join && !launch_ok((const void*)k_weights_join, p.joins, (hipStream_t)stream, a)) return SPH_ERR_HIP;
  return SPH_OK;
}

}  // extern "C"
