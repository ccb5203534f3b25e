// How much attention every cached token got (sph_attention_weights): sums over rows of exp(score - log of the row's softmax sum).
//
// For one kv head, row r = t * group + h is new token t under query head h of the head's group, as in the attention. S = Q K^T is computed
// by v_mfma_f32_32x32x16_f16 with a row per query row and a column per key, so a lane keeps 16 rows' scores of one key (rows
// 8 j + 4 (lane / 32) + i), and a key's sum stays with it: no key is shared, no atomics, and keys are read once, whatever the number of rows.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "sph_attn.h"

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

// The weights that rows 0 .. rows - 1 of 32 give to the lane's key, added up: scores st, logarithms lse_s and positions pos_s of all 32 in LDS.
template <bool WHOLE>
__device__ __forceinline__ float weigh(const f32x16& st, const float* lse_s, const int* pos_s, float scale, int rows, int key, int window, bool gone, int h) {
  float sum = 0.0f;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (8 * j < rows) {
      const f32x4 l = *(const f32x4*)(lse_s + 8 * j + 4 * h);
      float x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = __builtin_amdgcn_exp2f(fmaf(st[4 * j + i], scale, -l[i]));
      if constexpr (!WHOLE) {
        const int4 p = *(const int4*)(pos_s + 8 * j + 4 * h);
        const int pos[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const bool seen = key <= pos[i] && (!window || key > pos[i] - window);
          x[i] = !seen ? 0.0f : gone ? __builtin_nanf("") : x[i];
        }
      }
      sum += (x[0] + x[1]) + (x[2] + x[3]);
    }
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

// Up to 32 rows a kv head (single tokens, short drafts): each wave has keys of its own and goes through them once, or with one sum for
// all heads the workgroup's waves take the heads in turn and meet in LDS.
template <int DIM, int BITS>
__global__ __launch_bounds__(kThreads) void k_weights_few(WeightArgs) {
  const WeightArgs& a = *(const WeightArgs*)__builtin_amdgcn_kernarg_segment_ptr();
  typedef Keys<DIM, BITS> K;
  __shared__ __attribute__((aligned(16))) float lse_s[kWaves][32];
  __shared__ __attribute__((aligned(16))) int pos_s[kWaves][32];
  __shared__ float sum_s[kWaves][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, h = lane >> 5;
  uint32_t id = blockIdx.x;
  const int head = id % a.heads;
  id /= a.heads;
  const bool each = a.heads > 1 || a.c.kv_heads == 1;
  const int kt = (each ? id % a.tiles * kWaves + wave : id % a.tiles) * K::kKeys, b = id / a.tiles;
  if (kt >= a.max_len) return;                               // (with one sum for all heads for all waves alike)
  Seq s;
  s.load(a, b);
  const int nrow = s.n * a.group, first = s.len - s.n;
  const int lo = a.window ? max(0, first - a.window + 1) : 0;
  float sum = s.bad ? __builtin_nanf("") : 0.0f;
  if (!s.bad && nrow && kt < s.len && kt + K::kKeys > lo) {
    const int r = min(col, nrow - 1), t = r / a.group, pos = col < nrow ? first + t : -1;
    // every row sees every key
    const bool all = nrow == 32 && kt + K::kKeys <= first + 1 && (!a.window || kt > s.len - 1 - a.window);
    float acc[K::kBlocks] = {};
    if (h == 0) pos_s[wave][col] = pos;
    for (int kvh = each ? head : wave; kvh < a.c.kv_heads; kvh += each ? a.c.kv_heads : kWaves) {
      Pages pg;
      pg.set(a.c, kvh);
      const int hq = kvh * a.group + r % a.group;
      K keys;
      keys.load(pg, a.pages + b * a.pages_stride, kt, lo, s.len, lane);
      const char* qr = a.q + (s.start + t) * a.qt + hq * a.qh;
      f16x8 q[K::kSteps];
#pragma unroll
      for (int i = 0; i < K::kSteps; ++i) q[i] = *(const f16x8*)(qr + 16 * K::piece(i, h));
      if (h == 0) lse_s[wave][col] = log2_sum(a.lse[(int64_t)(s.start + t) * a.q_heads + hq]);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int u = 0; u < K::kBlocks; ++u) {
        f32x16 st = {};
#pragma unroll
        for (int i = 0; i < K::kSteps; ++i) st = __builtin_amdgcn_mfma_f32_32x32x16_f16(q[i], keys.k[u][i], st, 0, 0, 0);
        const int key = kt + 32 * u + col;
        if (all && !__any(keys.gone[u]))
          acc[u] += weigh<true>(st, lse_s[wave], pos_s[wave], a.scale, nrow, key, a.window, false, h);
        else
          acc[u] += weigh<false>(st, lse_s[wave], pos_s[wave], a.scale, nrow, key, a.window, keys.gone[u], h);
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
#pragma unroll
    for (int u = 0; u < K::kBlocks; ++u) acc[u] += __shfl_xor(acc[u], 32);
    sum = K::kBlocks == 2 && h ? acc[K::kBlocks - 1] : acc[0];
  }
  if (!each) {
    sum_s[wave][lane] = sum;
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int w = 1; w < kWaves; ++w) sum += sum_s[w][lane];
  }
  // lane l has key kt + l
  if (lane < K::kKeys) write_sum(a, b, head, kt + lane, s.bad ? a.max_len : s.len, sum);
}

constexpr int kManyRows = 64;                                // rows of a step

// More rows (prompts, long drafts): a workgroup's waves have keys of their own in registers, and go together through the rows that see any of
// them, which come 64 at a time through LDS.
template <int DIM, int BITS>
__global__ __launch_bounds__(kThreads, 2) void k_weights_many(WeightArgs) {
  const WeightArgs& a = *(const WeightArgs*)__builtin_amdgcn_kernarg_segment_ptr();
  typedef Keys<DIM, BITS> K;
  typedef RowPlaces<DIM> L;
  constexpr int kBytes = kManyRows * L::kRow, kShare = kManyRows * L::kPer / kThreads;
  static_assert(kManyRows * L::kPer % kThreads == 0, "whole shares");
  // two arrays, not one of two: loads on their way into one do not hold up reads of the other
  __shared__ __attribute__((aligned(16))) char rows_a[kBytes], rows_b[kBytes];
  __shared__ __attribute__((aligned(16))) float lse_s[2][kManyRows];
  __shared__ __attribute__((aligned(16))) int pos_s[2][kManyRows];
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
      auto load_rows = [&](int r0, char* to) {
#pragma unroll
        for (int i = 0; i < kShare; ++i) {
          const int idx = threadIdx.x + kThreads * i, row = idx / L::kPer, place = idx % L::kPer;
          const uint32_t r = min(r0 + row, r_hi - 1), t = r / (uint32_t)a.group, hq = kvh * a.group + r % (uint32_t)a.group;
          const char* from = a.q + (int64_t)(s.start + t) * a.qt + hq * a.qh + ((place ^ L::turn(row)) << 4);
          __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from,
                                           (__attribute__((address_space(3))) void*)(to + (kThreads * i + 64 * wave) * 16), 16, 0, 0);
        }
      };
      // logarithm and position of a step's row `threadIdx.x`: rows behind the last see nothing
      auto load_lse = [&](int r0, float& lse, int& pos) {
        const uint32_t r = min(r0 + (int)threadIdx.x, r_hi - 1), t = r / (uint32_t)a.group, hq = kvh * a.group + r % (uint32_t)a.group;
        lse = log2_sum(a.lse[(int64_t)(s.start + t) * a.q_heads + hq]);
        pos = r0 + (int)threadIdx.x < r_hi ? first + (int)t : -1;
      };
      float lse = 0.0f;
      int pos = 0;
      load_rows(r_lo, rows_a);
      if (threadIdx.x < kManyRows) {
        load_lse(r_lo, lse, pos);
        lse_s[0][threadIdx.x] = lse, pos_s[0][threadIdx.x] = pos;
      }
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
      auto step = [&](int r0, const char* from, char* to, int at) __attribute__((always_inline)) {
        const bool more = r0 + kManyRows < r_hi;
        if (more) {
          load_rows(r0 + kManyRows, to);
          if (threadIdx.x < kManyRows) load_lse(r0 + kManyRows, lse, pos);
        }
        const int p_lo = first + r0 / a.group, p_hi = first + (min(r0 + kManyRows, r_hi) - 1) / a.group;
        const bool whole = r0 + kManyRows <= r_hi && kt + K::kKeys - 1 <= p_lo && (!a.window || kt > p_hi - a.window) && !any_gone;
        if (kt <= p_hi && (!a.window || kt + K::kKeys > p_lo - a.window + 1)) {
#pragma unroll
          for (int rb = 0; rb < kManyRows / 32; ++rb) {
            f32x16 st[K::kBlocks] = {};
#pragma unroll
            for (int i = 0; i < K::kSteps; ++i) {
              const f16x8 q = *(const f16x8*)(from + L::at(32 * rb + col, K::piece(i, h)));
#pragma unroll
              for (int u = 0; u < K::kBlocks; ++u) st[u] = __builtin_amdgcn_mfma_f32_32x32x16_f16(q, keys.k[u][i], st[u], 0, 0, 0);
            }
#pragma unroll
            for (int u = 0; u < K::kBlocks; ++u) {
              const int key = kt + 32 * u + col;
              if (whole)
                acc[u] += weigh<true>(st[u], lse_s[at] + 32 * rb, pos_s[at] + 32 * rb, a.scale, 32, key, a.window, false, h);
              else
                acc[u] += weigh<false>(st[u], lse_s[at] + 32 * rb, pos_s[at] + 32 * rb, a.scale, 32, key, a.window, keys.gone[u], h);
            }
          }
        }
        if (more && threadIdx.x < kManyRows) lse_s[at ^ 1][threadIdx.x] = lse, pos_s[at ^ 1][threadIdx.x] = pos;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
      };
      for (int r0 = r_lo; r0 < r_hi; r0 += 2 * kManyRows) {
        step(r0, rows_a, rows_b, 0);
        if (r0 + kManyRows >= r_hi) break;
        step(r0 + kManyRows, rows_b, rows_a, 1);
      }
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

// Adds up k_weights_many's parts, in order.
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
  int tiles, splits, window;
  int64_t grid, joins;
  size_t bytes;
};

Plan plan_of(const sph_kv_cache* c, int64_t batch, int q_heads, int heads, int64_t max_q, int64_t max_len, int64_t window) {
  Plan p{};
  // one that hides nothing is none (and positions minus a window stay inside 32 bits)
  p.window = window > max_len ? 0 : (int)window;
  const int64_t rows = max_q * (q_heads / c->kv_heads), keys = c->head_dim <= 128 ? 64 : 32;
  const bool each = heads > 1 || c->kv_heads == 1;
  p.few = rows <= kFewRows;
  p.splits = 1;
  if (p.few) {
    p.tiles = (int)((max_len + keys * (each ? kWaves : 1) - 1) / (keys * (each ? kWaves : 1)));
    p.grid = batch * heads * p.tiles;
    return p;
  }
  p.tiles = (int)((max_len + keys * kWaves - 1) / (keys * kWaves));
  const int64_t units = batch * c->kv_heads * std::max(1, p.tiles);
  // rows are split where keys alone leave the chip idle, in parts of four steps at least
  p.splits = (int)std::max<int64_t>(1, std::min<int64_t>((2 * kCus + units - 1) / units, rows / (4 * kManyRows)));
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

template <int BITS>
const void* kernel_for(bool few, int dim) {
  switch (dim) {
    case 64: return few ? (const void*)k_weights_few<64, BITS> : (const void*)k_weights_many<64, BITS>;
    case 96: return few ? (const void*)k_weights_few<96, BITS> : (const void*)k_weights_many<96, BITS>;
    case 128: return few ? (const void*)k_weights_few<128, BITS> : (const void*)k_weights_many<128, BITS>;
    case 192: return few ? (const void*)k_weights_few<192, BITS> : (const void*)k_weights_many<192, BITS>;
    default: return few ? (const void*)k_weights_few<256, BITS> : (const void*)k_weights_many<256, BITS>;
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
  const void* fn = bits == 16 ? kernel_for<16>(p.few, dim) : bits == 8 ? kernel_for<8>(p.few, dim) : kernel_for<4>(p.few, dim);
  if (!launch_ok(fn, p.grid, (hipStream_t)stream, a)) return SPH_ERR_HIP;
  if (p.join && !launch_ok((const void*)k_weights_join, p.joins, (hipStream_t)stream, a)) return SPH_ERR_HIP;
  return SPH_OK;
}

}  // extern "C"
