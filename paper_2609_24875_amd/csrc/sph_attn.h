// What the attention's kernels share: their arguments, the pages of a kv head, which keys rows see, and how rows are written.
#pragma once
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "sph_cache.h"

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kAlone = -1;

struct AttnArgs {
  // (what sph_attention_shared's kernels do otherwise)
  static constexpr bool kParts = false;   // rows are always written as parts
  static constexpr bool kFlat = false;    // every row sees every key
  CacheView c;
  const char* q;
  char* o;
  int64_t qt, qh, ot, oh;  // strides in bytes
  const int32_t* q_start;
  const int32_t* pages;
  int64_t pages_stride;
  const int32_t* lens;
  float* lse;
  // Parts of rows whose keys several workgroups share: [slot][kv head][row of the sequence] (kParts of many rows: [split][kv head][token][row of its group])
  // of dim fp32 sums, of (m, l) pairs, and for k_attn each sequence's (first slot, slots).
  float* part;
  float2* ml;
  int2* where;
  int64_t tokens;
  int batch, q_heads, group, max_q, max_len, window, tiles, splits, chunk, shares, fold;
  // (fold: tiles of rows between k_attn_wide's workgroups that share a CU, 0 for the longest first)
  bool stream;             // k_attn reads values past the caches
  float scale;             // times log2 e
  int each;                // of kParts: workgroups a sequence and kv head, 0: one, or shares that are counted; kAlone: a wave
};

// The kernel for more rows a kv head than k_attn takes, and its rows a workgroup and keys a tile.
const void* sph_attn_wide_kernel(int bits, int dim);
constexpr int kWideRows = 128;
static inline int sph_attn_wide_tile(int dim) { return dim <= 192 ? 64 : 32; }

namespace {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;
constexpr int kWaves = 4, kThreads = 64 * kWaves;

// Weights are exp2(score - m + kLift), m a maximum that is raised, and o and l scaled down, only when a score passes it by kRise: below 2^16,
// inside fp16's range, and at full precision down to 2^-25 of m's, since those that fp16 loses would be missing from o and not from l.
// Against a rise of 8 with a lift of 7: 2048 tokens over themselves 61.9 and 62.1 us, 4096 of 192 channels 351 and 346, of 256 531 and 518, single tokens
// alike.
constexpr float kRise = 4.75f, kLift = 11.0f;
static_assert(kRise + kLift < 15.9f, "fp16's range, and room for three roundings of scores below kFar");
// Scores from here on are so far apart in fp32 (2^-6 and more) that a weight could end up above fp16's range: they are compared without a rise
// or a lift, and rounded before the maximum is subtracted.
constexpr float kFar = 1 << 17;

// A row's reference: weights are exp2(score - base), base 0 at first. It has to be raised where a score passes `top` (at first -inf).
struct Ref {
  float top, base;
  // To the score mn, where that raises it (so that what the sums are scaled by, `keep`, never grows them).
  __device__ __forceinline__ bool raise(float mn, float& keep) {
    const bool near = fabsf(mn) < kFar;
    const float to = near ? mn - kLift : mn, from = log();
    if (!(to > from)) return false;
    keep = __builtin_amdgcn_exp2f(from - to);
    top = near ? mn + kRise : mn, base = to;
    return true;
  }
  // what the sum of the weights is relative to: -inf with no score yet
  __device__ __forceinline__ float log() const { return top == -INFINITY ? -INFINITY : base; }
};

// The queries of one sequence: tokens start .. end - 1.
struct Seq {
  int start, end, n, len;
  bool bad;
  template <typename A>
  __device__ __forceinline__ void load(const A& a, int b) {
    if constexpr (A::kFlat) {
      a.tokens_of(b, start, end);
    } else {
      start = a.q_start ? a.q_start[b] : b;
      end = a.q_start ? a.q_start[b + 1] : b + 1;
    }
    len = a.lens[b];
    // (compared before they are subtracted: the difference of two arbitrary numbers need not fit)
    bad = len < 0 || len > a.max_len || start < 0 || end < start || end > a.tokens;
    n = bad ? 0 : end - start;
    bad |= n > a.max_q;
  }
  // k_attn's tiles of 32 keys, from the first that its rows see on: at least one where there are rows to write
  __device__ __forceinline__ int tiles(int window) const {
    if (bad) return 1;
    const int lo = window ? max(0, len - n - window + 1) : 0;
    return n == 0 ? 0 : max(1, (len - (lo & ~31) + 31) >> 5);
  }
};

// Four channels of a row: normalised, or as the part `slot` of it.
__device__ __forceinline__ void write_out(const AttnArgs& a, int64_t token, int head, int ch, f32x4 acc, float m, float l) {
  // l is NaN for poisoned rows, 0 where nothing is seen
  const float inv = 1.0f / l;
  f16x4 y;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float x = l == 0.0f ? 0.0f : acc[i] * inv;
    // a mean of finite values lies between them: above fp16's largest only what the weights' rounding adds
    if (__builtin_isfinite(x)) x = fminf(fmaxf(x, -65504.0f), 65504.0f);
    y[i] = (_Float16)x;
  }
  *(f16x4*)(a.o + token * a.ot + head * a.oh + 2 * ch) = y;
  if (ch == 0 && a.lse) a.lse[token * a.q_heads + head] = l == 0.0f ? -INFINITY : (m + __builtin_log2f(l)) * kLn2;
}

__device__ __forceinline__ int64_t part_at(const AttnArgs& a, int slot, int kvh, int row) {
  return ((int64_t)slot * a.c.kv_heads + kvh) * ((int64_t)a.max_q * a.group) + row;
}

// The same in the order of all tokens, row `row` of those from `token` on: no more parts than there are rows, however they are shared among sequences.
__device__ __forceinline__ int64_t token_part_at(const AttnArgs& a, int split, int kvh, int64_t token, int row) {
  return (((int64_t)split * a.c.kv_heads + kvh) * a.tokens + token) * a.group + row;
}

__device__ __forceinline__ void write_part(const AttnArgs& a, int64_t at, int ch, f32x4 acc, float m, float l) {
  *(f32x4*)(a.part + at * a.c.dim + ch) = acc;
  if (ch == 0) a.ml[at] = make_float2(m, l);
}

// Every row of a sequence that the device found to be outside its bounds becomes NaN.
__device__ inline void write_bad(const AttnArgs& a, const Seq& s, int kvh) {
  const int64_t t0 = max(s.start, 0), t1 = min((int64_t)s.end, a.tokens);
  const float nan = __builtin_nanf("");
  const int per = a.group * (a.c.dim / 4);
  for (int64_t t = t0; t < t1; ++t)
    for (int i = threadIdx.x; i < per; i += blockDim.x)
      write_out(a, t, kvh * a.group + i / (a.c.dim / 4), i % (a.c.dim / 4) * 4, f32x4{nan, nan, nan, nan}, 0.0f, nan);
}

template <int BYTES, bool STREAM = false>
__device__ __forceinline__ void load_words(const char* p, uint32_t* w) {
  if constexpr (BYTES == 4) {   // (not a vector of one: with it, k_attn_wide's 128 channels at 4 bits spill)
    w[0] = STREAM ? __builtin_nontemporal_load((const uint32_t*)p) : *(const uint32_t*)p;
  } else {
    typedef uint32_t V __attribute__((ext_vector_type(BYTES / 4)));
    const V v = STREAM ? __builtin_nontemporal_load((const V*)p) : *(const V*)p;
#pragma unroll
    for (int i = 0; i < BYTES / 4; ++i) w[i] = v[i];
  }
}

// One kv head's pages.
struct Pages {
  const char *k, *v, *k_par, *v_par;
  int64_t stride, par_stride;
  int token, par_token;      // bytes between tokens of a page
  int mask, shift, count;
  __device__ __forceinline__ void set(const CacheView& c, int head) {
    k = c.k + head * c.head_stride, v = c.v + head * c.head_stride;
    k_par = c.k_par + head * c.par_head_stride, v_par = c.v_par + head * c.par_head_stride;
    stride = c.page_stride, par_stride = c.par_page_stride;
    token = (int)c.token_stride, par_token = (int)c.par_token_stride;
    shift = c.page_shift, mask = (1 << shift) - 1, count = (int)c.n_pages;
  }
  __device__ __forceinline__ bool there(int page) const { return (unsigned)page < (unsigned)count; }
  __device__ __forceinline__ const char* row(const char* base, int64_t page_stride, int token_stride, int page, int key) const {
    return base + page * page_stride + (uint32_t)((key & mask) * token_stride);
  }
};

// A row's pieces of eight channels in LDS are permuted within it, piece p to place p ^ turn(row), so that lanes that read together (one
// piece of 16 rows, or two neighbouring pieces of eight) find 16 different 16-byte places of the 256 bytes of banks. kSkip is what a row
// adds to the place.
template <int DIM>
struct RowPlaces {
  static constexpr int kPer = DIM / 8, kRow = DIM * 2, kSkip = kPer % 16;
  __device__ static __forceinline__ int turn(int row) {
    if constexpr (kSkip == 0) return (row & 7) << 1 | (row >> 3 & 1);
    if constexpr (kSkip == 8) return (row >> 1 & 3) << 1 | (row >> 3 & 1);
    return (row >> 2 & 1) << 1 | (row >> 3 & 1);
  }
  __device__ static __forceinline__ int at(int row, int piece) { return row * kRow + ((piece ^ turn(row)) << 4); }
};

// Keys that a workgroup's rows see: [k_lo, k_hi) at most, of them each row those in (pos - window, pos].
struct Span {
  int k_lo, k_hi, p_lo, p_hi, window, tile;
  // every row sees the whole tile at kt
  __device__ __forceinline__ bool whole(int kt) const {
    return kt >= k_lo && kt + tile <= k_hi && kt + tile - 1 <= p_lo && (!window || kt > p_hi - window);
  }
  __device__ __forceinline__ bool seen(int key, int pos) const { return key >= k_lo && key < k_hi && key <= pos && (!window || key > pos - window); }
};

// Eight values in LDS: zero if no row sees them, otherwise with infinities and NaN taken out. Returns whether there was one.
__device__ __forceinline__ bool clean_piece(char* at, bool unseen) {
  u32x4 v = *(const u32x4*)at;
  uint32_t odd = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t w = unseen ? 0u : v[i];
    // a half's exponent bits all set: adding one to the exponent carries into the sign's place
    const uint32_t low = ((w & 0x7C00u) + 0x400u) >> 15 & 1u, high = (((w >> 16) & 0x7C00u) + 0x400u) >> 15;
    w &= ~((0u - low) & 0xFFFFu) & ~((0u - high) << 16);
    odd |= low | high;
    v[i] = w;
  }
  *(u32x4*)at = v;
  return odd != 0;
}

// The sum of the infinities and NaN among channels ch .. ch + 3 of the values that a row at position pos sees in tiles that not
// every row sees: a weight is positive, so it leaves them what they are. Only called where there are some.
template <int DIM, int BITS>
__device__ __forceinline__ f32x4 odd_values(const Span& s, const Pages& pg, const int32_t* pages, int pos, int ch) {
  f32x4 sum = {};
#pragma unroll 1
  for (int key = s.k_lo; key < s.k_hi; ++key) {
    const int page = pages[key >> pg.shift];
    if (s.whole(key & ~(s.tile - 1)) || !s.seen(key, pos) || !pg.there(page)) continue;
    const char* row = pg.row(pg.v, pg.stride, pg.token, page, key);
    f16x8 v;
    if constexpr (BITS == 16)
      v = *(const f16x8*)(row + 2 * (ch & ~7));
    else
      v = decode8<BITS>(row + (ch & ~7) * BITS / 8, *(const uint32_t*)(pg.row(pg.v_par, pg.par_stride, pg.par_token, page, key) + ch / 32 * 4));
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float f = (float)(ch & 4 ? v[4 + e] : v[e]);
      if (!__builtin_isfinite(f)) sum[e] += f;
    }
  }
  return sum;
}

}  // namespace
