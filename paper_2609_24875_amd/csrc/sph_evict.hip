// Eviction from the paged cache by accumulated attention weight: sph_kv_evict.
//
// Of n tokens the first `first` and the last `recent` are kept, and of the others the m = keep - first - recent with the largest sums, equal ones by the lower
// index. With B the m-th largest sum, T(j) the competing tokens up to j whose sum is B, and W = m - #{sum > B}: j is kept if its sum is above B, or is B and
// T(j) <= W, and its place is the number of kept ones before it.
//
// Two launches. k_evict_choose, a workgroup a sequence and row of sums, finds B digit by digit (of 12, 12 and 8 bits), then gives every kept
// token its place by counting in order; the choice needs no sort and depends on no order of atomics, which only count. k_evict_move takes their keys and
// values there, or within the same pages k_evict_within. Tokens keep their order, so a token's place is never behind where it was: moved inside the same pages, in
// ascending order and read before the same step's places are written, none is overwritten before it is read.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "sph_cache.h"

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct EvictArgs {
  CacheView c;
  const int32_t* pages;
  const int32_t* to;
  int64_t pages_stride, to_stride;
  const int32_t* lens;
  int32_t* new_lens;
  const float* sums;
  float* new_sums;
  int64_t ss, sh, ns, nh;  // strides in elements
  int32_t* kept;           // [batch][heads][keep]
  int64_t max_len, width;
  int heads, keep, recent, first, bits, chunks;
};

// (digits of 12, 12 and 8 bits: the first has a sum's sign, exponent and three bits more, the second mostly decides)
constexpr int kChooseThreads = 1024, kChooseWaves = kChooseThreads / 64, kDigits = 4096;

// Sums in the order of whole numbers: NaN above everything, -0 as 0. No sum gives 0, which stands for none.
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x + 0.0f);
  return x != x ? 0xFFFFFFFFu : u & 0x80000000u ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ int lanes_below(uint64_t mask) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}

// The sums of a wave's tokens, lane l those at 64 c + l of its stretch: R of them in registers, with R = 0 read again in every pass.
template <int R>
struct Keys {
  uint32_t k[R ? R : 1];
  const float* row;
  int count;               // tokens of the wave, 0 and less for none
  // keys of chunks c .. c + N - 1 (all loads on their way together: none is behind a branch)
  template <int N>
  __device__ __forceinline__ void read(int c, int lane, uint32_t* x) const {
    float v[N];
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = row[min(64 * (c + i) + lane, count - 1)];
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = 64 * (c + i) + lane < count ? ordered(v[i]) : 0u;
  }
  __device__ __forceinline__ void load(const float* r, int n, int lane) {
    row = r, count = n;
    if constexpr (R > 0) {
      if (count <= 0) return;
#pragma unroll
      for (int c = 0; c < R; c += 16) {
        if (64 * c < count)
          read<16>(c, lane, k + c);
        else
#pragma unroll
          for (int i = 0; i < 16; ++i) k[c + i] = 0u;
      }
    }
  }
  template <typename F>
  __device__ __forceinline__ void each(int lane, F f) const {
    if constexpr (R > 0) {
#pragma unroll
      for (int c = 0; c < R; ++c)
        if (64 * c < count) f(c, k[c]);
    } else {
      // (eight loads on their way together)
      for (int c0 = 0; 64 * c0 < count; c0 += 8) {
        uint32_t x[8];
        read<8>(c0, lane, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) f(c0 + i, x[i]);
      }
    }
  }
};

// The sum of the numbers of the waves before this one, all read at once.
__device__ __forceinline__ uint32_t before_wave(const uint32_t* of, int wave) {
  uint32_t sum = 0;
#pragma unroll
  for (int w = 0; w < kChooseWaves; ++w) sum += w < wave ? of[w] : 0u;
  return sum;
}

// Bound by the latency of its passes, three at most, one for each digit: the sums are read once and stay in registers (up to 65536
// tokens), and half its cycles are the counters in LDS, where those of one digit queue. A workgroup a row, since a row over several would have to wait for
// each other's counts: 32 sequences of up to 8192 tokens under 8 heads that choose for themselves 16.4 us, one of 517 with one choice for all 6.8.
template <int R>
__global__ __launch_bounds__(kChooseThreads) void k_evict_choose(EvictArgs a) {
  __shared__ __attribute__((aligned(16))) uint32_t hist[kDigits];
  __shared__ int found[3];                                   // digit, tokens above it, tokens with it
  __shared__ __attribute__((aligned(16))) uint32_t gts[kChooseWaves], eqs[kChooseWaves], totals[kChooseWaves];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int b = blockIdx.x / a.heads, h = blockIdx.x % a.heads;
  const int n = a.lens[b];
  const float* row = a.sums + b * a.ss + h * a.sh;
  float* out = a.new_sums + b * a.ns + h * a.nh;
  int32_t* kept = a.kept + (int64_t)blockIdx.x * a.keep;
  if (n < 0 || n > a.max_len) {
    for (int i = threadIdx.x; i < a.keep; i += kChooseThreads) kept[i] = -1;
    for (int64_t i = threadIdx.x; i < a.width; i += kChooseThreads) out[i] = __builtin_nanf("");
    return;
  }
  const int left = min(n, a.keep);
  if (n <= a.keep) {
    for (int i = threadIdx.x; i < a.keep; i += kChooseThreads) kept[i] = i < n ? i : -1;
  } else {
    const int all = n - a.first - a.recent, m = a.keep - a.first - a.recent;      // 0 <= m < all
    const int per = (all + kChooseThreads - 1) / kChooseThreads * 64;             // a wave's stretch
    Keys<R> keys;
    keys.load(row + a.first + wave * per, min(per, all - wave * per), lane);
    uint32_t prefix = 0, mask = 0;
    uint32_t bar = 0xFFFFFFFFu;                              // sums above it are kept, and `ties` of those that equal it
    int want = m, ties = 0;
    if (m > 0) {
      bool open = true;
#pragma unroll 1
      for (int shift = 20; shift >= 0 && open; shift = shift == 20 ? 8 : shift == 8 ? 0 : -1) {
        const uint32_t digits = shift ? kDigits : 256;
        ((uint4*)hist)[threadIdx.x] = make_uint4(0, 0, 0, 0);
        __syncthreads();
        keys.each(lane, [&](int, uint32_t key) {
          const bool in = key != 0 && (key & mask) == prefix;
          const uint64_t act = __ballot(in);
          if (!act) return;
          // (tokens that are all alike, as those that got nothing yet, are counted at once)
          const uint32_t digit = key >> shift & (digits - 1);
          if (act == ~0ull && __all(digit == (uint32_t)__builtin_amdgcn_readfirstlane(digit))) {
            if (lane == 0) atomicAdd(&hist[digit], 64u);
          } else if (in) {
            atomicAdd(&hist[digit], 1u);
          }
        });
        __syncthreads();
        // thread t has digits 4095 - 4 t .. 4092 - 4 t: tokens from the top down to each
        const uint4 four = ((const uint4*)hist)[kDigits / 4 - 1 - threadIdx.x];
        const uint32_t cnt[4] = {four.w, four.z, four.y, four.x}, sum = (cnt[0] + cnt[1]) + (cnt[2] + cnt[3]);
        uint32_t upto = sum;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
          const uint32_t v = __shfl_up(upto, d);
          upto += lane >= d ? v : 0;
        }
        if (lane == 63) totals[wave] = upto;
        __syncthreads();
        uint32_t above = upto - sum + before_wave(totals, wave);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (above < (uint32_t)want && above + cnt[i] >= (uint32_t)want) found[0] = kDigits - 1 - 4 * threadIdx.x - i, found[1] = above, found[2] = cnt[i];
          above += cnt[i];
        }
        __syncthreads();
        prefix |= (uint32_t)found[0] << shift;
        mask |= (digits - 1) << shift;
        want -= found[1];
        open = want < found[2];                              // otherwise all tokens with these digits are kept
      }
      bar = open ? prefix : prefix - 1;
      ties = open ? want : 0;
    }
    int gt = 0, eq = 0;
    keys.each(lane, [&](int, uint32_t key) {
      gt += __builtin_popcountll(__ballot(key > bar));
      eq += __builtin_popcountll(__ballot(key == bar));
    });
    if (lane == 0) gts[wave] = gt, eqs[wave] = eq;
    __syncthreads();
    gt = (int)before_wave(gts, wave), eq = (int)before_wave(eqs, wave);
    keys.each(lane, [&](int c, uint32_t key) {
      const uint64_t g = __ballot(key > bar), e = __ballot(key == bar);
      const int eq_before = eq + lanes_below(e);
      const int place = a.first + gt + lanes_below(g) + min(eq_before, ties);
      if (key > bar || (key == bar && eq_before < ties)) kept[place] = a.first + wave * per + 64 * c + lane;
      gt += __builtin_popcountll(g), eq += __builtin_popcountll(e);
    });
    for (int i = threadIdx.x; i < a.first; i += kChooseThreads) kept[i] = i;
    for (int i = threadIdx.x; i < a.recent; i += kChooseThreads) kept[a.keep - a.recent + i] = n - a.recent + i;
  }
  // the kept tokens' sums follow, in place if the caller says so: as in k_evict_within
  constexpr int kEach = 4;
  for (int i0 = 0; i0 < left; i0 += kEach * kChooseThreads) {
    __syncthreads();
    float v[kEach];
#pragma unroll
    for (int u = 0; u < kEach; ++u) {
      const int i = i0 + u * kChooseThreads + threadIdx.x;
      v[u] = i < left ? row[kept[i]] : 0.0f;
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kEach; ++u) {
      const int i = i0 + u * kChooseThreads + threadIdx.x;
      if (i < left) out[i] = v[u];
    }
  }
  for (int64_t i = left + threadIdx.x; i < a.width; i += kChooseThreads) out[i] = 0.0f;
}

constexpr int kMoveThreads = 256, kMoveEach = 4;

// What a token in a page outside the pool leaves behind: as the attention says of it, NaN.
__device__ __forceinline__ u32x4 lost_piece(int bits) { return bits == 16 ? u32x4{0x7E007E00u, 0x7E007E00u, 0x7E007E00u, 0x7E007E00u} : u32x4{}; }
constexpr uint32_t kLostPar = 0x00007E00u;

struct Place {
  int64_t code, par;       // byte offsets of a token's row under a head; code < 0: outside the pool
  __device__ __forceinline__ void set(const CacheView& c, const int32_t* pages, int head, int token) {
    const int page = pages[token >> c.page_shift], in_page = token & ((1 << c.page_shift) - 1);
    const bool there = (unsigned)page < (uint64_t)c.n_pages;
    code = there ? page * c.page_stride + head * c.head_stride + in_page * c.token_stride : -1;
    par = page * c.par_page_stride + head * c.par_head_stride + in_page * c.par_token_stride;
  }
};

__device__ __forceinline__ int kept_of(const EvictArgs& a, int b, int head, int i) {
  return a.kept[((int64_t)b * a.heads + (a.heads > 1 ? head : 0)) * a.keep + i];
}

// Into pages of their own. A thread copies 16 bytes of a key and of a value row, and the offset and step of 32 channels that
// start there, of kMoveEach tokens, whose loads are on their way together; past the caches, since each byte is read and written once. Bound by memory: 32
// sequences of up to 8192 tokens to 4096 each, 8 heads of 128 fp16 channels 113 us, 4.9 TB/s read and written.
template <int BITS>
__global__ __launch_bounds__(kMoveThreads) void k_evict_move(EvictArgs a) {
  const CacheView& c = a.c;
  const int pieces = c.dim * BITS / 128, per = kMoveThreads / pieces;
  uint32_t id = blockIdx.x;
  const int chunk = id % a.chunks;
  id /= a.chunks;
  const int head = id % c.kv_heads, b = id / c.kv_heads;
  const int n = a.lens[b];
  const bool bad = n < 0 || n > a.max_len;
  const int left = bad ? 0 : min(n, a.keep);
  if (chunk == 0 && head == 0 && threadIdx.x == 0) a.new_lens[b] = bad ? n : left;
  const int piece = threadIdx.x % pieces, t = threadIdx.x / pieces;
  if (t >= per) return;
  constexpr int kParPieces = BITS == 8 ? 2 : 1;              // pieces that share an offset and a step
  const bool par = BITS < 16 && piece % kParPieces == 0;
  const int i0 = chunk * per * kMoveEach + t;
  u32x4 k[kMoveEach], v[kMoveEach];
  uint32_t kp[kMoveEach], vp[kMoveEach];
#pragma unroll
  for (int u = 0; u < kMoveEach; ++u) {
    const int i = i0 + u * per;
    if (i >= left) continue;
    Place from;
    from.set(c, a.pages + b * a.pages_stride, head, kept_of(a, b, head, i));
    k[u] = v[u] = lost_piece(BITS), kp[u] = vp[u] = kLostPar;
    if (from.code < 0) continue;
    k[u] = __builtin_nontemporal_load((const u32x4*)(c.k + from.code + 16 * piece));
    v[u] = __builtin_nontemporal_load((const u32x4*)(c.v + from.code + 16 * piece));
    if (par) {
      kp[u] = *(const uint32_t*)(c.k_par + from.par + piece / kParPieces * 4);
      vp[u] = *(const uint32_t*)(c.v_par + from.par + piece / kParPieces * 4);
    }
  }
#pragma unroll
  for (int u = 0; u < kMoveEach; ++u) {
    const int i = i0 + u * per;
    if (i >= left) continue;
    Place to;
    to.set(c, a.to + b * a.to_stride, head, i);
    if (to.code < 0) continue;
    __builtin_nontemporal_store(k[u], (u32x4*)(c.k + to.code + 16 * piece));
    __builtin_nontemporal_store(v[u], (u32x4*)(c.v + to.code + 16 * piece));
    if (par) {
      *(uint32_t*)(c.k_par + to.par + piece / kParPieces * 4) = kp[u];
      *(uint32_t*)(c.v_par + to.par + piece / kParPieces * 4) = vp[u];
    }
  }
}

// Within the sequence's own pages: a workgroup takes up to 64 bytes of every key or value row of a sequence and head, or all offsets and steps, through
// all tokens in ascending order: nobody else reads or writes these bytes, and a step's tokens are read before any of its places is written. 32 sequences to
// 4096 tokens each, 8 heads of 128 fp16 channels 286 us (3.7 TB/s read and written), one sequence 24: the latency of its steps, of 1024 tokens each.
constexpr int kWithinThreads = 1024, kWithinEach = 4;

template <typename T>
__device__ __forceinline__ void move_within(const EvictArgs& a, char* base, bool par, int b, int head, int pieces, int first_piece, int left, T lost) {
  const CacheView& c = a.c;
  const int per = kWithinThreads / pieces, t = threadIdx.x / pieces;
  const int64_t at = (first_piece + threadIdx.x % pieces) * (int64_t)sizeof(T);
  const int32_t* pages = a.pages + b * a.pages_stride;
  for (int i0 = 0; i0 < left; i0 += per * kWithinEach) {
    T x[kWithinEach];
    bool moves[kWithinEach];
#pragma unroll
    for (int u = 0; u < kWithinEach; ++u) {
      const int i = i0 + u * per + t;
      moves[u] = false;
      if (t >= per || i >= left) continue;
      const int j = kept_of(a, b, head, i);
      moves[u] = j != i;
      if (!moves[u]) continue;
      Place from;
      from.set(c, pages, head, j);
      x[u] = from.code < 0 ? lost : *(const T*)(base + (par ? from.par : from.code) + at);
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kWithinEach; ++u) {
      if (!moves[u]) continue;
      Place to;
      to.set(c, pages, head, i0 + u * per + t);
      if (to.code >= 0) *(T*)(base + (par ? to.par : to.code) + at) = x[u];
    }
  }
}

__global__ __launch_bounds__(kWithinThreads) void k_evict_within(EvictArgs a) {
  const CacheView& c = a.c;
  const int pieces = c.dim * a.bits / 128, slices = (pieces + 3) / 4;
  uint32_t id = blockIdx.x;
  const int part = id % a.chunks;                            // of keys, of values, then both's offsets and steps
  id /= a.chunks;
  const int head = id % c.kv_heads, b = id / c.kv_heads;
  const int n = a.lens[b];
  const bool bad = n < 0 || n > a.max_len;
  const int left = bad ? 0 : min(n, a.keep);
  if (part == 0 && head == 0 && threadIdx.x == 0) a.new_lens[b] = bad ? n : left;
  if (part < 2 * slices) {
    const int slice = part % slices;
    move_within<u32x4>(a, part < slices ? c.k : c.v, false, b, head, min(4, pieces - 4 * slice), 4 * slice, left, lost_piece(a.bits));
  } else {
    move_within<uint32_t>(a, part == 2 * slices ? c.k_par : c.v_par, true, b, head, c.dim / 32, 0, left, kLostPar);
  }
}

template <typename... A>
bool launch_ok(const void* fn, uint32_t blocks, int threads, hipStream_t s, A... args) {
  void* kargs[] = {(void*)&args...};
  return hipLaunchKernel(fn, dim3(blocks), dim3(threads), kargs, 0, s) == hipSuccess && hipGetLastError() == hipSuccess;
}

}  // namespace

extern "C" {

sph_status sph_kv_evict(const sph_kv_cache* cache, int64_t batch, const int32_t* d_pages, int64_t pages_stride, const int32_t* d_seq_lens,
                        int64_t max_len, const float* d_sums, int32_t heads, int64_t sums_seq_stride, int64_t sums_head_stride,
                        int64_t keep, int64_t recent, int64_t first, const int32_t* d_to_pages, int64_t to_stride, int32_t* d_new_lens,
                        float* d_new_sums, int64_t new_width, int64_t new_seq_stride, int64_t new_head_stride, int32_t* d_kept,
                        void* stream) {
  if (!cache) return SPH_ERR_NULL;
  if (const int st = sph_cache_check(cache)) return (sph_status)st;
  if (batch < 0 || batch > 65536 || max_len < 0 || max_len > (1 << 30) || (heads != 1 && heads != cache->kv_heads) || keep < 1 ||
      keep > (1 << 30) || recent < 0 || first < 0 || recent > keep || first > keep - recent)
    return SPH_ERR_SHAPE;
  const int64_t most = std::min(keep, max_len), ps = cache->page_size, lim = int64_t(1) << 40;
  if (pages_stride < (max_len + ps - 1) / ps || pages_stride > INT32_MAX || to_stride < (most + ps - 1) / ps || to_stride > INT32_MAX ||
      new_width < most || new_width > (1 << 30))
    return SPH_ERR_SHAPE;
  for (int64_t s : {sums_seq_stride, sums_head_stride, new_seq_stride, new_head_stride})
    if (s < 0 || s >= lim) return SPH_ERR_SHAPE;
  // rows that are written must not overlap
  if ((batch > 1 && new_seq_stride < new_width) || (heads > 1 && new_head_stride < new_width)) return SPH_ERR_SHAPE;
  if (batch > 1 && heads > 1 && new_seq_stride < (heads - 1) * new_head_stride + new_width &&
      new_head_stride < (batch - 1) * new_seq_stride + new_width)
    return SPH_ERR_SHAPE;
  if (!batch) return SPH_OK;
  if (!d_seq_lens || !d_new_lens || !d_kept || (max_len > 0 && (!d_pages || !d_to_pages || !d_sums)) || (new_width > 0 && !d_new_sums)) return SPH_ERR_NULL;
  for (const void* p : {(const void*)d_pages, (const void*)d_to_pages, (const void*)d_seq_lens, (const void*)d_new_lens, (const void*)d_sums,
                        (const void*)d_new_sums, (const void*)d_kept})
    if ((uintptr_t)p % 4) return SPH_ERR_SHAPE;
  // sums rewritten in place have to be so row by row
  if (d_sums && d_new_sums == d_sums && ((batch > 1 && new_seq_stride != sums_seq_stride) || (heads > 1 && new_head_stride != sums_head_stride)))
    return SPH_ERR_SHAPE;
  const bool within = d_to_pages == d_pages;
  if (within && batch > 1 && to_stride != pages_stride) return SPH_ERR_SHAPE;
  EvictArgs a{};
  a.c = sph_cache_view(cache);
  a.pages = d_pages, a.to = d_to_pages, a.pages_stride = pages_stride, a.to_stride = to_stride;
  a.lens = d_seq_lens, a.new_lens = d_new_lens, a.sums = d_sums, a.new_sums = d_new_sums;
  a.ss = sums_seq_stride, a.sh = sums_head_stride, a.ns = new_seq_stride, a.nh = new_head_stride;
  a.kept = d_kept, a.max_len = max_len, a.width = new_width;
  a.heads = heads, a.keep = (int)keep, a.recent = (int)recent, a.first = (int)first, a.bits = cache->bits;
  const int pieces = cache->head_dim * cache->bits / 128;
  if (within) {
    a.chunks = 2 * ((pieces + 3) / 4) + (cache->bits < 16 ? 2 : 0);
  } else {
    const int64_t per = (int64_t)(kMoveThreads / pieces) * kMoveEach;
    a.chunks = (int)std::max<int64_t>(1, (most + per - 1) / per);
  }
  const int threads = within ? kWithinThreads : kMoveThreads;
  const int64_t rows = batch * heads, blocks = batch * cache->kv_heads * a.chunks;
  if (rows * kChooseThreads >= (int64_t(1) << 32) || blocks * threads >= (int64_t(1) << 32)) return SPH_ERR_SHAPE;
  const void* choose = max_len <= 16 * kChooseThreads   ? (const void*)k_evict_choose<16>
                       : max_len <= 64 * kChooseThreads ? (const void*)k_evict_choose<64>
                                                        : (const void*)k_evict_choose<0>;
  if (!launch_ok(choose, (uint32_t)rows, kChooseThreads, (hipStream_t)stream, a)) return SPH_ERR_HIP;
  const void* move = within              ? (const void*)k_evict_within
                     : cache->bits == 16 ? (const void*)k_evict_move<16>
                     : cache->bits == 8  ? (const void*)k_evict_move<8>
                                         : (const void*)k_evict_move<4>;
  if (!launch_ok(move, (uint32_t)blocks, threads, (hipStream_t)stream, a)) return SPH_ERR_HIP;
  return SPH_OK;
}

}  // extern "C"
