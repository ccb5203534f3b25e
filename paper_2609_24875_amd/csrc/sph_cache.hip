// Rotary positions and the paged key-value cache: sph_rope_table, sph_rope, sph_kv_append, sph_kv_read.
//
// All of them move each byte once and do a few operations on it, so they are bound by memory (by the
// launch for a decode step's few tokens). Rows are read and written 16 bytes a lane.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "sph_cache.h"

namespace {

constexpr int kThreads = 256;

// ------------------------------------------------------------------ rows

template <typename T>
struct Row8;
template <>
struct Row8<_Float16> {
  f16x8 v;
  __device__ __forceinline__ void load(const char* p) { v = *(const f16x8*)p; }
  __device__ __forceinline__ float at(int i) const { return (float)v[i]; }
};
template <>
struct Row8<float> {
  f32x4 v[2];
  __device__ __forceinline__ void load(const char* p) {
    v[0] = ((const f32x4*)p)[0];
    v[1] = ((const f32x4*)p)[1];
  }
  __device__ __forceinline__ float at(int i) const { return v[i >> 2][i & 3]; }
};

__device__ __forceinline__ void store8(_Float16* p, const float* y) {
  f16x8 o;
#pragma unroll
  for (int i = 0; i < 8; ++i) o[i] = (_Float16)y[i];
  *(f16x8*)p = o;
}

// ------------------------------------------------------------------ rotation

// (cos, sin) of N consecutive pairs of one position; NaN for a position outside the table.
template <int N>
struct Turn {
  float c[N], s[N];
  __device__ __forceinline__ void load(const float* table, int64_t max_pos, int half, int pos, int pair, float sign) {
    // (as a factor: stored on two branches, the angles would not stay in registers)
    const bool there = (unsigned)pos < (uint64_t)max_pos;
    const float one = there ? 1.0f : __builtin_nanf(""), turned = sign * one;
    const f32x4* t = (const f32x4*)(table + ((there ? (int64_t)pos : 0) * half + pair) * 2);
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      const f32x4 w = t[i];
      c[2 * i] = one * w[0], s[2 * i] = turned * w[1], c[2 * i + 1] = one * w[2], s[2 * i + 1] = turned * w[3];
    }
  }
};

// One pair turned. Each product is rounded before the sum, so that every path that rotates, whatever the
// compiler would fuse in it, gives the same bits: keys rotated on their way into the cache get the codes that they
// would get if they were rotated in fp32 first.
__device__ __forceinline__ void turn(float& p, float& q, float c, float s) {
#pragma clang fp contract(off)
  const float pc = p * c, qs = q * s, ps = p * s, qc = q * c;
  p = pc - qs;
  q = ps + qc;
}

struct RopeArgs {
  const char* x;
  char* y;
  int64_t xt, xh, yt, yh;  // strides in bytes
  const int32_t* pos;
  const float* table;
  int64_t max_pos;
  int64_t tokens;
  int heads, dim, rot;
  int hpt;                 // heads a thread takes
  float sign;
};

// One thread rotates two runs of 16 bytes of hpt heads of a token (eight pairs of fp16, four of fp32), each run beside its neighbouring
// lanes': loads and stores leave no gaps. The angles are read once for all heads. Channels behind rot_dim are copied. Four heads' loads
// are in flight together, past the caches, since each row is read once. STREAM: stores go past them, too, which is faster beside
// stores of the cache's pages (8192 tokens into 4 bits and back 58.5 us, otherwise 61.5; loads that stay in the caches 62) and
// slower alone (8192 tokens 41 us, otherwise 35.5; loads that stay 45).
template <typename T, typename O, bool INTER, bool STREAM>
__device__ __forceinline__ void rope_unit(const RopeArgs& a, int64_t token, int unit, int h0) {
  constexpr int N = 16 / sizeof(T);
  typedef T Run __attribute__((ext_vector_type(N)));
  typedef O Out __attribute__((ext_vector_type(N)));
  const int half = a.rot / 2, ch = N * unit;
  // first channels of the runs: of both elements of the pairs, or of the head's halves where pairs are neighbours
  int ca = ch, cb = a.dim / 2 + ch;
  if (!INTER) {
    const bool turns = ch < half;
    ca = turns ? ch : half + ch;                             // rot + (ch - half)
    cb = turns ? half + ch : a.dim / 2 + ch;                 // rot + (dim - rot) / 2 + (ch - half)
  }
  const bool turns_a = ca < a.rot, turns_b = cb < a.rot;
  Turn<N> w;
  if constexpr (INTER) {
    Turn<N / 2> u;
    if (turns_a) {
      u.load(a.table, a.max_pos, half, a.pos[token], ca / 2, a.sign);
#pragma unroll
      for (int j = 0; j < N / 2; ++j) w.c[j] = u.c[j], w.s[j] = u.s[j];
    }
    if (turns_b) {
      u.load(a.table, a.max_pos, half, a.pos[token], cb / 2, a.sign);
#pragma unroll
      for (int j = 0; j < N / 2; ++j) w.c[N / 2 + j] = u.c[j], w.s[N / 2 + j] = u.s[j];
    }
  } else {
    if (turns_a) w.load(a.table, a.max_pos, half, a.pos[token], ca, a.sign);
  }
  const int h1 = min(h0 + a.hpt, a.heads);
  const char* x = a.x + token * a.xt;
  char* y = a.y + token * a.yt;
  for (int h = h0; h < h1; h += 4) {
    Run ra[4], rb[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const char* p = x + min(h + i, h1 - 1) * a.xh;
      ra[i] = __builtin_nontemporal_load((const Run*)(p + ca * sizeof(T)));
      rb[i] = __builtin_nontemporal_load((const Run*)(p + cb * sizeof(T)));
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float e[2 * N];
#pragma unroll
      for (int j = 0; j < N; ++j) e[j] = (float)ra[i][j], e[N + j] = (float)rb[i][j];
      if (INTER) {
        if (turns_a)
#pragma unroll
          for (int j = 0; j < N / 2; ++j) turn(e[2 * j], e[2 * j + 1], w.c[j], w.s[j]);
        if (turns_b)
#pragma unroll
          for (int j = N / 2; j < N; ++j) turn(e[2 * j], e[2 * j + 1], w.c[j], w.s[j]);
      } else if (turns_a) {
#pragma unroll
        for (int j = 0; j < N; ++j) turn(e[j], e[N + j], w.c[j], w.s[j]);
      }
      if (h + i < h1) {
        O* r = (O*)(y + (h + i) * a.yh);
        Out oa, ob;
#pragma unroll
        for (int j = 0; j < N; ++j) oa[j] = (O)e[j], ob[j] = (O)e[N + j];
        if constexpr (STREAM) {
          __builtin_nontemporal_store(oa, (Out*)(r + ca));
          __builtin_nontemporal_store(ob, (Out*)(r + cb));
        } else {
          *(Out*)(r + ca) = oa;
          *(Out*)(r + cb) = ob;
        }
      }
    }
  }
}

// Thread `tid` of block `block` in a sequence of blocks over tokens of `per` units each: its token and unit. The
// long division is the block's, not the lane's.
__device__ __forceinline__ void place(uint32_t block, uint32_t per, int64_t& token, uint32_t& unit) {
  const uint64_t first = (uint64_t)block * kThreads;
  const uint64_t t0 = first / per;
  const uint32_t idx = (uint32_t)(first - t0 * per) + threadIdx.x;
  token = (int64_t)(t0 + idx / per);
  unit = idx % per;
}

// Bound by memory: 8192 tokens of 48 heads of 128 fp16 channels 35.5 us (5.7 TB/s read and written), 2051 tokens of 32 heads of
// 128 fp32 channels, half of them turned, 15 us (4.5 TB/s; a launch of a few tokens takes 3).
template <typename T, bool INTER>
__global__ __launch_bounds__(kThreads) void k_rope(RopeArgs a) {
  int64_t token;
  uint32_t unit;
  place(blockIdx.x, (uint32_t)a.dim / (32 / sizeof(T)), token, unit);
  if (token >= a.tokens) return;
  rope_unit<T, T, INTER, false>(a, token, (int)unit, blockIdx.y * a.hpt);
}

struct RopeFreqs {
  double f[256];
};

// One thread a position and pair. The angle and its cosine and sine are fp64: at position 10^6 an fp32 angle
// would be off by 0.03.
__global__ __launch_bounds__(kThreads) void k_rope_table(RopeFreqs f, int half, int64_t max_pos, double magnitude,
                                                         float* __restrict__ table) {
  int64_t p;
  uint32_t i;
  place(blockIdx.x, (uint32_t)half, p, i);
  if (p >= max_pos) return;
  double s, c;
  sincos((double)p * f.f[i], &s, &c);
  ((float2*)table)[p * half + i] = make_float2((float)(c * magnitude), (float)(s * magnitude));
}

// ------------------------------------------------------------------ writing

struct AppendArgs {
  CacheView c;
  const char *k, *v;
  int64_t kt, kh, vt, vh;  // strides in bytes
  const int32_t* slots;
  const int32_t* pos;      // NULL: keys are not rotated
  const float* table;
  int64_t max_pos;
  int64_t tokens;
  int rot;
  float sign;
  // The blocks that write the cache, bound by arithmetic when they quantise, are spread evenly among those that rotate queries, which
  // are bound by memory: block i is the (i kv_share / 2^32)-th of them if that number changes behind it.
  uint32_t kv_share;       // 0: all blocks write the cache
  uint32_t q_head_blocks;
  RopeArgs q;
};

template <int CTRL>
__device__ __forceinline__ float quad(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, false));
}
// over the four lanes that hold 32 channels
__device__ __forceinline__ float quad_min(float v) {
  v = fminf(v, quad<0xB1>(v));  // neighbours 1 0 3 2
  return fminf(v, quad<0x4E>(v));  // 2 3 0 1
}
__device__ __forceinline__ float quad_max(float v) {
  v = fmaxf(v, quad<0xB1>(v));
  return fmaxf(v, quad<0x4E>(v));
}

// One thread writes eight channels of one key or value row; four neighbouring lanes share an offset and a step.
// A rotated key's partner channels are read beside its own.
template <typename T, int BITS, bool INTER>
__device__ __forceinline__ void append_unit(const AppendArgs& a, int64_t token, uint32_t unit) {
  const CacheView& c = a.c;
  const uint32_t per_row = (uint32_t)c.dim / 8, per_kind = per_row * c.kv_heads;
  const bool is_v = unit >= per_kind;
  unit -= is_v ? per_kind : 0;
  const int head = unit / per_row, ch = 8 * (unit % per_row);
  const int slot = a.slots[token];
  if ((unsigned)slot >= (uint64_t)c.n_slots) return;  // the four lanes of a token's 32 channels leave together
  const char* row = is_v ? a.v + token * a.vt + head * a.vh : a.k + token * a.kt + head * a.kh;
  Row8<T> r;
  r.load(row + ch * sizeof(T));
  float x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = r.at(i);
  if (!is_v && a.pos && ch < a.rot) {
    const int half = a.rot / 2;
    Turn<8> w;
    if (INTER) {
      // four pairs: the second half of the eight that are loaded is unused and stays inside the row of the table
      const int pair = ch / 2, first = min(pair, half - 8);
      w.load(a.table, a.max_pos, half, a.pos[token], first, a.sign);
      const bool up = first != pair;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float cj = up ? w.c[j + 4] : w.c[j], sj = up ? w.s[j + 4] : w.s[j];
        turn(x[2 * j], x[2 * j + 1], cj, sj);
      }
    } else {
      const bool low = ch < half;
      w.load(a.table, a.max_pos, half, a.pos[token], low ? ch : ch - half, a.sign);
      Row8<T> o;
      o.load(row + (low ? ch + half : ch - half) * sizeof(T));
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float first = low ? x[i] : o.at(i), second = low ? o.at(i) : x[i];
        turn(first, second, w.c[i], w.s[i]);
        x[i] = low ? first : second;
      }
    }
  }
  const int64_t page = slot >> c.page_shift;
  const int in_page = slot & ((1 << c.page_shift) - 1);
  char* out = (is_v ? c.v : c.k) + page * c.page_stride + head * c.head_stride + in_page * c.token_stride;
  if constexpr (BITS == 16) {
    store8((_Float16*)out + ch, x);
  } else {
    constexpr float kTop = BITS == 8 ? 255.0f : 15.0f;
    float lo = x[0], hi = x[0], zero = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      lo = fminf(lo, x[i]);
      hi = fmaxf(hi, x[i]);
      zero = fmaf(x[i], 0.0f, zero);  // NaN from an infinity or a NaN on
    }
    lo = quad_min(lo), hi = quad_max(hi);
    const bool fits = quad_max(zero == 0.0f ? 0.0f : 1.0f) == 0.0f && lo >= -65504.0f && hi <= 65504.0f;
    _Float16 off = (_Float16)lo;
    float wide = fmaxf(hi - (float)off, 0.0f) * (1.0f / kTop);
    // an fp32 number, not a product rounded to fp16 at once: as in turn(), codes do not depend on what the compiler fuses
    asm("" : "+v"(wide));
    _Float16 step = (_Float16)wide;
    // rounded up, the step can carry the last level past fp16's range: then the next smaller one
    if ((float)off + kTop * (float)step > 65504.0f) step = __builtin_bit_cast(_Float16, (uint16_t)(__builtin_bit_cast(uint16_t, step) - 1));
    if (!fits) off = __builtin_bit_cast(_Float16, (uint16_t)0x7E00), step = (_Float16)0.0f;
    const float o = (float)off, d = (float)step, inv = d > 0.0f ? 1.0f / d : 0.0f;
    uint32_t q[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      // the quotient to its last bit, since fp16 inputs often lie exactly between two levels: one correction by the exact remainder
      const float y = x[i] - o, t = y * inv;
      q[i] = (uint32_t)__builtin_amdgcn_fmed3f(rintf(fmaf(fmaf(-t, d, y), inv, t)), 0.0f, kTop);
    }
    if constexpr (BITS == 8) {
      const uint32_t w0 = q[0] | q[1] << 8 | q[2] << 16 | q[3] << 24, w1 = q[4] | q[5] << 8 | q[6] << 16 | q[7] << 24;
      *(uint2*)(out + ch) = make_uint2(w0, w1);
    } else {
      uint32_t w = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) w |= q[i] << (4 * (i / 2) + 16 * (i % 2));
      *(uint32_t*)(out + ch / 2) = w;
    }
    if (ch % 32 == 0) {
      char* par = (is_v ? c.v_par : c.k_par) + page * c.par_page_stride + head * c.par_head_stride + in_page * c.par_token_stride;
      *(uint32_t*)(par + ch / 8) = (uint32_t)__builtin_bit_cast(uint16_t, off) | (uint32_t)__builtin_bit_cast(uint16_t, step) << 16;
    }
  }
}

// Bound by memory, and by the arithmetic of the codes beside it: 8192 tokens of 40 query and 8 kv heads of 128 channels into 4 bits 51 us
// (137 MB read, 97 written: 4.6 TB/s, vector ALU 42% busy); 64 tokens into 8 bits 3.6 us, the launch's latency.
template <typename T, int BITS, bool INTER>
__global__ __launch_bounds__(kThreads) void k_kv_append(AppendArgs a) {
  int64_t token;
  uint32_t unit;
  uint32_t kv_block = blockIdx.x;
  if (a.kv_share) {
    kv_block = __umulhi(blockIdx.x, a.kv_share);
    if (__umulhi(blockIdx.x + 1, a.kv_share) == kv_block) {
      const uint32_t q_block = blockIdx.x - kv_block;
      place(q_block / a.q_head_blocks, (uint32_t)a.c.dim / (32 / sizeof(T)), token, unit);
      if (token >= a.tokens) return;
      rope_unit<T, _Float16, INTER, true>(a.q, token, (int)unit, (int)(q_block % a.q_head_blocks) * a.q.hpt);
      return;
    }
  }
  place(kv_block, (uint32_t)(a.c.dim / 8) * 2 * a.c.kv_heads, token, unit);
  if (token >= a.tokens) return;
  append_unit<T, BITS, INTER>(a, token, unit);
}

// ------------------------------------------------------------------ reading

// One thread reads eight channels of one key row and of the value row beside it. Bound by memory: 32768 tokens of 8 heads of 128
// channels at 8 bits 34.8 us (6.0 TB/s; with stores that stay in the caches 43.5), 701 tokens of 3 heads of 96 in fp16 2.7 us, the launch's latency.
template <int BITS>
__global__ __launch_bounds__(kThreads) void k_kv_read(CacheView c, int64_t tokens, const int32_t* __restrict__ slots,
                                                      _Float16* __restrict__ ko, _Float16* __restrict__ vo) {
  int64_t token;
  uint32_t unit;
  const uint32_t per_row = (uint32_t)c.dim / 8;
  place(blockIdx.x, per_row * c.kv_heads, token, unit);
  if (token >= tokens) return;
  const int head = unit / per_row, ch = 8 * (unit % per_row);
  const int slot = slots[token];
  f16x8 k = {}, v = {};
  if ((unsigned)slot < (uint64_t)c.n_slots) {
    const int64_t page = slot >> c.page_shift;
    const int in_page = slot & ((1 << c.page_shift) - 1);
    const int64_t at = page * c.page_stride + head * c.head_stride + in_page * c.token_stride + ch * BITS / 8;
    if constexpr (BITS == 16) {
      k = *(const f16x8*)(c.k + at);
      v = *(const f16x8*)(c.v + at);
    } else {
      const int64_t par = page * c.par_page_stride + head * c.par_head_stride + in_page * c.par_token_stride + ch / 32 * 4;
      k = decode8<BITS>(c.k + at, *(const uint32_t*)(c.k_par + par));
      v = decode8<BITS>(c.v + at, *(const uint32_t*)(c.v_par + par));
    }
  }
  const int64_t to = (token * c.kv_heads + head) * c.dim + ch;
  __builtin_nontemporal_store(k, (f16x8*)(ko + to));
  __builtin_nontemporal_store(v, (f16x8*)(vo + to));
}

// ------------------------------------------------------------------ host side

template <typename... A>
sph_status launch(const void* fn, dim3 grid, hipStream_t s, A... args) {
  void* kargs[] = {(void*)&args...};
  if (hipLaunchKernel(fn, grid, dim3(kThreads), kargs, 0, s) != hipSuccess) return SPH_ERR_HIP;
  return hipGetLastError() == hipSuccess ? SPH_OK : SPH_ERR_HIP;
}

// Blocks over units * tokens threads. At most 2^26 tokens of 2 * 1024 * 32 units: 2^42 threads need more blocks than a
// launch takes, so such calls are refused (below 2^32 threads all fit).
bool blocks_for(int64_t tokens, int64_t per, uint32_t* blocks) {
  const int64_t b = (tokens * per + kThreads - 1) / kThreads;
  if (b >= (int64_t(1) << 24)) return false;
  *blocks = (uint32_t)b;
  return true;
}

// Heads a thread rotates: as many as leave about four waves a SIMD (2^18 threads), four at a time, so that a token's
// angles are read once for them.
int heads_per_thread(int64_t tokens, int heads, int units) {
  const int64_t threads = tokens * heads * units;
  const int64_t want = std::max<int64_t>(1, threads >> 18);
  return want < 4 ? (int)want : (int)std::min<int64_t>((want + 3) / 4 * 4, std::min(heads, 16));
}

sph_status check_rope(const sph_rope_desc* r, int head_dim) {
  if (!r->d_table) return SPH_ERR_NULL;
  if (r->max_pos < 1 || r->max_pos > INT32_MAX || r->rot_dim < 16 || r->rot_dim % 16 || r->rot_dim > head_dim ||
      (uintptr_t)r->d_table % 16 || (r->flags & ~(SPH_ROPE_INTERLEAVED | SPH_ROPE_INVERSE)))
    return SPH_ERR_SHAPE;
  return SPH_OK;
}

// 16-byte rows of elements of `size` bytes. Strides are only used by calls with more than one token or head, but have to be aligned always.
bool rows_ok(const void* p, int64_t ts, int64_t hs, int size) {
  const int64_t lim = int64_t(1) << 40;
  return (uintptr_t)p % 16 == 0 && ts >= 0 && hs >= 0 && ts < lim && hs < lim && ts * size % 16 == 0 && hs * size % 16 == 0;
}

// Rows that are written must not share their first byte.
bool apart(int64_t tokens, int64_t ts, int64_t heads, int64_t hs) { return (tokens < 2 || ts > 0) && (heads < 2 || hs > 0); }

bool tokens_ok(int64_t t) { return t >= 0 && t <= (int64_t(1) << 26); }

}  // namespace

int sph_cache_check(const sph_kv_cache* c) {
  if (c->bits != 16 && c->bits != 8 && c->bits != 4) return SPH_ERR_UNSUPPORTED_FORMAT;
  const int d = c->head_dim;
  if (d != 64 && d != 96 && d != 128 && d != 192 && d != 256) return SPH_ERR_UNSUPPORTED_FORMAT;
  if (!c->d_k || !c->d_v || (c->bits < 16 && (!c->d_k_par || !c->d_v_par))) return SPH_ERR_NULL;
  const int ps = c->page_size;
  if (ps < 1 || ps > 65536 || (ps & (ps - 1)) || c->kv_heads < 1 || c->kv_heads > 1024 || c->n_pages < 1 ||
      c->n_pages > INT32_MAX / ps)
    return SPH_ERR_SHAPE;
  const int64_t row = (int64_t)d * c->bits / 8, lim = int64_t(1) << 40;
  if ((uintptr_t)c->d_k % 16 || (uintptr_t)c->d_v % 16) return SPH_ERR_SHAPE;
  for (int64_t s : {c->page_stride, c->head_stride, c->token_stride})
    if (s < row || s >= lim || s % 16) return SPH_ERR_SHAPE;
  if ((int64_t)ps * c->token_stride > INT32_MAX) return SPH_ERR_SHAPE;
  if (c->bits < 16) {
    if ((uintptr_t)c->d_k_par % 4 || (uintptr_t)c->d_v_par % 4) return SPH_ERR_SHAPE;
    for (int64_t s : {c->par_page_stride, c->par_head_stride, c->par_token_stride})
      if (s < d / 8 || s >= lim || s % 4) return SPH_ERR_SHAPE;
    if ((int64_t)ps * c->par_token_stride > INT32_MAX) return SPH_ERR_SHAPE;
  }
  return SPH_OK;
}

CacheView sph_cache_view(const sph_kv_cache* c) {
  CacheView v{};
  v.k = (char*)c->d_k, v.v = (char*)c->d_v, v.k_par = (char*)c->d_k_par, v.v_par = (char*)c->d_v_par;
  v.page_stride = c->page_stride, v.head_stride = c->head_stride, v.token_stride = c->token_stride;
  v.par_page_stride = c->par_page_stride, v.par_head_stride = c->par_head_stride, v.par_token_stride = c->par_token_stride;
  v.n_pages = c->n_pages, v.n_slots = c->n_pages * c->page_size;
  v.kv_heads = c->kv_heads, v.dim = c->head_dim;
  while ((1 << v.page_shift) < c->page_size) ++v.page_shift;
  return v;
}

extern "C" {

sph_status sph_rope_table(int32_t rot_dim, int64_t max_pos, const double* inv_freq, double magnitude, float* d_table,
                          void* stream) {
  if (!inv_freq || !d_table) return SPH_ERR_NULL;
  if (rot_dim < 16 || rot_dim % 16 || rot_dim > 512 || max_pos < 1 || max_pos > INT32_MAX || (uintptr_t)d_table % 16) return SPH_ERR_SHAPE;
  RopeFreqs f{};
  for (int i = 0; i < rot_dim / 2; ++i) {
    if (!std::isfinite(inv_freq[i])) return SPH_ERR_BAD_VALUE;
    f.f[i] = inv_freq[i];
  }
  if (!std::isfinite(magnitude)) return SPH_ERR_BAD_VALUE;
  uint32_t blocks;
  if (!blocks_for(max_pos, rot_dim / 2, &blocks)) return SPH_ERR_SHAPE;
  return launch((const void*)k_rope_table, dim3(blocks), (hipStream_t)stream, f, (int)(rot_dim / 2), max_pos, magnitude, d_table);
}

sph_status sph_rope(const sph_rope_desc* rope, sph_dtype dtype, int64_t tokens, int32_t heads, int32_t head_dim,
                    const void* d_x, int64_t x_token_stride, int64_t x_head_stride, const int32_t* d_pos, void* d_y,
                    int64_t y_token_stride, int64_t y_head_stride, void* stream) {
  if (!rope) return SPH_ERR_NULL;
  if ((dtype != SPH_F16 && dtype != SPH_F32) || !tokens_ok(tokens) || heads < 1 || heads > 65535 || head_dim < 16 ||
      head_dim % 16 || head_dim > 512)
    return SPH_ERR_SHAPE;
  if (const sph_status st = check_rope(rope, head_dim)) return st;
  if (tokens == 0) return SPH_OK;
  if (!d_x || !d_y || !d_pos) return SPH_ERR_NULL;
  const int size = dtype == SPH_F16 ? 2 : 4;
  if (!rows_ok(d_x, x_token_stride, x_head_stride, size) || !rows_ok(d_y, y_token_stride, y_head_stride, size) || (uintptr_t)d_pos % 4 ||
      !apart(tokens, y_token_stride, heads, y_head_stride))
    return SPH_ERR_SHAPE;
  RopeArgs a{};
  a.x = (const char*)d_x, a.y = (char*)d_y;
  a.xt = x_token_stride * size, a.xh = x_head_stride * size, a.yt = y_token_stride * size, a.yh = y_head_stride * size;
  a.pos = d_pos, a.table = rope->d_table, a.max_pos = rope->max_pos;
  a.tokens = tokens, a.heads = heads, a.dim = head_dim, a.rot = rope->rot_dim;
  const int units = head_dim * size / 32;
  a.hpt = heads_per_thread(tokens, heads, units);
  a.sign = rope->flags & SPH_ROPE_INVERSE ? -1.0f : 1.0f;
  uint32_t blocks;
  if (!blocks_for(tokens, units, &blocks)) return SPH_ERR_SHAPE;
  const dim3 grid(blocks, (unsigned)((heads + a.hpt - 1) / a.hpt));
  const bool inter = rope->flags & SPH_ROPE_INTERLEAVED;
  const void* fn = dtype == SPH_F16 ? (inter ? (const void*)k_rope<_Float16, true> : (const void*)k_rope<_Float16, false>)
                                    : (inter ? (const void*)k_rope<float, true> : (const void*)k_rope<float, false>);
  return launch(fn, grid, (hipStream_t)stream, a);
}

sph_status sph_kv_append(const sph_kv_cache* cache, const sph_rope_desc* rope, sph_dtype dtype, int64_t tokens,
                         const void* d_k, int64_t k_token_stride, int64_t k_head_stride, const void* d_v,
                         int64_t v_token_stride, int64_t v_head_stride, const int32_t* d_slots, int32_t q_heads,
                         const void* d_q, int64_t q_token_stride, int64_t q_head_stride, void* d_q_out,
                         int64_t qo_token_stride, int64_t qo_head_stride, const int32_t* d_pos, void* stream) {
  if (!cache) return SPH_ERR_NULL;
  if (const int st = sph_cache_check(cache)) return (sph_status)st;
  if ((dtype != SPH_F16 && dtype != SPH_F32) || !tokens_ok(tokens) || q_heads < 0 || q_heads > 65535) return SPH_ERR_SHAPE;
  if (rope) {
    if (const sph_status st = check_rope(rope, cache->head_dim)) return st;
  } else if (q_heads) {
    return SPH_ERR_NULL;
  }
  if (tokens == 0) return SPH_OK;
  if (!d_k || !d_v || !d_slots || (rope && !d_pos) || (q_heads && (!d_q || !d_q_out))) return SPH_ERR_NULL;
  const int size = dtype == SPH_F16 ? 2 : 4;
  if (!rows_ok(d_k, k_token_stride, k_head_stride, size) || !rows_ok(d_v, v_token_stride, v_head_stride, size) ||
      (uintptr_t)d_slots % 4 || (uintptr_t)d_pos % 4)
    return SPH_ERR_SHAPE;
  if (q_heads && (!rows_ok(d_q, q_token_stride, q_head_stride, size) || !rows_ok(d_q_out, qo_token_stride, qo_head_stride, 2) ||
                  !apart(tokens, qo_token_stride, q_heads, qo_head_stride)))
    return SPH_ERR_SHAPE;
  AppendArgs a{};
  a.c = sph_cache_view(cache);
  a.k = (const char*)d_k, a.v = (const char*)d_v;
  a.kt = k_token_stride * size, a.kh = k_head_stride * size, a.vt = v_token_stride * size, a.vh = v_head_stride * size;
  a.slots = d_slots;
  a.tokens = tokens;
  bool inter = false;
  if (rope) {
    a.pos = d_pos, a.table = rope->d_table, a.max_pos = rope->max_pos, a.rot = rope->rot_dim;
    a.sign = rope->flags & SPH_ROPE_INVERSE ? -1.0f : 1.0f;
    inter = rope->flags & SPH_ROPE_INTERLEAVED;
  }
  uint32_t kv_blocks, unit_blocks = 0;
  uint64_t q_blocks = 0;
  if (!blocks_for(tokens, (int64_t)cache->head_dim / 8 * 2 * cache->kv_heads, &kv_blocks)) return SPH_ERR_SHAPE;
  if (q_heads) {
    RopeArgs& q = a.q;
    q.x = (const char*)d_q, q.y = (char*)d_q_out;
    q.xt = q_token_stride * size, q.xh = q_head_stride * size, q.yt = qo_token_stride * 2, q.yh = qo_head_stride * 2;
    q.pos = d_pos, q.table = rope->d_table, q.max_pos = rope->max_pos, q.sign = a.sign;
    q.tokens = tokens, q.heads = q_heads, q.dim = cache->head_dim, q.rot = rope->rot_dim;
    const int units = cache->head_dim * size / 32;
    q.hpt = heads_per_thread(tokens, q_heads, units);
    if (!blocks_for(tokens, units, &unit_blocks)) return SPH_ERR_SHAPE;
    a.q_head_blocks = (uint32_t)((q_heads + q.hpt - 1) / q.hpt);
    q_blocks = (uint64_t)unit_blocks * a.q_head_blocks;
    if (q_blocks + kv_blocks >= (1u << 24)) return SPH_ERR_SHAPE;
    // rounded up: floor(total * share / 2^32) is kv_blocks, since total < 2^32
    a.kv_share = (uint32_t)((((uint64_t)kv_blocks << 32) + q_blocks + kv_blocks - 1) / (q_blocks + kv_blocks));
  }
  const void* fn = nullptr;
#define SPH_PICK(B)                                                                                                    \
  fn = dtype == SPH_F16 ? (inter ? (const void*)k_kv_append<_Float16, B, true> : (const void*)k_kv_append<_Float16, B, false>) \
                        : (inter ? (const void*)k_kv_append<float, B, true> : (const void*)k_kv_append<float, B, false>)
  if (cache->bits == 16) SPH_PICK(16);
  if (cache->bits == 8) SPH_PICK(8);
  if (cache->bits == 4) SPH_PICK(4);
#undef SPH_PICK
  return launch(fn, dim3((uint32_t)q_blocks + kv_blocks), (hipStream_t)stream, a);
}

sph_status sph_kv_read(const sph_kv_cache* cache, int64_t tokens, const int32_t* d_slots, void* d_k_out, void* d_v_out,
                       void* stream) {
  if (!cache) return SPH_ERR_NULL;
  if (const int st = sph_cache_check(cache)) return (sph_status)st;
  if (!tokens_ok(tokens)) return SPH_ERR_SHAPE;
  if (tokens == 0) return SPH_OK;
  if (!d_slots || !d_k_out || !d_v_out) return SPH_ERR_NULL;
  if ((uintptr_t)d_slots % 4 || (uintptr_t)d_k_out % 16 || (uintptr_t)d_v_out % 16) return SPH_ERR_SHAPE;
  uint32_t blocks;
  if (!blocks_for(tokens, (int64_t)cache->head_dim / 8 * cache->kv_heads, &blocks)) return SPH_ERR_SHAPE;
  const CacheView v = sph_cache_view(cache);
  const void* fn = cache->bits == 16 ? (const void*)k_kv_read<16> : cache->bits == 8 ? (const void*)k_kv_read<8> : (const void*)k_kv_read<4>;
  return launch(fn, dim3(blocks), (hipStream_t)stream, v, tokens, d_slots, (_Float16*)d_k_out, (_Float16*)d_v_out);
}

}  // extern "C"
