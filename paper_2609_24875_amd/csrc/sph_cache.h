// What the cache's writer, its reader and the attention share: the view of the pages that kernels take and
// the numbers that codes stand for.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/sph.h"

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// sph_kv_cache as kernels read it; strides in bytes.
struct CacheView {
  char *k, *v, *k_par, *v_par;
  int64_t page_stride, head_stride, token_stride;
  int64_t par_page_stride, par_head_stride, par_token_stride;
  int64_t n_pages, n_slots;
  int kv_heads, dim, page_shift;
};

int sph_cache_check(const sph_kv_cache* c);
CacheView sph_cache_view(const sph_kv_cache* c);

// Two codes as fp16 numbers: a code below 1024 in the mantissa of 1024.0 (0x6400) is 1024 + code exactly, so the
// packed subtraction gives the code exactly, and one packed multiply-add rounds offset + code * step once.
__device__ __forceinline__ f16x2 decode2(uint32_t mantissas, f16x2 step, f16x2 off) {
  const f16x2 q = __builtin_bit_cast(f16x2, mantissas | 0x64006400u) - (f16x2){(_Float16)1024.0f, (_Float16)1024.0f};
  return __builtin_elementwise_fma(q, step, off);
}

// Eight channels from two words of bytes, or from one word of nibbles (channels 2i and 2i + 1 at bits 4i and 16 + 4i).
template <int BITS>
__device__ __forceinline__ f16x8 decode8w(uint32_t w0, uint32_t w1, uint32_t par) {
  const f16x2 p = __builtin_bit_cast(f16x2, par);
  const f16x2 off = {p[0], p[0]}, step = {p[1], p[1]};
  f16x2 r[4];
  if constexpr (BITS == 8) {
    // bytes 0 and 1 (2 and 3) of a word to the low bytes of two halves
    r[0] = decode2(__builtin_amdgcn_perm(0, w0, 0x0C010C00u), step, off);
    r[1] = decode2(__builtin_amdgcn_perm(0, w0, 0x0C030C02u), step, off);
    r[2] = decode2(__builtin_amdgcn_perm(0, w1, 0x0C010C00u), step, off);
    r[3] = decode2(__builtin_amdgcn_perm(0, w1, 0x0C030C02u), step, off);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = decode2((w0 >> (4 * i)) & 0x000F000Fu, step, off);
  }
  f16x8 y;
#pragma unroll
  for (int i = 0; i < 4; ++i) y[2 * i] = r[i][0], y[2 * i + 1] = r[i][1];
  return y;
}

template <int BITS>
__device__ __forceinline__ f16x8 decode8(const char* p, uint32_t par) {
  if constexpr (BITS == 8) {
    const uint2 w = *(const uint2*)p;
    return decode8w<8>(w.x, w.y, par);
  } else {
    return decode8w<4>(*(const uint32_t*)p, 0, par);
  }
}
