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

// Two codes as fp16 numbers, from halves that hold `one` + code (a power of two with the code in its mantissa): the packed
// subtraction gives the code exactly, and one packed multiply-add rounds offset + code * step once.
__device__ __forceinline__ f16x2 decode2(uint32_t halves, float one, f16x2 step, f16x2 off) {
  const f16x2 q = __builtin_bit_cast(f16x2, halves) - (f16x2){(_Float16)one, (_Float16)one};
  return __builtin_elementwise_fma(q, step, off);
}

// Eight channels from two words of bytes, or from one word of nibbles (channels 2i and 2i + 1 at bits 4i and 16 + 4i).
template <int BITS>
__device__ __forceinline__ f16x8 decode8w(uint32_t w0, uint32_t w1, uint32_t par) {
  const f16x2 p = __builtin_bit_cast(f16x2, par);
  const f16x2 off = {p[0], p[0]}, step = {p[1], p[1]};
  f16x2 r[4];
  if constexpr (BITS == 8) {
    // two bytes of a word below the high byte of 1024.0 (0x6400), whose last bit is worth 1
    r[0] = decode2(__builtin_amdgcn_perm(0x64646464u, w0, 0x04010400u), 1024.0f, step, off);
    r[1] = decode2(__builtin_amdgcn_perm(0x64646464u, w0, 0x04030402u), 1024.0f, step, off);
    r[2] = decode2(__builtin_amdgcn_perm(0x64646464u, w1, 0x04010400u), 1024.0f, step, off);
    r[3] = decode2(__builtin_amdgcn_perm(0x64646464u, w1, 0x04030402u), 1024.0f, step, off);
  } else {
    // bits 4..7 are worth 1..8 in 64.0 (0x5400), which spares every other shift
    uint32_t low = 0x000F000Fu, high = 0x00F000F0u, m1024 = 0x64006400u, m64 = 0x54005400u;
    // in registers, one of each pair scalar: v_and_or_b32 takes no literals
    asm("" : "+s"(low), "+s"(high), "+v"(m1024), "+v"(m64));
    const uint32_t w8 = w0 >> 8;
    r[0] = decode2((w0 & low) | m1024, 1024.0f, step, off);
    r[1] = decode2((w0 & high) | m64, 64.0f, step, off);
    r[2] = decode2((w8 & low) | m1024, 1024.0f, step, off);
    r[3] = decode2((w8 & high) | m64, 64.0f, step, off);
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
