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

#include "sph_attn_few.h"
#include "sph_attn_plan.h"

namespace {

template <int DIM, int BITS, int NB, bool UNI>
__global__ __launch_bounds__(kThreads, (DIM * NB <= 64 ? 3 : DIM * NB <= 128 ? (BITS == 4 ? 3 : 2) : 1)) void k_attn(AttnArgs) {
  // read where they are used: kept for the whole kernel, the arguments would push the loop's scalars out of their registers
  const AttnArgs& a = *(const AttnArgs*)__builtin_amdgcn_kernarg_segment_ptr();
  constexpr int kRows = 16 * NB, kVBytes = kTile * Lay<DIM, BITS>::kVStride, kOBytes = kRows * (DIM + 4) * 4;
  __shared__ __attribute__((aligned(16))) char lds[kWaves * (kVBytes > kOBytes ? kVBytes : kOBytes)];
  __shared__ float2 ml_s[kWaves][kRows];
  __shared__ int before[kEvenBatch + 1], sums[kEvenBatch / 32];
  typedef AttnArgs A;
  const uint32_t block = blockIdx.x;
#include "sph_attn_few.inc"
}


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

// Whether launches take it (and rows of a sequence fit 32 bits).
bool launchable(const Plan& p) { return p.grid < (1 << 24) && (!p.bytes || p.joins < (1 << 26)); }

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
