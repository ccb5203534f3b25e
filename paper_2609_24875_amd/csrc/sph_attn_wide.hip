// Attention of many new tokens: more rows a kv head than k_attn's 32 (prompts, long drafts).
//
// A workgroup takes 128 rows (tokens times the query heads of a kv head's group, so the group shares what is loaded) and
// goes through the keys they see in tiles that its four waves share in LDS, each wave 32 rows. Products are
// v_mfma_f32_32x32x16_f16: S^T = K Q^T with a row per key and a column per query row leaves a lane 16 keys of one row
// for every 32, and O^T = V^T P^T takes its weights from the same lane: keys 4 h .. 4 h + 3 and 8 + 4 h .. of each 16 (h = lane / 32), in
// which order V^T's operand is read by transposing reads.
#include "sph_attn_many.h"

namespace {

// What bounds it: matrix products and exponentials together, on two waves a SIMD (one above 128 channels). 2048 new tokens behind 14336
// others, 32 query heads over 8 kv heads of 128 channels, fp16: 577 to 602 us from card to card, 890 to 855 TFLOP/s at a clock
// that the products lower to about 2.0 GHz; MFMA
// 40%, vector ALU 42%, LDS 25% busy, no bank conflicts. Twice the rows a wave halve its LDS reads, but leave one wave a SIMD, which
// does not overlap its products with its weights well enough: 920 us. 4096 tokens over themselves at 8 bits 224 us, 4 bits 211, fp16 185.
template <int DIM, int BITS>
__global__ __launch_bounds__(kThreads, (DIM <= 128 ? 2 : 1)) void k_attn_wide(AttnArgs) {
  const AttnArgs& a = *(const AttnArgs*)__builtin_amdgcn_kernarg_segment_ptr();
  typedef Wide<DIM, BITS> W;
  // two arrays, not one of two: loads on their way into one do not hold up reads of the other
  __shared__ __attribute__((aligned(16))) char lds_a[2 * W::kHalf], lds_b[2 * W::kHalf];
  typedef AttnArgs A;
  const uint32_t block = blockIdx.x;
#include "sph_attn_many.inc"
}

template <int BITS>
const void* kernel_for(int dim) {
  return dim == 64    ? (const void*)k_attn_wide<64, BITS>
         : dim == 96  ? (const void*)k_attn_wide<96, BITS>
         : dim == 128 ? (const void*)k_attn_wide<128, BITS>
         : dim == 192 ? (const void*)k_attn_wide<192, BITS>
                      : (const void*)k_attn_wide<256, BITS>;
}

}  // namespace

const void* sph_attn_wide_kernel(int bits, int dim) { return bits == 16 ? kernel_for<16>(dim) : bits == 8 ? kernel_for<8>(dim) : kernel_for<4>(dim); }
