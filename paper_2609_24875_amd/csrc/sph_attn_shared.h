// The kernels of sph_attention_shared, whose sources are a file for each number of bits (see sph_attn_shared.hip).
#pragma once
#include "sph_attn_few.h"
#include "sph_attn_many.h"

// Which of the two ways (up to 32 rows of a kv head, or more) the prefixes and the own tokens go. Behind a prefix are at least as many rows as
// of any of its sequences.
enum SharedKind { kFewFew, kManyFew, kManyMany };

// The kernel for a number of bits; nb: blocks of 16 rows of the way for up to 32, uni: pages of 16 tokens and more.
const void* sph_attn_shared_kernel16(int dim, SharedKind kind, int nb, bool uni);
const void* sph_attn_shared_kernel8(int dim, SharedKind kind, int nb, bool uni);
const void* sph_attn_shared_kernel4(int dim, SharedKind kind, int nb, bool uni);

namespace {

// A sequence's own tokens.
struct OwnArgs : AttnArgs {
  static constexpr bool kParts = true;
};

// A prefix as a sequence whose new tokens are those of all sequences behind it: first[g] .. first[g + 1] - 1 of `seqs`, or with
// first NULL all.
struct PrefixArgs : AttnArgs {
  static constexpr bool kParts = true, kFlat = true;
  const int32_t* first;
  int seqs;
  __device__ __forceinline__ void tokens_of(int g, int& start, int& end) const {
    const int s0 = first ? first[g] : 0, s1 = first ? first[g + 1] : seqs;
    const bool there = s0 >= 0 && s0 <= s1 && s1 <= seqs;
    start = !there ? -1 : q_start ? q_start[s0] : s0;
    end = !there ? -1 : q_start ? q_start[s1] : s1;
  }
};

struct SharedArgs {
  OwnArgs own;
  PrefixArgs pre;
  int* descends;           // of more prefixes than a wave looks at at once: 1 if their starts descend anywhere, else 0
  uint32_t check, pre_blocks, blocks;   // workgroups before all others that find `descends`, 0 or 1; of the prefixes; of them and the own tokens
  int64_t pre_part;        // rows of parts before the prefixes'
  bool pre_many, own_many;
};

template <int DIM, int BITS, int NB, int KIND>
struct SharedLds {
  static constexpr int kFew = kWaves * (kTile * Lay<DIM, BITS>::kVStride > 16 * NB * (DIM + 4) * 4 ? kTile * Lay<DIM, BITS>::kVStride : 16 * NB * (DIM + 4) * 4);
  static constexpr int kMany = 2 * Wide<DIM, BITS>::kHalf;
  static constexpr int kA = KIND == kFewFew ? kFew : KIND == kManyMany || kMany > kFew ? kMany : kFew, kB = KIND == kFewFew ? 16 : kMany;
};

template <int DIM, int BITS, int NB, bool UNI, int KIND>
__global__ __launch_bounds__(kThreads, (DIM * NB <= 128 ? 2 : 1)) void k_attn_shared(SharedArgs) {
  const SharedArgs& both = *(const SharedArgs*)__builtin_amdgcn_kernarg_segment_ptr();
  typedef SharedLds<DIM, BITS, NB, KIND> L;
  // (two arrays, as k_attn_wide's; the other way uses the first)
  __shared__ __attribute__((aligned(16))) char lds_a[L::kA], lds_b[L::kB];
  __shared__ float2 ml_s[KIND == kManyMany ? 1 : kWaves][16 * NB];
  __shared__ int before[KIND == kManyMany ? 1 : kEvenBatch + 1], sums[KIND == kManyMany ? 1 : kEvenBatch / 32];
  const uint32_t place = blockIdx.x - both.check;            // (of the one that finds `descends`: above all others)
  if (place < both.pre_blocks) {
    typedef PrefixArgs A;
    const A& a = both.pre;
    const uint32_t block = place;
    if constexpr (KIND == kFewFew) {
      char* lds = lds_a;
#include "sph_attn_few.inc"
    } else {
      typedef Wide<DIM, BITS> W;
#include "sph_attn_many.inc"
    }
  } else if (place < both.blocks) {
    typedef OwnArgs A;
    const A& a = both.own;
    const uint32_t block = place - both.pre_blocks;
    if constexpr (KIND == kManyMany) {
      typedef Wide<DIM, BITS> W;
#include "sph_attn_many.inc"
    } else {
      char* lds = lds_a;
#include "sph_attn_few.inc"
    }
  } else {
    // (first of all: as the last it was the launch's end, 2 us of 603 with 1000 prefixes)
    const PrefixArgs& a = both.pre;
    bool down = false;
    for (int g = threadIdx.x; g < a.batch; g += kThreads) down |= a.first[g] > a.first[g + 1];
    const bool any = __syncthreads_or(down);
    if (threadIdx.x == 0) *both.descends = any;
  }
}

// (One block of rows where it does, also with pages of less than 16 tokens: two leave a CU one workgroup. Pages of 8: 8 prefixes of up to 4099 tokens with
// 8 sequences of up to 700 each at 8 bits 46 us, 74 by two blocks; 32 behind 8192 in fp16 28 and 39.)
template <int DIM, int BITS, bool UNI>
const void* shared_kernel(SharedKind kind, int nb) {
  if (kind == kFewFew) return nb == 1 ? (const void*)k_attn_shared<DIM, BITS, 1, UNI, kFewFew> : (const void*)k_attn_shared<DIM, BITS, 2, UNI, kFewFew>;
  return nb == 1 ? (const void*)k_attn_shared<DIM, BITS, 1, UNI, kManyFew> : (const void*)k_attn_shared<DIM, BITS, 2, UNI, kManyFew>;
}

template <int DIM, int BITS>
const void* shared_kernel(SharedKind kind, int nb, bool uni) {
  if (kind == kManyMany) return (const void*)k_attn_shared<DIM, BITS, 1, true, kManyMany>;
  if constexpr (DIM > 128) {
    if (kind == kFewFew) return uni ? (const void*)k_attn_shared<DIM, BITS, 1, true, kFewFew> : (const void*)k_attn_shared<DIM, BITS, 1, false, kFewFew>;
    return uni ? (const void*)k_attn_shared<DIM, BITS, 1, true, kManyFew> : (const void*)k_attn_shared<DIM, BITS, 1, false, kManyFew>;
  } else {
    return uni ? shared_kernel<DIM, BITS, true>(kind, nb) : shared_kernel<DIM, BITS, false>(kind, nb);
  }
}

template <int BITS>
const void* shared_kernel(int dim, SharedKind kind, int nb, bool uni) {
  switch (dim) {
    case 64: return shared_kernel<64, BITS>(kind, nb, uni);
    case 96: return shared_kernel<96, BITS>(kind, nb, uni);
    case 128: return shared_kernel<128, BITS>(kind, nb, uni);
    case 192: return shared_kernel<192, BITS>(kind, nb, uni);
    default: return shared_kernel<256, BITS>(kind, nb, uni);
  }
}

}  // namespace
