// The attention of more rows of a kv head, as sph_attn_wide.hip describes it: tiles of keys in LDS.
#pragma once
#include "sph_attn.h"

namespace {

template <int DIM, int BITS>
struct Wide {
  // Keys of a tile: 64 where the scores of so many leave room for the output's registers (4096 tokens of 32 heads of 192 channels: 351 us,
  // with 32 425).
  static constexpr int kTile = DIM <= 192 ? 64 : 32;
  // Codes are loaded a whole tile ahead where they fit the registers, else when the tile before begins: held through the weights'
  // products, 8-bit codes of 128 and 256 channels spill, and at 64 channels cost the third wave a SIMD (4096 tokens of 32 heads with either:
  // 4 bits, 64 channels 144 and 130 us, 128 211 and 220, 192 430 and 444, 256 648 and 666; 8 bits, 128 226 and 224, 192 434 and 432, 256 660 and 653).
  static constexpr bool kAhead = BITS == 4 && DIM > 64;
  static constexpr int kPer = DIM / 8;                       // pieces of eight channels in a row
  static constexpr int kPieces = kTile * kPer / kThreads;    // a thread's share of a tile's keys, and of its values
  static constexpr int kWords = BITS / 4;                    // of a piece as stored
  static constexpr int kRow = DIM * 2;                       // bytes of a row in LDS
  static constexpr int kHalf = kTile * kRow;                 // keys, then values
  static_assert(kTile * kPer % kThreads == 0, "whole shares");
  // Rows as in RowPlaces: for keys, one piece of 16 rows or two neighbouring pieces of eight are read together; for values, four
  // neighbouring pieces of four rows.
  static constexpr int kSkip = kPer % 16;
  __device__ static __forceinline__ int key_turn(int row) { return RowPlaces<DIM>::turn(row); }
  __device__ static __forceinline__ int value_turn(int row) {
    if constexpr (kSkip == 0) return (row & 3) << 2;
    if constexpr (kSkip == 8) return (row >> 1 & 1) << 2;
    return 0;
  }
  __device__ static __forceinline__ int key_at(int row, int piece) { return RowPlaces<DIM>::at(row, piece); }
  __device__ static __forceinline__ int value_at(int row, int piece) { return row * kRow + ((piece ^ value_turn(row)) << 4); }
};

template <int DIM, int BITS>
struct Share {
  typedef Wide<DIM, BITS> W;
  uint32_t k[W::kPieces][W::kWords], v[W::kPieces][W::kWords], k_par[W::kPieces], v_par[W::kPieces];
};

template <int BITS>
__device__ __forceinline__ f16x8 decoded(const uint32_t* w, uint32_t par) {
  if constexpr (BITS == 16) return __builtin_bit_cast(f16x8, make_uint4(w[0], w[1], w[2], w[3]));
  if constexpr (BITS == 8) return decode8w<8>(w[0], w[1], par);
  return decode8w<4>(w[0], 0, par);
}

__device__ __forceinline__ int64_t shuffled(int64_t v, int from) {
  return (int64_t)(uint32_t)__shfl((int)(uint32_t)v, from) | (int64_t)__shfl((int)(v >> 32), from) << 32;
}

// page: lane l holds the page of key kt + l % kTile.
template <int DIM, int BITS>
__device__ __forceinline__ void load_share(Share<DIM, BITS>& s, const Pages& pg, int page, int kt) {
  typedef Wide<DIM, BITS> W;
  const int in_page = (kt + ((threadIdx.x & 63) & (W::kTile - 1))) & pg.mask;
  const int64_t off = page * pg.stride + (uint32_t)(in_page * pg.token);
  const int64_t par_off = BITS < 16 ? page * pg.par_stride + (uint32_t)(in_page * pg.par_token) : 0;
#pragma unroll
  for (int i = 0; i < W::kPieces; ++i) {
    const int idx = threadIdx.x + kThreads * i, row = idx / W::kPer, piece = idx % W::kPer;
    const int64_t at = shuffled(off, row) + piece * BITS;
    load_words<BITS>(pg.k + at, s.k[i]);
    load_words<BITS>(pg.v + at, s.v[i]);
    if constexpr (BITS < 16) {
      const int64_t pat = shuffled(par_off, row) + piece / 4 * 4;
      s.k_par[i] = *(const uint32_t*)(pg.k_par + pat);
      s.v_par[i] = *(const uint32_t*)(pg.v_par + pat);
    }
  }
}

// fp16 pages go to LDS without passing registers: the wave's lanes fill 1 KiB in order, so each takes the piece that belongs there.
template <int DIM>
__device__ __forceinline__ void load_direct(char* lds, const Pages& pg, int page, int kt, int wave) {
  typedef Wide<DIM, 16> W;
  const int in_page = (kt + ((threadIdx.x & 63) & (W::kTile - 1))) & pg.mask;
  const int64_t off = page * pg.stride + (uint32_t)(in_page * pg.token);
#pragma unroll
  for (int i = 0; i < W::kPieces; ++i) {
    const int idx = threadIdx.x + kThreads * i, row = idx / W::kPer, piece = idx % W::kPer;
    const int64_t at = shuffled(off, row);
    char* to = lds + (kThreads * i + 64 * wave) * 16;
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(pg.k + at + ((piece ^ W::key_turn(row)) << 4)),
                                     (__attribute__((address_space(3))) void*)to, 16, 0, 0);
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(pg.v + at + ((piece ^ W::value_turn(row)) << 4)),
                                     (__attribute__((address_space(3))) void*)(to + W::kHalf), 16, 0, 0);
  }
}

template <int DIM, int BITS>
__device__ __forceinline__ void store_share(const Share<DIM, BITS>& s, char* lds) {
  typedef Wide<DIM, BITS> W;
  int thread = threadIdx.x;
  // (opaque: places are computed here, not kept in registers around the loop)
  if constexpr (!W::kAhead) asm volatile("" : "+v"(thread));
#pragma unroll
  for (int i = 0; i < W::kPieces; ++i) {
    const int idx = thread + kThreads * i, row = idx / W::kPer, piece = idx % W::kPer;
    *(f16x8*)(lds + W::key_at(row, piece)) = decoded<BITS>(s.k[i], s.k_par[i]);
    *(f16x8*)(lds + W::kHalf + W::value_at(row, piece)) = decoded<BITS>(s.v[i], s.v_par[i]);
  }
}

// The thread's own values of a tile that not every row sees, in LDS: see k_attn's loop. Returns whether there was an infinity or a NaN.
template <int DIM, int BITS>
__device__ __forceinline__ bool clean_share(char* lds, int kt, int k_lo, int k_hi, uint64_t gone) {
  typedef Wide<DIM, BITS> W;
  bool odd = false;
#pragma unroll 1
  for (int i = 0; i < W::kPieces; ++i) {
    const int idx = threadIdx.x + kThreads * i, row = idx / W::kPer, piece = idx % W::kPer;
    odd |= clean_piece(lds + W::kHalf + W::value_at(row, piece), kt + row < k_lo || kt + row >= k_hi || (gone >> row & 1));
  }
  return odd;
}

}  // namespace
