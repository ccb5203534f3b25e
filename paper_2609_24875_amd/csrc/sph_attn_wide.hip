// Attention of many new tokens: more rows a kv head than k_attn's 32 (prompts, long drafts).
//
// A workgroup takes 128 rows (tokens times the query heads of a kv head's group, so the group shares what is loaded) and
// goes through the keys they see in tiles that its four waves share in LDS, each wave 32 rows. Products are
// v_mfma_f32_32x32x16_f16: S^T = K Q^T with a row per key and a column per query row leaves a lane 16 keys of one row
// for every 32, and O^T = V^T P^T takes its weights from the same lane: keys 4 h .. 4 h + 3 and 8 + 4 h .. of each 16 (h = lane / 32), in
// which order V^T's operand is read by transposing reads.
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
  // A row's pieces are permuted within it, piece p to place p ^ turn(row), so that lanes that read together find 16 different 16-byte
  // places of the 256 bytes of banks: for keys, one piece of 16 rows or two neighbouring pieces of eight; for values, four neighbouring
  // pieces of four rows. kSkip is what a row adds to the place.
  static constexpr int kSkip = kPer % 16;
  __device__ static __forceinline__ int key_turn(int row) {
    if constexpr (kSkip == 0) return (row & 7) << 1 | (row >> 3 & 1);
    if constexpr (kSkip == 8) return (row >> 1 & 3) << 1 | (row >> 3 & 1);
    return (row >> 2 & 1) << 1 | (row >> 3 & 1);
  }
  __device__ static __forceinline__ int value_turn(int row) {
    if constexpr (kSkip == 0) return (row & 3) << 2;
    if constexpr (kSkip == 8) return (row >> 1 & 1) << 2;
    return 0;
  }
  __device__ static __forceinline__ int key_at(int row, int piece) { return row * kRow + ((piece ^ key_turn(row)) << 4); }
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

// What bounds it: matrix products and exponentials together, on two waves a SIMD (one above 128 channels). 2048 new tokens behind 14336
// others, 32 query heads over 8 kv heads of 128 channels, fp16: 577 to 602 us from card to card, 890 to 855 TFLOP/s at a clock
// that the products lower to about 2.0 GHz; MFMA
// 40%, vector ALU 42%, LDS 25% busy, no bank conflicts. Twice the rows a wave halve its LDS reads, but leave one wave a SIMD, which
// does not overlap its products with its weights well enough: 920 us. 4096 tokens over themselves at 8 bits 224 us, 4 bits 211, fp16 185.
template <int DIM, int BITS>
__global__ __launch_bounds__(kThreads, (DIM <= 128 ? 2 : 1)) void k_attn_wide(AttnArgs) {
  const AttnArgs& a = *(const AttnArgs*)__builtin_amdgcn_kernarg_segment_ptr();
  typedef Wide<DIM, BITS> W;
  constexpr int kTile = W::kTile, kSteps = DIM / 16, kBlocks = DIM / 32, kKeys = kTile / 32;
  // two arrays, not one of two: loads on their way into one do not hold up reads of the other
  __shared__ __attribute__((aligned(16))) char lds_a[2 * W::kHalf], lds_b[2 * W::kHalf];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, h = lane >> 5;
  uint32_t id = blockIdx.x;
  const int kvh = id % a.c.kv_heads;
  id /= a.c.kv_heads;
  const int place = id % a.tiles;
  id /= a.tiles;
  const int b = id % a.batch, split = id / a.batch;
  // The last rows see most, so they come first. Where all workgroups are resident at once, two on some CUs (see plan_of), the ones that
  // share a CU, a.fold places apart, are a long and a short one, and the longest have theirs alone.
  int tile = a.tiles - 1 - place;
  if (a.fold && a.batch > 1) {
    if (b * a.tiles >= a.fold) tile = place;
  } else if (a.fold) {
    const int shared = a.tiles - a.fold;
    tile = place < shared ? 2 * shared - 1 - place : place < a.fold ? a.tiles - 1 - (place - shared) : place - a.fold;
  }
  Seq s;
  s.load(a, b);
  if (s.bad) {
    if (tile == 0 && split == 0) write_bad(a, s, kvh);
    return;
  }
  const int rows = s.n * a.group, r0 = tile * kWideRows;
  if (r0 >= rows) return;
  const int nrow = min(kWideRows, rows - r0), first = s.len - s.n;
  const int p_lo = first + r0 / a.group, p_hi = first + (r0 + nrow - 1) / a.group;
  const int lo = a.window ? max(0, p_lo - a.window + 1) : 0, hi = p_hi + 1;
  const int k_lo = max(lo, (lo & ~(kTile - 1)) + split * a.chunk), k_hi = min(hi, (lo & ~(kTile - 1)) + (split + 1) * a.chunk);
  const Span span = {k_lo, k_hi, p_lo, p_hi, a.window, kTile};
  const int32_t* pages = a.pages + b * a.pages_stride;
  Pages pg;
  pg.set(a.c, kvh);

  const int w0 = 32 * wave;                                  // the wave's rows: none if w0 >= nrow
  const int r = r0 + min(w0 + col, nrow - 1), t = r / a.group, head = kvh * a.group + r % a.group, pos = first + t;
  const int wave_lo = first + (r0 + min(w0, nrow - 1)) / a.group, wave_hi = first + (r0 + min(w0 + 31, nrow - 1)) / a.group;
  f32x16 o[kBlocks] = {};
  Ref ref = {-INFINITY, 0.0f};
  float l = 0.0f;
  bool odd = false, far = false;
  if (k_lo < k_hi) {
    // |scale| is applied to the scores, its sign to the queries
    // (a scale of 0 as one that rounds every score to 0, since 0 times the -inf of an unseen key would be NaN)
    const float scale = fmaxf(fabsf(a.scale), 1e-30f);
    const uint32_t flip = a.scale < 0.0f ? 0x80008000u : 0u;
    f16x8 q[kSteps];
    const char* qr = a.q + (s.start + t) * a.qt + head * a.qh;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      u32x4 w = *(const u32x4*)(qr + 2 * (16 * i + 8 * h));
      w ^= flip;
      q[i] = __builtin_bit_cast(f16x8, w);
    }
    const int e_lo = k_lo >> pg.shift, e_hi = (k_hi - 1) >> pg.shift;
    auto page_of = [&](int kt) { return pages[min(max((kt + (lane & (kTile - 1))) >> pg.shift, e_lo), e_hi)]; };
    Share<DIM, BITS> S;
    constexpr bool kDirect = BITS == 16;
    const int k0 = k_lo & ~(kTile - 1), k_last = (k_hi - 1) & ~(kTile - 1);
    int page = page_of(k0), next = page_of(min(k0 + kTile, k_last));
    uint64_t gone = __ballot(!pg.there(page));
    page = pg.there(page) ? page : 0;
    if constexpr (kDirect) {
      load_direct<DIM>(lds_a, pg, page, k0, wave);
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    } else {
      load_share(S, pg, page, k0);
      store_share(S, lds_a);
    }
    if (!span.whole(k0) || gone) odd |= clean_share<DIM, BITS>(lds_a, k0, k_lo, k_hi, gone);
    if constexpr (W::kAhead) load_share(S, pg, pg.there(next) ? next : 0, min(k0 + kTile, k_last));
    __syncthreads();
    auto tile_at = [&](int kt, const char* ks, char* to) __attribute__((always_inline)) {
      const char* vs = ks + W::kHalf;
      const bool more = kt + kTile < k_hi;
      const uint64_t now_gone = gone;
      gone = __ballot(!pg.there(next));
      page = pg.there(next) ? next : 0;
      next = page_of(min(kt + 2 * kTile, k_last));
      if constexpr (!kDirect && !W::kAhead) {
        if (more) load_share(S, pg, page, kt + kTile);
      }
      const bool work = w0 < nrow && kt <= wave_hi && (!a.window || kt + kTile > wave_lo - a.window + 1);
      f32x16 st[kKeys] = {};
      if (work) {
        // keys are read two steps before their products, in this order
        f16x8 kf[kSteps][kKeys];
        auto read = [&](int i) {
#pragma unroll
          for (int u = 0; u < kKeys; ++u) kf[i][u] = *(const f16x8*)(ks + W::key_at(32 * u + col, 2 * i + h));
        };
        read(0);
        read(1);
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
          if (i + 2 < kSteps) read(i + 2);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int u = 0; u < kKeys; ++u) st[u] = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf[i][u], q[i], st[u], 0, 0, 0);
        }
      }
      // everyone left the other buffer at the last barrier; behind the products, whose time hides the addresses' arithmetic
      if constexpr (kDirect) {
        if (more) load_direct<DIM>(to, pg, page, kt + kTile, wave);
      }
      if constexpr (!kDirect) {
        if (more) {
          store_share(S, to);
          if constexpr (W::kAhead) load_share(S, pg, pg.there(next) ? next : 0, min(kt + 2 * kTile, k_last));
        }
      }
      if (work) {
        const bool whole = kt >= k_lo && kt + kTile <= k_hi && kt + kTile - 1 <= wave_lo && (!a.window || kt > wave_hi - a.window) && !now_gone;
        if (!whole) {
          // (opaque here: a branch stays, and what its tests compare with is not kept in registers around the loop)
          int at_pos = pos, key = kt + 4 * h;
          asm volatile("" : "+v"(at_pos), "+v"(key));
#pragma unroll
          for (int u = 0; u < kKeys; ++u) {
            uint32_t lost = (uint32_t)(now_gone >> (32 * u)) >> (4 * h);
            asm volatile("" : "+v"(lost));
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int kk = 8 * (i >> 2) + (i & 3);
              st[u][i] = !span.seen(key + 32 * u + kk, at_pos) ? -INFINITY : (lost >> kk & 1) ? __builtin_nanf("") : st[u][i];
            }
          }
        }
        float top = -INFINITY;
#pragma unroll
        for (int u = 0; u < kKeys; ++u)
#pragma unroll
          for (int i = 0; i < 16; i += 2) top = fmaxf(top, fmaxf(st[u][i], st[u][i + 1]));
        // (far scores are rounded here: one that is not before the subtraction may lie above a reference that is, by more than fp16 holds)
        float by = scale;
        if (far | __any(top * scale > ref.top)) {
          float mn = top * scale;
          mn = fmaxf(mn, __shfl_xor(mn, 32));
          float keep;
          if (ref.raise(mn, keep)) {
            l *= keep;
#pragma unroll
            for (int i = 0; i < kBlocks; ++i) o[i] *= keep;
          }
          far = __any(fabsf(ref.base) >= kFar);
          if (far) {
#pragma unroll
            for (int u = 0; u < kKeys; ++u) st[u] *= scale;
            by = 1.0f;
          }
        }
        // In steps of 16 keys: while a step's products run, the values of the next are read and its weights computed.
        constexpr int kGroups = 2 * kKeys;
        f16x8 vt[kGroups][kBlocks], p[kGroups];
        auto read_values = [&](int g) {
#pragma unroll
          for (int i = 0; i < kBlocks; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              const int row = 16 * g + 8 * j + 4 * h + ((lane & 15) >> 2), piece = 4 * i + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
              const s16x4 w = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                  (__attribute__((address_space(3))) s16x4*)(vs + W::value_at(row, piece) + 8 * (lane & 1)));
              const f16x4 f = __builtin_bit_cast(f16x4, w);
#pragma unroll
              for (int x = 0; x < 4; ++x) vt[g][i][4 * j + x] = f[x];
            }
        };
        auto weights = [&](int g) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float x = __builtin_amdgcn_exp2f(fmaf(st[g >> 1][8 * (g & 1) + i], by, -ref.base));
            l += x;
            p[g][i] = (_Float16)x;
          }
        };
        read_values(0);
        weights(0);
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
          if (g + 1 < kGroups) read_values(g + 1);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int i = 0; i < kBlocks; ++i) o[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vt[g][i], p[g], o[i], 0, 0, 0);
          if (g + 1 < kGroups) weights(g + 1);
        }
      }
      if constexpr (kDirect) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      if (more && (!span.whole(kt + kTile) || gone)) odd |= clean_share<DIM, BITS>(to, kt + kTile, k_lo, k_hi, gone);
      __syncthreads();
    };
    for (int kt = k0; kt < k_hi; kt += 2 * kTile) {
      tile_at(kt, lds_a, lds_b);
      if (kt + kTile >= k_hi) break;
      tile_at(kt + kTile, lds_b, lds_a);
    }
    l += __shfl_xor(l, 32);
  }
  const bool any_odd = __syncthreads_or(odd);
  if (w0 + col >= nrow) return;
#pragma unroll
  for (int i = 0; i < kBlocks; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int ch = 32 * i + 8 * j + 4 * h;
      f32x4 acc = {o[i][4 * j], o[i][4 * j + 1], o[i][4 * j + 2], o[i][4 * j + 3]};
      if (any_odd) acc += odd_values<DIM, BITS>(span, pg, pages, pos, ch);
      if (a.splits > 1)
        write_part(a, split * a.batch + b, kvh, r, ch, acc, ref.log(), l);
      else
        write_out(a, s.start + t, head, ch, acc, ref.log(), l);
    }
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
