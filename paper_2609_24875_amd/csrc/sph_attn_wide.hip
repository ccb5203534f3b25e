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
  static constexpr int kTile = DIM <= 128 ? 64 : 32;
  static constexpr int kPer = DIM / 8;                       // pieces of eight channels in a row
  static constexpr int kPieces = kTile * kPer / kThreads;    // a thread's share of a tile's keys, and of its values
  static constexpr int kWords = BITS / 4;                    // of a piece as stored
  static constexpr int kRow = DIM * 2;                       // bytes of a row in LDS
  static constexpr int kHalf = kTile * kRow;                 // keys, then values
  static_assert(kTile * kPer % kThreads == 0, "whole shares");
  // Where a row's piece lies in its LDS row. Keys: eight lanes read one piece of eight rows at once; values: 16 lanes read two
  // neighbouring pieces of four rows. Rows of a power of two would share their banks, so their pieces are permuted.
  __device__ static __forceinline__ int key_at(int row, int piece) {
    if constexpr (DIM == 64) return row * kRow + ((piece ^ ((row >> 1) & 7)) << 4);
    if constexpr (DIM == 128 || DIM == 256) return row * kRow + ((piece ^ (row & 15)) << 4);
    return row * kRow + (piece << 4);
  }
  __device__ static __forceinline__ int value_at(int row, int piece) {
    if constexpr (DIM == 64) return row * kRow + ((piece ^ (((row >> 1) & 3) << 1)) << 4);
    if constexpr (DIM == 128 || DIM == 256) return row * kRow + ((piece ^ ((row & 7) << 1)) << 4);
    return row * kRow + (piece << 4);
  }
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

template <int DIM, int BITS>
__device__ __forceinline__ void store_share(const Share<DIM, BITS>& s, char* lds) {
  typedef Wide<DIM, BITS> W;
#pragma unroll
  for (int i = 0; i < W::kPieces; ++i) {
    const int idx = threadIdx.x + kThreads * i, row = idx / W::kPer, piece = idx % W::kPer;
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

template <int DIM, int BITS>
__global__ __launch_bounds__(kThreads, (DIM <= 128 ? 2 : 1)) void k_attn_wide(AttnArgs) {
  const AttnArgs& a = *(const AttnArgs*)__builtin_amdgcn_kernarg_segment_ptr();
  typedef Wide<DIM, BITS> W;
  constexpr int kTile = W::kTile, kSteps = DIM / 16, kBlocks = DIM / 32, kKeys = kTile / 32;
  __shared__ __attribute__((aligned(16))) char lds[2][2 * W::kHalf];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, h = lane >> 5;
  uint32_t id = blockIdx.x;
  const int kvh = id % a.c.kv_heads;
  id /= a.c.kv_heads;
  const int tile = a.tiles - 1 - (int)(id % a.tiles);        // the last rows see most
  id /= a.tiles;
  const int b = id % a.batch, split = id / a.batch;
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
  float m = -INFINITY, base = 0.0f, l = 0.0f;
  bool odd = false;
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
    const int k0 = k_lo & ~(kTile - 1);
    int page = page_of(k0), next = page_of(min(k0 + kTile, k_hi - 1));
    uint64_t gone = __ballot(!pg.there(page));
    load_share(S, pg, pg.there(page) ? page : 0, k0);
    store_share(S, lds[0]);
    if (!span.whole(k0) || gone) odd |= clean_share<DIM, BITS>(lds[0], k0, k_lo, k_hi, gone);
    uint64_t next_gone = __ballot(!pg.there(next));
    load_share(S, pg, pg.there(next) ? next : 0, min(k0 + kTile, (k_hi - 1) & ~(kTile - 1)));
    __syncthreads();
    int buf = 0;
    for (int kt = k0; kt < k_hi; kt += kTile, buf ^= 1) {
      const char* ks = lds[buf];
      const char* vs = lds[buf] + W::kHalf;
      const bool more = kt + kTile < k_hi;
      const int nn = min(kt + 2 * kTile, (k_hi - 1) & ~(kTile - 1));
      next = page_of(nn);
      const bool work = w0 < nrow && kt <= wave_hi && (!a.window || kt + kTile > wave_lo - a.window + 1);
      f32x16 st[kKeys] = {};
      if (work) {
#pragma unroll
        for (int i = 0; i < kSteps; ++i)
#pragma unroll
          for (int u = 0; u < kKeys; ++u)
            st[u] = __builtin_amdgcn_mfma_f32_32x32x16_f16(*(const f16x8*)(ks + W::key_at(32 * u + col, 2 * i + h)), q[i], st[u], 0, 0, 0);
      }
      const uint64_t now_gone = gone;
      if (more) {
        char* to = lds[buf ^ 1];
        store_share(S, to);
        gone = next_gone;
        if (!span.whole(kt + kTile) || gone) odd |= clean_share<DIM, BITS>(to, kt + kTile, k_lo, k_hi, gone);
        next_gone = __ballot(!pg.there(next));
        load_share(S, pg, pg.there(next) ? next : 0, nn);
      }
      if (work) {
        const bool whole = kt >= k_lo && kt + kTile <= k_hi && kt + kTile - 1 <= wave_lo && (!a.window || kt > wave_hi - a.window) && !now_gone;
        if (!whole) {
          int at_pos = pos;
          asm volatile("" : "+v"(at_pos));  // keeps the branch
#pragma unroll
          for (int u = 0; u < kKeys; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int kk = 32 * u + 8 * (i >> 2) + 4 * h + (i & 3);
              st[u][i] = !span.seen(kt + kk, at_pos) ? -INFINITY : (now_gone >> kk & 1) ? __builtin_nanf("") : st[u][i];
            }
        }
        float top = -INFINITY;
#pragma unroll
        for (int u = 0; u < kKeys; ++u)
#pragma unroll
          for (int i = 0; i < 16; i += 2) top = fmaxf(top, fmaxf(st[u][i], st[u][i + 1]));
        // -inf times a scale of 0 is NaN, which raises nothing: with nothing seen m stays -inf
        if (__any(top * scale > m + 8.0f)) {
          float mn = fmaxf(m, top * scale);
          mn = fmaxf(mn, __shfl_xor(mn, 32));
          base = mn == -INFINITY ? 0.0f : mn;
          const float keep = __builtin_amdgcn_exp2f(m - base);
          m = mn;
          l *= keep;
#pragma unroll
          for (int i = 0; i < kBlocks; ++i) o[i] *= keep;
        }
#pragma unroll
        for (int u = 0; u < kKeys; ++u)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            f16x8 p;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const float x = __builtin_amdgcn_exp2f(fmaf(st[u][8 * e + i], scale, -base));
              l += x;
              p[i] = (_Float16)x;
            }
#pragma unroll
            for (int i = 0; i < kBlocks; ++i) {
              f16x8 vt;
#pragma unroll
              for (int j = 0; j < 2; ++j) {
                const int row = 32 * u + 16 * e + 8 * j + 4 * h + ((lane & 15) >> 2), piece = 4 * i + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
                const s16x4 w = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (__attribute__((address_space(3))) s16x4*)(vs + W::value_at(row, piece) + 8 * (lane & 1)));
                const f16x4 f = __builtin_bit_cast(f16x4, w);
#pragma unroll
                for (int x = 0; x < 4; ++x) vt[4 * j + x] = f[x];
              }
              o[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vt, p, o[i], 0, 0, 0);
            }
          }
      }
      __syncthreads();
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
        write_part(a, split * a.batch + b, kvh, r, ch, acc, m, l);
      else
        write_out(a, s.start + t, head, ch, acc, m, l);
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
