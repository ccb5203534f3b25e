// Attention of sequences that share long prefixes (sph_attention_shared).
//
// The rows of all sequences behind a prefix go through its keys together, as one sequence of so many rows that see all of it: what is read
// once serves all of them, and makes rows enough for the matrix products that prompts have. Beside that every sequence goes through its own tokens
// as ever. Both write parts (o, m, l), sums relative to 2^m, and the join adds a row's: o = sum_i o_i 2^(m_i - m), l = sum_i l_i 2^(m_i - m)
// with m the largest, and o / l at the end. One launch does both kinds, so that the prefix's products run beside the own tokens' reads; the
// join is the second. Parts are fp32, weights fp16 as in sph_attention: 2.2e-4 to 2.8e-4 relative to 64 bits, where a plain form has 2.1e-4.
//
// 32 query heads over 8 of 128 channels, fp16, kernel and join: 128 sequences of 1024 own tokens behind 32768 shared 161 + 8 us, bound by the prefix's
// products and the own tokens' reads side by side (alone 100 and 92); 32 of up to 512 behind 8192 19 + 7 (alone 17.7 and 12.6), the first tiles' and the
// join's latency: a workgroup's first tile of 64 keys takes 10 us, the second 2, later ones 1.3 each. Measured and not kept, of these two and of 8 times 8 at
// 8 bits (now 161, 19 and 41): own tokens' workgroups first 201, 28 and 50; prefixes by blocks of 32 rows through k_attn's way -, 40 and 52.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "sph_attn_plan.h"
#include "sph_attn_shared.h"

const void* sph_attn_shared_kernel16(int dim, SharedKind kind, int nb, bool uni) { return shared_kernel<16>(dim, kind, nb, uni); }

namespace {

// The prefix whose sequences are first[g] .. first[g + 1] - 1 with b among them, -1 for none. By a whole wave, 64 places at once. down: the starts descend
// anywhere, so that two prefixes may claim a sequence (and have written its parts over each other's), or one that belongs to a prefix be found by none.
__device__ __forceinline__ int prefix_of(const PrefixArgs& a, const int* descends, int b, bool& down) {
  if (!a.first) return 0;
  const int lane = threadIdx.x & 63, all = a.batch + 1;
  const int here = all > 64 ? *descends : a.first[min(lane, all - 1)], next = all > 64 ? 0 : a.first[min(lane + 1, all - 1)];
  if (all <= 64) {
    // (ascending, the lanes that are not above b are the first few)
    const int last = 63 - __builtin_clzll(__ballot(lane < all && here <= b) | 1);
    down = __any(here > next);
    return last < a.batch && __builtin_amdgcn_readlane(here, last) <= b ? last : -1;
  }
  int lo = 0, n = all;                                       // among the n entries from lo on, the last that is not above b
  while (n > 1) {
    const int step = (n + 63) / 64, at = lane * step;
    const int last = 63 - __builtin_clzll(__ballot(at < n && a.first[lo + min(at, n - 1)] <= b) | 1);
    lo += last * step;
    n = min(step, n - last * step);
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  down = __any(here > next);
  return lo < a.batch && a.first[lo] <= b && b < a.first[lo + 1] ? lo : -1;
}

// Joins the parts of a row, its own tokens' and then its prefix's, in this order: as k_attn_join. Bound by latency, 4 to 9 us: what a row needs to find its
// parts and the first of these are loaded at once, before it is known whether the lengths are right and which maximum is the largest.
template <bool FEW>
__global__ __launch_bounds__(kThreads) void k_attn_shared_join(SharedArgs both) {
  const OwnArgs& a = both.own;
  const int lane = threadIdx.x & 63;
  const uint32_t per = FEW ? a.c.dim / 4 : kJoinCh / 4, groups = 64 / per, chunks = FEW ? 1 : a.c.dim / kJoinCh, rows = a.max_q * a.group;
  uint32_t id = blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (id >= chunks * a.c.kv_heads * rows * a.batch) return;
  const uint32_t group = lane / per, ch = id % chunks * kJoinCh + lane % per * 4;
  id /= chunks;
  const int kvh = id % a.c.kv_heads;
  id /= a.c.kv_heads;
  const int row = id % rows, b = id / rows, head = kvh * a.group + row % a.group;
  // Where the row's parts are, whether or not its sequence and prefix turn out to be right: what is right is loaded beside the parts.
  const PrefixArgs& p = both.pre;
  Seq s;
  s.load(a, b);
  const int64_t token = (int64_t)s.start + row / a.group;
  bool down = false;
  const int g = prefix_of(p, both.descends, b, down);
  // (a token outside the arrays is a wrong one's: any part)
  const int64_t near = min(max(token, (int64_t)0), a.tokens - 1);
  int2 w = make_int2(b, both.own_many ? a.splits : 1);
  if (!both.own_many && (a.shares || a.each > 0)) w = a.where[b];
  const int64_t first = both.own_many ? token_part_at(a, 0, kvh, near, row % a.group) : part_at(a, w.x, kvh, row);
  const int64_t step = both.own_many ? (int64_t)a.c.kv_heads * (a.tokens * a.group) : part_at(a, 1, kvh, row) - part_at(a, 0, kvh, row);
  int64_t pre_first = 0, pre_step = 0;
  int parts = w.y, pre_parts = 0;
  bool bad = s.bad | down;
  if (g >= 0) {
    Seq q;
    q.load(p, g);
    // (a token that is not among the prefix's has starts that do not ascend)
    bad |= q.bad || token < q.start || token >= q.end;
    if (both.pre_many) {
      pre_step = (int64_t)a.c.kv_heads * (a.tokens * a.group);
      pre_first = both.pre_part + token_part_at(a, 0, kvh, near, row % a.group), pre_parts = p.splits;
    } else {
      w = p.shares || p.each > 0 ? p.where[g] : make_int2(g, 1);
      const int r = (int)min(max(token - q.start, (int64_t)0), (int64_t)p.max_q - 1) * a.group + row % a.group;
      pre_first = part_at(p, w.x, kvh, r), pre_step = part_at(p, w.x + 1, kvh, r) - pre_first, pre_parts = w.y;
      pre_first += both.pre_part;
    }
  }
  // (slots that no sequence wrote are anything)
  if (!both.own_many && (a.shares || a.each > 0) && (s.n == 0 || bad)) parts = 0;
  if (!both.pre_many && (p.shares || p.each > 0) && bad) pre_parts = 0;
  const int all = parts + pre_parts;
  auto at_of = [&](int i) { return i < parts ? first + i * step : pre_first + (i - parts) * pre_step; };
  constexpr int kLoads = 5;                                  // of a lane before it knows the maximum
  float2 ml[kLoads];
  f32x4 part[kLoads];
#pragma unroll
  for (int u = 0; u < kLoads; ++u) {
    const int i = group + u * groups;
    ml[u] = make_float2(-INFINITY, 0.0f), part[u] = f32x4{};
    if (group < groups && i < all) {
      const int64_t at = at_of(i);
      ml[u] = a.ml[at];
      part[u] = *(const f32x4*)(a.part + at * a.c.dim + ch);
    }
  }
  if (bad) {
    // every token that the sequence claims, though there may be more than max_q
    const float nan = __builtin_nanf("");
    const int64_t end = s.bad ? min((int64_t)s.end, a.tokens) : row < s.n * a.group ? token + 1 : token;
    const int64_t t0 = token < 0 ? token + (a.max_q - 1 - token) / a.max_q * a.max_q : token;
    if (group == 0)
      for (int64_t t = t0; t < end; t += a.max_q) write_out(a, t, head, ch, f32x4{nan, nan, nan, nan}, 0.0f, nan);
    return;
  }
  if (row >= s.n * a.group) return;
  float mm = -INFINITY;
#pragma unroll
  for (int u = 0; u < kLoads; ++u) mm = fmaxf(mm, ml[u].x);
  for (int i = kLoads * groups + lane; i < all; i += 64) mm = fmaxf(mm, a.ml[at_of(i)].x);
#pragma unroll
  for (int d = 32; d; d >>= 1) mm = fmaxf(mm, __shfl_xor(mm, d));
  const float ref = mm == -INFINITY ? 0.0f : mm;
  f32x4 acc = {};
  float l = 0.0f;
#pragma unroll
  for (int u = 0; u < kLoads; ++u) {
    const float f = __builtin_amdgcn_exp2f(ml[u].x - ref);
    l += f * ml[u].y;
    acc += f * part[u];
  }
  if (group < groups) {
#pragma unroll 4
    for (int i = group + kLoads * groups; i < all; i += groups) {
      const int64_t at = at_of(i);
      const float2 m = a.ml[at];
      const f32x4 x = *(const f32x4*)(a.part + at * a.c.dim + ch);
      const float f = __builtin_amdgcn_exp2f(m.x - ref);
      l += f * m.y;
      acc += f * x;
    }
  }
  // the groups' sums, in order, to the first
  for (uint32_t k = 1; k < groups; ++k) {
    const float more = __shfl(l, (int)(k * per + lane % per));
    l += group ? 0.0f : more;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float x = __shfl(acc[i], (int)(k * per + lane % per));
      acc[i] += group ? 0.0f : x;
    }
  }
  if (group == 0) write_out(a, token, head, ch, acc, mm, l);
}

// ------------------------------------------------------------------ host side

struct SharedPlan {
  Plan own, pre;
  int64_t pre_q;                           // tokens behind a prefix at most
  int own_each, pre_each;                  // as AttnArgs has it
  size_t own_parts, pre_parts, bytes;
  size_t flag;                             // of the bytes: SharedArgs::descends, behind everything else
  int64_t joins;
  bool few;
  SharedKind kind;
};

// Rows that are joined anyway can do with more workgroups than k_attn's plan gives short sequences: up to one a CU, by the host's bounds and without
// counting shares, and so for one sequence of any length. Three sequences behind 512 tokens 8.8 us with four workgroups a kv head for the prefix, 11.7
// with one; behind 768 8.5 and 14.3; four behind 1031 9.6, with shares that are counted 11.9.
// Many short ones go the other way: a wave for each and kv head, four to a workgroup, where there are waves enough for as many steps more (32 tokens
// a step). 8 kv heads of 128 channels behind 4096: 128 sequences of 128 tokens 39.4 -> 33.8 us, of 512 71 -> 66, of 2048 106 -> 108; 64 of 128 28.0 -> 25.9, of 512
// 49.5 -> 55; 32 of 128 23.0 -> 21.8, of 256 24.3 -> 24.5; 80 of 36 under 16 heads of 256, where a CU has one workgroup, behind 166 67 -> 37.
int each_of(const sph_kv_cache* c, Plan& p, int64_t n, int64_t max_len) {
  if (p.wide || !n || (p.shares && n > 1)) return 0;
  if (!p.shares && max_len <= kTile * std::min<int64_t>(32, n * c->kv_heads / 64)) {
    p.grid = c->kv_heads * ((n + kWaves - 1) / kWaves);
    return kAlone;
  }
  const int64_t steps = (max_len + kTile * kWaves - 1) / (kTile * kWaves);
  const int64_t most = n == 1 ? std::max<int64_t>(1, kCus * workgroups_per_cu(c) / c->kv_heads) : kCus / (c->kv_heads * n);
  const int64_t each = std::min({steps, most, (int64_t)kMaxSplits});
  if (each < 2) return 0;
  p.shares = 0, p.grid = c->kv_heads * n * each;
  return (int)each;
}

SharedPlan shared_plan(const sph_kv_cache* c, int64_t prefixes, int64_t max_group, int64_t max_prefix, int64_t batch, int64_t tokens,
                       int q_heads, int64_t max_q, int64_t max_len) {
  SharedPlan p{};
  const int64_t group = q_heads / c->kv_heads, rows = max_q * group;
  p.pre_q = std::max(max_q, std::min(tokens, max_group * max_q));
  p.own = plan_of(c, batch, q_heads, max_q, max_len, 0);
  p.pre = plan_of(c, prefixes, q_heads, p.pre_q, max_prefix, 0);
  p.own.fold = p.pre.fold = 0;             // (for workgroups that are alone in their launch)
  p.own_each = each_of(c, p.own, batch, max_len), p.pre_each = each_of(c, p.pre, prefixes, max_prefix);
  if (p.pre.wide) {
    // A workgroup a CU, beside which the own tokens' are, and two where prefixes are several, since ragged ones leave many with little to do. One
    // prefix of 32768 tokens before 128 sequences of 1024 161 us, with two 195; 8 of up to 4099 before 8 each of up to 700 at 8 bits 48 and 46. Above 128 channels
    // a CU holds one workgroup: one then, too (256 channels at 8 bits, 4 prefixes of up to 2000 before 32 each of up to 200: 76 us, with two 87).
    const int64_t units = c->kv_heads * prefixes * p.pre.tiles, tile = sph_attn_wide_tile(c->head_dim);
    const int64_t want = std::max<int64_t>(1, (prefixes > 1 && c->head_dim <= 128 ? 2 : 1) * kCus / units);
    p.pre.chunk = (int)std::max<int64_t>(4 * tile, ((max_prefix + want - 1) / want + tile - 1) / tile * tile);
    p.pre.splits = (int)std::max<int64_t>(1, (max_prefix + p.pre.chunk - 1) / p.pre.chunk);
    p.pre.grid = units * p.pre.splits;
  }
  p.kind = p.own.wide ? kManyMany : p.pre.wide ? kManyFew : kFewFew;
  const auto parts = [&](const Plan& q, int each, int64_t n, int64_t most) {
    if (q.wide) return (size_t)q.splits * tokens * q_heads;
    return (size_t)(each > 0 ? each * n : q.shares ? q.shares + n : n) * c->kv_heads * (most * group);
  };
  p.own_parts = parts(p.own, p.own_each, batch, max_q), p.pre_parts = parts(p.pre, p.pre_each, prefixes, p.pre_q);
  p.bytes = (p.own_parts + p.pre_parts) * (c->head_dim + 2) * sizeof(float) + (size_t)(batch + prefixes) * sizeof(int2);
  p.flag = prefixes > 63 ? sizeof(int2) : 0;
  p.bytes += p.flag;
  const int64_t each = (p.own.wide ? p.own.splits : std::max(1, p.own_each)) +
                       (p.pre.wide ? p.pre.splits : p.pre_each > 0 ? p.pre_each : 1 + p.pre.shares / prefixes);
  // a wave a row where they are many and of few parts, otherwise one for 32 channels of it: 4096 rows of 9 parts 13 us against 21, 2560 of 17 7 against 12;
  // 128 of 8 6 against 4.5, 1024 of 33 10 against 7
  p.few = each <= 20 && batch * max_q * q_heads >= 2048;
  p.joins = (int64_t)c->kv_heads * batch * rows * (p.few ? 1 : c->head_dim / kJoinCh);
  return p;
}

bool launchable(const SharedPlan& p) { return p.own.grid + p.pre.grid < (1 << 24) && p.joins < (1 << 26); }

sph_status check_shared(const sph_kv_cache* c, int64_t prefixes, int64_t max_group, int64_t max_prefix, int64_t batch, int64_t tokens,
                        int32_t q_heads, int64_t max_q, int64_t max_len) {
  if (const sph_status st = check_sizes(c, batch, tokens, q_heads, max_q, max_len, 0)) return st;
  if (prefixes < 1 || prefixes > 65536 || max_group < 1 || max_group > 65536 || max_prefix < 0 || max_prefix > (1 << 30) ||
      std::min(tokens, max_group * max_q) > (1 << 24))
    return SPH_ERR_SHAPE;
  return SPH_OK;
}

bool launch_ok(const void* fn, int64_t blocks, hipStream_t s, SharedArgs& a) {
  void* kargs[] = {(void*)&a};
  return hipLaunchKernel(fn, dim3((unsigned)blocks), dim3(kThreads), kargs, 0, s) == hipSuccess && hipGetLastError() == hipSuccess;
}

}  // namespace

extern "C" {

sph_status sph_attention_shared_workspace_bytes(const sph_kv_cache* cache, int64_t prefixes, int64_t max_group, int64_t max_prefix,
                                                int64_t batch, int64_t tokens, int32_t q_heads, int64_t max_q, int64_t max_len,
                                                size_t* bytes) {
  if (!bytes) return SPH_ERR_NULL;
  if (const sph_status st = check_shared(cache, prefixes, max_group, max_prefix, batch, tokens, q_heads, max_q, max_len)) return st;
  *bytes = 0;
  if (!batch || !tokens) return SPH_OK;
  const SharedPlan p = shared_plan(cache, prefixes, max_group, max_prefix, batch, tokens, q_heads, max_q, max_len);
  if (!launchable(p)) return SPH_ERR_SHAPE;
  *bytes = p.bytes;
  return SPH_OK;
}

sph_status sph_attention_shared(const sph_kv_cache* cache, int64_t prefixes, const int32_t* d_first, int64_t max_group,
                                const int32_t* d_prefix_pages, int64_t prefix_stride, const int32_t* d_prefix_lens, int64_t max_prefix,
                                int64_t batch, int64_t tokens, int32_t q_heads, const void* d_q, int64_t q_token_stride,
                                int64_t q_head_stride, const int32_t* d_q_start, int64_t max_q, const int32_t* d_pages,
                                int64_t pages_stride, const int32_t* d_seq_lens, int64_t max_len, float scale, void* d_o,
                                int64_t o_token_stride, int64_t o_head_stride, float* d_lse, void* d_ws, size_t ws_bytes, void* stream) {
  if (const sph_status st = check_shared(cache, prefixes, max_group, max_prefix, batch, tokens, q_heads, max_q, max_len)) return st;
  if (!std::isfinite(scale)) return SPH_ERR_BAD_VALUE;
  if ((!d_q_start && (max_q != 1 || tokens != batch)) || (!d_first && (prefixes != 1 || max_group < batch))) return SPH_ERR_SHAPE;
  const int64_t ps = cache->page_size;
  if (pages_stride < (max_len + ps - 1) / ps || pages_stride > INT32_MAX || prefix_stride < (max_prefix + ps - 1) / ps || prefix_stride > INT32_MAX)
    return SPH_ERR_SHAPE;
  if (!batch || !tokens) return SPH_OK;
  if (!d_q || !d_o || !d_seq_lens || !d_prefix_lens || (!d_pages && max_len > 0) || (!d_prefix_pages && max_prefix > 0)) return SPH_ERR_NULL;
  const int64_t lim = int64_t(1) << 40;
  for (int64_t s : {q_token_stride, q_head_stride, o_token_stride, o_head_stride})
    if (s < 0 || s >= lim || s % 8) return SPH_ERR_SHAPE;
  if ((uintptr_t)d_q % 16 || (uintptr_t)d_o % 16 || (uintptr_t)d_ws % 256) return SPH_ERR_SHAPE;
  for (const void* x : {(const void*)d_first, (const void*)d_prefix_pages, (const void*)d_prefix_lens, (const void*)d_q_start, (const void*)d_pages,
                        (const void*)d_seq_lens, (const void*)d_lse})
    if ((uintptr_t)x % 4) return SPH_ERR_SHAPE;
  if ((tokens > 1 && o_token_stride == 0) || (q_heads > 1 && o_head_stride == 0)) return SPH_ERR_SHAPE;  // rows written twice
  const SharedPlan p = shared_plan(cache, prefixes, max_group, max_prefix, batch, tokens, q_heads, max_q, max_len);
  if (!launchable(p)) return SPH_ERR_SHAPE;
  if (!d_ws) return SPH_ERR_NULL;
  if (ws_bytes < p.bytes) return SPH_ERR_BUFFER_TOO_SMALL;
  const int bits = cache->bits, dim = cache->head_dim;
  SharedArgs both{};
  AttnArgs& a = both.own;
  a.c = sph_cache_view(cache);
  a.q = (const char*)d_q, a.o = (char*)d_o;
  a.qt = 2 * q_token_stride, a.qh = 2 * q_head_stride, a.ot = 2 * o_token_stride, a.oh = 2 * o_head_stride;
  a.q_start = d_q_start, a.lse = d_lse, a.tokens = tokens, a.q_heads = q_heads, a.group = q_heads / cache->kv_heads;
  a.scale = scale * kLog2e;
  a.stream = cache->n_pages * cache->page_size * cache->kv_heads * (int64_t)dim * bits / 4 > kLastCache;
  a.part = (float*)d_ws;
  a.ml = (float2*)(a.part + (p.own_parts + p.pre_parts) * dim);
  a.where = (int2*)(a.ml + p.own_parts + p.pre_parts);
  (AttnArgs&)both.pre = a;
  const auto planned = [](AttnArgs& x, const Plan& q) { x.tiles = (int)q.tiles, x.splits = q.splits, x.chunk = q.chunk, x.shares = q.shares; };
  planned(a, p.own);
  both.own.each = p.own_each;
  a.pages = d_pages, a.pages_stride = pages_stride, a.lens = d_seq_lens;
  a.batch = (int)batch, a.max_q = (int)max_q, a.max_len = (int)max_len;
  PrefixArgs& b = both.pre;
  planned(b, p.pre);
  b.each = p.pre_each;
  b.pages = d_prefix_pages, b.pages_stride = prefix_stride, b.lens = d_prefix_lens;
  b.batch = (int)prefixes, b.max_q = (int)p.pre_q, b.max_len = (int)max_prefix;
  b.first = d_first, b.seqs = (int)batch;
  b.part = a.part + p.own_parts * dim, b.ml = a.ml + p.own_parts, b.where = a.where + batch;
  both.descends = (int*)(a.where + batch + prefixes);
  both.pre_blocks = (uint32_t)p.pre.grid, both.blocks = (uint32_t)(p.pre.grid + p.own.grid), both.check = d_first && p.flag ? 1 : 0;
  both.pre_part = (int64_t)p.own_parts;
  both.pre_many = p.pre.wide, both.own_many = p.own.wide;
  const bool uni = cache->page_size >= 16;
  const int nb = p.kind == kFewFew ? p.pre.nb : p.own.nb;
  const void* fn = bits == 16  ? sph_attn_shared_kernel16(dim, p.kind, nb, uni)
                   : bits == 8 ? sph_attn_shared_kernel8(dim, p.kind, nb, uni)
                               : sph_attn_shared_kernel4(dim, p.kind, nb, uni);
  if (!launch_ok(fn, both.check + p.pre.grid + p.own.grid, (hipStream_t)stream, both)) return SPH_ERR_HIP;
  if (!launch_ok(p.few ? (const void*)k_attn_shared_join<true> : (const void*)k_attn_shared_join<false>, (p.joins + kWaves - 1) / kWaves,
                 (hipStream_t)stream, both))
    return SPH_ERR_HIP;
  return SPH_OK;
}

}  // extern "C"
