// How the attention is cut into workgroups: host side, for sph_attention and sph_attention_shared.
#pragma once
#include <algorithm>

#include "sph_attn_few.h"

namespace {

constexpr int kMaxSplits = 512, kJoinCh = 32, kFewParts = 8;

struct Plan {
  int wide, nb, splits, chunk, shares, fold, window;
  int64_t tiles;                           // (up to 2^33 before the launch is refused)
  int64_t grid, joins;                     // workgroups; waves of the join
  bool few;                                // k_attn_join's form
  size_t parts;                            // rows of partial sums
  size_t bytes;
};

// k_attn: a workgroup a sequence and kv head where sequences are short (a few tiles a wave; joining would cost as much) or so many
// that they fill the chip; otherwise as many workgroups as are resident at once, with equal shares of all keys.
// k_attn_wide: stretches of at least four tiles where the rows alone would leave the chip idle.
constexpr int kCus = 256;

// Pools that the last cache before memory cannot hold are read past it (values: see load_values). One sequence of 131072 tokens in fp16 86 us
// instead of 95, 64 of up to 8192 at 8 bits 78 instead of 82; a pool of 41 MB that stays in that cache from call to call 26 instead of 24.
constexpr int64_t kLastCache = 256 << 20;

// Workgroups of k_attn on a CU: as many as keep about 64 KiB of pages on their way to it, a tile a wave. More lengthen the queue that every
// dependent load waits in, or wait for registers: 64 ragged sequences of up to 8192 tokens at 8 bits take 98, 78 and 95 us with one, two and three
// workgroups a CU; 16 of 32768 tokens at 4 bits 195, 135 and 123; one of 131072 tokens in fp16 86, 88 and 90, and its join 4.7, 5.9 and 6.9.
int workgroups_per_cu(const sph_kv_cache* c) {
  const int tile = kTile * 2 * c->head_dim * c->bits / 8;
  return std::max(1, std::min(3, (64 << 10) / (kWaves * tile)));
}

Plan plan_of(const sph_kv_cache* c, int64_t batch, int q_heads, int64_t max_q, int64_t max_len, int64_t window) {
  Plan p{};
  // one that hides nothing is none (and positions minus a window stay inside 32 bits)
  p.window = window > max_len ? 0 : (int)window;
  window = p.window;
  const int group = q_heads / c->kv_heads;
  const int64_t rows = max_q * group;
  // two blocks of rows of wider heads do not fit the registers
  p.nb = rows <= 16 || c->head_dim > 128 ? 1 : 2;
  p.wide = rows > 16 * p.nb;
  p.splits = 1;
  int64_t slots = 0;
  if (!p.wide) {
    p.tiles = 1;
    const int64_t span = window > 0 ? std::min<int64_t>(max_len, window + max_q + kTile) : max_len;
    // Short: up to 6 tiles of 128 channels a wave, or 16 where sequences and heads give half the CUs a workgroup, since the counting
    // of shares and their join cost about 8 us and such calls gain little from a few more workgroups. 8 kv heads, fp16, direct against
    // shares and join: one sequence of 512 keys 9.4 and 12.2 us, 768 11.9 and 11.9, 1024 14.5 and 12.3; 16 ragged ones of up to 1024
    // 16.0 and 17.6, 2048 24.5 and 23.5; 64 of up to 2048 52.8 and 54.4. 64 channels: one of 1536 12.2 and 11.8; 256: one of 384 14.4 and 15.4.
    const int64_t steps = (2 * batch * c->kv_heads >= kCus ? 16 : 6) * 128;
    const int64_t rounds = steps / c->head_dim;
    if (batch <= kEvenBatch && span > kTile * kWaves * rounds && batch * (span / kTile + 2) < (1 << 30)) {
      p.shares = (int)std::min<int64_t>(kMaxSplits - 1, std::max<int64_t>(1, kCus * workgroups_per_cu(c) / c->kv_heads));
      p.shares = (int)std::min<int64_t>(p.shares, batch * ((span + kTile * kWaves - 1) / (kTile * kWaves) + 1));
      slots = p.shares + batch;
    }
  } else {
    p.tiles = (rows + kWideRows - 1) / kWideRows;
    const int64_t tile = sph_attn_wide_tile(c->head_dim), step = 4 * tile;
    const int64_t span = window > 0 ? std::min<int64_t>(max_len, window + kWideRows / group + 1 + tile) : max_len;
    // None where the rows alone give half the CUs a workgroup: two parts save less than their join costs (900 rows of one prompt 35 us,
    // in two parts 33 + 17). Otherwise two a CU, and four where sequences are several, since ragged ones leave many with little
    // to do (8 of up to 8000 tokens, 40 of each new: 67 + 6 us with two, 40 + 7 with four).
    const int64_t units = c->kv_heads * batch * p.tiles, per_cu = batch > 1 ? 4 : 2;
    const int64_t want = 2 * units > kCus ? 1 : std::min<int64_t>(kMaxSplits, per_cu * kCus / units);
    p.chunk = (int)std::max<int64_t>(step, ((span + want - 1) / want + step - 1) / step * step);
    p.splits = (int)std::max<int64_t>(1, (span + p.chunk - 1) / p.chunk);
    if (p.splits > 1) slots = p.splits * batch;
    // All workgroups resident at once, two on some CUs (the i-th and the (i + 256)-th; of 64 channels a CU takes more, of 192 one): long
    // rows share theirs with short ones. 8 kv heads of 128 channels, so and with the longest first, fp16: prompts of 2048 tokens 62.0 and 65.0 us,
    // 1536 46.3 and 47.9, four of 512 26.8 and 30.1, 1300 behind 6700 others 236 and 243; four of 500 at 8 bits 30.7 and 35.6; 2048 of 96
    // channels 51.1 and 52.6, of 64 43.2 and 43.3.
    if (c->head_dim > 64 && c->head_dim <= 128 && p.splits == 1 && kCus % c->kv_heads == 0 && units > kCus && units <= 2 * kCus)
      p.fold = kCus / c->kv_heads;
  }
  p.parts = (size_t)slots * c->kv_heads * rows;
  if (slots) p.bytes = p.parts * (c->head_dim + 2) * sizeof(float) + (size_t)batch * sizeof(int2);
  const int64_t heads = c->kv_heads, all = heads * batch * rows;
  p.grid = p.wide ? heads * batch * p.tiles * p.splits : heads * (p.shares ? p.shares : batch);
  // k_attn_wide's parts are few, and k_attn's where sequences share a workgroup rather than the other way round
  p.few = p.wide ? p.splits <= kFewParts : 2 * batch > p.shares && p.shares <= kFewParts * batch;
  p.joins = p.few ? all : all * (c->head_dim / kJoinCh);
  return p;
}

sph_status check_sizes(const sph_kv_cache* c, int64_t batch, int64_t tokens, int32_t q_heads, int64_t max_q, int64_t max_len,
                       int64_t window) {
  if (!c) return SPH_ERR_NULL;
  if (const int st = sph_cache_check(c)) return (sph_status)st;
  if (batch < 0 || batch > 65536 || tokens < 0 || tokens > (1 << 26) || q_heads < 1 || q_heads > 65535 || q_heads % c->kv_heads ||
      max_q < 1 || max_q > (1 << 24) || max_len < 0 || max_len > (1 << 30) || window < 0)
    return SPH_ERR_SHAPE;
  return SPH_OK;
}

}  // namespace
