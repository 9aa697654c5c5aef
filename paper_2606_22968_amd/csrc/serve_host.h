// How the calls over paged batches and windows check their arguments and cut their
// work: shared by the host sides of mocap_serve.h and mocap_cache.h.
#pragma once

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <memory>
#include <new>

#include "host_common.h"
#include "serve.h"

namespace mocap {
namespace {

// A grid dimension holds fewer than 2^32 threads; no workgroup has more than 512.
constexpr int64_t kMaxGroups = ((int64_t)1 << 23) - 1;

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Integer and fp32 arrays are read and written value by value.
inline bool aligned4(const void* ptr) { return (reinterpret_cast<uintptr_t>(ptr) & 3u) == 0; }

// Whether [a, a + a_values) and [b, b + b_values) of 4-byte values share memory.
using wide = unsigned __int128;
inline bool overlap(const void* a, wide a_values, const void* b, wide b_values) {
  const wide x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + 4 * b_values && y < x + 4 * a_values;
}

// Values of rows `rows` of an array with this stride, the last of `used` values.
inline wide extent(int64_t rows, int64_t stride, int64_t used) { return (wide)(rows - 1) * (wide)stride + (wide)used; }

// The attention kernels step through a block's values of one KV head with 32-bit
// byte offsets.
inline bool block_too_large(const mocap_kv_store* kv) {
  return (int64_t)kv->head_dim * kv->block_size > ((int64_t)1 << 30) - 1;
}

inline bool valid_scale(float scale) { return scale > 0.f && std::isfinite(scale); }

inline mocap_status check_heads(int32_t h_q, int32_t h_kv, int32_t head_dim) {
  if (h_q <= 0 || h_kv <= 0 || h_q % h_kv != 0) return MOCAP_ERR_INVALID_ARG;
  return supported_head_dim(head_dim) ? MOCAP_OK : MOCAP_ERR_UNSUPPORTED;
}

// ---- Batches of sequences ----

// How a batch is cut (see SeqBatch).  More parts even out sequences of different
// lengths and keep more loads in flight, fewer save their fixed work and the join.
//   * At most about 5 workgroups per compute unit, for groups of more than 16 heads,
//     which have one wavefront per SIMD, 3 (four sequences of up to 131072 tokens,
//     64/8/128 heads: 294 us at 5, 302 at 8, 328 at 4; 60 of 9000, 32/1/128: 74 us at
//     3, 87 at 5); 16 for key weights, whose parts need no join (16 sequences of up to
//     32768 tokens: 135 us at 8, 130 at 16).
//   * Parts of at least 8 tiles; of 16 where no sequence has more or they fill the
//     device uncut (64 of 1024 tokens: 57 us cut, 49 uncut); down to 4 where parts of
//     8 leave compute units without one (one of 2048 tokens: 17.0 and 13.7 us).
constexpr int kDecodeGroupsPerCu = 5, kDecodeWideGroupsPerCu = 3, kDecodeWeightGroupsPerCu = 16;
constexpr int kDecodeTiles = 8, kDecodeLeastTiles = 4, kDecodeUncutTiles = 16;
constexpr int kDecodeHeads = 32;  // query heads of a workgroup, at most

// Fills in how a batch's tiles are cut: per_item workgroups work on an item; join:
// parts are joined by a second launch.
inline mocap_status plan_batch(int32_t batch, int64_t max_len, int64_t window, int64_t sinks, int64_t per_item,
                        int groups_per_cu, bool join, SeqBatch* s, bool* may_split) {
  int cus = 0;
  const mocap_status st = device_cu_count(&cus);
  if (st != MOCAP_OK) return st;
  if (window >= max_len) window = 0;
  int64_t most = ceil_div(max_len, kTileKeys);
  if (window > 0) most = std::min(most, ceil_div(window, kTileKeys) + 1 + ceil_div(std::min(sinks, max_len), kTileKeys));
  s->batch = batch;
  s->max_len = (int32_t)max_len;
  s->window = (int32_t)window;
  s->sinks = (int32_t)(window > 0 ? std::min(sinks, max_len) : 0);
  s->target = (int32_t)ceil_div((int64_t)cus * groups_per_cu, per_item);
  s->fill = (int32_t)ceil_div(cus, per_item);
  const bool uncut = join && (most <= kDecodeUncutTiles || (int64_t)batch * per_item >= 2 * cus);
  s->min_tiles = uncut ? kDecodeUncutTiles : kDecodeTiles;
  s->least_tiles = uncut ? kDecodeUncutTiles : kDecodeLeastTiles;
  const int64_t items =
      std::min<int64_t>((int64_t)s->target + batch, batch * std::max<int64_t>(1, ceil_div(most, s->least_tiles)));
  if (items * per_item > kMaxGroups - 8 * per_item) return MOCAP_ERR_UNSUPPORTED;
  s->items = (int32_t)items;
  *may_split = most > s->least_tiles;
  return MOCAP_OK;
}

// Checks of a batch's tables and lengths.
inline mocap_status check_batch(const mocap_kv_store* kv, const int32_t* block_tables, int32_t table_stride,
                         const int32_t* seq_lens, int32_t batch, int64_t max_len) {
  const mocap_status st = check_store(kv);
  if (st != MOCAP_OK) return st;
  if (batch < 0 || table_stride < 0 || max_len < 0 || max_len > kMaxPositions) return MOCAP_ERR_INVALID_ARG;
  if (max_len > (int64_t)table_stride * kv->block_size) return MOCAP_ERR_INVALID_ARG;
  if (batch == 0) return MOCAP_OK;
  if (!kv->k_pool || !kv->v_pool || !block_tables || !seq_lens) return MOCAP_ERR_INVALID_ARG;
  if (!aligned16(kv->k_pool) || !aligned16(kv->v_pool) || !aligned4(block_tables) || !aligned4(seq_lens))
    return MOCAP_ERR_INVALID_ARG;
  return MOCAP_OK;
}

inline void set_tables(const mocap_kv_store* kv, const int32_t* block_tables, int32_t table_stride, const int32_t* seq_lens,
                SeqBatch* s) {
  s->tables = block_tables;
  s->seq_lens = seq_lens;
  s->table_stride = table_stride;
  s->block_size = kv->block_size;
  block_divider((uint32_t)kv->block_size, &s->block_magic, &s->block_shift);
}

#ifdef MOCAP_DEBUG_TABLES
// Every entry that the visible positions of a sequence use names a block; a sequence
// longer than max_len ends there, or with skip_longer uses none.  Sequences may share
// blocks.
inline mocap_status debug_check_batch(const mocap_kv_store* kv, const int32_t* block_tables, int32_t table_stride,
                               const int32_t* seq_lens, int32_t batch, int64_t max_len, int64_t window, int64_t sinks,
                               bool skip_longer = false) {
  const int64_t entries = (int64_t)batch * table_stride;
  std::unique_ptr<int32_t[]> host(new (std::nothrow) int32_t[entries + batch]);
  if (!host) return MOCAP_ERR_UNSUPPORTED;
  if (hipMemcpy(host.get(), block_tables, entries * sizeof(int32_t), hipMemcpyDeviceToHost) != hipSuccess ||
      hipMemcpy(host.get() + entries, seq_lens, batch * sizeof(int32_t), hipMemcpyDeviceToHost) != hipSuccess)
    return MOCAP_ERR_HIP;
  for (int32_t b = 0; b < batch; ++b) {
    if (skip_longer && host[entries + b] > max_len) continue;
    const int64_t n = std::min<int64_t>(host[entries + b], max_len);
    const int64_t low = window > 0 ? std::max<int64_t>(0, n - window) : 0;
    for (int64_t lb = 0; lb * kv->block_size < n; ++lb) {
      if ((lb + 1) * kv->block_size <= low && lb * kv->block_size >= sinks) continue;
      const int32_t block = host[b * (int64_t)table_stride + lb];
      if (block < 0 || block >= kv->num_blocks) return MOCAP_ERR_INVALID_ARG;
    }
  }
  return MOCAP_OK;
}
#define MOCAP_DEBUG_CHECK_BATCH(...)                             \
  do {                                                           \
    const mocap_status debug_st_ = debug_check_batch(__VA_ARGS__); \
    if (debug_st_ != MOCAP_OK) return debug_st_;                 \
  } while (0)
#else
#define MOCAP_DEBUG_CHECK_BATCH(...) \
  do {                               \
  } while (0)
#endif

inline mocap_status plan_decode(int32_t batch, int64_t max_len, int32_t h_q, int32_t h_kv, int64_t window, int64_t sinks,
                         DecodeAttnLaunch* p) {
  p->h_q = h_q;
  p->h_kv = h_kv;
  p->group = h_q / h_kv;
  p->row_blocks = (int32_t)ceil_div(p->group, p->group <= 16 ? 16 : kDecodeHeads);
  if ((int64_t)batch * h_q > kMaxGroups) return MOCAP_ERR_UNSUPPORTED;
  return plan_batch(batch, max_len, window, sinks, (int64_t)h_kv * p->row_blocks,
                    p->group <= 16 ? kDecodeGroupsPerCu : kDecodeWideGroupsPerCu, true, &p->seqs, &p->may_split);
}

inline size_t decode_workspace(const DecodeAttnLaunch& p, int32_t head_dim) {
  if (!p.may_split) return 0;
  const size_t rows = (size_t)p.seqs.items * p.h_q;
  return round_up(rows * head_dim * sizeof(float), 256) + round_up(rows * sizeof(float), 256);
}

// ---- A chunk in a window ----

// Time model for the number of ranges: a workgroup of 256 rows costs a tile time
// per 64-key tile, two wavefronts on each SIMD, plus fixed work, one workgroup
// per compute unit at a time; a split adds the merge's launch and traffic.  It ranks
// counts and gives no times: at head_dim 128 a tile takes 1.7 us where few compute
// units are busy and 2 where all are, and 10 us are fixed.  The counts that it chose
// for seven shapes of 1 to 1000 tokens took at most 7% more than the best of 1 to 64
// (64 tokens of 32/8/128 in a window of 4096: 14 ranges 24.0 us, 24 ranges 22.4, one 115).
constexpr double kWindowTileUs128 = 1.4, kWindowTileUs64 = 0.9;
constexpr double kWindowGroupUs = 4.0, kWindowMergeUs = 5.0, kWindowMergeBytesPerUs = 4.0e6;
constexpr int64_t kWindowMaxRanges = 64;

inline mocap_status plan_window(int64_t prefix_len, int32_t chunk_len, int32_t h_q, int32_t h_kv, int32_t head_dim,
                         int64_t window, int64_t sinks, int32_t num_splits, WindowLaunch* p) {
  const int64_t group = h_q / h_kv, rows = chunk_len * group;
  if (rows > ((int64_t)1 << 31) - 2 * kWindowRows) return MOCAP_ERR_UNSUPPORTED;
  p->prefix_len = (int32_t)prefix_len;
  p->chunk_len = chunk_len;
  p->h_q = h_q;
  p->h_kv = h_kv;
  p->group = (int32_t)group;
  block_divider((uint32_t)group, &p->group_magic, &p->group_shift);
  p->row_blocks = (int32_t)ceil_div(rows, kWindowRows);
  p->window = (int32_t)std::min<int64_t>(window, kMaxPositions);
  p->sinks = (int32_t)std::min<int64_t>(sinks, kMaxPositions);
  const int64_t wgs = (int64_t)p->row_blocks * h_kv;
  // Tiles of the workgroup with the most.
  const int64_t span = std::min<int64_t>(chunk_len, ceil_div(kWindowRows, group) + 1) + p->window;
  const int64_t tiles = std::min(ceil_div(prefix_len + chunk_len, kTileKeys),
                                 ceil_div(span, kTileKeys) + 1 + ceil_div(p->sinks, kTileKeys));
  int64_t best = 1;
  if (num_splits > 1) {
    best = std::min<int64_t>(num_splits, tiles);
  } else if (num_splits == 0) {
    int cus = 0;
    const mocap_status st = device_cu_count(&cus);
    if (st != MOCAP_OK) return st;
    const double tile_us = head_dim == 128 ? kWindowTileUs128 : kWindowTileUs64;
    double best_us = INFINITY;
    for (int64_t n = 1; n <= std::min(kWindowMaxRanges, tiles); ++n) {
      double us = (double)ceil_div(wgs * n, cus) * (ceil_div(tiles, n) * tile_us + kWindowGroupUs);
      if (n > 1) us += kWindowMergeUs + 2.0 * n * chunk_len * h_q * (head_dim + 1) * 4.0 / kWindowMergeBytesPerUs;
      if (us < best_us * 0.98) {
        best_us = us;
        best = n;
      }
    }
  }
  if (wgs * best > kMaxGroups) return MOCAP_ERR_UNSUPPORTED;
  p->n_ranges = (int32_t)best;
  p->total_wgs = (int32_t)(wgs * best);
  return MOCAP_OK;
}

inline size_t window_workspace(const WindowLaunch& p, int32_t head_dim) {
  if (p.n_ranges <= 1) return 0;
  const size_t rows = (size_t)p.n_ranges * p.h_q * p.chunk_len;
  return round_up(rows * head_dim * sizeof(float), 256) + round_up(rows * sizeof(float), 256);
}

inline mocap_status check_chunk(int64_t prefix_len, int32_t chunk_len) {
  if (prefix_len < 0 || chunk_len < 0 || prefix_len + (int64_t)chunk_len > kMaxPositions) return MOCAP_ERR_INVALID_ARG;
  return MOCAP_OK;
}

// Checks shared by the calls on one chunk of one sequence.
inline mocap_status check_chunk_args(const mocap_kv_store* kv, const int32_t* block_table, int32_t n_table, const void* q,
                              int64_t prefix_len, int32_t chunk_len, int32_t h_q, int32_t h_kv, int32_t head_dim,
                              float scale) {
  mocap_status st = check_store(kv);
  if (st != MOCAP_OK) return st;
  if (h_q <= 0 || h_kv <= 0 || h_q % h_kv != 0 || h_kv != kv->h_kv || head_dim != kv->head_dim || !valid_scale(scale))
    return MOCAP_ERR_INVALID_ARG;
  st = check_positions(kv, n_table, prefix_len, chunk_len);
  if (st != MOCAP_OK) return st;
  if (chunk_len == 0) return MOCAP_OK;
  if (!kv->k_pool || !kv->v_pool || !block_table || !q) return MOCAP_ERR_INVALID_ARG;
  if (!aligned16(kv->k_pool) || !aligned16(kv->v_pool) || !aligned4(block_table) || !aligned16(q))
    return MOCAP_ERR_INVALID_ARG;
  return MOCAP_OK;
}

}  // namespace
}  // namespace mocap
