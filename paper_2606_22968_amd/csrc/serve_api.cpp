// Host side of the calls that follow the prefill (mocap_serve.h): argument
// validation, how the work is cut, and kernel dispatch.  Every check runs before
// anything is enqueued.
#include "mocap_serve.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <memory>
#include <new>

#include "host_common.h"
#include "serve.h"

namespace {

using mocap::aligned16;
using mocap::block_divider;
using mocap::check_positions;
using mocap::check_store;
using mocap::device_cu_count;
using mocap::kMaxPositions;
using mocap::kTileKeys;
using mocap::round_up;
using mocap::supported_head_dim;

// A grid dimension holds fewer than 2^32 threads; no workgroup has more than 512.
constexpr int64_t kMaxGroups = ((int64_t)1 << 23) - 1;

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Integer and fp32 arrays are read and written value by value.
bool aligned4(const void* ptr) { return (reinterpret_cast<uintptr_t>(ptr) & 3u) == 0; }

// Whether [a, a + a_values) and [b, b + b_values) of 4-byte values share memory.
using wide = unsigned __int128;
bool overlap(const void* a, wide a_values, const void* b, wide b_values) {
  const wide x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + 4 * b_values && y < x + 4 * a_values;
}

// Values of rows `rows` of an array with this stride, the last of `used` values.
wide extent(int64_t rows, int64_t stride, int64_t used) { return (wide)(rows - 1) * (wide)stride + (wide)used; }

// The attention kernels step through a block's values of one KV head with 32-bit
// byte offsets.
bool block_too_large(const mocap_kv_store* kv) {
  return (int64_t)kv->head_dim * kv->block_size > ((int64_t)1 << 30) - 1;
}

bool valid_scale(float scale) { return scale > 0.f && std::isfinite(scale); }

mocap_status check_heads(int32_t h_q, int32_t h_kv, int32_t head_dim) {
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
mocap_status plan_batch(int32_t batch, int64_t max_len, int64_t window, int64_t sinks, int64_t per_item,
                        int groups_per_cu, bool join, mocap::SeqBatch* s, bool* may_split) {
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
mocap_status check_batch(const mocap_kv_store* kv, const int32_t* block_tables, int32_t table_stride,
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

void set_tables(const mocap_kv_store* kv, const int32_t* block_tables, int32_t table_stride, const int32_t* seq_lens,
                mocap::SeqBatch* s) {
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
mocap_status debug_check_batch(const mocap_kv_store* kv, const int32_t* block_tables, int32_t table_stride,
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

mocap_status plan_decode(int32_t batch, int64_t max_len, int32_t h_q, int32_t h_kv, int64_t window, int64_t sinks,
                         mocap::DecodeAttnLaunch* p) {
  p->h_q = h_q;
  p->h_kv = h_kv;
  p->group = h_q / h_kv;
  p->row_blocks = (int32_t)ceil_div(p->group, p->group <= 16 ? 16 : kDecodeHeads);
  if ((int64_t)batch * h_q > kMaxGroups) return MOCAP_ERR_UNSUPPORTED;
  return plan_batch(batch, max_len, window, sinks, (int64_t)h_kv * p->row_blocks,
                    p->group <= 16 ? kDecodeGroupsPerCu : kDecodeWideGroupsPerCu, true, &p->seqs, &p->may_split);
}

size_t decode_workspace(const mocap::DecodeAttnLaunch& p, int32_t head_dim) {
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

mocap_status plan_window(int64_t prefix_len, int32_t chunk_len, int32_t h_q, int32_t h_kv, int32_t head_dim,
                         int64_t window, int64_t sinks, int32_t num_splits, mocap::WindowLaunch* p) {
  const int64_t group = h_q / h_kv, rows = chunk_len * group;
  if (rows > ((int64_t)1 << 31) - 2 * mocap::kWindowRows) return MOCAP_ERR_UNSUPPORTED;
  p->prefix_len = (int32_t)prefix_len;
  p->chunk_len = chunk_len;
  p->h_q = h_q;
  p->h_kv = h_kv;
  p->group = (int32_t)group;
  block_divider((uint32_t)group, &p->group_magic, &p->group_shift);
  p->row_blocks = (int32_t)ceil_div(rows, mocap::kWindowRows);
  p->window = (int32_t)std::min<int64_t>(window, kMaxPositions);
  p->sinks = (int32_t)std::min<int64_t>(sinks, kMaxPositions);
  const int64_t wgs = (int64_t)p->row_blocks * h_kv;
  // Tiles of the workgroup with the most.
  const int64_t span = std::min<int64_t>(chunk_len, ceil_div(mocap::kWindowRows, group) + 1) + p->window;
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

size_t window_workspace(const mocap::WindowLaunch& p, int32_t head_dim) {
  if (p.n_ranges <= 1) return 0;
  const size_t rows = (size_t)p.n_ranges * p.h_q * p.chunk_len;
  return round_up(rows * head_dim * sizeof(float), 256) + round_up(rows * sizeof(float), 256);
}

// ---- Key weights ----

// A row tile (32 rows by 512 keys), fixed work of a workgroup, and the join of row
// parts; the fewest tiles of a part, and the most parts (1000 tokens of 64/1/64 heads
// without a prefix: 37 us at 64, 25 at 128, 24 at 256).  The tile times are those of
// whole stages without masked tiles; first chunks, which have many others, take a
// quarter to a half more than the model says (2048 tokens of 32/8/128 heads: 38 us for 25).
constexpr double kWeightTileUs128 = 0.75, kWeightTileUs64 = 0.55, kWeightGroupUs = 4.0, kWeightJoinUs = 4.0;
// Up to this many rows the keys stream past the rows instead: 65501 keys of 8 heads
// of 128 by 4, 64, 128 and 256 rows, 29, 31, 37 and 60 us against 38, 42, 46 and 63;
// 8000 keys, 8.2, -, 10.7 and 17.8 against 8.4, -, 10.3 and 14.9.  Three of its
// workgroups fit a compute unit (four or six of them per unit: 38 and 41 us for 37).
constexpr int64_t kWeightFewRows = 128, kWeightFewGroupsPerCu = 3;
constexpr int64_t kWeightMinTiles = 4, kWeightMaxParts = 256, kWeightMaxRounds = 4;

mocap_status plan_weights(int64_t prefix_len, int32_t chunk_len, int32_t h_q, int32_t h_kv, int32_t head_dim,
                          mocap::KeyWeightsLaunch* p) {
  const int64_t group = h_q / h_kv, rows = chunk_len * group, n = prefix_len + chunk_len;
  if (rows > ((int64_t)1 << 31) - 1024) return MOCAP_ERR_UNSUPPORTED;
  // A stage's rows (128, of 128 / group + 2 tokens at most) are addressed with 32-bit
  // byte offsets.
  if ((128 / group + 2) * h_q * head_dim * 2 > ((int64_t)1 << 31) - 1) return MOCAP_ERR_UNSUPPORTED;
  int cus = 0;
  const mocap_status st = device_cu_count(&cus);
  if (st != MOCAP_OK) return st;
  p->prefix_len = (int32_t)prefix_len;
  p->chunk_len = chunk_len;
  p->h_q = h_q;
  p->h_kv = h_kv;
  p->group = (int32_t)group;
  block_divider((uint32_t)group, &p->group_magic, &p->group_shift);
  p->few = rows <= kWeightFewRows;
  if (p->few) {
    // Every wavefront a tile at least; about three workgroups per compute unit.
    p->key_blocks = (int32_t)std::min(ceil_div(n, 4 * kTileKeys), ceil_div((int64_t)cus * kWeightFewGroupsPerCu, h_kv));
    p->row_parts = 1;
    return (int64_t)p->key_blocks * h_kv > kMaxGroups ? MOCAP_ERR_UNSUPPORTED : MOCAP_OK;
  }
  const int64_t block_keys = mocap::kWeightKeys * mocap::kWeightWaves;
  p->key_blocks = (int32_t)ceil_div(n, block_keys);
  // Parts: one workgroup per compute unit at a time, a round costs its longest
  // one's row tiles plus fixed work.
  const int64_t wgs = (int64_t)p->key_blocks * h_kv, tiles = ceil_div(rows, 32);
  if (wgs > kMaxGroups || h_kv > 65535) return MOCAP_ERR_UNSUPPORTED;
  const double tile_us = head_dim == 128 ? kWeightTileUs128 : kWeightTileUs64;
  // Key blocks that all rows see from their first key on; the others have the later
  // rows only, and fewer parts of this many tiles.
  const int64_t seen = std::min<int64_t>(p->key_blocks, prefix_len / block_keys + 1);
  p->row_parts = 1;
  p->part_tiles = (int32_t)tiles;
  p->head_wgs = p->key_blocks;
  double best_us = ceil_div(wgs, cus) * (tiles * tile_us + kWeightGroupUs);
  for (int64_t parts = 2; parts <= std::min<int64_t>(kWeightMaxParts, ceil_div(tiles, kWeightMinTiles)); ++parts) {
    if (std::max(seen * parts, (int64_t)p->key_blocks) * h_kv > kWeightMaxRounds * cus) break;
    const int64_t most = ceil_div(tiles, parts);
    int64_t head_wgs = seen * ceil_div(tiles, most);
    for (int64_t b = seen; b < p->key_blocks; ++b)
      head_wgs += ceil_div(tiles - (b * block_keys - prefix_len) * group / 32, most);
    if (head_wgs * h_kv > kWeightMaxRounds * cus) break;
    double us = (double)ceil_div(head_wgs * h_kv, cus) * (most * tile_us + kWeightGroupUs);
    us += kWeightJoinUs + 8.0 * parts * h_kv * n / kWindowMergeBytesPerUs;
    if (us < best_us * 0.98) {
      best_us = us;
      p->row_parts = (int32_t)ceil_div(tiles, most);
      p->part_tiles = (int32_t)most;
      p->head_wgs = (int32_t)head_wgs;
    }
  }
  return MOCAP_OK;
}

size_t weights_workspace(const mocap::KeyWeightsLaunch& p) {
  if (p.row_parts <= 1) return 0;
  return (size_t)p.row_parts * p.h_kv * ((size_t)p.prefix_len + p.chunk_len) * sizeof(float);
}

// ---- Eviction ----

// Its kernels step over positions in 32 bits, its grids have four threads a position.
constexpr int64_t kEvictMaxPositions = ((int64_t)1 << 30) - 64;

// The workspace is sized for all n positions as candidates; sinks and recent
// ones only make them fewer.
int32_t evict_chunks(int64_t candidates) {
  if (candidates <= mocap::kEvictOneGroup) return 0;
  return (int32_t)std::min<int64_t>(mocap::kEvictMaxChunks, ceil_div(candidates, 4096));
}

mocap_status check_chunk(int64_t prefix_len, int32_t chunk_len) {
  if (prefix_len < 0 || chunk_len < 0 || prefix_len + (int64_t)chunk_len > kMaxPositions) return MOCAP_ERR_INVALID_ARG;
  return MOCAP_OK;
}

// Checks shared by the calls on one chunk of one sequence.
mocap_status check_chunk_args(const mocap_kv_store* kv, const int32_t* block_table, int32_t n_table, const void* q,
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

extern "C" {

mocap_status mocap_decode_append(const mocap_kv_store* kv, const int32_t* block_tables, int32_t table_stride,
                                 const int32_t* seq_lens, int32_t batch, const void* k, const void* v, void* stream) {
  const mocap_status st = check_batch(kv, block_tables, table_stride, seq_lens, batch, 0);
  if (st != MOCAP_OK || batch == 0) return st;
  if (!k || !v || !aligned16(k) || !aligned16(v)) return MOCAP_ERR_INVALID_ARG;
  if (batch > kMaxGroups || (int64_t)kv->h_kv * (kv->head_dim / 8) > 65535 * 64) return MOCAP_ERR_UNSUPPORTED;
  MOCAP_DEBUG_CHECK_BATCH(kv, block_tables, table_stride, seq_lens, batch, (int64_t)table_stride * kv->block_size, 1, 0,
                          true);
  mocap::DecodeAppendLaunch p;
  p.k = static_cast<const uint16_t*>(k);
  p.v = static_cast<const uint16_t*>(v);
  p.k_pool = static_cast<uint16_t*>(kv->k_pool);
  p.v_pool = static_cast<uint16_t*>(kv->v_pool);
  p.tables = block_tables;
  p.seq_lens = seq_lens;
  p.table_stride = table_stride;
  p.batch = batch;
  p.h_kv = kv->h_kv;
  p.block_size = kv->block_size;
  return mocap::launch_decode_append(p, kv->head_dim, static_cast<hipStream_t>(stream)) == hipSuccess ? MOCAP_OK
                                                                                                      : MOCAP_ERR_HIP;
}

mocap_status mocap_decode_attn_workspace_size(int32_t batch, int64_t max_len, int32_t h_q, int32_t h_kv,
                                              int32_t head_dim, int64_t window, int64_t sinks, size_t* bytes_out) {
  if (bytes_out == nullptr || batch < 0 || max_len < 0 || max_len > kMaxPositions || window < 0 || sinks < 0)
    return MOCAP_ERR_INVALID_ARG;
  mocap_status st = check_heads(h_q, h_kv, head_dim);
  if (st != MOCAP_OK) return st;
  *bytes_out = 0;
  if (batch == 0) return MOCAP_OK;
  mocap::DecodeAttnLaunch p;
  st = plan_decode(batch, max_len, h_q, h_kv, window, sinks, &p);
  if (st == MOCAP_OK) *bytes_out = decode_workspace(p, head_dim);
  return st;
}

mocap_status mocap_decode_attn(const mocap_kv_store* kv, const int32_t* block_tables, int32_t table_stride,
                               const int32_t* seq_lens, int32_t batch, int64_t max_len, const void* q, int32_t h_q,
                               int32_t h_kv, int32_t head_dim, float scale, int64_t window, int64_t sinks, void* o,
                               float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  mocap_status st = check_batch(kv, block_tables, table_stride, seq_lens, batch, max_len);
  if (st != MOCAP_OK) return st;
  if (h_q <= 0 || h_kv <= 0 || h_q % h_kv != 0 || h_kv != kv->h_kv || head_dim != kv->head_dim || !valid_scale(scale) ||
      window < 0 || sinks < 0)
    return MOCAP_ERR_INVALID_ARG;
  if (batch == 0) return MOCAP_OK;
  if (!q || !o || !lse || !aligned16(q) || !aligned16(o) || !aligned4(lse)) return MOCAP_ERR_INVALID_ARG;
  if (block_too_large(kv)) return MOCAP_ERR_UNSUPPORTED;
  mocap::DecodeAttnLaunch p;
  st = plan_decode(batch, max_len, h_q, h_kv, window, sinks, &p);
  if (st != MOCAP_OK) return st;
  if (p.may_split && (!workspace || !aligned16(workspace) || workspace_bytes < decode_workspace(p, head_dim)))
    return MOCAP_ERR_WORKSPACE;
  MOCAP_DEBUG_CHECK_BATCH(kv, block_tables, table_stride, seq_lens, batch, max_len, window, sinks);
  set_tables(kv, block_tables, table_stride, seq_lens, &p.seqs);
  p.q = static_cast<const uint16_t*>(q);
  p.k_pool = static_cast<const uint16_t*>(kv->k_pool);
  p.v_pool = static_cast<const uint16_t*>(kv->v_pool);
  p.o = static_cast<uint16_t*>(o);
  p.lse = lse;
  p.ws_o = nullptr;
  p.ws_lse = nullptr;
  if (p.may_split) {
    p.ws_o = static_cast<float*>(workspace);
    p.ws_lse = reinterpret_cast<float*>(static_cast<char*>(workspace) +
                                        round_up((size_t)p.seqs.items * h_q * head_dim * sizeof(float), 256));
  }
  p.scale_log2 = (float)((double)scale * 1.4426950408889634);
  return mocap::launch_decode_attn(p, head_dim, static_cast<hipStream_t>(stream)) == hipSuccess ? MOCAP_OK
                                                                                                : MOCAP_ERR_HIP;
}

mocap_status mocap_window_attn_workspace_size(int64_t prefix_len, int32_t chunk_len, int32_t h_q, int32_t h_kv,
                                              int32_t head_dim, int64_t window, int64_t sinks, int32_t num_splits,
                                              int32_t* splits_out, size_t* bytes_out) {
  if (bytes_out == nullptr || window < 1 || sinks < 0 || num_splits < 0) return MOCAP_ERR_INVALID_ARG;
  mocap_status st = check_chunk(prefix_len, chunk_len);
  if (st == MOCAP_OK) st = check_heads(h_q, h_kv, head_dim);
  if (st != MOCAP_OK) return st;
  mocap::WindowLaunch p;
  p.n_ranges = 1;
  if (chunk_len > 0) st = plan_window(prefix_len, chunk_len, h_q, h_kv, head_dim, window, sinks, num_splits, &p);
  if (st != MOCAP_OK) return st;
  if (splits_out) *splits_out = p.n_ranges;
  *bytes_out = chunk_len > 0 ? window_workspace(p, head_dim) : 0;
  return MOCAP_OK;
}

mocap_status mocap_window_attn(const mocap_kv_store* kv, const int32_t* block_table, int32_t n_table, const void* q,
                               int64_t prefix_len, int32_t chunk_len, int32_t h_q, int32_t h_kv, int32_t head_dim,
                               float scale, int64_t window, int64_t sinks, void* o, float* lse, void* workspace,
                               size_t workspace_bytes, int32_t num_splits, void* stream) {
  mocap_status st = check_chunk_args(kv, block_table, n_table, q, prefix_len, chunk_len, h_q, h_kv, head_dim, scale);
  if (st != MOCAP_OK) return st;
  if (window < 1 || sinks < 0 || num_splits < 0) return MOCAP_ERR_INVALID_ARG;
  if (chunk_len == 0) return MOCAP_OK;
  if (!o || !lse || !aligned16(o) || !aligned4(lse)) return MOCAP_ERR_INVALID_ARG;
  if (block_too_large(kv)) return MOCAP_ERR_UNSUPPORTED;
  mocap::WindowLaunch p;
  st = plan_window(prefix_len, chunk_len, h_q, h_kv, head_dim, window, sinks, num_splits, &p);
  if (st != MOCAP_OK) return st;
  if (p.n_ranges > 1 && (!workspace || !aligned16(workspace) || workspace_bytes < window_workspace(p, head_dim)))
    return MOCAP_ERR_WORKSPACE;
  MOCAP_DEBUG_CHECK(block_table, 0, std::min<int64_t>(sinks, prefix_len + chunk_len), kv);
  MOCAP_DEBUG_CHECK(block_table, std::max<int64_t>(0, prefix_len - window + 1), prefix_len + chunk_len, kv);
  p.q = static_cast<const uint16_t*>(q);
  p.k_pool = static_cast<const uint16_t*>(kv->k_pool);
  p.v_pool = static_cast<const uint16_t*>(kv->v_pool);
  p.table = block_table;
  p.o = static_cast<uint16_t*>(o);
  p.lse = lse;
  p.block_size = kv->block_size;
  block_divider((uint32_t)kv->block_size, &p.block_magic, &p.block_shift);
  p.scale_log2 = (float)((double)scale * 1.4426950408889634);
  p.ws_o = nullptr;
  p.ws_lse = nullptr;
  if (p.n_ranges > 1) {
    p.ws_o = static_cast<float*>(workspace);
    p.ws_lse = reinterpret_cast<float*>(
        static_cast<char*>(workspace) + round_up((size_t)p.n_ranges * h_q * chunk_len * head_dim * sizeof(float), 256));
  }
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (mocap::launch_window_attn(p, head_dim, s) != hipSuccess) return MOCAP_ERR_HIP;
  if (p.n_ranges > 1) {
    const mocap::MergeLaunch m{p.ws_o, p.ws_lse, p.o, lse, chunk_len, h_q, p.n_ranges};
    if (mocap::launch_lse_merge(m, head_dim, s) != hipSuccess) return MOCAP_ERR_HIP;
  }
  return MOCAP_OK;
}

mocap_status mocap_key_weights_workspace_size(int64_t prefix_len, int32_t chunk_len, int32_t h_q, int32_t h_kv,
                                              int32_t head_dim, size_t* bytes_out) {
  if (bytes_out == nullptr) return MOCAP_ERR_INVALID_ARG;
  mocap_status st = check_chunk(prefix_len, chunk_len);
  if (st == MOCAP_OK) st = check_heads(h_q, h_kv, head_dim);
  if (st != MOCAP_OK) return st;
  *bytes_out = 0;
  if (chunk_len == 0) return MOCAP_OK;
  mocap::KeyWeightsLaunch p;
  st = plan_weights(prefix_len, chunk_len, h_q, h_kv, head_dim, &p);
  if (st == MOCAP_OK) *bytes_out = weights_workspace(p);
  return st;
}

mocap_status mocap_key_weights(const mocap_kv_store* kv, const int32_t* block_table, int32_t n_table, const void* q,
                               int64_t prefix_len, int32_t chunk_len, int32_t h_q, int32_t h_kv, int32_t head_dim,
                               float scale, const float* lse, const float* prev, float* weights, int64_t weight_stride,
                               void* workspace, size_t workspace_bytes, void* stream) {
  mocap_status st = check_chunk_args(kv, block_table, n_table, q, prefix_len, chunk_len, h_q, h_kv, head_dim, scale);
  if (st != MOCAP_OK) return st;
  if (weight_stride < prefix_len + chunk_len) return MOCAP_ERR_INVALID_ARG;
  if (chunk_len == 0) return MOCAP_OK;
  if (!lse || !weights || !aligned4(lse) || !aligned4(weights) || !aligned4(prev)) return MOCAP_ERR_INVALID_ARG;
  const wide values = extent(h_kv, weight_stride, prefix_len + chunk_len);
  if (prev != nullptr && prev != weights && overlap(prev, values, weights, values)) return MOCAP_ERR_INVALID_ARG;
  mocap::KeyWeightsLaunch p;
  st = plan_weights(prefix_len, chunk_len, h_q, h_kv, head_dim, &p);
  if (st != MOCAP_OK) return st;
  if (p.row_parts > 1 && (!workspace || !aligned16(workspace) || workspace_bytes < weights_workspace(p)))
    return MOCAP_ERR_WORKSPACE;
  MOCAP_DEBUG_CHECK(block_table, 0, prefix_len + chunk_len, kv);
  p.q = static_cast<const uint16_t*>(q);
  p.k_pool = static_cast<const uint16_t*>(kv->k_pool);
  p.table = block_table;
  p.lse = lse;
  p.prev = prev;
  p.weights = weights;
  p.ws = static_cast<float*>(workspace);
  p.weight_stride = weight_stride;
  p.block_size = kv->block_size;
  block_divider((uint32_t)kv->block_size, &p.block_magic, &p.block_shift);
  p.scale_log2 = (float)((double)scale * 1.4426950408889634);
  return mocap::launch_key_weights(p, head_dim, static_cast<hipStream_t>(stream)) == hipSuccess ? MOCAP_OK
                                                                                                : MOCAP_ERR_HIP;
}

mocap_status mocap_decode_key_weights(const mocap_kv_store* kv, const int32_t* block_tables, int32_t table_stride,
                                      const int32_t* seq_lens, int32_t batch, int64_t max_len, const void* q,
                                      int32_t h_q, int32_t h_kv, int32_t head_dim, float scale, const float* lse,
                                      const float* prev, float* weights, int64_t weight_stride, void* stream) {
  mocap_status st = check_batch(kv, block_tables, table_stride, seq_lens, batch, max_len);
  if (st != MOCAP_OK) return st;
  if (h_q <= 0 || h_kv <= 0 || h_q % h_kv != 0 || h_kv != kv->h_kv || head_dim != kv->head_dim || !valid_scale(scale) ||
      weight_stride < max_len)
    return MOCAP_ERR_INVALID_ARG;
  if (batch == 0) return MOCAP_OK;
  if (!q || !lse || !weights || !aligned16(q) || !aligned4(lse) || !aligned4(weights) || !aligned4(prev))
    return MOCAP_ERR_INVALID_ARG;
  const wide values = extent((int64_t)batch * h_kv, weight_stride, max_len);
  if (prev != nullptr && prev != weights && overlap(prev, values, weights, values)) return MOCAP_ERR_INVALID_ARG;
  mocap::DecodeKeyWeightsLaunch p;
  bool may_split;
  st = plan_batch(batch, max_len, 0, 0, h_kv, kDecodeWeightGroupsPerCu, false, &p.seqs, &may_split);
  if (st != MOCAP_OK) return st;
  MOCAP_DEBUG_CHECK_BATCH(kv, block_tables, table_stride, seq_lens, batch, max_len, 0, 0);
  set_tables(kv, block_tables, table_stride, seq_lens, &p.seqs);
  p.q = static_cast<const uint16_t*>(q);
  p.k_pool = static_cast<const uint16_t*>(kv->k_pool);
  p.lse = lse;
  p.prev = prev;
  p.weights = weights;
  p.weight_stride = weight_stride;
  p.h_q = h_q;
  p.h_kv = h_kv;
  p.group = h_q / h_kv;
  block_divider((uint32_t)p.group, &p.group_magic, &p.group_shift);
  p.scale_log2 = (float)((double)scale * 1.4426950408889634);
  return mocap::launch_decode_key_weights(p, head_dim, static_cast<hipStream_t>(stream)) == hipSuccess ? MOCAP_OK
                                                                                                       : MOCAP_ERR_HIP;
}

mocap_status mocap_kv_evict_workspace_size(int64_t n, int32_t h_kv, int32_t keep, size_t* bytes_out) {
  if (bytes_out == nullptr || n < 0 || n > kMaxPositions || h_kv <= 0 || keep < 0 || keep > n || (n > 0 && keep == 0))
    return MOCAP_ERR_INVALID_ARG;
  if (h_kv > 65535 || n > kEvictMaxPositions) return MOCAP_ERR_UNSUPPORTED;
  const int32_t chunks = evict_chunks(n);
  *bytes_out = chunks > 0 ? (size_t)h_kv * mocap::evict_head_words(chunks) * sizeof(uint32_t) : 0;
  return MOCAP_OK;
}

mocap_status mocap_kv_evict(const mocap_kv_store* src, const int32_t* src_table, int32_t n_src_table,
                            const mocap_kv_store* dst, const int32_t* dst_table, int32_t n_dst_table, int64_t n,
                            int32_t keep, int32_t sinks, int32_t recent, const float* weights, int64_t weight_stride,
                            int32_t* kept, float* kept_weights, void* workspace, size_t workspace_bytes, void* stream) {
  mocap_status st = check_store(src);
  if (st == MOCAP_OK) st = check_store(dst);
  if (st != MOCAP_OK) return st;
  if (src->h_kv != dst->h_kv || src->head_dim != dst->head_dim || n < 0 || n > kMaxPositions || keep < 0 || keep > n ||
      (n > 0 && keep == 0) || sinks < 0 || recent < 0 || (int64_t)sinks + recent > keep || weight_stride < n)
    return MOCAP_ERR_INVALID_ARG;
  st = check_positions(src, n_src_table, n, 0);
  if (st == MOCAP_OK) st = check_positions(dst, n_dst_table, 0, keep);
  if (st != MOCAP_OK) return st;
  if (n == 0) return MOCAP_OK;
  if (!src->k_pool || !src->v_pool || !dst->k_pool || !dst->v_pool || !src_table || !dst_table || !weights || !kept)
    return MOCAP_ERR_INVALID_ARG;
  if (!aligned16(src->k_pool) || !aligned16(src->v_pool) || !aligned16(dst->k_pool) || !aligned16(dst->v_pool) ||
      !aligned4(src_table) || !aligned4(dst_table) || !aligned4(weights) || !aligned4(kept) ||
      !aligned4(kept_weights))
    return MOCAP_ERR_INVALID_ARG;
  if ((src->k_pool == dst->k_pool || src->v_pool == dst->v_pool) && src_table == dst_table) return MOCAP_ERR_INVALID_ARG;
  if (kept_weights != nullptr &&
      overlap(weights, extent(src->h_kv, weight_stride, n), kept_weights, (wide)src->h_kv * (wide)keep))
    return MOCAP_ERR_INVALID_ARG;
  size_t need = 0;
  st = mocap_kv_evict_workspace_size(n, src->h_kv, keep, &need);
  if (st != MOCAP_OK) return st;
  if (need > 0 && (!workspace || !aligned16(workspace) || workspace_bytes < need)) return MOCAP_ERR_WORKSPACE;
  MOCAP_DEBUG_CHECK(src_table, 0, n, src);
  MOCAP_DEBUG_CHECK(dst_table, 0, keep, dst);
  mocap::EvictLaunch p;
  p.k_src = static_cast<const uint16_t*>(src->k_pool);
  p.v_src = static_cast<const uint16_t*>(src->v_pool);
  p.k_dst = static_cast<uint16_t*>(dst->k_pool);
  p.v_dst = static_cast<uint16_t*>(dst->v_pool);
  p.src_table = src_table;
  p.dst_table = dst_table;
  p.weights = weights;
  p.kept = kept;
  p.kept_weights = kept_weights;
  p.weight_stride = weight_stride;
  p.n = (int32_t)n;
  p.keep = keep;
  p.sinks = sinks;
  p.recent = recent;
  p.h_kv = src->h_kv;
  p.src_block_size = src->block_size;
  p.dst_block_size = dst->block_size;
  p.chunks = evict_chunks(n - sinks - recent);
  p.ws = static_cast<uint32_t*>(workspace);
  return mocap::launch_kv_evict(p, src->head_dim, static_cast<hipStream_t>(stream)) == hipSuccess ? MOCAP_OK
                                                                                                  : MOCAP_ERR_HIP;
}

}  // extern "C"
