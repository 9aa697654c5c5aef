// Host side of the rotating appends and of the 4-bit store (mocap_cache.h):
// argument validation, how the work is cut, and kernel dispatch.  Every check runs
// before anything is enqueued.
#include "mocap_cache.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "cache.h"
#include "serve_host.h"

namespace {

using namespace mocap;

// A 4-bit store as the checks of sizes, tables and pool pointers see it.
mocap_kv_store view_of(const mocap_kv4_store* kv) {
  return mocap_kv_store{kv->k_pool, kv->v_pool, kv->num_blocks, kv->block_size, kv->h_kv, kv->head_dim};
}

bool scales_missing(const mocap_kv4_store* kv) {
  return !kv->k_scale || !kv->v_scale || !aligned16(kv->k_scale) || !aligned16(kv->v_scale);
}

StorePools pools_of(const mocap_kv_store* kv) { return StorePools{kv->k_pool, kv->v_pool, nullptr, nullptr}; }
StorePools pools_of(const mocap_kv4_store* kv) {
  return StorePools{kv->k_pool, kv->v_pool, static_cast<uint8_t*>(kv->k_scale), static_cast<uint8_t*>(kv->v_scale)};
}

mocap_status done(hipError_t e) { return e == hipSuccess ? MOCAP_OK : MOCAP_ERR_HIP; }

// ---- A chunk's attention ----

// A chunk of few rows, or with few keys, takes decoding's way (kv4_decode.hip): tiles from the
// store to registers, a wavefront each, without barriers, in blocks of 16 or 32 rows that each
// read them.  A block's four wavefronts take 1.4 or 1.75 us for a tile each, where 256 rows take
// 1.9 us a tile in kv4_chunk.hip, but few rows 1.5 there as well; and their fixed part is shorter.
// Measured in us, blocks of 16, of 32, workgroups of 256, d 128, 8 KV heads with groups of 4: 300
// tokens without a prefix 9.4, 10.9, 15.7; 1000 29.5, 29.3, 30.8; 2000 80, 73, 52; 100 in a window of
// 1000 11.8, 17.0, 20.7.  One of 32 and of 256: 16 rows a KV head behind 120000 positions 34 and
// 95; 64 rows behind 30000 25 and 31, 128 rows 38 and 34.  The rule is a time of each way: turns of
// the fullest compute unit, a fixed part, the merge's traffic.  Of 142 shapes the way it
// chose took at most 1.15 of the best one's time, 1.002 on average, and 0.68 of that of 256.
constexpr double kMergeUs = 3.5, kBigUs = 6.0, kSmallUs16 = 4.0, kSmallUs32 = 6.0;
// Rows that see all keys before them: long and short row groups together where every
// workgroup starts at once (32/8/128 heads, 2048 tokens without a prefix 74 -> 60 us,
// behind 2048 140 -> 124), neighbours, longest first, where they follow one another (8192
// tokens 577 us, mirrored 645).
bool mirrored_rows(const WindowLaunch& p, int cus) {
  return p.window >= p.prefix_len + p.chunk_len && p.total_wgs <= cus;
}
struct ChunkWork {
  int64_t tiles;       // of the block with the most
  double mean;         // of all blocks
};
ChunkWork work_of(const WindowLaunch& p, int64_t block) {
  const int64_t end = (int64_t)p.prefix_len + p.chunk_len;
  const int64_t span = std::min<int64_t>(p.chunk_len, ceil_div(block, p.group) + 1) + p.window;
  ChunkWork w;
  w.tiles = std::min(ceil_div(end, kTileKeys), ceil_div(span, kTileKeys) + 1 + ceil_div(p.sinks, kTileKeys));
  w.mean = std::min((double)w.tiles, (p.prefix_len + 0.5 * p.chunk_len) / kTileKeys + 1.0);
  return w;
}
double merge_us(const WindowLaunch& p, int32_t head_dim, int64_t n) {
  return n > 1 ? kMergeUs + 8.0 * n * p.chunk_len * p.h_q * (head_dim + 1) / kWindowMergeBytesPerUs : 0.0;
}

mocap_status plan_chunk(int64_t prefix_len, int32_t chunk_len, int32_t h_q, int32_t h_kv, int32_t head_dim,
                        int64_t window, int64_t sinks, int32_t num_splits, WindowLaunch* p, bool* few) {
  if (window == 0) window = kMaxPositions, sinks = 0;
  *few = false;
  mocap_status st = plan_window(prefix_len, chunk_len, h_q, h_kv, head_dim, window, sinks, num_splits, p);
  if (st != MOCAP_OK) return st;
  int cus = 0;
  st = device_cu_count(&cus);
  if (st != MOCAP_OK) return st;
  const int64_t rows = (int64_t)chunk_len * p->group;
  const ChunkWork big = work_of(*p, kWindowRows);
  const bool d64 = head_dim == 64;
  const double big_tile = rows <= kWindowRows / 2 ? (d64 ? 1.1 : 1.5) : (d64 ? 1.4 : 1.9);
  // (A workgroup with mirrored row groups walks the later one's tiles, half of them for both.)
  const double big_tiles = mirrored_rows(*p, cus)
                               ? 0.5 * (big.tiles + big.mean)
                               : std::max((double)big.tiles, ceil_div(p->total_wgs, cus) * big.mean);
  double best_us = big_tiles / p->n_ranges * big_tile + kBigUs + merge_us(*p, head_dim, p->n_ranges);
  int64_t best = 0, best_blocks = 0;
  for (const int64_t block : {16, 32}) {
    const int64_t blocks = ceil_div(rows, block);
    if (block == 32 && rows <= 16) break;
    const ChunkWork small = work_of(*p, block);
    const double turn = block == 16 ? (d64 ? 1.1 : 1.4) : (d64 ? 1.25 : 1.75);  // of a workgroup's four wavefronts
    const double fixed = block == 16 ? kSmallUs16 : kSmallUs32;
    const int64_t most = std::min<int64_t>(num_splits > 0 ? num_splits : 128, small.tiles);
    for (int64_t n = num_splits > 0 ? most : 1; n <= most; n += n < 32 ? 1 : 8) {
      if (blocks * h_kv * n > kMaxGroups) break;
      // (Two workgroups of 16 rows share a compute unit's time; of 32, one after the other.)
      const int64_t wgs = blocks * h_kv * n;
      const double per_cu = wgs <= cus ? 1.0 : block == 16 ? 0.5 * ceil_div(2 * wgs, cus) : (double)ceil_div(wgs, cus);
      const double turns = std::max((double)ceil_div(small.tiles, 4 * n), per_cu * (small.mean / (4 * n) + 0.5));
      const double us = turns * turn + fixed + merge_us(*p, head_dim, n);
      if (us < best_us) best_us = us, best = n, best_blocks = blocks;
    }
  }
  if (best == 0) return MOCAP_OK;
  *few = true;
  p->row_blocks = (int32_t)best_blocks;
  p->n_ranges = (int32_t)best;
  p->total_wgs = (int32_t)(best_blocks * h_kv * best);
  return MOCAP_OK;
}

// ---- A batch's attention ----

// Groups of more than 16 heads: blocks of 16, which start sooner (NT 1: less to join in LDS), or of
// 32, which read and convert keys and values once, where a compute unit has more than kBlockTurns
// turns of four tiles at the most.  Measured in us, blocks of 16 and of 32: one sequence of 2048,
// 32/1/128 10.6 and 12.7; 8 of 1024, 64/2/128 10.3 and 14.3; at 8 turns 64/2/128 22.5 and 23.1,
// 128/2/64 21.9 and 22.4, 40/2/128 21.9 and 21.2; at 24 64/1/64 29.4 and 27.7; at 64 128/2/64 61.1
// and 52.3.
constexpr int64_t kBlockTurns = 8;
// Workgroups a compute unit, at most, of blocks of 16 heads of such groups: as for wide groups over the
// bf16 store.  With so few turns it hardly matters: 2, 3, 4, 5 and 8 were within 2% of one another
// for 40 batches (1 of 572 to 32 of 1024; 32/1/128, 64/1/64, 64/2/128, 40/2/128, 128/2/64).
constexpr int kBlockGroupsPerCu = 3;
mocap_status plan_batch_rows(int32_t batch, int64_t max_len, int32_t h_q, int32_t h_kv, int64_t window, int64_t sinks,
                             DecodeAttnLaunch* p) {
  mocap_status st = plan_decode(batch, max_len, h_q, h_kv, window, sinks, p);
  if (st != MOCAP_OK || p->group <= 16) return st;
  int cus = 0;
  st = device_cu_count(&cus);
  if (st != MOCAP_OK) return st;
  int64_t tiles = ceil_div(max_len, kTileKeys);
  if (p->seqs.window > 0)
    tiles = std::min(tiles, ceil_div(p->seqs.window, kTileKeys) + 1 + ceil_div(p->seqs.sinks, kTileKeys));
  const int64_t blocks = ceil_div(p->group, 16);
  if (batch * tiles * h_kv * blocks > kBlockTurns * 4 * cus) return MOCAP_OK;
  p->row_blocks = (int32_t)blocks;
  return plan_batch(batch, max_len, window, sinks, h_kv * blocks, kBlockGroupsPerCu, true, &p->seqs, &p->may_split);
}

// ---- Rows ----

// 2-byte values of `tokens` rows of `heads` heads.
bool overlap_bf16(const void* a, int64_t a_stride, const void* b, int64_t b_stride, int64_t tokens, int64_t a_row,
                  int64_t b_row) {
  const wide x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + 2 * extent(tokens, b_stride, b_row) && y < x + 2 * extent(tokens, a_stride, a_row);
}

// Checks the rotation and the rows of Q, K and V of `tokens` tokens, and fills in
// their part of the launch.
mocap_status set_rows(const mocap_kv_store& kv, const mocap_rope* rope, const void* q, int64_t q_stride, int32_t h_q,
                      const void* k, int64_t k_stride, const void* v, int64_t v_stride, void* q_out, int64_t tokens,
                      RopeAppendLaunch* p) {
  p->inv_freq = nullptr;
  p->rot = 0;
  p->interleaved = false;
  if (rope != nullptr) {
    if (!rope->inv_freq || !aligned4(rope->inv_freq) || rope->rot_dim <= 0 || rope->rot_dim > kv.head_dim)
      return MOCAP_ERR_INVALID_ARG;
    if (rope->rot_dim % 16 != 0) return MOCAP_ERR_UNSUPPORTED;
    p->inv_freq = rope->inv_freq;
    p->rot = rope->rot_dim;
    p->interleaved = rope->interleaved != 0;
  }
  const int64_t kv_row = (int64_t)kv.h_kv * kv.head_dim, q_row = (int64_t)h_q * kv.head_dim;
  if (h_q < 0 || h_q % kv.h_kv != 0) return MOCAP_ERR_INVALID_ARG;
  if (k_stride < kv_row || v_stride < kv_row || k_stride % 8 != 0 || v_stride % 8 != 0) return MOCAP_ERR_INVALID_ARG;
  if (!k || !v || !aligned16(k) || !aligned16(v)) return MOCAP_ERR_INVALID_ARG;
  if (h_q > 0) {
    if (!q || !q_out || !aligned16(q) || !aligned16(q_out) || q_stride < q_row || q_stride % 8 != 0)
      return MOCAP_ERR_INVALID_ARG;
    const bool in_place = q_out == q && q_stride == q_row;
    if ((!in_place && overlap_bf16(q_out, q_row, q, q_stride, tokens, q_row, q_row)) ||
        overlap_bf16(q_out, q_row, k, k_stride, tokens, q_row, kv_row) ||
        overlap_bf16(q_out, q_row, v, v_stride, tokens, q_row, kv_row))
      return MOCAP_ERR_INVALID_ARG;
  }
  p->q = static_cast<const uint16_t*>(q);
  p->k = static_cast<const uint16_t*>(k);
  p->v = static_cast<const uint16_t*>(v);
  p->q_out = static_cast<uint16_t*>(q_out);
  p->q_stride = q_stride;
  p->k_stride = k_stride;
  p->v_stride = v_stride;
  p->h_q = h_q;
  p->h_kv = kv.h_kv;
  p->block_size = kv.block_size;
  return MOCAP_OK;
}

mocap_status append_chunk(const mocap_kv_store& kv, const StorePools& pools, bool scales_bad,
                          const int32_t* block_table, int32_t n_table, int64_t start_pos, int32_t chunk_len,
                          const mocap_rope* rope, int64_t first_pos, const void* q, int64_t q_stride, int32_t h_q,
                          const void* k, int64_t k_stride, const void* v, int64_t v_stride, void* q_out, void* stream) {
  mocap_status st = check_store(&kv);
  if (st == MOCAP_OK) st = check_positions(&kv, n_table, start_pos, chunk_len);
  if (st != MOCAP_OK) return st;
  if (first_pos < 0 || first_pos > kMaxPositions - chunk_len)
    return MOCAP_ERR_INVALID_ARG;
  if (chunk_len == 0) return MOCAP_OK;
  if (!kv.k_pool || !kv.v_pool || !block_table || !aligned16(kv.k_pool) || !aligned16(kv.v_pool) || scales_bad ||
      !aligned4(block_table))
    return MOCAP_ERR_INVALID_ARG;
  RopeAppendLaunch p{};
  st = set_rows(kv, rope, q, q_stride, h_q, k, k_stride, v, v_stride, q_out, chunk_len, &p);
  if (st != MOCAP_OK) return st;
  if (ceil_div(start_pos % kTileKeys + chunk_len, kTileKeys) > kMaxGroups ||
      kv.h_kv + ceil_div(h_q, kRopeHeads) > 65535)
    return MOCAP_ERR_UNSUPPORTED;
  MOCAP_DEBUG_CHECK(block_table, start_pos, start_pos + chunk_len, &kv);
  p.pools = pools;
  p.tables = block_table;
  p.start_pos = start_pos;
  p.first_pos = first_pos;
  p.chunk_len = chunk_len;
  return done(launch_rope_append(p, kv.head_dim, static_cast<hipStream_t>(stream)));
}

mocap_status append_batch(const mocap_kv_store& kv, const StorePools& pools, bool scales_bad,
                          const int32_t* block_tables, int32_t table_stride, const int32_t* seq_lens, int32_t batch,
                          const mocap_rope* rope, const int32_t* positions, const void* q, int64_t q_stride,
                          int32_t h_q, const void* k, int64_t k_stride, const void* v, int64_t v_stride, void* q_out,
                          void* stream) {
  mocap_status st = check_batch(&kv, block_tables, table_stride, seq_lens, batch, 0);
  if (st != MOCAP_OK || batch == 0) return st;
  if (scales_bad || !aligned4(positions)) return MOCAP_ERR_INVALID_ARG;
  RopeAppendLaunch p{};
  st = set_rows(kv, rope, q, q_stride, h_q, k, k_stride, v, v_stride, q_out, batch, &p);
  if (st != MOCAP_OK) return st;
  if (batch > kMaxGroups || ((int64_t)kv.h_kv + h_q) * (kv.head_dim / 16) > 65535 * 64) return MOCAP_ERR_UNSUPPORTED;
  MOCAP_DEBUG_CHECK_BATCH(&kv, block_tables, table_stride, seq_lens, batch, (int64_t)table_stride * kv.block_size, 1, 0,
                          true);
  p.pools = pools;
  p.tables = block_tables;
  p.seq_lens = seq_lens;
  p.positions = positions;
  p.table_stride = table_stride;
  p.batch = batch;
  return done(launch_decode_rope_append(p, kv.head_dim, static_cast<hipStream_t>(stream)));
}

}  // namespace

extern "C" {

mocap_status mocap_rope_append(const mocap_kv_store* kv, const int32_t* block_table, int32_t n_table,
                               int64_t start_pos, int32_t chunk_len, const mocap_rope* rope, int64_t first_pos,
                               const void* q, int64_t q_stride, int32_t h_q, const void* k, int64_t k_stride,
                               const void* v, int64_t v_stride, void* q_out, void* stream) {
  if (kv == nullptr) return MOCAP_ERR_INVALID_ARG;
  return append_chunk(*kv, pools_of(kv), false, block_table, n_table, start_pos, chunk_len, rope, first_pos, q,
                      q_stride, h_q, k, k_stride, v, v_stride, q_out, stream);
}

mocap_status mocap_kv4_append(const mocap_kv4_store* kv, const int32_t* block_table, int32_t n_table,
                              int64_t start_pos, int32_t chunk_len, const mocap_rope* rope, int64_t first_pos,
                              const void* q, int64_t q_stride, int32_t h_q, const void* k, int64_t k_stride,
                              const void* v, int64_t v_stride, void* q_out, void* stream) {
  if (kv == nullptr) return MOCAP_ERR_INVALID_ARG;
  return append_chunk(view_of(kv), pools_of(kv), scales_missing(kv), block_table, n_table, start_pos, chunk_len, rope,
                      first_pos, q, q_stride, h_q, k, k_stride, v, v_stride, q_out, stream);
}

mocap_status mocap_decode_rope_append(const mocap_kv_store* kv, const int32_t* block_tables, int32_t table_stride,
                                      const int32_t* seq_lens, int32_t batch, const mocap_rope* rope,
                                      const int32_t* positions, const void* q, int64_t q_stride, int32_t h_q,
                                      const void* k, int64_t k_stride, const void* v, int64_t v_stride, void* q_out,
                                      void* stream) {
  if (kv == nullptr) return MOCAP_ERR_INVALID_ARG;
  return append_batch(*kv, pools_of(kv), false, block_tables, table_stride, seq_lens, batch, rope, positions, q,
                      q_stride, h_q, k, k_stride, v, v_stride, q_out, stream);
}

mocap_status mocap_kv4_decode_append(const mocap_kv4_store* kv, const int32_t* block_tables, int32_t table_stride,
                                     const int32_t* seq_lens, int32_t batch, const mocap_rope* rope,
                                     const int32_t* positions, const void* q, int64_t q_stride, int32_t h_q,
                                     const void* k, int64_t k_stride, const void* v, int64_t v_stride, void* q_out,
                                     void* stream) {
  if (kv == nullptr) return MOCAP_ERR_INVALID_ARG;
  return append_batch(view_of(kv), pools_of(kv), scales_missing(kv), block_tables, table_stride, seq_lens, batch, rope,
                      positions, q, q_stride, h_q, k, k_stride, v, v_stride, q_out, stream);
}

mocap_status mocap_kv4_load(const mocap_kv4_store* kv, const int32_t* block_tables, int32_t table_stride,
                            const int32_t* ends, int32_t batch, int32_t n, void* k, void* v, void* stream) {
  if (kv == nullptr || n < 0 || n > kMaxPositions) return MOCAP_ERR_INVALID_ARG;
  const mocap_kv_store view = view_of(kv);
  const mocap_status st = check_batch(&view, block_tables, table_stride, ends, batch, 0);
  if (st != MOCAP_OK || batch == 0) return st;
  if (scales_missing(kv)) return MOCAP_ERR_INVALID_ARG;
  if (n == 0) return MOCAP_OK;
  if (!k || !v || !aligned16(k) || !aligned16(v)) return MOCAP_ERR_INVALID_ARG;
  if (batch > 65535 || kv->h_kv > 65535 || ceil_div(n, kTileKeys) + 1 > kMaxGroups) return MOCAP_ERR_UNSUPPORTED;
  MOCAP_DEBUG_CHECK_BATCH(&view, block_tables, table_stride, ends, batch, (int64_t)table_stride * kv->block_size, n, 0,
                          true);
  const Kv4LoadLaunch p{pools_of(kv), block_tables, ends, table_stride, static_cast<uint16_t*>(k),
                        static_cast<uint16_t*>(v), batch, n, kv->h_kv, kv->block_size};
  return done(launch_kv4_load(p, kv->head_dim, static_cast<hipStream_t>(stream)));
}

mocap_status mocap_kv4_decode_attn_workspace_size(int32_t batch, int64_t max_len, int32_t h_q, int32_t h_kv,
                                                  int32_t head_dim, int64_t window, int64_t sinks, size_t* bytes_out) {
  if (bytes_out == nullptr || batch < 0 || max_len < 0 || max_len > kMaxPositions || window < 0 || sinks < 0)
    return MOCAP_ERR_INVALID_ARG;
  mocap_status st = check_heads(h_q, h_kv, head_dim);
  if (st != MOCAP_OK) return st;
  *bytes_out = 0;
  if (batch == 0) return MOCAP_OK;
  DecodeAttnLaunch p;
  st = plan_batch_rows(batch, max_len, h_q, h_kv, window, sinks, &p);
  if (st == MOCAP_OK) *bytes_out = decode_workspace(p, head_dim);
  return st;
}

mocap_status mocap_kv4_decode_attn(const mocap_kv4_store* kv, const int32_t* block_tables, int32_t table_stride,
                                   const int32_t* seq_lens, int32_t batch, int64_t max_len, const void* q, int32_t h_q,
                                   int32_t h_kv, int32_t head_dim, float scale, int64_t window, int64_t sinks, void* o,
                                   float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  if (kv == nullptr) return MOCAP_ERR_INVALID_ARG;
  const mocap_kv_store view = view_of(kv);
  mocap_status st = check_batch(&view, block_tables, table_stride, seq_lens, batch, max_len);
  if (st != MOCAP_OK) return st;
  if (h_q <= 0 || h_kv <= 0 || h_q % h_kv != 0 || h_kv != kv->h_kv || head_dim != kv->head_dim || !valid_scale(scale) ||
      window < 0 || sinks < 0)
    return MOCAP_ERR_INVALID_ARG;
  if (batch == 0) return MOCAP_OK;
  if (scales_missing(kv) || !q || !o || !lse || !aligned16(q) || !aligned16(o) || !aligned4(lse))
    return MOCAP_ERR_INVALID_ARG;
  Kv4DecodeLaunch p;
  st = plan_batch_rows(batch, max_len, h_q, h_kv, window, sinks, &p.a);
  if (st != MOCAP_OK) return st;
  if (p.a.may_split && (!workspace || !aligned16(workspace) || workspace_bytes < decode_workspace(p.a, head_dim)))
    return MOCAP_ERR_WORKSPACE;
  MOCAP_DEBUG_CHECK_BATCH(&view, block_tables, table_stride, seq_lens, batch, max_len, window, sinks);
  set_tables(&view, block_tables, table_stride, seq_lens, &p.a.seqs);
  p.a.q = static_cast<const uint16_t*>(q);
  p.a.k_pool = static_cast<const uint16_t*>(kv->k_pool);
  p.a.v_pool = static_cast<const uint16_t*>(kv->v_pool);
  p.k_scale = static_cast<const uint8_t*>(kv->k_scale);
  p.v_scale = static_cast<const uint8_t*>(kv->v_scale);
  p.a.o = static_cast<uint16_t*>(o);
  p.a.lse = lse;
  p.a.ws_o = nullptr;
  p.a.ws_lse = nullptr;
  if (p.a.may_split) {
    p.a.ws_o = static_cast<float*>(workspace);
    p.a.ws_lse = reinterpret_cast<float*>(static_cast<char*>(workspace) +
                                          round_up((size_t)p.a.seqs.items * h_q * head_dim * sizeof(float), 256));
  }
  p.a.scale_log2 = (float)((double)scale * 1.4426950408889634);
  return done(launch_kv4_decode(p, head_dim, static_cast<hipStream_t>(stream)));
}

mocap_status mocap_kv4_chunk_attn_workspace_size(int64_t prefix_len, int32_t chunk_len, int32_t h_q, int32_t h_kv,
                                                 int32_t head_dim, int64_t window, int64_t sinks, int32_t num_splits,
                                                 int32_t* splits_out, size_t* bytes_out) {
  if (bytes_out == nullptr || window < 0 || sinks < 0 || num_splits < 0) return MOCAP_ERR_INVALID_ARG;
  mocap_status st = check_chunk(prefix_len, chunk_len);
  if (st == MOCAP_OK) st = check_heads(h_q, h_kv, head_dim);
  if (st != MOCAP_OK) return st;
  WindowLaunch p;
  p.n_ranges = 1;
  bool few;
  if (chunk_len > 0) st = plan_chunk(prefix_len, chunk_len, h_q, h_kv, head_dim, window, sinks, num_splits, &p, &few);
  if (st != MOCAP_OK) return st;
  if (splits_out) *splits_out = p.n_ranges;
  *bytes_out = chunk_len > 0 ? window_workspace(p, head_dim) : 0;
  return MOCAP_OK;
}

mocap_status mocap_kv4_chunk_attn(const mocap_kv4_store* kv, const int32_t* block_table, int32_t n_table, const void* q,
                                  int64_t prefix_len, int32_t chunk_len, int32_t h_q, int32_t h_kv, int32_t head_dim,
                                  float scale, int64_t window, int64_t sinks, void* o, float* lse, void* workspace,
                                  size_t workspace_bytes, int32_t num_splits, void* stream) {
  if (kv == nullptr) return MOCAP_ERR_INVALID_ARG;
  const mocap_kv_store view = view_of(kv);
  mocap_status st = check_chunk_args(&view, block_table, n_table, q, prefix_len, chunk_len, h_q, h_kv, head_dim, scale);
  if (st != MOCAP_OK) return st;
  if (window < 0 || sinks < 0 || num_splits < 0) return MOCAP_ERR_INVALID_ARG;
  if (chunk_len == 0) return MOCAP_OK;
  if (scales_missing(kv) || !o || !lse || !aligned16(o) || !aligned4(lse)) return MOCAP_ERR_INVALID_ARG;
  Kv4ChunkLaunch p;
  bool few;
  st = plan_chunk(prefix_len, chunk_len, h_q, h_kv, head_dim, window, sinks, num_splits, &p.a, &few);
  if (st != MOCAP_OK) return st;
  if (p.a.n_ranges > 1 && (!workspace || !aligned16(workspace) || workspace_bytes < window_workspace(p.a, head_dim)))
    return MOCAP_ERR_WORKSPACE;
  MOCAP_DEBUG_CHECK(block_table, 0, std::min<int64_t>(p.a.sinks, prefix_len + chunk_len), &view);
  MOCAP_DEBUG_CHECK(block_table, std::max<int64_t>(0, prefix_len - p.a.window + 1), prefix_len + chunk_len, &view);
  p.a.q = static_cast<const uint16_t*>(q);
  p.a.k_pool = static_cast<const uint16_t*>(kv->k_pool);
  p.a.v_pool = static_cast<const uint16_t*>(kv->v_pool);
  p.k_scale = static_cast<const uint8_t*>(kv->k_scale);
  p.v_scale = static_cast<const uint8_t*>(kv->v_scale);
  int cus = 0;
  st = device_cu_count(&cus);
  if (st != MOCAP_OK) return st;
  p.mirrored = mirrored_rows(p.a, cus);
  p.a.table = block_table;
  p.a.o = static_cast<uint16_t*>(o);
  p.a.lse = lse;
  p.a.block_size = kv->block_size;
  block_divider((uint32_t)kv->block_size, &p.a.block_magic, &p.a.block_shift);
  p.a.scale_log2 = (float)((double)scale * 1.4426950408889634);
  p.a.ws_o = nullptr;
  p.a.ws_lse = nullptr;
  if (p.a.n_ranges > 1) {
    p.a.ws_o = static_cast<float*>(workspace);
    p.a.ws_lse = reinterpret_cast<float*>(
        static_cast<char*>(workspace) + round_up((size_t)p.a.n_ranges * h_q * chunk_len * head_dim * sizeof(float), 256));
  }
  hipStream_t s = static_cast<hipStream_t>(stream);
  if ((few ? launch_kv4_few_rows : launch_kv4_chunk)(p, head_dim, s) != hipSuccess) return MOCAP_ERR_HIP;
  if (p.a.n_ranges > 1) {
    const MergeLaunch m{p.a.ws_o, p.a.ws_lse, p.a.o, lse, chunk_len, h_q, p.a.n_ranges};
    if (launch_lse_merge(m, head_dim, s) != hipSuccess) return MOCAP_ERR_HIP;
  }
  return MOCAP_OK;
}

}  // extern "C"
