/*
 * mocap_serve.h -- the calls of libmocap_attn that follow the prefill: decoding
 * over the paged KV store, attention in a sliding window, accumulated key
 * weights and eviction by them, on AMD Instinct MI355X (gfx950).
 *
 * The store, its block tables, the GQA groups, the precision of the inputs and
 * the conventions on pointers, streams, alignment and errors are those of
 * mocap_attn.h; every call only enqueues kernel launches (no allocation, no
 * memset) and can be captured into a HIP graph.  In addition:
 *   - A batch of sequences shares one store.  block_tables is a device int32
 *     array [batch][table_stride]; row b is the block table of sequence b.
 *     Sequences may share physical blocks that are only read (a common
 *     prefix); a block that is written to must belong to one sequence.
 *   - seq_lens is a device int32 array [batch]: n_b, the number of positions of
 *     sequence b, its new token included.  0 or less is a row without a
 *     sequence (a padded batch).  The host never reads it, so a captured call
 *     may be replayed with other lengths.  No position at or beyond the call's
 *     bound (max_len, table_stride * block_size) is ever accessed, whatever
 *     seq_lens holds; a sequence longer than max_len is taken to end there.
 *   - Block tables, lengths, positions and fp32 arrays (lse, weights) need only
 *     the alignment of their type, so rows of larger arrays may be passed.
 *   - Outputs and the workspace must overlap no input and no other output, except
 *     where a call says so, and inputs must stay as they are until a call is done.
 *   - Calls that are given a workspace share nothing else, so calls with
 *     different workspaces (and outputs) may run at the same time.  Two
 *     captured graphs whose replays can overlap need a workspace each.
 *
 * With a window W > 0 and s sinks, the query at position t sees the keys
 *   j <= t  with  j < s  or  j > t - W
 * (the last W positions, its own included, and the first s); W = 0 means all
 * j <= t.
 */
#ifndef MOCAP_SERVE_H
#define MOCAP_SERVE_H

#include "mocap_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * mocap_decode_append -- store the new token's keys and values of every
 * sequence of a batch: mocap_kv_append of one position per sequence, in one
 * launch.
 *
 *   kv            store to write into
 *   block_tables, table_stride, seq_lens, batch   as above (batch 0 is a no-op)
 *   k, v          device bf16 [batch][h_kv][head_dim]
 *
 * Row b is written bit for bit to position n_b - 1 of sequence b; nothing is
 * written for n_b <= 0 or n_b > table_stride * block_size.  The positions
 * written must be distinct slots.
 * Errors: INVALID_ARG for null/misaligned pointers or negative sizes;
 * UNSUPPORTED as mocap_kv_append, or for a batch of 2^23 or
 * more, or h_kv * head_dim above 512 * 65535.
 */
mocap_status mocap_decode_append(const mocap_kv_store* kv, const int32_t* block_tables, int32_t table_stride,
                                 const int32_t* seq_lens, int32_t batch, const void* k, const void* v, void* stream);

/*
 * mocap_decode_attn_workspace_size -- workspace bytes of mocap_decode_attn.
 * Depends on the sizes alone, not on the sequences' lengths.  0 when no
 * sequence of up to max_len positions would be split.
 * Errors: INVALID_ARG for a null bytes_out or malformed sizes; UNSUPPORTED for
 * head_dim not in {64, 128} or too many workgroups; HIP if the device query fails.
 */
mocap_status mocap_decode_attn_workspace_size(int32_t batch, int64_t max_len, int32_t h_q, int32_t h_kv,
                                              int32_t head_dim, int64_t window, int64_t sinks, size_t* bytes_out);

/*
 * mocap_decode_attn -- attention of one new token of every sequence over its
 * paged keys and values (Section 2.2's step for a chunk of one token, for a
 * whole batch), with an optional window and sinks.
 *
 *   max_len       no sequence has more positions (>= 0); max_len <=
 *                 table_stride * block_size
 *   q             device bf16 [batch][h_q][head_dim]; the query of sequence b sits
 *                 at position n_b - 1, whose key and value are in the store
 *   scale         as in mocap_chunk_attn
 *   window, sinks >= 0 (window 0: all keys; sinks is then not used)
 *   o             device bf16 [batch][h_q][head_dim]               (output)
 *   lse           device fp32 [batch][h_q], natural log              (output)
 *   workspace     device scratch of workspace_bytes, or NULL when
 *                 mocap_decode_attn_workspace_size gives 0; its contents on entry
 *                 do not matter
 *
 * The visible keys of all sequences are cut into about equal parts, as many as
 * fill the device, whatever the sequences' lengths are; the parts of a sequence
 * are joined by their log-sum-exp in a fixed order, so equal inputs give equal
 * bits.  A row without a sequence gives O = 0 and LSE = -infinity.  What hidden
 * or unwritten positions hold (NaN included) does not matter.  An infinite value
 * is infinite in its dim of O for every row that sees it, NaN where both infinities
 * meet.  Scores, softmax and partials are fp32; the probabilities enter the P*V
 * product as the sum of two bf16 values (2^-17 relative).
 * Errors: as mocap_chunk_attn (INVALID_ARG also for a negative window or sinks,
 * a max_len beyond the tables, or null seq_lens); UNSUPPORTED also for a block of
 * 2^30 or more values per head, or batch * h_q of 2^23; WORKSPACE when the
 * workspace is missing or too small.
 */
mocap_status mocap_decode_attn(const mocap_kv_store* kv, const int32_t* block_tables, int32_t table_stride,
                               const int32_t* seq_lens, int32_t batch, int64_t max_len, const void* q, int32_t h_q,
                               int32_t h_kv, int32_t head_dim, float scale, int64_t window, int64_t sinks, void* o,
                               float* lse, void* workspace, size_t workspace_bytes, void* stream);

/*
 * mocap_window_attn_workspace_size -- the range count and workspace bytes of
 * mocap_window_attn.  num_splits as a request: 1 = one range, n >= 2 = the tiles
 * that any row of a workgroup sees cut into n ranges, 0 = chosen from the shape.
 * A request is clamped to the tiles that a workgroup's windows and sinks can touch
 * wherever in a tile they begin: at most two more than they do touch, and the ranges
 * that are then empty cost their workspace only.  splits_out may be NULL.
 * Errors: as mocap_chunk_attn_workspace_size; INVALID_ARG for window < 1 or
 * sinks < 0.
 */
mocap_status mocap_window_attn_workspace_size(int64_t prefix_len, int32_t chunk_len, int32_t h_q, int32_t h_kv,
                                              int32_t head_dim, int64_t window, int64_t sinks, int32_t num_splits,
                                              int32_t* splits_out, size_t* bytes_out);

/*
 * mocap_window_attn -- mocap_chunk_attn in which the row at position t sees only
 * its last `window` positions and the first `sinks` ones.  Blocks that no row
 * sees are not read, and neither are their table entries.
 *
 *   window >= 1, sinks >= 0; other arguments, outputs and precision as in
 *   mocap_chunk_attn
 *
 * Non-finite keys and values reach exactly the rows that see them (an infinite
 * value as infinity, or as NaN where its probability rounds to 0).  (Where the
 * window hides nothing, W >= P + L, mocap_chunk_attn gives the same rows in less
 * time, but a non-finite value there also reaches rows of its 64-key tile that do
 * not see it.)
 * Errors: as mocap_chunk_attn, plus INVALID_ARG for window < 1 or sinks < 0, and
 * UNSUPPORTED for a block of 2^30 or more values per head.
 */
mocap_status mocap_window_attn(const mocap_kv_store* kv, const int32_t* block_table, int32_t n_table, const void* q,
                               int64_t prefix_len, int32_t chunk_len, int32_t h_q, int32_t h_kv, int32_t head_dim,
                               float scale, int64_t window, int64_t sinks, void* o, float* lse, void* workspace,
                               size_t workspace_bytes, int32_t num_splits, void* stream);

/*
 * mocap_key_weights_workspace_size -- workspace bytes of mocap_key_weights (0 when
 * the rows are not cut).
 * Errors: as mocap_chunk_attn_workspace_size.
 */
mocap_status mocap_key_weights_workspace_size(int64_t prefix_len, int32_t chunk_len, int32_t h_q, int32_t h_kv,
                                              int32_t head_dim, size_t* bytes_out);

/*
 * mocap_key_weights -- the attention weight that every key received from a
 * chunk's rows, summed over the rows and the query heads of its group:
 *   weights[h][j] = (j < P ? prev[h][j] : 0)
 *                   + sum over rows i with P + i >= j and heads g of group h of
 *                     exp(scale <q_{i,g}, k_{j,h}> - lse_{g,i})
 * for j < P + L: accumulated over the chunks of a prompt, what eviction
 * (mocap_kv_evict) goes by.  A chunk may be the last rows of a longer one
 * (observers): P then counts the rows before them.
 *
 *   kv, block_table, n_table, q, prefix_len P, chunk_len L, h_q, h_kv, head_dim,
 *   scale         as in mocap_chunk_attn; only keys are read
 *   lse           device fp32 [h_q][L], natural log: that of mocap_chunk_attn for
 *                 these rows.  A row whose LSE is -infinity (every score of it is) adds
 *                 nothing; a NaN score or LSE makes the weight of the keys it meets NaN
 *   prev          device fp32 [h_kv][weight_stride], or NULL: 0 everywhere; may be
 *                 `weights` itself, and must not overlap it otherwise
 *   weights       device fp32 [h_kv][weight_stride], weight_stride >= P + L (output;
 *                 values at P + L and beyond are left as they were)
 *   workspace     device scratch of workspace_bytes, NULL when the size is 0
 *
 * Sums are fp32, added in a fixed order.  L = 0 is a no-op.
 * Errors: as mocap_chunk_attn; INVALID_ARG for a weight_stride below P + L, or a
 * prev that overlaps weights without being it; UNSUPPORTED also for more than
 * 65535 KV heads with more than 128 rows, or 128 rows of Q beyond 2 GiB.
 */
mocap_status mocap_key_weights(const mocap_kv_store* kv, const int32_t* block_table, int32_t n_table, const void* q,
                               int64_t prefix_len, int32_t chunk_len, int32_t h_q, int32_t h_kv, int32_t head_dim,
                               float scale, const float* lse, const float* prev, float* weights, int64_t weight_stride,
                               void* workspace, size_t workspace_bytes, void* stream);

/*
 * mocap_decode_key_weights -- mocap_key_weights for the new token of every
 * sequence of a batch (P = n_b - 1, L = 1):
 *   weights[b][h][j] = (j < n_b - 1 ? prev[b][h][j] : 0)
 *                      + sum over heads g of group h of
 *                        exp(scale <q_{b,g}, k_{j,h}> - lse_{b,g}),   j < n_b
 *
 *   block_tables, table_stride, seq_lens, batch, max_len, q   as in mocap_decode_attn
 *   lse           device fp32 [batch][h_q]: that of mocap_decode_attn with window 0
 *   prev, weights device fp32 [batch][h_kv][weight_stride], weight_stride >= max_len;
 *                 prev may be NULL or `weights` itself; weights of positions n_b
 *                 and beyond are left as they were
 * Errors: as mocap_decode_attn and mocap_key_weights.
 */
mocap_status mocap_decode_key_weights(const mocap_kv_store* kv, const int32_t* block_tables, int32_t table_stride,
                                      const int32_t* seq_lens, int32_t batch, int64_t max_len, const void* q,
                                      int32_t h_q, int32_t h_kv, int32_t head_dim, float scale, const float* lse,
                                      const float* prev, float* weights, int64_t weight_stride, void* stream);

/*
 * mocap_kv_evict_workspace_size -- workspace bytes of mocap_kv_evict.
 * Errors: INVALID_ARG for a null bytes_out or malformed sizes; UNSUPPORTED for
 * more than 65535 heads or 2^30 - 64 positions.
 */
mocap_status mocap_kv_evict_workspace_size(int64_t n, int32_t h_kv, int32_t keep, size_t* bytes_out);

/*
 * mocap_kv_evict -- keep `keep` of the n positions of a sequence, chosen for each
 * KV head by weight, and copy their keys and values to positions 0 .. keep - 1 of
 * other blocks.
 *
 * Head h keeps the first `sinks` positions, the last `recent` ones, and of the
 * others the keep - sinks - recent with the largest weights; among equal ones
 * the lower position.  NaN counts as the largest weight; -0 equals 0.  Kept
 * positions stay in order: position i of the result is kept[h][i], ascending.
 * (Positions of different heads then differ, which attention does not notice:
 * it sees keys, not positions.)
 *
 *   src, src_table, n_src_table   the store of positions [0, n)
 *   dst, dst_table, n_dst_table   the store that receives positions [0, keep);
 *                 the same h_kv and head_dim, any supported block size.  It may
 *                 be the same store; the blocks it is given must not be among
 *                 those of src (the same pool with the same table is refused).
 *   n             positions (>= 0); 1 <= keep <= n, or n = keep = 0, a no-op;
 *                 sinks, recent >= 0, sinks + recent <= keep
 *   weights       device fp32 [h_kv][weight_stride], weight_stride >= n
 *   kept          device int32 [h_kv][keep]        (output; must overlap neither
 *                 weights nor kept_weights)
 *   kept_weights  device fp32 [h_kv][keep], or NULL: the kept positions' weights
 *                 (output; must not overlap weights)
 *   workspace     device scratch of workspace_bytes, NULL when the size is 0
 *
 * Slots of dst at position keep and beyond are left as they were.
 * Errors: INVALID_ARG for null/misaligned pointers, malformed sizes, stores that
 * differ in h_kv or head_dim, tables that are too short, dst = src (see above),
 * or kept_weights that overlap weights; UNSUPPORTED as mocap_kv_evict_workspace_size, or for a head_dim or
 * block_size that mocap_kv_append does not take; WORKSPACE when the workspace is
 * missing or too small; HIP if a launch fails.
 */
mocap_status mocap_kv_evict(const mocap_kv_store* src, const int32_t* src_table, int32_t n_src_table,
                            const mocap_kv_store* dst, const int32_t* dst_table, int32_t n_dst_table, int64_t n,
                            int32_t keep, int32_t sinks, int32_t recent, const float* weights, int64_t weight_stride,
                            int32_t* kept, float* kept_weights, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* MOCAP_SERVE_H */
