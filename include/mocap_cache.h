/*
 * mocap_cache.h -- the calls of libmocap_attn that rotate keys and queries on
 * the way into the paged store, and a store that holds keys and values in
 * 4 bits with the attention that reads it, on AMD Instinct MI355X (gfx950).
 *
 * Conventions, batches of sequences, windows and sinks are those of
 * mocap_attn.h and mocap_serve.h: device pointers owned by the caller, checks
 * on the host before anything is enqueued, kernel launches only (no
 * allocation, no memset), so every call can be captured into a HIP graph;
 * seq_lens, positions and ends stay on the device and are never read by the
 * host.  Inputs must stay as they are until a call is done, and outputs overlap
 * no input and no other output, except where a call says so.
 */
#ifndef MOCAP_CACHE_H
#define MOCAP_CACHE_H

#include "mocap_serve.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Rotation of a head's first rot_dim dims by its position p: for i < rot_dim / 2
 * the pair (x, y) becomes
 *   (x cos a - y sin a, x sin a + y cos a),   a = p * inv_freq[i],
 * where x, y are dims i and i + rot_dim / 2, or 2 i and 2 i + 1 if interleaved.
 * Other dims stay as they are.  Angles are taken exactly, so far positions lose
 * nothing; a pair whose angle is 2^48 radians or more, or no number, becomes NaN.
 *   inv_freq      device fp32 [rot_dim / 2]; below 2^17 (a layer's are at most 1) no
 *                 position reaches that
 *   rot_dim       16 .. head_dim, a multiple of 16
 */
typedef struct mocap_rope {
  const float* inv_freq;
  int32_t rot_dim;
  int32_t interleaved;
} mocap_rope;

/*
 * A paged store in 4 bits (4.25 with its scales).  32 consecutive dims of one
 * position and KV head share a scale 2^e, e the smallest with
 * max |x| <= 6 * 2^e; a value is held as the nearest of 0, 0.5, 1, 1.5, 2, 3, 4,
 * 6 (codes 0 to 7; ties to the even code; bit 3 is the sign), times 2^e.  The
 * scale's byte is e + 127, from 2 to 252 (larger values are cut to 6 * 2^125); a
 * block that holds a NaN or an infinity has the byte 255 and reads as NaN.
 *
 *   k_pool   uint8 [num_blocks][h_kv][block_size][head_dim / 2]
 *            byte i: dims 2 i (low four bits) and 2 i + 1
 *   v_pool   uint8 [num_blocks][h_kv][block_size / 64][head_dim / 2][64]
 *            row 16 b + i: dims 32 b + i (low) and 32 b + 16 + i of 64 positions
 *   k_scale, v_scale   uint8 [num_blocks][h_kv][block_size / 64][head_dim / 32][64]
 *
 * head_dim 64 or 128, block_size a multiple of 64.  (The layouts are those in
 * which 64 lanes read a 64-position tile in whole lines; a byte belongs to one
 * position, so positions can be stored one at a time.)
 */
typedef struct mocap_kv4_store {
  void* k_pool;
  void* v_pool;
  void* k_scale;
  void* v_scale;
  int32_t num_blocks;
  int32_t block_size;
  int32_t h_kv;
  int32_t head_dim;
} mocap_kv4_store;

/*
 * mocap_rope_append -- mocap_kv_append of a chunk whose keys are rotated on the
 * way, and whose queries are rotated in the same launch.
 *
 *   kv, block_table, n_table, start_pos, chunk_len   as in mocap_kv_append
 *   rope          the rotation, or NULL: none
 *   first_pos     the rotation's position of the chunk's first token (>= 0; the
 *                 others follow).  Equal to start_pos unless positions were evicted
 *   q, q_stride, h_q   device bf16, token i at q + i * q_stride: [h_q][head_dim]; h_q
 *                 a multiple of h_kv, or 0 without queries (q and q_out then not used)
 *   k, k_stride, v, v_stride   device bf16, token i: [h_kv][head_dim]
 *   q_out         device bf16 [chunk_len][h_q][head_dim] (output); may be q itself if
 *                 q_stride = h_q * head_dim
 *
 * Strides are in values, multiples of 8, and at least the heads' values, so Q, K
 * and V can be parts of one projection's rows.  Products are fp32, results are
 * rounded to bf16 once; V and dims that are not rotated are copied bit for bit.
 * Errors: INVALID_ARG for null or misaligned pointers (inv_freq: 4 bytes, others
 * 16), malformed sizes, strides or tables, positions beyond 2^31 - 128, or a q_out
 * that overlaps q, k or v otherwise; UNSUPPORTED for a head_dim or block_size that
 * mocap_kv_append does not take, a rot_dim that is no multiple of 16, or too many
 * workgroups; HIP if a launch fails.
 */
mocap_status mocap_rope_append(const mocap_kv_store* kv, const int32_t* block_table, int32_t n_table,
                               int64_t start_pos, int32_t chunk_len, const mocap_rope* rope, int64_t first_pos,
                               const void* q, int64_t q_stride, int32_t h_q, const void* k, int64_t k_stride,
                               const void* v, int64_t v_stride, void* q_out, void* stream);

/*
 * mocap_decode_rope_append -- the same, to the bit, for the new token of every
 * sequence of a batch: its key and value are stored at position n_b - 1 (see
 * mocap_decode_append).
 *
 *   positions     device int32 [batch]: the rotation's positions, or NULL: n_b - 1
 *   q, k, v       token b is sequence b's
 *   q_out         device bf16 [batch][h_q][head_dim]; rows of sequences with
 *                 n_b <= 0 or n_b > table_stride * block_size are left as they were
 * Errors: as mocap_rope_append and mocap_decode_append.
 */
mocap_status mocap_decode_rope_append(const mocap_kv_store* kv, const int32_t* block_tables, int32_t table_stride,
                                      const int32_t* seq_lens, int32_t batch, const mocap_rope* rope,
                                      const int32_t* positions, const void* q, int64_t q_stride, int32_t h_q,
                                      const void* k, int64_t k_stride, const void* v, int64_t v_stride, void* q_out,
                                      void* stream);

/*
 * mocap_kv4_append, mocap_kv4_decode_append -- mocap_rope_append and
 * mocap_decode_rope_append into a 4-bit store.  Keys are rotated in fp64 and
 * rounded once, to 4 bits; q_out is as there.
 */
mocap_status mocap_kv4_append(const mocap_kv4_store* kv, const int32_t* block_table, int32_t n_table,
                              int64_t start_pos, int32_t chunk_len, const mocap_rope* rope, int64_t first_pos,
                              const void* q, int64_t q_stride, int32_t h_q, const void* k, int64_t k_stride,
                              const void* v, int64_t v_stride, void* q_out, void* stream);
mocap_status mocap_kv4_decode_append(const mocap_kv4_store* kv, const int32_t* block_tables, int32_t table_stride,
                                     const int32_t* seq_lens, int32_t batch, const mocap_rope* rope,
                                     const int32_t* positions, const void* q, int64_t q_stride, int32_t h_q,
                                     const void* k, int64_t k_stride, const void* v, int64_t v_stride, void* q_out,
                                     void* stream);

/*
 * mocap_kv4_load -- the keys and values that a 4-bit store stands for, of the
 * last n of the positions [0, ends[b]) of every sequence of a batch, in bf16 (which
 * holds them exactly): to move a sequence into a bf16 store, or to look at it.
 *
 *   block_tables, table_stride, batch   as in mocap_decode_attn
 *   ends          device int32 [batch]
 *   k, v          device bf16 [batch][n][h_kv][head_dim] (outputs): row i is position
 *                 ends[b] - n + i; rows before position 0, and all rows of a
 *                 sequence with ends[b] <= 0 or beyond the tables, are 0
 * Errors: as mocap_decode_append; INVALID_ARG for a negative n; UNSUPPORTED also
 * for more than 65535 sequences or KV heads.
 */
mocap_status mocap_kv4_load(const mocap_kv4_store* kv, const int32_t* block_tables, int32_t table_stride,
                            const int32_t* ends, int32_t batch, int32_t n, void* k, void* v, void* stream);

/*
 * mocap_kv4_decode_attn_workspace_size, mocap_kv4_decode_attn --
 * mocap_decode_attn over a 4-bit store: the same arguments, results, precision
 * and errors (but blocks of any size are taken), with the values that the store
 * stands for.  A key block that reads as NaN makes the rows that see it NaN, a
 * value block its 32 dims of them.  Weighted values are summed in fp32 before they
 * are divided by the weights' sum: values up to 2^96 in magnitude never leave it, at
 * any length; larger ones may make O infinite or NaN where it should be finite.
 */
mocap_status mocap_kv4_decode_attn_workspace_size(int32_t batch, int64_t max_len, int32_t h_q, int32_t h_kv,
                                                  int32_t head_dim, int64_t window, int64_t sinks, size_t* bytes_out);
mocap_status mocap_kv4_decode_attn(const mocap_kv4_store* kv, const int32_t* block_tables, int32_t table_stride,
                                   const int32_t* seq_lens, int32_t batch, int64_t max_len, const void* q, int32_t h_q,
                                   int32_t h_kv, int32_t head_dim, float scale, int64_t window, int64_t sinks, void* o,
                                   float* lse, void* workspace, size_t workspace_bytes, void* stream);

/*
 * mocap_kv4_chunk_attn_workspace_size, mocap_kv4_chunk_attn -- a chunk's causal
 * attention over a 4-bit store: mocap_chunk_attn with window = 0,
 * mocap_window_attn with window >= 1 (sinks then count), with their arguments,
 * results and precision (probabilities in bf16, or nearer).  The chunk's own keys
 * and values are read from the store as well.  num_splits as in
 * mocap_window_attn_workspace_size.  NaN blocks reach exactly the rows that see
 * them, as in mocap_kv4_decode_attn.  Weights may exceed 1 here, by 2^62 a tile, so
 * the values that never leave fp32 are those up to 2^40.
 * Errors: as mocap_window_attn, but window = 0 and blocks of any size are taken.
 */
mocap_status mocap_kv4_chunk_attn_workspace_size(int64_t prefix_len, int32_t chunk_len, int32_t h_q, int32_t h_kv,
                                                 int32_t head_dim, int64_t window, int64_t sinks, int32_t num_splits,
                                                 int32_t* splits_out, size_t* bytes_out);
mocap_status mocap_kv4_chunk_attn(const mocap_kv4_store* kv, const int32_t* block_table, int32_t n_table, const void* q,
                                  int64_t prefix_len, int32_t chunk_len, int32_t h_q, int32_t h_kv, int32_t head_dim,
                                  float scale, int64_t window, int64_t sinks, void* o, float* lse, void* workspace,
                                  size_t workspace_bytes, int32_t num_splits, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* MOCAP_CACHE_H */
