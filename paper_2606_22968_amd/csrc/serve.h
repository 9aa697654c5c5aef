// Launch descriptions of the calls that follow the prefill (mocap_serve.h),
// shared by their host side and kernels.  Not part of the public ABI.
#pragma once

#include "internal.h"

namespace mocap {

// Sequences of a batch and how their visible 64-key tiles are cut into items.
// A sequence's tiles are those that hold a visible key, in order: the sinks'
// tiles, then the window's.  With T the tiles of all sequences, a part has at
// most max(T / target + 1, few) tiles, where few is min_tiles, or down to
// least_tiles when T / fill is less (when parts of min_tiles leave compute units
// free); a sequence with c tiles is cut evenly into ceil(c / that) parts (one, if
// it has none), and the items are the parts of all sequences in order.  `items`
// bounds their number for any lengths: sum ceil(c_b / part) <= T / part + batch
// <= target + batch.
struct SeqBatch {
  const int32_t* tables;    // [batch][table_stride]
  const int32_t* seq_lens;  // [batch]
  int64_t table_stride;
  int32_t batch;
  int32_t max_len;
  int32_t window;           // 0: all keys
  int32_t sinks;            // 0 when window is 0
  int32_t target;
  int32_t fill;
  int32_t min_tiles;
  int32_t least_tiles;
  int32_t items;
  int32_t block_size;
  uint32_t block_magic;     // as in AttnLaunch
  int32_t block_shift;
};

struct DecodeAppendLaunch {
  const uint16_t* k;        // bf16 [batch][Hkv][D]
  const uint16_t* v;
  uint16_t* k_pool;
  uint16_t* v_pool;
  const int32_t* tables;
  const int32_t* seq_lens;
  int64_t table_stride;
  int32_t batch;
  int32_t h_kv;
  int32_t block_size;
};

struct DecodeAttnLaunch {
  SeqBatch seqs;
  const uint16_t* q;        // bf16 [batch][Hq][D]
  const uint16_t* k_pool;
  const uint16_t* v_pool;
  uint16_t* o;              // bf16 [batch][Hq][D]
  float* lse;               // fp32 [batch][Hq]
  float* ws_o;              // fp32 [items][Hq][D]
  float* ws_lse;            // fp32 [items][Hq]
  int32_t h_q;
  int32_t h_kv;
  int32_t group;
  int32_t row_blocks;       // blocks of query heads of a group
  bool may_split;           // some sequence of up to max_len positions is cut
  float scale_log2;
};

// One launch of the window kernel.  Rows are counted as in AttnLaunch; a
// workgroup owns kWindowRows consecutive ones and walks the tiles that any of
// them sees (the sinks', then the window's), or one of n_ranges even cuts of
// those.
constexpr int kWindowRows = 256;
struct WindowLaunch {
  const uint16_t* q;
  const uint16_t* k_pool;
  const uint16_t* v_pool;
  const int32_t* table;
  uint16_t* o;
  float* lse;
  float* ws_o;              // fp32 [R][L][Hq][D]
  float* ws_lse;            // fp32 [R][L][Hq]
  int32_t prefix_len;
  int32_t chunk_len;
  int32_t h_q;
  int32_t h_kv;
  int32_t group;
  uint32_t group_magic;
  int32_t group_shift;
  int32_t row_blocks;       // ceil(L group / kWindowRows)
  int32_t block_size;
  uint32_t block_magic;
  int32_t block_shift;
  int32_t window;
  int32_t sinks;
  int32_t n_ranges;
  int32_t total_wgs;
  float scale_log2;
};

// One launch of the key weight kernel: a workgroup's eight wavefronts hold 64 keys
// each and walk an even cut of the row tiles that see some of them, part_tiles at
// most.  Keys of the prefix are seen by all tiles, in row_parts cuts.
constexpr int kWeightKeys = 64;
constexpr int kWeightWaves = 8;
struct KeyWeightsLaunch {
  const uint16_t* q;
  const uint16_t* k_pool;
  const int32_t* table;
  const float* lse;         // fp32 [Hq][L]
  const float* prev;        // fp32 [Hkv][weight_stride] or null
  float* weights;
  float* ws;                // fp32 [row_parts][Hkv][P + L] when row_parts > 1
  int64_t weight_stride;
  int32_t prefix_len;
  int32_t chunk_len;
  int32_t h_q;
  int32_t h_kv;
  int32_t group;
  uint32_t group_magic;
  int32_t group_shift;
  int32_t block_size;
  uint32_t block_magic;
  int32_t block_shift;
  bool few;                 // the kernel for few rows
  int32_t key_blocks;       // ceil((P + L) / 512); few: workgroups of a KV head
  int32_t row_parts;
  int32_t part_tiles;
  int32_t head_wgs;         // workgroups of a KV head
  float scale_log2;
};

struct DecodeKeyWeightsLaunch {
  SeqBatch seqs;
  const uint16_t* q;
  const uint16_t* k_pool;
  const float* lse;         // fp32 [batch][Hq]
  const float* prev;        // fp32 [batch][Hkv][weight_stride] or null
  float* weights;
  int64_t weight_stride;
  int32_t h_q;
  int32_t h_kv;
  int32_t group;
  uint32_t group_magic;
  int32_t group_shift;
  float scale_log2;
};

// Selection: up to kEvictOneGroup candidates by one workgroup per head (chunks
// = 0), more by `chunks` of them, with counts in the workspace.
constexpr int kEvictOneGroup = 16384;
constexpr int kEvictMaxChunks = 32;
constexpr int kEvictFirstBins = 1024, kEvictSecondBins = 4096, kEvictThirdBins = 1024;
// 32-bit words of workspace per head.
constexpr int64_t evict_head_words(int chunks) {
  return (int64_t)chunks * (kEvictFirstBins + kEvictThirdBins + 1) + kEvictSecondBins + 4;
}
struct EvictLaunch {
  const uint16_t* k_src;
  const uint16_t* v_src;
  uint16_t* k_dst;
  uint16_t* v_dst;
  const int32_t* src_table;
  const int32_t* dst_table;
  const float* weights;     // fp32 [Hkv][weight_stride]
  int32_t* kept;            // int32 [Hkv][keep]
  float* kept_weights;      // fp32 [Hkv][keep] or null
  int64_t weight_stride;
  int32_t n;
  int32_t keep;
  int32_t sinks;
  int32_t recent;
  int32_t h_kv;
  int32_t src_block_size;
  int32_t dst_block_size;
  int32_t chunks;
  uint32_t* ws;
};

hipError_t launch_decode_append(const DecodeAppendLaunch& p, int head_dim, hipStream_t stream);
hipError_t launch_decode_attn(const DecodeAttnLaunch& p, int head_dim, hipStream_t stream);
hipError_t launch_window_attn(const WindowLaunch& p, int head_dim, hipStream_t stream);
hipError_t launch_key_weights(const KeyWeightsLaunch& p, int head_dim, hipStream_t stream);
hipError_t launch_decode_key_weights(const DecodeKeyWeightsLaunch& p, int head_dim, hipStream_t stream);
hipError_t launch_kv_evict(const EvictLaunch& p, int head_dim, hipStream_t stream);

}  // namespace mocap
