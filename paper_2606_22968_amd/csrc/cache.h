// Launch descriptions of the rotating appends and of the 4-bit store
// (mocap_cache.h), shared by their host side and kernels.  Not part of the public
// ABI.
#pragma once

#include "serve.h"

namespace mocap {

// A store of either kind: bf16 pools, or 4-bit pools and their scales.
struct StorePools {
  void* k;
  void* v;
  uint8_t* k_scale;         // null: bf16
  uint8_t* v_scale;
};

// Query heads that a workgroup of the chunk append rotates (their tokens' angles are
// made once).
constexpr int kRopeHeads = 4;
struct RopeAppendLaunch {
  const uint16_t* q;        // bf16, token i at q + i q_stride: [Hq][D]
  const uint16_t* k;
  const uint16_t* v;
  uint16_t* q_out;          // bf16 [tokens][Hq][D]
  int64_t q_stride;
  int64_t k_stride;
  int64_t v_stride;
  const float* inv_freq;    // [rot / 2]
  int32_t rot;              // rotated dims, 0: none; a multiple of 16
  bool interleaved;
  StorePools pools;
  const int32_t* tables;    // of the sequence, or [batch][table_stride]
  int32_t h_q;
  int32_t h_kv;
  int32_t block_size;
  // A chunk of one sequence.
  int64_t start_pos;
  int64_t first_pos;
  int32_t chunk_len;
  // One token of every sequence of a batch.
  const int32_t* seq_lens;
  const int32_t* positions; // or null
  int64_t table_stride;
  int32_t batch;
};

struct Kv4LoadLaunch {
  StorePools pools;
  const int32_t* tables;
  const int32_t* ends;
  int64_t table_stride;
  uint16_t* k;              // bf16 [batch][n][Hkv][D]
  uint16_t* v;
  int32_t batch;
  int32_t n;
  int32_t h_kv;
  int32_t block_size;
};

// The bf16 kernels' launches; their pool pointers are the 4-bit pools.
struct Kv4DecodeLaunch {
  DecodeAttnLaunch a;
  const uint8_t* k_scale;
  const uint8_t* v_scale;
};
struct Kv4ChunkLaunch {
  WindowLaunch a;
  const uint8_t* k_scale;
  const uint8_t* v_scale;
  bool mirrored;            // a workgroup's two row groups: the x-th from either end
};

hipError_t launch_rope_append(const RopeAppendLaunch& p, int head_dim, hipStream_t stream);
hipError_t launch_decode_rope_append(const RopeAppendLaunch& p, int head_dim, hipStream_t stream);
hipError_t launch_kv4_load(const Kv4LoadLaunch& p, int head_dim, hipStream_t stream);
hipError_t launch_kv4_decode(const Kv4DecodeLaunch& p, int head_dim, hipStream_t stream);
hipError_t launch_kv4_chunk(const Kv4ChunkLaunch& p, int head_dim, hipStream_t stream);
hipError_t launch_kv4_few_rows(const Kv4ChunkLaunch& p, int head_dim, hipStream_t stream);
// Joins the parts of a batch's sequences (decode_attn.hip); short_too: with the shorter way
// for few parts.
hipError_t launch_decode_join(const DecodeAttnLaunch& p, int head_dim, bool short_too, hipStream_t stream);

}  // namespace mocap
