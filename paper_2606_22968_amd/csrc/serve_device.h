// Device code shared by the kernels that read a batch of paged sequences.
#pragma once

#include "attn_device.h"
#include "serve.h"

namespace mocap {
namespace {

__device__ __forceinline__ float quad_rows_max(float x) {
  // max over the lanes l, l ^ 16, l ^ 32, l ^ 48.
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return lane_pair_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}

__device__ __forceinline__ float quad_rows_sum(float x) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return lane_pair_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

// The visible keys of a sequence: positions j < len with j < sink_end or
// j >= low; its tiles are [0, sink_tiles) and [low / 64, ceil(len / 64)).
struct SeqSpan {
  int len, low, sink_end, sink_tiles, tiles;
  __device__ __forceinline__ int tile(int i) const { return i < sink_tiles ? i : i - sink_tiles + low / kTileKeys; }
};
__device__ __forceinline__ SeqSpan seq_span(const SeqBatch& s, int seq_len) {
  SeqSpan x;
  x.len = max(0, min(seq_len, s.max_len));
  x.low = s.window > 0 ? max(0, x.len - s.window) : 0;
  x.sink_end = min(s.sinks, x.low);
  x.sink_tiles = min((x.sink_end + kTileKeys - 1) / kTileKeys, x.low / kTileKeys);
  x.tiles = x.sink_tiles + (x.len + kTileKeys - 1) / kTileKeys - x.low / kTileKeys;
  return x;
}

__device__ __forceinline__ int wave_total(int x) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) x += __shfl_xor(x, off);
  return x;
}

// Tiles of a part, from the lengths of all sequences; every wavefront makes it
// for itself (4 bytes per sequence, from the L2).
__device__ __forceinline__ int part_tiles(const SeqBatch& s, int lane) {
  int64_t total = 0;
  for (int b0 = 0; b0 < s.batch; b0 += 64) {
    const int b = b0 + lane;
    total += wave_total(b < s.batch ? seq_span(s, s.seq_lens[b]).tiles : 0);
  }
  return max(s.min_tiles, (int)((total + s.target - 1) / s.target));
}

// Item -> (sequence, part): `batch` if there is no such item.
struct SeqPart {
  int seq, part, parts;
  SeqSpan span;
};
__device__ __forceinline__ SeqPart locate_item(const SeqBatch& s, int lane, int item) {
  const int per = part_tiles(s, lane);
  SeqPart r;
  r.seq = s.batch;
  int base = 0;
  for (int b0 = 0; b0 < s.batch; b0 += 64) {
    const int b = b0 + lane;
    const int parts = b < s.batch ? max(1, (seq_span(s, s.seq_lens[b]).tiles + per - 1) / per) : 0;
    int upto = parts;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const int x = __shfl_up(upto, off);
      upto += lane >= off ? x : 0;
    }
    const uint64_t past = __builtin_amdgcn_ballot_w64(item < base + upto);
    if (past != 0) {
      const int at = __builtin_ctzll(past);
      r.seq = b0 + at;
      r.parts = __builtin_amdgcn_readlane(parts, at);
      r.part = item - base - (__builtin_amdgcn_readlane(upto, at) - r.parts);
      r.span = seq_span(s, s.seq_lens[r.seq]);
      return r;
    }
    base += __builtin_amdgcn_readlane(upto, 63);
  }
  return r;
}

// The parts of sequence `seq` and the first one's item.
__device__ __forceinline__ SeqPart parts_of(const SeqBatch& s, int lane, int seq, int* first) {
  const int per = part_tiles(s, lane);
  int base = 0;
  for (int b0 = 0; b0 < seq; b0 += 64) {
    const int b = b0 + lane;
    base += wave_total(b < seq ? max(1, (seq_span(s, s.seq_lens[b]).tiles + per - 1) / per) : 0);
  }
  SeqPart r;
  r.seq = seq;
  r.part = 0;
  r.span = seq_span(s, s.seq_lens[seq]);
  r.parts = max(1, (r.span.tiles + per - 1) / per);
  *first = base;
  return r;
}

// Tiles [begin, end) of a part, counted along the sequence's visible tiles.
__device__ __forceinline__ void part_range(const SeqPart& w, int* begin, int* end) {
  *begin = (int)((int64_t)w.span.tiles * w.part / w.parts);
  *end = (int)((int64_t)w.span.tiles * (w.part + 1) / w.parts);
}

}  // namespace
}  // namespace mocap
