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

// Inclusive sums over the wavefront's lanes, with data-parallel moves: within
// rows of 16 lanes, then from the row before and the half before.
template <int kMove, int kRows>
__device__ __forceinline__ int add_moved(int x) {
  return x + __builtin_amdgcn_update_dpp(0, x, kMove, kRows, 0xF, false);
}
__device__ __forceinline__ int wave_sums(int x) {
  x = add_moved<0x111, 0xF>(x);  // row_shr:1, 2, 4, 8
  x = add_moved<0x112, 0xF>(x);
  x = add_moved<0x114, 0xF>(x);
  x = add_moved<0x118, 0xF>(x);
  x = add_moved<0x142, 0xA>(x);  // row_bcast:15 to rows 1 and 3
  return add_moved<0x143, 0xC>(x);  // row_bcast:31 to rows 2 and 3
}

// The same in fp32 (in a fixed order), and the maximum; of all lanes, in every lane.
template <int kMove, int kRows>
__device__ __forceinline__ float moved(float x, float none) {
  return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(none), __float_as_int(x), kMove, kRows, 0xF, false));
}
__device__ __forceinline__ float wave_total(float x) {
  x += moved<0x111, 0xF>(x, 0.f);
  x += moved<0x112, 0xF>(x, 0.f);
  x += moved<0x114, 0xF>(x, 0.f);
  x += moved<0x118, 0xF>(x, 0.f);
  x += moved<0x142, 0xA>(x, 0.f);
  x += moved<0x143, 0xC>(x, 0.f);
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}
__device__ __forceinline__ float wave_largest(float x) {
  x = fmaxf(x, moved<0x111, 0xF>(x, x));
  x = fmaxf(x, moved<0x112, 0xF>(x, x));
  x = fmaxf(x, moved<0x114, 0xF>(x, x));
  x = fmaxf(x, moved<0x118, 0xF>(x, x));
  x = fmaxf(x, moved<0x142, 0xA>(x, x));
  x = fmaxf(x, moved<0x143, 0xC>(x, x));
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}

// Tiles of a part, from the lengths of all sequences; every wavefront makes it
// for itself (4 bytes per sequence, from the L2).
__device__ __forceinline__ int part_tiles(const SeqBatch& s, int lane) {
  float t = 0.f;
  for (int b0 = 0; b0 < s.batch; b0 += 64) {
    const int b = b0 + lane;
    // At most 2^25 tiles a sequence: 64 of them fit.
    const int sums = wave_sums(b < s.batch ? seq_span(s, s.seq_lens[b]).tiles : 0);
    t += (float)(uint32_t)__builtin_amdgcn_readlane(sums, 63);
  }
  // (Floating point: no 64-bit division; a tile more or less in a part is no matter,
  // but a part must not have fewer than total / target.)
  const int few = min(s.min_tiles, max(s.least_tiles, (int)(t / (float)s.fill) + 1));
  return max(few, (int)(t * 1.000001f / (float)s.target) + 1);
}

__device__ __forceinline__ int parts_for(int tiles, int per) { return max(1, (tiles + per - 1) / per); }

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
    const int len = b < s.batch ? s.seq_lens[b] : 0;
    const int parts = b < s.batch ? parts_for(seq_span(s, len).tiles, per) : 0;
    const int upto = wave_sums(parts);
    const uint64_t past = __builtin_amdgcn_ballot_w64(item < base + upto);
    if (past != 0) {
      const int at = __builtin_ctzll(past);
      r.seq = b0 + at;
      r.parts = __builtin_amdgcn_readlane(parts, at);
      r.part = item - base - (__builtin_amdgcn_readlane(upto, at) - r.parts);
      r.span = seq_span(s, __builtin_amdgcn_readlane(len, at));
      return r;
    }
    base += __builtin_amdgcn_readlane(upto, 63);
  }
  return r;
}

// The parts of sequence `seq` and the first one's item.
__device__ __forceinline__ SeqPart parts_of(const SeqBatch& s, int lane, int seq, int* first) {
  const int per = part_tiles(s, lane);
  SeqPart r;
  r.seq = seq;
  r.part = 0;
  int base = 0;
  for (int b0 = 0; b0 <= seq; b0 += 64) {
    const int b = b0 + lane;
    const int len = b <= seq ? s.seq_lens[b] : 0;
    const int upto = wave_sums(b < seq ? parts_for(seq_span(s, len).tiles, per) : 0);
    base += __builtin_amdgcn_readlane(upto, 63);
    if (seq - b0 < 64) r.span = seq_span(s, __builtin_amdgcn_readlane(len, seq - b0));
  }
  r.parts = parts_for(r.span.tiles, per);
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
