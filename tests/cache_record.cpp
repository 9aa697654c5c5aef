// A CPU build of the host side of mocap_cache.h (cache_api.cpp) in which every
// launch is recorded and none is made, on a device of 256 compute units.
#include <hip/hip_runtime.h>

#include <cstring>

#include "cache.h"

namespace {
mocap::RopeAppendLaunch append;
mocap::Kv4ChunkLaunch chunk;
bool few = false;
mocap::SeqBatch seqs;
int row_blocks = 0;
int launches = 0;
}  // namespace

namespace mocap {
hipError_t launch_rope_append(const RopeAppendLaunch& p, int, hipStream_t) {
  append = p;
  return ++launches, hipSuccess;
}
hipError_t launch_decode_rope_append(const RopeAppendLaunch& p, int, hipStream_t) {
  append = p;
  return ++launches, hipSuccess;
}
hipError_t launch_kv4_load(const Kv4LoadLaunch&, int, hipStream_t) { return ++launches, hipSuccess; }
hipError_t launch_kv4_decode(const Kv4DecodeLaunch& p, int, hipStream_t) {
  seqs = p.a.seqs;
  row_blocks = p.a.row_blocks;
  return ++launches, hipSuccess;
}
hipError_t launch_kv4_chunk(const Kv4ChunkLaunch& p, int, hipStream_t) {
  chunk = p;
  few = false;
  return ++launches, hipSuccess;
}
hipError_t launch_kv4_few_rows(const Kv4ChunkLaunch& p, int, hipStream_t) {
  chunk = p;
  few = true;
  return ++launches, hipSuccess;
}
hipError_t launch_lse_merge(const MergeLaunch&, int, hipStream_t) { return ++launches, hipSuccess; }
}  // namespace mocap

extern "C" {

hipError_t hipGetDevice(int* dev) {
  *dev = 0;
  return hipSuccess;
}
hipError_t hipDeviceGetAttribute(int* value, hipDeviceAttribute_t, int) {
  *value = 256;
  return hipSuccess;
}
hipError_t hipMemcpy(void* dst, const void* src, size_t bytes, hipMemcpyKind) {
  std::memcpy(dst, src, bytes);
  return hipSuccess;
}

int record_launches() { return launches; }
int record_row_blocks() { return row_blocks; }
void record_append(long long* out) {
  const long long v[] = {append.rot, append.interleaved, append.h_q, append.h_kv, append.q_stride, append.k_stride,
                         append.v_stride, append.start_pos, append.first_pos, append.chunk_len,
                         append.pools.k_scale != nullptr};
  for (int i = 0; i < 11; ++i) out[i] = v[i];
}
void record_chunk(int* out) {
  const int v[] = {chunk.a.row_blocks, chunk.a.n_ranges, chunk.a.total_wgs, chunk.a.window, chunk.a.sinks, chunk.mirrored,
                   few};
  for (int i = 0; i < 7; ++i) out[i] = v[i];
}
void record_batch(int* out) {
  const int v[] = {seqs.target, seqs.fill,  seqs.min_tiles, seqs.least_tiles,
                   seqs.items,  seqs.window, seqs.sinks,    seqs.max_len};
  for (int i = 0; i < 8; ++i) out[i] = v[i];
}

}  // extern "C"
