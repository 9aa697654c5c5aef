// A CPU build of the host side of mocap_serve.h (serve_api.cpp) in which every
// launch is recorded and none is made, on a device of 256 compute units.
#include <hip/hip_runtime.h>

#include <cstring>

#include "serve.h"

namespace {
mocap::SeqBatch seqs;
mocap::WindowLaunch window;
mocap::KeyWeightsLaunch weights;
int launches = 0;
}  // namespace

namespace mocap {
hipError_t launch_decode_append(const DecodeAppendLaunch&, int, hipStream_t) { return ++launches, hipSuccess; }
hipError_t launch_decode_attn(const DecodeAttnLaunch& p, int, hipStream_t) {
  seqs = p.seqs;
  return ++launches, hipSuccess;
}
hipError_t launch_window_attn(const WindowLaunch& p, int, hipStream_t) {
  window = p;
  return ++launches, hipSuccess;
}
hipError_t launch_key_weights(const KeyWeightsLaunch& p, int, hipStream_t) {
  weights = p;
  return ++launches, hipSuccess;
}
hipError_t launch_decode_key_weights(const DecodeKeyWeightsLaunch& p, int, hipStream_t) {
  seqs = p.seqs;
  return ++launches, hipSuccess;
}
hipError_t launch_kv_evict(const EvictLaunch&, int, hipStream_t) { return ++launches, hipSuccess; }
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
// How the last batch is cut.
void record_batch(int* out) {
  const int v[] = {seqs.target, seqs.fill,  seqs.min_tiles, seqs.least_tiles,
                   seqs.items,  seqs.window, seqs.sinks,    seqs.max_len};
  for (int i = 0; i < 8; ++i) out[i] = v[i];
}
void record_window(int* out) {
  const int v[] = {window.row_blocks, window.n_ranges, window.total_wgs, window.window, window.sinks};
  for (int i = 0; i < 5; ++i) out[i] = v[i];
}
void record_weights(int* out) {
  const int v[] = {weights.few, weights.key_blocks, weights.row_parts};
  for (int i = 0; i < 3; ++i) out[i] = v[i];
}
void record_weights_cut(int* out) {
  const int v[] = {weights.row_parts, weights.part_tiles, weights.head_wgs};
  for (int i = 0; i < 3; ++i) out[i] = v[i];
}

}  // extern "C"
