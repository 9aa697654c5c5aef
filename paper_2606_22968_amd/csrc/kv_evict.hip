// Eviction by weight for gfx950 (CDNA4): which positions each KV head keeps, and
// their compaction into other blocks.
//
// Selection: the positions between the sinks and the recent ones are candidates,
// c of them stay.  A weight becomes a 32-bit key whose unsigned order is the
// order of the weights (NaN the largest, -0 as 0); the c-th largest key is found
// digit by digit from histograms of the candidates that share the digits found
// so far; keys above it stay, and of those equal to it the first ones.  Counts
// are integers, so the result does not depend on the order of the atomics.
#include "attn_device.h"
#include "serve.h"

namespace mocap {
namespace {

constexpr int kSelectThreads = 1024;
constexpr int kSelectWaves = kSelectThreads / 64;
constexpr int kBins = 256;

__device__ __forceinline__ uint32_t weight_key(float w) {
  if (w != w) return 0xFFFFFFFFu;
  const uint32_t x = __float_as_uint(w == 0.f ? 0.f : w);
  return x >> 31 ? ~x : x | 0x80000000u;
}

__global__ __launch_bounds__(kSelectThreads) void evict_select_kernel(const EvictLaunch p) {
  __shared__ uint32_t hist[kBins];
  __shared__ uint32_t digit_s, left_s;
  __shared__ uint32_t counts[2][kSelectWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int h = blockIdx.x;
  const float* w = p.weights + h * p.weight_stride;
  const int first = p.sinks, end = p.n - p.recent;  // candidates [first, end)
  uint32_t left = (uint32_t)(p.keep - p.sinks - p.recent);  // still to be found among those with this prefix
  uint32_t prefix = 0;
  // Digit by digit, the highest first.  With nothing or everything to keep the
  // border is found all the same, and `left` of the keys equal to it stay.
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = tid; i < kBins; i += kSelectThreads) hist[i] = 0;
    __syncthreads();
    for (int i = first + tid; i < end; i += kSelectThreads) {
      const uint32_t k = weight_key(w[i]);
      if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[k >> shift & (kBins - 1)], 1u);
    }
    __syncthreads();
    if (wave == 0) {
      // Lane l holds bins 255 - 4 l .. 252 - 4 l; counts above them by a scan.
      uint32_t c[4], sum = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) sum += c[j] = hist[kBins - 1 - 4 * lane - j];
      uint32_t upto = sum;
#pragma unroll
      for (int off = 1; off < 64; off <<= 1) {
        const uint32_t x = __shfl_up(upto, off);
        upto += lane >= off ? x : 0;
      }
      uint32_t above = upto - sum;
      // The bin that holds the left-th largest (left >= 1); with left = 0 none is needed.
      if (left > above && left <= upto) {
        for (int j = 0; j < 4; ++j) {
          if (left <= above + c[j]) {
            digit_s = kBins - 1 - 4 * lane - j;
            left_s = left - above;
            break;
          }
          above += c[j];
        }
      } else if (left == 0 && lane == 0) {
        digit_s = kBins - 1;
        left_s = 0;
      }
    }
    __syncthreads();
    prefix |= digit_s << shift;
    left = left_s;
    __syncthreads();
  }

  // Kept positions in order: sinks, candidates, recent ones.
  int32_t* kept = p.kept + (int64_t)h * p.keep;
  float* kept_w = p.kept_weights ? p.kept_weights + (int64_t)h * p.keep : nullptr;
  auto put = [&](int at, int pos) {
    kept[at] = pos;
    if (kept_w) kept_w[at] = w[pos];
  };
  for (int i = tid; i < p.sinks; i += kSelectThreads) put(i, i);
  for (int i = tid; i < p.recent; i += kSelectThreads) put(p.keep - p.recent + i, end + i);
  uint32_t equal_before = 0;
  int at0 = p.sinks;
  const uint64_t below = (1ull << lane) - 1;
  for (int i0 = first; i0 < end; i0 += kSelectThreads) {
    const int i = i0 + tid;
    const uint32_t k = i < end ? weight_key(w[i]) : 0;
    const bool equal = i < end && k == prefix;
    const uint64_t eq = __builtin_amdgcn_ballot_w64(equal);
    if (lane == 0) counts[0][wave] = __builtin_popcountll(eq);
    __syncthreads();
    uint32_t eq_at = equal_before + __builtin_popcountll(eq & below), eq_all = 0;
    for (int x = 0; x < kSelectWaves; ++x) {
      eq_at += x < wave ? counts[0][x] : 0;
      eq_all += counts[0][x];
    }
    const bool stays = i < end && (k > prefix || (equal && eq_at < left));
    const uint64_t st = __builtin_amdgcn_ballot_w64(stays);
    if (lane == 0) counts[1][wave] = __builtin_popcountll(st);
    __syncthreads();
    uint32_t at = __builtin_popcountll(st & below), all = 0;
    for (int x = 0; x < kSelectWaves; ++x) {
      at += x < wave ? counts[1][x] : 0;
      all += counts[1][x];
    }
    if (stays) put(at0 + at, i);
    at0 += all;
    equal_before += eq_all;
  }
}

// Copies the kept positions' keys and values: one workgroup per 64 positions of
// dst and KV head.  A kept key is one row; a kept value's dims are spread over as
// many rows of V, where neighbouring kept positions share lines.
template <int D>
__global__ __launch_bounds__(256) void evict_copy_kernel(const EvictLaunch p) {
  constexpr int T = 64, CHUNKS = D / 8;
  __shared__ int64_t src_block[T];  // first element of the source block's head, K and V alike
  __shared__ int src_slot[T];
  const int tid = threadIdx.x, h = blockIdx.y;
  const int pos0 = blockIdx.x * T;
  const int count = min(T, p.keep - pos0);
  if (tid < count) {
    const int pos = p.kept[(int64_t)h * p.keep + pos0 + tid];
    const int lb = pos / p.src_block_size;
    src_block[tid] = ((int64_t)p.src_table[lb] * p.h_kv + h) * D * p.src_block_size;
    src_slot[tid] = pos - lb * p.src_block_size;
  }
  __syncthreads();
  const int lb = pos0 / p.dst_block_size;  // 64 positions lie in one block
  const int slot0 = pos0 - lb * p.dst_block_size;
  const int64_t dst = ((int64_t)p.dst_table[lb] * p.h_kv + h) * D * p.dst_block_size;
#pragma unroll 4
  for (int i = tid; i < count * CHUNKS; i += 256) {
    const int r = i / CHUNKS, c = i % CHUNKS;
    *reinterpret_cast<u32x4*>(p.k_dst + dst + (int64_t)(slot0 + r) * D + c * 8) =
        *reinterpret_cast<const u32x4*>(p.k_src + src_block[r] + (int64_t)src_slot[r] * D + c * 8);
  }
  const int r = tid & (T - 1), e0 = tid / T;
  if (r >= count) return;
  const uint16_t* v = p.v_src + src_block[r] + src_slot[r];
  uint16_t* o = p.v_dst + dst + slot0 + r;
#pragma unroll 16
  for (int e = e0; e < D; e += 256 / T) o[(int64_t)e * p.dst_block_size] = v[(int64_t)e * p.src_block_size];
}

}  // namespace

hipError_t launch_kv_evict(const EvictLaunch& p, int head_dim, hipStream_t stream) {
  hipLaunchKernelGGL(evict_select_kernel, dim3(p.h_kv), dim3(kSelectThreads), 0, stream, p);
  const dim3 grid((p.keep + 63) / 64, p.h_kv), block(256);
  if (head_dim == 128) {
    hipLaunchKernelGGL(evict_copy_kernel<128>, grid, block, 0, stream, p);
  } else {
    hipLaunchKernelGGL(evict_copy_kernel<64>, grid, block, 0, stream, p);
  }
  return hipGetLastError();
}

}  // namespace mocap
