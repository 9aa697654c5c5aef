// Eviction by weight for gfx950 (CDNA4): which positions each KV head keeps, and
// their compaction into other blocks.
//
// Selection: the positions between the sinks and the recent ones are candidates,
// c of them stay.  A weight becomes a 32-bit key whose unsigned order is the
// order of the weights (NaN the largest, -0 as 0); the c-th largest key (the
// border) is found digit by digit, 10, 12 and 10 bits, from histograms of the
// candidates that have the digits found so far; keys above it stay, and of those
// equal to it the first ones.  Counts are integers, so the result does not depend
// on the order of the atomics.
//
// Up to kEvictOneGroup candidates are held by one workgroup per head, which needs one
// launch (8 heads of 128, 100 of 16384 positions kept: 17 us in all, 26 in chunks);
// more are cut into chunks, in four launches, which is what a workgroup's registers
// ask for (131072 positions: 27 of 101 us, bound by four chains of launch, load and
// count; 8, 16, 32 and 64 chunks: 43, 34, 31 and 32 us with 256 kept).  Up to 4096
// candidates a workgroup holds four a thread instead of sixteen (13.3 us and 16.0).
//
// Bounds: the copy by HBM, not by the bytes that stay but by the lines they lie in.
// A value's dim lies in a line with 63 other positions', so at a share of 1/8 nearly
// every line of V is read: 131072 positions to 16384, 8 heads of 128: 369 MB in
// 75 us, 4.9 TB/s.
#include "attn_device.h"
#include "serve.h"

#include <type_traits>

namespace mocap {
namespace {

constexpr int kSelectThreads = 1024;
constexpr int kSelectWaves = kSelectThreads / 64;
constexpr int kDigitBits[3] = {10, 12, 10}, kDigitShift[3] = {22, 10, 0};
constexpr int kMostBins = 4096;
constexpr int bins(int d) { return 1 << kDigitBits[d]; }

__device__ __forceinline__ uint32_t weight_key(float w) {
  if (w != w) return 0xFFFFFFFFu;
  const uint32_t x = __float_as_uint(w == 0.f ? 0.f : w);
  return x >> 31 ? ~x : x | 0x80000000u;
}

// Whether a key has the digits before digit d of the border found so far.
template <int d>
__device__ __forceinline__ bool in_prefix(uint32_t key, uint32_t prefix) {
  if constexpr (d == 0) {
    return true;
  } else {
    return (key ^ prefix) >> kDigitShift[d - 1] == 0;
  }
}
template <int d>
__device__ __forceinline__ uint32_t digit_of(uint32_t key) {
  return key >> kDigitShift[d] & (bins(d) - 1);
}

// `left` of the candidates with the digits in `prefix` stay.
struct Border {
  uint32_t prefix, left;
};

// Adds digit d: the bin that holds the left-th largest of those candidates,
// count(bin) being their histogram.  Every thread calls it and gets the result;
// with left = 0 it is the highest digit, so that no key lies above the border.
template <int d, class Count>
__device__ __forceinline__ void find_digit(Count count, Border& x) {
  constexpr int EACH = bins(d) / kSelectThreads;
  __shared__ uint32_t totals[kSelectWaves], found[2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int top = bins(d) - 1 - EACH * tid;  // this thread's bins, downwards
  uint32_t c[EACH], sum = 0;
#pragma unroll
  for (int j = 0; j < EACH; ++j) sum += c[j] = count(top - j);
  uint32_t upto = sum;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const uint32_t y = __shfl_up(upto, off);
    upto += lane >= off ? y : 0;
  }
  if (lane == 63) totals[wave] = upto;
  if (tid == 0) {
    found[0] = bins(d) - 1;
    found[1] = 0;
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kSelectWaves; ++w) upto += w < wave ? totals[w] : 0;
  uint32_t above = upto - sum;
  if (x.left > above && x.left <= upto) {
#pragma unroll
    for (int j = 0; j < EACH; ++j) {
      if (x.left > above && x.left <= above + c[j]) {
        found[0] = top - j;
        found[1] = x.left - above;
      }
      above += c[j];
    }
  }
  __syncthreads();
  x.prefix |= found[0] << kDigitShift[d];
  x.left = found[1];
  __syncthreads();
}

struct Output {
  int32_t* kept;
  float* kept_weights;
  __device__ __forceinline__ void put(int at, int pos, float w) const {
    kept[at] = pos;
    if (kept_weights) kept_weights[at] = w;
  }
};
__device__ __forceinline__ Output output_of(const EvictLaunch& p, int h) {
  return Output{p.kept + (int64_t)h * p.keep, p.kept_weights ? p.kept_weights + (int64_t)h * p.keep : nullptr};
}
__device__ __forceinline__ void put_always_kept(const EvictLaunch& p, const Output& out, const float* w, int64_t first,
                                                int64_t step) {
  for (int64_t i = first; i < p.sinks; i += step) out.put((int)i, (int)i, w[i]);
  for (int64_t i = first; i < p.recent; i += step) {
    const int pos = p.n - p.recent + (int)i;
    out.put(p.keep - p.recent + (int)i, pos, w[pos]);
  }
}

// Writes those that stay of 1024 ROUNDS consecutive candidates, in order:
// candidate r 1024 + tid is key[r], w[r] at position pos0 + r 1024 + tid, the
// first `count` exist.  above and equal: how many candidates above the border and
// equal to it have come before; moved on by this call.  The candidates that stay
// have the output positions at0 .. at0 + stay - 1, and nothing is written elsewhere:
// in several launches each reads the weights anew, and weights that someone writes to
// meanwhile can put more candidates above the border than were counted.
template <int ROUNDS>
__device__ __forceinline__ void compact(const uint32_t (&key)[ROUNDS], const float (&w)[ROUNDS], int pos0, int count,
                                        const Border& border, int at0, uint32_t stay, uint32_t& above, uint32_t& equal,
                                        const Output& out) {
  constexpr int SLOTS = ROUNDS * kSelectWaves;
  static_assert(SLOTS <= kSelectThreads, "a thread for every (round, wave)");
  __shared__ uint32_t above_n[SLOTS + 1], equal_n[SLOTS + 1], totals[2][kSelectWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const uint64_t below = (1ull << lane) - 1;
  // Counts of every (round, wave), then the sums before each.
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r) {
    const bool live = r * kSelectThreads + tid < count;
    const uint64_t gt = __builtin_amdgcn_ballot_w64(live && key[r] > border.prefix);
    const uint64_t eq = __builtin_amdgcn_ballot_w64(live && key[r] == border.prefix);
    if (lane == 0) {
      above_n[r * kSelectWaves + wave] = __builtin_popcountll(gt);
      equal_n[r * kSelectWaves + wave] = __builtin_popcountll(eq);
    }
  }
  __syncthreads();
  const uint32_t a0 = tid < SLOTS ? above_n[tid] : 0, b0 = tid < SLOTS ? equal_n[tid] : 0;
  uint32_t a = a0, b = b0;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const uint32_t y = __shfl_up(a, off), z = __shfl_up(b, off);
    a += lane >= off ? y : 0;
    b += lane >= off ? z : 0;
  }
  if (lane == 63) {
    totals[0][wave] = a;
    totals[1][wave] = b;
  }
  __syncthreads();
#pragma unroll
  for (int x = 0; x < kSelectWaves; ++x) {
    a += x < wave ? totals[0][x] : 0;
    b += x < wave ? totals[1][x] : 0;
  }
  if (tid < SLOTS) {
    above_n[tid] = a - a0;
    equal_n[tid] = b - b0;
  }
  if (tid == kSelectThreads - 1) {
    above_n[SLOTS] = a;
    equal_n[SLOTS] = b;
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r) {
    const int i = r * kSelectThreads + tid;
    const bool live = i < count;
    const bool gt = live && key[r] > border.prefix, eq = live && key[r] == border.prefix;
    const uint32_t gt_at = above + above_n[r * kSelectWaves + wave] + __builtin_popcountll(__builtin_amdgcn_ballot_w64(gt) & below);
    const uint32_t eq_at = equal + equal_n[r * kSelectWaves + wave] + __builtin_popcountll(__builtin_amdgcn_ballot_w64(eq) & below);
    // Of the equal ones the first `left` stay.
    const uint32_t at = gt_at + min(eq_at, border.left);
    if ((gt || (eq && eq_at < border.left)) && at < stay) out.put(at0 + (int)at, pos0 + i, w[r]);
  }
  above += above_n[SLOTS];
  equal += equal_n[SLOTS];
  __syncthreads();
}

// ---- One workgroup per head ----
template <int ROUNDS>
__global__ __launch_bounds__(kSelectThreads) void evict_select_kernel(const EvictLaunch p) {
  __shared__ uint32_t hist[kMostBins];
  const int tid = threadIdx.x, h = blockIdx.x;
  const float* w = p.weights + h * p.weight_stride;
  const int first = p.sinks, count = p.n - p.recent - p.sinks;
  float x[ROUNDS];
  uint32_t key[ROUNDS];
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r) {
    const int i = r * kSelectThreads + tid;
    x[r] = i < count ? w[first + i] : 0.f;
  }
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r) key[r] = weight_key(x[r]);
  const Output out = output_of(p, h);
  put_always_kept(p, out, w, tid, kSelectThreads);
  const uint32_t stay = p.keep - p.sinks - p.recent;
  Border border{0, stay};
  auto digit = [&](auto dd) __attribute__((always_inline)) {
    constexpr int d = decltype(dd)::value;
    for (int i = tid; i < bins(d); i += kSelectThreads) hist[i] = 0;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r)
      if (r * kSelectThreads + tid < count && in_prefix<d>(key[r], border.prefix)) atomicAdd(&hist[digit_of<d>(key[r])], 1u);
    __syncthreads();
    find_digit<d>([&](int bin) { return hist[bin]; }, border);
  };
  digit(std::integral_constant<int, 0>());
  digit(std::integral_constant<int, 1>());
  digit(std::integral_constant<int, 2>());
  uint32_t above = 0, equal = 0;
  compact<ROUNDS>(key, x, first, count, border, p.sinks, stay, above, equal, out);
}

// ---- p.chunks workgroups per head ----
// Each takes an even run of the candidates.  Every launch finds the digit that
// the one before has counted, every workgroup for itself (it reads 128 KiB at
// most, from the L2), and counts the next.  The first and the last digit are
// counted per chunk, so nothing needs clearing beforehand and the last launch
// knows how many of the chunks before its own stay; the second is counted with
// atomics in memory that the first launch clears.
struct ChunkCounts {  // of one head
  uint32_t* first;    // [chunks][bins(0)]
  uint32_t* second;   // [bins(1)]
  uint32_t* third;    // [chunks][bins(2)]
  uint32_t* above;    // [chunks]: candidates above the first two digits of the border
  uint32_t* border;   // prefix and left behind the first, then the second digit
};
__device__ __forceinline__ ChunkCounts counts_of(const EvictLaunch& p, int h) {
  uint32_t* x = p.ws + (int64_t)h * evict_head_words(p.chunks);
  ChunkCounts c;
  c.first = x;
  c.second = c.first + p.chunks * bins(0);
  c.third = c.second + bins(1);
  c.above = c.third + p.chunks * bins(2);
  c.border = c.above + p.chunks;
  return c;
}
static_assert(bins(0) == kEvictFirstBins && bins(1) == kEvictSecondBins && bins(2) == kEvictThirdBins, "workspace layout");

struct Chunk {
  const float* w;  // of candidate 0
  int begin, end;  // its candidates
};
__device__ __forceinline__ Chunk chunk_of(const EvictLaunch& p, int h, int chunk) {
  const int64_t all = p.n - p.recent - p.sinks;
  return Chunk{p.weights + h * p.weight_stride + p.sinks, (int)(all * chunk / p.chunks), (int)(all * (chunk + 1) / p.chunks)};
}

// A thread's candidates of a chunk, in batches whose loads are all in flight: first()
// asks for the first batch (before other work, where there is some), each() hands
// every candidate's key to f.  (Loaded one by one: 70 instead of 63 us for 8
// heads of 500000 positions, of which the copy takes 25.)
struct Batches {
  static constexpr int ROUNDS = 8;
  const Chunk& x;
  int tid;
  float w[ROUNDS];
  __device__ __forceinline__ Batches(const Chunk& chunk, int thread) : x(chunk), tid(thread) {}
  __device__ __forceinline__ void load(int i0) {
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
      const int i = r * kSelectThreads + tid;
      w[r] = i < x.end - i0 ? x.w[i0 + i] : 0.f;
    }
  }
  __device__ __forceinline__ void first() { load(x.begin); }
  template <class F>
  __device__ __forceinline__ void each(F f) {
    for (int i0 = x.begin; i0 < x.end; i0 += ROUNDS * kSelectThreads) {
      uint32_t key[ROUNDS];
#pragma unroll
      for (int r = 0; r < ROUNDS; ++r) key[r] = weight_key(w[r]);
      const int count = x.end - i0;
      if (count > ROUNDS * kSelectThreads) load(i0 + ROUNDS * kSelectThreads);
#pragma unroll
      for (int r = 0; r < ROUNDS; ++r)
        if (r * kSelectThreads + tid < count) f(key[r]);
    }
  }
};

__global__ __launch_bounds__(kSelectThreads) void evict_first_kernel(const EvictLaunch p) {
  __shared__ uint32_t hist[bins(0)];
  const int tid = threadIdx.x, chunk = blockIdx.x, h = blockIdx.y;
  const ChunkCounts c = counts_of(p, h);
  const Chunk x = chunk_of(p, h, chunk);
  Batches batches(x, tid);
  batches.first();
  hist[tid] = 0;
  if (chunk == 0)
    for (int i = tid; i < bins(1); i += kSelectThreads) c.second[i] = 0;
  put_always_kept(p, output_of(p, h), x.w - p.sinks, (int64_t)chunk * kSelectThreads + tid,
                  (int64_t)p.chunks * kSelectThreads);
  __syncthreads();
  batches.each([&](uint32_t key) { atomicAdd(&hist[digit_of<0>(key)], 1u); });
  __syncthreads();
  c.first[chunk * bins(0) + tid] = hist[tid];
}
static_assert(bins(0) == kSelectThreads && bins(2) == kSelectThreads, "a thread per bin of the first and last digit");

__global__ __launch_bounds__(kSelectThreads) void evict_second_kernel(const EvictLaunch p) {
  __shared__ uint32_t hist[bins(1)];
  const int tid = threadIdx.x, chunk = blockIdx.x, h = blockIdx.y;
  const ChunkCounts c = counts_of(p, h);
  const Chunk x = chunk_of(p, h, chunk);
  Batches batches(x, tid);
  for (int i = tid; i < bins(1); i += kSelectThreads) hist[i] = 0;
  Border border{0, (uint32_t)(p.keep - p.sinks - p.recent)};
  find_digit<0>([&](int bin) {
    uint32_t v[kEvictMaxChunks], sum = 0;  // all loads in flight
#pragma unroll
    for (int y = 0; y < kEvictMaxChunks; ++y) v[y] = y < p.chunks ? c.first[y * bins(0) + bin] : 0;
    batches.first();
#pragma unroll
    for (int y = 0; y < kEvictMaxChunks; ++y) sum += v[y];
    return sum;
  }, border);
  if (chunk == 0 && tid == 0) {
    c.border[0] = border.prefix;
    c.border[1] = border.left;
  }
  batches.each([&](uint32_t key) {
    if (in_prefix<1>(key, border.prefix)) atomicAdd(&hist[digit_of<1>(key)], 1u);
  });
  __syncthreads();
  for (int i = tid; i < bins(1); i += kSelectThreads)
    if (hist[i] != 0) atomicAdd(&c.second[i], hist[i]);
}

__global__ __launch_bounds__(kSelectThreads) void evict_third_kernel(const EvictLaunch p) {
  __shared__ uint32_t hist[bins(2)], above_s;
  const int tid = threadIdx.x, chunk = blockIdx.x, h = blockIdx.y;
  const ChunkCounts c = counts_of(p, h);
  const Chunk x = chunk_of(p, h, chunk);
  Batches batches(x, tid);
  batches.first();
  hist[tid] = 0;
  if (tid == 0) above_s = 0;
  Border border{c.border[0], c.border[1]};
  find_digit<1>([&](int bin) { return c.second[bin]; }, border);
  if (chunk == 0 && tid == 0) {
    c.border[2] = border.prefix;
    c.border[3] = border.left;
  }
  uint32_t above = 0;
  batches.each([&](uint32_t key) {
    if (in_prefix<2>(key, border.prefix)) {
      atomicAdd(&hist[digit_of<2>(key)], 1u);
    } else {
      above += key > border.prefix;
    }
  });
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) above += __shfl_xor(above, off);
  if ((tid & 63) == 0) atomicAdd(&above_s, above);
  __syncthreads();
  c.third[chunk * bins(2) + tid] = hist[tid];
  if (tid == 0) c.above[chunk] = above_s;
}

__global__ __launch_bounds__(kSelectThreads) void evict_compact_kernel(const EvictLaunch p) {
  constexpr int ROUNDS = 4;
  __shared__ uint32_t above_s, equal_s;
  const int tid = threadIdx.x, chunk = blockIdx.x, h = blockIdx.y;
  const ChunkCounts c = counts_of(p, h);
  const Chunk x = chunk_of(p, h, chunk);
  if (tid == 0) above_s = equal_s = 0;
  // Thread t looks at bin 1023 - t: in all chunks, and in those before this one.
  const int bin = bins(2) - 1 - tid;
  uint32_t counts[kEvictMaxChunks], sum = 0, before = 0;
#pragma unroll
  for (int y = 0; y < kEvictMaxChunks; ++y) counts[y] = y < p.chunks ? c.third[y * bins(2) + bin] : 0;
  Border border{c.border[2], c.border[3]};
  float w[ROUNDS];
  auto load = [&](int i0) __attribute__((always_inline)) {
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
      const int i = r * kSelectThreads + tid;
      w[r] = i < x.end - i0 ? x.w[i0 + i] : 0.f;
    }
  };
  load(x.begin);
#pragma unroll
  for (int y = 0; y < kEvictMaxChunks; ++y) {
    sum += counts[y];
    before += y < chunk ? counts[y] : 0;
  }
  find_digit<2>([&](int) { return sum; }, border);
  const int digit = (int)digit_of<2>(border.prefix);
  uint32_t above = bin > digit ? before : 0;
  for (int y = tid; y < chunk; y += kSelectThreads) above += c.above[y];
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) above += __shfl_xor(above, off);
  if ((tid & 63) == 0) atomicAdd(&above_s, above);
  if (bin == digit) equal_s = before;
  __syncthreads();
  above = above_s;
  uint32_t equal = equal_s;
  const Output out = output_of(p, h);
  for (int i0 = x.begin; i0 < x.end; i0 += ROUNDS * kSelectThreads) {
    uint32_t key[ROUNDS];
    const int count = min(x.end - i0, ROUNDS * kSelectThreads);
    float now[ROUNDS];
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
      now[r] = w[r];
      key[r] = weight_key(w[r]);
    }
    if (i0 + ROUNDS * kSelectThreads < x.end) load(i0 + ROUNDS * kSelectThreads);
    compact<ROUNDS>(key, now, p.sinks + i0, count, border, p.sinks, p.keep - p.sinks - p.recent, above, equal, out);
  }
}

// ---- Copy ----
// One workgroup per 64 positions of dst, KV head and D / 32-th of the work: a kept key
// is one row, of which a workgroup copies whole ones (all keys' 32 dims instead, which
// reads and writes every line in pieces at different times: 110.8 and 101.5 us for
// 131072 positions to 16384, 206 and 164 to 65536); a kept value's dims lie in as many
// rows of V, where neighbouring kept positions share lines: a wavefront takes one dim
// of the 64 positions at a time, the workgroup 32 dims.  Giving neighbouring
// positions, which share lines, to one XCD changes nothing (102, 168 us).
template <int D>
__global__ __launch_bounds__(256) void evict_copy_kernel(const EvictLaunch p) {
  constexpr int T = 64, DIMS = 32;
  const int tid = threadIdx.x, h = blockIdx.y, dim0 = blockIdx.z * DIMS;
  const int pos0 = blockIdx.x * T;
  const int count = min(T, p.keep - pos0);
  const int32_t* kept = p.kept + (int64_t)h * p.keep + pos0;
  auto source = [&](int r, int* slot) __attribute__((always_inline)) {  // first element of the block's head
    // (In range also where the weights were written to while positions were chosen.)
    const int pos = max(0, min(kept[min(r, count - 1)], p.n - 1));
    const int lb = pos / p.src_block_size;
    *slot = pos - lb * p.src_block_size;
    return ((int64_t)p.src_table[lb] * p.h_kv + h) * D * p.src_block_size;
  };
  const int lb = pos0 / p.dst_block_size;  // 64 positions lie in one block
  const int slot0 = pos0 - lb * p.dst_block_size;
  const int64_t dst = ((int64_t)p.dst_table[lb] * p.h_kv + h) * D * p.dst_block_size;
  const int kr = blockIdx.z * (DIMS * T / D) + tid / (D / 8), kc = tid % (D / 8) * 8;  // K: row and first dim
  const int vr = tid & (T - 1), ve = dim0 + tid / T;                  // V: position and first dim, 4 apart
  int k_slot, v_slot;
  const uint16_t* k = p.k_src + source(kr, &k_slot);
  const uint16_t* v = p.v_src + source(vr, &v_slot) + v_slot;
  const u32x4 key = *reinterpret_cast<const u32x4*>(k + (int64_t)k_slot * D + kc);
  uint16_t value[DIMS / 4];
#pragma unroll
  for (int i = 0; i < DIMS / 4; ++i) value[i] = v[(int64_t)(ve + 4 * i) * p.src_block_size];
  if (kr < count) *reinterpret_cast<u32x4*>(p.k_dst + dst + (int64_t)(slot0 + kr) * D + kc) = key;
  if (vr < count) {
#pragma unroll
    for (int i = 0; i < DIMS / 4; ++i) p.v_dst[dst + (int64_t)(ve + 4 * i) * p.dst_block_size + slot0 + vr] = value[i];
  }
}

template <int D>
void launch_copy(const EvictLaunch& p, hipStream_t stream) {
  hipLaunchKernelGGL(evict_copy_kernel<D>, dim3((p.keep + 63) / 64, p.h_kv, D / 32), dim3(256), 0, stream, p);
}

}  // namespace

hipError_t launch_kv_evict(const EvictLaunch& p, int head_dim, hipStream_t stream) {
  const dim3 block(kSelectThreads);
  const int candidates = p.n - p.sinks - p.recent;
  if (p.chunks > 0) {
    const dim3 grid(p.chunks, p.h_kv);
    hipLaunchKernelGGL(evict_first_kernel, grid, block, 0, stream, p);
    hipLaunchKernelGGL(evict_second_kernel, grid, block, 0, stream, p);
    hipLaunchKernelGGL(evict_third_kernel, grid, block, 0, stream, p);
    hipLaunchKernelGGL(evict_compact_kernel, grid, block, 0, stream, p);
  } else if (candidates <= 4 * kSelectThreads) {
    hipLaunchKernelGGL(evict_select_kernel<4>, dim3(p.h_kv), block, 0, stream, p);
  } else {
    hipLaunchKernelGGL(evict_select_kernel<kEvictOneGroup / kSelectThreads>, dim3(p.h_kv), block, 0, stream, p);
  }
  if (head_dim == 128) {
    launch_copy<128>(p, stream);
  } else {
    launch_copy<64>(p, stream);
  }
  return hipGetLastError();
}

}  // namespace mocap
