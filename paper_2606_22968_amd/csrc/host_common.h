// Argument checks and small host helpers shared by the library's entry points.
#pragma once

#include "mocap_attn.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <cstddef>
#include <cstdint>
#include <utility>
#include <vector>

#include "internal.h"

namespace mocap {

// Magic number and shift for unsigned division by an invariant d >= 1, valid
// for dividends below 2^31: l = ceil(log2 d), m = floor(2^32 (2^l - d) / d) + 1,
// and n / d = (umulhi(n, m) + n) >> l (Granlund and Montgomery, 1994, round-up
// method; the sum cannot overflow 32 bits because umulhi(n, m) <= n < 2^31).
inline void block_divider(uint32_t d, uint32_t* magic, int32_t* shift) {
  int l = 0;
  while ((1ull << l) < d) ++l;
  *magic = (uint32_t)((((1ull << l) - d) << 32) / d + 1);
  *shift = l;
}

constexpr int kMaxDevices = 64;
constexpr int64_t kMaxPositions = ((int64_t)1 << 31) - 128;
inline std::atomic<int> g_cu_count[kMaxDevices];  // 0 = not yet queried

inline bool aligned16(const void* ptr) { return (reinterpret_cast<uintptr_t>(ptr) & 15u) == 0; }

inline bool supported_head_dim(int d) { return d == 64 || d == 128; }

inline mocap_status device_cu_count(int* out) {
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess) return MOCAP_ERR_HIP;
  if (dev >= 0 && dev < kMaxDevices) {
    const int cached = g_cu_count[dev].load(std::memory_order_relaxed);
    if (cached > 0) {
      *out = cached;
      return MOCAP_OK;
    }
  }
  int cus = 0;
  if (hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || cus <= 0)
    return MOCAP_ERR_HIP;
  if (dev >= 0 && dev < kMaxDevices) g_cu_count[dev].store(cus, std::memory_order_relaxed);
  *out = cus;
  return MOCAP_OK;
}

inline size_t round_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

inline mocap_status check_store(const mocap_kv_store* kv) {
  if (kv == nullptr) return MOCAP_ERR_INVALID_ARG;
  if (kv->num_blocks <= 0 || kv->block_size <= 0 || kv->h_kv <= 0 || kv->head_dim <= 0)
    return MOCAP_ERR_INVALID_ARG;
  if (!supported_head_dim(kv->head_dim)) return MOCAP_ERR_UNSUPPORTED;
  if (kv->block_size % kTileKeys != 0) return MOCAP_ERR_UNSUPPORTED;
  return MOCAP_OK;
}

inline mocap_status check_positions(const mocap_kv_store* kv, int32_t n_table, int64_t start, int32_t len) {
  if (start < 0 || len < 0 || n_table < 0) return MOCAP_ERR_INVALID_ARG;
  // Kernels index positions with 32-bit integers.
  if (start + (int64_t)len > kMaxPositions) return MOCAP_ERR_INVALID_ARG;
  const int64_t end = start + len;
  const int64_t blocks_needed = (end + kv->block_size - 1) / kv->block_size;
  if (blocks_needed > n_table) return MOCAP_ERR_INVALID_ARG;
  return MOCAP_OK;
}

// Host-side check of the block-table entries that positions [first, end) use:
// each in [0, num_blocks), no two logical blocks on one physical block.
inline mocap_status check_table_entries(const int32_t* table, int32_t n_table, int64_t first, int64_t end,
                                        int32_t block_size, int32_t num_blocks, int32_t* bad_out) {
  if (bad_out) *bad_out = -1;
  if (first < 0 || end < first || block_size <= 0 || num_blocks <= 0 || n_table < 0) return MOCAP_ERR_INVALID_ARG;
  if (end == first) return MOCAP_OK;
  const int64_t b0 = first / block_size, b1 = (end + block_size - 1) / block_size;
  if (b1 > n_table || table == nullptr) return MOCAP_ERR_INVALID_ARG;
  std::vector<std::pair<int32_t, int64_t>> used;
  used.reserve((size_t)(b1 - b0));
  for (int64_t b = b0; b < b1; ++b) {
    if (table[b] < 0 || table[b] >= num_blocks) {
      if (bad_out) *bad_out = (int32_t)b;
      return MOCAP_ERR_INVALID_ARG;
    }
    used.emplace_back(table[b], b);
  }
  std::sort(used.begin(), used.end());
  for (size_t i = 1; i < used.size(); ++i) {
    if (used[i].first == used[i - 1].first) {
      if (bad_out) *bad_out = (int32_t)used[i].second;
      return MOCAP_ERR_INVALID_ARG;
    }
  }
  return MOCAP_OK;
}

// In a build with MOCAP_DEBUG_TABLES, every call copies the table entries it
// will use to the host (a synchronous copy) and checks them before anything
// is enqueued; a bad entry returns MOCAP_ERR_INVALID_ARG.
#ifdef MOCAP_DEBUG_TABLES
inline mocap_status debug_check_table(const int32_t* dev_table, int64_t first, int64_t end, const mocap_kv_store* kv) {
  if (end <= first) return MOCAP_OK;
  const int64_t b0 = first / kv->block_size, b1 = (end + kv->block_size - 1) / kv->block_size;
  std::vector<int32_t> host((size_t)b1, 0);
  if (hipMemcpy(host.data() + b0, dev_table + b0, (size_t)(b1 - b0) * sizeof(int32_t), hipMemcpyDeviceToHost) !=
      hipSuccess)
    return MOCAP_ERR_HIP;
  return check_table_entries(host.data(), (int32_t)b1, first, end, kv->block_size, kv->num_blocks, nullptr);
}
#define MOCAP_DEBUG_CHECK(table, first, end, kv)                                            \
  do {                                                                                      \
    const mocap_status debug_st_ = mocap::debug_check_table((table), (first), (end), (kv)); \
    if (debug_st_ != MOCAP_OK) return debug_st_;                                            \
  } while (0)
#else
#define MOCAP_DEBUG_CHECK(table, first, end, kv) \
  do {                                           \
  } while (0)
#endif

}  // namespace mocap
