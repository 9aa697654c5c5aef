// Attention weight received by every key, for gfx950 (CDNA4):
//   w[h][j] = sum over rows i that see key j and heads g of group h of
//             exp(scale <q_ig, k_jh> - lse_gi)
// Many rows are bound by the matrix unit (2 D FLOP a pair) and the exponentials
// beside it (one a pair, as many issue cycles as the products at head_dim 128),
// few rows by HBM (the keys, once).
//
//   * The keys stay, the rows stream: a wavefront holds 64 keys as B operands in
//     registers and walks the rows, S = Q K^T with v_mfma_f32_32x32x16_bf16.  Lane
//     l then holds key l % 32 of each product and 16 of its 32 rows, so the sum
//     over the rows stays within the lane: one exponential, one FMA and one add a
//     score, and no exchange between lanes before the end.
//   * Rows ((token, query head) pairs of the group, token-major) come in tiles of
//     32 through LDS, Q copied straight to it, a row's LSE in base 2 beside it.
//     key_waves wavefronts along the keys share a tile; 8 / key_waves row tiles
//     are worked on at a time, whose sums meet in LDS at the end.
//   * Sums are fp32: 16 rows first, then tile by tile.
#include "serve_device.h"

namespace mocap {
namespace {

constexpr int kRowTile = 32;
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
  __builtin_amdgcn_s_barrier();
}

__device__ __forceinline__ uint32_t div_by(uint32_t n, uint32_t magic, int shift) {
  return (__umulhi(n, magic) + n) >> shift;
}

template <int D>
__device__ __forceinline__ int q_swizzle(int r) {
  return D == 128 ? (r & 15) : ((r >> 1) & 7);
}

// KW: wavefronts along the keys.
template <int D, int KW>
__global__ __launch_bounds__(64 * kWeightWaves, 2) void key_weights_kernel(const KeyWeightsLaunch p) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int KS = D / 16;
  constexpr int RW = kWeightWaves / KW;           // row tiles at a time
  constexpr int ROW_CHUNKS = D / 8;
  constexpr int TILE_ELEMS = kRowTile * D;
  constexpr int STAGE_ROWS = RW * kRowTile;
  constexpr int COPIES = RW * TILE_ELEMS / 8 / (64 * kWeightWaves);  // 16-byte copies of a thread per stage (0: half of them)
  constexpr int COPY_THREADS = COPIES > 0 ? 64 * kWeightWaves : RW * TILE_ELEMS / 8;
  constexpr int COPIES_EACH = COPIES > 0 ? COPIES : 1;
  constexpr int STAGES = 2;
  __shared__ __attribute__((aligned(1024))) uint16_t ring[STAGES][RW * TILE_ELEMS];
  __shared__ __attribute__((aligned(16))) float lse2[STAGES][STAGE_ROWS];
  __shared__ float sums[RW > 1 ? RW : 1][KW * kWeightKeys];

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = lane >> 5, l32 = lane & 31;
  const int kw = wave % KW, rw = wave / KW;
  const int P = p.prefix_len, n = P + p.chunk_len;

  // Logical order: KV head, row part, key block.
  const int total = p.key_blocks * p.row_parts * p.h_kv;
  const int logical = xcd_contiguous(blockIdx.x, total);
  const int kv_head = logical / (p.key_blocks * p.row_parts);
  const int in_kv = logical - kv_head * p.key_blocks * p.row_parts;
  const int part = in_kv / p.key_blocks;
  const int block0 = (in_kv - part * p.key_blocks) * (KW * kWeightKeys);
  const int key0 = block0 + kw * kWeightKeys;  // this wavefront's keys

  // Rows [begin, end) of this part, in tiles; rows before begin see no key of
  // the workgroup (row r sees key j if r >= (j - P) G).
  const int rows = p.chunk_len * p.group;
  const int row_tiles = (rows + kRowTile - 1) / kRowTile;
  const int first_tile = max(0, block0 - P) * p.group / kRowTile;
  const int span = row_tiles - first_tile;
  const int t0 = first_tile + (int)((int64_t)span * part / p.row_parts);
  const int t1 = first_tile + (int)((int64_t)span * (part + 1) / p.row_parts);

  // K as the B operand: lane l holds key l % 32 of a 32-key half, dims 16 ks + 8 (l / 32) .. + 7.
  // Keys past the last take it; nothing of theirs is stored.
  bf16x8 kf[2][KS];
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    const int key = min(key0 + b * 32 + l32, n - 1);
    const int lb = (int)div_by((uint32_t)key, p.block_magic, p.block_shift);
    const int64_t slot = key - lb * p.block_size;
    const uint16_t* k = p.k_pool + ((((int64_t)p.table[lb] * p.h_kv + kv_head) * p.block_size) + slot) * D + half * 8;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) kf[b][ks] = *reinterpret_cast<const bf16x8*>(k + ks * 16);
  }

  // Stage s of the ring holds row tiles t0 + s RW ..; copy j of a thread moves
  // 16-byte chunk j * 512 + tid, from a column XORed with the row.  Rows past the
  // last take it, with an LSE of +infinity (a weight of 0).
  auto issue = [&](int s) __attribute__((always_inline)) {
    // Offsets from the stage's first token: a stage spans few tokens, all of Q
    // may not fit in 32 bits.
    const int base_row = (t0 + s * RW) * kRowTile;
    const int base_token = (int)div_by((uint32_t)min(base_row, rows - 1), p.group_magic, p.group_shift);
    const uint16_t* base = p.q + ((int64_t)base_token * p.h_q + kv_head * p.group) * D;
    const __amdgpu_buffer_rsrc_t q = __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, -1, kBufferWord3);
    if (tid < COPY_THREADS) {
#pragma unroll
      for (int j = 0; j < COPIES_EACH; ++j) {
        const int chunk = j * COPY_THREADS + tid;
        const int lr = chunk / ROW_CHUNKS, c = (chunk % ROW_CHUNKS) ^ q_swizzle<D>(lr);
        const int r = min(base_row + lr, rows - 1);
        const int token = (int)div_by((uint32_t)r, p.group_magic, p.group_shift);
        const int at = ((token - base_token) * p.h_q + (r - token * p.group)) * D + c * 8;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(q, (lds_ptr_t)(&ring[s % STAGES][(j * COPY_THREADS + wave * 64) * 8]),
                                                 16, at * 2, 0, 0, 0);
      }
    }
  };
  auto load_lse = [&](int s) __attribute__((always_inline)) -> float {
    if (tid >= STAGE_ROWS) return 0.f;
    const int r = (t0 + s * RW) * kRowTile + tid;
    const int q = min(r, rows - 1);
    const int token = (int)div_by((uint32_t)q, p.group_magic, p.group_shift);
    const float x = p.lse[(int64_t)(kv_head * p.group + (q - token * p.group)) * p.chunk_len + token];
    return r < rows && x != -INFINITY ? x * kLog2e : INFINITY;
  };
  auto put_lse = [&](int s, float x) __attribute__((always_inline)) {
    if (tid < STAGE_ROWS) lse2[s % STAGES][tid] = x;
  };

  const float sl2 = p.scale_log2;
  float w[2] = {0.f, 0.f};
  const int stages = (t1 - t0 + RW - 1) / RW;
  if (stages > 0) {
    issue(0);
    put_lse(0, load_lse(0));
    for (int s = 0; s < stages; ++s) {
      float next_lse = 0.f;
      wait_vmem<0>();
      lds_barrier();
      if (s + 1 < stages) {
        issue(s + 1);
        next_lse = load_lse(s + 1);
      }
      const int t = t0 + s * RW + rw;
      // Rows of tile t: the first sees keys up to P + r / G, the last ...
      const int r0 = t * kRowTile, r1 = min(r0 + kRowTile, rows) - 1;
      const bool any = t < t1 && key0 <= P + (int)div_by((uint32_t)max(r1, 0), p.group_magic, p.group_shift);
      if (any) {
        const bool masked = r0 + kRowTile > rows ||
                            key0 + kWeightKeys - 1 > P + (int)div_by((uint32_t)r0, p.group_magic, p.group_shift);
        const uint16_t* ql = &ring[s % STAGES][rw * TILE_ELEMS];
        f32x16 sc[2] = {f32x16{}, f32x16{}};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const bf16x8 a = *reinterpret_cast<const bf16x8*>(ql + l32 * D + (((ks * 2 + half) ^ q_swizzle<D>(l32)) << 3));
          sc[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, kf[0][ks], sc[0], 0, 0, 0);
          sc[1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, kf[1][ks], sc[1], 0, 0, 0);
        }
        // Score j of this lane belongs to row r0 + 8 (j / 4) + 4 half + j % 4.
        float l2[16];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const f32x4 x = *reinterpret_cast<const f32x4*>(&lse2[s % STAGES][rw * kRowTile + j * 8 + half * 4]);
#pragma unroll
          for (int e = 0; e < 4; ++e) l2[j * 4 + e] = x[e];
        }
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          float e[16];
#pragma unroll
          for (int j = 0; j < 16; ++j) e[j] = __builtin_amdgcn_exp2f(fmaf(sc[b][j], sl2, -l2[j]));
          if (masked) {
            // The first row that sees this lane's key.
            const int64_t from = max((int64_t)(key0 + b * 32 + l32 - P) * p.group, (int64_t)0);
#pragma unroll
            for (int j = 0; j < 16; ++j) {
              const int r = r0 + (j >> 2) * 8 + half * 4 + (j & 3);
              e[j] = r >= from && r < rows ? e[j] : 0.f;
            }
          }
#pragma unroll
          for (int off = 8; off > 0; off >>= 1)
#pragma unroll
            for (int j = 0; j < off; ++j) e[j] += e[j + off];
          w[b] += e[0];
        }
      }
      if (s + 1 < stages) put_lse(s + 1, next_lse);
    }
  }

  w[0] = lane_pair_sum(w[0]);
  w[1] = lane_pair_sum(w[1]);
  float total_w = half ? w[1] : w[0];  // of key key0 + lane
  if constexpr (RW > 1) {
    sums[rw][kw * kWeightKeys + lane] = total_w;
    __syncthreads();
    if (rw != 0) return;
    total_w = 0.f;
#pragma unroll
    for (int r = 0; r < RW; ++r) total_w += sums[r][kw * kWeightKeys + lane];
  }
  const int key = key0 + lane;
  if (key >= n) return;
  if (p.row_parts == 1) {
    const int64_t at = kv_head * p.weight_stride + key;
    p.weights[at] = (p.prev != nullptr && key < P ? p.prev[at] : 0.f) + total_w;
  } else {
    p.ws[((int64_t)part * p.h_kv + kv_head) * n + key] = total_w;
  }
#endif  // __HIP_DEVICE_COMPILE__
}

// Sums the row parts, in order.
__global__ __launch_bounds__(256) void key_weights_join_kernel(const KeyWeightsLaunch p) {
  const int n = p.prefix_len + p.chunk_len;
  const int key = blockIdx.x * 256 + threadIdx.x, h = blockIdx.y;
  if (key >= n) return;
  float w = 0.f;
  for (int part = 0; part < p.row_parts; ++part) w += p.ws[((int64_t)part * p.h_kv + h) * n + key];
  const int64_t at = h * p.weight_stride + key;
  p.weights[at] = (p.prev != nullptr && key < p.prefix_len ? p.prev[at] : 0.f) + w;
}

// ---- One row per sequence ----
// Bound by HBM (every key once).  A wavefront takes 64 keys at a time, all of
// them in flight, in registers: S = Q K^T with v_mfma_f32_16x16x32_bf16, 16 query
// heads by 16 keys, so lane l holds key l % 16 and four heads of each product;
// groups of more heads go through the same keys 16 at a time.
constexpr int kDecodeWaves = 4;

template <int D>
__global__ __launch_bounds__(64 * kDecodeWaves) void decode_key_weights_kernel(const DecodeKeyWeightsLaunch p) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int KS = D / 32;
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, g4 = lane >> 4;
  const int item = blockIdx.x / p.h_kv;
  const int kv_head = blockIdx.x - item * p.h_kv;
  const SeqPart x = locate_item(p.seqs, lane, item);
  if (x.seq == p.seqs.batch) return;
  int begin, end;
  part_range(x, &begin, &end);

  const const_i32_ptr table = (const_i32_ptr)(p.seqs.tables + x.seq * p.seqs.table_stride);
  const int bs = p.seqs.block_size;
  const int64_t q0 = (int64_t)x.seq * p.h_q + kv_head * p.group;
  const int64_t w0 = ((int64_t)x.seq * p.h_kv + kv_head) * p.weight_stride;
  const float sl2 = p.scale_log2;
  for (int t = begin + wave; t < end; t += kDecodeWaves) {
    const int pos = t * kTileKeys;
    const int lb = (int)div_by((uint32_t)pos, p.seqs.block_magic, p.seqs.block_shift);
    const int64_t slot = pos - lb * bs;
    const uint16_t* k = p.k_pool + (((int64_t)table[lb] * p.h_kv + kv_head) * bs + slot + l16) * D + g4 * 8;
    bf16x8 kf[4][KS];
#pragma unroll
    for (int b = 0; b < 4; ++b)
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) kf[b][ks] = *reinterpret_cast<const bf16x8*>(k + b * 16 * D + ks * 32);
    const int key = pos + lane;
    const bool live = key < x.span.len;
    const float old = live && p.prev != nullptr && key < x.span.len - 1 ? p.prev[w0 + key] : 0.f;
    float w = 0.f;  // of key pos + lane
    for (int h0 = 0; h0 < p.group; h0 += 16) {
      const uint16_t* q = p.q + (q0 + min(h0 + l16, p.group - 1)) * D + g4 * 8;
      bf16x8 qf[KS];
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) qf[ks] = *reinterpret_cast<const bf16x8*>(q + ks * 32);
      float l2[4];  // of heads h0 + 4 g4 + e
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int head = h0 + g4 * 4 + e;
        const float v = p.lse[q0 + min(head, p.group - 1)];
        l2[e] = head < p.group && v != -INFINITY ? v * kLog2e : INFINITY;
      }
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        f32x4 s = f32x4{};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qf[ks], kf[b][ks], s, 0, 0, 0);
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float v = __builtin_amdgcn_exp2f(fmaf(s[e], sl2, -l2[e]));
          sum += h0 + g4 * 4 + e < p.group ? v : 0.f;
        }
        sum = quad_rows_sum(sum);
        w += g4 == b ? sum : 0.f;
      }
    }
    if (live) p.weights[w0 + key] = old + w;
  }
#endif  // __HIP_DEVICE_COMPILE__
}

template <int D>
void launch(const KeyWeightsLaunch& p, hipStream_t stream) {
  const dim3 grid((unsigned)((int64_t)p.key_blocks * p.row_parts * p.h_kv)), block(64 * kWeightWaves);
  switch (p.key_waves) {
    case 1: hipLaunchKernelGGL((key_weights_kernel<D, 1>), grid, block, 0, stream, p); break;
    case 2: hipLaunchKernelGGL((key_weights_kernel<D, 2>), grid, block, 0, stream, p); break;
    case 4: hipLaunchKernelGGL((key_weights_kernel<D, 4>), grid, block, 0, stream, p); break;
    default: hipLaunchKernelGGL((key_weights_kernel<D, 8>), grid, block, 0, stream, p); break;
  }
  if (p.row_parts > 1) {
    const int n = p.prefix_len + p.chunk_len;
    hipLaunchKernelGGL(key_weights_join_kernel, dim3((n + 255) / 256, p.h_kv), dim3(256), 0, stream, p);
  }
}

}  // namespace

hipError_t launch_key_weights(const KeyWeightsLaunch& p, int head_dim, hipStream_t stream) {
  if (head_dim == 128) {
    launch<128>(p, stream);
  } else {
    launch<64>(p, stream);
  }
  return hipGetLastError();
}

hipError_t launch_decode_key_weights(const DecodeKeyWeightsLaunch& p, int head_dim, hipStream_t stream) {
  const dim3 grid((unsigned)((int64_t)p.seqs.items * p.h_kv)), block(64 * kDecodeWaves);
  if (head_dim == 128) {
    hipLaunchKernelGGL(decode_key_weights_kernel<128>, grid, block, 0, stream, p);
  } else {
    hipLaunchKernelGGL(decode_key_weights_kernel<64>, grid, block, 0, stream, p);
  }
  return hipGetLastError();
}

}  // namespace mocap
