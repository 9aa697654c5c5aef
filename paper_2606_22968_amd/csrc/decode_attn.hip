// Decoding over the paged store for gfx950 (CDNA4): the batch append of one
// token per sequence, and the attention of one token per sequence.
//
// For query head g of KV head h and sequence b, over its visible keys j:
//   s_j = scale <q_g, k_j>,  lse = ln sum_j exp s_j,  o = sum_j exp(s_j - lse) v_j
// Every key and value is used by the G query heads of its group only: 2 G FLOP a
// byte, so HBM bounds it (and latency, when there is little to read).
//
//   * Work is cut by what is there and not by sequence (see SeqBatch): a
//     workgroup takes one part of one sequence for one KV head and up to 16 or 32
//     of its query heads, and every part has about the same number of tiles.
//   * A part's four wavefronts take its keys in turn, 32 at a time, each with a
//     softmax state of its own, so there is no barrier before the end.
//   * Scores are computed transposed, S^T = K Q^T, with
//     v_mfma_f32_16x16x32_bf16: 16 keys by 16 query heads.  Lane l then holds
//     head l % 16 and four keys of each product.  The K rows of a pair of
//     products are taken in an order that gives lane group g = l / 16 the keys
//     8 g .. 8 g + 7 of the 32, which is what the P*V product wants as its B
//     operand, and in the store V's 8 consecutive keys of a dim are 16 bytes.
//     Both operands come straight from the store in registers: a load
//     instruction takes 64 contiguous bytes of 16 rows, the rate of the vector
//     cache, and nothing is used twice, so LDS has nothing to give.
//   * MFMAs are some percent busy, so precision is cheap: the probabilities go
//     in as two bf16 values, p = hi + lo.
#include "serve_device.h"

namespace mocap {
namespace {

constexpr int kDecodeWaves = 4;
constexpr int kDecodeThreads = 64 * kDecodeWaves;
constexpr int kStepKeys = 32;

// ---- Append ----
// One thread per 16 bytes of a position's K and V.  V is stored with the
// positions contiguous, so each of its values goes to a line of its own.
template <int D>
__global__ __launch_bounds__(256) void decode_append_kernel(const DecodeAppendLaunch p) {
  constexpr int CHUNKS = D / 8;
  const int b = blockIdx.x;
  const int64_t n = p.seq_lens[b];
  if (n <= 0 || n > p.table_stride * p.block_size) return;
  const uint32_t pos = (uint32_t)(n - 1);
  const uint32_t lb = pos / (uint32_t)p.block_size;
  const int64_t slot = pos - lb * (uint32_t)p.block_size;
  const int64_t block = p.tables[b * p.table_stride + lb];
  for (int i = blockIdx.y * 256 + threadIdx.x; i < p.h_kv * CHUNKS; i += gridDim.y * 256) {
    const int h = i / CHUNKS, c = i % CHUNKS;
    const int64_t src = ((int64_t)b * p.h_kv + h) * D + c * 8;
    const int64_t head = (block * p.h_kv + h) * D * p.block_size;
    const u32x4 k = *reinterpret_cast<const u32x4*>(p.k + src);
    const u32x4 v = *reinterpret_cast<const u32x4*>(p.v + src);
    *reinterpret_cast<u32x4*>(p.k_pool + head + slot * D + c * 8) = k;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      uint16_t* dst = p.v_pool + head + (int64_t)(c * 8 + 2 * w) * p.block_size + slot;
      dst[0] = (uint16_t)(v[w] & 0xFFFFu);
      dst[p.block_size] = (uint16_t)(v[w] >> 16);
    }
  }
}

// ---- Attention ----
// NT: 16-head blocks of the group that a workgroup takes.
template <int D, int NT>
__global__ __launch_bounds__(kDecodeThreads) void decode_attn_kernel(const DecodeAttnLaunch p) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int KS = D / 32;  // k-steps of a score product
  constexpr int MD = D / 16;  // 16-dim blocks of O
  __shared__ __attribute__((aligned(16))) float part_o[kDecodeWaves][NT * 16][D];
  __shared__ float part_m[kDecodeWaves][NT * 16], part_l[kDecodeWaves][NT * 16];

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, g4 = lane >> 4;

  // Logical order: item, KV head, block of query heads.
  const int per_item = p.h_kv * p.row_blocks;
  const int item = blockIdx.x / per_item;
  const int in_item = blockIdx.x - item * per_item;
  const int kv_head = in_item / p.row_blocks;
  const int head0 = (in_item - kv_head * p.row_blocks) * (NT * 16);  // of the group
  const SeqPart w = locate_item(p.seqs, lane, item);
  if (w.seq == p.seqs.batch) return;
  int begin, end;
  part_range(w, &begin, &end);

  // Q as the B operand: lane l holds head l % 16, dims 32 ks + 8 (l / 16) .. + 7.
  // Lanes past the group's last head take that head; nothing of theirs is stored.
  bf16x8 qf[NT][KS];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int g = min(head0 + t * 16 + l16, p.group - 1);
    const uint16_t* row = p.q + ((int64_t)w.seq * p.h_q + kv_head * p.group + g) * D + g4 * 8;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[t][ks] = *reinterpret_cast<const bf16x8*>(row + ks * 32);
  }

  const const_i32_ptr table = (const_i32_ptr)(p.seqs.tables + w.seq * p.seqs.table_stride);
  const int bs = p.seqs.block_size;
  const int64_t head_stride = (int64_t)D * bs;
  const int k_lane = (8 * (l16 >> 2) + (l16 & 3)) * D + g4 * 8;  // key of the first product; the second's is 4 on
  const int v_lane = l16 * bs + g4 * 8;

  struct Tile {
    bf16x8 k[2][KS], v[MD];
  };
  auto step_key = [&](int i) __attribute__((always_inline)) {  // first key of step i of the part
    return w.span.tile(begin + (i >> 1)) * kTileKeys + (i & 1) * kStepKeys;
  };
  auto fetch = [&](int i, Tile& x) __attribute__((always_inline)) {
    const int pos = step_key(i);
    const int lb = (int)((__umulhi((uint32_t)pos, p.seqs.block_magic) + (uint32_t)pos) >> p.seqs.block_shift);
    const int slot = pos - lb * bs;
    const int64_t base = ((int64_t)table[lb] * p.h_kv + kv_head) * head_stride;
    const uint16_t* k = p.k_pool + base + (int64_t)slot * D + k_lane;
    const uint16_t* v = p.v_pool + base + slot + v_lane;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) x.k[h][ks] = *reinterpret_cast<const bf16x8*>(k + h * 4 * D + ks * 32);
#pragma unroll
    for (int md = 0; md < MD; ++md) x.v[md] = *reinterpret_cast<const bf16x8*>(v + (int64_t)md * 16 * bs);
  };

  f32x4 oacc[NT][MD];
  float m_run[NT], l_run[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    m_run[t] = -INFINITY;
    l_run[t] = 0.f;
#pragma unroll
    for (int md = 0; md < MD; ++md) oacc[t][md] = f32x4{};
  }
  const float sl2 = p.scale_log2;

  // Steps of this wavefront; the last tile's second half may lie past the end.
  const int steps = 2 * (end - begin);
  Tile cur;
  if (wave < steps) fetch(wave, cur);
  for (int i = wave; i < steps; i += kDecodeWaves) {
    Tile next;
    const bool more = i + kDecodeWaves < steps;
    if (more) fetch(i + kDecodeWaves, next);
    const int key0 = step_key(i);
    // Hidden keys of this lane's eight, key0 + 8 g4 .. + 7, as bits.
    uint32_t hidden = 0;
    const bool masked = key0 + kStepKeys > w.span.len || (key0 < w.span.low && key0 + kStepKeys > w.span.sink_end);
    if (masked) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int key = key0 + g4 * 8 + e;
        const bool seen = key < w.span.len && (key < w.span.sink_end || key >= w.span.low);
        hidden |= seen ? 0u : 1u << e;
      }
      // What a hidden position holds may be NaN; its probability is 0.
#pragma unroll
      for (int md = 0; md < MD; ++md) {
        u32x4 x = __builtin_bit_cast(u32x4, cur.v[md]);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          x[e] &= (hidden >> (2 * e) & 1 ? 0u : 0x0000FFFFu) | (hidden >> (2 * e + 1) & 1 ? 0u : 0xFFFF0000u);
        cur.v[md] = __builtin_bit_cast(bf16x8, x);
      }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      f32x4 s[2] = {f32x4{}, f32x4{}};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        s[0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(cur.k[0][ks], qf[t][ks], s[0], 0, 0, 0);
        s[1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(cur.k[1][ks], qf[t][ks], s[1], 0, 0, 0);
      }
      float x[8];  // of keys key0 + 8 g4 + e
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = hidden >> e & 1 ? -INFINITY : s[e >> 2][e & 3];
      float mx = x[0];
#pragma unroll
      for (int e = 1; e < 8; ++e) mx = fmaxf(mx, x[e]);
      const float m_new = fmaxf(m_run[t], quad_rows_max(mx) * sl2);
      const float ref = m_new == -INFINITY ? 0.f : m_new;
      // The accumulators are scaled only when some row's maximum has grown.
      if (__builtin_amdgcn_ballot_w64(m_new != m_run[t]) != 0) {
        const float f = __builtin_amdgcn_exp2f(m_run[t] - ref);
        l_run[t] *= f;
#pragma unroll
        for (int md = 0; md < MD; ++md) oacc[t][md] *= f;
        m_run[t] = m_new;
      }
      float e2[8], lo[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        e2[e] = __builtin_amdgcn_exp2f(fmaf(x[e], sl2, -ref));
        l_run[t] += e2[e];
        lo[e] = e2[e] - (float)(__bf16)e2[e];
      }
      u32x4 ph, pl;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        ph[e] = pack_bf16x2(e2[2 * e], e2[2 * e + 1]);
        pl[e] = pack_bf16x2(lo[2 * e], lo[2 * e + 1]);
      }
      const bf16x8 hi8 = __builtin_bit_cast(bf16x8, ph), lo8 = __builtin_bit_cast(bf16x8, pl);
#pragma unroll
      for (int md = 0; md < MD; ++md) {
        oacc[t][md] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(cur.v[md], hi8, oacc[t][md], 0, 0, 0);
        oacc[t][md] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(cur.v[md], lo8, oacc[t][md], 0, 0, 0);
      }
    }
    cur = next;
  }

  // The wavefronts' partials meet in LDS.  Lane l holds head l % 16 and dims
  // 16 md + 4 (l / 16) .. + 3.
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const float l = quad_rows_sum(l_run[t]);
    if (g4 == 0) {
      part_m[wave][t * 16 + l16] = m_run[t];
      part_l[wave][t * 16 + l16] = l;
    }
#pragma unroll
    for (int md = 0; md < MD; ++md)
      *reinterpret_cast<f32x4*>(&part_o[wave][t * 16 + l16][md * 16 + g4 * 4]) = oacc[t][md];
  }
  __syncthreads();
  constexpr int QUADS = D / 4;
  for (int i = tid; i < min(NT * 16, p.group - head0) * QUADS; i += kDecodeThreads) {
    const int row = i / QUADS, quad = i % QUADS;
    float m = -INFINITY;
#pragma unroll
    for (int x = 0; x < kDecodeWaves; ++x) m = fmaxf(m, part_m[x][row]);
    float l = 0.f;
    f32x4 acc = f32x4{};
#pragma unroll
    for (int x = 0; x < kDecodeWaves; ++x) {
      // A partial counts if its sum is not 0 (a NaN score leaves m = -inf and a NaN sum).
      const float l_x = part_l[x][row];
      const float f = l_x != 0.f ? __builtin_amdgcn_exp2f(part_m[x][row] - m) : 0.f;
      l += l_x != 0.f ? l_x * f : 0.f;
      const f32x4 o_x = *reinterpret_cast<const f32x4*>(&part_o[x][row][quad * 4]);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] += l_x != 0.f ? o_x[e] * f : 0.f;
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const float row_lse = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
    const int head = kv_head * p.group + head0 + row;
    acc *= inv;
    if (w.parts == 1) {
      const int64_t at = (int64_t)w.seq * p.h_q + head;
      bf16x4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = (__bf16)acc[e];
      *reinterpret_cast<bf16x4*>(p.o + at * D + quad * 4) = v;
      if (quad == 0) p.lse[at] = row_lse;
    } else {
      const int64_t at = (int64_t)item * p.h_q + head;
      *reinterpret_cast<f32x4*>(p.ws_o + at * D + quad * 4) = acc;
      if (quad == 0) p.ws_lse[at] = row_lse;
    }
  }
#endif  // __HIP_DEVICE_COMPILE__
}

// ---- Join ----
// One wavefront per (sequence, query head) that was cut: lse = ln sum exp lse_r,
// o = sum exp(lse_r - lse) o_r over its parts r, in order.
template <int D>
__global__ __launch_bounds__(kDecodeThreads) void decode_join_kernel(const DecodeAttnLaunch p) {
  constexpr int QUADS = D / 4, SIDE = 64 / QUADS;  // parts read at a time
  const int lane = threadIdx.x & 63;
  const int64_t at = (int64_t)blockIdx.x * kDecodeWaves + (threadIdx.x >> 6);
  if (at >= (int64_t)p.seqs.batch * p.h_q) return;
  const int seq = (int)(at / p.h_q), head = (int)(at - (int64_t)seq * p.h_q);
  int first;
  const SeqPart w = parts_of(p.seqs, lane, seq, &first);
  if (w.parts == 1) return;
  const int quad = lane % QUADS, side = lane / QUADS;
  const float* lse = p.ws_lse + (int64_t)first * p.h_q + head;
  const float* o = p.ws_o + ((int64_t)first * p.h_q + head) * D + quad * 4;
  float m = -INFINITY;
  for (int r = lane; r < w.parts; r += 64) m = fmaxf(m, lse[(int64_t)r * p.h_q]);
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor(m, off));
  float z = 0.f;
  f32x4 acc = f32x4{};
  for (int r = side; r < w.parts; r += SIDE) {
    const float lr = lse[(int64_t)r * p.h_q];
    const f32x4 v = *reinterpret_cast<const f32x4*>(o + (int64_t)r * p.h_q * D);
    const bool used = lr != -INFINITY;
    const float f = used ? expf(lr - m) : 0.f;
    z += f;
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] = fmaf(f, used ? v[e] : 0.f, acc[e]);
  }
#pragma unroll
  for (int off = 32; off >= QUADS; off >>= 1) {
    z += __shfl_xor(z, off);
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] += __shfl_xor(acc[e], off);
  }
  if (side != 0) return;
  const float inv = z == 0.f ? 0.f : 1.f / z;
  bf16x4 out;
#pragma unroll
  for (int e = 0; e < 4; ++e) out[e] = (__bf16)(acc[e] * inv);
  *reinterpret_cast<bf16x4*>(p.o + at * D + quad * 4) = out;
  if (quad == 0) p.lse[at] = z == 0.f ? -INFINITY : m + logf(z);
}

template <int D>
void launch(const DecodeAttnLaunch& p, hipStream_t stream) {
  const dim3 grid((unsigned)((int64_t)p.seqs.items * p.h_kv * p.row_blocks)), block(kDecodeThreads);
  if (p.group <= 16) {
    hipLaunchKernelGGL((decode_attn_kernel<D, 1>), grid, block, 0, stream, p);
  } else {
    hipLaunchKernelGGL((decode_attn_kernel<D, 2>), grid, block, 0, stream, p);
  }
  if (!p.may_split) return;
  const int64_t rows = (int64_t)p.seqs.batch * p.h_q;
  hipLaunchKernelGGL((decode_join_kernel<D>), dim3((unsigned)((rows + kDecodeWaves - 1) / kDecodeWaves)), block, 0,
                     stream, p);
}

}  // namespace

hipError_t launch_decode_attn(const DecodeAttnLaunch& p, int head_dim, hipStream_t stream) {
  if (head_dim == 128) {
    launch<128>(p, stream);
  } else {
    launch<64>(p, stream);
  }
  return hipGetLastError();
}

hipError_t launch_decode_append(const DecodeAppendLaunch& p, int head_dim, hipStream_t stream) {
  const int chunks = p.h_kv * (head_dim / 8);
  const dim3 grid(p.batch, (chunks + 255) / 256), block(256);
  if (head_dim == 128) {
    hipLaunchKernelGGL(decode_append_kernel<128>, grid, block, 0, stream, p);
  } else {
    hipLaunchKernelGGL(decode_append_kernel<64>, grid, block, 0, stream, p);
  }
  return hipGetLastError();
}

}  // namespace mocap
