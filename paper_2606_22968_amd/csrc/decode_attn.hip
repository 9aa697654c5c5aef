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
//   * A part's four wavefronts take its 64-key tiles in turn, each with a softmax
//     state of its own, so there is no barrier before the end.
//   * Scores are computed transposed, S^T = K Q^T, with
//     v_mfma_f32_16x16x32_bf16: 16 keys by 16 query heads.  Lane l then holds
//     head l % 16 and four keys of each product.  The K rows of a pair of
//     products are taken in an order that gives lane group g = l / 16 the keys
//     8 g .. 8 g + 7 of the 32, which is what the P*V product wants as its B
//     operand, and in the store V's 8 consecutive keys of a dim are 16 bytes.
//     Both operands come straight from the store in registers: a load
//     instruction takes 64 contiguous bytes of 16 rows, the rate of the vector
//     cache, and nothing is used twice, so LDS has nothing to give.
//   * MFMAs are busy 6% of the time, so precision is cheap: the probabilities go
//     in as two bf16 values, p = hi + lo.  lo is 0 or negative as often as not, which
//     an infinite value turns into NaN or the other infinity; where an accumulator is
//     not finite, the part's values are searched for what its dim gets by definition
//     (an infinity in every block of the four long sequences below: 483 us for 299).
// Measured: four sequences of 65537 to 131072 positions, 64/8/128 heads, 1.70 GB
// in 293 us, 5.8 TB/s (a large copy runs at 5.1); 32 of 1 to 8192, 32/8/128, 340 MB
// in 68 us and the join's 6; one of 572 positions, 9 us: lengths, table, keys and
// values, one after the other.
#include "serve_device.h"

namespace mocap {
namespace {

constexpr int kDecodeWaves = 4;
constexpr int kDecodeThreads = 64 * kDecodeWaves;

// ---- Append ----
// One thread per 16 bytes of a position's K and V, small workgroups for many
// compute units.  V is stored with the positions contiguous, so each of its values
// goes to a line of its own.  Bound by latency: lengths, table, stores (1.9 us for
// one sequence, 4.9 for 32 of 8 heads of 128).
template <int D>
__global__ __launch_bounds__(64) void decode_append_kernel(const DecodeAppendLaunch p) {
  constexpr int CHUNKS = D / 8;
  const int b = blockIdx.x;
  const int i = blockIdx.y * 64 + threadIdx.x;
  if (i >= p.h_kv * CHUNKS) return;
  const int h = i / CHUNKS, c = i % CHUNKS;
  const int64_t src = ((int64_t)b * p.h_kv + h) * D + c * 8;
  const u32x4 k = *reinterpret_cast<const u32x4*>(p.k + src);
  const u32x4 v = *reinterpret_cast<const u32x4*>(p.v + src);
  const int64_t n = p.seq_lens[b];
  if (n <= 0 || n > p.table_stride * p.block_size) return;
  const uint32_t pos = (uint32_t)(n - 1);
  const uint32_t lb = pos / (uint32_t)p.block_size;
  const int64_t slot = pos - lb * (uint32_t)p.block_size;
  const int64_t head = ((int64_t)p.tables[b * p.table_stride + lb] * p.h_kv + h) * D * p.block_size;
  *reinterpret_cast<u32x4*>(p.k_pool + head + slot * D + c * 8) = k;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    uint16_t* dst = p.v_pool + head + (int64_t)(c * 8 + 2 * w) * p.block_size + slot;
    dst[0] = (uint16_t)(v[w] & 0xFFFFu);
    dst[p.block_size] = (uint16_t)(v[w] >> 16);
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
  __shared__ uint32_t part_apart[kDecodeWaves];  // some accumulator is not finite
  // What the part's values hold of each dim: 1 for +infinity, 2 for -infinity, both for NaN.
  __shared__ uint32_t marks[D];

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, g4 = lane >> 4;

  // Logical order: item, KV head; the blocks of query heads that read the same
  // keys are 8 workgroups apart, on one XCD.
  const int stripe = blockIdx.x / (8 * p.row_blocks), in_stripe = blockIdx.x - stripe * 8 * p.row_blocks;
  const int work = stripe * 8 + (in_stripe & 7);
  const int item = work / p.h_kv;
  const int kv_head = work - item * p.h_kv;
  const int head0 = (in_stripe >> 3) * (NT * 16);  // of the group
  if (item >= p.seqs.items) return;
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
  // The K rows of products 0 and 1 of a 32-key half: keys 8 (l16 / 4) + l16 % 4, and 4 on.
  const int k_lane = (8 * (l16 >> 2) + (l16 & 3)) * D + g4 * 8;
  const int v_lane = l16 * bs + g4 * 8;

  struct Source {
    const uint16_t *k, *v;
  };
  // Position pos, the first of a tile: its slot, and the first element of its block's head.
  auto find = [&](int pos, int* slot) __attribute__((always_inline)) {
    const int lb = (int)((__umulhi((uint32_t)pos, p.seqs.block_magic) + (uint32_t)pos) >> p.seqs.block_shift);
    *slot = pos - lb * bs;
    return ((int64_t)table[lb] * p.h_kv + kv_head) * head_stride;
  };
  auto locate = [&](int i) __attribute__((always_inline)) {  // tile i of the part
    int slot;
    const int64_t base = find(w.span.tile(begin + i) * kTileKeys, &slot);
    return Source{p.k_pool + base + (int64_t)slot * D + k_lane, p.v_pool + base + slot + v_lane};
  };
  auto visible = [&](int key) { return key < w.span.len && (key < w.span.sink_end || key >= w.span.low); };
  bf16x8 k[4][KS], v[2][MD];  // of a tile: K by product, V by 32-key half
  auto fetch_k = [&](const uint16_t* src) __attribute__((always_inline)) {
#pragma unroll
    for (int h = 0; h < 4; ++h)
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
        k[h][ks] = *reinterpret_cast<const bf16x8*>(src + ((h >> 1) * 32 + (h & 1) * 4) * D + ks * 32);
  };
  auto fetch_v = [&](const uint16_t* src) __attribute__((always_inline)) {
#pragma unroll
    for (int md = 0; md < MD; ++md)
#pragma unroll
      for (int h = 0; h < 2; ++h) v[h][md] = *reinterpret_cast<const bf16x8*>(src + (int64_t)md * 16 * bs + h * 32);
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

  // A wavefront's tiles: wave, wave + 4, ...  The next tile's K is requested as
  // soon as this one's is used up, its V likewise.
  const int tiles = end - begin;
  if (wave < tiles) {
    const Source first = locate(wave);
    fetch_k(first.k);
    fetch_v(first.v);
  }
  for (int i = wave; i < tiles; i += kDecodeWaves) {
    const bool more = i + kDecodeWaves < tiles;
    const Source next = locate(more ? i + kDecodeWaves : i);
    f32x4 s[NT][4];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        s[t][h] = f32x4{};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
          s[t][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[h][ks], qf[t][ks], s[t][h], 0, 0, 0);
      }
    if (more) fetch_k(next.k);
    // Score e of a lane belongs to key key0 + 32 (e / 8) + 8 g4 + e % 8; hidden ones as bits.
    const int key0 = w.span.tile(begin + i) * kTileKeys;
    uint32_t hidden = 0;
    if (key0 + kTileKeys > w.span.len || (key0 < w.span.low && key0 + kTileKeys > w.span.sink_end)) {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        hidden |= visible(key0 + (e >> 3) * 32 + g4 * 8 + (e & 7)) ? 0u : 1u << e;
      }
      // What a hidden position holds may be NaN; its probability is 0.
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int md = 0; md < MD; ++md) {
          u32x4 x = __builtin_bit_cast(u32x4, v[h][md]);
#pragma unroll
          for (int e = 0; e < 4; ++e)
            x[e] &= (hidden >> (8 * h + 2 * e) & 1 ? 0u : 0x0000FFFFu) | (hidden >> (8 * h + 2 * e + 1) & 1 ? 0u : 0xFFFF0000u);
          v[h][md] = __builtin_bit_cast(bf16x8, x);
        }
    }
    bf16x8 hi[NT][2], lo[NT][2];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      float x[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) x[e] = hidden >> e & 1 ? -INFINITY : s[t][e >> 2][e & 3];
      float mx = x[0];
#pragma unroll
      for (int e = 1; e < 16; ++e) mx = fmaxf(mx, x[e]);
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
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        u32x4 ph, pl;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float a = __builtin_amdgcn_exp2f(fmaf(x[8 * h + 2 * e], sl2, -ref));
          const float b = __builtin_amdgcn_exp2f(fmaf(x[8 * h + 2 * e + 1], sl2, -ref));
          l_run[t] += a + b;
          ph[e] = pack_bf16x2(a, b);
          pl[e] = pack_bf16x2(a - __uint_as_float(ph[e] << 16), b - __uint_as_float(ph[e] & 0xFFFF0000u));
        }
        hi[t][h] = __builtin_bit_cast(bf16x8, ph);
        lo[t][h] = __builtin_bit_cast(bf16x8, pl);
      }
    }
#pragma unroll
    for (int md = 0; md < MD; ++md)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          oacc[t][md] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[h][md], hi[t][h], oacc[t][md], 0, 0, 0);
          oacc[t][md] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[h][md], lo[t][h], oacc[t][md], 0, 0, 0);
        }
    if (more) fetch_v(next.v);
  }

  // The wavefronts' partials meet in LDS.  Lane l holds head l % 16 and dims
  // 16 md + 4 (l / 16) .. + 3.
  float probe = 0.f;  // NaN if some accumulator is not finite
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    // A score whose product with the scale is beyond fp32 makes every other exponential
    // 0 and its own too; the row is NaN, as with an infinite score.
    const float l = m_run[t] == INFINITY ? NAN : quad_rows_sum(l_run[t]);
    if (g4 == 0) {
      part_m[wave][t * 16 + l16] = m_run[t];
      part_l[wave][t * 16 + l16] = l;
    }
#pragma unroll
    for (int md = 0; md < MD; ++md) {
      *reinterpret_cast<f32x4*>(&part_o[wave][t * 16 + l16][md * 16 + g4 * 4]) = oacc[t][md];
#pragma unroll
      for (int e = 0; e < 4; ++e) probe = fmaf(oacc[t][md][e], 0.f, probe);
    }
  }
  const bool wave_apart = __builtin_amdgcn_ballot_w64(probe != probe) != 0;
  if (lane == 0) part_apart[wave] = wave_apart;
  if (tid < D) marks[tid] = 0;
  __syncthreads();
  uint32_t apart = 0;
#pragma unroll
  for (int x = 0; x < kDecodeWaves; ++x) apart |= part_apart[x];
  if (apart != 0) {  // the same for the whole workgroup
    constexpr int SIDE = kDecodeThreads / D;  // tiles searched side by side
    const int dim = tid % D;
    uint32_t mark = 0;
#pragma unroll 1
    for (int i = tid / D; i < tiles; i += SIDE) {
      const int key0 = w.span.tile(begin + i) * kTileKeys;
      int slot;
      const uint16_t* src = p.v_pool + find(key0, &slot) + (int64_t)dim * bs;
      u32x4 x[kTileKeys / 8];  // all loads in flight
#pragma unroll
      for (int c = 0; c < kTileKeys / 8; ++c) x[c] = *reinterpret_cast<const u32x4*>(src + slot + c * 8);
#pragma unroll
      for (int e = 0; e < kTileKeys; ++e) {
        const uint32_t v = x[e / 8][e / 2 % 4] >> (16 * (e & 1)) & 0xFFFFu;
        if ((v & 0x7F80u) == 0x7F80u && visible(key0 + e)) mark |= (v & 0x7Fu) ? 3u : v >> 15 ? 2u : 1u;
      }
    }
    if (mark != 0) atomicOr(&marks[dim], mark);
    __syncthreads();
  }
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
    if (apart != 0 && l > 0.f) {  // (a NaN score's row is NaN)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t mark = marks[quad * 4 + e];
        if (mark != 0) acc[e] = mark == 1 ? INFINITY : mark == 2 ? -INFINITY : NAN;
      }
    }
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
// One workgroup per (sequence, query head) that was cut: lse = ln sum exp lse_r,
// o = sum exp(lse_r - lse) o_r over its parts r, in order.  Bound by the chain of
// loads: every wavefront takes a quarter of the parts, lane r the LSE of its r-th,
// forms 64 weights together, and requests the partials of 8 (head_dim 128: 16)
// parts at once, the first before any weight is known.  6 us for 4 sequences of 64
// heads in 164 parts in all (14 with one wavefront for a row), and for 32 of 32 heads.

// The weight of a part with keys is never 0, so that infinities and NaN in its O count
// however far it lies below the others; the least fp32 value times a finite O adds
// less than 5e-7.
__device__ __forceinline__ float part_weight(float lse, float m) {
  const float w = expf(lse - m);
  return w == 0.f ? 1.4e-45f : w;
}

template <int D>
__global__ __launch_bounds__(kDecodeThreads) void decode_join_kernel(const DecodeAttnLaunch p) {
  constexpr int QUADS = D / 4, SIDE = 64 / QUADS;  // parts read side by side
  constexpr int kAhead = 8;
  __shared__ float wave_m[kDecodeWaves], wave_z[kDecodeWaves];
  __shared__ __attribute__((aligned(16))) f32x4 wave_o[kDecodeWaves][QUADS];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t at = blockIdx.x;
  const int seq = (int)(at / p.h_q), head = (int)(at - (int64_t)seq * p.h_q);
  int first;
  const SeqPart w = parts_of(p.seqs, lane, seq, &first);
  if (w.parts == 1) return;
  const int begin = w.parts * wave / kDecodeWaves, end = w.parts * (wave + 1) / kDecodeWaves;
  const int quad = lane % QUADS, side = lane / QUADS;
  const float* lse = p.ws_lse + (int64_t)first * p.h_q + head;
  const float* o = p.ws_o + ((int64_t)first * p.h_q + head) * D + quad * 4;
  f32x4 v[kAhead];
  auto fetch = [&](int r0) __attribute__((always_inline)) {  // parts r0 + side, ...
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
      v[j] = *reinterpret_cast<const f32x4*>(o + (int64_t)min(r0 + j * SIDE + side, w.parts - 1) * p.h_q * D);
  };
  auto load_lse = [&](int r) { return r < end ? lse[(int64_t)r * p.h_q] : -INFINITY; };
  fetch(begin);
  float lr = load_lse(begin + lane);
  float m = lr;
  for (int r = begin + lane + 64; r < end; r += 64) m = fmaxf(m, load_lse(r));
  m = wave_largest(m);
  float z = 0.f;
  f32x4 acc = f32x4{};
  for (int r0 = begin; r0 < end; r0 += 64) {
    if (r0 > begin) lr = load_lse(r0 + lane);
    const float weight = lr != -INFINITY ? part_weight(lr, m) : 0.f;  // NaN reaches the result
    z += weight;
    const int n = min(64, end - r0);
    for (int i0 = 0; i0 < n; i0 += kAhead * SIDE) {
      if (r0 + i0 > begin) fetch(r0 + i0);
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        // Lanes past the last part hold a weight of 0.
        float f = 0.f;
#pragma unroll
        for (int x = 0; x < SIDE; ++x) {
          const float fx = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(weight), (i0 + j * SIDE + x) & 63));
          f = side == x ? fx : f;
        }
        const bool used = f != 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] = fmaf(used ? f : 0.f, used ? v[j][e] : 0.f, acc[e]);
      }
    }
  }
  z = wave_total(z);
#pragma unroll
  for (int e = 0; e < 4; ++e) acc[e] = SIDE == 2 ? lane_pair_sum(acc[e]) : quad_rows_sum(acc[e]);
  if (lane == 0) {
    wave_m[wave] = m;
    wave_z[wave] = z;
  }
  if (side == 0) wave_o[wave][quad] = acc;
  __syncthreads();
  if (threadIdx.x >= QUADS) return;
  m = wave_m[0];
#pragma unroll
  for (int x = 1; x < kDecodeWaves; ++x) m = fmaxf(m, wave_m[x]);
  z = 0.f;
  acc = f32x4{};
#pragma unroll
  for (int x = 0; x < kDecodeWaves; ++x) {
    // A wavefront without parts, or whose parts have no keys, has a sum of 0 and is left
    // out: not its factor tells, which is next to 0 where a NaN part has left the
    // maximum to the other wavefronts.
    const bool counts = wave_z[x] != 0.f;
    const float f = counts ? part_weight(wave_m[x], m) : 0.f;
    z += counts ? f * wave_z[x] : 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] += counts ? f * wave_o[x][quad][e] : 0.f;
  }
  const float inv = z == 0.f ? 0.f : 1.f / z;
  bf16x4 out;
#pragma unroll
  for (int e = 0; e < 4; ++e) out[e] = (__bf16)(acc[e] * inv);
  *reinterpret_cast<bf16x4*>(p.o + at * D + quad * 4) = out;
  if (quad == 0) p.lse[at] = z == 0.f ? -INFINITY : m + logf(z);
}

template <int D>
void launch(const DecodeAttnLaunch& p, hipStream_t stream) {
  const int64_t work = ((int64_t)p.seqs.items * p.h_kv + 7) / 8 * 8;
  const dim3 grid((unsigned)(work * p.row_blocks)), block(kDecodeThreads);
  if (p.group <= 16 * p.row_blocks) {
    hipLaunchKernelGGL((decode_attn_kernel<D, 1>), grid, block, 0, stream, p);
  } else {
    hipLaunchKernelGGL((decode_attn_kernel<D, 2>), grid, block, 0, stream, p);
  }
  if (!p.may_split) return;
  hipLaunchKernelGGL((decode_join_kernel<D>), dim3((unsigned)(p.seqs.batch * p.h_q)), block, 0, stream, p);
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
  const dim3 grid(p.batch, (chunks + 63) / 64), block(64);
  if (head_dim == 128) {
    hipLaunchKernelGGL(decode_append_kernel<128>, grid, block, 0, stream, p);
  } else {
    hipLaunchKernelGGL(decode_append_kernel<64>, grid, block, 0, stream, p);
  }
  return hipGetLastError();
}

}  // namespace mocap
