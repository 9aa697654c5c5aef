// Causal attention of a chunk in a sliding window with sinks, for gfx950 (CDNA4).
//
// The row at position t sees keys j <= t with j < sinks or j > t - window:
//   s_j = scale <q, k_j>,  lse = ln sum_j exp s_j,  o = sum_j exp(s_j - lse) v_j
// Long chunks are bound by the matrix unit and the softmax beside it, short ones
// by the walk over their tiles.
//
//   * A workgroup owns 256 consecutive rows of a KV head ((token, query head)
//     pairs in token-major order), 32 per wavefront, and walks the 64-key tiles
//     that any of them sees: the sinks' tiles, then the window's.  256 rows of a
//     group of 4 lie on 64 tokens, so a window of W keys costs W / 64 + 2 tiles at
//     most; tiles that no row of a wavefront sees are left out by it.
//   * Every workgroup has about the same number of tiles (the window's), so no
//     pairing of long and short ones is needed.  Where workgroups are too few,
//     the tiles are cut into ranges that lse_merge.hip joins.
//   * K/V tiles go straight to a 4-stage LDS ring, two tiles ahead, even ones
//     copied by wavefronts 0-3 and odd ones by 4-7; one barrier per tile.
//   * Products, softmax bookkeeping and outputs are those of chunk_attn.hip:
//     S^T = K Q^T and O^T += V^T P^T with v_mfma_f32_32x32x16_bf16, the
//     probabilities rounded to bf16 (their bf16 sum normalises O, the fp32 sum of
//     the exponentials gives the LSE).  A layer's windowed and full rows then have
//     one precision (O 0.0023 of its norm from 64 bits; 0.0017, its own rounding, with
//     exact probabilities), and a low part beside them, as in decode_attn.hip, would
//     double the P*V products of a kernel that is bound by issue.
//   * A wavefront makes tile k's scores, then tile k - 1's P*V with tile k's
//     exponentials, packing and row sums woven in between the MFMAs.
//   * Tiles that some row of the workgroup does not see in full are masked.  A
//     hidden key's probability is exactly 0, but 0 times a NaN or infinite value
//     is NaN: such tiles are searched for non-finite values as they arrive, and
//     where there are any (never, in ordinary use) they are left out of the
//     product, and the rows that see them receive them in the end.
// Measured: 2048 tokens of 32/8/128 heads in a window of 4096, 141 us, 974 TFLOP/s
// over visible pairs, one workgroup per compute unit; 2 us a tile and 10 us fixed
// (first copies, the masked ends, outputs).  The matrix unit is busy 43% of the
// time, and vector work runs beside it for a third of that: issue bounds it.
#include "attn_device.h"
#include "serve.h"

namespace mocap {
namespace {

template <int D>
__device__ __forceinline__ int k_swizzle(int r) {
  return D == 128 ? (r & 15) : ((r >> 1) & 7);
}
__device__ __forceinline__ int v_swizzle(int e) { return (e >> 1) & 7; }

__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
  __builtin_amdgcn_s_barrier();
}

__device__ __forceinline__ uint32_t div_by(uint32_t n, uint32_t magic, int shift) {
  return (__umulhi(n, magic) + n) >> shift;
}

// A 16-bit word of a packed pair is NaN or infinite where its exponent is all ones.
__device__ __forceinline__ bool nonfinite(uint32_t x) { return (x & 0x7F80u) == 0x7F80u; }

// The tiles of a run of rows at positions [first, last]: the sinks' [0, sinks),
// then [begin, end).
struct Tiles {
  int sinks, begin, end;
  __device__ __forceinline__ int count() const { return sinks + end - begin; }
  __device__ __forceinline__ int at(int i) const { return i < sinks ? i : i - sinks + begin; }
};
__device__ __forceinline__ Tiles tiles_of(const WindowLaunch& p, int first, int last) {
  const int low = max(0, first - p.window + 1);
  Tiles t;
  t.begin = low / kTileKeys;
  t.end = last / kTileKeys + 1;
  t.sinks = min((min(p.sinks, low) + kTileKeys - 1) / kTileKeys, t.begin);
  return t;
}

template <int D>
__global__ __launch_bounds__(kAttnThreads, 2) void window_attn_kernel(const WindowLaunch p) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int KS = D / 16;
  constexpr int MD = D / 32;
  constexpr int K_ROW_CHUNKS = D / 8;
  constexpr int V_ROW_CHUNKS = kTileKeys / 8;
  constexpr int K_ELEMS = kTileKeys * D;
  constexpr int BUF_ELEMS = 2 * K_ELEMS;
  constexpr int LOADS = K_ELEMS / 8 / (kAttnThreads / 2);
  constexpr int STAGES = 4;
  // One array for the ring and what lies beside it: with several, the compiler
  // tells them apart, takes every read of the ring to depend on the copies in
  // flight, and waits for those (143 instead of 141 us for 2048 tokens in a window
  // of 4096).
  constexpr int ROW_BITS = kWindowRows * MD;  // words
  __shared__ __attribute__((aligned(1024))) uint16_t lds[STAGES * BUF_ELEMS + 2 * (STAGES + 2 * ROW_BITS)];
  int* const found = reinterpret_cast<int*>(lds + STAGES * BUF_ELEMS);  // the stage's tile holds non-finite values
  // Dims of the workgroup's rows that receive +infinity or -infinity (NaN: both), as bits.
  uint32_t* const plus = reinterpret_cast<uint32_t*>(found + STAGES);
  uint32_t* const minus = plus + ROW_BITS;

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = lane >> 5;
  const int l32 = lane & 31;
  const int P = p.prefix_len, L = p.chunk_len;

  // Within a KV head: row block (the last ones first), then range; a row block's
  // ranges share no tile, neighbouring row blocks most of them.
  const int logical = xcd_contiguous(blockIdx.x, p.total_wgs);
  const int per_kv = p.row_blocks * p.n_ranges;
  const int kv_head = logical / per_kv;
  const int in_kv = logical - kv_head * per_kv;
  const int range = in_kv / p.row_blocks;
  const int block = p.row_blocks - 1 - (in_kv - range * p.row_blocks);

  // Row r of the KV head is token r / G, head r % G.  The workgroup's and the
  // wavefront's positions.
  const int64_t rows_end = (int64_t)L * p.group;
  const int wg_row0 = block * kWindowRows, row0 = wg_row0 + wave * kAttnWaveRows;
  auto token_of = [&](int64_t r) { return (int)div_by((uint32_t)min(r, rows_end - 1), p.group_magic, p.group_shift); };
  const int wg_first = P + token_of(wg_row0), wg_last = P + token_of((int64_t)wg_row0 + kWindowRows - 1);
  const int first = P + token_of(row0), last = P + token_of((int64_t)row0 + kAttnWaveRows - 1);
  const bool wave_on = row0 < rows_end;
  const Tiles tiles = tiles_of(p, wg_first, wg_last), own = tiles_of(p, first, last);
  const int i0 = (int)((int64_t)tiles.count() * range / p.n_ranges);
  const int i1 = (int)((int64_t)tiles.count() * (range + 1) / p.n_ranges);
  // A tile that all rows of [a, b] see in full; one that some row of this wavefront sees.
  auto full_for = [&](int t, int a, int b) __attribute__((always_inline)) -> bool {
    const int k0 = t * kTileKeys, k1 = k0 + kTileKeys;
    return k1 <= a + 1 && (k0 > b - p.window || k1 <= p.sinks);
  };
  auto seen = [&](int t) __attribute__((always_inline)) -> bool {
    return wave_on && (t < own.sinks || (t >= own.begin && t < own.end));
  };

  // This lane's row: its token, and its head of the group.  Lanes past the last
  // row take the last; nothing of theirs is stored.
  const int lane_r = (int)min((int64_t)row0 + l32, rows_end - 1);
  const int token = token_of(lane_r);
  const int head = kv_head * p.group + lane_r - token * p.group;
  const int pos = P + token;

  bf16x8 qf[KS];
  {
    const uint16_t* qrow = p.q + ((int64_t)token * p.h_q + head) * D + half * 8;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = *reinterpret_cast<const bf16x8*>(qrow + ks * 16);
  }

  // Copies (see chunk_attn.hip): copy j moves 16-byte chunk (j * 4 + gwave) * 64 + lane.
  const int64_t head_stride = (int64_t)D * p.block_size;
  const int my_group = wave >> 2, gwave = wave & 3;
  int k_src, v_src;
  {
    const int chunk = gwave * 64 + lane;
    const int kr = chunk / K_ROW_CHUNKS, kc = (chunk % K_ROW_CHUNKS) ^ k_swizzle<D>(kr);
    k_src = (kr * D + kc * 8) * 2;
    const int vr = chunk / V_ROW_CHUNKS, vc = (chunk % V_ROW_CHUNKS) ^ v_swizzle(vr);
    v_src = (vr * p.block_size + vc * 8) * 2;
  }
  constexpr int K_ROWS_PER_COPY = kAttnThreads / 2 / K_ROW_CHUNKS;
  constexpr int V_ROWS_PER_COPY = kAttnThreads / 2 / V_ROW_CHUNKS;
  const const_i32_ptr table = (const_i32_ptr)p.table;
  auto issue = [&](int i) __attribute__((always_inline)) {
    if ((i & 1) != my_group) return;
    const int pos0 = tiles.at(i) * kTileKeys;
    const int lb = (int)div_by((uint32_t)pos0, p.block_magic, p.block_shift);
    const int slot0 = pos0 - lb * p.block_size;
    const int64_t base = ((int64_t)table[lb] * p.h_kv + kv_head) * head_stride;
    const uint16_t* kb = p.k_pool + base + (int64_t)slot0 * D;
    const uint16_t* vb = p.v_pool + base + slot0;
    uint16_t* kl = lds + (i % STAGES) * BUF_ELEMS;
    uint16_t* vl = kl + K_ELEMS;
    const __amdgpu_buffer_rsrc_t kr = __builtin_amdgcn_make_buffer_rsrc((void*)kb, 0, -1, kBufferWord3);
    const __amdgpu_buffer_rsrc_t vr = __builtin_amdgcn_make_buffer_rsrc((void*)vb, 0, -1, kBufferWord3);
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      const int dst = (j * 4 + gwave) * 64 * 8;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(kr, (lds_ptr_t)(kl + dst), 16, k_src, j * K_ROWS_PER_COPY * D * 2, 0, 0);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(vr, (lds_ptr_t)(vl + dst), 16, v_src,
                                               j * V_ROWS_PER_COPY * p.block_size * 2, 0, 0);
    }
  };
  const int valid_end = P + L;
  // Tile i is published: its copies are complete, and every wavefront is done
  // with tile i - 1.  True if the tile holds non-finite values that some row may
  // not see.
  auto publish = [&](int i) __attribute__((always_inline)) -> bool {
    if ((i & 1) == my_group) wait_vmem<0>();
    const int t = tiles.at(i), stage = i % STAGES;
    const bool search = !full_for(t, wg_first, wg_last);
    if (search && tid == 0) found[stage] = 0;
    lds_barrier();
    if (!search) return false;
    // Unwritten store memory becomes 0.
    u32x4* vl = reinterpret_cast<u32x4*>(lds + stage * BUF_ELEMS + K_ELEMS);
    bool bad = false;
    for (int c = tid; c < K_ELEMS / 8; c += kAttnThreads) {
      const int e = c / V_ROW_CHUNKS, key0 = t * kTileKeys + ((c % V_ROW_CHUNKS) ^ v_swizzle(e)) * 8;
      u32x4 x = vl[c];
      if (key0 + 8 > valid_end) {
#pragma unroll
        for (int w = 0; w < 4; ++w)
          x[w] &= (key0 + 2 * w < valid_end ? 0x0000FFFFu : 0u) | (key0 + 2 * w + 1 < valid_end ? 0xFFFF0000u : 0u);
        vl[c] = x;
      }
#pragma unroll
      for (int w = 0; w < 4; ++w) bad |= nonfinite(x[w]) || nonfinite(x[w] >> 16);
    }
    if (bad) found[stage] = 1;
    lds_barrier();
    return __builtin_amdgcn_readfirstlane(found[stage]) != 0;
  };

  f32x16 oacc[MD];
#pragma unroll
  for (int md = 0; md < MD; ++md) oacc[md] = f32x16{};
  float m_run = -INFINITY, l_run = 0.f, f_run = 0.f;
  const float sl2 = p.scale_log2;
  const int k_row_lo = key_row_order(l32);
  const int v_row_sw = v_swizzle(l32);

  // Tile i holds non-finite values: which dims of which rows receive one from a
  // key they see is noted, and in LDS the values become 0.  A lane notes half of
  // its row's dims.  Every wavefront calls this for the same tiles.
  bool apart = false;
  const int row_bits = (wave * kAttnWaveRows + l32) * MD;
  auto set_apart = [&](int i) __attribute__((always_inline)) {
    uint16_t* vl = lds + (i % STAGES) * BUF_ELEMS + K_ELEMS;
    const int k0 = tiles.at(i) * kTileKeys;
#pragma unroll 1
    for (int x = half * (MD / 2); x < (half + 1) * (MD / 2); ++x) {
      uint32_t up = apart ? plus[row_bits + x] : 0u;
      uint32_t down = apart ? minus[row_bits + x] : 0u;
#pragma unroll 1
      for (int bit = 0; bit < 32; ++bit) {
        const int e = x * 32 + bit;
#pragma unroll 1
        for (int key = 0; key < kTileKeys; ++key) {
          const int at = k0 + key;
          const bool sees = at <= pos && (at > pos - p.window || at < p.sinks);
          const uint32_t v = vl[e * kTileKeys + (((key >> 3) ^ v_swizzle(e)) << 3) + (key & 7)];
          if (sees && nonfinite(v)) {
            const bool nan = (v & 0x7Fu) != 0;
            up |= (nan || !(v >> 15) ? 1u : 0u) << bit;
            down |= (nan || v >> 15 ? 1u : 0u) << bit;
          }
        }
      }
      plus[row_bits + x] = up;
      minus[row_bits + x] = down;
    }
    apart = true;
    lds_barrier();
    for (int c = tid; c < K_ELEMS / 2; c += kAttnThreads) {
      uint32_t* x = reinterpret_cast<uint32_t*>(vl) + c;
      *x &= (nonfinite(*x) ? 0u : 0x0000FFFFu) | (nonfinite(*x >> 16) ? 0u : 0xFFFF0000u);
    }
    lds_barrier();
  };

  // Visible keys of this lane's 16 of a 32-key half: keys base + {0..7, 16..23}, as bits.
  auto visible_bits = [&](int base) __attribute__((always_inline)) -> uint32_t {
    auto below = [&](int x) {  // keys below x
      x -= base;
      const int n = x <= 0 ? 0 : x <= 8 ? x : x <= 16 ? 8 : x <= 24 ? x - 8 : 16;
      return (1u << n) - 1u;
    };
    return below(pos + 1) & (~below(max(pos - p.window + 1, 0)) | below(p.sinks));
  };

  // Scores of tile i, all MFMAs, K fragments read two k-steps ahead.
  f32x16 s[2];
  uint32_t pk[16];          // probabilities in pairs: pair 8 sb + j holds scores 2 j, 2 j + 1 of half sb
  float rs[2], fs[2];       // per 32-key half: sums of the rounded probabilities, of the exponentials
  auto scores = [&](int i) __attribute__((always_inline)) {
    const int t = tiles.at(i);
    const uint16_t* kl = lds + (i % STAGES) * BUF_ELEMS;
    const int kr0 = k_row_lo, kr1 = 32 + k_row_lo;
    const int ksw0 = k_swizzle<D>(kr0), ksw1 = k_swizzle<D>(kr1);
    auto kfrag = [&](int kr, int ksw, int ks) __attribute__((always_inline)) {
      return *reinterpret_cast<const bf16x8*>(kl + kr * D + (((ks * 2 + half) ^ ksw) << 3));
    };
    bf16x8 a0[KS], a1[KS];
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      a0[ks] = kfrag(kr0, ksw0, ks);
      a1[ks] = kfrag(kr1, ksw1, ks);
    }
    s[0] = s[1] = f32x16{};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      if (ks + 2 < KS) {
        a0[ks + 2] = kfrag(kr0, ksw0, ks + 2);
        a1[ks + 2] = kfrag(kr1, ksw1, ks + 2);
      }
      s[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a0[ks], qf[ks], s[0], 0, 0, 0);
      s[1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a1[ks], qf[ks], s[1], 0, 0, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x100, 4, 1);  // LDS reads
#pragma unroll
    for (int k = 0; k < 2 * KS; ++k) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 1);  // MFMA
      if (k + 4 < 2 * KS) __builtin_amdgcn_sched_group_barrier(0x100, 1, 1);
    }
    if (!full_for(t, first, last)) {
#pragma unroll
      for (int sb = 0; sb < 2; ++sb) {
        const uint32_t vm = visible_bits(t * kTileKeys + sb * 32 + half * 8);
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const int keep = __builtin_amdgcn_sbfe((int)vm, j, 1);
          s[sb][j] = __int_as_float((__float_as_int(s[sb][j]) & keep) | (~keep & (int)0xFF800000u));
        }
      }
    }
  };
  auto probs = [&](float neg_m) __attribute__((always_inline)) {
#pragma unroll
    for (int sb = 0; sb < 2; ++sb) {
      float fa = 0.f, acc = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float e0 = __builtin_amdgcn_exp2f(fmaf(s[sb][2 * j], sl2, neg_m));
        const float e1 = __builtin_amdgcn_exp2f(fmaf(s[sb][2 * j + 1], sl2, neg_m));
        pk[sb * 8 + j] = pack_bf16x2(e0, e1);
        fa += e0 + e1;
        acc = dot2_bf16(pk[sb * 8 + j], 0x3F803F80u, acc);
      }
      fs[sb] = fa;
      rs[sb] = acc;
    }
  };
  // Raises the reference exponents of rows that need it (see attn_device.h).
  auto settle = [&]() __attribute__((always_inline)) {
    const bool over = !(rs[0] <= kSumLimit) || !(rs[1] <= kSumLimit);
    if (__builtin_amdgcn_ballot_w64(over) != 0) {
      const bool row_over = lane_pair_max(over ? 1.f : 0.f) > 0.f;
      float mx = -INFINITY;
#pragma unroll
      for (int sb = 0; sb < 2; ++sb)
#pragma unroll
        for (int j = 0; j < 16; ++j) mx = fmaxf(mx, s[sb][j]);
      mx = lane_pair_max(mx) * sl2;
      if (row_over) {
        if (lane_pair_sum(l_run) != 0.f) {
          const float f = __builtin_amdgcn_exp2f(m_run - mx);
#pragma unroll
          for (int md = 0; md < MD; ++md) oacc[md] *= f;
          l_run *= f;
          f_run *= f;
        }
        m_run = mx;
        probs(m_run == -INFINITY ? 0.f : -m_run);
      }
    }
    l_run += rs[0] + rs[1];
    f_run += fs[0] + fs[1];
  };
  // P*V takes the keys 16 at a time (quad q = pairs 4 q .. 4 q + 3) for each
  // 32-dim block: MFMA k is quad k / MD, block k % MD.
  constexpr int NF = 4 * MD;
  auto vfrag = [&](const uint16_t* vl, int k) __attribute__((always_inline)) {
    const int q = k / MD, md = k % MD;
    return *reinterpret_cast<const bf16x8*>(vl + (md * 32 + l32) * kTileKeys + (((q * 2 + half) ^ v_row_sw) << 3));
  };
  auto pfrag = [&](int k) __attribute__((always_inline)) {
    const int q = k / MD * 4;
    return __builtin_bit_cast(bf16x8, u32x4{pk[q], pk[q + 1], pk[q + 2], pk[q + 3]});
  };
  auto v_tile = [&](int i) __attribute__((always_inline)) { return lds + (i % STAGES) * BUF_ELEMS + K_ELEMS; };
  // Tile i's P*V alone.
  auto pv = [&](int i) __attribute__((always_inline)) {
    constexpr int AHEAD = 3;
    const uint16_t* vl = v_tile(i);
    bf16x8 vf[AHEAD + 1];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) vf[k] = vfrag(vl, k);
#pragma unroll
    for (int k = 0; k < NF; ++k) {
      if (k + AHEAD < NF) vf[(k + AHEAD) % (AHEAD + 1)] = vfrag(vl, k + AHEAD);
      oacc[k % MD] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[k % (AHEAD + 1)], pfrag(k), oacc[k % MD], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // Tile i's P*V with the next tile's probabilities (from s) woven in after the
  // MFMAs, in place: a pair is packed four pairs after its exponentials, when the
  // MFMAs of the quad it replaces are issued, and summed two pairs later.
  auto pv_probs = [&](int i, float neg_m) __attribute__((always_inline)) {
    constexpr int AHEAD = 2, NPAIRS = 16, PAIRS = NPAIRS / NF, LAG_PACK = 4, LAG_SUM = 6;
    static_assert(PAIRS * NF == NPAIRS, "whole pairs per MFMA");
    const uint16_t* vl = v_tile(i);
    bf16x8 vf[AHEAD + 1];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) vf[k] = vfrag(vl, k);
    float acc[2] = {0.f, 0.f}, facc[2] = {0.f, 0.f};
    float ex[NPAIRS][2];
    auto trail = [&](int pr) __attribute__((always_inline)) {
      if (pr >= LAG_PACK && pr - LAG_PACK < NPAIRS) {
        const int x = pr - LAG_PACK;
        pk[x] = pack_bf16x2(ex[x][0], ex[x][1]);
      }
      if (pr >= LAG_SUM) {
        const int x = pr - LAG_SUM;
        acc[x / 8] = dot2_bf16(pk[x], 0x3F803F80u, acc[x / 8]);
        facc[x / 8] += ex[x][0] + ex[x][1];
      }
    };
#pragma unroll
    for (int k = 0; k < NF; ++k) {
      if (k + AHEAD < NF) vf[(k + AHEAD) % (AHEAD + 1)] = vfrag(vl, k + AHEAD);
      oacc[k % MD] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[k % (AHEAD + 1)], pfrag(k), oacc[k % MD], 0, 0, 0);
#pragma unroll
      for (int x = 0; x < PAIRS; ++x) {
        const int pr = k * PAIRS + x;
        ex[pr][0] = __builtin_amdgcn_exp2f(fmaf(s[pr / 8][pr % 8 * 2], sl2, neg_m));
        ex[pr][1] = __builtin_amdgcn_exp2f(fmaf(s[pr / 8][pr % 8 * 2 + 1], sl2, neg_m));
        trail(pr);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int pr = NPAIRS; pr < NPAIRS + LAG_SUM; ++pr) trail(pr);
#pragma unroll
    for (int sb = 0; sb < 2; ++sb) {
      rs[sb] = acc[sb];
      fs[sb] = facc[sb];
    }
  };
  // Tile by tile: its scores, then the tile before's P*V with its probabilities
  // woven in.  A tile that this wavefront does not see ends the chain: the tile
  // before's P*V is made alone (its stage is refilled after the next barrier),
  // and the next tile begins a new one.
  if (i0 < i1) {
    issue(i0);
    if (i0 + 1 < i1) issue(i0 + 1);
    bool pending = false;  // tile i - 1's P*V is still to be made
    for (int i = i0; i < i1; ++i) {
      if (publish(i)) set_apart(i);
      if (i + 2 < i1) issue(i + 2);
      const bool on = seen(tiles.at(i));
      if (pending && !on) {
        pv(i - 1);
        pending = false;
      }
      if (!on) continue;
      scores(i);
      if (pending) {
        pv_probs(i - 1, -m_run);
      } else {
        probs(-m_run);
      }
      settle();
      pending = true;
    }
    if (pending) pv(i1 - 1);
  }

  // A score whose product with the scale is beyond fp32 makes every exponential 0, its
  // own too; the row is NaN, as with an infinite score.
  const bool beyond = m_run == INFINITY;
  const float l_tot = lane_pair_sum(l_run), f_tot = beyond ? NAN : lane_pair_sum(f_run);
  if (row0 + l32 >= rows_end) return;
  const float inv = beyond ? NAN : l_tot > 0.f ? 1.f / l_tot : 0.f;
  const float row_lse = f_tot == 0.f ? -INFINITY : (m_run + log2f(f_tot)) * kLn2;
  const int64_t out_row = (int64_t)token * p.h_q + head;
  const int64_t part_row = (int64_t)range * L * p.h_q + out_row;
#pragma unroll
  for (int md = 0; md < MD; ++md) {
    const uint32_t up = apart ? plus[row_bits + md] : 0u;
    const uint32_t down = apart ? minus[row_bits + md] : 0u;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int dim = md * 32 + j * 8 + half * 4;
      f32x4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[e] = oacc[md][j * 4 + e] * inv;
        const int bit = j * 8 + half * 4 + e;
        if (up >> bit & 1) v[e] += INFINITY;
        if (down >> bit & 1) v[e] -= INFINITY;
      }
      if (p.n_ranges == 1) {
        bf16x4 x;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = (__bf16)v[e];
        *reinterpret_cast<bf16x4*>(p.o + out_row * D + dim) = x;
      } else {
        *reinterpret_cast<f32x4*>(p.ws_o + part_row * D + dim) = v;
      }
    }
  }
  if (half == 0) {
    if (p.n_ranges == 1) {
      p.lse[(int64_t)head * L + token] = row_lse;
    } else {
      p.ws_lse[part_row] = row_lse;
    }
  }
#endif  // __HIP_DEVICE_COMPILE__
}

}  // namespace

hipError_t launch_window_attn(const WindowLaunch& p, int head_dim, hipStream_t stream) {
  const dim3 grid(p.total_wgs), block(kAttnThreads);
  if (head_dim == 128) {
    hipLaunchKernelGGL(window_attn_kernel<128>, grid, block, 0, stream, p);
  } else {
    hipLaunchKernelGGL(window_attn_kernel<64>, grid, block, 0, stream, p);
  }
  return hipGetLastError();
}

}  // namespace mocap
