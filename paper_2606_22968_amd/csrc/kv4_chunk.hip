// Causal attention of a chunk over the 4-bit store, in full or in a sliding window
// with sinks, for gfx950 (CDNA4).
//
// As window_attn.hip, which see for the walk, the products and the softmax; what is
// different is how a tile comes into LDS:
//   * A 64-key tile is 4 KiB of K and 4 KiB of V codes (d 128) and 512 bytes of
//     scales.  Each of wavefronts 0-3 loads K, 4-7 V, 16 bytes a lane (d 64: 8), a tile
//     ahead in registers; during the step before its own the tile is turned into bf16
//     (exact) and stored in LDS in the layout that the products read.  Every row of the
//     workgroup then uses it, so 256 rows pay for one conversion.
//   * K has two stages, V three (a tile's P*V follows the next tile's scores); one
//     barrier per tile.
//   * A value block that reads as NaN is left to the product where all rows of the
//     workgroup see its tile.  In other tiles its scale is set next to 0, and the rows
//     that see it get NaN in its dims at the end.
// Measured: 2048 tokens of 32/8/128 heads behind 30720, 960 to 1030 us by the card, 1.03 to
// 1.11 PFLOP/s.  Issue bounds it: MFMAs hold 45% of the SIMDs' cycles, a third of those beside
// vector instructions (2.3 GHz).  The conversion is 5.5% of it, half of that the stores to LDS.
// At head_dim 64 a tile has half the MFMAs beside the same exponentials, packing and sums (12 vector
// instructions an MFMA for 6.6, 2 of them exponentials for 1): 2048 tokens of 16/2/64 behind 16384
// 217 to 230 us, 0.64 to 0.67 PFLOP/s, MFMAs busy 26% of the cycles, vector instructions 49%.
// Tried: a table entry looked up a tile ahead (no difference); pieces dealt to the lanes so
// that those stores, 16 lanes over 32 banks, meet no bank twice, with loads 64 bytes apart
// (1% more); the conversion of wavefronts 0-3 or 4-7 between the scores and the products or
// after them (0 to 3% more), of all (10 to 14%).
#include "kv4_device.h"

#include <type_traits>

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

template <int D>
__global__ __launch_bounds__(kAttnThreads, 2) void kv4_chunk_kernel(const Kv4ChunkLaunch launch) {
#if defined(__HIP_DEVICE_COMPILE__)
  const WindowLaunch& p = launch.a;
  constexpr int KS = D / 16;
  constexpr int MD = D / 32;                 // 32-dim blocks
  constexpr int TILE_ELEMS = kTileKeys * D;
  // Where the next tile is turned into bf16: between the MFMAs of this one's scores (from a
  // second set of registers), or ahead of them.  2048 tokens of 32/8/128 heads behind 30720
  // 1030 and 993 us, of 16/2/64 behind 16384 217 and 231: at head_dim 128 a tile's MFMAs
  // are twice as many beside the same exponentials, and take the issue slots.
  constexpr bool kWeave = D == 64;
  constexpr int K_STAGES = 2, V_STAGES = 3;
  // One array: with several, the compiler takes reads of one to depend on writes of another.
  __shared__ __attribute__((aligned(1024))) uint16_t lds[(K_STAGES + V_STAGES) * TILE_ELEMS + 2 * 4];
  int* const found = reinterpret_cast<int*>(lds + (K_STAGES + V_STAGES) * TILE_ELEMS);  // [4]: tile i holds NaN value blocks
  auto k_tile = [&](int i) __attribute__((always_inline)) { return lds + (i % K_STAGES) * TILE_ELEMS; };
  auto v_tile = [&](int i) __attribute__((always_inline)) { return lds + (K_STAGES + i % V_STAGES) * TILE_ELEMS; };

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = lane >> 5;
  const int l32 = lane & 31;
  const int P = p.prefix_len, L = p.chunk_len;

  // Within a KV head: row block, then range; a row block's ranges share no tile, neighbouring
  // row blocks most of them.
  const int logical = xcd_contiguous(blockIdx.x, p.total_wgs);
  const int per_kv = p.row_blocks * p.n_ranges;
  const int kv_head = logical / per_kv;
  const int in_kv = logical - kv_head * per_kv;
  const int range = in_kv / p.row_blocks;
  const int block = in_kv - range * p.row_blocks;

  // Row r of the KV head is token r / G, head r % G.  Wavefronts 0-3 and 4-7 take 128 rows each:
  // neighbouring row groups, the last ones first, or (mirrored) the x-th from either end,
  // the later one for wavefronts 0-3 (its V is more work to convert than K: 60 us for 65),
  // the middle one of an odd count alone.
  const int64_t rows_end = (int64_t)L * p.group;
  constexpr int kGroupRows = kWindowRows / 2;
  const int groups = (int)((rows_end + kGroupRows - 1) / kGroupRows);
  const int low = launch.mirrored ? block : 2 * (p.row_blocks - 1 - block);
  const int high = launch.mirrored ? groups - 1 - block : min(low + 1, groups - 1);
  const int row0 = ((wave < 4) == launch.mirrored ? high : low) * kGroupRows + (wave & 3) * kAttnWaveRows;
  auto token_of = [&](int64_t r) { return (int)div_by((uint32_t)min(r, rows_end - 1), p.group_magic, p.group_shift); };
  const int wg_first = P + token_of((int64_t)low * kGroupRows);
  const int wg_last = P + token_of((int64_t)high * kGroupRows + kGroupRows - 1);
  const int first = P + token_of(row0), last = P + token_of((int64_t)row0 + kAttnWaveRows - 1);
  const bool wave_on = row0 < rows_end && (wave < 4 || low < high);  // (equal: wavefronts 0-3 alone)
  const Tiles tiles = tiles_of(p, wg_first, wg_last), own = tiles_of(p, first, last);
  const int i0 = (int)((int64_t)tiles.count() * range / p.n_ranges);
  const int i1 = (int)((int64_t)tiles.count() * (range + 1) / p.n_ranges);
  // A tile that some row of this wavefront sees.
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

  // A thread's piece of a tile: of wavefronts 0-3 D / 4 dims of a key, of 4-7 D / 8 keys of V row
  // (block, dim), that is of dims 32 block + dim and 16 on.
  const int block_tiles = p.block_size / kTileKeys;
  const uint8_t* const k_pool = reinterpret_cast<const uint8_t*>(p.k_pool);
  const uint8_t* const v_pool = reinterpret_cast<const uint8_t*>(p.v_pool);
  constexpr int WORDS = D / 32;              // of codes, a thread
  constexpr int STEPS = 2 * WORDS;           // of their conversion
  constexpr int TILE_BYTES = kTileKeys * D / 2, SCALE_BYTES = kTileKeys * MD;
  const bool takes_v = wave >= 4;
  const int piece = tid & 255;
  const const_i32_ptr table = (const_i32_ptr)p.table;
  typedef uint32_t words __attribute__((ext_vector_type(WORDS)));
  struct Raw {
    words codes, scales;                     // K: one scale
  } raw, next;  // of the tile to be turned into bf16; kWeave: and of the one after it
  const int k_key = piece / 4, k_part = piece % 4;   // dims D / 4 k_part ..
  constexpr int V_PARTS = 512 / D;
  const int v_row = piece / V_PARTS, v_part = piece % V_PARTS;
  const int scale_at = takes_v ? v_row / 16 * kTileKeys + v_part * (D / 8) : k_part * (D / 4) / 32 * kTileKeys + k_key;
  auto tile_number = [&](int i) __attribute__((always_inline)) {
    const int pos0 = tiles.at(i) * kTileKeys;
    const int lb = (int)div_by((uint32_t)pos0, p.block_magic, p.block_shift);
    return ((int64_t)table[lb] * p.h_kv + kv_head) * block_tiles + (pos0 - lb * p.block_size) / kTileKeys;
  };
  auto fetch = [&](int i, Raw& to) __attribute__((always_inline)) {
    const int64_t t = tile_number(i);
    if (takes_v) {
      to.codes = *reinterpret_cast<const words*>(v_pool + t * TILE_BYTES + piece * (D / 8));
      to.scales = *reinterpret_cast<const words*>(launch.v_scale + t * SCALE_BYTES + scale_at);
    } else {
      to.codes = *reinterpret_cast<const words*>(k_pool + t * TILE_BYTES + piece * (D / 8));
      to.scales[0] = launch.k_scale[t * SCALE_BYTES + scale_at];
    }
  };
  // Where all rows see a whole tile, a NaN value block reaches all of them as NaN; in other
  // tiles it is noted and its scale set next to 0, as are scales of unwritten positions.
  auto set_apart = [&](int i) __attribute__((always_inline)) {
    if (!takes_v || seen_in_full(p, tiles.at(i), wg_first, wg_last)) return;
    uint32_t bad = 0;
#pragma unroll
    for (int w = 0; w < WORDS; ++w) bad |= beyond_252(raw.scales[w]);
    if (bad == 0) return;
    const int behind = wg_last + 1 - tiles.at(i) * kTileKeys - v_part * (D / 8);  // the first byte that no row sees
#pragma unroll
    for (int w = 0; w < WORDS; ++w) {
      const uint32_t b = beyond_252(raw.scales[w]);
      if (b != 0 && w * 4 + __builtin_ctz(b) / 8 < behind) found[i % 4] = 1;
      raw.scales[w] &= ~((b >> 7) * 0xFFu);
    }
  };
  // Turns the fetched codes into bf16 in the stages of tile i, in STEPS steps.
  u32x4 out[2];
  auto k_step = [&](int i, int step) __attribute__((always_inline)) {
    const uint32_t c = raw.codes[step / 2];
    const float s = scale_of(raw.scales[0], 0);
    if (step % 2 == 0) {
      out[0] = u32x4{two_values<0>(c, s), two_values<1>(c, s), two_values<2>(c, s), two_values<3>(c, s)};
    } else {
      *reinterpret_cast<u32x4*>(k_tile(i) + k_key * D + (((k_part * WORDS + step / 2) ^ k_swizzle<D>(k_key)) << 3)) = out[0];
    }
  };
  auto v_step = [&](int i, int step) __attribute__((always_inline)) {
    if (step % 4 < 2) {
      const int w = step % 4;
      const uint32_t v = raw.codes[step / 4 * 2 + w], sc = raw.scales[step / 4 * 2 + w];
      const uint32_t v0 = two_values<0>(v, scale_of(sc, 0)), v1 = two_values<1>(v, scale_of(sc, 1));
      const uint32_t v2 = two_values<2>(v, scale_of(sc, 2)), v3 = two_values<3>(v, scale_of(sc, 3));
      out[0][2 * w] = low_halves(v0, v1);
      out[0][2 * w + 1] = low_halves(v2, v3);
      out[1][2 * w] = high_halves(v0, v1);
      out[1][2 * w + 1] = high_halves(v2, v3);
    } else {
      const int e = v_row / 16 * 32 + v_row % 16 + (step % 4 - 2) * 16;
      *reinterpret_cast<u32x4*>(v_tile(i) + e * kTileKeys + (((v_part * (WORDS / 2) + step / 4) ^ v_swizzle(e)) << 3)) =
          out[step % 4 - 2];
    }
  };
  auto convert = [&](int i) __attribute__((always_inline)) {
    if (takes_v) {
#pragma unroll
      for (int step = 0; step < STEPS; ++step) v_step(i, step);
    } else {
#pragma unroll
      for (int step = 0; step < STEPS; ++step) k_step(i, step);
    }
  };

  f32x16 oacc[MD];
#pragma unroll
  for (int md = 0; md < MD; ++md) oacc[md] = f32x16{};
  float m_run = -INFINITY, l_run = 0.f, f_run = 0.f;
  const float sl2 = p.scale_log2;
  const int k_row_lo = key_row_order(l32);
  const int v_row_sw = v_swizzle(l32);

  // Tile i holds NaN value blocks: the 32-dim blocks in which this lane's row sees one, as bits.
  uint32_t nan_dims = 0;
  auto note_nan = [&](int i) __attribute__((always_inline)) {
    const int k0 = tiles.at(i) * kTileKeys;
    each_nan<MD>(launch.v_scale + tile_number(i) * (MD * kTileKeys), [&](int b, int slot) {
      const int at = k0 + slot;
      if (at <= pos && (at > pos - p.window || at < p.sinks)) nan_dims |= 1u << b;
    });
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
  auto scores = [&](int i, auto with_next) __attribute__((always_inline)) {
    constexpr int NEXT = decltype(with_next)::value;  // 1, 2: turns tile i + 1's K or V into bf16 between the MFMAs
    const uint16_t* kl = k_tile(i);
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
    auto between = [&](int mfma) __attribute__((always_inline)) {
      constexpr int EVERY = 2 * KS / STEPS;
      if (NEXT == 1 && mfma % EVERY == 0) k_step(i + 1, mfma / EVERY);
      if (NEXT == 2 && mfma % EVERY == 0) v_step(i + 1, mfma / EVERY);
    };
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      if (ks + 2 < KS) {
        a0[ks + 2] = kfrag(kr0, ksw0, ks + 2);
        a1[ks + 2] = kfrag(kr1, ksw1, ks + 2);
      }
      s[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a0[ks], qf[ks], s[0], 0, 0, 0);
      between(2 * ks);
      __builtin_amdgcn_sched_barrier(0);
      s[1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a1[ks], qf[ks], s[1], 0, 0, 0);
      between(2 * ks + 1);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  auto mask = [&](int i) __attribute__((always_inline)) {
    const int t = tiles.at(i);
    if (!seen_in_full(p, t, first, last)) {
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
  if (tid < 4) found[tid] = 0;
  __syncthreads();
  if (i0 < i1) {
    fetch(i0, raw);
    set_apart(i0);
    convert(i0);
    if (i0 + 1 < i1) fetch(i0 + 1, kWeave ? next : raw);
    bool pending = false;  // tile i - 1's P*V is still to be made
    for (int i = i0; i < i1; ++i) {
      lds_barrier();
      const bool more = i + 1 < i1;
      if (__builtin_amdgcn_readfirstlane(found[i % 4]) != 0) note_nan(i);
      if (tid == 0) found[(i + 2) % 4] = 0;
      if (kWeave) {
        raw = next;
        if (i + 2 < i1) fetch(i + 2, next);
      }
      if (more) set_apart(i + 1);
      if (!kWeave) {
        if (more) convert(i + 1);
        if (i + 2 < i1) fetch(i + 2, raw);
      }
      const bool on = seen(tiles.at(i));
      if (pending && !on) {
        pv(i - 1);
        pending = false;
      }
      if (!kWeave || !on || !more) {
        if (kWeave && more) convert(i + 1);
        if (!on) continue;
        scores(i, std::integral_constant<int, 0>{});
      } else if (takes_v) {
        scores(i, std::integral_constant<int, 2>{});
      } else {
        scores(i, std::integral_constant<int, 1>{});
      }
      mask(i);
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
  if (!wave_on || row0 + l32 >= rows_end) return;
  const float inv = beyond ? NAN : l_tot > 0.f ? 1.f / l_tot : 0.f;
  const float row_lse = f_tot == 0.f ? -INFINITY : (m_run + log2f(f_tot)) * kLn2;
  const int64_t out_row = (int64_t)token * p.h_q + head;
  const int64_t part_row = (int64_t)range * L * p.h_q + out_row;
#pragma unroll
  for (int md = 0; md < MD; ++md) {
    const float scale = nan_dims >> md & 1 ? NAN : inv;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int dim = md * 32 + j * 8 + half * 4;
      f32x4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[e] = oacc[md][j * 4 + e] * scale;
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

hipError_t launch_kv4_chunk(const Kv4ChunkLaunch& p, int head_dim, hipStream_t stream) {
  const dim3 grid(p.a.total_wgs), block(kAttnThreads);
  if (head_dim == 128) {
    hipLaunchKernelGGL(kv4_chunk_kernel<128>, grid, block, 0, stream, p);
  } else {
    hipLaunchKernelGGL(kv4_chunk_kernel<64>, grid, block, 0, stream, p);
  }
  return hipGetLastError();
}

}  // namespace mocap
