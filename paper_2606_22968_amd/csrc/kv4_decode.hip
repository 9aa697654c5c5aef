// Decoding over the 4-bit store for gfx950 (CDNA4): the attention of one token per
// sequence, decode_attn.hip's over keys and values of 4.25 bits; and of a chunk's few rows, which
// are then as many heads of one token, each with its own last key.
//
// A key or value of d dims is d / 2 + d / 32 bytes and 4 d G FLOP for the G query
// heads of a group: HBM bounds groups of up to 16 heads still, at 3.8 times the keys a second.
// Larger groups are bound by issue: each 16 or 32 of their heads load and convert a tile again,
// and one wavefront carries that, the exponentials and the doubled P V product of its tile.
//
//   * How work is cut, the products, the softmax and the join are decode_attn.hip's:
//     the fp4 values become bf16 in registers (exact), and enter the same bf16 MFMAs.
//     (The scaled fp4 x fp8 MFMA would take K as it is, and q as the sum of two fp8
//     values, but sums only to 2^-14 of its terms' magnitudes.)
//   * A lane's share of a K row is d / 4 consecutive dims, with one scale, and the
//     query's dims are taken in the same order: one 16-byte load (d 128) a product.
//   * K rows m of product h are keys 16 (m / 4) + 4 h + m % 4 of the tile, so lane group
//     g holds the scores of keys 16 g .. + 15, in order over the four products.  That
//     is what a 16-byte load of a V row gives it: 16 keys of dims 32 b + i and
//     32 b + 16 + i, one byte a key, which with that key's scale become a pair.
// Measured: four sequences of 65537 to 131072 positions, 64/8/128 heads, 452 MB in 85 to 89 us,
// 5.3 TB/s, 5.9 without the 6 us that a launch of one tile a wavefront takes; 32 of up to
// 8192, 32/8/128, 23 us for 83 MB; one of 2048, 6 us.  HBM and that latency bound it:
// without V's conversion it takes 3% less, without the low halves of the probabilities 2%.
// 32 of 32768 in larger groups, us and what their bytes take: 32/1/128 50 and 28, 64/1/128 75 and 28, 64/1/64
// 51 and 14, 128/2/64 88 and 28, 64/2/128 83 and 56.
// Tried: the next tile's codes in a second set of registers (two wavefronts a SIMD, 89
// us), 1 to 9 workgroups per compute unit, parts of whole turns of the four wavefronts, 128
// registers and four wavefronts a SIMD (6 to 37 of them spilled: 117 to 158 us), Q in LDS,
// V's scales loaded once for 16 lanes (none faster than +-3%).
#include "kv4_device.h"
#include "serve_device.h"

#include <type_traits>

namespace mocap {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;

// NT: 16-row blocks that a workgroup takes (1 or 2: see cache_api.cpp).  Rows are the heads of a sequence's group, or
// (CHUNK) those of all tokens of a chunk, row r token r / G.  (CHUNK with NT 2 keeps 39 scalar values, at head_dim 64
// 45, in lanes of vector registers.)
template <int D, int NT, bool CHUNK>
__global__ __launch_bounds__(kThreads) void kv4_rows_kernel(
    const typename std::conditional<CHUNK, Kv4ChunkLaunch, Kv4DecodeLaunch>::type launch) {
#if defined(__HIP_DEVICE_COMPILE__)
  const auto& p = launch.a;
  constexpr int KS = D / 32;   // k-steps of a score product
  constexpr int B = D / 32;    // blocks of 32 dims
  constexpr int MD = D / 16;   // 16-dim blocks of O
  constexpr int KW = D / 32;   // words of a lane's share of a K row
  __shared__ __attribute__((aligned(16))) float part_o[kWaves][NT * 16][D];
  __shared__ float part_m[kWaves][NT * 16], part_l[kWaves][NT * 16];

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, g4 = lane >> 4;

  // Logical order: item (a sequence's part, or a range of the chunk's tiles), KV head.  The blocks
  // of rows that read the same keys are 8 workgroups apart, on one XCD, or (a chunk) as many as
  // there are items and heads, the last rows first: on 8 / gcd(8, that) XCDs, each with late
  // and early rows (a contiguous share of all for each XCD: 80 us for 2882 tokens of 12/4/128
  // without a prefix).
  int work, row0;  // (row0: of the KV head)
  if constexpr (CHUNK) {
    const int works = p.n_ranges * p.h_kv, block = blockIdx.x / works;
    work = blockIdx.x - block * works;
    row0 = (p.row_blocks - 1 - block) * (NT * 16);
  } else {
    const int stripe = blockIdx.x / (8 * p.row_blocks), in_stripe = blockIdx.x - stripe * 8 * p.row_blocks;
    work = stripe * 8 + (in_stripe & 7);
    row0 = (in_stripe >> 3) * (NT * 16);
  }
  const int item = work / p.h_kv;
  const int kv_head = work - item * p.h_kv;
  SeqPart w;         // of a batch
  Tiles chunk;       // of a chunk's rows, at positions first to last
  int begin, end, rows, first = 0, last = 0;
  const_i32_ptr table;
  int bs, block_shift;
  uint32_t block_magic;
  // Row r's token of the chunk; its row of Q and O.
  auto token_of = [&](int row) __attribute__((always_inline)) {
    if constexpr (CHUNK) return (int)div_by((uint32_t)min(row, rows - 1), p.group_magic, p.group_shift);
    return 0;
  };
  auto out_row = [&](int row) __attribute__((always_inline)) -> int64_t {
    if constexpr (CHUNK) {
      const int token = token_of(row);
      return (int64_t)token * p.h_q + kv_head * p.group + row - token * p.group;
    } else {
      return (int64_t)w.seq * p.h_q + kv_head * p.group + row;
    }
  };
  if constexpr (CHUNK) {
    rows = p.chunk_len * p.group;
    first = p.prefix_len + token_of(row0);
    last = p.prefix_len + token_of(row0 + NT * 16 - 1);
    chunk = tiles_of(p, first, last);
    begin = (int)((int64_t)chunk.count() * item / p.n_ranges);
    end = (int)((int64_t)chunk.count() * (item + 1) / p.n_ranges);
    table = (const_i32_ptr)p.table;
    bs = p.block_size, block_magic = p.block_magic, block_shift = p.block_shift;
  } else {
    if (item >= p.seqs.items) return;
    w = locate_item(p.seqs, lane, item);
    if (w.seq == p.seqs.batch) return;
    part_range_longer_first(w, &begin, &end);
    rows = p.group;
    table = (const_i32_ptr)(p.seqs.tables + w.seq * p.seqs.table_stride);
    bs = p.seqs.block_size, block_magic = p.seqs.block_magic, block_shift = p.seqs.block_shift;
  }
  // Tile i of the part or range.
  auto tile_of = [&](int i) __attribute__((always_inline)) {
    if constexpr (CHUNK) {
      return chunk.at(begin + i);
    } else {
      return w.span.tile(begin + i);
    }
  };

  // Q as the B operand: lane l holds row l % 16, dims D / 4 (l / 16) + 8 ks .. + 7.
  // Lanes past the last row take that row; nothing of theirs is stored.
  bf16x8 qf[NT][KS];
  int pos[NT];  // the row's position (CHUNK)
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int at = min(row0 + t * 16 + l16, rows - 1);
    if constexpr (CHUNK) pos[t] = p.prefix_len + token_of(at);
    const uint16_t* row = p.q + out_row(at) * D + g4 * (D / 4);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[t][ks] = *reinterpret_cast<const bf16x8*>(row + ks * 8);
  }

  const int block_tiles = bs / kTileKeys;
  const uint8_t* const k_pool = reinterpret_cast<const uint8_t*>(p.k_pool);
  const uint8_t* const v_pool = reinterpret_cast<const uint8_t*>(p.v_pool);
  const int k_lane = (16 * (l16 >> 2) + (l16 & 3)) * (D / 2) + g4 * (D / 8);
  const int k_scale_lane = g4 * (D / 4) / 32 * kTileKeys + 16 * (l16 >> 2);
  const int v_lane = l16 * kTileKeys + g4 * 16;
  const int v_scale_lane = g4 * 16;

  // A tile's codes and scales.
  typedef uint32_t k_words __attribute__((ext_vector_type(KW)));
  struct {
    k_words k[4];       // by product
    u32x4 k_scale;      // word h: byte l % 4 is product h's
    u32x4 v[B], v_scale[B];
  } raw;
  // The number of tile i of the part in [blocks][Hkv][bs / 64].
  auto tile_at = [&](int i) __attribute__((always_inline)) {
    const int key0 = tile_of(i) * kTileKeys;
    const int lb = (int)div_by((uint32_t)key0, block_magic, block_shift);
    return ((int64_t)table[lb] * p.h_kv + kv_head) * block_tiles + (key0 - lb * bs) / kTileKeys;
  };
  auto fetch_k = [&](int64_t tile) __attribute__((always_inline)) {
    const uint8_t* src = k_pool + tile * (kTileKeys * D / 2) + k_lane;
#pragma unroll
    for (int h = 0; h < 4; ++h) raw.k[h] = *reinterpret_cast<const k_words*>(src + h * 4 * (D / 2));
    raw.k_scale = *reinterpret_cast<const u32x4*>(launch.k_scale + tile * (B * kTileKeys) + k_scale_lane);
  };
  auto fetch_v = [&](int64_t tile) __attribute__((always_inline)) {
    const uint8_t* src = v_pool + tile * (kTileKeys * D / 2) + v_lane;
    const uint8_t* scales = launch.v_scale + tile * (B * kTileKeys) + v_scale_lane;
#pragma unroll
    for (int b = 0; b < B; ++b) {
      raw.v[b] = *reinterpret_cast<const u32x4*>(src + b * 16 * kTileKeys);
      raw.v_scale[b] = *reinterpret_cast<const u32x4*>(scales + b * kTileKeys);
    }
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

  // CHUNK: hides keys that a row does not see.  A tile's NaN value blocks would reach all rows
  // of the product: their scales are set next to 0, and rows that see one are noted.
  uint32_t nan_dims[NT] = {};
  auto mask_chunk = [&](int i, int key0, f32x4 (&s)[NT][4]) __attribute__((always_inline)) {
    if constexpr (CHUNK) {
      const int base = key0 + g4 * 16;
      auto below = [&](int x) { return (1u << min(max(x - base, 0), 16)) - 1u; };  // keys below x, as bits
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const uint32_t seen = below(pos[t] + 1) & (~below(max(pos[t] - p.window + 1, 0)) | below(p.sinks));
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float x = s[t][e >> 2][e & 3];
          if constexpr (NT == 1) {
            const int keep = __builtin_amdgcn_sbfe((int)seen, e, 1);
            s[t][e >> 2][e & 3] = __int_as_float((__float_as_int(x) & keep) | (~keep & (int)0xFF800000u));
          } else {  // (fewer vector registers: two wavefronts a SIMD at head_dim 128, three at 64)
            s[t][e >> 2][e & 3] = seen >> e & 1 ? x : -INFINITY;
          }
        }
      }
      uint32_t bad = 0;
#pragma unroll
      for (int b = 0; b < B; ++b)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const uint32_t y = beyond_252(raw.v_scale[b][x]);
          if (y != 0 && base + x * 4 + __builtin_ctz(y) / 8 <= last) bad = 1;
          raw.v_scale[b][x] &= ~((y >> 7) * 0xFFu);
        }
      if (__builtin_amdgcn_ballot_w64(bad != 0) != 0) {
        const uint8_t* scales = launch.v_scale + tile_at(i) * (B * kTileKeys);
        each_nan<B>(scales, [&](int b, int slot) {
          const int at = key0 + slot;
#pragma unroll
          for (int t = 0; t < NT; ++t)
            if (at <= pos[t] && (at > pos[t] - p.window || at < p.sinks)) nan_dims[t] |= 1u << b;
        });
      }
    }
  };

  // A wavefront's tiles: wave, wave + 4, ...  The next tile's K is requested as
  // soon as this one's is used up, its V likewise.
  const int tiles = end - begin;
  if (wave < tiles) {
    const int64_t first = tile_at(wave);
    fetch_k(first);
    fetch_v(first);
  }
  for (int i = wave; i < tiles; i += kWaves) {
    const bool more = i + kWaves < tiles;
    const int64_t next = tile_at(more ? i + kWaves : i);
    f32x4 s[NT][4];
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      // The lane's byte, then the exponent's place.
      const float scale = __uint_as_float((raw.k_scale[h] << (24 - 8 * (l16 & 3))) >> 1);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const uint32_t c = raw.k[h][ks];
        const bf16x8 k = __builtin_bit_cast(
            bf16x8, u32x4{two_values<0>(c, scale), two_values<1>(c, scale), two_values<2>(c, scale), two_values<3>(c, scale)});
#pragma unroll
        for (int t = 0; t < NT; ++t)
          s[t][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, qf[t][ks], ks == 0 ? f32x4{} : s[t][h], 0, 0, 0);
      }
    }
    if (more) fetch_k(next);
    // Score e of a lane (product e / 4) belongs to key key0 + 16 g4 + e.
    const int key0 = tile_of(i) * kTileKeys;
    if constexpr (CHUNK) {
      if (!seen_in_full(p, key0 / kTileKeys, first, last)) mask_chunk(i, key0, s);
    } else if (key0 + kTileKeys > w.span.len || (key0 < w.span.low && key0 + kTileKeys > w.span.sink_end)) {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int key = key0 + g4 * 16 + e;
        const bool gone = key >= w.span.len || (key >= w.span.sink_end && key < w.span.low);
#pragma unroll
        for (int t = 0; t < NT; ++t) s[t][e >> 2][e & 3] = gone ? -INFINITY : s[t][e >> 2][e & 3];
        // A hidden position's scale may be NaN; its probability is 0.
#pragma unroll
        for (int b = 0; b < B; ++b) raw.v_scale[b][e >> 2] &= gone ? ~(0xFFu << (8 * (e & 3))) : ~0u;
      }
    }
    bf16x8 hi[NT][2], lo[NT][2];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      float mx = s[t][0][0];
#pragma unroll
      for (int e = 1; e < 16; ++e) mx = fmaxf(mx, s[t][e >> 2][e & 3]);
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
          const float a = __builtin_amdgcn_exp2f(fmaf(s[t][2 * h + e / 2][2 * e & 3], sl2, -ref));
          const float b = __builtin_amdgcn_exp2f(fmaf(s[t][2 * h + e / 2][(2 * e & 3) + 1], sl2, -ref));
          l_run[t] += a + b;
          ph[e] = pack_bf16x2(a, b);
          pl[e] = pack_bf16x2(a - __uint_as_float(ph[e] << 16), b - __uint_as_float(ph[e] & 0xFFFF0000u));
        }
        hi[t][h] = __builtin_bit_cast(bf16x8, ph);
        lo[t][h] = __builtin_bit_cast(bf16x8, pl);
      }
    }
#pragma unroll
    for (int b = 0; b < B; ++b)
#pragma unroll
      for (int h = 0; h < 2; ++h) {  // keys 16 g4 + 8 h .. + 7
        u32x4 low, high;             // dims 32 b + l16, and 16 on
#pragma unroll
        for (int w2 = 0; w2 < 2; ++w2) {
          const uint32_t c = raw.v[b][2 * h + w2], sc = raw.v_scale[b][2 * h + w2];
          const uint32_t x0 = two_values<0>(c, scale_of(sc, 0)), x1 = two_values<1>(c, scale_of(sc, 1));
          const uint32_t x2 = two_values<2>(c, scale_of(sc, 2)), x3 = two_values<3>(c, scale_of(sc, 3));
          low[2 * w2] = low_halves(x0, x1);
          low[2 * w2 + 1] = low_halves(x2, x3);
          high[2 * w2] = high_halves(x0, x1);
          high[2 * w2 + 1] = high_halves(x2, x3);
        }
        const bf16x8 vl = __builtin_bit_cast(bf16x8, low), vh = __builtin_bit_cast(bf16x8, high);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          oacc[t][2 * b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vl, hi[t][h], oacc[t][2 * b], 0, 0, 0);
          oacc[t][2 * b + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vh, hi[t][h], oacc[t][2 * b + 1], 0, 0, 0);
          oacc[t][2 * b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vl, lo[t][h], oacc[t][2 * b], 0, 0, 0);
          oacc[t][2 * b + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vh, lo[t][h], oacc[t][2 * b + 1], 0, 0, 0);
        }
      }
    if (more) fetch_v(next);
  }

  // The wavefronts' partials meet in LDS.  Lane l holds head l % 16 and dims
  // 16 md + 4 (l / 16) .. + 3.
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
      if (CHUNK && nan_dims[t] >> md / 2 & 1) oacc[t][md] = f32x4{NAN, NAN, NAN, NAN};
      *reinterpret_cast<f32x4*>(&part_o[wave][t * 16 + l16][md * 16 + g4 * 4]) = oacc[t][md];
    }
  }
  __syncthreads();
  constexpr int QUADS = D / 4;
  for (int i = tid; i < min(NT * 16, rows - row0) * QUADS; i += kThreads) {
    const int row = i / QUADS, quad = i % QUADS;
    float m = -INFINITY;
#pragma unroll
    for (int x = 0; x < kWaves; ++x) m = fmaxf(m, part_m[x][row]);
    float l = 0.f;
    f32x4 acc = f32x4{};
#pragma unroll
    for (int x = 0; x < kWaves; ++x) {
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
    acc *= inv;
    const int64_t at = out_row(row0 + row);
    bool alone;
    int64_t part_at;
    if constexpr (CHUNK) {
      alone = p.n_ranges == 1;
      part_at = (int64_t)item * p.chunk_len * p.h_q + at;
    } else {
      alone = w.parts == 1;
      part_at = (int64_t)(item - w.seq) * p.h_q + at;
    }
    if (alone) {
      bf16x4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = (__bf16)acc[e];
      *reinterpret_cast<bf16x4*>(p.o + at * D + quad * 4) = v;
      if (quad == 0) {
        if constexpr (CHUNK) {
          const int token = token_of(row0 + row);
          p.lse[(at - (int64_t)token * p.h_q) * p.chunk_len + token] = row_lse;
        } else {
          p.lse[at] = row_lse;
        }
      }
    } else {
      *reinterpret_cast<f32x4*>(p.ws_o + part_at * D + quad * 4) = acc;
      if (quad == 0) p.ws_lse[part_at] = row_lse;
    }
  }
#endif  // __HIP_DEVICE_COMPILE__
}

template <int D>
void launch(const Kv4DecodeLaunch& p, hipStream_t stream) {
  const int64_t work = ((int64_t)p.a.seqs.items * p.a.h_kv + 7) / 8 * 8;
  const dim3 grid((unsigned)(work * p.a.row_blocks)), block(kThreads);
  if (p.a.group <= 16 * p.a.row_blocks) {
    hipLaunchKernelGGL((kv4_rows_kernel<D, 1, false>), grid, block, 0, stream, p);
  } else {
    hipLaunchKernelGGL((kv4_rows_kernel<D, 2, false>), grid, block, 0, stream, p);
  }
}

template <int D>
void launch(const Kv4ChunkLaunch& p, hipStream_t stream) {
  const dim3 grid(p.a.total_wgs), block(kThreads);
  if ((int64_t)p.a.chunk_len * p.a.group <= (int64_t)16 * p.a.row_blocks) {
    hipLaunchKernelGGL((kv4_rows_kernel<D, 1, true>), grid, block, 0, stream, p);
  } else {
    hipLaunchKernelGGL((kv4_rows_kernel<D, 2, true>), grid, block, 0, stream, p);
  }
}

}  // namespace

hipError_t launch_kv4_decode(const Kv4DecodeLaunch& p, int head_dim, hipStream_t stream) {
  if (head_dim == 128) {
    launch<128>(p, stream);
  } else {
    launch<64>(p, stream);
  }
  const hipError_t e = hipGetLastError();
  return e != hipSuccess || !p.a.may_split ? e : launch_decode_join(p.a, head_dim, true, stream);
}

hipError_t launch_kv4_few_rows(const Kv4ChunkLaunch& p, int head_dim, hipStream_t stream) {
  if (head_dim == 128) {
    launch<128>(p, stream);
  } else {
    launch<64>(p, stream);
  }
  return hipGetLastError();
}

}  // namespace mocap
