// Attention weight received by every key, for gfx950 (CDNA4):
//   w[h][j] = sum over rows i that see key j and heads g of group h of
//             exp(scale <q_ig, k_jh> - lse_gi)
// Many rows are bound by the matrix unit (2 D FLOP a pair) and the exponentials
// beside it (one a pair, with an FMA and an add as many issue cycles as the
// products at head_dim 128), few rows by HBM (the keys, once).
//
// Many rows: the keys stay, the rows stream.
//   * A wavefront holds 64 keys as B operands in registers and walks the rows,
//     S = Q K^T with v_mfma_f32_32x32x16_bf16.  Lane l then holds key l % 32 of
//     each product and 16 of its 32 rows, so the sum over the rows stays within
//     the lane, with no exchange between lanes before the end.
//   * Rows ((token, query head) pairs of the group, token-major) come in tiles of
//     32, four tiles a stage, through a 3-stage LDS ring that a workgroup's eight
//     wavefronts (512 keys) share, two stages ahead; a row's LSE in base 2 lies
//     beside it.
//   * A tile's products have the exponentials and sums of the tile before woven
//     in between, two scores per MFMA at head_dim 128, through all of a stage and
//     on into the next.  A wavefront's first tiles, whose rows do not all see its
//     keys, and those of an incomplete last stage are done one by one.
//   * Where keys are few, the rows are cut into parts whose sums a second launch
//     adds in order: parts of about as many tiles everywhere, so a block of keys that
//     only the later rows see has fewer (the same number for every block: 48 instead
//     of 37 us for a first chunk of 2048 tokens of 32/8/128 heads, 128 and 98 for 4096).
//   * Sums are fp32: 16 rows first, then tile by tile.
// Measured: 2048 tokens of 32/8/128 heads behind 30720, 490 us, 1.09 PFLOP/s; the
// matrix unit is busy half of the time, with vector work beside it for 60% of that.
#include "serve_device.h"

namespace mocap {
namespace {

constexpr int kRowTile = 32;
constexpr int kStageTiles = 4;
constexpr int kStageRows = kRowTile * kStageTiles;
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

constexpr int kBlockKeys = kWeightWaves * kWeightKeys;

// Row r sees key j if r >= (j - P) G.
__device__ __forceinline__ int first_row_of(const KeyWeightsLaunch& p, int key) {
  return (int)min((int64_t)max(key - p.prefix_len, 0) * p.group, (int64_t)p.chunk_len * p.group);
}
// Key blocks whose first key all rows see; of the others, the row parts.
__device__ __forceinline__ int blocks_seen(const KeyWeightsLaunch& p) {
  return min(p.key_blocks, p.prefix_len / kBlockKeys + 1);
}
__device__ __forceinline__ int parts_of_block(const KeyWeightsLaunch& p, int block) {
  const int tiles = (p.chunk_len * p.group + kRowTile - 1) / kRowTile - first_row_of(p, block * kBlockKeys) / kRowTile;
  return (tiles + p.part_tiles - 1) / p.part_tiles;
}
// The block and part of workgroup `at` of those behind block `from`.
__device__ __forceinline__ void locate_part(const KeyWeightsLaunch& p, int lane, int from, int at, int* block, int* part,
                                            int* parts) {
  for (int b0 = from; b0 < p.key_blocks; b0 += 64) {
    const int b = b0 + lane;
    const int mine = b < p.key_blocks ? parts_of_block(p, b) : 0;
    const int upto = wave_sums(mine);
    const uint64_t past = __builtin_amdgcn_ballot_w64(at < upto);
    if (past != 0) {
      const int i = __builtin_ctzll(past);
      *block = b0 + i;
      *parts = __builtin_amdgcn_readlane(mine, i);
      *part = at - (__builtin_amdgcn_readlane(upto, i) - *parts);
      return;
    }
    at -= __builtin_amdgcn_readlane(upto, 63);
  }
}

template <int D>
__global__ __launch_bounds__(64 * kWeightWaves, 2) void key_weights_kernel(const KeyWeightsLaunch p) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int KS = D / 16;
  constexpr int ROW_CHUNKS = D / 8;
  constexpr int STAGE_ELEMS = kStageRows * D;
  constexpr int COPIES = STAGE_ELEMS / 8 / (64 * kWeightWaves);  // 16-byte copies of a thread per stage
  constexpr int STAGES = 3;
  // One array for the ring and the LSE beside it: with two, the compiler tells
  // them apart, takes every read of the ring to depend on the copies in flight,
  // and waits for those (588 -> 566 us for 2048 tokens of 32/8/128
  // heads behind 30720).
  __shared__ __attribute__((aligned(1024))) uint16_t lds[STAGES * (STAGE_ELEMS + 2 * kStageRows)];
  float* const lse2 = reinterpret_cast<float*>(lds + STAGES * STAGE_ELEMS);

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = lane >> 5, l32 = lane & 31;
  const int P = p.prefix_len, n = P + p.chunk_len;

  // Logical order: KV head; the key blocks that all rows see, by row part; the others.
  const int logical = xcd_contiguous(blockIdx.x, p.head_wgs * p.h_kv);
  const int kv_head = logical / p.head_wgs;
  const int in_kv = logical - kv_head * p.head_wgs;
  const int seen_blocks = blocks_seen(p);
  int part = in_kv / seen_blocks, key_block = in_kv - part * seen_blocks, parts = p.row_parts;
  if (part >= p.row_parts) {
    const int other = in_kv - seen_blocks * p.row_parts;
    if (p.row_parts == 1) {
      part = 0;
      key_block = seen_blocks + other;
    } else {
      locate_part(p, lane, seen_blocks, other, &key_block, &part, &parts);
    }
  }
  const int block0 = key_block * kBlockKeys;
  const int key0 = block0 + wave * kWeightKeys;  // this wavefront's keys

  // The row tiles [t0, t1) of this part, of those that see some key of the
  // workgroup; this wavefront starts at tile `from` and masks those before `full`.
  const int rows = p.chunk_len * p.group;
  auto first_row = [&](int key) { return first_row_of(p, key); };
  const int first_tile = first_row(block0) / kRowTile;
  const int span = (rows + kRowTile - 1) / kRowTile - first_tile;
  const int t0 = first_tile + (int)((int64_t)span * part / parts);
  const int t1 = first_tile + (int)((int64_t)span * (part + 1) / parts);
  const int from = first_row(key0) / kRowTile;
  const int full = (first_row(key0 + kWeightKeys - 1) + kRowTile - 1) / kRowTile;

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

  // Stage s of the ring holds row tiles t0 + 4 s .. + 3; copy j of a thread moves
  // 16-byte chunk j * 512 + tid, from a column XORed with the row.
  // Rows past the last take it, with an LSE of +infinity (a weight of 0).
  // Offsets of this thread's chunks of rows that start at base_row, from the first
  // one's token: all of Q may not fit in 32 bits.
  auto offsets = [&](int base_row, int base_token, int* at) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < COPIES; ++j) {
      const int chunk = j * 64 * kWeightWaves + tid;
      const int lr = chunk / ROW_CHUNKS, c = (chunk % ROW_CHUNKS) ^ q_swizzle<D>(lr);
      const int r = min(base_row + lr, rows - 1);
      const int token = (int)div_by((uint32_t)r, p.group_magic, p.group_shift);
      at[j] = (((token - base_token) * p.h_q + (r - token * p.group)) * D + c * 8) * 2;
    }
  };
  // A group that divides a stage's rows: every whole stage has the same ones.
  const bool same = kStageRows % p.group == 0 && rows >= kStageRows;
  int usual[COPIES];
  if (same) offsets(0, 0, usual);
  auto issue = [&](int s) __attribute__((always_inline)) {
    const int base_row = (t0 + s * kStageTiles) * kRowTile;
    const int base_token = (int)div_by((uint32_t)min(base_row, rows - 1), p.group_magic, p.group_shift);
    const uint16_t* base = p.q + ((int64_t)base_token * p.h_q + kv_head * p.group) * D;
    const __amdgpu_buffer_rsrc_t q = __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, -1, kBufferWord3);
    int at[COPIES];
    if (same && base_row + kStageRows <= rows && base_token * p.group == base_row) {
#pragma unroll
      for (int j = 0; j < COPIES; ++j) at[j] = usual[j];
    } else {
      offsets(base_row, base_token, at);
    }
#pragma unroll
    for (int j = 0; j < COPIES; ++j)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          q, (lds_ptr_t)(lds + s % STAGES * STAGE_ELEMS + (j * 64 * kWeightWaves + wave * 64) * 8), 16, at[j], 0, 0, 0);
  };
  // The first two wavefronts bring the stage's LSE: requested with its copies, used
  // (waited for) one stage later.
  static_assert(kStageRows == 128, "a row for every lane of two wavefronts");
  auto load_lse = [&](int s) __attribute__((always_inline)) -> float {
    const int r = min((t0 + s * kStageTiles) * kRowTile + tid, rows - 1);
    const int token = (int)div_by((uint32_t)r, p.group_magic, p.group_shift);
    return p.lse[(int64_t)(kv_head * p.group + (r - token * p.group)) * p.chunk_len + token];
  };
  auto put_lse = [&](int s, float x) __attribute__((always_inline)) {
    const bool live = (t0 + s * kStageTiles) * kRowTile + tid < rows;
    lse2[s % STAGES * kStageRows + tid] = live && x != -INFINITY ? x * kLog2e : INFINITY;
  };

  const float sl2 = p.scale_log2;
  float w[2] = {0.f, 0.f};
  f32x16 acc[2][2];  // scores of even and odd tiles, per 32-key half
  // Fragment i of a stage: k-step i % KS of its tile i / KS.
  auto qfrag = [&](int s, int i) __attribute__((always_inline)) {
    return *reinterpret_cast<const bf16x8*>(lds + s % STAGES * STAGE_ELEMS + (i / KS * kRowTile + l32) * D +
                                            (((i % KS * 2 + half) ^ q_swizzle<D>(l32)) << 3));
  };
  // Score j of a lane belongs to row 8 (j / 4) + 4 half + j % 4 of its tile.
  auto lse_quad = [&](int s, int u, int quad) __attribute__((always_inline)) {
    return *reinterpret_cast<const f32x4*>(lse2 + s % STAGES * kStageRows + u * kRowTile + quad * 8 + half * 4);
  };
  constexpr int NM = 2 * KS;      // MFMAs of a tile
  constexpr int EACH = 32 / NM;   // scores woven in behind one
  // All tiles of stage s, each with the weights of the tile before woven in; the
  // first one's are those of the stage before, if `cont`.  The last tile's scores
  // stay in acc[1].
  //
  // Behind an MFMA come the FMAs of the scores after next, the exponentials of
  // the next ones and the sums of the last, so nothing there waits for the
  // instruction before it.  Scores are taken in the order (quad, half, row): a
  // quad's LSE serves eight, and the half whose products were issued last is not
  // touched in the first turns.
  auto stage = [&](int s, auto continued) __attribute__((always_inline)) {
    constexpr bool cont = decltype(continued)::value;
    constexpr int AHEAD = 3;
    bf16x8 f[AHEAD + 1];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) f[i] = qfrag(s, i);
    f32x4 l2[2];
    if constexpr (cont) l2[0] = lse_quad(s - 1, kStageTiles - 1, 0);
#pragma unroll
    for (int u = 0; u < kStageTiles; ++u) {
      f32x16* const a = acc[u % 2];
      const f32x16* const before = acc[1 - u % 2];
      float sum[2] = {0.f, 0.f}, x[2][EACH], v[2][EACH];  // arguments and exponentials of even and odd turns
      auto fmas = [&](int k) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
          const int j = k * EACH + i, quad = j / 8, h = j / 4 % 2, e = j % 4;
          x[k % 2][i] = fmaf(before[h][quad * 4 + e], sl2, -l2[quad % 2][e]);
        }
      };
      auto exps = [&](int k) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < EACH; ++i) v[k % 2][i] = __builtin_amdgcn_exp2f(x[k % 2][i]);
      };
      auto sums = [&](int k) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < EACH; i += 2) sum[(k * EACH + i) / 4 % 2] += v[k % 2][i] + v[k % 2][i + 1];
      };
#pragma unroll
      for (int k = 0; k < NM; ++k) {
        const int i = u * KS + k / 2, b = k % 2;
        if (b == 0 && i + AHEAD < kStageTiles * KS) f[(i + AHEAD) % (AHEAD + 1)] = qfrag(s, i + AHEAD);
        a[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[i % (AHEAD + 1)], kf[b][k / 2], k < 2 ? f32x16{} : a[b], 0, 0, 0);
        if (cont || u > 0) {
          if (k * EACH % 8 == 0 && k * EACH < 24)
            l2[(k * EACH / 8 + 1) % 2] = lse_quad(u ? s : s - 1, u ? u - 1 : kStageTiles - 1, k * EACH / 8 + 1);
          if (k >= 2) sums(k - 2);
          if (k >= 1) exps(k - 1);
          fmas(k);
        }
        if (k == NM - 1 && u + 1 < kStageTiles) l2[0] = lse_quad(s, u, 0);
        // Kept in this order by groups (an MFMA, an LDS read, the vector work of a
        // turn) rather than a barrier per turn: 575 -> 556 us.
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x402, 3 * EACH, 0);
      }
      if (cont || u > 0) {
        sums(NM - 2);
        exps(NM - 1);
        sums(NM - 1);
        w[0] += sum[0];
        w[1] += sum[1];
      }
    }
  };
  // The weights of tile u of stage s, from a, alone; t: its number, masked if some
  // key is not seen by all of its rows.
  auto finish = [&](int s, int u, int t, bool masked, const f32x16* a) __attribute__((always_inline)) {
    float sum[2] = {0.f, 0.f};
#pragma unroll
    for (int quad = 0; quad < 4; ++quad) {
      const f32x4 l2 = lse_quad(s, u, quad);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int seen_from = masked ? first_row(key0 + h * 32 + l32) : 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float v = __builtin_amdgcn_exp2f(fmaf(a[h][quad * 4 + e], sl2, -l2[e]));
          sum[h] += t * kRowTile + quad * 8 + half * 4 + e >= seen_from ? v : 0.f;
        }
      }
    }
    w[0] += sum[0];
    w[1] += sum[1];
  };
  auto alone = [&](int s, int u, int t) __attribute__((always_inline)) {
    f32x16* const a = acc[0];
    a[0] = a[1] = f32x16{};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const bf16x8 f = qfrag(s, u * KS + ks);
      a[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, kf[0][ks], a[0], 0, 0, 0);
      a[1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, kf[1][ks], a[1], 0, 0, 0);
    }
    finish(s, u, t, t < full, a);
  };

  const int stages = (t1 - t0 + kStageTiles - 1) / kStageTiles;
  // Whole stages of tiles that need no mask.
  const int whole0 = max(0, (full - t0 + kStageTiles - 1) / kStageTiles), whole1 = (t1 - t0) / kStageTiles;
  if (stages > 0) {
    issue(0);
    float coming = 0.f;  // the LSE of the next stage
    if (wave < 2) put_lse(0, load_lse(0));
    // Also the keys: without this the loop waits for them in every turn.
    wait_vmem<0>();
    if (stages > 1) {
      issue(1);
      if (wave < 2) coming = load_lse(1);
    }
    for (int s = 0; s < stages; ++s) {
      // In flight, oldest first: this stage's copies, the next one's (and in the
      // first wavefronts the next one's LSE).
      if (s + 1 == stages) {
        wait_vmem<0>();
      } else {
        wait_vmem<COPIES>();
      }
      lds_barrier();
      float later = 0.f;
      if (s + 2 < stages) {
        issue(s + 2);
        if (wave < 2) later = load_lse(s + 2);
      }
      if (s >= whole0 && s < whole1) {
        if (s > whole0) {
          stage(s, std::integral_constant<bool, true>());
        } else {
          stage(s, std::integral_constant<bool, false>());
        }
        if (s + 1 == whole1) finish(s, kStageTiles - 1, 0, false, acc[1]);
      } else {
#pragma unroll 1
        for (int u = 0; u < kStageTiles; ++u) {
          const int t = t0 + s * kStageTiles + u;
          if (t >= from && t < t1) alone(s, u, t);
        }
      }
      if (wave < 2 && s + 1 < stages) put_lse(s + 1, coming);
      coming = later;
    }
  }

  w[0] = lane_pair_sum(w[0]);
  w[1] = lane_pair_sum(w[1]);
  const float total = half ? w[1] : w[0];  // of key key0 + lane
  const int key = key0 + lane;
  if (key >= n) return;
  if (p.row_parts == 1) {
    const int64_t at = kv_head * p.weight_stride + key;
    p.weights[at] = (p.prev != nullptr && key < P ? p.prev[at] : 0.f) + total;
  } else {
    p.ws[((int64_t)part * p.h_kv + kv_head) * n + key] = total;
  }
#endif  // __HIP_DEVICE_COMPILE__
}

// Sums the row parts, in order.
__global__ __launch_bounds__(256) void key_weights_join_kernel(const KeyWeightsLaunch p) {
  const int n = p.prefix_len + p.chunk_len;
  const int key = blockIdx.x * 256 + threadIdx.x, h = blockIdx.y;
  if (key >= n) return;
  const int parts = key / kBlockKeys < blocks_seen(p) ? p.row_parts : parts_of_block(p, key / kBlockKeys);
  float w = 0.f;
  constexpr int AHEAD = 16;  // loads in flight (one by one: 48 instead of 37 us with 64 parts)
  for (int part0 = 0; part0 < parts; part0 += AHEAD) {
    float v[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) v[i] = p.ws[((int64_t)min(part0 + i, parts - 1) * p.h_kv + h) * n + key];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) w += part0 + i < parts ? v[i] : 0.f;
  }
  const int64_t at = h * p.weight_stride + key;
  p.weights[at] = (p.prev != nullptr && key < p.prefix_len ? p.prev[at] : 0.f) + w;
}

// ---- Few rows ----
// One row per sequence of a batch, or a chunk of few rows.  Bound by HBM: every key
// once.  A workgroup keeps up to 128 rows in LDS, as the A operands of their
// products; a wavefront takes 64 keys at a time straight from the store in
// registers: S = Q K^T with v_mfma_f32_16x16x32_bf16, 16 rows by 16 keys, so lane l
// holds key l % 16 and four rows of each product.  The 64 keys are worked through as
// two halves, and the next tile's half is asked for as soon as its registers are
// free, so keys are on their way during the products; the first ones come in behind
// the rows.  (All 64 keys loaded, then used: 38.3 instead of 36.9 us for 32 tokens of
// 32/8/128 heads by 65533 keys, 13.6 instead of 10.6 by 8032; one token of 64
// sequences of 3000, 91 instead of 86.)  134 MB of keys in 29 us with up to 8 tokens,
// 4.7 TB/s; with 32 tokens the last tiles' exponentials stand behind their loads.
constexpr int kFewWaves = 4;
constexpr int kFewBlock = 128;  // rows kept at a time

struct FewRows {
  const uint16_t* q;       // row r of the group: token r / G, head r % G
  const uint16_t* k_pool;
  const float* lse;        // of head h, token t: lse[h lse_head + t]
  const float* prev;       // of the KV head, or null
  float* weights;
  const_i32_ptr table;
  int64_t lse_head;
  int rows, group, h_q, h_kv, kv_head, block_size, len, prefix;
  uint32_t block_magic, group_magic;
  int block_shift, group_shift;
  float scale_log2;
};

// The weights of the keys of tiles begin, begin + 1, .. end - 1.
template <int D>
__device__ __forceinline__ void few_rows(const FewRows& x, int begin, int end) {
  constexpr int KS = D / 32;
  constexpr int STAGINGS = kFewBlock / 16 * KS / kFewWaves;
  __shared__ __attribute__((aligned(16))) u32x4 rows_q[kFewBlock / 16 * KS * 64];  // [16 rows][k-step][lane]
  __shared__ __attribute__((aligned(16))) float rows_l2[kFewBlock];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, g4 = lane >> 4;
  // Row r sees key j if r >= (j - prefix) G.
  auto first_row = [&](int j) { return (int)min((int64_t)max(j - x.prefix, 0) * x.group, (int64_t)x.rows); };
  for (int block = 0; block < x.rows; block += kFewBlock) {
    const int count = min(kFewBlock, x.rows - block), tiles16 = (count + 15) / 16;
    // Rows past the last take it, with an LSE of +infinity (a weight of 0).
    u32x4 rows_in[STAGINGS];
#pragma unroll
    for (int j = 0; j < STAGINGS; ++j) {
      const int at = j * kFewWaves + wave;  // (row tile, k-step)
      if (at < tiles16 * KS) {
        const int r = min(block + at / KS * 16 + l16, x.rows - 1);
        const int token = (int)div_by((uint32_t)r, x.group_magic, x.group_shift);
        rows_in[j] = *reinterpret_cast<const u32x4*>(x.q + ((int64_t)token * x.h_q + r - token * x.group) * D +
                                                     at % KS * 32 + g4 * 8);
      }
    }
    float lse_in = 0.f;
    if (tid < kFewBlock) {
      const int r = min(block + tid, x.rows - 1);
      const int token = (int)div_by((uint32_t)r, x.group_magic, x.group_shift);
      lse_in = x.lse[(r - token * x.group) * x.lse_head + token];
    }
    // Keys 32 half + .. of tile t, and what they had: from former queries, then from
    // the rows before this block.
    bf16x8 kf[4][KS];
    float old = 0.f;
    auto load = [&](int t, int half) __attribute__((always_inline)) {
      const int pos = t * kTileKeys;
      const int lb = (int)div_by((uint32_t)pos, x.block_magic, x.block_shift);
      const int64_t slot = pos - lb * x.block_size;
      const uint16_t* k =
          x.k_pool + (((int64_t)x.table[lb] * x.h_kv + x.kv_head) * x.block_size + slot + l16) * D + g4 * 8;
#pragma unroll
      for (int b = 2 * half; b < 2 * half + 2; ++b)
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) kf[b][ks] = *reinterpret_cast<const bf16x8*>(k + b * 16 * D + ks * 32);
    };
    auto load_old = [&](int t) __attribute__((always_inline)) {
      const int key = t * kTileKeys + lane;
      if (block > 0) {
        old = key < x.len ? x.weights[key] : 0.f;
      } else if (x.prev != nullptr) {
        old = key < x.prefix ? x.prev[key] : 0.f;
      }
    };
    // The first keys come in behind the rows.
    int t = begin + wave;
    if (t < end) {
      load_old(t);
      load(t, 0);
    }
    if (block > 0) lds_barrier();
#pragma unroll
    for (int j = 0; j < STAGINGS; ++j) {
      const int at = j * kFewWaves + wave;
      if (at < tiles16 * KS) rows_q[at * 64 + lane] = rows_in[j];
    }
    if (tid < kFewBlock) rows_l2[tid] = tid < count && lse_in != -INFINITY ? lse_in * kLog2e : INFINITY;
    if (t < end) load(t, 1);
    lds_barrier();
    for (; t < end; t += kFewWaves) {
      const int pos = t * kTileKeys;
      const int key = pos + lane;
      const float had = old;
      float w[4] = {0.f, 0.f, 0.f, 0.f};  // of key pos + 16 b + l16, from this lane's rows
      // Rows that see no key of the tile are left out; those from `full` on see all.
      const int from = max(0, first_row(pos) - block) / 16, full = first_row(pos + kTileKeys - 1) - block;
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        for (int rt = from; rt < tiles16; ++rt) {
          bf16x8 qf[KS];
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) qf[ks] = __builtin_bit_cast(bf16x8, rows_q[(rt * KS + ks) * 64 + lane]);
          const f32x4 l2 = *reinterpret_cast<const f32x4*>(&rows_l2[rt * 16 + g4 * 4]);
          const bool masked = rt * 16 < full || rt * 16 + 16 > count;
#pragma unroll
          for (int b = 2 * half; b < 2 * half + 2; ++b) {
            f32x4 s = f32x4{};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qf[ks], kf[b][ks], s, 0, 0, 0);
            f32x4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = __builtin_amdgcn_exp2f(fmaf(s[e], x.scale_log2, -l2[e]));
            if (masked) {
              const int seen_from = first_row(pos + b * 16 + l16) - block;
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const int r = rt * 16 + g4 * 4 + e;
                v[e] = r >= seen_from && r < count ? v[e] : 0.f;
              }
            }
            w[b] += (v[0] + v[1]) + (v[2] + v[3]);
          }
        }
        // The next tile's keys take the place of those that are done.
        if (t + kFewWaves < end) {
          if (half == 0) load_old(t + kFewWaves);
          load(t + kFewWaves, half);
        }
      }
      float total = 0.f;  // of key pos + lane
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const float sum = quad_rows_sum(w[b]);
        total = g4 == b ? sum : total;
      }
      if (key < x.len) x.weights[key] = had + total;
    }
  }
}

template <int D>
__global__ __launch_bounds__(64 * kFewWaves, 3) void decode_key_weights_kernel(const DecodeKeyWeightsLaunch p) {
#if defined(__HIP_DEVICE_COMPILE__)
  const int item = blockIdx.x / p.h_kv;
  const int kv_head = blockIdx.x - item * p.h_kv;
  const SeqPart w = locate_item(p.seqs, threadIdx.x & 63, item);
  if (w.seq == p.seqs.batch) return;
  int begin, end;
  part_range(w, &begin, &end);
  const int64_t row0 = (int64_t)w.seq * p.h_q + kv_head * p.group;
  const int64_t at = ((int64_t)w.seq * p.h_kv + kv_head) * p.weight_stride;
  FewRows x;
  x.q = p.q + row0 * D;
  x.k_pool = p.k_pool;
  x.lse = p.lse + row0;
  x.prev = p.prev != nullptr ? p.prev + at : nullptr;
  x.weights = p.weights + at;
  x.table = (const_i32_ptr)(p.seqs.tables + w.seq * p.seqs.table_stride);
  x.lse_head = 1;
  x.rows = x.group = p.group;
  x.h_q = p.h_q;
  x.h_kv = p.h_kv;
  x.kv_head = kv_head;
  x.block_size = p.seqs.block_size;
  x.len = w.span.len;
  x.prefix = w.span.len - 1;
  x.block_magic = p.seqs.block_magic;
  x.block_shift = p.seqs.block_shift;
  x.group_magic = p.group_magic;
  x.group_shift = p.group_shift;
  x.scale_log2 = p.scale_log2;
  few_rows<D>(x, begin, end);
#endif  // __HIP_DEVICE_COMPILE__
}

// A chunk of few rows: key_blocks workgroups per KV head take even runs of tiles.
template <int D>
__global__ __launch_bounds__(64 * kFewWaves, 3) void few_key_weights_kernel(const KeyWeightsLaunch p) {
#if defined(__HIP_DEVICE_COMPILE__)
  const int part = blockIdx.x / p.h_kv;
  const int kv_head = blockIdx.x - part * p.h_kv;
  const int n = p.prefix_len + p.chunk_len, tiles = (n + kTileKeys - 1) / kTileKeys;
  const int begin = (int)((int64_t)tiles * part / p.key_blocks), end = (int)((int64_t)tiles * (part + 1) / p.key_blocks);
  FewRows x;
  x.q = p.q + (int64_t)kv_head * p.group * D;
  x.k_pool = p.k_pool;
  x.lse = p.lse + (int64_t)kv_head * p.group * p.chunk_len;
  x.prev = p.prev != nullptr ? p.prev + kv_head * p.weight_stride : nullptr;
  x.weights = p.weights + kv_head * p.weight_stride;
  x.table = (const_i32_ptr)p.table;
  x.lse_head = p.chunk_len;
  x.rows = p.chunk_len * p.group;
  x.group = p.group;
  x.h_q = p.h_q;
  x.h_kv = p.h_kv;
  x.kv_head = kv_head;
  x.block_size = p.block_size;
  x.len = n;
  x.prefix = p.prefix_len;
  x.block_magic = p.block_magic;
  x.block_shift = p.block_shift;
  x.group_magic = p.group_magic;
  x.group_shift = p.group_shift;
  x.scale_log2 = p.scale_log2;
  few_rows<D>(x, begin, end);
#endif  // __HIP_DEVICE_COMPILE__
}

template <int D>
void launch(const KeyWeightsLaunch& p, hipStream_t stream) {
  if (p.few) {
    hipLaunchKernelGGL((few_key_weights_kernel<D>), dim3((unsigned)((int64_t)p.key_blocks * p.h_kv)),
                       dim3(64 * kFewWaves), 0, stream, p);
    return;
  }
  const dim3 grid((unsigned)((int64_t)p.head_wgs * p.h_kv)), block(64 * kWeightWaves);
  hipLaunchKernelGGL((key_weights_kernel<D>), grid, block, 0, stream, p);
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
  const dim3 grid((unsigned)((int64_t)p.seqs.items * p.h_kv)), block(64 * kFewWaves);
  if (head_dim == 128) {
    hipLaunchKernelGGL(decode_key_weights_kernel<128>, grid, block, 0, stream, p);
  } else {
    hipLaunchKernelGGL(decode_key_weights_kernel<64>, grid, block, 0, stream, p);
  }
  return hipGetLastError();
}

}  // namespace mocap
