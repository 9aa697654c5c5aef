// Appends of keys and values to the paged store, in bf16 or in 4 bits, with the
// rotation of keys and queries on the way (mocap_cache.h).
//
// For a token at position p and pair (x, y) of a head:
//   a = p inv_freq_i,  (x cos a - y sin a, x sin a + y cos a)
// Every value is read once and written once: HBM bounds a chunk, latency a batch of
// single tokens.
//
//   * A thread holds the same 16 dims of a token in every head it handles: two
//     16-byte pieces that hold eight whole pairs (dims 8 c .. and rot / 2 + 8 c ..,
//     or 16 c .. with neighbours paired), so pairs never leave a thread, and its
//     eight angles serve all its heads.
//   * p inv_freq has 31 + 24 bits and is taken as the sum of two fp64 values, exact, and
//     reduced to a quarter turn with pi/2 in two parts; sine and cosine of the rest
//     are Taylor polynomials.  gfx950 runs fp64 at the fp32 rate.
//   * For 4 bits the products stay in fp64, and the result goes to fp32 rounded to odd
//     (the last bit set if anything was cut off): it then lies on the right side of
//     every border between codes, so the one rounding that counts is exact.
//   * V is stored with the positions contiguous, through LDS (see kv_append.hip).
// Measured (kernel time, inputs out of cache): 2048 tokens of 32/8/128 heads 10.8 us into the
// bf16 store (50 MB, 4.7 TB/s) and 12.4 into the 4-bit one (44 MB).  All workgroups start at
// once, and for 4 bits those of K and V take longer than those of Q: a chain of V's conversion
// and turn, 8 fp64 angles, 16 fp64 products and K's conversion (passes with the rotation 9.8 us into
// bf16 and 11.6 into 4 bits, without 9.4 and 8.9).  20011 tokens of 8 KV heads of 128,
// without a rotation, into 4 bits 29 us (104 MB), of which 25 are its reads; without the
// conversion and the turn in LDS 29.  One token 3.1 us, 32 of 32/8/128 4.2.  Tried, none
// faster than +-2%: 2 or 8 query heads a workgroup, half the registers and a third more
// wavefronts, a grid with the heads of a tile in a row, pieces of 8 neighbouring dims,
// shorter polynomials, angles from two tables in LDS (a wavefront's first token's turned by the
// steps': a third of the fp64 work, 12 us where 10.7 were).
#include "kv4_device.h"

namespace mocap {
namespace {

// cos and sin of p f.  T: what the polynomials are evaluated in.  fp64 results are within 2^-52;
// without the product's low part they would lose 2^-54 of the angle where p f has more than
// 53 bits (1e-7 at positions near 2^31).  From kMaxAngle on, where the number of turns would lose
// its fraction, they are NaN.  (Here and in rotate(), sums of products are written as they are
// rounded: a token gets the same bits in a chunk and in a batch.)
constexpr double kMaxAngle = 281474976710656.;  // 2^48
template <typename T>
__device__ __forceinline__ void turn(double p, double f, T* c, T* s) {
  const double x = p * f, x_low = fma(p, f, -x);
  // Quarter turns, x 2 / pi, rounded by a sum of which the last bits hold whole numbers.
  constexpr double kWhole = 6755399441055744.;  // 1.5 * 2^52
  const double shifted = fma(x, 0.63661977236758134, kWhole), n = shifted - kWhole;
  // pi / 2 = 1.5707963267948966 + 6.123233995736766e-17 (to 2^-107); the first sum is exact.
  const double rest = fma(-n, 1.5707963267948966, x) + fma(-n, 6.123233995736766e-17, x_low);
  const T r = fabs(x) < kMaxAngle ? (T)rest : (T)NAN;
  const T r2 = r * r;
  T sine, cosine;  // |r| < 0.81: the terms left out are below 1e-16 (fp32: 4e-9)
  if (sizeof(T) == 8) {
    sine = T(-1. / 1307674368000);
    sine = fma(sine, r2, T(1. / 6227020800));
    sine = fma(sine, r2, T(-1. / 39916800));
    cosine = T(1. / 20922789888000);
    cosine = fma(cosine, r2, T(-1. / 87178291200));
    cosine = fma(cosine, r2, T(1. / 479001600));
    cosine = fma(cosine, r2, T(-1. / 3628800));
  } else {
    sine = T(0);
    cosine = T(-1. / 3628800);
  }
  sine = fma(sine, r2, T(1. / 362880));
  sine = fma(sine, r2, T(-1. / 5040));
  sine = fma(sine, r2, T(1. / 120));
  sine = fma(sine, r2, T(-1. / 6));
  sine = fma(sine, r2 * r, r);
  cosine = fma(cosine, r2, T(1. / 40320));
  cosine = fma(cosine, r2, T(-1. / 720));
  cosine = fma(cosine, r2, T(1. / 24));
  cosine = fma(cosine, r2, T(-0.5));
  cosine = fma(cosine, r2, T(1));
  const uint32_t quarter = (uint32_t)__double2loint(shifted);
  const T a = quarter & 1 ? sine : cosine, b = quarter & 1 ? cosine : sine;
  *c = (quarter + 1) & 2 ? -a : a;
  *s = quarter & 2 ? -b : b;
}

// What thread c of a token's D / 16 holds: dims first .. + 7 and second .. + 7, of
// which pair j is (first + j, second + j), or the neighbours 2 j, 2 j + 1 of the 16;
// their angles are 8 c + j.
struct Piece {
  int first, second;
  bool turned;
};
__device__ __forceinline__ Piece piece_of(const RopeAppendLaunch& p, int c) {
  Piece x;
  x.turned = c * 16 < p.rot;
  if (x.turned && !p.interleaved) {
    x.first = c * 8;
    x.second = c * 8 + p.rot / 2;
  } else {
    x.first = c * 16;
    x.second = c * 16 + 8;
  }
  return x;
}

template <typename T>
struct Turns {
  T c[8], s[8];
};
template <typename T>
__device__ __forceinline__ void make_turns(const RopeAppendLaunch& p, int c, int64_t pos, Turns<T>* t) {
  float f[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) f[j] = p.inv_freq[c * 8 + j];
#pragma unroll
  for (int j = 0; j < 8; ++j) turn((double)pos, (double)f[j], &t->c[j], &t->s[j]);
}

__device__ __forceinline__ void widen(const u32x4& x, float* y) {
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    y[2 * w] = __uint_as_float(x[w] << 16);
    y[2 * w + 1] = __uint_as_float(x[w] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ u32x4 narrow(const float* y) {
  return u32x4{pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]), pack_bf16x2(y[4], y[5]), pack_bf16x2(y[6], y[7])};
}

// The fp32 neighbour of y towards 0, its last bit set, where y is not an fp32 value:
// no comparison with a value of 23 bits or fewer changes, and no finite y becomes
// infinite.
__device__ __forceinline__ float to_odd(double y) {
  const float f = (float)y;
  const double back = (double)f;
  uint32_t bits = __float_as_uint(f);
  if (back != y) {
    bits -= fabs(back) > fabs(y) ? 1u : 0u;
    bits |= 1u;
  }
  return __uint_as_float(bits);
}
__device__ __forceinline__ float finish(float y) { return y; }
__device__ __forceinline__ float finish(double y) { return to_odd(y); }

// Turns the eight pairs of 16 values (the first piece's, then the second's).
template <typename T>
__device__ __forceinline__ void rotate(float* x, const Turns<T>& t, bool interleaved) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const T a = (T)(interleaved ? x[2 * j] : x[j]), b = (T)(interleaved ? x[2 * j + 1] : x[8 + j]);
    const float u = finish(fma(a, t.c[j], -(b * t.s[j]))), v = finish(fma(a, t.s[j], b * t.c[j]));
    x[interleaved ? 2 * j : j] = u;
    x[interleaved ? 2 * j + 1 : 8 + j] = v;
  }
}
template <typename T>
__device__ __forceinline__ void rotate_any(const RopeAppendLaunch& p, float* x, const Turns<T>& t) {
  if (p.interleaved) {
    rotate(x, t, true);
  } else {
    rotate(x, t, false);
  }
}

// A thread's 16 values of a head: loaded, turned, and stored in bf16.
__device__ __forceinline__ void load_pieces(const uint16_t* head, const Piece& at, u32x4* x) {
  x[0] = *reinterpret_cast<const u32x4*>(head + at.first);
  x[1] = *reinterpret_cast<const u32x4*>(head + at.second);
}
__device__ __forceinline__ void store_turned(const RopeAppendLaunch& p, u32x4* x, const Piece& at,
                                             const Turns<float>& t, uint16_t* head) {
  if (at.turned) {
    float y[16];
    widen(x[0], y);
    widen(x[1], y + 8);
    rotate_any(p, y, t);
    x[0] = narrow(y);
    x[1] = narrow(y + 8);
  }
  *reinterpret_cast<u32x4*>(head + at.first) = x[0];
  *reinterpret_cast<u32x4*>(head + at.second) = x[1];
}

// The bytes of one token's V rows from two threads' codes: those of dims 32 b .. + 15
// (even threads) and of the 16 dims after them (odd ones).  An even thread makes rows
// 16 b .. + 7, an odd one the next eight: even rows' bytes in x, odd rows' in y.
__device__ __forceinline__ void v_row_bytes(const uint32_t* codes, bool odd, uint32_t* x, uint32_t* y) {
  constexpr uint32_t kLow = 0x0F0F0F0Fu;
  const uint32_t sent = odd ? codes[0] : codes[1];
  const uint32_t got = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)sent, 0xB1, 0xF, 0xF, false);  // lane ^ 1
  const uint32_t low = odd ? got : codes[0], high = odd ? codes[1] : got;
  *x = (low & kLow) | (high & kLow) << 4;
  *y = (low >> 4 & kLow) | (high & ~kLow);
}
__device__ __forceinline__ int other_of_pair(int x) { return __builtin_amdgcn_update_dpp(0, x, 0xB1, 0xF, 0xF, false); }

// ---- A chunk ----
// One workgroup: the slots of one 64-slot tile of the store, for one KV head's K and V
// or for kRopeHeads query heads.
constexpr int kTile = kTileKeys;

// Element of (dim e, slot) in the bf16 V tile (see kv_append.hip).
__device__ __forceinline__ int v_index(int e, int slot) {
  return (((e * (kTile / 8) + (slot >> 3)) ^ ((e >> 3) & 15)) << 3) + (slot & 7);
}

template <int D, bool FOUR>
__global__ __launch_bounds__(4 * D) void rope_append_kernel(const RopeAppendLaunch p) {
  constexpr int C = D / 16, THREADS = kTile * C;
  constexpr int V_ROW = kTile + 8;  // bytes of a row of the 4-bit V tile in LDS
  __shared__ __attribute__((aligned(16))) uint8_t lds[FOUR ? D / 2 * V_ROW + kTile * (D / 8 + D / 32) : D * kTile * 2];

  const int tid = threadIdx.x;
  const int64_t tile0 = (p.start_pos / kTile + blockIdx.x) * kTile;
  const int first = (int)max(p.start_pos - tile0, (int64_t)0);
  const int last = (int)min(p.start_pos + p.chunk_len - tile0, (int64_t)kTile);
  const int slot = tid / C, c = tid % C;
  const bool mine = slot >= first && slot < last;
  const int64_t token = tile0 + slot - p.start_pos;
  const Piece at = piece_of(p, c);

  if ((int)blockIdx.y >= p.h_kv) {
    const int head0 = ((int)blockIdx.y - p.h_kv) * kRopeHeads, heads = min(kRopeHeads, p.h_q - head0);
    if (!mine) return;
    u32x4 x[kRopeHeads][2];
    const uint16_t* src = p.q + token * p.q_stride + (int64_t)head0 * D;
#pragma unroll
    for (int h = 0; h < kRopeHeads; ++h)
      if (h < heads) load_pieces(src + h * D, at, x[h]);
    Turns<float> t;
    if (at.turned) make_turns(p, c, p.first_pos + token, &t);
    uint16_t* dst = p.q_out + (token * p.h_q + head0) * D;
#pragma unroll
    for (int h = 0; h < kRopeHeads; ++h)
      if (h < heads) store_turned(p, x[h], at, t, dst + h * D);
    return;
  }

  const int h = blockIdx.y;
  const uint32_t lb = (uint32_t)tile0 / (uint32_t)p.block_size;
  const int slot0 = (int)(tile0 - (int64_t)lb * p.block_size);
  const int64_t head = (int64_t)p.tables[lb] * p.h_kv + h;  // of the pools' [blocks][Hkv]
  const uint16_t* k_src = p.k + token * p.k_stride + (int64_t)h * D;
  const uint16_t* v_src = p.v + token * p.v_stride + (int64_t)h * D;

  if constexpr (!FOUR) {
    uint16_t* vt = reinterpret_cast<uint16_t*>(lds);
    if (mine) {
      u32x4 k[2], v[2];
      load_pieces(k_src, at, k);
      load_pieces(v_src, Piece{c * 8, c * 8 + D / 2, false}, v);
      Turns<float> t;
      if (at.turned) make_turns(p, c, p.first_pos + token, &t);
      store_turned(p, k, at, t, static_cast<uint16_t*>(p.pools.k) + (head * p.block_size + slot0 + slot) * D);
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const int e = c * 8 + x * (D / 2) + 2 * w;
          vt[v_index(e, slot)] = (uint16_t)(v[x][w] & 0xFFFFu);
          vt[v_index(e + 1, slot)] = (uint16_t)(v[x][w] >> 16);
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = tid; i < D * (kTile / 8); i += THREADS) {
      const int e = i / (kTile / 8), s = i % (kTile / 8) * 8;
      uint16_t* dst = static_cast<uint16_t*>(p.pools.v) + (head * D + e) * p.block_size + slot0 + s;
      const uint16_t* tile = vt + v_index(e, s);
      if (s >= first && s + 8 <= last) {
        *reinterpret_cast<u32x4*>(dst) = *reinterpret_cast<const u32x4*>(tile);
      } else {
        for (int j = max(first - s, 0); j < min(last - s, 8); ++j) dst[j] = tile[j];
      }
    }
  } else {
    uint8_t* vt = lds;                           // [D / 2][V_ROW]
    uint8_t* k_max = lds + D / 2 * V_ROW;        // [slot][D / 8]: scale bytes that 8 dims would have
    uint8_t* v_max = k_max + kTile * (D / 8);    // [slot][D / 32]: scale bytes
    float y[16];
    if (mine) {
      u32x4 k[2], v[2];
      load_pieces(k_src, at, k);
      load_pieces(v_src, Piece{c * 16, c * 16 + 8, false}, v);
      widen(v[0], y);
      widen(v[1], y + 8);
      const int own = scale_byte(max(largest_bits(y), largest_bits(y + 8)));
      const int byte = max(own, other_of_pair(own));  // the bytes grow with the values
      const uint32_t codes[2] = {eight_codes(y, byte), eight_codes(y + 8, byte)};
      uint32_t even, odd;
      v_row_bytes(codes, c & 1, &even, &odd);
      uint8_t* rows = vt + ((c >> 1) * 16 + (c & 1) * 8) * V_ROW + slot;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        rows[2 * i * V_ROW] = (uint8_t)(even >> 8 * i);
        rows[(2 * i + 1) * V_ROW] = (uint8_t)(odd >> 8 * i);
      }
      if ((c & 1) == 0) v_max[slot * (D / 32) + (c >> 1)] = (uint8_t)byte;
      widen(k[0], y);
      widen(k[1], y + 8);
      if (at.turned) {
        Turns<double> t;
        make_turns(p, c, p.first_pos + token, &t);
        rotate_any(p, y, t);
      }
      k_max[slot * (D / 8) + at.first / 8] = (uint8_t)scale_byte(largest_bits(y));
      k_max[slot * (D / 8) + at.second / 8] = (uint8_t)scale_byte(largest_bits(y + 8));
    }
    __syncthreads();
    // A block's scale byte is the largest of its four pieces'.
    auto block_byte = [&](int s, int b) {
      const uint32_t m = *reinterpret_cast<const uint32_t*>(k_max + s * (D / 8) + b * 4);
      return (int)max(max(m & 255, m >> 8 & 255), max(m >> 16 & 255, m >> 24));
    };
    if (mine) {
      uint8_t* dst = static_cast<uint8_t*>(p.pools.k) + (head * p.block_size + slot0 + slot) * (D / 2);
      *reinterpret_cast<uint32_t*>(dst + at.first / 2) = eight_codes(y, block_byte(slot, at.first / 32));
      *reinterpret_cast<uint32_t*>(dst + at.second / 2) = eight_codes(y + 8, block_byte(slot, at.second / 32));
    }
    const int64_t tile = head * (p.block_size / kTile) + slot0 / kTile;  // of [blocks][Hkv][bs / 64]
    for (int i = tid; i < D / 2 * (kTile / 8); i += THREADS) {
      const int r = i / (kTile / 8), s = i % (kTile / 8) * 8;
      uint8_t* dst = static_cast<uint8_t*>(p.pools.v) + (tile * (D / 2) + r) * kTile + s;
      if (s >= first && s + 8 <= last) {
        *reinterpret_cast<u32x2*>(dst) = *reinterpret_cast<const u32x2*>(vt + r * V_ROW + s);
      } else {
        for (int j = max(first - s, 0); j < min(last - s, 8); ++j) dst[j] = vt[r * V_ROW + s + j];
      }
    }
    if (tid < D / 32 * kTile) {
      const int b = tid / kTile, s = tid % kTile;
      if (s >= first && s < last) {
        p.pools.k_scale[(tile * (D / 32) + b) * kTile + s] = (uint8_t)block_byte(s, b);
        p.pools.v_scale[(tile * (D / 32) + b) * kTile + s] = v_max[s * (D / 32) + b];
      }
    }
  }
}

// ---- One token of every sequence of a batch ----
// One wavefront: 64 / (D / 16) heads of one token, the KV heads before the query heads.
// The heads share their angles, one a lane, through LDS (each thread its eight: 1 us more), in
// fp32 for bf16 results and in fp64 for 4 bits, as in a chunk.
template <int D, bool FOUR>
__global__ __launch_bounds__(64) void decode_rope_append_kernel(const RopeAppendLaunch p) {
  constexpr int C = D / 16;
  __shared__ __attribute__((aligned(4))) uint8_t k_max[FOUR ? 64 / C * (D / 8) : 4];
  __shared__ float cosines[D / 2], sines[D / 2];
  __shared__ double key_cosines[FOUR ? D / 2 : 1], key_sines[FOUR ? D / 2 : 1];  // for 4 bits
  const int b = blockIdx.x;
  const int local = threadIdx.x / C, c = threadIdx.x % C;
  const int h = blockIdx.y * (64 / C) + local;
  const int64_t n = p.seq_lens[b];
  const int pos = p.positions ? p.positions[b] : (int)n - 1;
  if (n <= 0 || n > p.table_stride * p.block_size) return;  // the whole workgroup
  const Piece at = piece_of(p, c);
  const bool is_q = h >= p.h_kv && h < p.h_kv + p.h_q, is_kv = h < p.h_kv;
  const uint32_t slot_pos = (uint32_t)(n - 1);
  const uint32_t lb = slot_pos / (uint32_t)p.block_size;
  const int slot = (int)(slot_pos - lb * (uint32_t)p.block_size);

  u32x4 x[2], v[2];
  if (is_q) {
    load_pieces(p.q + b * p.q_stride + (int64_t)(h - p.h_kv) * D, at, x);
  } else if (is_kv) {
    load_pieces(p.k + b * p.k_stride + (int64_t)h * D, at, x);
    load_pieces(p.v + b * p.v_stride + (int64_t)h * D, Piece{c * 16, c * 16 + 8, false}, v);
  }
  if ((int)threadIdx.x < p.rot / 2) {
    const double f = p.inv_freq[threadIdx.x];
    turn((double)pos, f, &cosines[threadIdx.x], &sines[threadIdx.x]);
    if (FOUR) turn((double)pos, f, &key_cosines[threadIdx.x], &key_sines[threadIdx.x]);
  }
  __syncthreads();
  auto shared_turns = [&](auto* t, const auto* cos, const auto* sin) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      t->c[j] = cos[c * 8 + j];
      t->s[j] = sin[c * 8 + j];
    }
  };
  if (is_q || (is_kv && !FOUR)) {
    Turns<float> t;
    if (at.turned) shared_turns(&t, cosines, sines);
    uint16_t* dst;
    if (is_q) {
      dst = p.q_out + ((int64_t)b * p.h_q + h - p.h_kv) * D;
    } else {
      const int64_t head = (int64_t)p.tables[b * p.table_stride + lb] * p.h_kv + h;
      dst = static_cast<uint16_t*>(p.pools.k) + (head * p.block_size + slot) * D;
      uint16_t* vd = static_cast<uint16_t*>(p.pools.v) + (head * D + c * 16) * p.block_size + slot;
#pragma unroll
      for (int i = 0; i < 16; ++i)
        vd[(int64_t)i * p.block_size] = (uint16_t)(i & 1 ? v[i / 8][i / 2 % 4] >> 16 : v[i / 8][i / 2 % 4] & 0xFFFFu);
    }
    store_turned(p, x, at, t, dst);
  }
  if constexpr (FOUR) {
    float y[16];
    int64_t head = 0, tile = 0;
    int s = 0;
    if (is_kv) {
      head = (int64_t)p.tables[b * p.table_stride + lb] * p.h_kv + h;
      tile = head * (p.block_size / kTile) + slot / kTile;
      s = slot % kTile;
      widen(v[0], y);
      widen(v[1], y + 8);
      const int own = scale_byte(max(largest_bits(y), largest_bits(y + 8)));
      const int byte = max(own, other_of_pair(own));
      const uint32_t codes[2] = {eight_codes(y, byte), eight_codes(y + 8, byte)};
      uint32_t even, odd;
      v_row_bytes(codes, c & 1, &even, &odd);
      uint8_t* rows = static_cast<uint8_t*>(p.pools.v) + (tile * (D / 2) + (c >> 1) * 16 + (c & 1) * 8) * kTile + s;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        rows[2 * i * kTile] = (uint8_t)(even >> 8 * i);
        rows[(2 * i + 1) * kTile] = (uint8_t)(odd >> 8 * i);
      }
      if ((c & 1) == 0) p.pools.v_scale[(tile * (D / 32) + (c >> 1)) * kTile + s] = (uint8_t)byte;
      widen(x[0], y);
      widen(x[1], y + 8);
      if (at.turned) {
        Turns<double> t;
        shared_turns(&t, key_cosines, key_sines);
        rotate_any(p, y, t);
      }
      k_max[local * (D / 8) + at.first / 8] = (uint8_t)scale_byte(largest_bits(y));
      k_max[local * (D / 8) + at.second / 8] = (uint8_t)scale_byte(largest_bits(y + 8));
    }
    __syncthreads();
    if (is_kv) {
      auto block_byte = [&](int i) {
        const uint32_t m = *reinterpret_cast<const uint32_t*>(k_max + local * (D / 8) + i * 4);
        return (int)max(max(m & 255, m >> 8 & 255), max(m >> 16 & 255, m >> 24));
      };
      uint8_t* dst = static_cast<uint8_t*>(p.pools.k) + (head * p.block_size + slot) * (D / 2);
      *reinterpret_cast<uint32_t*>(dst + at.first / 2) = eight_codes(y, block_byte(at.first / 32));
      *reinterpret_cast<uint32_t*>(dst + at.second / 2) = eight_codes(y + 8, block_byte(at.second / 32));
      if (c < D / 32) p.pools.k_scale[(tile * (D / 32) + c) * kTile + s] = (uint8_t)block_byte(c);
    }
  }
}

// ---- The values that a 4-bit store stands for ----
// One workgroup: the wanted positions of one 64-slot tile, for one KV head.  A thread makes
// 8 dims of a position at a time, so that the lanes' 16-byte stores run along the rows (a
// thread with 32 dims, its stores 64 bytes apart: 29 us for 20011 positions of 8 heads of
// 128; now 17, 104 MB).  V's rows are turned in LDS.
constexpr int kLoadThreads = 256;
template <int D>
__global__ __launch_bounds__(kLoadThreads) void kv4_load_kernel(const Kv4LoadLaunch p) {
  constexpr int B = D / 32, C = D / 8, V_ROW = kTile + 4;
  __shared__ __attribute__((aligned(16))) uint8_t vt[D / 2 * V_ROW];
  const int tid = threadIdx.x;
  const int b = blockIdx.z, h = blockIdx.y;
  const int64_t end = p.ends[b];
  const int64_t begin = end - p.n;
  const bool none = end <= 0 || end > p.table_stride * p.block_size;
  const int64_t first_tile = begin >= 0 ? begin / kTile : -((-begin + kTile - 1) / kTile);
  const int64_t tile0 = (first_tile + blockIdx.x) * kTile;
  if (tile0 >= end) return;
  const bool stored = !none && tile0 >= 0;  // tiles start at multiples of 64: before 0 as a whole or not at all
  const int first = (int)max(begin - tile0, (int64_t)0), last = (int)min(end - tile0, (int64_t)kTile);
  int64_t head = 0, tile = 0;
  int slot0 = 0;
  if (stored) {
    const uint32_t lb = (uint32_t)tile0 / (uint32_t)p.block_size;
    slot0 = (int)(tile0 - (int64_t)lb * p.block_size);
    head = (int64_t)p.tables[b * p.table_stride + lb] * p.h_kv + h;
    tile = head * (p.block_size / kTile) + slot0 / kTile;
  }
  const uint8_t* const k_src = static_cast<const uint8_t*>(p.pools.k) + (head * p.block_size + slot0) * (D / 2);
  const uint8_t* const v_src = static_cast<const uint8_t*>(p.pools.v) + tile * (D / 2) * kTile;
  const uint8_t* const k_scale = p.pools.k_scale + tile * B * kTile;
  const uint8_t* const v_scale = p.pools.v_scale + tile * B * kTile;
  const int64_t row = (int64_t)p.h_kv * D;
  const int64_t to = ((int64_t)b * p.n + (tile0 - begin)) * row + h * D;  // of slot 0
  // Thread: dims 8 c .. + 7 of slots first + i, ...
  constexpr int SLOTS = kLoadThreads / C, TURNS = kTile / SLOTS;
  const int c = tid % C;
  uint32_t codes[TURNS] = {}, ks[TURNS] = {}, vs[TURNS] = {};
  if (stored) {
#pragma unroll
    for (int i = 0; i < TURNS; ++i) {
      const int s = first + i * SLOTS + tid / C;
      if (s >= last) break;
      codes[i] = *reinterpret_cast<const uint32_t*>(k_src + s * (D / 2) + c * 4);
      ks[i] = k_scale[c / 4 * kTile + s];
      vs[i] = v_scale[c / 4 * kTile + s];
    }
    if (tid < 2 * D) {  // 16 bytes each
      const u32x4 x = *reinterpret_cast<const u32x4*>(v_src + tid * 16);
      uint32_t* dst = reinterpret_cast<uint32_t*>(vt + tid / 4 * V_ROW + tid % 4 * 16);
#pragma unroll
      for (int w = 0; w < 4; ++w) dst[w] = x[w];
    }
  }
  __syncthreads();
  // V dims 8 c .. are four bits of rows 16 (c / 4) + 8 (c % 2) ..: the low ones where c % 4 < 2.
  const uint8_t* const v_rows = vt + (c / 4 * 16 + (c & 1) * 8) * V_ROW;
  const int shift = c % 4 / 2 * 4;
#pragma unroll
  for (int i = 0; i < TURNS; ++i) {
    const int s = first + i * SLOTS + tid / C;
    if (s >= last) break;
    u32x4 k = {}, v = {};
    if (stored) {
      const float k_s = scale_of(ks[i], 0), v_s = scale_of(vs[i], 0);
      k = u32x4{two_values<0>(codes[i], k_s), two_values<1>(codes[i], k_s), two_values<2>(codes[i], k_s),
                two_values<3>(codes[i], k_s)};
      uint32_t w = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) w |= ((uint32_t)v_rows[j * V_ROW + s] >> shift & 15u) << (4 * j);
      v = u32x4{two_values<0>(w, v_s), two_values<1>(w, v_s), two_values<2>(w, v_s), two_values<3>(w, v_s)};
    }
    *reinterpret_cast<u32x4*>(p.k + to + s * row + c * 8) = k;
    *reinterpret_cast<u32x4*>(p.v + to + s * row + c * 8) = v;
  }
}

template <int D>
void launch_chunk(const RopeAppendLaunch& p, hipStream_t stream) {
  const int64_t first_tile = p.start_pos / kTile, end_tile = (p.start_pos + p.chunk_len + kTile - 1) / kTile;
  const dim3 grid((unsigned)(end_tile - first_tile), p.h_kv + (p.h_q + kRopeHeads - 1) / kRopeHeads), block(4 * D);
  if (p.pools.k_scale) {
    hipLaunchKernelGGL((rope_append_kernel<D, true>), grid, block, 0, stream, p);
  } else {
    hipLaunchKernelGGL((rope_append_kernel<D, false>), grid, block, 0, stream, p);
  }
}

template <int D>
void launch_batch(const RopeAppendLaunch& p, hipStream_t stream) {
  constexpr int HEADS = 64 / (D / 16);
  const dim3 grid(p.batch, (p.h_kv + p.h_q + HEADS - 1) / HEADS), block(64);
  if (p.pools.k_scale) {
    hipLaunchKernelGGL((decode_rope_append_kernel<D, true>), grid, block, 0, stream, p);
  } else {
    hipLaunchKernelGGL((decode_rope_append_kernel<D, false>), grid, block, 0, stream, p);
  }
}

}  // namespace

hipError_t launch_rope_append(const RopeAppendLaunch& p, int head_dim, hipStream_t stream) {
  if (head_dim == 128) {
    launch_chunk<128>(p, stream);
  } else {
    launch_chunk<64>(p, stream);
  }
  return hipGetLastError();
}

hipError_t launch_decode_rope_append(const RopeAppendLaunch& p, int head_dim, hipStream_t stream) {
  if (head_dim == 128) {
    launch_batch<128>(p, stream);
  } else {
    launch_batch<64>(p, stream);
  }
  return hipGetLastError();
}

hipError_t launch_kv4_load(const Kv4LoadLaunch& p, int head_dim, hipStream_t stream) {
  const dim3 grid((p.n + kTile - 1) / kTile + 1, p.h_kv, p.batch), block(kLoadThreads);
  if (head_dim == 128) {
    hipLaunchKernelGGL(kv4_load_kernel<128>, grid, block, 0, stream, p);
  } else {
    hipLaunchKernelGGL(kv4_load_kernel<64>, grid, block, 0, stream, p);
  }
  return hipGetLastError();
}

}  // namespace mocap
