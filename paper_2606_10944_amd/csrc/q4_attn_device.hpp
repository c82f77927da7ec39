// Device-side pieces of attention over the 4-bit cache.
//
// o = sum_j p_j v_j / sum_j p_j,  p_j = exp(<q, k_j> / sqrt(d) - max).
//
// A code times its power of two is exactly a bf16, so keys and values enter the bf16
// matrix instructions without loss, and so do bf16 queries; float32 queries and their
// weights p split into three bf16 parts.  Weights of bf16 queries are two parts (off by
// 2^-17) where few rows read a cache, and one (2^-8 at most, as the output's rounding)
// where the matrix instructions of many rows bound the call; there the sum of the weights
// is that of the rounded ones, so that they make one in all.
//
// (The scaled instruction would take keys' codes as they are stored, beside bf16 queries in
// two e4m3 parts: 687 us instead of 800 for 4096 tokens over 16384 rows.  But it cuts
// products below about 2^-15 of the largest under its scale, and the parts lose bits of
// channels 2^-9 below the row's largest: one outlier channel then hides the others.)
//
// Lanes are l = 16 g + m.  Scores S^T = K Q^T (keys x query rows): lane (m, g) feeds
// key row m's share of the channels, and query row m's.  It then holds the scores of
// keys 4 g .. 4 g + 3 for query row m, which is what the product O^T = V^T P^T wants as
// its second operand.  Its first, V^T, is read from LDS, where value rows lie decoded,
// by the transposing read.
#pragma once

#include <math.h>

#include <algorithm>

#include "common.hpp"
#include "q4.hpp"
#include "q4_device.hpp"

namespace thin {

constexpr float kLowest = -3.0e38f;
// Scores are to base 2: exp(z / sqrt d - max) = 2^(z c2 - mrun).  mrun moves only when a
// score passes it by more than kSlack: until then weights up to 2^kSlack are as exact
// as weights up to 1, and neither maxima nor sums pass between lanes.
constexpr float kSlack = 8.0f;
constexpr double kQ4Log2e = 1.44269504088896340736;

typedef short s16x4 __attribute__((ext_vector_type(4)));

// bf16 parts of eight float32 values: 1 (rounded) or 3 (their sum is the value).
template <int NP>
__device__ __forceinline__ void split8(const float* f, bf16x8_t* out) {
  float r[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = f[i];
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w[i] = cvt_pk_bf16(r[2 * i], r[2 * i + 1]);
      if (p + 1 < NP) {
        r[2 * i] -= __uint_as_float(w[i] << 16);
        r[2 * i + 1] -= __uint_as_float(w[i] & 0xffff0000u);
      }
    }
    out[p] = __builtin_bit_cast(bf16x8_t, (u32x4){w[0], w[1], w[2], w[3]});
  }
}

template <int N>
__device__ __forceinline__ void load_words(const uint8_t* p, uint32_t* w) {
  if constexpr (N == 4) {
    const u32x4 x = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = x[i];
  } else if constexpr (N == 2) {
    const uint2 x = *reinterpret_cast<const uint2*>(p);
    w[0] = x.x;
    w[1] = x.y;
  } else {
    w[0] = *reinterpret_cast<const uint32_t*>(p);
  }
}

// A slice's rows: offsets within it fit 32 bits (n_max * d / 2 <= 2^27 bytes).
struct Slice {
  const uint8_t *kc, *ks, *vc, *vs;
};
template <int D>
__device__ __forceinline__ Slice slice_of(const Q4View& c, int64_t s) {
  const int64_t row = s * c.n_max;
  return {c.k_codes + row * (D / 2), c.k_scales + row * (D / 32), c.v_codes + row * (D / 2),
          c.v_scales + row * (D / 32)};
}

// A tile's 16 query rows as the second operand of the scores, and the scores of 16 keys.
// Queries are bf16 as they are, or three bf16 parts of float32 (24 bits); keys are decoded
// to bf16.  Both are exact, and products are summed in float32.
template <typename T, int D>
struct Queries {
  static constexpr int KS = D / 32, QP = Elem<T>::bytes == 2 ? 1 : 3;
  bf16x8_t q[QP][KS];
  // row: this lane's query row (null: zeros); g: lane / 16
  __device__ __forceinline__ void load(const T* row, int g) {
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      float f[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      if (row) load8<T>(row + g * (D / 4) + k * 8, f);
      bf16x8_t part[QP];
      split8<QP>(f, part);
#pragma unroll
      for (int p = 0; p < QP; ++p) q[p][k] = part[p];
    }
  }
  __device__ __forceinline__ floatx4_t scores(const uint32_t* codes, uint32_t byte) const {
    floatx4_t z = {0.f, 0.f, 0.f, 0.f};
    const float ks = q4_scale(byte);
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      uint32_t w[4];
      decode8(codes[k], ks, w);
      const bf16x8_t kf = __builtin_bit_cast(bf16x8_t, (u32x4){w[0], w[1], w[2], w[3]});
#pragma unroll
      for (int p = QP - 1; p >= 0; --p)
        z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, q[p][k], z, 0, 0, 0);
    }
    return z;
  }
};

// Bytes per value row in LDS: 32 past the row put the four rows that 16 lanes read
// together on different banks.
template <int D>
constexpr int kVStride = 2 * D + 32;

// The V^T operand of 32 keys (rows 0 .. 31 of `rows`) and channels 16 dt .. 16 dt + 15.
template <int D>
__device__ __forceinline__ bf16x8_t value_columns(unsigned char* rows, int dt, int m, int g) {
  typedef __attribute__((address_space(3))) s16x4 lds_t;
  typedef short s16x8 __attribute__((ext_vector_type(8)));
  unsigned char* from = rows + (4 * g + m / 4) * kVStride<D> + dt * 32 + m % 4 * 8;
  const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t*)from);
  const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t*)(from + 16 * kVStride<D>));
  return __builtin_bit_cast(bf16x8_t, (s16x8)__builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
}

}  // namespace thin
