// Device-side pieces of attention over the 4-bit cache.
//
// o = sum_j p_j v_j / sum_j p_j,  p_j = exp(<q, k_j> / sqrt(d) - max).
//
// A code times its power of two is exactly a bf16, so values (and, for float32
// queries, keys) enter the bf16 matrix instructions without loss.  float32 weights p
// split into three bf16 parts; bf16 queries use one bf16 weight: its rounding (2^-8 of
// a term at most) is that of the output.
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
//
// float32: three bf16 parts (24 bits), the keys decoded to bf16.
template <typename T, int D>
struct Queries {
  static constexpr int KS = D / 32, N = 3 * KS;  // N: matrix instructions for 16 keys
  bf16x8_t q[3][KS];
  // row: this lane's query row (null: zeros); g: lane / 16
  __device__ __forceinline__ void load(const T* row, int g) {
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      float f[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      if (row) load8<T>(row + g * (D / 4) + k * 8, f);
      bf16x8_t part[3];
      split8<3>(f, part);
#pragma unroll
      for (int p = 0; p < 3; ++p) q[p][k] = part[p];
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
      for (int p = 2; p >= 0; --p)
        z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, q[p][k], z, 0, 0, 0);
    }
    return z;
  }
};

// bf16: the scaled 16x16x128 instruction takes the codes and their scales as they are
// stored, 128 channels at a time, beside fp8 queries.  A bf16 is the sum of two e4m3
// numbers (four significant bits each) under one power of two per row, exactly for
// values down to 2^-9 of the row's largest, within 2^-18 of that below.  (The
// instruction cuts products below about 2^-15 of its largest one: 1e-6 of the sum of
// magnitudes for normal values.)  Against decoding the keys to bf16 it saves 32 of 64
// conversions per step of 32 keys and takes two thirds of the matrix cores' time.
//
// Channels of k-slot 16 g + i and 64 + 16 g + i in lane (m, g) of the fp8 operand; the
// fp4 operand's lane (m, g) holds k-slots 32 g .. 32 g + 31, all under its own scale.
// d = 128: an instruction for each part; d = 64: k-slots 0 .. 63 take the first part,
// the others the second, beside the same keys; d = 32: 0 .. 31 and 32 .. 63.
typedef int i32x8 __attribute__((ext_vector_type(8)));
template <int D>
struct Queries<bf16_t, D> {
  static constexpr int N = D == 128 ? 2 : 1;  // matrix instructions for 16 keys
  i32x8 q[N];
  int scale;
  __device__ __forceinline__ void load(const bf16_t* row, int g) {
    // this lane's 16 channels (d = 128: 32) and the part that it holds
    constexpr int C = D == 128 ? 32 : 16;
    float f[C];
    const int c0 = D == 32 ? g % 2 * 16 : g * 16;
    float amax = 0.0f;
#pragma unroll
    for (int i = 0; i < C; i += 8) {
      if (row)
        load8<bf16_t>(row + c0 + i / 16 * 64 + i % 16, f + i);
      else
#pragma unroll
        for (int j = 0; j < 8; ++j) f[i + j] = 0.0f;
    }
#pragma unroll
    for (int i = 0; i < C; ++i) amax = fmaxf(amax, fabsf(f[i]));
    amax = across_rows(amax, true, [](float a, float b) { return fmaxf(a, b); });
    // the largest value lands in [2^7, 2^8)
    int byte = (int)(__float_as_uint(amax) >> 23) - 7;
    byte = byte < 1 ? 1 : byte;
    scale = byte;
    const float up = __uint_as_float((uint32_t)(254 - byte) << 23);
    int part[2][C / 4];
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int i = 0; i < C / 4; ++i) {
        float* x = f + 4 * i;
        if (p == 0)
#pragma unroll
          for (int j = 0; j < 4; ++j) x[j] *= up;
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], w, true);
        part[p][i] = w;
        x[0] -= __builtin_amdgcn_cvt_f32_fp8(w, 0);
        x[1] -= __builtin_amdgcn_cvt_f32_fp8(w, 1);
        x[2] -= __builtin_amdgcn_cvt_f32_fp8(w, 2);
        x[3] -= __builtin_amdgcn_cvt_f32_fp8(w, 3);
      }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (D == 128) {
        q[0][i] = part[0][i];
        q[N - 1][i] = part[1][i];
      } else if (D == 64) {
        q[0][i] = part[i / 4][i % 4];
      } else {
        q[0][i] = i < 4 ? part[g / 2][i % 4] : 0;
      }
    }
  }
  __device__ __forceinline__ floatx4_t scores(const uint32_t* codes, uint32_t byte) const {
    floatx4_t z = {0.f, 0.f, 0.f, 0.f};
    const i32x8 k = {(int)codes[0], (int)codes[1], (int)codes[2], (int)codes[3], 0, 0, 0, 0};
#pragma unroll
    for (int i = N - 1; i >= 0; --i)
      z = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(k, q[i], z, 4, 0, 0, (int)byte, 0, scale);
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
