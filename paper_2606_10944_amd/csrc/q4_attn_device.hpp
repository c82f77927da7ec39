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

// Which cached rows a call's tokens attend to: every row up to their own, those of listed
// blocks, or those before the drafts and the drafts of their masks.
constexpr int kQ4All = 0, kQ4List = 1, kQ4Tree = 2;

// What a lane's query row of a drafted tree sees: cached rows 0 .. before - 1, and row at + j
// for the drafts j < there whose bit is set.
struct Drafts {
  const uint64_t* seen;
  int before, at, there;
  __device__ __forceinline__ Drafts() {}
  // Token t of sequence b; t = T or a token that is not there: no row at all.
  __device__ __forceinline__ Drafts(const Q4AttnArgs& a, int b, int t, int n_max) {
    const int cnt = a.tok.count ? std::min(a.tok.count[b], a.tok.T) : a.tok.T;
    const int x = a.tok.at[b];
    at = x > n_max ? n_max : (x < -kQ4MaxDrafts ? -kQ4MaxDrafts : x);
    there = t < cnt ? std::min(cnt, n_max - at) : 0;
    before = t < cnt ? std::max(at, 0) : 0;
    seen = a.seen + ((int64_t)b * a.tok.T + std::min(t, a.tok.T - 1)) * a.words;
  }
  // Rows row0 .. row0 + 63 (row0 >= 0): bit i is row row0 + i.
  __device__ __forceinline__ uint64_t window(int row0) const {
    const int off = row0 - at, j = off > 0 ? off : 0;  // the first draft among them
    uint64_t x = 0;
    if (j < there) {
      x = seen[j / 64] >> (j % 64);
      if (j % 64 != 0 && (j | 63) + 1 < there) x |= seen[j / 64 + 1] << (64 - j % 64);
      if (there - j < 64) x &= ((uint64_t)1 << (there - j)) - 1;
    }
    const int old = before - row0;  // rows before the drafts
    if (old <= 0) return x;
    return old >= 64 ? ~(uint64_t)0 : x << old | (((uint64_t)1 << old) - 1);
  }
};

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

// How the workgroups of a key head and tile share the sequences' steps.  Every
// sequence gets workgroups by its length: a share is what a workgroup takes of one
// sequence, the least for which the workgroups are enough.  Lane l holds sequences
// l, l + 64, ..
struct Shares {
  static constexpr int N = kQ4SharedEntries / 64;
  int steps[N];  // of this lane's sequences
  int upto[N];   // shares of the sequences up to each of them
  uint32_t share;

  __device__ __forceinline__ uint32_t count(int i) const {
    return ((uint32_t)steps[i] + share - 1) / share;
  }

  // steps_of(b): the tile's steps of sequence b
  template <typename F>
  __device__ __forceinline__ Shares(const Q4View& c, const Q4AttnArgs& a, int lane, F steps_of) {
    auto add = [](uint32_t x, uint32_t y) { return x + y; };
    int sum = 0;  // (at most 2^24: 256 sequences, 2^16 steps each)
#pragma unroll
    for (int i = 0; i < N; ++i) {
      steps[i] = 0;
      if (i * 64 < c.B && i * 64 + lane < c.B) steps[i] = steps_of(i * 64 + lane);
      sum += steps[i];
    }
    sum = (int)wave_reduce<uint32_t>((uint32_t)sum, 0u, add);
    // Rounded up per sequence, the shares are up to B more than the sum's: none of that is
    // set aside at first, then quarters of B, until the workgroups are enough.  (Setting B
    // aside at once left 32 sequences of one length half of theirs.)
    const int groups = c.B * a.shape.splits;
    for (int q = 0; q <= 4; ++q) {
      const uint32_t spare = (uint32_t)(groups - c.B * q / 4);
      const uint32_t even = ((uint32_t)sum + spare - 1) / spare;
      share = (uint32_t)__builtin_amdgcn_readfirstlane(
          (int)std::max(even, (uint32_t)a.shape.least));
      uint32_t taken = 0;
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (i * 64 < c.B) taken += count(i);
      if (wave_reduce<uint32_t>(taken, 0u, add) <= (uint32_t)groups) break;
    }
    int before = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      upto[i] = before;
      if (i * 64 >= c.B) continue;
      upto[i] += (int)wave_scan<uint32_t>(count(i), 0u, add);
      before = __builtin_amdgcn_readlane(upto[i], 63);
    }
  }

  // Workgroup j's sequence (-1: none is left for it) and steps i0 .. i1 - 1.
  __device__ __forceinline__ int find(const Q4View& c, int j, int* i0, int* i1) const {
    int b = -1;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (i * 64 >= c.B || b >= 0) continue;
      const uint64_t past = __ballot(upto[i] > j);
      if (!past) continue;
      const int l = __ffsll((unsigned long long)past) - 1;
      const int first = __builtin_amdgcn_readlane(upto[i] - (int)count(i), l);
      *i0 = __builtin_amdgcn_readfirstlane((j - first) * (int)share);
      const int end = __builtin_amdgcn_readlane(steps[i], l);
      *i1 = *i0 + (int)share < end ? *i0 + (int)share : end;
      b = i * 64 + l;
    }
    return b;
  }

  // The first of every sequence's workgroups and how many there are.
  __device__ __forceinline__ void write(const Q4View& c, int2* table, int lane) const {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i * 64 + lane < c.B)
        table[i * 64 + lane] = make_int2(upto[i] - (int)count(i), (int)count(i));
  }
};

}  // namespace thin
