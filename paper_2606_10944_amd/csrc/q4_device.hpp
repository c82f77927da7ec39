// Device-side pieces of the 4-bit cache's kernels.
#pragma once

#include "common.hpp"
#include "q4.hpp"

namespace thin {

// 2^(byte - 127)
__device__ __forceinline__ float q4_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// Eight codes as bf16 pairs (exact: a code times a power of two).
__device__ __forceinline__ void decode8(uint32_t c, float scale, uint32_t* w) {
  w[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 0));
  w[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 1));
  w[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 2));
  w[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 3));
}

template <typename T>
__device__ __forceinline__ float elem(const T* p, int64_t i);
template <>
__device__ __forceinline__ float elem<float>(const float* p, int64_t i) {
  return p[i];
}
template <>
__device__ __forceinline__ float elem<bf16_t>(const bf16_t* p, int64_t i) {
  return bf16_to_float(p[i].bits);
}

// Eight elements from a 16-byte aligned place.
template <typename T>
__device__ __forceinline__ void load8(const T* p, float* f);
template <>
__device__ __forceinline__ void load8<float>(const float* p, float* f) {
  const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
  f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
  f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
}
template <>
__device__ __forceinline__ void load8<bf16_t>(const bf16_t* p, float* f) {
  const u32x4 w = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = __uint_as_float(w[i] << 16);
    f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}

// The last cached row that token t of batch entry b sees (its own); -1 for a
// token that is not there or stands before row 0.
__device__ __forceinline__ int q4_last_row(const Q4Tokens& tok, int b, int t, int n_max) {
  if (tok.count && t >= tok.count[b]) return -1;
  int at = tok.at[b];
  at = at > n_max ? n_max : (at < -kQ4MaxTokens ? -kQ4MaxTokens : at);  // t < kQ4MaxTokens
  const int r = at + t;
  return r < 0 ? -1 : (r < n_max ? r : n_max - 1);
}

// Workgroups are dealt to the eight XCDs in turn.  Which of the launch's n = gridDim.x *
// gridDim.y pieces of work this one takes so that every XCD has a contiguous eighth of
// them, and its L2 the rows of few slices.
__device__ __forceinline__ uint32_t xcd_contiguous() {
  const uint32_t l = blockIdx.y * gridDim.x + blockIdx.x, n = gridDim.x * gridDim.y;
  const uint32_t x = l % 8;
  return x * (n / 8) + (x < n % 8 ? x : n % 8) + l / 8;
}

// One step of a reduction over the wave's lanes: the value of another lane by data
// parallel primitives (lanes that have no source keep `none`).
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t lane_move(uint32_t x, uint32_t none) {
  return (uint32_t)__builtin_amdgcn_update_dpp((int)none, (int)x, CTRL, ROWS, 0xf, false);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ uint64_t lane_move(uint64_t x, uint64_t none) {
  return (uint64_t)lane_move<CTRL, ROWS>((uint32_t)(x >> 32), (uint32_t)(none >> 32)) << 32 |
         lane_move<CTRL, ROWS>((uint32_t)x, (uint32_t)none);
}
// Lanes of four, of eight and of a row of 16.
constexpr int kSwapOnes = 0xb1, kSwapTwos = 0x4e;  // lane ^ 1, lane ^ 2
constexpr int kMirror8 = 0x141, kMirror16 = 0x140;  // lane i of eight: 7 - i; of 16: 15 - i
constexpr int kTurn4 = 0x124, kTurn8 = 0x128;      // four, eight lanes round
template <int CTRL>
__device__ __forceinline__ int lane_move(int x) {
  return (int)lane_move<CTRL, 0xf>((uint32_t)x, 0u);
}
template <int CTRL>
__device__ __forceinline__ float lane_move(float x) {
  return __uint_as_float(lane_move<CTRL, 0xf>(__float_as_uint(x), 0u));
}
template <int CTRL>
__device__ __forceinline__ double lane_move(double x) {
  return __longlong_as_double(
      (long long)lane_move<CTRL, 0xf>((uint64_t)__double_as_longlong(x), (uint64_t)0));
}

// op over a row of 16 lanes, the same in each of them.
template <typename K, typename F>
__device__ __forceinline__ K row_reduce(K x, F op) {
  x = op(x, lane_move<kSwapOnes>(x));
  x = op(x, lane_move<kSwapTwos>(x));
  x = op(x, lane_move<kMirror8>(x));
  return op(x, lane_move<kMirror16>(x));
}

// The upper half of a for the lower half of b (halves), or the odd rows of 16 lanes of a for
// the even ones of b: a then holds the lower (even) lanes' a and b, b the others'.
__device__ __forceinline__ void trade(bool halves, float& a, float& b) {
  const auto r = halves ? __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b),
                                                           false, false)
                        : __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b),
                                                           false, false);
  a = __uint_as_float(r[0]);
  b = __uint_as_float(r[1]);
}

// op over lanes 16 (and, with all, 32) apart, the same in each of them.
template <typename F>
__device__ __forceinline__ float across_rows(float x, bool all, F op) {
  float y = x;
  trade(false, x, y);
  x = op(x, y);
  if (!all) return x;
  y = x;
  trade(true, x, y);
  return op(x, y);
}

// op over the lanes up to each; op(x, none) = x.  Rows of 16 lanes by shifts, then across
// rows: six steps of a few cycles where a shuffle takes an LDS trip.
template <typename K, typename F>
__device__ __forceinline__ K wave_scan(K x, K none, F op) {
  x = op(x, lane_move<0x111, 0xf>(x, none));  // from 1, 2, 4, 8 lanes below
  x = op(x, lane_move<0x112, 0xf>(x, none));
  x = op(x, lane_move<0x114, 0xf>(x, none));
  x = op(x, lane_move<0x118, 0xf>(x, none));
  x = op(x, lane_move<0x142, 0xa>(x, none));  // lane 15 of a row to the next row
  return op(x, lane_move<0x143, 0xc>(x, none));  // lane 31 to the upper half
}
// op over all lanes, the same in each.
template <typename K, typename F>
__device__ __forceinline__ K wave_reduce(K x, K none, F op) {
  x = wave_scan<K>(x, none, op);
  if constexpr (sizeof(K) == 8)
    return (K)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(x >> 32), 63) << 32 |
           (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)x, 63);
  else
    return (K)__builtin_amdgcn_readlane((int)x, 63);
}
template <typename K>
__device__ __forceinline__ K wave_min(K x) {
  return wave_reduce<K>(x, ~(K)0, [](K a, K b) { return a < b ? a : b; });
}
template <typename K>
__device__ __forceinline__ K wave_max(K x) {
  return wave_reduce<K>(x, (K)0, [](K a, K b) { return a > b ? a : b; });
}

__device__ __forceinline__ double wave_sum(double x) {
  const uint64_t r = wave_reduce<uint64_t>(
      (uint64_t)__double_as_longlong(x), 0ull, [](uint64_t a, uint64_t b) {
        return (uint64_t)__double_as_longlong(__longlong_as_double((long long)a) +
                                              __longlong_as_double((long long)b));
      });
  return __longlong_as_double((long long)r);
}

// Instance F<element type, head dimension> of a launch.
#define Q4_BY_D(F, ...)                                                                      \
  return dtype == 0 ? (d == 32   ? F<float, 32>(__VA_ARGS__)                                 \
                       : d == 64 ? F<float, 64>(__VA_ARGS__)                                 \
                                 : F<float, 128>(__VA_ARGS__))                               \
                    : (d == 32   ? F<bf16_t, 32>(__VA_ARGS__)                                \
                       : d == 64 ? F<bf16_t, 64>(__VA_ARGS__)                                \
                                 : F<bf16_t, 128>(__VA_ARGS__))

}  // namespace thin
