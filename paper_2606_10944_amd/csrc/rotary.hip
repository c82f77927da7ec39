// Rotary positions on gfx950.  A pair (x_i, x_j) of a row's channels is turned by
// the angle 2 pi pos f: x_i' = amp (x_i cos - x_j sin), x_j' = amp (x_j cos + x_i sin);
// turning back (the gradient of it) negates the sine.
//
// A thread owns P pairs of one token and keeps their cosines and sines in
// registers while it walks its share of the heads, so an angle is formed once
// for all of them.  Angles: position times turns in float64, whole turns taken
// off before the rounding to float32 (a float32 product would lose 2^-24 of a
// position of a million: a tenth of a radian).
//
// Bound by HBM: 16384 tokens x 40 heads x 128 channels, bf16, 62 us = 5.4 TB/s read and
// written (a large copy runs at 5.1); one token of 16 sequences, 40 heads: 3.8 us, a
// launch and the latency of positions, sines and rows.
#include "common.hpp"
#include "q4.hpp"

namespace thin {

namespace {

constexpr int THREADS = 256;

// P pairs are two 16-byte words of a row: P = 8 (bf16) or 4 (float32).
template <typename T>
struct Pairs {
  static constexpr int n = 16 / Elem<T>::bytes;
};

template <typename T>
__device__ __forceinline__ void unpack(const u32x4& w, float* f);
template <>
__device__ __forceinline__ void unpack<float>(const u32x4& w, float* f) {
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(w[i]);
}
template <>
__device__ __forceinline__ void unpack<bf16_t>(const u32x4& w, float* f) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = __uint_as_float(w[i] << 16);
    f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
template <typename T>
__device__ __forceinline__ u32x4 pack(const float* f);
template <>
__device__ __forceinline__ u32x4 pack<float>(const float* f) {
  return (u32x4){__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]),
                 __float_as_uint(f[3])};
}
template <>
__device__ __forceinline__ u32x4 pack<bf16_t>(const float* f) {
  return (u32x4){cvt_pk_bf16(f[0], f[1]), cvt_pk_bf16(f[2], f[3]), cvt_pk_bf16(f[4], f[5]),
                 cvt_pk_bf16(f[6], f[7])};
}

// INTER: a pair is two neighbouring channels, else channels i and i + rot / 2.
template <typename T, int D, bool INTER>
__global__ __launch_bounds__(THREADS) void rotary_kernel(RotaryArgs a, int heads) {
  constexpr int P = Pairs<T>::n;
  constexpr int VT = D / (2 * P);  // threads per token
  const int64_t item = blockIdx.x * (int64_t)(THREADS / VT) + threadIdx.x / VT;
  if (item >= a.B * a.T) return;
  const int v = threadIdx.x % VT;
  const int64_t b = item / a.T, t = item % a.T;
  const bool turn = v * 2 * P < a.rot;
  // the thread's two words of a row: where its pairs' first and second channels
  // are (half layout), or 2 P channels in a row
  const int half = a.rot / 2;
  const int c0 = INTER || !turn ? v * 2 * P : v * P;
  const int c1 = INTER || !turn ? c0 + P : c0 + half;
  float cs[P], sn[P];
  if (turn) {
    const double pos =
        a.pos_per_token ? (double)a.pos[item] : (double)((int64_t)a.pos[b] + t);
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const double n = pos * a.turns[v * P + i];
      float s, c;
      sincospif((float)(2.0 * (n - rint(n))), &s, &c);
      cs[i] = c * a.amp;
      sn[i] = (a.inverse ? -s : s) * a.amp;
    }
  }
  const int64_t h0 = (int64_t)blockIdx.y * heads;
  const int64_t h1 = h0 + heads < a.Hx + a.Hy ? h0 + heads : a.Hx + a.Hy;
#pragma unroll 4
  for (int64_t h = h0; h < h1; ++h) {
    const bool x = h < a.Hx;
    const RowsView& in = x ? a.x : a.y;
    const RowsView& out = x ? a.xo : a.yo;
    const int64_t hh = x ? h : h - a.Hx;
    const T* ip = static_cast<const T*>(in.p) + b * in.sb + hh * in.sh + t * in.sr;
    T* op = static_cast<T*>(const_cast<void*>(out.p)) + b * out.sb + hh * out.sh + t * out.sr;
    u32x4 w0 = *reinterpret_cast<const u32x4*>(ip + c0);
    u32x4 w1 = *reinterpret_cast<const u32x4*>(ip + c1);
    if (turn) {
      float f[2 * P], r[2 * P];
      unpack<T>(w0, f);
      unpack<T>(w1, f + P);
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const int lo = INTER ? 2 * i : i, hi = INTER ? 2 * i + 1 : P + i;
        r[lo] = f[lo] * cs[i] - f[hi] * sn[i];
        r[hi] = f[hi] * cs[i] + f[lo] * sn[i];
      }
      w0 = pack<T>(r);
      w1 = pack<T>(r + P);
    }
    *reinterpret_cast<u32x4*>(op + c0) = w0;
    *reinterpret_cast<u32x4*>(op + c1) = w1;
  }
}

template <typename T, int D>
hipError_t launch(const RotaryArgs& a, hipStream_t st) {
  constexpr int per = THREADS / (D / (2 * Pairs<T>::n));
  const int64_t tiles = (a.B * a.T + per - 1) / per, H = a.Hx + a.Hy;
  int64_t parts = (1024 + tiles - 1) / tiles;
  if (parts > H) parts = H;
  const int64_t heads = (H + parts - 1) / parts;
  const dim3 grid((uint32_t)tiles, (uint32_t)((H + heads - 1) / heads));
  if (a.layout)
    rotary_kernel<T, D, true><<<grid, THREADS, 0, st>>>(a, (int)heads);
  else
    rotary_kernel<T, D, false><<<grid, THREADS, 0, st>>>(a, (int)heads);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rotary(int dtype, int64_t d, const RotaryArgs& a, hipStream_t st) {
  if (dtype == 0)
    return d == 32 ? launch<float, 32>(a, st) : d == 64 ? launch<float, 64>(a, st)
                                                        : launch<float, 128>(a, st);
  return d == 32 ? launch<bf16_t, 32>(a, st) : d == 64 ? launch<bf16_t, 64>(a, st)
                                                       : launch<bf16_t, 128>(a, st);
}

}  // namespace thin
