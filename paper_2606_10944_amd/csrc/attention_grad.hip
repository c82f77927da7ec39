// The gradient of coreset attention on gfx950.  With z_qj = <q, k_j> / sqrt(d) + lw_j,
// p = softmax_j(z) and g_qj = <do_q, v_j>:
//   ds_qj = p_qj (g_qj - sum_i p_qi g_qi),       dlw_j = sum_q ds_qj,
//   dq = sum_j ds_qj k_j / sqrt(d),   dk_j = sum_q ds_qj q / sqrt(d),   dv_j = sum_q p_qj do_q.
// Probabilities are formed anew from the queries and keys; the sum p g of a row too, so
// neither the forward's output nor its statistics are read.
//
// Up to 256 coreset rows (float32: 128; bf16 with all of a float32 dO: 192 of 128 channels) a
// workgroup holds every key of a slice, 16 to 64 per wave, and walks a range of its queries, 32 at
// a time (16 of float32 rows over up to 32 keys): one launch reads Q and dO once and writes dQ,
// and the sums of dK and dV stay in registers.  Wider coresets take a launch that owns query rows
// (statistics, then dQ), and the same walk per chunk of keys for dK and dV.
// Workgroups leave their sums of dK and dV for the join, which adds them in order.  Rows off the
// coreset are zeros that the walk writes beside its own work, or a launch of their own.
//
// 64 slices of 16384 queries over 192 keys, d = 128, bf16: 470 to 500 us, 550 TFLOP/s at 10 d per
// (query, key), 2.9 TB/s; the walk takes 450 of it, the join 16.  The matrix cores are busy for
// 26 % of the cycles that the walk's waves live, the vector ALU 42 %, LDS 50 % (conflicts 1 %):
// a wave owns 16 keys alone, so twelve of them read Q and dO from LDS, by rows and by columns, for
// few products each, and 8 of the 12 have units of dQ.  Without the traffic with HBM it takes 284
// us of 360 (128 keys), without that and the products 200: the row statistics' way through LDS,
// that of p and ds, and two barriers per 32 queries.  Over 128 keys 350 us; 32 slices of 32768 over
// 256 keys 520.  float32 rows over 512 keys (16 slices of 2048) 345 us, the matrix cores busy for 75
// and 78 % of the two large launches, which form scores and g three times.  The smallest calls are
// two dependent launches, 6 + 5 us, behind 14 us of host time.
//
// Registers.  Waves of 32 and 64 keys leave some in scratch: bytes per lane for dO of bf16, of
// float32, and of float32 with dlogw: d = 32 2 x 4 0, 40, 40, 4 x 4 68, 84, 80; d = 64 8 x 2 36, 20,
// 28; d = 128 8 x 2 8, 48.  The other shapes that were measured there are slower (see grad_shape).
//
// Types.  bf16 rows: bf16 products summed in float32; p and ds round to bf16 (half a step, as
// the gradients' own rounding) for the products over queries and over keys; a float32 dO is
// two bf16 parts (17 bits), or in g all three where dlw, a float32 sum of differences, is asked
// for.  float32 rows: float32 products throughout.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "common.hpp"
#include "grad.hpp"
#include "q4_device.hpp"

namespace thin {

// float32 rows of dO of which bf16 products take all three bf16 parts.
struct exact_t {
  float f;
};
template <>
struct Elem<exact_t> {
  static constexpr int bytes = 4;
};

namespace {

// Rows of a product over rows: the bf16 instruction takes 32, of the float32 one, which takes
// four, 16 are counted as one.
template <typename T>
constexpr int kUnit = Elem<T>::bytes == 2 ? 32 : 16;

constexpr float kLeast = -3.0e38f;
constexpr double kLog2e = 1.44269504088896340736;

// Scores of bf16 rows are to base 2.  Those of float32 rows are not: a score of 10 would round by
// as much again once more, where its distance from the maximum, which a weight goes by, is small.
// (64 slices of 4096 queries over 128 keys of 64 channels 219 -> 235 us for it.)
template <typename T>
constexpr float kUnitScore = Elem<T>::bytes == 2 ? (float)kLog2e : 1.0f;
template <typename T>
__device__ __forceinline__ float weight(float x) {
  return __builtin_amdgcn_exp2f(Elem<T>::bytes == 2 ? x : x * (float)kLog2e);
}
// The score of a product x.  (float32 rows: the scale's rounding would move every score alike.)
template <typename T, int D>
__device__ __forceinline__ float score(float x, float bias) {
  const double c = (Elem<T>::bytes == 2 ? kLog2e : 1.0) / sqrt((double)D);
  if constexpr (Elem<T>::bytes == 4 && D != 64)
    bias = fmaf(x, (float)(c - (double)(float)c), bias);
  return fmaf(x, (float)c, bias);
}

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef short s16x8_t __attribute__((ext_vector_type(8)));

// Rows of D elements of T in LDS.  32 bytes past the row put rows that lanes read together on
// different banks, in both ways of reading.
template <typename T, int D>
struct LdsRows {
  static constexpr int CW = D * Elem<T>::bytes / 16;  // words per row
  static constexpr int stride = D * Elem<T>::bytes + 32;
};

// Word v of this lane's row fragment (row m, word 4 v + g) of a tile of 16 rows.
template <typename T, int D>
__device__ __forceinline__ uint4 lds_word(const unsigned char* rows, int v, int m, int g) {
  return *reinterpret_cast<const uint4*>(rows + m * LdsRows<T, D>::stride + (4 * v + g) * 16);
}

// Column 16 dt + m of rows 4 g .. 4 g + 3 and 16 + 4 g .. (of 32 rows `stride` bytes apart).
__device__ __forceinline__ bf16x8_t lds_columns(const unsigned char* rows, int stride, int dt,
                                                int m, int g) {
  typedef __attribute__((address_space(3))) s16x4_t lds_t;
  unsigned char* from =
      const_cast<unsigned char*>(rows) + (4 * g + m / 4) * stride + dt * 32 + m % 4 * 8;
  const s16x4_t v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t*)from);
  const s16x4_t v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t*)(from + 16 * stride));
  return __builtin_bit_cast(bf16x8_t,
                            (s16x8_t)__builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
}

__device__ __forceinline__ bf16x8_t pack8(const float* a, const float* b) {
  return __builtin_bit_cast(bf16x8_t, (u32x4){cvt_pk_bf16(a[0], a[1]), cvt_pk_bf16(a[2], a[3]),
                                              cvt_pk_bf16(b[0], b[1]), cvt_pk_bf16(b[2], b[3])});
}

// Operands of a product over a unit of rows: lane (m, g) holds rows 4 g .. 4 g + 3 (and of bf16
// 16 + 4 g ..) of its column: of rows in LDS (column 16 dt + m), or of values it has.
template <typename T>
struct Column;
template <>
struct Column<bf16_t> {
  bf16x8_t x;
  __device__ __forceinline__ Column() {}
  __device__ __forceinline__ Column(const unsigned char* rows, int stride, int dt, int m, int g)
      : x(lds_columns(rows, stride, dt, m, g)) {}
  __device__ __forceinline__ Column(const float (*w)[4]) : x(pack8(w[0], w[1])) {}
  // The same of a row (of a column m) in LDS.
  __device__ __forceinline__ Column(const unsigned char* row, int g) {
    const uint2 a = *reinterpret_cast<const uint2*>(row + 8 * g);
    const uint2 b = *reinterpret_cast<const uint2*>(row + 32 + 8 * g);
    x = __builtin_bit_cast(bf16x8_t, (u32x4){a.x, a.y, b.x, b.y});
  }
  // acc (this' columns x b's) += this^T b: lane (m, g) has columns 4 g .. 4 g + 3 of this and m
  // of b.
  __device__ __forceinline__ floatx4_t times(const Column& b, floatx4_t acc) const {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, b.x, acc, 0, 0, 0);
  }
};
template <>
struct Column<float> {
  float x[4];
  __device__ __forceinline__ Column() {}
  __device__ __forceinline__ Column(const unsigned char* rows, int stride, int dt, int m, int g) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      x[i] = *reinterpret_cast<const float*>(rows + (4 * g + i) * stride + (16 * dt + m) * 4);
  }
  __device__ __forceinline__ Column(const float (*w)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = w[0][i];
  }
  __device__ __forceinline__ Column(const unsigned char* row, int g) {
    const floatx4_t a = *reinterpret_cast<const floatx4_t*>(row + 16 * g);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = a[i];
  }
  __device__ __forceinline__ floatx4_t times(const Column& b, floatx4_t acc) const {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      acc = __builtin_amdgcn_mfma_f32_16x16x4f32(x[i], b.x[i], acc, 0, 0, 0);
    return acc;
  }
};

// `bytes` bytes at p: loads past them give 0 and stores past them are dropped, without a branch,
// so that the compiler can count a step's memory operations.  p and bytes are the wave's.
struct Span {
  __amdgpu_buffer_rsrc_t r;
  __device__ __forceinline__ Span(const void* p, int bytes)
      : r(__builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, bytes, 0x00027000)) {}
  __device__ __forceinline__ u32x4 load16(uint32_t at) const {
    return __builtin_amdgcn_raw_buffer_load_b128(r, at, 0, 0);
  }
  __device__ __forceinline__ uint32_t load4(uint32_t at) const {
    return __builtin_amdgcn_raw_buffer_load_b32(r, at, 0, 0);
  }
  __device__ __forceinline__ u32x2 load8(uint32_t at) const {
    return __builtin_amdgcn_raw_buffer_load_b64(r, at, 0, 0);
  }
  __device__ __forceinline__ void store(u32x4 w, uint32_t at) const {
    __builtin_amdgcn_raw_buffer_store_b128(w, r, at, 0, 0);
  }
  // (not to be kept in the caches: the zeros of dK and dV, 87 -> 76 us for 64 slices of 8192
  // queries over 64 keys of 64 channels; dQ, whose lines several waves write, 360 -> 440 us)
  __device__ __forceinline__ void stream(u32x4 w, uint32_t at) const {
    __builtin_amdgcn_raw_buffer_store_b128(w, r, at, 0, 2);
  }
  __device__ __forceinline__ void store(u32x2 w, uint32_t at) const {
    __builtin_amdgcn_raw_buffer_store_b64(w, r, at, 0, 0);
  }
};

// A 16-byte word of T from a row of TO: one part, or the bf16 parts of float32, each the rounding
// of what those before it leave.
template <typename T, typename TO>
struct Parts {
  static constexpr bool mixed = Elem<T>::bytes == 2 && Elem<TO>::bytes == 4;
  static constexpr int n = mixed ? (std::is_same<TO, exact_t>::value ? 3 : 2) : 1;
};
template <typename T, typename TO>
struct RawWord;  // as it is in memory; word `item` of a span
template <typename T>
struct RawWord<T, T> {
  u32x4 w;
  __device__ __forceinline__ void load(const Span& p, uint32_t item) { w = p.load16(item * 16); }
  __device__ __forceinline__ void parts(u32x4* o) const { o[0] = w; }
};
template <>
struct RawWord<float, bf16_t> {
  u32x2 w;
  __device__ __forceinline__ void load(const Span& p, uint32_t item) { w = p.load8(item * 8); }
  __device__ __forceinline__ void parts(u32x4* o) const {
    o[0] = (u32x4){w[0] << 16, w[0] & 0xffff0000u, w[1] << 16, w[1] & 0xffff0000u};
  }
};
template <int N>
struct SplitWord {
  u32x4 w[2];
  __device__ __forceinline__ void load(const Span& p, uint32_t item) {
    w[0] = p.load16(item * 32);
    w[1] = p.load16(item * 32 + 16);
  }
  __device__ __forceinline__ void parts(u32x4* o) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float a = __uint_as_float(w[i / 2][i % 2 * 2]), b = __uint_as_float(w[i / 2][i % 2 * 2 + 1]);
#pragma unroll
      for (int p = 0; p < N; ++p) {
        o[p][i] = cvt_pk_bf16(a, b);
        a -= __uint_as_float(o[p][i] << 16);
        b -= __uint_as_float(o[p][i] & 0xffff0000u);
      }
    }
  }
};
template <>
struct RawWord<bf16_t, float> : SplitWord<2> {};
template <>
struct RawWord<bf16_t, exact_t> : SplitWord<3> {};

// Four consecutive channels of a gradient.
template <typename T>
struct Four;
template <>
struct Four<bf16_t> {
  u32x2 w;
  __device__ __forceinline__ Four() {}
  __device__ __forceinline__ Four(floatx4_t o)
      : w((u32x2){cvt_pk_bf16(o[0], o[1]), cvt_pk_bf16(o[2], o[3])}) {}
  __device__ __forceinline__ void store(bf16_t* p) const { *reinterpret_cast<u32x2*>(p) = w; }
};
template <>
struct Four<float> {
  u32x4 w;
  __device__ __forceinline__ Four() {}
  __device__ __forceinline__ Four(floatx4_t o) : w(__builtin_bit_cast(u32x4, o)) {}
  __device__ __forceinline__ void store(float* p) const { *reinterpret_cast<u32x4*>(p) = w; }
};
template <typename T>
__device__ __forceinline__ void store4(T* p, floatx4_t o) {
  Four<T>(o).store(p);
}

// The row that an entry of the list stands for, as in the forward: the nearest one.
__device__ __forceinline__ int32_t nearest_row(int32_t r, int64_t n) {
  return (int32_t)std::min<int64_t>(std::max(r, 0), n - 1);
}

// Coreset row j of slice s: its row of K and V (-1: none, or its weight is 0) and log-weight as
// scores are.
template <typename T>
__device__ __forceinline__ int coreset_row(const GradArgs& a, int64_t s, int64_t j, float* bias) {
  *bias = -INFINITY;
  if (j >= a.n_out) return -1;
  const float lw = a.logw ? a.logw[s * a.n_out + j] : 0.0f;
  if (lw == -INFINITY) return -1;
  *bias = lw * kUnitScore<T>;
  return nearest_row(a.idx[s * a.n_out + j], a.n);
}

// ---------------------------------------------------------------------------
// Zeros of dK and dV, where the rows are many more than the queries.
// ---------------------------------------------------------------------------
constexpr int ZT = 256, ZW = 8;  // threads, 16-byte words of each tensor per thread

__global__ __launch_bounds__(ZT) void grad_zeros_kernel(u32x4* k, u32x4* v, int64_t words) {
  const int64_t z = (int64_t)blockIdx.x * ZT * ZW + threadIdx.x;
#pragma unroll
  for (int i = 0; i < ZW; ++i)
    if (z + i * ZT < words) {
      k[z + i * ZT] = (u32x4){0, 0, 0, 0};
      v[z + i * ZT] = (u32x4){0, 0, 0, 0};
    }
}

// ---------------------------------------------------------------------------
// Keys: see above.  W waves of 16 KT keys.  ONE: every key of the slice is here.
//
// Lanes are l = 16 g + m.  Scores S^T = K Q^T by 16 keys x 16 queries: lane (m, g) holds keys
// 4 g .. 4 g + 3 of query m, so that a row's maximum and sums need few moves between lanes;
// the waves' meet in LDS.  p and ds pass through LDS, [query, key]: a wave reads its own keys'
// columns back by the transposing read for the products over queries, as it reads the columns
// of Q and dO, and every wave reads all of ds for its 16 channels of dQ.
// ---------------------------------------------------------------------------
template <typename T, typename TO, int D, int W, int KT, bool ONE>
__global__ __launch_bounds__(64 * W, W > 8 ? W / 4 : 2) void grad_keys_kernel(GradArgs a) {
  using R = LdsRows<T, D>;
  constexpr int NV = Frag<T, D>::NV, DT = D / 16, NK = 16 * W * KT;
  constexpr int OP = Parts<T, TO>::n, E = 16 / Elem<T>::bytes;
  // queries of a step, tiles of 16 of them, and units
  constexpr int QT = (int)grad_tile(Elem<T>::bytes == 2, W), TQ = QT / 16, UR = kUnit<T>;
  constexpr int QU = QT / UR;
  constexpr int PLANE = QT * R::stride;
  constexpr int IT = (QT * R::CW + 64 * W - 1) / (64 * W);  // words of a tile per thread
  // bytes per query of p and ds in LDS (bf16: 24 of padding, 0 8 16 24 32 40 took 1485 531 549 528
  // 645 530 us at [32,32768,128], 256 keys)
  constexpr int SS = NK * Elem<T>::bytes + (Elem<T>::bytes == 2 ? 24 : 16);
  // dQ: a wave's units are (16 channels, 16 queries), UN of them in all; of two tiles it takes
  // both, where it has several
  constexpr int UN = TQ * DT, U = (UN + W - 1) / W;
  constexpr int UQ = TQ == 2 && U > 1 ? 2 : 1, SL = U / UQ;
  // Where registers run out, keys are read from LDS in every step: a wave's own and 16 channels
  // of all of them would take KR.
  constexpr int KR = 4 * NV * KT + SL * (NK / UR) * 4;
  constexpr bool KL = ONE && (KR > 48 || W > 8);
  constexpr bool TIGHT = KT * DT >= 16;
  static_assert(NK % UR == 0 && QT % UR == 0, "whole units of keys");
  __shared__ __align__(16) unsigned char tile_[2][1 + OP][PLANE];
  __shared__ __align__(16) unsigned char ds_[QT * SS];
  __shared__ float st[ONE ? W : 1][3][QT];
  __shared__ int rows_[NK];
  __shared__ float bias_[NK];
  __shared__ __align__(16) unsigned char sk[KL ? NK * R::stride : 16];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int m = lane & 15, g = lane >> 4;
  const int part = blockIdx.x % a.shape.parts, chunk = blockIdx.x / a.shape.parts % a.shape.chunks;
  const int64_t s = blockIdx.x / (a.shape.parts * a.shape.chunks);
  const int64_t steps = (a.n_q + QT - 1) / QT;
  const int64_t t0 = (int64_t)part * a.shape.run, t1 = std::min(steps, t0 + a.shape.run);
  const T* Q = static_cast<const T*>(a.Q) + s * a.n_q * D;
  const TO* dO = static_cast<const TO*>(a.dO) + s * a.n_q * D;
  const T* K = static_cast<const T*>(a.K) + s * a.n * D;
  const T* V = static_cast<const T*>(a.V) + s * a.n * D;

  RawWord<T, T> rq[IT];
  RawWord<T, TO> ro[IT];
  // (a tile's words lie behind one another)
  constexpr bool EVEN = QT * R::CW % (64 * W) == 0;
  auto load = [&](int64_t t) __attribute__((always_inline)) {
    const int rows = t < t1 ? (int)std::min<int64_t>(QT, a.n_q - t * QT) : 0;
    const int64_t at = rows > 0 ? t * QT * D : 0;
    const Span q(Q + at, rows * D * Elem<T>::bytes), o(dO + at, rows * D * Elem<TO>::bytes);
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      rq[i].load(q, i * 64 * W + threadIdx.x);
      ro[i].load(o, i * 64 * W + threadIdx.x);
    }
  };
  // without ONE, the next step's statistics: maximum, 1 / sum (0 past the last row), sum p g
  uint32_t next[3][TQ];
  auto statistics = [&](int64_t t) __attribute__((always_inline)) {
    const int rows = t < t1 ? (int)std::min<int64_t>(QT, a.n_q - t * QT) : 0;
    const int64_t at = s * a.n_q + (rows > 0 ? t * QT : 0);
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      const Span x(a.stats + k * a.S * a.n_q + at, rows * 4);
#pragma unroll
      for (int tq = 0; tq < TQ; ++tq) next[k][tq] = x.load4((16 * tq + m) * 4);
    }
  };
  auto put = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      const int item = i * 64 * W + (int)threadIdx.x;
      if (!EVEN && item >= QT * R::CW) continue;
      const int to = item / R::CW * R::stride + item % R::CW * 16;
      u32x4 w[3];
      rq[i].parts(w);
      *reinterpret_cast<u32x4*>(tile_[buf][0] + to) = w[0];
      ro[i].parts(w);
#pragma unroll
      for (int p = 0; p < OP; ++p) *reinterpret_cast<u32x4*>(tile_[buf][1 + p] + to) = w[p];
    }
  };
  load(t0);

  // the rows of the workgroup's keys, then this wave's
  for (int j = threadIdx.x; j < NK; j += 64 * W)
    rows_[j] = coreset_row<T>(a, s, (int64_t)chunk * NK + j, &bias_[j]);
  __syncthreads();
  uint4 kf[KL ? 1 : KT][NV], vf[KT][NV];
  float bias[KT][4];
#pragma unroll
  for (int kt = 0; kt < KT; ++kt) {
    const int key = (wave * KT + kt) * 16 + m, r = rows_[key];
#pragma unroll
    for (int j = 0; j < 4; ++j) bias[kt][j] = bias_[(wave * KT + kt) * 16 + 4 * g + j];
    uint4* kw = kf[KL ? 0 : kt];
    load_frag<T, D>(K, r, g, r >= 0, kw);
    load_frag<T, D>(V, r, g, r >= 0, vf[kt]);
    if (KL) {
#pragma unroll
      for (int v = 0; v < NV; ++v)
        *reinterpret_cast<uint4*>(sk + key * R::stride + (4 * v + g) * 16) = kw[v];
    }
  }
  // columns of every key for dQ
  Column<T> kc[KL ? 1 : SL][NK / UR];
  const int unit0 = wave * U;
  const bool has_unit = U * W == UN || unit0 < UN;
  const int dt0 = TQ == 2 ? unit0 / 2 : unit0;
  if (ONE && !KL && has_unit) {
#pragma unroll
    for (int x = 0; x < NK / UR; ++x) {
      float f[SL][UR / 16][4];
#pragma unroll
      for (int i = 0; i < UR / 4; ++i) {
        const int r = rows_[UR * x + i / 4 * 16 + 4 * g + i % 4];
        // (loaded in any case: a branch would wait for every load by itself)
        const T* row = K + (int64_t)std::max(r, 0) * D;
#pragma unroll
        for (int y = 0; y < SL; ++y) {
          const float v = elem<T>(row, 16 * (dt0 + y) + m);
          f[y][i / 4][i % 4] = r >= 0 ? v : 0.0f;
        }
      }
#pragma unroll
      for (int y = 0; y < SL; ++y) kc[y][x] = Column<T>(f[y]);
    }
  }
  // whether this wave has keys at all, and the units of keys that some wave has
  const int64_t have = a.n_out - (int64_t)chunk * NK;
  // (not in waves of several tiles, where the branches cost registers, 69 -> 82 us for 128 keys of
  // 32 channels, nor among twelve, most of which have keys, 488 -> 511 us for 192)
  constexpr bool SKIP = KT == 1 && W < 12;
  const bool active = !SKIP || wave * 16 < have;
  const int units = !SKIP ? NK / UR : (int)std::min<int64_t>(NK / UR, (have + UR - 1) / UR);
  put(0);
  load(t0 + 1);
  if (!ONE) statistics(t0);

  floatx4_t ak[KT][DT], av[KT][DT];
  float aw[KT][4];
#pragma unroll
  for (int kt = 0; kt < KT; ++kt) {
#pragma unroll
    for (int j = 0; j < 4; ++j) aw[kt][j] = 0.0f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) ak[kt][dt] = av[kt][dt] = (floatx4_t){0.f, 0.f, 0.f, 0.f};
  }
  const float rd = (float)(1.0 / sqrt((double)D));

  // this workgroup's share of the zeros of dK and dV, in 16-byte words: as many in a step as the
  // step's queries have, the rest of them behind the last step
  const int64_t words = a.n * D / E;
  const int64_t zs = (words + a.shape.parts - 1) / a.shape.parts;
  int64_t z = chunk == 0 && !a.zeros ? std::min(words, part * zs) : words;
  const int64_t z1 = std::min(words, z + zs);
  auto zeros = [&]() __attribute__((always_inline)) {
    const int64_t at = s * a.n * D + std::min(z, z1) * E;
    const int left = (int)std::max<int64_t>(0, std::min<int64_t>(z1 - z, IT * 64 * W)) * 16;
    const Span k(static_cast<T*>(a.dK) + at, left), v(static_cast<T*>(a.dV) + at, left);
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      k.stream((u32x4){0, 0, 0, 0}, (i * 64 * W + threadIdx.x) * 16);
      v.stream((u32x4){0, 0, 0, 0}, (i * 64 * W + threadIdx.x) * 16);
    }
    z += IT * 64 * W;
  };

  // dQ of the step before from its ds, and its stores
  Four<T> dq[SL][UQ];
  auto tile_of = [&](int u) { return UQ == 2 ? u : TQ == 2 ? unit0 % 2 : 0; };
  auto queries = [&]() __attribute__((always_inline)) {
    if (!has_unit) return;
#pragma unroll
    for (int y = 0; y < SL; ++y) {
      floatx4_t o[UQ];
#pragma unroll
      for (int u = 0; u < UQ; ++u) o[u] = (floatx4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int x = 0; x < NK / UR; ++x) {
        if (SKIP && x > 0 && x >= units) break;
        const Column<T> k = KL ? Column<T>(sk + UR * x * R::stride, R::stride, dt0 + y, m, g)
                               : kc[KL ? 0 : y][x];
#pragma unroll
        for (int u = 0; u < UQ; ++u)
          o[u] = k.times(Column<T>(ds_ + (16 * tile_of(u) + m) * SS + UR * x * Elem<T>::bytes, g),
                         o[u]);
        if (TIGHT) __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int u = 0; u < UQ; ++u) dq[y][u] = Four<T>(o[u] * rd);
    }
  };
  auto put_queries = [&](int64_t t) __attribute__((always_inline)) {
    const int rows = has_unit && t >= t0 ? (int)std::min<int64_t>(QT, a.n_q - t * QT) : 0;
    const Span o(static_cast<T*>(a.dQ) + (s * a.n_q + std::max(t, t0) * QT) * D,
                 rows * D * Elem<T>::bytes);
#pragma unroll
    for (int y = 0; y < SL; ++y)
#pragma unroll
      for (int u = 0; u < UQ; ++u)
        o.store(dq[y][u].w,
                (uint32_t)((16 * tile_of(u) + m) * D + 16 * (dt0 + y) + 4 * g) * Elem<T>::bytes);
  };

  // scores (of bf16 rows to base 2, of float32 to e) and g of keys 4 g + j, query 16 tq + m
  auto scores = [&](int buf, float (&p)[KT][TQ][4], float (&gd)[KT][TQ][4])
                    __attribute__((always_inline)) {
    floatx4_t x[KT][TQ], y[KT][TQ];
#pragma unroll
    for (int i = 0; i < TQ * KT; ++i)
      x[i / TQ][i % TQ] = y[i / TQ][i % TQ] = (floatx4_t){0.f, 0.f, 0.f, 0.f};
    // (a word of the keys serves both tiles, or, where registers are short, one after the other)
    constexpr int QS = TIGHT ? 1 : TQ;
    // float32 rows' sums over many channels, or of many keys, in two halves: errors of a gradient
    // over 532 keys of 128 channels 1.5e-6 -> 7e-7 (128 keys of 64 in one workgroup gain little
    // and would take 239 us for 235)
    constexpr bool HALVES = Elem<T>::bytes == 4 && QS == TQ && (!ONE || D == 128);
    floatx4_t x0[KT][TQ], y0[KT][TQ];
#pragma unroll
    for (int q0 = 0; q0 < TQ; q0 += QS)
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        if (HALVES && v == NV / 2) {
#pragma unroll
          for (int i = 0; i < TQ * KT; ++i) {
            x0[i / TQ][i % TQ] = x[i / TQ][i % TQ];
            y0[i / TQ][i % TQ] = y[i / TQ][i % TQ];
            x[i / TQ][i % TQ] = y[i / TQ][i % TQ] = (floatx4_t){0.f, 0.f, 0.f, 0.f};
          }
        }
        uint4 kw[KT];
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
          kw[kt] = KL ? lds_word<T, D>(sk + (wave * KT + kt) * 16 * R::stride, v, m, g)
                      : kf[KL ? 0 : kt][v];
#pragma unroll
        for (int tq = q0; tq < q0 + QS; ++tq) {
          const uint4 qw = lds_word<T, D>(tile_[buf][0] + 16 * tq * R::stride, v, m, g);
#pragma unroll
          for (int kt = 0; kt < KT; ++kt) x[kt][tq] = mma_word<T>(kw[kt], qw, x[kt][tq]);
#pragma unroll
          for (int o = OP - 1; o >= 0; --o) {
            const uint4 ow = lds_word<T, D>(tile_[buf][1 + o] + 16 * tq * R::stride, v, m, g);
#pragma unroll
            for (int kt = 0; kt < KT; ++kt) y[kt][tq] = mma_word<T>(vf[kt][v], ow, y[kt][tq]);
          }
        }
        if (TIGHT) __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
    for (int i = 0; i < 4 * TQ * KT; ++i) {
      const int kt = i / (4 * TQ), tq = i / 4 % TQ, j = i % 4;
      if (HALVES) {
        x[kt][tq][j] += x0[kt][tq][j];
        y[kt][tq][j] += y0[kt][tq][j];
      }
      p[kt][tq][j] = score<T, D>(x[kt][tq][j], bias[kt][j]);
      gd[kt][tq][j] = y[kt][tq][j];
    }
  };
  auto add = [](float x, float y) { return x + y; };
  auto larger = [](float x, float y) { return fmaxf(x, y); };
  // weights under the wave's own maxima (top), and the wave's statistics
  auto local = [&](float (&p)[KT][TQ][4], const float (&gd)[KT][TQ][4], float (&top)[TQ])
                   __attribute__((always_inline)) {
#pragma unroll
    for (int tq = 0; tq < TQ; ++tq) {
      float x = kLeast, l = 0.0f, e = 0.0f;
#pragma unroll
      for (int i = 0; i < 4 * KT; ++i) x = fmaxf(x, p[i / 4][tq][i % 4]);
      x = across_rows(x, true, larger);
#pragma unroll
      for (int i = 0; i < 4 * KT; ++i) {
        float& w = p[i / 4][tq][i % 4];
        w = weight<T>(w - x);
        l += w;
        e = fmaf(w, gd[i / 4][tq][i % 4], e);
      }
      l = across_rows(l, true, add);
      e = across_rows(e, true, add);
      top[tq] = x;
      if (g == 0) {
        st[wave][0][16 * tq + m] = x;
        st[wave][1][16 * tq + m] = l;
        st[wave][2][16 * tq + m] = e;
      }
    }
  };
  // The waves' statistics under one maximum: lane l takes row l % 32 of half of the waves, then
  // the halves meet, and rows of 16 lanes trade the two tiles' queries.
  auto joined = [&](const float (&top)[TQ], float (&f)[TQ], float (&dm)[TQ])
                    __attribute__((always_inline)) {
    if constexpr (TQ == 1) {  // (float32: every lane its own row)
      float mx = kLeast, l = 0.0f, e = 0.0f;
#pragma unroll
      for (int w = 0; w < W; ++w) mx = fmaxf(mx, st[w][0][m]);
#pragma unroll
      for (int w = 0; w < W; ++w) {
        const float k = weight<T>(st[w][0][m] - mx);
        l = fmaf(st[w][1][m], k, l);
        e = fmaf(st[w][2][m], k, e);
      }
      const float inv = l > 0.0f ? 1.0f / l : 0.0f;
      dm[0] = e * inv;
      f[0] = weight<T>(top[0] - mx) * inv;
    } else {
      const int r = lane & 31, h = lane / 32;
      float x[W / 2], mx = kLeast, l = 0.0f, e = 0.0f;
  #pragma unroll
      for (int w = 0; w < W / 2; ++w) {
        x[w] = st[2 * w + h][0][r];
        mx = fmaxf(mx, x[w]);
      }
      auto halves = [](float v, auto op) {
        float u = v;
        trade(true, v, u);
        return op(v, u);
      };
      mx = halves(mx, larger);
  #pragma unroll
      for (int w = 0; w < W / 2; ++w) {
        const float k = weight<T>(x[w] - mx);
        l = fmaf(st[2 * w + h][1][r], k, l);
        e = fmaf(st[2 * w + h][2][r], k, e);
      }
      l = halves(l, add);
      e = halves(e, add);
      float inv = l > 0.0f ? 1.0f / l : 0.0f, i1 = inv, m1 = mx;
      dm[0] = dm[1] = e * inv;
      trade(false, dm[0], dm[1]);
      trade(false, inv, i1);
      trade(false, mx, m1);
      f[0] = weight<T>(top[0] - mx) * inv;
      f[1] = weight<T>(top[1] - m1) * i1;
    }
  };
  // dK and dV of a step: p times f, ds in place of g, both through LDS by columns, in one place
  auto keys = [&](int buf, float (&p)[KT][TQ][4], float (&gd)[KT][TQ][4], const float (&f)[TQ],
                  const float (&dm)[TQ]) __attribute__((always_inline)) {
    Column<T> wp[KT][QU], ws[KT][QU];
    unsigned char* mine = ds_ + (wave * KT * 16 + 4 * g) * Elem<T>::bytes + m * SS;
    auto put4 = [&](const float* v, int i) {
      store4<T>(reinterpret_cast<T*>(mine + i / TQ * 16 * Elem<T>::bytes + i % TQ * 16 * SS),
                (floatx4_t){v[0], v[1], v[2], v[3]});
    };
#pragma unroll
    for (int i = 0; i < 4 * TQ * KT; ++i) {
      const int kt = i / (4 * TQ), tq = i / 4 % TQ, j = i % 4;
      p[kt][tq][j] *= f[tq];
      gd[kt][tq][j] = p[kt][tq][j] * (gd[kt][tq][j] - dm[tq]);
    }
    if (a.part_w) {
#pragma unroll
      for (int i = 0; i < 4 * TQ * KT; ++i)
        aw[i / (4 * TQ)][i % 4] += gd[i / (4 * TQ)][i / 4 % TQ][i % 4];
    }
#pragma unroll
    for (int i = 0; i < TQ * KT; ++i) put4(p[i / TQ][i % TQ], i);
#pragma unroll
    for (int i = 0; i < KT * QU; ++i)
      wp[i / QU][i % QU] = Column<T>(ds_ + i % QU * UR * SS, SS, wave * KT + i / QU, m, g);
#pragma unroll
    for (int i = 0; i < TQ * KT; ++i) put4(gd[i / TQ][i % TQ], i);
#pragma unroll
    for (int i = 0; i < KT * QU; ++i)
      ws[i / QU][i % QU] = Column<T>(ds_ + i % QU * UR * SS, SS, wave * KT + i / QU, m, g);
    // (of wide waves one pair of columns at a time: more of them on their way cost registers
    // that are not there)
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
#pragma unroll
      for (int h = 0; h < QU; ++h) {
        const int at = h * UR * R::stride;
#pragma unroll
        for (int o = std::min(OP, 2) - 1; o >= 0; --o) {  // (dV rounds to bf16: 17 bits do)
          const Column<T> x(tile_[buf][1 + o] + at, R::stride, dt, m, g);
#pragma unroll
          for (int kt = 0; kt < KT; ++kt) av[kt][dt] = x.times(wp[kt][h], av[kt][dt]);
        }
        const Column<T> x(tile_[buf][0] + at, R::stride, dt, m, g);
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) ak[kt][dt] = x.times(ws[kt][h], ak[kt][dt]);
      }
      if (TIGHT) __builtin_amdgcn_sched_barrier(0);
    }
  };

  // (Memory operations end in order, stores too: a step makes a number of them that the compiler
  // knows, so that its wait for the next tile's words is none for the stores made since.)
  __syncthreads();
  float p[KT][TQ][4], gd[KT][TQ][4], f[TQ], dm[TQ], top[TQ];
  if (ONE && !active) {  // (a wave without keys: nothing to add, in any step)
    for (int i = lane; i < QT; i += 64) {
      st[wave][0][i] = kLeast;
      st[wave][1][i] = st[wave][2][i] = 0.0f;
    }
    // (the ds that dQ's last unit of keys reads)
#pragma unroll
    for (int i = 0; i < TQ * KT; ++i)
      store4<T>(reinterpret_cast<T*>(ds_ + (i % TQ * 16 + m) * SS +
                                     ((wave * KT + i / TQ) * 16 + 4 * g) * Elem<T>::bytes),
                (floatx4_t){0.f, 0.f, 0.f, 0.f});
  }
  for (int64_t t = t0; t < t1; ++t) {
    const int buf = (int)(t - t0) & 1;
    if (active) {
      scores(buf, p, gd);
      if (ONE) local(p, gd, top);
    }
    if (ONE) {
      if (t > t0) queries();
      __syncthreads();
      if (active) joined(top, f, dm);
      put_queries(t - 1);
    } else {
#pragma unroll
      for (int tq = 0; tq < TQ; ++tq) {
        f[tq] = __uint_as_float(next[1][tq]);
        dm[tq] = __uint_as_float(next[2][tq]);
        // (a row past the last has scores of the log-weights alone, under no maximum)
        const float mx = f[tq] > 0.0f ? __uint_as_float(next[0][tq]) : INFINITY;
#pragma unroll
        for (int i = 0; i < 4 * KT; ++i)
          p[i / 4][tq][i % 4] = weight<T>(p[i / 4][tq][i % 4] - mx);
      }
      statistics(t + 1);
    }
    zeros();
    if (active) keys(buf, p, gd, f, dm);
    put(buf ^ 1);
    load(t + 2);
    __syncthreads();
  }
  if (ONE) {
    queries();
    put_queries(t1 - 1);
  }
  for (int64_t i = (z1 - z + IT * 64 * W - 1) / (IT * 64 * W); i > 0; --i) zeros();

  float* out = a.part + (int64_t)blockIdx.x * NK * 2 * D;
#pragma unroll
  for (int kt = 0; kt < KT; ++kt) {
    const int key = (wave * KT + kt) * 16 + m;
    float* o = out + (int64_t)key * 2 * D + 4 * g;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      *reinterpret_cast<floatx4_t*>(o + 16 * dt) = ak[kt][dt];
      *reinterpret_cast<floatx4_t*>(o + D + 16 * dt) = av[kt][dt];
    }
    if (a.part_w) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float w = row_reduce(aw[kt][j], [](float x, float y) { return x + y; });
        if (m == 0) a.part_w[(int64_t)blockIdx.x * NK + key + 4 * g + j] = w;
      }
    }
  }
}

// ---------------------------------------------------------------------------
// Rows, for coresets wider than a workgroup holds: SH waves take 16 queries and walk the keys
// twice, for the rows' statistics, then for dQ; of a step's keys each takes its share, and they
// join statistics and sums through LDS.  Scores S^T = K Q^T: lane (m, g) holds keys 4 g .. 4 g + 3
// of query m.
//
// 15 slices of 2047 queries over 333 keys, d = 128, bf16 with a float32 dO: 39 us, the matrix
// cores busy for 30 % of the waves' cycles, LDS 27 %, the vector ALU 37 %: the rest are a step's
// latencies, two waves per SIMD that meet at a barrier every 64 keys.  About half of it is the
// second pass, which forms scores and g again: up to a few hundred keys they could stay in
// registers between the passes, which has not been tried.
// ---------------------------------------------------------------------------
constexpr int RW = 8;  // waves

template <typename T, typename TO, int D, int SH>
__global__ __launch_bounds__(64 * RW) void grad_rows_kernel(GradArgs a) {
  using R = LdsRows<T, D>;
  constexpr int NV = Frag<T, D>::NV, DT = D / 16, OP = Parts<T, TO>::n;
  constexpr bool HALVES = Elem<T>::bytes == 4;  // (as above)
  // a wave's tiles of a step's keys, and these
  constexpr int KT = std::max(4 / SH, kUnit<T> / 16), CK = 16 * KT * SH;
  constexpr int IT = (CK * R::CW + 64 * RW - 1) / (64 * RW);  // words of a step per thread
  __shared__ __align__(16) unsigned char sk[2][CK * R::stride], sv[2][CK * R::stride];
  __shared__ float sb[2][CK];
  __shared__ float st[SH > 1 ? RW : 1][3][16];
  constexpr int RT = RW / SH;  // tiles of 16 queries
  const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), sub = wave % SH;
  const int64_t blocks = (a.n_q + 16 * RT - 1) / (16 * RT);
  const int64_t s = blockIdx.x / blocks;
  const int64_t r0 = (blockIdx.x % blocks * RT + wave / SH) * 16;  // the wave's first query
  const int64_t r = r0 + m;                                        // this lane's
  const bool there = r < a.n_q, active = r0 < a.n_q;
  // A step's rows are on their way while the step before is worked on, and their numbers and
  // log-weights a step before that, without branches: no load waits for another.
  int32_t at[IT];
  float lw[IT], bias[IT];
  u32x4 kw[IT], vw[IT];
  const T* K = static_cast<const T*>(a.K) + s * a.n * D;
  const T* V = static_cast<const T*>(a.V) + s * a.n * D;
  const int32_t* idx = a.idx + s * a.n_out;
  const float* logw = a.logw ? a.logw + s * a.n_out : reinterpret_cast<const float*>(idx);
  auto place = [&](int64_t k0, int i) { return k0 + (i * 64 * RW + (int)threadIdx.x) / R::CW; };
  auto number = [&](int64_t k0) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      const int64_t j = std::min(place(k0, i), a.n_out - 1);
      at[i] = idx[j];
      lw[i] = logw[j];
    }
  };
  auto load = [&](int64_t k0) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      const float w = a.logw ? lw[i] : 0.0f;
      const bool is = place(k0, i) < a.n_out && w != -INFINITY;
      bias[i] = is ? w * kUnitScore<T> : -INFINITY;
      const int64_t word = (int64_t)nearest_row(at[i], a.n) * R::CW + threadIdx.x % R::CW;
      kw[i] = reinterpret_cast<const u32x4*>(K)[word];
      vw[i] = reinterpret_cast<const u32x4*>(V)[word];
    }
  };
  auto put = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      const int item = i * 64 * RW + (int)threadIdx.x;
      if (CK * R::CW % (64 * RW) != 0 && item >= CK * R::CW) continue;
      const int to = item / R::CW * R::stride + item % R::CW * 16;
      const u32x4 none = {0, 0, 0, 0};
      const bool is = bias[i] != -INFINITY;
      *reinterpret_cast<u32x4*>(sk[buf] + to) = is ? kw[i] : none;
      *reinterpret_cast<u32x4*>(sv[buf] + to) = is ? vw[i] : none;
      if (item % R::CW == 0) sb[buf][item / R::CW] = bias[i];
    }
  };
  static_assert(64 * RW % R::CW == 0, "a thread's words lie in one column");
  const int64_t steps = (a.n_out + CK - 1) / CK;
  // step i of 2 * steps: the keys twice
  auto first = [&](int64_t i) { return (i < steps ? i : i - steps) * CK; };
  number(0);
  load(0);
  number(first(1));

  uint4 qf[NV], of[OP][NV];
  load_frag<T, D>(static_cast<const T*>(a.Q), s * a.n_q + r, g, there, qf);
  const Span dO(static_cast<const TO*>(a.dO) + (s * a.n_q + std::min(r0, a.n_q - 1)) * D,
                (int)std::max<int64_t>(0, std::min<int64_t>(16, a.n_q - r0)) * D *
                    Elem<TO>::bytes);
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    RawWord<T, TO> w;
    w.load(dO, m * R::CW + 4 * v + g);
    u32x4 x[3];
    w.parts(x);
#pragma unroll
    for (int p = 0; p < OP; ++p) of[p][v] = __builtin_bit_cast(uint4, x[p]);
  }
  const float rd = (float)(1.0 / sqrt((double)D));
  // all parts of dO for the statistics, from which dlogw is; two for dQ, which rounds to bf16
  auto products = [&](int buf, auto parts, float (&p)[KT][4], float (&gd)[KT][4])
                      __attribute__((always_inline)) {
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
      floatx4_t x = {0.f, 0.f, 0.f, 0.f}, y = x, x0 = x, y0 = x;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        if (HALVES && v == NV / 2) {
          x0 = x;
          y0 = y;
          x = y = (floatx4_t){0.f, 0.f, 0.f, 0.f};
        }
        const int at = 16 * (sub * KT + kt) * R::stride;
        x = mma_word<T>(lds_word<T, D>(sk[buf] + at, v, m, g), qf[v], x);
        const uint4 vw = lds_word<T, D>(sv[buf] + at, v, m, g);
#pragma unroll
        for (int o = decltype(parts)::value - 1; o >= 0; --o) y = mma_word<T>(vw, of[o][v], y);
      }
      if (HALVES) {
        x += x0;
        y += y0;
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        p[kt][j] = score<T, D>(x[j], sb[buf][16 * (sub * KT + kt) + 4 * g + j]);
        gd[kt][j] = y[j];
      }
    }
  };
  put(0);
  load(first(1));
  number(first(2));
  __syncthreads();

  float mx = kLeast, l = 0.0f, e = 0.0f;
  int64_t i = 0;
  auto turn = [&]() __attribute__((always_inline)) {
    put((int)(i + 1) & 1);
    load(first(i + 2));
    number(first(i + 3));
    __syncthreads();
  };
  for (; i < steps; ++i) {
    if (active) {
      float p[KT][4], gd[KT][4];
      products((int)i & 1, std::integral_constant<int, OP>(), p, gd);
      float x = mx;
#pragma unroll
      for (int j = 0; j < 4 * KT; ++j) x = fmaxf(x, p[j / 4][j % 4]);
      const float k = weight<T>(mx - x);
      mx = x;
      l *= k;
      e *= k;
#pragma unroll
      for (int j = 0; j < 4 * KT; ++j) {
        const float w = weight<T>(p[j / 4][j % 4] - mx);
        l += w;
        e = fmaf(w, gd[j / 4][j % 4], e);
      }
    }
    turn();
  }
  auto add = [](float x, float y) { return x + y; };
  float top = across_rows(mx, true, [](float x, float y) { return fmaxf(x, y); });
  const float k = weight<T>(mx - top);
  l = across_rows(l * k, true, add);
  e = across_rows(e * k, true, add);
  if constexpr (SH > 1) {
    if (g == 0) {
      st[wave][0][m] = top;
      st[wave][1][m] = l;
      st[wave][2][m] = e;
    }
    __syncthreads();
    const int w0 = wave - sub;
#pragma unroll
    for (int w = 0; w < SH; ++w) top = fmaxf(top, st[w0 + w][0][m]);
    l = e = 0.0f;
#pragma unroll
    for (int w = 0; w < SH; ++w) {
      const float k = weight<T>(st[w0 + w][0][m] - top);
      l = fmaf(st[w0 + w][1][m], k, l);
      e = fmaf(st[w0 + w][2][m], k, e);
    }
  }
  // (a row that no key weighs in: probabilities of 0)
  const float inv = l > 0.0f ? 1.0f / l : 0.0f, dm = e * inv;
  if (there && g == 0 && sub == 0) {
    a.stats[s * a.n_q + r] = top;
    a.stats[(a.S + s) * a.n_q + r] = inv;
    a.stats[(2 * a.S + s) * a.n_q + r] = dm;
  }
  floatx4_t acc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) acc[dt] = (floatx4_t){0.f, 0.f, 0.f, 0.f};
  for (; i < 2 * steps; ++i) {
    const int buf = (int)i & 1;
    if (active) {
      float p[KT][4], gd[KT][4];
      products(buf, std::integral_constant<int, (OP < 2 ? OP : 2)>(), p, gd);
#pragma unroll
      for (int j = 0; j < 4 * KT; ++j)
        p[j / 4][j % 4] =
            weight<T>(p[j / 4][j % 4] - top) * inv * (gd[j / 4][j % 4] - dm);
#pragma unroll
      for (int h = 0; h < 16 * KT / kUnit<T>; ++h) {
        const Column<T> w(p + h * (kUnit<T> / 16));
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
          acc[dt] = Column<T>(sk[buf] + (16 * KT * sub + kUnit<T> * h) * R::stride, R::stride, dt,
                              m, g)
                        .times(w, acc[dt]);
      }
    }
    turn();
  }
  if constexpr (SH > 1) {  // the keys' place is free now
    constexpr int PER = (SH - 1) * 64;
    static_assert(RT * PER * DT * 16 <= (int)sizeof(sk), "room for the waves' sums");
    floatx4_t* sums = reinterpret_cast<floatx4_t*>(sk[0]) + wave / SH * PER * DT;
    if (sub > 0)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) sums[(dt * (SH - 1) + sub - 1) * 64 + lane] = acc[dt];
    __syncthreads();
    if (sub > 0) return;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int w = 0; w < SH - 1; ++w) acc[dt] += sums[(dt * (SH - 1) + w) * 64 + lane];
  }
  if (!there) return;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
    store4<T>(static_cast<T*>(a.dQ) + (s * a.n_q + r) * D + 16 * dt + 4 * g, acc[dt] * rd);
}

// ---------------------------------------------------------------------------
// Join: a wave adds the sums of one coreset row in the order of the queries and writes its row
// of dK and dV; where there are many parts, four waves share them (64 parts of 32 rows: 8.2 us
// with one).  A row that the coreset lists more than once is written by the first place whose
// key is there, with the sums of all of them; a row whose keys are not there keeps its zeros, so
// that a list's padding (one row, listed by every place of it) is no chain of sums.
// ---------------------------------------------------------------------------
template <typename T, int D, int PER>
__global__ __launch_bounds__(256) void grad_join_kernel(GradArgs a) {
  __shared__ floatx4_t sums[PER][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sub = wave % PER;
  const int64_t w = blockIdx.x * (int64_t)(4 / PER) + wave / PER;
  if (w >= a.S * a.n_out) return;
  const int64_t s = w / a.n_out, j = w % a.n_out;
  const int64_t NK = a.shape.keys();
  const int32_t* idx = a.idx + s * a.n_out;
  auto slot = [&](int64_t i, int part) {
    return ((s * a.shape.chunks + i / NK) * a.shape.parts + part) * NK + i % NK;
  };
  if (a.dlogw && sub == 0) {
    float x = 0.0f;
    for (int p = lane; p < a.shape.parts; p += 64) x += a.part_w[slot(j, p)];
#pragma unroll
    for (int i = 32; i > 0; i /= 2) x += __shfl_xor(x, i);
    if (lane == 0) a.dlogw[w] = x;
  }
  const float* logw = a.logw ? a.logw + s * a.n_out : nullptr;
  const int32_t r = nearest_row(idx[j], a.n);
  if (logw && logw[j] == -INFINITY) return;
  constexpr int V = 2 * D / 4;  // lanes of a row of sums, four channels each
  floatx4_t o = {0.f, 0.f, 0.f, 0.f};
  constexpr int BATCH = 8;  // places of the list per lane at a time
  for (int64_t i0 = 0; i0 < a.n_out; i0 += 64 * BATCH) {
    int32_t at[BATCH];
#pragma unroll
    for (int x = 0; x < BATCH; ++x) {
      const int64_t i = i0 + x * 64 + lane;
      at[x] = nearest_row(idx[i < a.n_out ? i : a.n_out - 1], a.n);
    }
#pragma unroll
    for (int x = 0; x < BATCH; ++x) {
      const int64_t place = i0 + x * 64 + lane;
      uint64_t same = __ballot(at[x] == r && place < a.n_out);
      // (the weights of other places alone: 1024 keys' join 4 us longer with all of them)
      if (logw && __ballot(at[x] == r && place < a.n_out && place != j))
        same &= __ballot(logw[std::min(place, a.n_out - 1)] != -INFINITY);
      while (same) {
        const int64_t i = i0 + x * 64 + __ffsll((unsigned long long)same) - 1;
        same &= same - 1;
        if (i < j) return;  // (all waves of the row)
        if (lane < V) {
          const float* p = a.part + slot(i, 0) * 2 * D + lane * 4;
#pragma unroll 8
          for (int y = sub; y < a.shape.parts; y += PER)
            o += *reinterpret_cast<const floatx4_t*>(p + y * NK * 2 * D);
        }
      }
    }
  }
  if constexpr (PER > 1) {
    sums[sub][lane] = o;
    __syncthreads();
    if (sub > 0) return;
#pragma unroll
    for (int x = 1; x < PER; ++x) o += sums[x][lane];
  }
  if (lane >= V) return;
  const bool key = lane < D / 4;
  if (key) o *= (float)(1.0 / sqrt((double)D));
  store4<T>(static_cast<T*>(key ? a.dK : a.dV) + (s * a.n + r) * D + lane % (D / 4) * 4, o);
}

template <typename T, typename TO, int D, int W, int KT, bool ONE>
hipError_t keys_as(const GradArgs& a, hipStream_t st) {
  const uint32_t grid = (uint32_t)(a.S * a.shape.chunks * a.shape.parts);
  grad_keys_kernel<T, TO, D, W, KT, ONE><<<grid, 64 * W, 0, st>>>(a);
  return hipGetLastError();
}

// The shapes of grad_shape.
template <typename T, typename TO, int D>
hipError_t keys_d(const GradArgs& a, hipStream_t st) {
  constexpr bool LOW = Elem<T>::bytes == 2;
  constexpr int CHUNK = LOW && D < 128 ? 2 : 1;
  if (!a.shape.one) return keys_as<T, TO, D, 8, CHUNK, false>(a, st);
  const int w = a.shape.waves, t = a.shape.tiles;
  if (w == 2 && t == 1) return keys_as<T, TO, D, 2, 1, true>(a, st);
  if constexpr (LOW && D == 32) {
    if (w == 2 && t == 2) return keys_as<T, TO, D, 2, 2, true>(a, st);
    if (w == 2 && t == 4) return keys_as<T, TO, D, 2, 4, true>(a, st);
    if (w == 4 && t == 4) return keys_as<T, TO, D, 4, 4, true>(a, st);
  } else if constexpr (LOW && D == 64) {
    if (w == 4 && t == 1) return keys_as<T, TO, D, 4, 1, true>(a, st);
    if (w == 4 && t == 2) return keys_as<T, TO, D, 4, 2, true>(a, st);
    if (w == 8 && t == 2) return keys_as<T, TO, D, 8, 2, true>(a, st);
  } else if constexpr (LOW) {
    if (w == 4 && t == 1) return keys_as<T, TO, D, 4, 1, true>(a, st);
    if (w == 8 && t == 1) return keys_as<T, TO, D, 8, 1, true>(a, st);
    if (w == 12 && t == 1) return keys_as<T, TO, D, 12, 1, true>(a, st);
    if constexpr (!std::is_same<TO, exact_t>::value)
      if (w == 8 && t == 2) return keys_as<T, TO, D, 8, 2, true>(a, st);
  } else {
    if (w == 4 && t == 1) return keys_as<T, TO, D, 4, 1, true>(a, st);
    if constexpr (D == 32) {
      if (w == 4 && t == 2) return keys_as<T, TO, D, 4, 2, true>(a, st);
    } else {
      if (w == 8 && t == 1) return keys_as<T, TO, D, 8, 1, true>(a, st);
    }
  }
  return hipErrorInvalidValue;
}

template <typename T, typename TO, int D>
hipError_t rows_d(const GradArgs& a, hipStream_t st) {
  const int share = grad_share(a.S, a.n_q);
  const int64_t rows = 16 * RW / share;
  const uint32_t grid = (uint32_t)(a.S * ((a.n_q + rows - 1) / rows));
  if (share == 4)
    grad_rows_kernel<T, TO, D, 4><<<grid, 64 * RW, 0, st>>>(a);
  else if (share == 2)
    grad_rows_kernel<T, TO, D, 2><<<grid, 64 * RW, 0, st>>>(a);
  else
    grad_rows_kernel<T, TO, D, 1><<<grid, 64 * RW, 0, st>>>(a);
  return hipGetLastError();
}

template <typename T, int D>
hipError_t join_d(const GradArgs& a, hipStream_t st) {
  if (a.shape.parts >= 16)  // (and so few rows)
    grad_join_kernel<T, D, 4><<<(uint32_t)(a.S * a.n_out), 256, 0, st>>>(a);
  else
    grad_join_kernel<T, D, 1><<<(uint32_t)((a.S * a.n_out + 3) / 4), 256, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace

// Instance F<rows, gradient of the output, head dimension> of a launch.
#define GRAD_BY_D(F, T, TO)                   \
  return d == 32   ? F<T, TO, 32>(a, st)      \
         : d == 64 ? F<T, TO, 64>(a, st)      \
                   : F<T, TO, 128>(a, st)
#define GRAD_BY_TYPES(F)                                       \
  if (dtype == 0 && out_dtype == 0) GRAD_BY_D(F, float, float);   \
  if (dtype == 0) GRAD_BY_D(F, float, bf16_t);                    \
  if (out_dtype == 0 && a.dlogw) GRAD_BY_D(F, bf16_t, exact_t);   \
  if (out_dtype == 0) GRAD_BY_D(F, bf16_t, float);                \
  GRAD_BY_D(F, bf16_t, bf16_t)

hipError_t launch_grad_zeros(int64_t row_bytes, const GradArgs& a, hipStream_t st) {
  const int64_t words = a.S * a.n * row_bytes / 16;
  grad_zeros_kernel<<<(uint32_t)((words + ZT * ZW - 1) / (ZT * ZW)), ZT, 0, st>>>(
      static_cast<u32x4*>(a.dK), static_cast<u32x4*>(a.dV), words);
  return hipGetLastError();
}
hipError_t launch_grad_rows(int dtype, int out_dtype, int64_t d, const GradArgs& a,
                            hipStream_t st) {
  GRAD_BY_TYPES(rows_d);
}
hipError_t launch_grad_keys(int dtype, int out_dtype, int64_t d, const GradArgs& a,
                            hipStream_t st) {
  GRAD_BY_TYPES(keys_d);
}
hipError_t launch_grad_join(int dtype, int64_t d, const GradArgs& a, hipStream_t st) {
  Q4_BY_D(join_d, a, st);
}

}  // namespace thin
