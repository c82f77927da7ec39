// Store, load and selection of the 4-bit key/value cache on gfx950.
//
// A group of 32 channels with largest magnitude amax takes e = the least integer
// in [-125, 125] with amax <= 7 * 2^e and the codes of x / 2^e rounded to nearest
// (ties to even) in {0, .5, 1, 1.5, 2, 3, 4, 6}: 7 is the value beyond which 6
// would be off by more than half a step.  NaN is stored as 0, values beyond
// 6 * 2^125 as that, so every cached value is a finite normal bf16 or 0: a
// masked row's weight of 0 stays 0 in a product.
#include "common.hpp"
#include "q4.hpp"
#include "q4_device.hpp"

namespace thin {

namespace {

constexpr int THREADS = 256;

// ---------------------------------------------------------------------------
// Store.  A workgroup owns one block of 64 rows of one slice: it encodes the new
// rows that fall into it and forms the block's bounds anew from them and the rows
// before them, so bounds never depend on how rows were grouped into calls, nor on
// rows that a rewound sequence no longer holds.  Four lanes hold a group, eight
// channels each.
// ---------------------------------------------------------------------------
// Codes of eight channels of a group that four neighbouring lanes hold; *byte
// gets the group's scale byte.
__device__ __forceinline__ uint32_t encode8(float* f, uint32_t* byte) {
  float amax = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    f[i] = f[i] != f[i] ? 0.0f : f[i];
    amax = fmaxf(amax, fabsf(f[i]));
  }
  amax = fmaxf(amax, __shfl_xor(amax, 1));
  amax = fmaxf(amax, __shfl_xor(amax, 2));
  // amax = 1.m * 2^(E - 127): e = E - 129 if 1.m <= 1.75, else E - 128
  const uint32_t bits = __float_as_uint(amax);
  int s = (int)(bits >> 23) - ((bits & 0x7fffffu) <= 0x600000u ? 2 : 1);
  s = s < 2 ? 2 : (s > 252 ? 252 : s);
  *byte = (uint32_t)s;
  const float scale = __uint_as_float((uint32_t)s << 23);
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[0], f[1], scale, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[2], f[3], scale, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[4], f[5], scale, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[6], f[7], scale, 3);
  return c;
}

template <typename T, int D>
__global__ __launch_bounds__(THREADS) void q4_store_kernel(Q4View c, RowsView k, RowsView v,
                                                           Q4Tokens tok) {
  constexpr int LR = D / 8;           // lanes per row
  constexpr int RPP = THREADS / LR;   // rows per pass
  const int64_t s = blockIdx.y;
  const int b = blockIdx.y / c.H, h = blockIdx.y % c.H;
  const int64_t at = tok.at[b];
  int64_t cnt = tok.count ? tok.count[b] : tok.T;
  cnt = cnt < 0 ? 0 : (cnt > tok.T ? tok.T : cnt);
  // the new rows that are rows of the cache
  const int64_t lo = at < 0 ? 0 : at, hi = at + cnt < c.n_max ? at + cnt : c.n_max;
  const int64_t r0 = (lo / kQ4Block + blockIdx.x) * kQ4Block;
  if (r0 >= hi) return;
  const int l = threadIdx.x % LR, rp = threadIdx.x / LR;
  float mn[8], mx[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    mn[i] = INFINITY;
    mx[i] = -INFINITY;
  }
#pragma unroll
  for (int p = 0; p < kQ4Block; p += RPP) {
    const int64_t r = r0 + p + rp;
    if (r >= hi) continue;  // (lanes of a row together: the shuffles stay within it)
    const int64_t row = s * c.n_max + r;
    uint32_t code, byte;
    if (r >= lo) {
      float f[8];
      load8<T>(static_cast<const T*>(k.p) + b * k.sb + h * k.sh + (r - at) * k.sr + l * 8, f);
      code = encode8(f, &byte);
      *reinterpret_cast<uint32_t*>(c.k_codes + row * (D / 2) + l * 4) = code;
      if ((l & 3) == 0) c.k_scales[row * (D / 32) + l / 4] = (uint8_t)byte;
      float g[8];
      uint32_t vb;
      load8<T>(static_cast<const T*>(v.p) + b * v.sb + h * v.sh + (r - at) * v.sr + l * 8, g);
      *reinterpret_cast<uint32_t*>(c.v_codes + row * (D / 2) + l * 4) = encode8(g, &vb);
      if ((l & 3) == 0) c.v_scales[row * (D / 32) + l / 4] = (uint8_t)vb;
    } else {
      code = *reinterpret_cast<const uint32_t*>(c.k_codes + row * (D / 2) + l * 4);
      byte = c.k_scales[row * (D / 32) + l / 4];
    }
    uint32_t w[4];
    decode8(code, q4_scale(byte), w);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float a = __uint_as_float(w[i] << 16), d = __uint_as_float(w[i] & 0xffff0000u);
      mn[2 * i] = fminf(mn[2 * i], a);
      mx[2 * i] = fmaxf(mx[2 * i], a);
      mn[2 * i + 1] = fminf(mn[2 * i + 1], d);
      mx[2 * i + 1] = fmaxf(mx[2 * i + 1], d);
    }
  }
  // over the wave's rows, then the four waves
#pragma unroll
  for (int m = LR; m < 64; m *= 2)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      mn[i] = fminf(mn[i], __shfl_xor(mn[i], m));
      mx[i] = fmaxf(mx[i], __shfl_xor(mx[i], m));
    }
  __shared__ float sm[4][2][D];
  if ((threadIdx.x & 63) < LR)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      sm[threadIdx.x / 64][0][l * 8 + i] = mn[i];
      sm[threadIdx.x / 64][1][l * 8 + i] = mx[i];
    }
  __syncthreads();
  if (threadIdx.x < 2 * D) {
    const int which = threadIdx.x / D, ch = threadIdx.x % D;
    float x = sm[0][which][ch];
#pragma unroll
    for (int w = 1; w < 4; ++w) x = which ? fmaxf(x, sm[w][1][ch]) : fminf(x, sm[w][0][ch]);
    const int64_t nb = (c.n_max + kQ4Block - 1) / kQ4Block;
    // (exact: every cached value is a bf16)
    c.bounds[((s * nb + r0 / kQ4Block) * 2 + which) * D + ch] = (uint16_t)(__float_as_uint(x) >> 16);
  }
}

// ---------------------------------------------------------------------------
// Load: rows at[b] .. at[b] + T - 1 as the values they stand for, zeros outside the cache.
// ---------------------------------------------------------------------------
template <typename T, int D>
__global__ __launch_bounds__(THREADS) void q4_load_kernel(Q4View c, const int32_t* at, int64_t T_,
                                                          T* k, T* v) {
  constexpr int LR = D / 8;
  const int64_t s = blockIdx.y, t = blockIdx.x * (int64_t)(THREADS / LR) + threadIdx.x / LR;
  const int l = threadIdx.x % LR;
  if (t >= T_) return;
  const int64_t r = (int64_t)at[blockIdx.y / c.H] + t;
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) {
    uint32_t w[4] = {0, 0, 0, 0};
    if (r >= 0 && r < c.n_max) {
      const int64_t row = s * c.n_max + r;
      const uint32_t code = *reinterpret_cast<const uint32_t*>(
          (kv ? c.v_codes : c.k_codes) + row * (D / 2) + l * 4);
      const uint32_t byte = (kv ? c.v_scales : c.k_scales)[row * (D / 32) + l / 4];
      decode8(code, q4_scale(byte), w);
    }
    T* out = (kv ? v : k) + (s * T_ + t) * D + l * 8;
    if constexpr (Elem<T>::bytes == 2) {
      *reinterpret_cast<u32x4*>(out) = (u32x4){w[0], w[1], w[2], w[3]};
    } else {
      u32x4* o = reinterpret_cast<u32x4*>(out);
      o[0] = (u32x4){w[0] << 16, w[0] & 0xffff0000u, w[1] << 16, w[1] & 0xffff0000u};
      o[1] = (u32x4){w[2] << 16, w[2] & 0xffff0000u, w[3] << 16, w[3] & 0xffff0000u};
    }
  }
}

// ---------------------------------------------------------------------------
// Selection.  The score of a block for a token and key head is the sum over the
// heads g of the group and the channels c of max(q_gc lo_c, q_gc hi_c), the most
// that the block's keys could give: <q+, hi> + <q-, lo> with q+ and q- the sums
// over the group of the positive and the negative parts.  In float64, where the
// products of bf16 values and their sums are exact (or nearly, for float32
// queries), so that the order of a border does not depend on the order of sums.
// ---------------------------------------------------------------------------

// Scores as integers of the same order; NaN below everything, 0 left free for
// blocks that are not there.
__device__ __forceinline__ uint64_t score_key(double s) {
  if (s != s) return 1;
  const uint64_t u = (uint64_t)__double_as_longlong(s + 0.0);  // -0 is 0
  const uint64_t k = (u >> 63) ? ~u : u | 0x8000000000000000ull;
  return k < 2 ? 2 : k;
}

constexpr int SLANES = 8;  // lanes per block's bounds

template <typename T, int D>
__global__ __launch_bounds__(THREADS) void q4_scores_kernel(Q4View c, Q4SelectArgs a) {
  const int64_t s = blockIdx.y;
  const int b = blockIdx.y / c.H, h = blockIdx.y % c.H;
  const int t = a.t0 + blockIdx.x % a.tn, part = blockIdx.x / a.tn;
  const int nb = (c.n_max + kQ4Block - 1) / kQ4Block;
  const int last_row = q4_last_row(a.tok, b, t, c.n_max);
  if (last_row < 0) return;
  const int last = last_row / kQ4Block;
  __shared__ double sq[2 * D];  // q- beside lo, then q+ beside hi
  if (threadIdx.x < D) {
    const T* q = static_cast<const T*>(a.q.p) + b * a.q.sb + (int64_t)h * a.G * a.q.sh + t * a.q.sr;
    double neg = 0.0, pos = 0.0;
    for (int g = 0; g < a.G; ++g) {
      const double x = (double)elem<T>(q + g * a.q.sh, threadIdx.x);
      if (!(x >= 0.0)) neg += x;  // (NaN here, and so in the score)
      if (x > 0.0) pos += x;
    }
    sq[threadIdx.x] = neg;
    sq[D + threadIdx.x] = pos;
  }
  __syncthreads();
  const int j = threadIdx.x % SLANES;
  constexpr int W = 2 * D / 8 / SLANES;  // 16-byte words of bounds per lane
  double q[W][8];
#pragma unroll
  for (int w = 0; w < W; ++w)
#pragma unroll
    for (int i = 0; i < 8; ++i) q[w][i] = sq[(w * SLANES + j) * 8 + i];
  const int step = (int)(gridDim.x / a.tn) * (THREADS / SLANES);
  for (int k = part * (THREADS / SLANES) + threadIdx.x / SLANES; k <= last; k += step) {
    const u32x4* p = reinterpret_cast<const u32x4*>(c.bounds + (s * nb + k) * 2 * D);
    double sum = 0.0;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const u32x4 x = p[w * SLANES + j];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        sum += q[w][2 * i] * (double)__uint_as_float(x[i] << 16);
        sum += q[w][2 * i + 1] * (double)__uint_as_float(x[i] & 0xffff0000u);
      }
    }
#pragma unroll
    for (int m = 1; m < SLANES; m *= 2) sum += __shfl_xor(sum, m);
    if (j == 0) a.scores[(s * a.tn + t - a.t0) * nb + k] = score_key(sum);
  }
}

// The n_sel best of a row's blocks, in order.  A workgroup of W waves holds the
// row's keys, KPL per lane; the least key that stays in is found by halving the
// interval of keys (at most 64 steps, as many as it takes until the count of
// keys above the middle is what is wanted).  Equal keys at the border: the lowest
// blocks.
template <int W, int KPL>
__global__ __launch_bounds__(64 * W) void q4_pick_kernel(Q4View c, Q4SelectArgs a) {
  const int64_t s = blockIdx.y;
  const int b = blockIdx.y / c.H, t = a.t0 + blockIdx.x;
  const int nb = (c.n_max + kQ4Block - 1) / kQ4Block;
  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64;
  int32_t* out = a.blocks + (s * a.tok.T + t) * a.n_sel;
  const uint64_t* keys = a.scores + (s * a.tn + blockIdx.x) * nb;
  const int lr = q4_last_row(a.tok, b, t, c.n_max);
  const int n = lr < 0 ? 0 : lr / kQ4Block + 1;  // blocks that are there
  __shared__ int cnt[2][W];
  // a wave's keys are its KPL runs of 64 blocks
  uint64_t key[KPL];
  const int base = wave * KPL * 64;
#pragma unroll
  for (int i = 0; i < KPL; ++i) {
    const int k = base + i * 64 + lane;
    key[i] = 0;
    if (k < n) key[i] = k < a.n_sinks || k >= n - a.n_window ? ~0ull : keys[k];
  }
  // how many of the workgroup's keys are at least x
  int parity = 0;
  auto count = [&](uint64_t x) {
    int m = 0;
#pragma unroll
    for (int i = 0; i < KPL; ++i) m += __popcll(__ballot(key[i] >= x));
    if (W > 1) {
      if (lane == 0) cnt[parity][wave] = m;
      __syncthreads();
      m = 0;
#pragma unroll
      for (int w = 0; w < W; ++w) m += cnt[parity][w];
      parity ^= 1;
    }
    return m;
  };
  // least x with count(x) <= n_sel: the keys at least x stay, and of those equal
  // to x - 1 the lowest blocks as far as they fit
  uint64_t x = 1;
  int above = n < a.n_sel ? n : a.n_sel;
  if (n > a.n_sel) {
    uint64_t lo = 1, hi = ~0ull;  // count(lo) > n_sel >= count(hi): sinks and window fit
    above = count(hi);
    while (hi - lo > 1) {
      const uint64_t mid = lo + (hi - lo) / 2;
      const int m = count(mid);
      if (m > a.n_sel) {
        lo = mid;
      } else {
        hi = mid;
        above = m;
        if (m == a.n_sel) break;
      }
    }
    x = hi;
  }
  const int ties = (n < a.n_sel ? n : a.n_sel) - above;  // keys equal to x - 1 that stay
  // places in order: waves, then runs of 64
  const uint64_t below = (1ull << lane) - 1;
  int nabove = 0, nties = 0;
#pragma unroll
  for (int i = 0; i < KPL; ++i) {
    nabove += __popcll(__ballot(key[i] >= x));
    nties += __popcll(__ballot(key[i] == x - 1 && key[i] != 0));
  }
  int pa = 0, pt = 0;  // above and ties of the waves before
  if (W > 1) {
    __syncthreads();
    if (lane == 0) {
      cnt[0][wave] = nabove;
      cnt[1][wave] = nties;
    }
    __syncthreads();
    for (int w = 0; w < wave; ++w) {
      pa += cnt[0][w];
      pt += cnt[1][w];
    }
  }
#pragma unroll
  for (int i = 0; i < KPL; ++i) {
    const bool in = key[i] >= x && key[i] != 0, tie = key[i] == x - 1 && key[i] != 0;
    const uint64_t mi = __ballot(in), mt = __ballot(tie);
    const int before = pt + __popcll(mt & below);
    // ties that stay before this one: min(before, ties)
    const int place = pa + __popcll(mi & below) + (before < ties ? before : ties);
    if (in || (tie && before < ties)) out[place] = base + i * 64 + lane;
    pa += __popcll(mi);
    pt += __popcll(mt);
  }
  const int used = n < a.n_sel ? n : a.n_sel;
  for (int i = used + (int)threadIdx.x; i < a.n_sel; i += 64 * W) out[i] = -1;
}

template <typename T, int D>
hipError_t store_d(const Q4View& c, const RowsView& k, const RowsView& v, const Q4Tokens& tok,
                   hipStream_t st) {
  const dim3 grid((uint32_t)((tok.T + kQ4Block - 2) / kQ4Block + 1), (uint32_t)(c.B * c.H));
  q4_store_kernel<T, D><<<grid, THREADS, 0, st>>>(c, k, v, tok);
  return hipGetLastError();
}

template <typename T, int D>
hipError_t load_d(const Q4View& c, const int32_t* at, int64_t T_, void* k, void* v, hipStream_t st) {
  constexpr int per = THREADS / (D / 8);
  const dim3 grid((uint32_t)((T_ + per - 1) / per), (uint32_t)(c.B * c.H));
  q4_load_kernel<T, D><<<grid, THREADS, 0, st>>>(c, at, T_, static_cast<T*>(k), static_cast<T*>(v));
  return hipGetLastError();
}

template <typename T, int D>
hipError_t scores_d(const Q4View& c, const Q4SelectArgs& a, hipStream_t st) {
  const int64_t nb = (c.n_max + kQ4Block - 1) / kQ4Block;
  const int64_t rows = (int64_t)c.B * c.H * a.tn, per = THREADS / SLANES;
  int64_t x = (nb + per - 1) / per;
  const int64_t most = (4096 + rows - 1) / rows;  // workgroups enough to fill the device
  if (x > most) x = most;
  const dim3 grid((uint32_t)(x * a.tn), (uint32_t)(c.B * c.H));
  q4_scores_kernel<T, D><<<grid, THREADS, 0, st>>>(c, a);
  return hipGetLastError();
}

template <int W, int KPL>
hipError_t pick(const Q4View& c, const Q4SelectArgs& a, hipStream_t st) {
  const dim3 grid((uint32_t)a.tn, (uint32_t)(c.B * c.H));
  q4_pick_kernel<W, KPL><<<grid, 64 * W, 0, st>>>(c, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_q4_store(int dtype, int64_t d, const Q4View& c, const RowsView& k,
                           const RowsView& v, const Q4Tokens& tok, hipStream_t st) {
  Q4_BY_D(store_d, c, k, v, tok, st);
}

hipError_t launch_q4_load(int dtype, int64_t d, const Q4View& c, const int32_t* at, int64_t T,
                          void* k, void* v, hipStream_t st) {
  Q4_BY_D(load_d, c, at, T, k, v, st);
}

hipError_t launch_q4_scores(int dtype, int64_t d, const Q4View& c, const Q4SelectArgs& a,
                            hipStream_t st) {
  Q4_BY_D(scores_d, c, a, st);
}

hipError_t launch_q4_pick(const Q4View& c, const Q4SelectArgs& a, hipStream_t st) {
  const int64_t runs = (c.n_max + kQ4Block * 64 - 1) / (kQ4Block * 64);  // runs of 64 blocks
  if (runs <= 2) return pick<1, 2>(c, a, st);
  if (runs <= 8) return pick<1, 8>(c, a, st);
  if (runs <= 32) return pick<4, 8>(c, a, st);
  if (runs <= 128) return pick<16, 8>(c, a, st);
  return pick<16, 32>(c, a, st);
}

}  // namespace thin
