// Attention over the 4-bit key/value cache on gfx950: causal over every cached
// row, or over the rows of the blocks listed for a token and key head.
//
// o = sum_j p_j v_j / sum_j p_j,  p_j = exp(<q, k_j> / sqrt(d) - max).
//
// A code times its power of two is exactly a bf16, so keys and values enter the
// bf16 matrix instructions without loss, for float32 queries too: those split
// into three bf16 parts (24 bits), and so do their weights p.  bf16 queries use
// one bf16 weight: its rounding (2^-9 of a term) is that of the output.
//
// Lane layout of the 16x16x32 instruction: lane l = 16 g + m.  Scores S^T = K Q^T
// (keys x query rows): lane (m, g) feeds key row m's channels of quarter g of the
// head, as they lie in memory (d / 8 bytes of codes, one scale), and of query row
// m the same channels.  Lane (m, g) then holds the scores of keys 4 g .. 4 g + 3
// for query row m, which is what the product O^T = V^T P^T wants as its second
// operand.  Its first, V^T, is read from LDS by the transposing read: a wave keeps
// 32 decoded value rows there.
#include <math.h>

#include <algorithm>

#include "common.hpp"
#include "q4.hpp"
#include "q4_device.hpp"

namespace thin {

namespace {

constexpr int WAVES = 4;
constexpr int CH = 32;  // keys per step of a wave
constexpr float kLowest = -3.0e38f;
constexpr double kLog2e = 1.44269504088896340736;

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

// One wave's step: the codes of 32 keys and values.
template <int D>
struct Codes {
  static constexpr int KB = D / 8;  // bytes of a lane's quarter of a key row
  static constexpr int KW = KB / 4;
  uint32_t k[2][KW];
  uint32_t ks[2];
  // values: VL bytes per lane and item, VI items
  static constexpr int VL = D == 32 ? 8 : 16;
  static constexpr int VR = D / 2 / VL;           // lanes per row
  static constexpr int VI = CH * VR / 64;
  uint32_t v[VI][VL / 4];
  uint32_t vs[VI];
};

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

// Rows row0 .. row0 + 31 of a slice; rows past `last` stand for `last`.
template <int D>
__device__ __forceinline__ void load_codes(const Q4View& c, int64_t s, int64_t row0, int64_t last,
                                           int lane, Codes<D>& x) {
  using C = Codes<D>;
  const int m = lane & 15, g = lane >> 4;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    int64_t r = row0 + t * 16 + m;
    r = s * c.n_max + (r < last ? r : last);
    load_words<C::KW>(c.k_codes + r * (D / 2) + g * C::KB, x.k[t]);
    x.ks[t] = c.k_scales[r * (D / 32) + g * C::KB * 2 / 32];
  }
#pragma unroll
  for (int i = 0; i < C::VI; ++i) {
    const int item = i * 64 + lane;
    int64_t r = row0 + item / C::VR;
    r = s * c.n_max + (r < last ? r : last);
    load_words<C::VL / 4>(c.v_codes + r * (D / 2) + item % C::VR * C::VL, x.v[i]);
    x.vs[i] = c.v_scales[r * (D / 32) + item % C::VR * C::VL * 2 / 32];
  }
}

// Bytes per value row in LDS: 32 past the row put the four rows that 16 lanes read
// together on different banks.
template <int D>
constexpr int kVStride = 2 * D + 32;

// Channels ch .. ch + 3 of query row r of a tile, if there is such a row.
template <typename T, bool LIST>
__device__ __forceinline__ void store_row4(const Q4AttnArgs& a, int64_t b, int64_t h, int64_t tile,
                                           int r, int ch, floatx4_t o) {
  int64_t t, head;
  if (LIST) {
    const int64_t gt = (a.G + 15) / 16;
    t = tile / gt;
    head = tile % gt * 16 + r;
    if (head >= a.G) return;
  } else {
    const int64_t row = tile * 16 + r;
    if (row >= a.tok.T * a.G) return;
    t = row / a.G;
    head = row % a.G;
  }
  T* p = static_cast<T*>(const_cast<void*>(a.o.p)) + b * a.o.sb + (h * a.G + head) * a.o.sh +
         t * a.o.sr + ch;
  if constexpr (Elem<T>::bytes == 2)
    *reinterpret_cast<uint2*>(p) = make_uint2(cvt_pk_bf16(o[0], o[1]), cvt_pk_bf16(o[2], o[3]));
  else
    *reinterpret_cast<floatx4_t*>(p) = o;
}

template <typename T, int D, bool LIST>
__global__ __launch_bounds__(64 * WAVES) void q4_attn_kernel(Q4View c, Q4AttnArgs a) {
  constexpr int NP = Elem<T>::bytes == 2 ? 1 : 3;
  constexpr int KS = D / 32;  // k-steps of the scores
  using C = Codes<D>;
  __shared__ __align__(16) unsigned char lds[WAVES * CH * kVStride<D>];
  __shared__ float sm[WAVES][16], sl[WAVES][16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int m = lane & 15, g = lane >> 4;
  const int64_t s = blockIdx.y, b = s / c.H, h = s % c.H;
  const int64_t split = blockIdx.x % a.splits, tile = blockIdx.x / a.splits;
  // the tile's 16 query rows: heads of one token (LIST), or tokens x heads in a row
  const int64_t gt = (a.G + 15) / 16;
  int64_t t, head, tl;  // this lane's token and head, the tile's last token
  bool there;
  if (LIST) {
    t = tl = tile / gt;
    head = tile % gt * 16 + m;
    there = head < a.G;
  } else {
    const int64_t row = tile * 16 + m, rows = a.tok.T * a.G;
    const int64_t end = std::min(tile * 16 + 15, rows - 1);
    there = row < rows;
    t = there ? row / a.G : 0;
    head = there ? row % a.G : 0;
    tl = end / a.G;
  }
  const int64_t qlast = there ? q4_last_row(a.tok, b, t, c.n_max) : -1;
  // the last row that any of the tile's queries sees
  int64_t last = -1;
  if (LIST) {
    last = q4_last_row(a.tok, b, tl, c.n_max);
  } else {
    const int64_t cnt = a.tok.count ? (int64_t)a.tok.count[b] : a.tok.T;
    if (tl >= cnt) tl = cnt - 1;
    if (tl >= 0 && tl * a.G + a.G > tile * 16) last = q4_last_row(a.tok, b, tl, c.n_max);
  }

  bf16x8_t q[NP][KS];
  {
    const T* qp = static_cast<const T*>(a.q.p) + b * a.q.sb + (h * a.G + head) * a.q.sh +
                  t * a.q.sr + g * (D / 4);
#pragma unroll
    for (int i = 0; i < KS; ++i) {
      float f[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      if (there) load8<T>(qp + i * 8, f);
      bf16x8_t part[NP];
      split8<NP>(f, part);
#pragma unroll
      for (int p = 0; p < NP; ++p) q[p][i] = part[p];
    }
  }

  // steps of 32 keys: the split's share, the waves in turn
  const int64_t steps = LIST ? a.n_sel * (kQ4Block / CH) : (last + CH) / CH;
  const int64_t share = (steps + a.splits - 1) / a.splits;
  const int64_t i1 = std::min(steps, (split + 1) * share);
  const int32_t* list = LIST ? a.blocks + (s * a.tok.T + tl) * a.n_sel : nullptr;
  const int64_t nb = (c.n_max + kQ4Block - 1) / kQ4Block;
  auto row_of = [&](int64_t i) -> int64_t {  // first row of step i, or past `last`
    if (!LIST) return i * CH;
    const int64_t k = list[i / (kQ4Block / CH)];
    return k < 0 || k >= nb ? c.n_max : k * kQ4Block + i % (kQ4Block / CH) * CH;
  };

  const float c2 = (float)(kLog2e / sqrt((double)D));
  float mrun = kLowest, lrun = 0.0f;
  floatx4_t acc[D / 16];
#pragma unroll
  for (int i = 0; i < D / 16; ++i) acc[i] = (floatx4_t){0.f, 0.f, 0.f, 0.f};
  unsigned char* sv = lds + wave * CH * kVStride<D>;

  if (last >= 0) {
    for (int64_t i = split * share + wave; i < i1; i += WAVES) {
      const int64_t row0 = row_of(i);
      if (row0 > last) continue;
      C x;
      load_codes<D>(c, s, row0, last, lane, x);
      float sc[8];
#pragma unroll
      for (int t2 = 0; t2 < 2; ++t2) {
        floatx4_t z = {0.f, 0.f, 0.f, 0.f};
        const float ks = q4_scale(x.ks[t2]);
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          uint32_t w[4];
          decode8(x.k[t2][k], ks, w);
          const bf16x8_t kf = __builtin_bit_cast(bf16x8_t, (u32x4){w[0], w[1], w[2], w[3]});
#pragma unroll
          for (int p = NP - 1; p >= 0; --p)
            z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, q[p][k], z, 0, 0, 0);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
          sc[t2 * 4 + j] = row0 + t2 * 16 + 4 * g + j <= qlast ? z[j] : -INFINITY;
      }
      float mx = sc[0];
#pragma unroll
      for (int j = 1; j < 8; ++j) mx = fmaxf(mx, sc[j]);
      mx = fmaxf(mx, __shfl_xor(mx, 16));
      mx = fmaxf(mx, __shfl_xor(mx, 32));
      const float mnew = fmaxf(mrun, mx);
      const float scale = __builtin_amdgcn_exp2f((mrun - mnew) * c2);
      mrun = mnew;
      float sum = 0.0f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        sc[j] = __builtin_amdgcn_exp2f((sc[j] - mnew) * c2);
        sum += sc[j];
      }
      lrun = lrun * scale + sum;
#pragma unroll
      for (int dt = 0; dt < D / 16; ++dt) acc[dt] *= scale;
      bf16x8_t pp[NP];
      split8<NP>(sc, pp);
      // values to LDS
#pragma unroll
      for (int n = 0; n < C::VI; ++n) {
        const int item = n * 64 + lane;
        unsigned char* to = sv + item / C::VR * kVStride<D> + item % C::VR * C::VL * 4;
        const float vs = q4_scale(x.vs[n]);
#pragma unroll
        for (int w8 = 0; w8 < C::VL / 4; ++w8) {
          uint32_t w[4];
          decode8(x.v[n][w8], vs, w);
          *reinterpret_cast<u32x4*>(to + w8 * 16) = (u32x4){w[0], w[1], w[2], w[3]};
        }
      }
#pragma unroll
      for (int dt = 0; dt < D / 16; ++dt) {
        typedef __attribute__((address_space(3))) s16x4 lds_t;
        unsigned char* from = sv + (4 * g + m / 4) * kVStride<D> + dt * 32 + m % 4 * 8;
        const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t*)from);
        const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t*)(from + 16 * kVStride<D>));
        typedef short s16x8 __attribute__((ext_vector_type(8)));
        const bf16x8_t vf = __builtin_bit_cast(
            bf16x8_t, (s16x8)__builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
        for (int p = NP - 1; p >= 0; --p)
          acc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pp[p], acc[dt], 0, 0, 0);
      }
    }
  }
  lrun += __shfl_xor(lrun, 16);
  lrun += __shfl_xor(lrun, 32);

  // the waves' sums under one maximum
  if (g == 0) {
    sm[wave][m] = mrun;
    sl[wave][m] = lrun;
  }
  __syncthreads();  // (also: every wave is done with its value rows)
  float mall = sm[0][m], lall = 0.0f;
#pragma unroll
  for (int w = 1; w < WAVES; ++w) mall = fmaxf(mall, sm[w][m]);
#pragma unroll
  for (int w = 0; w < WAVES; ++w) lall += sl[w][m] * __builtin_amdgcn_exp2f((sm[w][m] - mall) * c2);
  constexpr int OS = D + 4;  // floats per row of a wave's sums
  static_assert(WAVES * 16 * OS * 4 <= (int)sizeof(lds), "the waves' sums fit the value rows");
  float* so = reinterpret_cast<float*>(lds);
  {
    const float scale = __builtin_amdgcn_exp2f((mrun - mall) * c2);
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) {
      const floatx4_t r = acc[dt] * scale;
      *reinterpret_cast<floatx4_t*>(so + (wave * 16 + m) * OS + dt * 16 + 4 * g) = r;
    }
  }
  // sl and sm of all rows for the threads that write them
  __syncthreads();
  if (wave == 0 && g == 0) {
    sm[0][m] = mall;
    sl[0][m] = lall;
  }
  __syncthreads();
  constexpr int V = D / 4;  // threads per row, four channels each
  for (int i = threadIdx.x; i < 16 * V; i += 64 * WAVES) {
    const int r = i / V, ch = i % V * 4;
    floatx4_t o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < WAVES; ++w)
      o += *reinterpret_cast<const floatx4_t*>(so + (w * 16 + r) * OS + ch);
    if (a.splits > 1) {
      const int64_t slot = (s * (gridDim.x / a.splits) + tile) * a.splits + split;
      *reinterpret_cast<floatx4_t*>(a.part + (slot * 16 + r) * D + ch) = o;
      float* ml = a.part + (int64_t)gridDim.y * gridDim.x * 16 * D + slot * 32;
      if (ch == 0) {
        ml[r] = sm[0][r];
        ml[16 + r] = sl[0][r];
      }
    } else {
      store_row4<T, LIST>(a, b, h, tile, r, ch, o * (sl[0][r] > 0.0f ? 1.0f / sl[0][r] : 0.0f));
    }
  }
}

// The splits' sums of a tile of rows under one maximum.
template <typename T, int D, bool LIST>
__global__ __launch_bounds__(64 * WAVES) void q4_join_kernel(Q4View c, Q4AttnArgs a) {
  const int64_t s = blockIdx.y, b = s / c.H, h = s % c.H, tile = blockIdx.x;
  const int64_t slot0 = (s * gridDim.x + tile) * a.splits;
  const float* ml = a.part + (int64_t)gridDim.y * gridDim.x * a.splits * 16 * D + slot0 * 32;
  const float c2 = (float)(kLog2e / sqrt((double)D));
  constexpr int V = D / 4;
  for (int i = threadIdx.x; i < 16 * V; i += 64 * WAVES) {
    const int r = i / V, ch = i % V * 4;
    float mall = kLowest;
    for (int64_t p = 0; p < a.splits; ++p) mall = fmaxf(mall, ml[p * 32 + r]);
    floatx4_t o = {0.f, 0.f, 0.f, 0.f};
    float l = 0.0f;
    for (int64_t p = 0; p < a.splits; ++p) {
      const float w = __builtin_amdgcn_exp2f((ml[p * 32 + r] - mall) * c2);
      o += *reinterpret_cast<const floatx4_t*>(a.part + ((slot0 + p) * 16 + r) * D + ch) * w;
      l += ml[p * 32 + 16 + r] * w;
    }
    store_row4<T, LIST>(a, b, h, tile, r, ch, o * (l > 0.0f ? 1.0f / l : 0.0f));
  }
}

template <typename T, int D>
hipError_t attn_d(const Q4View& c, const Q4AttnArgs& a, hipStream_t st) {
  const int64_t tiles = q4_row_tiles(a.G, a.tok.T, a.blocks != nullptr);
  const dim3 grid((uint32_t)(tiles * a.splits), (uint32_t)(c.B * c.H));
  if (a.blocks)
    q4_attn_kernel<T, D, true><<<grid, 64 * WAVES, 0, st>>>(c, a);
  else
    q4_attn_kernel<T, D, false><<<grid, 64 * WAVES, 0, st>>>(c, a);
  return hipGetLastError();
}

template <typename T, int D>
hipError_t join_d(const Q4View& c, const Q4AttnArgs& a, hipStream_t st) {
  const dim3 grid((uint32_t)q4_row_tiles(a.G, a.tok.T, a.blocks != nullptr),
                  (uint32_t)(c.B * c.H));
  if (a.blocks)
    q4_join_kernel<T, D, true><<<grid, 64 * WAVES, 0, st>>>(c, a);
  else
    q4_join_kernel<T, D, false><<<grid, 64 * WAVES, 0, st>>>(c, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_q4_attention(int dtype, int64_t d, const Q4View& c, const Q4AttnArgs& a,
                               hipStream_t st) {
  Q4_BY_D(attn_d, c, a, st);
}

hipError_t launch_q4_join(int dtype, int64_t d, const Q4View& c, const Q4AttnArgs& a,
                          hipStream_t st) {
  Q4_BY_D(join_d, c, a, st);
}

}  // namespace thin
