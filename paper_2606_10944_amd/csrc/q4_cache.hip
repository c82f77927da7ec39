// Store, load, moves and selection of the 4-bit key/value cache on gfx950, and trees of drafts.
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
#include "q4_attn_device.hpp"

namespace thin {

namespace {

constexpr int THREADS = 256;

// ---------------------------------------------------------------------------
// Store.  A workgroup owns one block of 64 rows of one slice: it encodes the new
// rows that fall into it and forms the block's bounds anew from them and the rows
// before them, so bounds never depend on how rows were grouped into calls, nor on
// rows that a rewound sequence no longer holds.  Four lanes hold a group, eight
// channels each.
//
// Bound by HBM: 2 x 8 x 16384 rows of keys and values, d = 128, bf16, 37 us for 134 MB
// read and 36 written, 4.6 TB/s; one row for 64 x 8 slices, 4.9 us, of which the reading
// back of the block's older rows (up to 4 KB a slice) is 2.  20240 slices of 8 tokens, d =
// 32: 66 us, vector ALU (126 with the rows' values passed on by LDS shuffles).
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
  amax = fmaxf(amax, lane_move<kSwapOnes>(amax));
  amax = fmaxf(amax, lane_move<kSwapTwos>(amax));
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

// The bounds of a block of slice s from the least and largest values of eight channels (l * 8
// on, l = threadIdx.x % (D / 8)) that each of a workgroup's four waves' threads holds.
template <int D>
__device__ __forceinline__ void write_bounds(const Q4View& c, int64_t s, int64_t block, float* mn,
                                             float* mx) {
  constexpr int LR = D / 8;
  const int l = threadIdx.x % LR;
  // over the wave's rows, then the four waves.  Halves of the wave, then its quarters,
  // trade values so that each keeps half of them: quarter g is left with channels 2 g and
  // 2 g + 1 of the eight.
#pragma unroll
  for (int n = 4; n > 1; n /= 2)
#pragma unroll
    for (int i = 0; i < n; ++i) {
      trade(n == 4, mn[i], mn[i + n]);
      trade(n == 4, mx[i], mx[i + n]);
      mn[i] = fminf(mn[i], mn[i + n]);
      mx[i] = fmaxf(mx[i], mx[i + n]);
    }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if (LR <= 8) {
      mn[i] = fminf(mn[i], lane_move<kTurn8>(mn[i]));
      mx[i] = fmaxf(mx[i], lane_move<kTurn8>(mx[i]));
    }
    if (LR <= 4) {
      mn[i] = fminf(mn[i], lane_move<kTurn4>(mn[i]));
      mx[i] = fmaxf(mx[i], lane_move<kTurn4>(mx[i]));
    }
  }
  __shared__ float sm[4][2][D];
  if ((threadIdx.x & 15) < LR) {
    const int ch = l * 8 + (threadIdx.x & 63) / 16 * 2;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      sm[threadIdx.x / 64][0][ch + i] = mn[i];
      sm[threadIdx.x / 64][1][ch + i] = mx[i];
    }
  }
  __syncthreads();
  if (threadIdx.x < 2 * D) {
    const int which = threadIdx.x / D, ch = threadIdx.x % D;
    float x = sm[0][which][ch];
#pragma unroll
    for (int w = 1; w < 4; ++w) x = which ? fmaxf(x, sm[w][1][ch]) : fminf(x, sm[w][0][ch]);
    const int64_t nb = (c.n_max + kQ4Block - 1) / kQ4Block;
    // (exact: every cached value is a bf16)
    c.bounds[((s * nb + block) * 2 + which) * D + ch] = (uint16_t)(__float_as_uint(x) >> 16);
  }
}

// The values of eight codes (channels 0 .. 7) into running bounds.
__device__ __forceinline__ void take_bounds(uint32_t code, uint32_t byte, float* mn, float* mx) {
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
  if (lo >= hi || r0 >= hi) return;  // (no new row, here or at all)
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
    take_bounds(code, byte, mn, mx);
  }
  write_bounds<D>(c, s, r0 / kQ4Block, mn, mx);
}

// ---------------------------------------------------------------------------
// Load: rows at[b] .. at[b] + T - 1 as the values they stand for, zeros outside the cache.
// Bound by HBM: 2 x 8 x 16384 rows, d = 128, as bf16: 25 us, 6.6 TB/s (mostly writes).
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
// Keep: the rows of an accepted path of drafts move to the places behind the rows before
// them, and the bounds of the blocks that hold these places are formed anew, as a store of
// these rows forms them.  A workgroup takes the keys or the values of a slice.  The rows pass
// through LDS whole before the first is written, so a path may name rows in any order, and rows
// that it also writes.
//
// 8 x 8 slices, 7 of 64 drafts kept, d = 128: 4.8 us, a chain of the path, its rows and the
// block's older rows.  64 x 8 slices, 500 of 1024: 21 us for 70 MB (3.3 TB/s; 28 with one workgroup
// for keys and values), 24 where other caches were worked on in between; a workgroup's rows all
// wait for the path, and its blocks' bounds are formed in turn, two barriers each.
// ---------------------------------------------------------------------------
template <int D, int CAP>
__global__ __launch_bounds__(THREADS) void q4_keep_kernel(Q4View c, const int32_t* at_,
                                                          const int32_t* path, int P,
                                                          int32_t* end) {
  constexpr int CW = D / 32;  // 16-byte words of a row's codes, and bytes of its scales
  __shared__ u32x4 codes[CAP * CW];
  __shared__ uint8_t scales[CAP * CW];
  __shared__ int32_t from[CAP];
  __shared__ int first_bad;
  const int64_t s = blockIdx.x;
  const int b = blockIdx.x / c.H;
  const bool keys = blockIdx.y == 0;
  const int64_t at = at_[b];
  if (threadIdx.x == 0) first_bad = P;
  __syncthreads();
  for (int i = threadIdx.x; i < P; i += THREADS) {
    const int32_t p = path[(int64_t)b * P + i];
    const int64_t row = at + p;
    from[i] = (int32_t)row;
    if (p < 0 || at < 0 || row >= c.n_max || at + i >= c.n_max) atomicMin(&first_bad, i);
  }
  __syncthreads();
  const int n = first_bad;
  if (keys && blockIdx.x % c.H == 0 && threadIdx.x == 0) end[b] = (int32_t)(at + n);
  const int64_t base = s * c.n_max;
  uint8_t* cp = keys ? c.k_codes : c.v_codes;
  uint8_t* sp = keys ? c.k_scales : c.v_scales;
#pragma unroll 4
  for (int i = threadIdx.x; i < n * CW; i += THREADS) {
    const int64_t row = base + from[i / CW];
    codes[i] = reinterpret_cast<const u32x4*>(cp + row * (D / 2))[i % CW];
    scales[i] = sp[row * CW + i % CW];
  }
  __syncthreads();
  for (int i = threadIdx.x; i < n * CW; i += THREADS) {
    // (n * CW words in a row: the new rows lie behind one another)
    reinterpret_cast<u32x4*>(cp + (base + at) * (D / 2))[i] = codes[i];
    sp[(base + at) * CW + i] = scales[i];
  }
  // bounds of the blocks from the last row before the drafts to the last row kept
  const int64_t last = at + n - 1, r0 = (at > 0 ? at - 1 : 0) / kQ4Block;
  if (!keys || last < 0 || last >= c.n_max) return;
  constexpr int LR = D / 8, RPP = THREADS / LR;
  const int l = threadIdx.x % LR, rp = threadIdx.x / LR;
  for (int64_t k = r0; k <= last / kQ4Block; ++k) {
    float mn[8], mx[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      mn[i] = INFINITY;
      mx[i] = -INFINITY;
    }
#pragma unroll
    for (int p = 0; p < kQ4Block; p += RPP) {
      const int64_t r = k * kQ4Block + p + rp;
      if (r > last) continue;
      uint32_t code, byte;
      if (r >= at) {
        const int i = (int)(r - at);
        code = reinterpret_cast<const uint32_t*>(codes)[i * (D / 8) + l];
        byte = scales[i * CW + l / 4];
      } else {
        code = *reinterpret_cast<const uint32_t*>(c.k_codes + (base + r) * (D / 2) + l * 4);
        byte = c.k_scales[(base + r) * CW + l / 4];
      }
      take_bounds(code, byte, mn, mx);
    }
    __syncthreads();  // (the block before is done with the waves' bounds)
    write_bounds<D>(c, s, k, mn, mx);
  }
}

// ---------------------------------------------------------------------------
// A tree of drafts.  seen[t] has the bits of t and its ancestors, pos[t] = at + their number
// - 1.  Parents come before their children, so a chain of ancestors runs down through the
// words of 64 drafts.  A wave closes a word over itself by jumping from ancestor to ancestor's
// ancestor, six times at most, and finds every draft's first ancestor below the word; then a
// draft takes one such step per word.  A workgroup takes 256 drafts of a sequence.
//
// 8 trees of 64: 2.9 us, a launch and two chains of loads; 64 of 1024: 7.2 us for 8.9 MB, six jumps
// through LDS and up to sixteen steps up the words.
// ---------------------------------------------------------------------------
constexpr int kTreeWords = kQ4MaxDrafts / 64;

__global__ __launch_bounds__(THREADS) void q4_tree_kernel(const int32_t* parents,
                                                          const int32_t* at, int T, uint64_t* seen,
                                                          int32_t* pos) {
  __shared__ uint64_t chain[kQ4MaxDrafts];  // the draft and its ancestors in its word
  __shared__ int32_t below[kQ4MaxDrafts];   // the first one below it, -1: none
  constexpr int RS = kTreeWords + 1;
  __shared__ uint64_t rows[THREADS * RS];
  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64;
  const int64_t b = blockIdx.y;
  const int t0 = blockIdx.x * THREADS, t1 = std::min(T, t0 + THREADS);
  const int words = (T + 63) / 64;
  for (int w = wave; w * 64 < t1; w += THREADS / 64) {
    const int t = w * 64 + lane;
    int p = t < T ? parents[b * T + t] : -1;
    if (p < 0 || p >= t) p = -1;
    uint64_t bits = (uint64_t)1 << lane;
    int jump = p >= w * 64 ? p - w * 64 : -1;  // a lane of this word
    int up = p >= w * 64 ? -1 : p;
    for (int i = 0; i < 6 && __any(jump >= 0); ++i) {
      const int from = jump < 0 ? lane : jump;
      const uint64_t more = __shfl(bits, from);
      const int next = __shfl(jump, from), theirs = __shfl(up, from);
      if (jump >= 0) {
        bits |= more;
        jump = next;
        up = theirs;
      }
    }
    chain[t] = bits;
    below[t] = up;
  }
  __syncthreads();
  const int t = t0 + threadIdx.x;
  if (t < T) {
    int a = t, n = 0;
    for (int w = words - 1; w >= 0; --w) {
      uint64_t x = 0;
      if (a >= w * 64) {
        x = chain[a];
        a = below[a];
        n += __popcll(x);
      }
      rows[threadIdx.x * RS + w] = x;
    }
    pos[b * T + t] = (int32_t)((uint32_t)at[b] + (uint32_t)n - 1u);
  }
  __syncthreads();
  uint64_t* out = seen + (b * T + t0) * words;
  for (int i = threadIdx.x; i < (t1 - t0) * words; i += THREADS)
    out[i] = rows[i / words * RS + i % words];
}

// ---------------------------------------------------------------------------
// Selection.  The score of a block for a token and key head is the sum over the
// heads g of the group and the channels c of max(q_gc lo_c, q_gc hi_c), the most
// that the block's keys could give: <q+, hi> + <q-, lo> with q+ and q- the sums
// over the group of the positive and the negative parts.  In float64, where the
// products of bf16 values and their sums are exact (or nearly, for float32
// queries), so that the order of a border does not depend on the order of sums.
//
// Scores for few tokens: eight lanes hold the sums beside a block's bounds in registers,
// and the first bounds are on their way while the queries are summed.  4 x 8 slices over
// up to 2048 blocks, d = 128: 7.0 us for 23 MB, four workgroups per compute unit (8.4 with
// eight, 8.2 with one).
// ---------------------------------------------------------------------------

// Scores as integers of the same order; NaN below everything, 0 left free for
// blocks that are not there.
__device__ __forceinline__ uint64_t score_key(double s) {
  if (s != s) return 1;
  const uint64_t u = (uint64_t)__double_as_longlong(s + 0.0);  // -0 is 0
  const uint64_t k = (u >> 63) ? ~u : u | 0x8000000000000000ull;
  return k < 2 ? 2 : k;
}

constexpr int SLANES = 8;  // lanes per block's bounds, whose sums meet by moves within eight

// The sums of a token's queries over its group, q- beside lo, then q+ beside hi, by the
// first D threads.
template <typename T, int D>
__device__ __forceinline__ void sum_queries(const Q4SelectArgs& a, int b, int h, int t, double* sq) {
  if (threadIdx.x >= D) return;
  const T* q = static_cast<const T*>(a.q.p) + b * a.q.sb + (int64_t)h * a.G * a.q.sh + t * a.q.sr;
  double neg = 0.0, pos = 0.0;
  for (int g = 0; g < a.G; ++g) {
    const double v = (double)elem<T>(q + g * a.q.sh, threadIdx.x);
    if (!(v >= 0.0)) neg += v;  // (NaN here, and so in the score)
    if (v > 0.0) pos += v;
  }
  sq[threadIdx.x] = neg;
  sq[D + threadIdx.x] = pos;
}

// A lane's share of blocks' scores: SLANES lanes to a block.
template <int D>
struct BlockScores {
  static constexpr int W = 2 * D / 8 / SLANES;  // 16-byte words of bounds per lane
  u32x4 x[W];
  double q[W][8];
  const uint16_t* bounds;  // the slice's
  int nb, j;

  __device__ __forceinline__ BlockScores(const Q4View& c, int64_t s)
      : nb((c.n_max + kQ4Block - 1) / kQ4Block), j(threadIdx.x % SLANES) {
    bounds = c.bounds + s * nb * 2 * D;
  }
  __device__ __forceinline__ void fetch(int block) {
    const u32x4* p =
        reinterpret_cast<const u32x4*>(bounds + (int64_t)(block < nb ? block : nb - 1) * 2 * D);
#pragma unroll
    for (int w = 0; w < W; ++w) x[w] = p[w * SLANES + j];
  }
  __device__ __forceinline__ void queries(const double* sq) {
#pragma unroll
    for (int w = 0; w < W; ++w)
#pragma unroll
      for (int i = 0; i < 8; ++i) q[w][i] = sq[(w * SLANES + j) * 8 + i];
  }
  // Scores of blocks k, k + step, .. up to `last` to `out`; block k's bounds are fetched.
  __device__ __forceinline__ void run(int k, int step, int last, uint64_t* out) {
    for (; k <= last; k += step) {
      double sum = 0.0;
#pragma unroll
      for (int w = 0; w < W; ++w)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          sum += q[w][2 * i] * (double)__uint_as_float(x[w][i] << 16);
          sum += q[w][2 * i + 1] * (double)__uint_as_float(x[w][i] & 0xffff0000u);
        }
      sum += lane_move<kSwapOnes>(sum);
      sum += lane_move<kSwapTwos>(sum);
      sum += lane_move<kMirror8>(sum);
      if (j == 0) out[k] = score_key(sum);
      fetch(k + step);
    }
  }
};

template <typename T, int D>
__global__ __launch_bounds__(THREADS) void q4_scores_kernel(Q4View c, Q4SelectArgs a) {
  const int64_t s = blockIdx.y;
  const int b = blockIdx.y / c.H, h = blockIdx.y % c.H;
  const int t = a.t0 + blockIdx.x % a.tn, part = blockIdx.x / a.tn;
  const int step = (int)(gridDim.x / a.tn) * (THREADS / SLANES);
  const int k = part * (THREADS / SLANES) + threadIdx.x / SLANES;
  BlockScores<D> sc(c, s);
  sc.fetch(k);  // (on its way while the queries are summed)
  const int last_row = q4_last_row(a.tok, b, t, c.n_max);
  if (last_row < 0) return;
  __shared__ double sq[2 * D];
  sum_queries<T, D>(a, b, h, t, sq);
  __syncthreads();
  sc.queries(sq);
  sc.run(k, step, last_row / kQ4Block, a.scores + (s * a.tn + t - a.t0) * sc.nb);
}

// The n_sel best of a row's blocks, in order.  A workgroup of W waves holds the
// row's keys, KPL per lane.  The border is found by counting keys in equal parts of
// the interval that it lies in, 512 W at a time (a step or two for scores that differ; for
// the key's 64 bits 8 at most with one wave, 6 with four, 5 with 16).  Equal keys at the border: the lowest blocks.
// (Halving the interval instead took 6 of 9.5 us for 32 rows of 2048 blocks.)
// keys: the scores of the n blocks that are there; out: the token's list.
template <int W, int KPL>
__device__ __forceinline__ void pick_blocks(const Q4SelectArgs& a, const uint64_t* keys, int n,
                                            int32_t* out) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64;
  __shared__ int cnt[2][W];
  __shared__ uint64_t ends[2][W];
  // a wave's keys are its KPL runs of 64 blocks
  uint64_t key[KPL];
  const int base = wave * KPL * 64;
  uint64_t lo = ~0ull, hi = 0;  // least and largest score
#pragma unroll
  for (int i = 0; i < KPL; ++i) {
    const int k = base + i * 64 + lane;
    key[i] = 0;
    if (k >= n) continue;
    if (k < a.n_sinks || k >= n - a.n_window) {
      key[i] = ~0ull;
    } else {
      key[i] = keys[k];
      lo = key[i] < lo ? key[i] : lo;
      hi = key[i] > hi ? key[i] : hi;
    }
  }
  lo = wave_min(lo);
  hi = wave_max(hi);
  if (W > 1) {
    if (lane == 0) {
      ends[0][wave] = lo;
      ends[1][wave] = hi;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < W; ++w) {
      lo = ends[0][w] < lo ? ends[0][w] : lo;
      hi = ends[1][w] > hi ? ends[1][w] : hi;
    }
  }
  const int want = n < a.n_sel ? n : a.n_sel;
  // keys of at least x stay, and `ties` of those equal to x - 1
  uint64_t x = 1;
  int ties = 0;
  if (n > a.n_sel) {
    constexpr int TH = 64 * W, PER = 8, BITS = W == 1 ? 9 : W == 4 ? 11 : 13;
    static_assert(1 << BITS == TH * PER, "parts of the interval");
    // part p lies where the thread that sums it reads without bank conflicts
    __shared__ int part[TH * PER];
    auto place_of = [](int p) { return p % PER * TH + p / PER; };
    __shared__ int sums[W], found[3];
    const int forced = (a.n_sinks < n ? a.n_sinks : n) + (a.n_window < n ? a.n_window : n);
    int need = want - forced;  // (n > n_sel >= sinks + window: they do not overlap)
    x = need > 0 ? 0 : hi + 1;
    while (x == 0) {
      const uint64_t range = hi - lo;
      const int len = 64 - __clzll((long long)range), shift = len > BITS ? len - BITS : 0;
      for (int p = 0; p < PER; ++p) part[p * TH + threadIdx.x] = 0;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < KPL; ++i)
        if (key[i] >= lo && key[i] <= hi && key[i] != 0)
          atomicAdd(&part[place_of((int)((key[i] - lo) >> shift))], 1);
      __syncthreads();
      // thread t: the t-th eight parts from the top, and how many keys lie above them
      const int top = TH * PER - 1 - (int)threadIdx.x * PER;
      int c8[PER], mine = 0;
#pragma unroll
      for (int p = 0; p < PER; ++p) {
        c8[p] = part[place_of(top - p)];
        mine += c8[p];
      }
      int upto = (int)wave_scan<uint32_t>((uint32_t)mine, 0u,
                                          [](uint32_t a, uint32_t b) { return a + b; });
      if (lane == 63) sums[wave] = upto;
      __syncthreads();
      for (int w = 0; w < wave; ++w) upto += sums[w];
      if (upto - mine < need && upto >= need) {
        int over = upto - mine;
        bool past = false;
#pragma unroll
        for (int p = 0; p < PER; ++p) {
          if (!past && over + c8[p] >= need) {
            past = true;
            found[0] = top - p;
            found[1] = over;
            found[2] = c8[p];
          }
          over += c8[p];
        }
      }
      __syncthreads();
      need -= found[1];
      lo += (uint64_t)found[0] << shift;
      if (found[2] == need) {
        x = lo;
      } else if (shift == 0) {
        x = lo + 1;
        ties = need;
      } else {
        const uint64_t end = lo + ((1ull << shift) - 1);
        hi = end < hi ? end : hi;
      }
    }
  }
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
  for (int i = want + (int)threadIdx.x; i < a.n_sel; i += 64 * W) out[i] = -1;
}

template <int W, int KPL>
__global__ __launch_bounds__(64 * W) void q4_pick_kernel(Q4View c, Q4SelectArgs a) {
  const int64_t s = blockIdx.y;
  const int b = blockIdx.y / c.H, t = a.t0 + blockIdx.x;
  const int nb = (c.n_max + kQ4Block - 1) / kQ4Block;
  const int lr = q4_last_row(a.tok, b, t, c.n_max);
  pick_blocks<W, KPL>(a, a.scores + (s * a.tn + blockIdx.x) * nb, lr < 0 ? 0 : lr / kQ4Block + 1,
                      a.blocks + (s * a.tok.T + t) * a.n_sel);
}

// The tokens that launch_q4_select leaves: those of whose 16 one sees more blocks than LDS
// holds.  A sequence's are the last ones of it, padding among their 16 included.
struct TokenRange {
  int first, end;
};
__device__ __forceinline__ TokenRange q4_left_tokens(const Q4View& c, const Q4Tokens& tok, int b) {
  constexpr int64_t kRows = kQ4SelectBlocks * kQ4Block;
  const int cnt = tok.count ? std::min(tok.count[b], tok.T) : tok.T;
  if (cnt <= 0 || q4_last_row(tok, b, cnt - 1, c.n_max) < kRows) return {0, 0};
  // the first 16 whose last token there, 16 g + 15 or cnt - 1, stands at kRows or behind
  const int64_t upto = kRows - tok.at[b] + 1;  // tokens up to it (<= cnt)
  return {upto <= 16 ? 0 : (int)((upto - 1) / 16 * 16), std::min((cnt + 15) / 16 * 16, tok.T)};
}

// Those tokens' selection in one launch, in float64: a workgroup takes a token and key head,
// its scores to a slot of the workspace and the choice from there, then its next ones.  What
// is left is counted here, so that a launch costs as little as there is left of it (8 key
// heads, 4096 tokens at row 8192 of a cache of 262144: 293 us with the launch before it, 399
// where scores and choices had launches over all tokens).  4096 tokens over 200000 rows: 4.15
// ms, 512 over 1000000 2.3; d = 128.
template <typename T, int D, int KPL>
__global__ __launch_bounds__(1024) void q4_select_rest_kernel(Q4View c, Q4SelectArgs a) {
  constexpr int W = 16;
  __shared__ double sq[2 * D];
  const int lane = threadIdx.x & 63;
  const int nb = (c.n_max + kQ4Block - 1) / kQ4Block;
  uint64_t* slot = a.scores + (int64_t)blockIdx.x * nb;
  int64_t item = blockIdx.x;  // of the tokens x heads left, sequence by sequence, head by head
  int64_t before = 0;         // items of the sequences before this lane's
  for (int b0 = 0; b0 < c.B; b0 += 64) {  // 64 sequences at a time, one per lane
    TokenRange mine = {0, 0};
    if (b0 + lane < c.B) mine = q4_left_tokens(c, a.tok, b0 + lane);
    const uint64_t upto = before + wave_scan<uint64_t>((uint64_t)(mine.end - mine.first) * c.H, 0ull,
                                                       [](uint64_t x, uint64_t y) { return x + y; });
    for (;; item += gridDim.x) {
      const uint64_t past = __ballot(upto > (uint64_t)item);
      if (!past) break;  // (the same in every wave)
      const int l = __ffsll((unsigned long long)past) - 1;
      const int first = __builtin_amdgcn_readlane(mine.first, l);
      const int tokens = __builtin_amdgcn_readlane(mine.end, l) - first;
      const int64_t end = (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(upto >> 32), l) << 32 |
                                    (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)upto, l));
      const int64_t i = item - (end - (int64_t)tokens * c.H);  // of this sequence's
      const int b = b0 + l, h = (int)(i / tokens), t = first + (int)(i % tokens);
      const int64_t s = (int64_t)b * c.H + h;
      const int lr = q4_last_row(a.tok, b, t, c.n_max);
      if (lr >= 0) {
        BlockScores<D> sc(c, s);
        sc.fetch(threadIdx.x / SLANES);
        sum_queries<T, D>(a, b, h, t, sq);
        __syncthreads();
        sc.queries(sq);
        sc.run(threadIdx.x / SLANES, 64 * W / SLANES, lr / kQ4Block, slot);
      }
      __syncthreads();  // scores, and behind the last choice
      pick_blocks<W, KPL>(a, slot, lr < 0 ? 0 : lr / kQ4Block + 1,
                          a.blocks + (s * a.tok.T + t) * a.n_sel);
      __syncthreads();  // the slot is read
    }
    before = (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(upto >> 32), 63) << 32 |
                       (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)upto, 63));
  }
}

// Selection for several tokens of a slice in one launch.  A workgroup takes 16 tokens:
// their scores of every block come from the bf16 matrix instructions, the queries'
// float64 sums split into two bf16 parts (bounds are bf16), and stay in LDS.  Such a
// score is off by less than eps = (4 d 2^-23 + 2^-16) (1 + 2^-6) size, size = the token's
// largest sum of the products' magnitudes as the instructions add it up: 4 d additions,
// rounded or cut to float32, lose at most 2^-23 of it each, the split 2^-16 of each query
// sum (two roundings by half a step, 2^-8), and size itself may be short by 2^-7 (first
// parts only, and its additions).  So a block more than 2 eps
// above the last one that fits is in, one more than 2 eps below it is out, whatever the
// rounding; the others between (mostly that one alone) are scored again in float64.
//
// 2047 tokens x 8 key heads over up to 512 blocks, d = 128 (8e6 scores of 256 products:
// 62 us in float64 at the rate of a large float64 matrix product): 64 us, of which the
// scores take about half, second scores a fifth, and the choice the rest.  In float64
// throughout: 343.

// A float's key: integers of the same order, NaN below everything, 0 left free.
__device__ __forceinline__ uint32_t float_key(float f) {
  if (f != f) return 1;
  const uint32_t u = __float_as_uint(f + 0.0f);
  const uint32_t k = (u >> 31) ? ~u : u | 0x80000000u;
  return k < 2 ? 2 : k;
}
__device__ __forceinline__ float key_float(uint32_t k) {
  return __uint_as_float((k >> 31) ? k & 0x7fffffffu : ~k);
}

// N elements from an aligned place, N * sizeof(T) a power of two up to 16.
template <typename T, int N>
__device__ __forceinline__ void load_few(const T* p, float* f) {
  constexpr int BYTES = N * Elem<T>::bytes;
  typedef uint32_t words __attribute__((ext_vector_type(BYTES >= 4 ? BYTES / 4 : 1)));
  if constexpr (BYTES < 4) {
#pragma unroll
    for (int j = 0; j < N; ++j) f[j] = elem<T>(p, j);
  } else {
    words w = *reinterpret_cast<const words*>(p);
    uint32_t u[BYTES / 4];
    __builtin_memcpy(u, &w, BYTES);
#pragma unroll
    for (int j = 0; j < N; ++j)
      f[j] = Elem<T>::bytes == 4 ? __uint_as_float(u[j])
                                 : __uint_as_float(j % 2 ? u[j / 2] & 0xffff0000u : u[j / 2] << 16);
  }
}

// Of the keys of a wave (key i of lane l stands at place 64 i + l) the largest `want`,
// ties to the lowest places: bit i of the result says whether this lane's key i is one.
// Keys of 0 are none; there are at least `want` others.
template <typename K, int KPL>
__device__ __forceinline__ uint32_t largest(const K* key, int want, int lane) {
  K lo = ~(K)0, hi = 0;
#pragma unroll
  for (int i = 0; i < KPL; ++i) {
    if (key[i] != 0 && key[i] < lo) lo = key[i];
    if (key[i] > hi) hi = key[i];
  }
  lo = wave_min(lo);
  hi = wave_max(hi);
  auto count = [&](K x) {
    int n = 0;
#pragma unroll
    for (int i = 0; i < KPL; ++i) n += __popcll(__ballot(key[i] >= x));
    return n;
  };
  // least x in (lo, hi + 1] with count(x) <= want; hi + 1 overflows at most to 0: a key of
  // all ones does not occur
  int above = 0;
  hi += 1;
  if (count(lo) <= want) {
    hi = lo;
    above = want;
  }
  while (hi - lo > 1) {
    const K mid = lo + (hi - lo) / 2;
    const int n = count(mid);
    if (n > want) {
      lo = mid;
    } else {
      hi = mid;
      above = n;
      if (n == want) break;
    }
  }
  int ties = want - above;  // keys equal to lo that are in
  uint32_t in = 0;
#pragma unroll
  for (int i = 0; i < KPL; ++i) {
    const bool tie = key[i] == lo && lo < hi;
    const uint64_t t = __ballot(tie);
    const int before = __popcll(t & ((1ull << lane) - 1));
    if (key[i] != 0 && (key[i] >= hi || (tie && before < ties))) in |= 1u << i;
    const int taken = __popcll(t);
    ties -= taken < ties ? taken : ties;
  }
  return in;
}

// SW waves.
template <typename T, int D, int KPL, int SW>
__global__ __launch_bounds__(64 * SW, SW == 8 ? 6 : KPL > 8 ? 4 : 8) void q4_select_kernel(
    Q4View c, Q4SelectArgs a, int stride) {
  constexpr int KS = 2 * D / 32;  // k-steps: q- beside lo, then q+ beside hi
  extern __shared__ __align__(16) float score[];  // [16, stride], then the queries' parts
  __shared__ uint32_t ssize[SW][16];
  const int64_t s = blockIdx.y;
  const int b = blockIdx.y / c.H, h = blockIdx.y % c.H, t0 = blockIdx.x * 16;
  const int nb = (c.n_max + kQ4Block - 1) / kQ4Block;
  const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const T* qh = static_cast<const T*>(a.q.p) + b * a.q.sb + (int64_t)h * a.G * a.q.sh;
  const uint16_t* bounds = c.bounds + s * nb * 2 * D;

  // the first bounds of this wave are on their way while the queries are summed
  u32x4 w[KS];
  auto fetch = [&](int k0, u32x4* to) __attribute__((always_inline)) {
    const u32x4* row =
        reinterpret_cast<const u32x4*>(bounds + (int64_t)std::min(k0 + m, nb - 1) * 2 * D);
#pragma unroll
    for (int i = 0; i < KS; ++i) to[i] = row[4 * i + g];
  };

  // the last block that any of the tokens sees
  const bool there = t0 + m < a.tok.T;
  const int most = (int)wave_max((uint32_t)(
      (there ? q4_last_row(a.tok, b, t0 + m, c.n_max) : -1) + 1));
  const int blocks = (most + kQ4Block - 1) / kQ4Block;
  if (blocks > kQ4SelectBlocks) return;  // (left to q4_select_rest_kernel)

  // The tokens' sums in parts: [k-step, part, lane] 16-byte words, lane (m, g) token m's
  // channels of words 4 i + g.  The waves share the words.
  u32x4* parts = reinterpret_cast<u32x4*>(score + 16 * stride);
  // sums whose second part may lie below the normal numbers: not 0, less than 2^-100
  bool small = false, some = false;  // some: a sum that is not 0
  auto below = [](float x) {
    return (__float_as_uint(x) << 1) - 1 < (__float_as_uint(0x1p-100f) << 1) - 1;
  };
  for (int i = wave; i < KS / 2; i += SW) {
    double neg[8], pos[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) neg[j] = pos[j] = 0.0;
    if (there) {
      const T* p = qh + (int64_t)(t0 + m) * a.q.sr + (4 * i + g) * 8;
#pragma unroll 2
      for (int x = 0; x < a.G; ++x) {
        float f[8];
        load8<T>(p + x * a.q.sh, f);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (!(f[j] >= 0.0f)) neg[j] += (double)f[j];
          if (f[j] > 0.0f) pos[j] += (double)f[j];
        }
      }
    }
    // (float32 keeps 2^-24 of a sum, the first bf16 part 2^-8, the second 2^-16 of it)
    float n[8], p[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      n[j] = (float)neg[j];
      p[j] = (float)pos[j];
      small |= below(n[j]) || below(p[j]);
      some |= n[j] != 0.0f || p[j] != 0.0f;
    }
    bf16x8_t np[2], pp[2];
    split8<2>(n, np);
    split8<2>(p, pp);
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      parts[(i * 2 + x) * 64 + lane] = __builtin_bit_cast(u32x4, np[x]);
      parts[((i + KS / 2) * 2 + x) * 64 + lane] = __builtin_bit_cast(u32x4, pp[x]);
    }
  }
  fetch(wave * 16, w);
  __syncthreads();

  // largest sum of magnitudes of this lane's scores (token m), as bits: NaN above all, and
  // infinite for sums that the parts do not hold (all its blocks are scored again).  0 only
  // where every query is: products of others may lie below the normal numbers.
  uint32_t size = small ? 0x7f800000u : some ? 0x00800000u : 0;
  auto tile = [&](int k0, const u32x4* x) __attribute__((always_inline)) {
    floatx4_t z = {0.f, 0.f, 0.f, 0.f}, y = {0.f, 0.f, 0.f, 0.f};
    const u32x4 sign = {0x80008000u, 0x80008000u, 0x80008000u, 0x80008000u};
#pragma unroll
    for (int i = 0; i < KS; ++i) {
      const u32x4 q0 = parts[i * 2 * 64 + lane], q1 = parts[(i * 2 + 1) * 64 + lane];
      const bf16x8_t v = __builtin_bit_cast(bf16x8_t, x[i]);
      z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, __builtin_bit_cast(bf16x8_t, q1), z, 0, 0, 0);
      z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, __builtin_bit_cast(bf16x8_t, q0), z, 0, 0, 0);
      y = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, x[i] & ~sign),
                                                  __builtin_bit_cast(bf16x8_t, q0 & ~sign), y, 0, 0,
                                                  0);
    }
    *reinterpret_cast<floatx4_t*>(score + m * stride + k0 + 4 * g) = z;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (k0 + 4 * g + j < blocks) size = std::max(size, __float_as_uint(y[j]) & 0x7fffffffu);
  };
  for (int k0 = wave * 16; k0 < blocks; k0 += SW * 16) {
    tile(k0, w);
    fetch(k0 + SW * 16, w);
  }
  size = __float_as_uint(across_rows(__uint_as_float(size), true, [](float x, float y) {
    return __uint_as_float(std::max(__float_as_uint(x), __float_as_uint(y)));
  }));
  if (lane < 16) ssize[wave][lane] = size;
  __syncthreads();

  for (int r = wave; r < 16; r += SW) {
    const int t = t0 + r;
    if (t >= a.tok.T) break;
    int32_t* out = a.blocks + (s * a.tok.T + t) * a.n_sel;
    const int lr = q4_last_row(a.tok, b, t, c.n_max);
    const int n = lr < 0 ? 0 : lr / kQ4Block + 1;  // blocks that are there
    const int want = n < a.n_sel ? n : a.n_sel;
    uint32_t in = 0;  // bit i: block 64 i + lane is taken
    if (n <= a.n_sel) {
#pragma unroll
      for (int i = 0; i < KPL; ++i)
        if (i * 64 + lane < n) in |= 1u << i;
    } else {
      uint32_t key[KPL];
      int forced = 0;  // sinks and window
#pragma unroll
      for (int i = 0; i < KPL; ++i) {
        const int k = i * 64 + lane;
        const bool f = k < n && (k < a.n_sinks || k >= n - a.n_window);
        if (f) in |= 1u << i;
        forced += __popcll(__ballot(f));
        key[i] = k < n && !f ? float_key(score[r * stride + k]) : 0;
      }
      const int free = want - forced;
      if (free > 0) {
        uint32_t best = largest<uint32_t, KPL>(key, free, lane);
        uint32_t least = ~0u;  // of the chosen keys
#pragma unroll
        for (int i = 0; i < KPL; ++i)
          if ((best >> i & 1) && key[i] < least) least = key[i];
        least = wave_min(least);
        // 2 eps (at least what products below the normal numbers can make); not a number or
        // infinite: every block is scored again
        uint32_t bits = 0;
#pragma unroll
        for (int x = 0; x < SW; ++x) bits = std::max(bits, ssize[x][r]);
        const float size = __uint_as_float(bits);
        constexpr float kEps2 = 2.0f * (4.0f * D * 0x1p-23f + 0x1p-16f) * (1.0f + 0x1p-6f);
        const float eps2 = fmaxf(kEps2 * size, 0x1p-110f);
        const float mid = key_float(least), up = mid + eps2, down = mid - eps2;
        const bool wild = !(size < INFINITY) || !(fabsf(mid) < INFINITY);
        int sure = 0, open = 0;
        uint32_t maybe = 0;
#pragma unroll
        for (int i = 0; i < KPL; ++i) {
          const float f = key_float(key[i]);
          const bool x = key[i] != 0 && (wild || (f <= up && f >= down));
          if (x) maybe |= 1u << i;
          open += __popcll(__ballot(x));
          sure += __popcll(__ballot((best >> i & 1) && !x));
        }
        // (all queries 0: the lowest blocks are chosen already)
        if (open > free - sure && !(size == 0.0f)) {
          // products of 2 D / 64 neighbouring channels per lane, q- beside lo, q+ beside hi
          constexpr int N = 2 * D / 64;
          const bool low = lane < 32;
          double qd[N];
#pragma unroll
          for (int j = 0; j < N; ++j) qd[j] = 0.0;
          const T* row = qh + (int64_t)t * a.q.sr + lane % 32 * N;
#pragma unroll 4
          for (int x = 0; x < a.G; ++x) {
            float f[N];
            load_few<T, N>(row + x * a.q.sh, f);
#pragma unroll
            for (int j = 0; j < N; ++j)
              if (low ? !(f[j] >= 0.0f) : f[j] > 0.0f) qd[j] += (double)f[j];
          }
          uint64_t wide[KPL];
#pragma unroll
          for (int i = 0; i < KPL; ++i) {
            wide[i] = 0;
            for (uint64_t todo = __ballot(maybe >> i & 1); todo; todo &= todo - 1) {
              const int l = __ffsll((unsigned long long)todo) - 1;
              float f[N];
              load_few<bf16_t, N>(reinterpret_cast<const bf16_t*>(bounds) +
                                      (int64_t)(i * 64 + l) * 2 * D + lane * N, f);
              double sum = 0.0;
#pragma unroll
              for (int j = 0; j < N; ++j) sum += qd[j] * (double)f[j];
              sum = wave_sum(sum);
              if (lane == l) wide[i] = score_key(sum);
            }
          }
          best = (best & ~maybe) | largest<uint64_t, KPL>(wide, free - sure, lane);
        }
        in |= best;
      }
    }
    int place = 0;
#pragma unroll
    for (int i = 0; i < KPL; ++i) {
      const uint64_t mask = __ballot(in >> i & 1);
      if (in >> i & 1) out[place + __popcll(mask & ((1ull << lane) - 1))] = i * 64 + lane;
      place += __popcll(mask);
    }
    for (int i = want + lane; i < a.n_sel; i += 64) out[i] = -1;
  }
}

template <typename T, int D>
hipError_t store_d(const Q4View& c, const RowsView& k, const RowsView& v, const Q4Tokens& tok,
                   hipStream_t st) {
  const dim3 grid((uint32_t)((tok.T + kQ4Block - 2) / kQ4Block + 1), (uint32_t)(c.B * c.H));
  q4_store_kernel<T, D><<<grid, THREADS, 0, st>>>(c, k, v, tok);
  return hipGetLastError();
}

template <int D>
hipError_t keep_d(const Q4View& c, const int32_t* at, const int32_t* path, int64_t P, int32_t* end,
                  hipStream_t st) {
  const dim3 grid((uint32_t)(c.B * c.H), 2);
  if (P <= 64)
    q4_keep_kernel<D, 64><<<grid, THREADS, 0, st>>>(c, at, path, (int)P, end);
  else if (P <= 512)
    q4_keep_kernel<D, 512><<<grid, THREADS, 0, st>>>(c, at, path, (int)P, end);
  else
    q4_keep_kernel<D, kQ4MaxDrafts><<<grid, THREADS, 0, st>>>(c, at, path, (int)P, end);
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
  const int64_t most = (1024 + rows - 1) / rows;  // four workgroups per compute unit
  if (x > most) x = most;
  const dim3 grid((uint32_t)(x * a.tn), (uint32_t)(c.B * c.H));
  q4_scores_kernel<T, D><<<grid, THREADS, 0, st>>>(c, a);
  return hipGetLastError();
}

template <typename T, int D>
hipError_t rest_d(const Q4View& c, const Q4SelectArgs& a, hipStream_t st) {
  const int64_t nb = (c.n_max + kQ4Block - 1) / kQ4Block;
  const dim3 grid((uint32_t)q4_select_slots((int64_t)c.B * c.H, nb, a.tok.T));
  if (nb <= 16 * 64 * 8)
    q4_select_rest_kernel<T, D, 8><<<grid, 1024, 0, st>>>(c, a);
  else if (nb <= 16 * 64 * 16)
    q4_select_rest_kernel<T, D, 16><<<grid, 1024, 0, st>>>(c, a);
  else
    q4_select_rest_kernel<T, D, 32><<<grid, 1024, 0, st>>>(c, a);
  return hipGetLastError();
}

template <int W, int KPL>
hipError_t pick(const Q4View& c, const Q4SelectArgs& a, hipStream_t st) {
  const dim3 grid((uint32_t)a.tn, (uint32_t)(c.B * c.H));
  q4_pick_kernel<W, KPL><<<grid, 64 * W, 0, st>>>(c, a);
  return hipGetLastError();
}

template <typename T, int D, int KPL, int SW>
hipError_t select_k(const Q4View& c, const Q4SelectArgs& a, hipStream_t st) {
  const int nb = std::min<int>((c.n_max + kQ4Block - 1) / kQ4Block, kQ4SelectBlocks);
  const int stride = (nb + 15) / 16 * 16 + 4;
  const dim3 grid((uint32_t)((a.tok.T + 15) / 16), (uint32_t)(c.B * c.H));
  constexpr size_t kParts = 2 * D / 32 * 2 * 64 * 16;
  const size_t lds = (size_t)16 * stride * 4 + kParts;
  // Dynamic LDS past 64 KiB is allowed by an attribute of the kernel, which all host threads
  // share: every call sets it to the most that this instance takes, never to its own need.
  constexpr size_t most = (size_t)16 * (64 * KPL + 4) * 4 + kParts;
  if constexpr (most > 64 * 1024) {
    const hipError_t e =
        hipFuncSetAttribute(reinterpret_cast<const void*>(&q4_select_kernel<T, D, KPL, SW>),
                            hipFuncAttributeMaxDynamicSharedMemorySize, (int)most);
    if (e != hipSuccess) return e;
  }
  q4_select_kernel<T, D, KPL, SW><<<grid, 64 * SW, lds, st>>>(c, a, stride);
  return hipGetLastError();
}

// Up to 1024 workgroups (two per compute unit at a time) 16 waves share a workgroup's blocks
// and tokens, beyond that eight, three workgroups to a compute unit (8 key heads over up to
// 512 blocks: 1024 workgroups 62.6 us against 71.1, 256 11.0 and 13.9; all 16384 tokens of
// a cache, 8192 workgroups 291 and 252).  Scores of more blocks leave one workgroup to a
// compute unit: 16 waves (1024 tokens over 1024 blocks: 72.5 against 88.7 with eight).
template <typename T, int D>
hipError_t select_d(const Q4View& c, const Q4SelectArgs& a, hipStream_t st) {
  const int nb = (c.n_max + kQ4Block - 1) / kQ4Block;
  if (nb > 1024) return select_k<T, D, 32, 16>(c, a, st);
  if (nb > 512) return select_k<T, D, 16, 16>(c, a, st);
  if ((int64_t)c.B * c.H * ((a.tok.T + 15) / 16) > 1024)
    return nb <= 128 ? select_k<T, D, 2, 8>(c, a, st) : select_k<T, D, 8, 8>(c, a, st);
  return nb <= 128 ? select_k<T, D, 2, 16>(c, a, st) : select_k<T, D, 8, 16>(c, a, st);
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

hipError_t launch_q4_keep(int64_t d, const Q4View& c, const int32_t* at, const int32_t* path,
                          int64_t P, int32_t* end, hipStream_t st) {
  return d == 32   ? keep_d<32>(c, at, path, P, end, st)
         : d == 64 ? keep_d<64>(c, at, path, P, end, st)
                   : keep_d<128>(c, at, path, P, end, st);
}

hipError_t launch_q4_tree(const int32_t* parents, const int32_t* at, int64_t B, int64_t T,
                          uint64_t* seen, int32_t* pos, hipStream_t st) {
  const dim3 grid((uint32_t)((T + THREADS - 1) / THREADS), (uint32_t)B);
  q4_tree_kernel<<<grid, THREADS, 0, st>>>(parents, at, (int)T, seen, pos);
  return hipGetLastError();
}

hipError_t launch_q4_scores(int dtype, int64_t d, const Q4View& c, const Q4SelectArgs& a,
                            hipStream_t st) {
  Q4_BY_D(scores_d, c, a, st);
}

hipError_t launch_q4_select(int dtype, int64_t d, const Q4View& c, const Q4SelectArgs& a,
                            hipStream_t st) {
  Q4_BY_D(select_d, c, a, st);
}

hipError_t launch_q4_select_rest(int dtype, int64_t d, const Q4View& c, const Q4SelectArgs& a,
                                 hipStream_t st) {
  Q4_BY_D(rest_d, c, a, st);
}

hipError_t launch_q4_pick(const Q4View& c, const Q4SelectArgs& a, hipStream_t st) {
  const int64_t runs = (c.n_max + kQ4Block * 64 - 1) / (kQ4Block * 64);  // runs of 64 blocks
  if (runs <= 2) return pick<1, 2>(c, a, st);
  if (runs <= 8) return pick<1, 8>(c, a, st);
  if (runs <= 32) return pick<4, 8>(c, a, st);
  if (runs <= 128) return pick<16, 8>(c, a, st);
  if (runs <= 256) return pick<16, 16>(c, a, st);
  return pick<16, 32>(c, a, st);
}

}  // namespace thin
