// Attention over the 4-bit key/value cache on gfx950: causal over every cached
// row, over the rows of the blocks listed for a token and key head, or of a tree of
// drafted tokens over the rows before the drafts and the drafts of its ancestors.
//
// The kernel for few query rows: a wave takes 32 keys at a time on its own, its
// decoded value rows in LDS, the next step's codes on their way meanwhile.
//
// d = 128, bf16, 8 key heads.  8 sequences of 3000 to 65536 rows, one token: 51 us for 298
// MB, 5.8 TB/s (a stream of reads reaches 6.5), then 5 us for the join of the shared
// tiles.  64 of 2048 blocks for 8 sequences: 12 + 4 us for 36 MB, latencies (a launch,
// positions, lists, codes, four steps per wave, the join's three loads in turn).  32
// blocks for each of 509 tokens: 123 us; the vector ALU is busy two thirds of it, the
// matrix cores a third, and of the 290 cycles that a step takes a compute unit, writing 32
// decoded value rows to LDS costs 128 (64 bytes each) and reading them transposed 53.  Trees of 9
// drafts behind up to 1000 rows, 2 sequences, 16 heads over 4, d = 64, float32: 8.3 us, one launch's
// chain of positions, codes, products, sums.
#include "q4_attn_device.hpp"

namespace thin {

namespace {

constexpr int CH = kQ4Step;

// Buffers of codes of a wave: the step in work and the next (three cost registers: 8
// sequences of up to 65536 rows 64.5 -> 66.6 us, 64 of 2048 blocks 15.6 -> 17.4).
constexpr int PF = 2;

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

// Rows row0 .. row0 + 31; rows past `last` stand for `last`.
template <int D>
__device__ __forceinline__ void load_codes(const Slice& c, int row0, int last, int lane,
                                           Codes<D>& x) {
  using C = Codes<D>;
  const int m = lane & 15, g = lane >> 4;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const uint32_t r = std::min(row0 + t * 16 + m, last);
    load_words<C::KW>(c.kc + (r * (D / 2) + g * C::KB), x.k[t]);
    x.ks[t] = c.ks[r * (D / 32) + g * C::KB * 2 / 32];
  }
#pragma unroll
  for (int i = 0; i < C::VI; ++i) {
    const int item = i * 64 + lane;
    const uint32_t r = std::min(row0 + item / C::VR, last);
    load_words<C::VL / 4>(c.vc + (r * (D / 2) + item % C::VR * C::VL), x.v[i]);
    x.vs[i] = c.vs[r * (D / 32) + item % C::VR * C::VL * 2 / 32];
  }
}

// Channels ch .. ch + 3 of query row r (there is one) of a tile.
template <typename T, bool LIST>
__device__ __forceinline__ void store_row4(const Q4AttnArgs& a, int b, int h, int tile, int r,
                                           int ch, floatx4_t o) {
  int t, head;
  if (LIST) {
    const int gt = (a.G + 15) / 16;
    t = tile / gt;
    head = tile % gt * 16 + r;
  } else {
    t = (tile * 16 + r) / a.G;
    head = (tile * 16 + r) % a.G;
  }
  T* p = static_cast<T*>(const_cast<void*>(a.o.p)) + b * a.o.sb +
         ((int64_t)h * a.G + head) * a.o.sh + t * a.o.sr + ch;
  if constexpr (Elem<T>::bytes == 2)
    *reinterpret_cast<uint2*>(p) = make_uint2(cvt_pk_bf16(o[0], o[1]), cvt_pk_bf16(o[2], o[3]));
  else
    *reinterpret_cast<floatx4_t*>(p) = o;
}

// The tokens of which tile `tile` (tokens x heads in a row) holds a head.
struct TileTokens {
  int first, last;
};
__device__ __forceinline__ TileTokens tile_tokens(const Q4AttnArgs& a, int tile) {
  const int rows = a.tok.T * a.G;
  return {tile * 16 / a.G, (tile * 16 + 16 < rows ? tile * 16 + 15 : rows - 1) / a.G};
}

// The last cached row that any of a tile's tokens of sequence b sees, -1 if none.  (Which
// drafts a drafted token sees is its mask's matter: it may be any of them.)
template <int MODE>
__device__ __forceinline__ int tile_row(const Q4View& c, const Q4AttnArgs& a, int b, TileTokens tt) {
  const int cnt = a.tok.count ? a.tok.count[b] : a.tok.T;
  if (MODE == kQ4Tree)
    return cnt <= tt.first ? -1 : q4_last_row(a.tok, b, std::min(cnt, a.tok.T) - 1, c.n_max);
  return cnt <= tt.first ? -1 : q4_last_row(a.tok, b, tt.last < cnt ? tt.last : cnt - 1, c.n_max);
}

// Steps of 32 keys up to there.
template <int MODE>
__device__ __forceinline__ int steps_of(const Q4View& c, const Q4AttnArgs& a, int b, TileTokens tt) {
  return (tile_row<MODE>(c, a, b, tt) + CH) / CH;
}

// WV waves.  Without splits a workgroup takes a tile's whole keys; with them
// workgroups share the keys and leave sums in a.part, one slot of existing rows each.
// (bf16 lists: 128 registers hold four workgroups in a compute unit, 128 -> 123 us for 32
// blocks of each of 509 tokens; over all rows they cost 64 -> 66 us for long caches.)
template <typename T, int D, int MODE, int WV>
__global__ __launch_bounds__(64 * WV, Elem<T>::bytes == 2 && MODE == kQ4List && WV == 4 ? 4 : 2)
void q4_attn_kernel(Q4View c, Q4AttnArgs a) {
  constexpr bool LIST = MODE == kQ4List;
  // bf16 parts of the weights.  (bf16, two: 17 bits, while the sum of the weights is that of
  // the unrounded ones.  One would save 1 % of one token's calls at d = 128, a tenth at 64 and
  // 32 (24 sequences of up to 10156 rows, 8 key heads, d = 64: 31.1 -> 27.9 us), and 123 -> 110
  // us for 32 blocks of each of 509 tokens.)
  constexpr int NP = Elem<T>::bytes == 2 ? 2 : 3;
  using C = Codes<D>;
  __shared__ __align__(16) unsigned char lds[WV * CH * kVStride<D>];
  __shared__ float sm[WV][16], sl[WV][16];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int m = lane & 15, g = lane >> 4;
  // the workgroup's slice, tile and share of the steps
  const int splits = a.shape.splits;
  const int64_t slot = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
  int b, h, tile, i0, i1;
  if (splits == 1) {
    const uint32_t piece = xcd_contiguous(), slice = piece / gridDim.x;
    b = slice / c.H;
    h = slice % c.H;
    tile = piece % gridDim.x;
    i0 = 0;
    i1 = LIST ? a.n_sel * (kQ4Block / CH) : steps_of<MODE>(c, a, b, tile_tokens(a, tile));
  } else if (LIST) {
    b = blockIdx.y / c.H;
    h = blockIdx.y % c.H;
    tile = blockIdx.x / splits;
    const int steps = a.n_sel * (kQ4Block / CH);
    const int share = (steps + splits - 1) / splits;
    i0 = blockIdx.x % splits * share;
    i1 = i0 + share < steps ? i0 + share : steps;
  } else {
    const int groups = c.B * splits;
    h = blockIdx.y;
    tile = blockIdx.x / groups;
    const TileTokens tt = tile_tokens(a, tile);
    const Shares sh(c, a, lane, [&](int i) { return steps_of<MODE>(c, a, i, tt); });
    // one workgroup per tile leaves the table that the join goes by
    if (h == 0 && blockIdx.x % groups == 0 && wave == 0) sh.write(c, a.table + tile * c.B, lane);
    b = sh.find(c, blockIdx.x % groups, &i0, &i1);
    if (b < 0) return;
  }
  const int64_t s = (int64_t)b * c.H + h;
  const Slice rows = slice_of<D>(c, s);
  // the tile's query rows: heads of one token (LIST), or tokens x heads in a row
  int t, head, nrows;  // this lane's
  if (LIST) {
    const int gt = (a.G + 15) / 16;
    t = tile / gt;
    head = tile % gt * 16 + m;
    nrows = std::min(16, a.G - tile % gt * 16);
  } else {
    nrows = std::min(16, a.tok.T * a.G - tile * 16);
    t = (tile * 16 + m) / a.G;
    head = (tile * 16 + m) % a.G;
  }
  const bool there = m < nrows;
  const int qlast = there ? q4_last_row(a.tok, b, t, c.n_max) : -1;
  Drafts drafts;
  if (MODE == kQ4Tree) drafts = Drafts(a, b, there ? t : a.tok.T, c.n_max);
  // the last row that any of them sees
  const int last = __builtin_amdgcn_readfirstlane(
      LIST ? q4_last_row(a.tok, b, t, c.n_max) : tile_row<MODE>(c, a, b, tile_tokens(a, tile)));

  // a wave's steps are i0 + wave + WV n.  LIST: lane n % 64 holds the listed block
  // of step n, for 64 steps at a time.
  const int nb = (c.n_max + kQ4Block - 1) / kQ4Block;
  const int32_t* list = LIST ? a.blocks + (s * a.tok.T + t) * a.n_sel : nullptr;
  int entry = -1;
  // the wave's first step with rows to read from step n on; past i1 there is none, and
  // *row0 keeps its value
  auto next = [&](int n, int* row0) {
    for (;; ++n) {
      const int i = i0 + wave + WV * n;
      if (i >= i1) break;
      if (!LIST) {
        *row0 = i * CH;
        break;
      }
      if ((n & 63) == 0) {
        const int k = i + WV * lane;
        entry = k < i1 ? list[k / (kQ4Block / CH)] : -1;
      }
      const int k = __builtin_amdgcn_readlane(entry, n & 63);
      if (k < 0 || k >= nb) continue;
      const int r = k * kQ4Block + i % (kQ4Block / CH) * CH;
      if (r > last) continue;
      *row0 = r;
      break;
    }
    return n;
  };
  auto more = [&](int n) { return i0 + wave + WV * n < i1; };
  if (last < 0) i1 = i0;
  // the codes of this step and of the next one, which are on their way.  (Past the end
  // the last row is loaded again: a load that is sometimes not made would have every
  // use wait for all loads.)
  C buf[PF];
  int row0[PF], n = -1;
  bool go[PF];
  auto fetch = [&](int k) __attribute__((always_inline)) {
    row0[k] = c.n_max;
    n = next(n + 1, &row0[k]);
    go[k] = more(n);
    load_codes<D>(rows, row0[k], std::max(last, 0), lane, buf[k]);
  };
#pragma unroll
  for (int k = 0; k + 1 < PF; ++k) fetch(k);

  Queries<T, D> q;
  q.load(there ? static_cast<const T*>(a.q.p) + b * a.q.sb + ((int64_t)h * a.G + head) * a.q.sh +
                     t * a.q.sr
               : nullptr,
         g);

  const float c2 = (float)(kQ4Log2e / sqrt((double)D));
  float mrun = kLowest, lrun = 0.0f;
  floatx4_t acc[D / 16];
#pragma unroll
  for (int dt = 0; dt < D / 16; ++dt) acc[dt] = (floatx4_t){0.f, 0.f, 0.f, 0.f};
  unsigned char* sv = lds + wave * CH * kVStride<D>;
  // rows that every query of the tile sees need no mask
  int all = there ? (MODE == kQ4Tree ? drafts.before - 1 : qlast) : 0x7fffffff;
  all = __builtin_amdgcn_readfirstlane(
      row_reduce(all, [](int x, int y) { return std::min(x, y); }));

  auto step = [&](const C& x, int row0) __attribute__((always_inline)) {
    float sc[8];
#pragma unroll
    for (int t2 = 0; t2 < 2; ++t2) {
      const floatx4_t z = q.scores(x.k[t2], x.ks[t2]);
#pragma unroll
      for (int j = 0; j < 4; ++j) sc[t2 * 4 + j] = z[j];
    }
    // values to LDS
#pragma unroll
    for (int n2 = 0; n2 < C::VI; ++n2) {
      const int item = n2 * 64 + lane;
      unsigned char* to = sv + item / C::VR * kVStride<D> + item % C::VR * C::VL * 4;
      const float vs = q4_scale(x.vs[n2]);
#pragma unroll
      for (int w8 = 0; w8 < C::VL / 4; ++w8) {
        uint32_t w[4];
        decode8(x.v[n2][w8], vs, w);
        *reinterpret_cast<u32x4*>(to + w8 * 16) = (u32x4){w[0], w[1], w[2], w[3]};
      }
    }
    if (MODE == kQ4Tree && row0 + CH - 1 > all) {
      const uint32_t see = (uint32_t)drafts.window(row0) >> (4 * g);
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (!(see >> (j / 4 * 16 + j % 4) & 1)) sc[j] = -INFINITY;
    } else if (row0 + CH - 1 > all) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (row0 + j / 4 * 16 + 4 * g + j % 4 > qlast) sc[j] = -INFINITY;
    }
    float mx = sc[0];
#pragma unroll
    for (int j = 1; j < 8; ++j) mx = fmaxf(mx, sc[j]);
    mx *= c2;
    if (__any(mx > mrun + kSlack)) {
      mx = across_rows(mx, true, [](float x, float y) { return fmaxf(x, y); });
      const float mnew = fmaxf(mrun, mx);
      const float scale = __builtin_amdgcn_exp2f(mrun - mnew);
      mrun = mnew;
      lrun *= scale;
#pragma unroll
      for (int dt = 0; dt < D / 16; ++dt) acc[dt] *= scale;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      sc[j] = __builtin_amdgcn_exp2f(fmaf(sc[j], c2, -mrun));
      lrun += sc[j];
    }
    bf16x8_t pp[NP];
    split8<NP>(sc, pp);
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) {
      const bf16x8_t vf = value_columns<D>(sv, dt, m, g);
#pragma unroll
      for (int p = NP - 1; p >= 0; --p)
        acc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pp[p], acc[dt], 0, 0, 0);
    }
  };
  for (bool done = false; !done;) {
#pragma unroll
    for (int k = 0; k < PF; ++k) {
      if (!go[k]) {
        done = true;
        break;
      }
      fetch((k + PF - 1) % PF);
      step(buf[k], row0[k]);
    }
  }
  lrun = across_rows(lrun, true, [](float x, float y) { return x + y; });

  // the waves' sums under one maximum
  if (g == 0) {
    sm[wave][m] = mrun;
    sl[wave][m] = lrun;
  }
  __syncthreads();  // (also: every wave is done with its value rows)
  float mall = sm[0][m], lall = 0.0f;
#pragma unroll
  for (int w = 1; w < WV; ++w) mall = fmaxf(mall, sm[w][m]);
#pragma unroll
  for (int w = 0; w < WV; ++w) lall += sl[w][m] * __builtin_amdgcn_exp2f(sm[w][m] - mall);
  constexpr int OS = D + 4;  // floats per row of a wave's sums
  static_assert(WV * 16 * OS * 4 <= (int)sizeof(lds), "the waves' sums fit the value rows");
  float* so = reinterpret_cast<float*>(lds);
  if (there) {
    const float scale = __builtin_amdgcn_exp2f(mrun - mall);
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) {
      const floatx4_t r = acc[dt] * scale;
      *reinterpret_cast<floatx4_t*>(so + (wave * 16 + m) * OS + dt * 16 + 4 * g) = r;
    }
  }
  __syncthreads();
  if (wave == 0 && g == 0) {
    sm[0][m] = mall;
    sl[0][m] = lall;
  }
  __syncthreads();
  constexpr int V = D / 4;  // threads per row, four channels each
  for (int k = threadIdx.x; k < nrows * V; k += 64 * WV) {
    const int r = k / V, ch = k % V * 4;
    floatx4_t o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < WV; ++w)
      o += *reinterpret_cast<const floatx4_t*>(so + (w * 16 + r) * OS + ch);
    if (splits > 1) {
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

// The splits' sums of a tile of rows under one maximum.  A workgroup takes a tile, or the
// z-th part of its channels: its threads take rows x four channels, and share the splits
// where that leaves threads.  (One row of 128 channels in 512 splits, a workgroup: 22 us, by
// one compute unit's loads; in eight parts 9.6.)
constexpr int JT = 512;  // threads
template <typename T, int D, bool LIST>
__global__ __launch_bounds__(JT) void q4_join_kernel(Q4View c, Q4AttnArgs a) {
  const int V = D / 4 / gridDim.z, c0 = (int)blockIdx.z * V;
  __shared__ float w[kQ4MaxSplits][16];  // the splits' factors
  __shared__ float inv[16];
  __shared__ floatx4_t part[JT];
  const int b = blockIdx.y / c.H, h = blockIdx.y % c.H, tile = blockIdx.x;
  const int splits = a.shape.splits;
  int nrows;
  if (LIST) {
    const int gt = (a.G + 15) / 16;
    nrows = std::min(16, a.G - tile % gt * 16);
  } else {
    nrows = std::min(16, a.tok.T * a.G - tile * 16);
  }
  // the tile's slots: `splits` of them, or those that its sequence got by its length
  int n = splits;
  int64_t slot0 = ((int64_t)blockIdx.y * gridDim.x + tile) * splits;
  if (a.table) {
    const int2 mine = a.table[tile * c.B + b];
    slot0 = ((int64_t)h * gridDim.x + tile) * c.B * splits + mine.x;
    n = mine.y;
  }
  const int64_t slots = (int64_t)gridDim.y * gridDim.x * splits;
  const float* ml = a.part + slots * 16 * D + slot0 * 32;
  // rows x four channels: `ways` threads per item, split way, way + ways, ..; the first
  // of them are on their way while the factors are formed
  const int items = nrows * V;
  const int ways = items >= JT ? 1 : JT / items;
  const int span = JT / ways;
  const int way = (int)threadIdx.x / span;
  constexpr int EARLY = 4;
  floatx4_t early[EARLY];
#pragma unroll
  for (int e = 0; e < EARLY; ++e) {
    const int k = (int)threadIdx.x % span, p = way + e * ways;
    early[e] = (floatx4_t){0.f, 0.f, 0.f, 0.f};
    if (k < items && way < ways && p < n)
      early[e] = *reinterpret_cast<const floatx4_t*>(a.part + ((slot0 + p) * 16 + k / V) * D +
                                                     (c0 + k % V) * 4);
  }
  {
    // JT / 16 threads per row
    constexpr int RT = JT / 16;
    static_assert(RT == 32, "lanes of two rows of 16");
    const int r = threadIdx.x / RT, k = threadIdx.x % RT;
    float mall = kLowest, l = 0.0f;
    if (r < nrows) {
      constexpr int MOST = kQ4MaxSplits / RT;  // (n is at most that: all loads at once)
      float mx[MOST], sums[MOST];
#pragma unroll
      for (int i = 0; i < MOST; ++i) {
        mx[i] = kLowest;
        sums[i] = 0.0f;
        if (i * RT < n && i * RT + k < n) {
          mx[i] = ml[(i * RT + k) * 32 + r];
          sums[i] = ml[(i * RT + k) * 32 + 16 + r];
        }
      }
#pragma unroll
      for (int i = 0; i < MOST; ++i) mall = fmaxf(mall, mx[i]);
      auto larger = [](float x, float y) { return fmaxf(x, y); };
      mall = across_rows(row_reduce(mall, larger), false, larger);
#pragma unroll
      for (int i = 0; i < MOST; ++i) {
        if (i * RT >= n) break;
        const float f = __builtin_amdgcn_exp2f(mx[i] - mall);
        if (i * RT + k < n) w[i * RT + k][r] = f;
        l += sums[i] * f;
      }
      auto add = [](float x, float y) { return x + y; };
      l = across_rows(row_reduce(l, add), false, add);
      if (k == 0) inv[r] = l > 0.0f ? 1.0f / l : 0.0f;
    }
  }
  __syncthreads();
  for (int k0 = 0; k0 < items; k0 += span) {
    const int k = k0 + (int)threadIdx.x % span;
    const int r = k / V, ch = (c0 + k % V) * 4;
    floatx4_t o = {0.f, 0.f, 0.f, 0.f};
    if (k < items && way < ways) {
      int p = way;
      if (k0 == 0)
#pragma unroll
        for (int e = 0; e < EARLY; ++e, p += ways)
          if (p < n) o += early[e] * w[p][r];
      const float* p0 = a.part + (slot0 * 16 + r) * D + ch;
#pragma unroll 4
      for (; p < n; p += ways)
        o += *reinterpret_cast<const floatx4_t*>(p0 + (int64_t)p * 16 * D) * w[p][r];
    }
    if (ways > 1) {
      part[threadIdx.x] = o;
      __syncthreads();
      if (way == 0 && k < items)
        for (int x = 1; x < ways; ++x) o += part[threadIdx.x + x * span];
    }
    if (way == 0 && k < items) store_row4<T, LIST>(a, b, h, tile, r, ch, o * inv[r]);
  }
}

template <typename T, int D, int MODE, int WV>
hipError_t attn(const Q4View& c, const Q4AttnArgs& a, hipStream_t st) {
  const int64_t tiles = q4_row_tiles(a.G, a.tok.T, MODE == kQ4List);
  const int64_t splits = a.shape.splits;
  const dim3 grid = MODE == kQ4List || splits == 1
                        ? dim3((uint32_t)(tiles * splits), (uint32_t)(c.B * c.H))
                        : dim3((uint32_t)(tiles * splits * c.B), (uint32_t)c.H);
  q4_attn_kernel<T, D, MODE, WV><<<grid, 64 * WV, 0, st>>>(c, a);
  return hipGetLastError();
}

template <typename T, int D>
hipError_t attn_d(const Q4View& c, const Q4AttnArgs& a, hipStream_t st) {
  if (a.shape.waves == 8)
    return a.seen     ? attn<T, D, kQ4Tree, 8>(c, a, st)
           : a.blocks ? attn<T, D, kQ4List, 8>(c, a, st)
                      : attn<T, D, kQ4All, 8>(c, a, st);
  return a.seen     ? attn<T, D, kQ4Tree, 4>(c, a, st)
         : a.blocks ? attn<T, D, kQ4List, 4>(c, a, st)
                    : attn<T, D, kQ4All, 4>(c, a, st);
}

template <typename T, int D>
hipError_t join_d(const Q4View& c, const Q4AttnArgs& a, hipStream_t st) {
  const int64_t tiles = q4_row_tiles(a.G, a.tok.T, a.blocks != nullptr);
  // parts of at least 16 channels, while compute units are left for them
  int parts = 1;
  while (parts * 2 <= D / 16 && tiles * c.B * c.H * parts * 2 <= 256) parts *= 2;
  const dim3 grid((uint32_t)tiles, (uint32_t)(c.B * c.H), (uint32_t)parts);
  if (a.blocks)
    q4_join_kernel<T, D, true><<<grid, JT, 0, st>>>(c, a);
  else
    q4_join_kernel<T, D, false><<<grid, JT, 0, st>>>(c, a);
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
