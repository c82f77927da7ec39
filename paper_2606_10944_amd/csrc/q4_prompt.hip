// Attention over the 4-bit key/value cache on gfx950 for many query rows of a slice (a
// prompt or a chunk of one): causal over every cached row.
//
// A workgroup of four waves takes 64 RT query rows, RT tiles of 16 per wave, and walks
// the cached rows 64 at a time.  Its threads bring codes to LDS once for all of them:
// keys as stored, values decoded, one 16-byte word of each per thread, while the
// tile before is worked on.  Against the kernel for few rows, a value row is decoded
// once per 64 RT query rows instead of once per 16, and each operand read from LDS
// serves RT products.
//
// 4096 tokens over 16384 rows, 32 heads of 128 channels, 8 key heads, bf16: 800 us (842 on
// another card), 1.20 PFLOP/s, as a library bf16 product of 8192^3; float32 2.0 ms, three
// products for one.  The matrix cores alone need 410 us of the bf16 call (68 instructions of 16
// cycles per wave and tile), the vector ALU 475; without the reads of the values' columns it
// takes 49 us less, without the exponentials 59, without decoding the keys 16.
#include "q4_attn_device.hpp"

namespace thin {

namespace {

constexpr int PW = 4;    // waves
constexpr int PK = 64;   // cached rows per tile

// SPLIT: workgroups share a tile's keys and leave sums for the join.
template <typename T, int D, int RT, bool SPLIT>
__global__ __launch_bounds__(64 * PW, 2) void q4_prompt_kernel(Q4View c, Q4AttnArgs a) {
  constexpr bool MX = Elem<T>::bytes == 2;
  // bf16 parts of the weights, whose sum is that of the rounded ones.  (bf16, one: two take
  // 1145 us instead of 800 at the size above.)
  constexpr int NP = MX ? 1 : 3;
  constexpr int GR = D / 32;                      // groups per row
  constexpr int KW = D / 32;                      // words of a key row that a lane feeds
  constexpr int ROWS = 16 * RT;                   // query rows of a wave
  __shared__ __align__(16) unsigned char sv[2][PK * kVStride<D>];
  __shared__ __align__(16) uint32_t sk[2][PK * D / 8];
  __shared__ uint8_t sks[2][PK * GR];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int m = lane & 15, g = lane >> 4;

  // slice by slice; a slice's last tiles, which see the most rows, come first; the
  // workgroups that share a tile's keys side by side
  const uint32_t piece = xcd_contiguous();
  const int slice = piece / gridDim.x, b = slice / c.H, h = slice % c.H;
  const int splits = SPLIT ? a.shape.splits : 1, split = SPLIT ? piece % splits : 0;
  const int tile = (int)(gridDim.x / splits) - 1 - (int)(piece % gridDim.x / splits);
  const int nrows = a.tok.T * a.G;
  const int r0 = tile * (ROWS * PW);  // the workgroup's first query row
  const int cnt = a.tok.count ? std::min(a.tok.count[b], a.tok.T) : a.tok.T;
  // the last cached row that query rows up to r see
  auto seen = [&](int r) {
    const int t = std::min(std::min(r, nrows - 1) / a.G, cnt - 1);
    return t < 0 ? -1 : q4_last_row(a.tok, b, t, c.n_max);
  };
  const int last = __builtin_amdgcn_readfirstlane(r0 / a.G < cnt ? seen(r0 + ROWS * PW - 1) : -1);
  const int w0 = r0 + wave * ROWS;
  const int wlast =
      __builtin_amdgcn_readfirstlane(w0 < nrows && w0 / a.G < cnt ? seen(w0 + ROWS - 1) : -1);

  int qlast[RT];
  int all = 0x7fffffff;  // rows up to here are seen by every query of the wave
  Queries<T, D> q[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int r = w0 + rt * 16 + m;
    const bool there = r < nrows;
    const int t = there ? r / a.G : 0, head = there ? r % a.G : 0;
    qlast[rt] = there ? q4_last_row(a.tok, b, t, c.n_max) : -1;
    if (there) all = std::min(all, qlast[rt]);
    q[rt].load(there ? static_cast<const T*>(a.q.p) + b * a.q.sb +
                           ((int64_t)h * a.G + head) * a.q.sh + t * a.q.sr
                     : nullptr,
               g);
  }
  all = __builtin_amdgcn_readfirstlane(
      row_reduce(all, [](int x, int y) { return std::min(x, y); }));

  // this workgroup's share of the rows: k0 .. k1 - 1, whole tiles of them
  const int share = (last / PK + splits) / splits * PK;
  const int k0 = split * share, k1 = SPLIT ? std::min(last + 1, k0 + share) : last + 1;

  // this thread's word of a tile: row and group
  const int srow = threadIdx.x / GR, sgr = threadIdx.x % GR;
  const bool stages = srow < PK;
  const Slice rows = slice_of<D>(c, (int64_t)b * c.H + h);
  u32x4 kw, vw;
  uint32_t kb, vb;
  auto load_keys = [&](int row0) __attribute__((always_inline)) {
    const uint32_t r = std::min(row0 + srow, last);
    kw = *reinterpret_cast<const u32x4*>(rows.kc + (r * (D / 2) + sgr * 16));
    kb = rows.ks[r * GR + sgr];
  };
  auto load_values = [&](int row0) __attribute__((always_inline)) {
    const uint32_t r = std::min(row0 + srow, last);
    vw = *reinterpret_cast<const u32x4*>(rows.vc + (r * (D / 2) + sgr * 16));
    vb = rows.vs[r * GR + sgr];
  };
  auto put_keys = [&](int to) __attribute__((always_inline)) {
    if (!stages) return;
    *reinterpret_cast<u32x4*>(sk[to] + (srow * GR + sgr) * 4) = kw;
    sks[to][srow * GR + sgr] = (uint8_t)kb;
  };
  auto put_values = [&](int to) __attribute__((always_inline)) {
    if (!stages) return;
    const float scale = q4_scale(vb);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t w[4];
      decode8(vw[i], scale, w);
      *reinterpret_cast<u32x4*>(sv[to] + srow * kVStride<D> + sgr * 64 + i * 16) =
          (u32x4){w[0], w[1], w[2], w[3]};
    }
  };
  // raw scores of a tile whose keys lie in buffer `from`
  auto score = [&](int from, float (&sc)[RT][PK / 4]) __attribute__((always_inline)) {
#pragma unroll
    for (int kt = 0; kt < PK / 16; ++kt) {
      const int key = kt * 16 + m;
      uint32_t kc[KW];
      load_words<KW>(reinterpret_cast<const uint8_t*>(sk[from] + key * (D / 8) + g * KW), kc);
      const uint32_t byte = sks[from][key * GR + g * GR / 4];
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        const floatx4_t z = q[rt].scores(kc, byte);
#pragma unroll
        for (int j = 0; j < 4; ++j) sc[rt][kt * 4 + j] = z[j];
      }
    }
  };

  const float c2 = (float)(kQ4Log2e / sqrt((double)D));
  float mrun[RT];
  floatx4_t acc[RT][D / 16];
  // sums of weights: one more row of values, all ones (32 vector additions less per tile)
  floatx4_t lrun[RT];
  bf16x8_t ones;
#pragma unroll
  for (int j = 0; j < 8; ++j) ones[j] = (__bf16)1.0f;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    mrun[rt] = kLowest;
    lrun[rt] = (floatx4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) acc[rt][dt] = (floatx4_t){0.f, 0.f, 0.f, 0.f};
  }

  // Keys are a tile ahead of values: while a tile's weights are formed on the vector ALU,
  // the matrix cores work on the next tile's scores.
  float sc[2][RT][PK / 4];
  if (k0 < k1) {
    load_keys(k0);
    load_values(k0);
    put_keys(0);
    put_values(0);
    load_keys(k0 + PK);
    put_keys(1);
    load_keys(k0 + 2 * PK);
    load_values(k0 + PK);
    __syncthreads();
    score(0, sc[0]);
    __syncthreads();  // (the first tile overwrites these keys)
  }
  // One tile, its scores in s, the next one's to ns; i: its buffers.
  auto tile_step = [&](int row0, int i, float (&s)[RT][PK / 4],
                       float (&ns)[RT][PK / 4]) __attribute__((always_inline)) {
    if (row0 <= wlast) {
      if (row0 + PK - 1 > all) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
          for (int j = 0; j < PK / 4; ++j)
            if (row0 + j / 4 * 16 + 4 * g + j % 4 > qlast[rt]) s[rt][j] = -INFINITY;
      }
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        float mx = s[rt][0];
#pragma unroll
        for (int j = 1; j < PK / 4; ++j) mx = fmaxf(mx, s[rt][j]);
        mx *= c2;
        if (__any(mx > mrun[rt] + kSlack)) {
          mx = across_rows(mx, true, [](float x, float y) { return fmaxf(x, y); });
          const float mnew = fmaxf(mrun[rt], mx);
          const float scale = __builtin_amdgcn_exp2f(mrun[rt] - mnew);
          mrun[rt] = mnew;
          lrun[rt] *= scale;
#pragma unroll
          for (int dt = 0; dt < D / 16; ++dt) acc[rt][dt] *= scale;
        }
      }
      // The next tile's scores among this one's exponentials, and whichever wave of a SIMD has
      // products to issue goes first (852 -> 800 us by the priority).
      __builtin_amdgcn_s_setprio(1);
      __builtin_amdgcn_sched_barrier(0);
      score(i ^ 1, ns);
      bf16x8_t pp[RT][PK / 32][NP];
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
        for (int j = 0; j < PK / 4; ++j)
          s[rt][j] = __builtin_amdgcn_exp2f(fmaf(s[rt][j], c2, -mrun[rt]));
#pragma unroll
        for (int ch = 0; ch < PK / 32; ++ch) split8<NP>(s[rt] + ch * 8, pp[rt][ch]);
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int ch = 0; ch < PK / 32; ++ch) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
          for (int p = NP - 1; p >= 0; --p)
            lrun[rt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pp[rt][ch][p], lrun[rt], 0, 0, 0);
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) {
          const bf16x8_t vf = value_columns<D>(sv[i] + ch * 32 * kVStride<D>, dt, m, g);
#pragma unroll
          for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int p = NP - 1; p >= 0; --p)
              acc[rt][dt] =
                  __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pp[rt][ch][p], acc[rt][dt], 0, 0, 0);
        }
      }
      __builtin_amdgcn_s_setprio(0);
    }
    put_keys(i);         // (the tile's own keys were last read in the tile before)
    put_values(i ^ 1);   // (the tile before, which lay there, is behind the barrier)
    load_keys(row0 + 3 * PK);
    load_values(row0 + 2 * PK);
    __syncthreads();
  };
  for (int row0 = k0; row0 < k1; row0 += 2 * PK) {
    tile_step(row0, 0, sc[0], sc[1]);
    if (row0 + PK >= k1) break;
    tile_step(row0 + PK, 1, sc[1], sc[0]);
  }

#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const float l = lrun[rt][0];
    const int r = w0 + rt * 16 + m;
    if (r >= nrows) continue;
    if (SPLIT) {  // sums, maximum and sum of weights of the row, for the join
      const int tiles = (nrows + 15) / 16;
      const int64_t slots = (int64_t)gridDim.y * tiles * splits;
      const int64_t slot = ((int64_t)slice * tiles + r / 16) * splits + split;
#pragma unroll
      for (int dt = 0; dt < D / 16; ++dt)
        *reinterpret_cast<floatx4_t*>(a.part + (slot * 16 + m) * D + dt * 16 + 4 * g) = acc[rt][dt];
      float* ml = a.part + slots * 16 * D + slot * 32;
      if (g == 0) {
        ml[m] = mrun[rt];
        ml[16 + m] = l;
      }
      continue;
    }
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
    T* p = static_cast<T*>(const_cast<void*>(a.o.p)) + b * a.o.sb +
           ((int64_t)h * a.G + r % a.G) * a.o.sh + r / a.G * a.o.sr + 4 * g;
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) {
      const floatx4_t o = acc[rt][dt] * inv;
      if constexpr (MX)
        *reinterpret_cast<uint2*>(p + dt * 16) =
            make_uint2(cvt_pk_bf16(o[0], o[1]), cvt_pk_bf16(o[2], o[3]));
      else
        *reinterpret_cast<floatx4_t*>(p + dt * 16) = o;
    }
  }
}

template <typename T, int D>
hipError_t prompt_d(const Q4View& c, const Q4AttnArgs& a, hipStream_t st) {
  constexpr int RT = Elem<T>::bytes == 2 ? 2 : 1;
  static_assert(16 * RT * PW == q4_prompt_rows(Elem<T>::bytes == 2), "rows of a workgroup");
  const int64_t tiles = ((int64_t)a.tok.T * a.G + 16 * RT * PW - 1) / (16 * RT * PW);
  const dim3 grid((uint32_t)(tiles * a.shape.splits), (uint32_t)(c.B * c.H));
  if (a.shape.splits > 1)
    q4_prompt_kernel<T, D, RT, true><<<grid, 64 * PW, 0, st>>>(c, a);
  else
    q4_prompt_kernel<T, D, RT, false><<<grid, 64 * PW, 0, st>>>(c, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_q4_prompt(int dtype, int64_t d, const Q4View& c, const Q4AttnArgs& a,
                            hipStream_t st) {
  Q4_BY_D(prompt_d, c, a, st);
}

}  // namespace thin
