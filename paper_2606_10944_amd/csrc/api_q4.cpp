// C ABI of rotary positions and the 4-bit key/value cache: argument validation and launches.
#include <math.h>
#include <stdint.h>

#include "../../include/thin.h"
#include "observe.hpp"
#include "q4.hpp"

using thin::observed;

static_assert(THIN_Q4_MAX_DRAFTS == thin::kQ4MaxDrafts, "one bound of drafts");

namespace {

constexpr int64_t kMaxSlices = 65535;  // grid y
constexpr int64_t kMaxTokens = thin::kQ4MaxTokens;
// Query rows of an attention call, of a key head and in all: tiles of 16 of them (at least
// one per token) stay below 2^24 a grid row, whose threads the runtime counts in 32 bits,
// and below 2^31 in all.
constexpr int64_t kMaxGroupRows = (int64_t)1 << 27;
constexpr int64_t kMaxRows = (int64_t)1 << 30;

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
bool aligned16(const void* p) { return aligned(p, 16); }
// device int32 arguments: the first required, the second nullable
bool valid_ints(const int32_t* p, const int32_t* q) { return p && aligned(p, 4) && aligned(q, 4); }

bool supported_d(int64_t d) { return d == 32 || d == 64 || d == 128; }

bool known_dtype(int32_t t) { return t == THIN_FP32 || t == THIN_BF16; }

// Rows [B, heads, T, d] at p: THIN_EINVAL for what the kernels cannot address.
int rows_view(const void* p, const int64_t* strides, int64_t B, int64_t heads, int64_t T, int64_t d,
              int32_t dtype, bool output, thin::RowsView* v) {
  if (!p || !aligned16(p)) return THIN_EINVAL;
  *v = {p, heads * T * d, T * d, d};
  if (!strides) return THIN_OK;
  const int64_t word = dtype == THIN_BF16 ? 8 : 4;  // elements of 16 bytes
  const int64_t len[3] = {B, heads, T};
  int64_t out[3];
  for (int i = 0; i < 3; ++i) {
    if (len[i] == 1) {
      out[i] = 0;
      continue;
    }
    if (strides[i] % word != 0 || (output && strides[i] == 0)) return THIN_EINVAL;
    out[i] = strides[i];
  }
  v->sb = out[0];
  v->sh = out[1];
  v->sr = out[2];
  return THIN_OK;
}

int cache_view(const thin_q4_cache_t* c, thin::Q4View* v) {
  if (!c || c->B < 1 || c->H < 1 || c->B > kMaxSlices || c->H > kMaxSlices ||
      c->B * c->H > kMaxSlices || !supported_d(c->d))
    return THIN_EINVAL;
  if (c->n_max < 1 || c->n_max > THIN_Q4_MAX_ROWS) return THIN_EINVAL;
  const void* all[5] = {c->k_codes, c->k_scales, c->v_codes, c->v_scales, c->bounds};
  for (const void* p : all)
    if (!p || !aligned16(p)) return THIN_EINVAL;
  *v = {static_cast<uint8_t*>(c->k_codes), static_cast<uint8_t*>(c->k_scales),
        static_cast<uint8_t*>(c->v_codes), static_cast<uint8_t*>(c->v_scales),
        static_cast<uint16_t*>(c->bounds), (int32_t)c->B, (int32_t)c->H, (int32_t)c->n_max};
  return THIN_OK;
}

bool valid_sizes(int64_t B, int64_t H, int64_t n_max, int64_t T) {
  return B >= 1 && H >= 1 && B <= kMaxSlices && H <= kMaxSlices && B * H <= kMaxSlices &&
         n_max >= 1 && n_max <= THIN_Q4_MAX_ROWS && T >= 1 && T <= kMaxTokens;
}

int64_t blocks_of(int64_t n_max) { return (n_max + THIN_Q4_BLOCK - 1) / THIN_Q4_BLOCK; }

// Query heads per key head, 0 if there is no such grouping.
int64_t group_of(int64_t q_heads, int64_t H) {
  return q_heads >= H && q_heads % H == 0 && q_heads / H <= thin::kQ4MaxGroup ? q_heads / H : 0;
}

struct AttnPlan {
  thin::Q4AttnShape shape;
  size_t bytes, sums;
};

bool plan_attention(int64_t B, int64_t H, int64_t q_heads, int64_t n_max, int64_t d, int64_t T,
                    int64_t n_sel, bool bf16, AttnPlan* p) {
  if (!valid_sizes(B, H, n_max, T) || !supported_d(d) || !group_of(q_heads, H) || n_sel < 0 ||
      n_sel > 32768)
    return false;
  if (T * (q_heads / H) > kMaxGroupRows || B * q_heads * T > kMaxRows) return false;
  const int64_t tiles = thin::q4_row_tiles(q_heads / H, T, n_sel > 0);
  p->shape = thin::q4_attention_shape(B, H, q_heads / H, T, n_sel > 0,
                                      n_sel > 0 ? n_sel * THIN_Q4_BLOCK : n_max, d, bf16);
  p->bytes = thin::q4_attention_bytes(B, H, tiles, p->shape.splits, d);
  p->sums = thin::q4_sums_bytes(B, H, tiles, p->shape.splits, d);
  return true;
}

// thin_q4_attention, or with `seen` thin_q4_tree_attention.
int attention(const thin_q4_cache_t* cache, const void* Q, const int64_t* q_strides,
              int64_t q_heads, int32_t dtype, int64_t T, const int32_t* at, const int32_t* count,
              const int32_t* blocks, int64_t n_sel, const uint64_t* seen, void* O,
              const int64_t* o_strides, void* workspace, size_t workspace_bytes, void* stream) {
  thin::Q4View c;
  int rc = cache_view(cache, &c);
  if (rc) return rc;
  if (!known_dtype(dtype)) return THIN_EDTYPE;
  AttnPlan p;
  if (!valid_ints(at, count) || !aligned(blocks, 4) || (blocks != nullptr) != (n_sel > 0) ||
      !plan_attention(c.B, c.H, q_heads, c.n_max, cache->d, T, n_sel, dtype == THIN_BF16, &p))
    return THIN_EINVAL;
  thin::Q4AttnArgs a{};
  rc = rows_view(Q, q_strides, c.B, q_heads, T, cache->d, dtype, false, &a.q);
  if (!rc) rc = rows_view(O, o_strides, c.B, q_heads, T, cache->d, dtype, true, &a.o);
  if (rc) return rc;
  if (p.bytes && (!workspace || workspace_bytes < p.bytes || !aligned16(workspace)))
    return THIN_EWORKSPACE;
  a.G = (int32_t)group_of(q_heads, c.H);
  a.tok = {at, count, (int32_t)T};
  a.blocks = blocks;
  a.n_sel = (int32_t)n_sel;
  a.seen = seen;
  a.words = (int32_t)((T + 63) / 64);
  a.shape = p.shape;
  if (p.bytes) {
    a.part = static_cast<float*>(workspace);
    // (the kernel for many rows shares keys out by length for trees alone)
    const bool several = seen && c.B > 1 && c.B <= thin::kQ4SharedEntries;
    if (!blocks && (p.shape.waves || several))
      a.table = reinterpret_cast<int2*>(static_cast<char*>(workspace) + p.sums);
  }
  hipStream_t st = static_cast<hipStream_t>(stream);
  hipError_t e = observed(THIN_KERNEL_Q4_ATTENTION, -1, st, [&] {
    return p.shape.waves == 0 ? thin::launch_q4_prompt(dtype, cache->d, c, a, st)
                              : thin::launch_q4_attention(dtype, cache->d, c, a, st);
  });
  if (e == hipSuccess && p.shape.splits > 1)
    e = observed(THIN_KERNEL_Q4_ATTENTION, -1, st,
                 [&] { return thin::launch_q4_join(dtype, cache->d, c, a, st); });
  return e == hipSuccess ? THIN_OK : THIN_EHIP;
}

// thin_rotary, or with `axis` thin_rotary_axes.
int rotary(const void* X, const int64_t* x_strides, int64_t x_heads, void* X_out,
           const int64_t* x_out_strides, const void* Y, const int64_t* y_strides, int64_t y_heads,
           void* Y_out, const int64_t* y_out_strides, int32_t dtype, int64_t B, int64_t T,
           int64_t d, int64_t rot, int32_t layout, const int32_t* pos, int32_t pos_per_token,
           int32_t axes, const int32_t* axis, const double* turns, double amp, int32_t inverse,
           void* stream) {
  if (!known_dtype(dtype)) return THIN_EDTYPE;
  if (B < 1 || T < 1 || B > ((int64_t)1 << 27) || T > ((int64_t)1 << 27) ||
      B * T > ((int64_t)1 << 27) || !supported_d(d))
    return THIN_EINVAL;
  if (rot < 16 || rot > d || rot % 16 != 0) return THIN_EINVAL;
  if (layout != THIN_ROTARY_HALF && layout != THIN_ROTARY_INTERLEAVED) return THIN_EINVAL;
  if (x_heads < 1 || x_heads > kMaxSlices || !valid_ints(pos, nullptr) ||
      !turns || !aligned(turns, 8) || !isfinite((float)amp))
    return THIN_EINVAL;
  if (Y ? (y_heads < 1 || y_heads > kMaxSlices) : (y_heads != 0 || Y_out)) return THIN_EINVAL;
  thin::RotaryArgs a{};
  int rc = rows_view(X, x_strides, B, x_heads, T, d, dtype, false, &a.x);
  if (!rc) rc = rows_view(X_out, x_out_strides, B, x_heads, T, d, dtype, true, &a.xo);
  if (!rc && Y) rc = rows_view(Y, y_strides, B, y_heads, T, d, dtype, false, &a.y);
  if (!rc && Y) rc = rows_view(Y_out, y_out_strides, B, y_heads, T, d, dtype, true, &a.yo);
  if (rc) return rc;
  a.Hx = x_heads;
  a.Hy = y_heads;
  a.B = B;
  a.T = T;
  a.pos = pos;
  a.pos_per_token = pos_per_token;
  a.axes = axes;
  a.axis = axis;
  a.turns = turns;
  a.rot = (int32_t)rot;
  a.layout = layout;
  a.inverse = inverse;
  a.amp = (float)amp;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const hipError_t e =
      observed(THIN_KERNEL_ROTARY, -1, st, [&] { return thin::launch_rotary(dtype, d, a, st); });
  return e == hipSuccess ? THIN_OK : THIN_EHIP;
}

}  // namespace

extern "C" {

int thin_rotary(const void* X, const int64_t* x_strides, int64_t x_heads, void* X_out,
                const int64_t* x_out_strides, const void* Y, const int64_t* y_strides,
                int64_t y_heads, void* Y_out, const int64_t* y_out_strides, int32_t dtype,
                int64_t B, int64_t T, int64_t d, int64_t rot, int32_t layout, const int32_t* pos,
                int32_t pos_per_token, const double* turns, double amp, int32_t inverse,
                void* stream) {
  return rotary(X, x_strides, x_heads, X_out, x_out_strides, Y, y_strides, y_heads, Y_out,
                y_out_strides, dtype, B, T, d, rot, layout, pos, pos_per_token, 0, nullptr, turns,
                amp, inverse, stream);
}

int thin_rotary_axes(const void* X, const int64_t* x_strides, int64_t x_heads, void* X_out,
                     const int64_t* x_out_strides, const void* Y, const int64_t* y_strides,
                     int64_t y_heads, void* Y_out, const int64_t* y_out_strides, int32_t dtype,
                     int64_t B, int64_t T, int64_t d, int64_t rot, int32_t layout,
                     const int32_t* pos, int32_t axes, const int32_t* axis, const double* turns,
                     double amp, int32_t inverse, void* stream) {
  if (!known_dtype(dtype)) return THIN_EDTYPE;
  if (axes < 1 || axes > THIN_ROTARY_MAX_AXES || !valid_ints(axis, nullptr)) return THIN_EINVAL;
  return rotary(X, x_strides, x_heads, X_out, x_out_strides, Y, y_strides, y_heads, Y_out,
                y_out_strides, dtype, B, T, d, rot, layout, pos, 1, axes, axis, turns, amp,
                inverse, stream);
}

int thin_rotary_turns(int64_t rot, double base, int32_t scaling, double factor, double length,
                      double slow, double fast, double* turns, double* amp) {
  if (!turns || !amp || rot < 2 || rot % 2 != 0 || !(base > 1.0) || !isfinite(base))
    return THIN_EINVAL;
  if (scaling < THIN_ROTARY_PLAIN || scaling > THIN_ROTARY_BANDS) return THIN_EINVAL;
  if (scaling != THIN_ROTARY_PLAIN && (!(factor >= 1.0) || !isfinite(factor))) return THIN_EINVAL;
  if (scaling == THIN_ROTARY_BASE && rot < 4) return THIN_EINVAL;
  if (scaling == THIN_ROTARY_BANDS &&
      (!(length > 0.0) || !isfinite(length) || !(slow < fast) || !isfinite(slow) || !isfinite(fast)))
    return THIN_EINVAL;
  if (scaling == THIN_ROTARY_BASE) base *= pow(factor, (double)rot / (double)(rot - 2));
  if (!isfinite(base)) return THIN_EINVAL;
  for (int64_t i = 0; i < rot / 2; ++i) {
    double f = pow(base, -2.0 * (double)i / (double)rot) / (2.0 * M_PI);
    if (scaling == THIN_ROTARY_LINEAR) f /= factor;
    if (scaling == THIN_ROTARY_BANDS) {
      double keep = (length * f - slow) / (fast - slow);
      keep = keep < 0.0 ? 0.0 : (keep > 1.0 ? 1.0 : keep);
      f = f * keep + f / factor * (1.0 - keep);
    }
    turns[i] = f;
  }
  *amp = scaling == THIN_ROTARY_BANDS ? 0.1 * log(factor) + 1.0 : 1.0;
  return THIN_OK;
}

int thin_q4_store(const thin_q4_cache_t* cache, const void* K, const int64_t* k_strides,
                  const void* V, const int64_t* v_strides, int32_t dtype, int64_t T,
                  const int32_t* at, const int32_t* count, void* stream) {
  thin::Q4View c;
  int rc = cache_view(cache, &c);
  if (rc) return rc;
  if (!known_dtype(dtype)) return THIN_EDTYPE;
  if (T < 1 || T > kMaxTokens || !valid_ints(at, count)) return THIN_EINVAL;
  thin::RowsView k, v;
  rc = rows_view(K, k_strides, c.B, c.H, T, cache->d, dtype, false, &k);
  if (!rc) rc = rows_view(V, v_strides, c.B, c.H, T, cache->d, dtype, false, &v);
  if (rc) return rc;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const hipError_t e = observed(THIN_KERNEL_Q4_STORE, -1, st, [&] {
    return thin::launch_q4_store(dtype, cache->d, c, k, v, {at, count, (int32_t)T}, st);
  });
  return e == hipSuccess ? THIN_OK : THIN_EHIP;
}

int thin_q4_load(const thin_q4_cache_t* cache, int64_t T, const int32_t* at, void* K, void* V,
                 int32_t dtype, void* stream) {
  thin::Q4View c;
  const int rc = cache_view(cache, &c);
  if (rc) return rc;
  if (!known_dtype(dtype)) return THIN_EDTYPE;
  if (T < 1 || T > THIN_Q4_MAX_ROWS || !valid_ints(at, nullptr) || !K || !V || !aligned16(K) ||
      !aligned16(V))
    return THIN_EINVAL;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const hipError_t e = observed(THIN_KERNEL_Q4_LOAD, -1, st, [&] {
    return thin::launch_q4_load(dtype, cache->d, c, at, T, K, V, st);
  });
  return e == hipSuccess ? THIN_OK : THIN_EHIP;
}

int thin_q4_select_plan(int64_t B, int64_t H, int64_t n_max, int64_t T, size_t* workspace_bytes) {
  if (!workspace_bytes || !valid_sizes(B, H, n_max, T)) return THIN_EINVAL;
  const int64_t nb = blocks_of(n_max);
  int64_t rows = 0;  // of scores
  if (!thin::q4_select_grouped(B * H, T))
    rows = B * H * thin::q4_select_tokens(B * H, nb, T);
  else if (!thin::q4_select_fused(B * H, nb, T))
    rows = thin::q4_select_slots(B * H, nb, T);
  *workspace_bytes = (size_t)(rows * nb) * 8;
  return THIN_OK;
}

int thin_q4_select(const thin_q4_cache_t* cache, const void* Q, const int64_t* q_strides,
                   int64_t q_heads, int32_t dtype, int64_t T, const int32_t* at,
                   const int32_t* count, int64_t n_sel, int64_t n_sinks, int64_t n_window,
                   int32_t* blocks, void* workspace, size_t workspace_bytes, void* stream) {
  thin::Q4View c;
  int rc = cache_view(cache, &c);
  if (rc) return rc;
  if (!known_dtype(dtype)) return THIN_EDTYPE;
  size_t need = 0;
  if (thin_q4_select_plan(c.B, c.H, c.n_max, T, &need) != THIN_OK ||
      !valid_ints(at, count) || !valid_ints(blocks, nullptr))
    return THIN_EINVAL;
  if (!group_of(q_heads, c.H)) return THIN_EINVAL;
  if (n_sel < 1 || n_sel > 32768 || n_sinks < 0 || n_window < 1 || n_sinks > n_sel ||
      n_window > n_sel || n_sinks + n_window > n_sel)
    return THIN_EINVAL;
  thin::Q4SelectArgs a{};
  rc = rows_view(Q, q_strides, c.B, q_heads, T, cache->d, dtype, false, &a.q);
  if (rc) return rc;
  if (need && (!workspace || workspace_bytes < need || !aligned16(workspace)))
    return THIN_EWORKSPACE;
  a.G = (int32_t)group_of(q_heads, c.H);
  a.tok = {at, count, (int32_t)T};
  a.n_sel = (int32_t)n_sel;
  a.n_sinks = (int32_t)n_sinks;
  a.n_window = (int32_t)n_window;
  a.blocks = blocks;
  a.scores = static_cast<uint64_t*>(workspace);
  hipStream_t st = static_cast<hipStream_t>(stream);
  hipError_t e = hipSuccess;
  const int64_t slices = (int64_t)c.B * c.H, nb = blocks_of(c.n_max);
  if (thin::q4_select_grouped(slices, T)) {
    e = observed(THIN_KERNEL_Q4_SELECT, -1, st,
                 [&] { return thin::launch_q4_select(dtype, cache->d, c, a, st); });
    if (e == hipSuccess && !thin::q4_select_fused(slices, nb, T))
      e = observed(THIN_KERNEL_Q4_SELECT, -1, st,
                   [&] { return thin::launch_q4_select_rest(dtype, cache->d, c, a, st); });
    return e == hipSuccess ? THIN_OK : THIN_EHIP;
  }
  const int64_t step = thin::q4_select_tokens(slices, nb, T);
  for (int64_t t0 = 0; t0 < T && e == hipSuccess; t0 += step) {
    a.t0 = (int32_t)t0;
    a.tn = (int32_t)(T - t0 < step ? T - t0 : step);
    e = observed(THIN_KERNEL_Q4_SELECT, -1, st,
                 [&] { return thin::launch_q4_scores(dtype, cache->d, c, a, st); });
    if (e == hipSuccess)
      e = observed(THIN_KERNEL_Q4_SELECT, -1, st, [&] { return thin::launch_q4_pick(c, a, st); });
  }
  return e == hipSuccess ? THIN_OK : THIN_EHIP;
}

int thin_q4_attention_plan(int64_t B, int64_t H, int64_t q_heads, int64_t n_max, int64_t d,
                           int64_t T, int64_t n_sel, size_t* workspace_bytes) {
  AttnPlan p;
  if (!workspace_bytes) return THIN_EINVAL;
  *workspace_bytes = 0;
  for (const bool bf16 : {false, true}) {  // the larger of the two types'
    if (!plan_attention(B, H, q_heads, n_max, d, T, n_sel, bf16, &p)) return THIN_EINVAL;
    if (p.bytes > *workspace_bytes) *workspace_bytes = p.bytes;
  }
  return THIN_OK;
}

int thin_q4_attention(const thin_q4_cache_t* cache, const void* Q, const int64_t* q_strides,
                      int64_t q_heads, int32_t dtype, int64_t T, const int32_t* at,
                      const int32_t* count, const int32_t* blocks, int64_t n_sel, void* O,
                      const int64_t* o_strides, void* workspace, size_t workspace_bytes,
                      void* stream) {
  return attention(cache, Q, q_strides, q_heads, dtype, T, at, count, blocks, n_sel, nullptr, O,
                   o_strides, workspace, workspace_bytes, stream);
}

int thin_q4_tree(const int32_t* parents, const int32_t* at, int64_t B, int64_t T, uint64_t* seen,
                 int32_t* pos, void* stream) {
  if (B < 1 || B > kMaxSlices || T < 1 || T > THIN_Q4_MAX_DRAFTS) return THIN_EINVAL;
  if (!valid_ints(parents, nullptr) || !valid_ints(at, nullptr) || !seen || !aligned(seen, 8) ||
      !valid_ints(pos, nullptr))
    return THIN_EINVAL;
  const void* masks = seen;
  if (masks == parents || masks == at || masks == pos || pos == parents || pos == at)
    return THIN_EINVAL;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const hipError_t e = observed(THIN_KERNEL_Q4_TREE, -1, st, [&] {
    return thin::launch_q4_tree(parents, at, B, T, seen, pos, st);
  });
  return e == hipSuccess ? THIN_OK : THIN_EHIP;
}

int thin_q4_tree_attention(const thin_q4_cache_t* cache, const void* Q, const int64_t* q_strides,
                           int64_t q_heads, int32_t dtype, int64_t T, const int32_t* at,
                           const int32_t* count, const uint64_t* seen, void* O,
                           const int64_t* o_strides, void* workspace, size_t workspace_bytes,
                           void* stream) {
  if (T > THIN_Q4_MAX_DRAFTS || !seen || !aligned(seen, 8)) return THIN_EINVAL;
  return attention(cache, Q, q_strides, q_heads, dtype, T, at, count, nullptr, 0, seen, O,
                   o_strides, workspace, workspace_bytes, stream);
}

int thin_q4_keep(const thin_q4_cache_t* cache, const int32_t* at, const int32_t* path, int64_t P,
                 int32_t* end, void* stream) {
  thin::Q4View c;
  const int rc = cache_view(cache, &c);
  if (rc) return rc;
  if (P < 1 || P > THIN_Q4_MAX_DRAFTS || !valid_ints(at, nullptr) || !valid_ints(path, nullptr) ||
      !valid_ints(end, nullptr) || end == at || end == path)
    return THIN_EINVAL;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const hipError_t e = observed(THIN_KERNEL_Q4_KEEP, -1, st, [&] {
    return thin::launch_q4_keep(cache->d, c, at, path, P, end, st);
  });
  return e == hipSuccess ? THIN_OK : THIN_EHIP;
}

}  // extern "C"
