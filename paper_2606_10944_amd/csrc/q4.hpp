// The 4-bit key/value cache (MX format: groups of 32 channels, e2m1 codes, one
// power-of-two scale byte) and the launchers of the operators over it.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "q4_plan.hpp"

namespace thin {

constexpr int kQ4Block = 64;  // rows per block of the selection

// Device pointers of a cache; slice s = b * H + h owns rows [s * n_max, (s + 1) * n_max).
struct Q4View {
  uint8_t* k_codes;   // [B, H, n_max, d / 2]
  uint8_t* k_scales;  // [B, H, n_max, d / 32]
  uint8_t* v_codes;
  uint8_t* v_scales;
  uint16_t* bounds;   // bf16 [B, H, ceil(n_max / 64), 2, d]: least and largest key values
  int32_t B, H, n_max;
};

// Rows [B, heads, T, d] of any strides (elements; channels are contiguous).
struct RowsView {
  const void* p;
  int64_t sb, sh, sr;
};

// New tokens: token t of batch entry b stands at position at[b] + t and is
// there if t < count[b] (count null: all T).
struct Q4Tokens {
  const int32_t* at;
  const int32_t* count;
  int32_t T;
};

struct RotaryArgs {
  RowsView x, xo, y, yo;  // y.p null: x alone
  int64_t Hx, Hy, B, T;
  const int32_t* pos;
  int32_t pos_per_token;  // pos [B, T] instead of [B] + t
  const double* turns;    // [rot / 2]
  int32_t rot, layout, inverse;
  float amp;
};
hipError_t launch_rotary(int dtype, int64_t d, const RotaryArgs& a, hipStream_t st);

hipError_t launch_q4_store(int dtype, int64_t d, const Q4View& c, const RowsView& k,
                           const RowsView& v, const Q4Tokens& tok, hipStream_t st);
hipError_t launch_q4_load(int dtype, int64_t d, const Q4View& c, const int32_t* at, int64_t T,
                          void* k, void* v, hipStream_t st);

struct Q4SelectArgs {
  RowsView q;
  int32_t G;  // query heads per key head
  Q4Tokens tok;
  int32_t n_sel, n_sinks, n_window;
  int32_t* blocks;   // [B, H, T, n_sel]
  int32_t t0, tn;    // the launch's tokens: t0 .. t0 + tn - 1
  uint64_t* scores;  // [B, H, tn, ceil(n_max / 64)], or a slot per workgroup (the rest)
};
// Many tokens: scores and choice in one launch, without a workspace, of the tokens whose 16
// see at most kQ4SelectBlocks blocks, then of the others.  Few: scores, then the choice by
// them, of tokens t0 .. t0 + tn - 1.
hipError_t launch_q4_select(int dtype, int64_t d, const Q4View& c, const Q4SelectArgs& a,
                            hipStream_t st);
hipError_t launch_q4_select_rest(int dtype, int64_t d, const Q4View& c, const Q4SelectArgs& a,
                                 hipStream_t st);
hipError_t launch_q4_scores(int dtype, int64_t d, const Q4View& c, const Q4SelectArgs& a,
                            hipStream_t st);
hipError_t launch_q4_pick(const Q4View& c, const Q4SelectArgs& a, hipStream_t st);

struct Q4AttnArgs {
  RowsView q, o;
  int32_t G;
  Q4Tokens tok;
  const int32_t* blocks;  // null: every cached row
  int32_t n_sel;
  Q4AttnShape shape;
  // shape.splits > 1: [slot, 16, d] sums, then [slot, 2, 16] maxima and sums
  float* part;
  // where the slots follow the sequences' lengths, the first and the number of each
  // sequence's ([tile, B], the same for every head), else null
  int2* table;
};
hipError_t launch_q4_attention(int dtype, int64_t d, const Q4View& c, const Q4AttnArgs& a,
                               hipStream_t st);
hipError_t launch_q4_prompt(int dtype, int64_t d, const Q4View& c, const Q4AttnArgs& a,
                            hipStream_t st);
hipError_t launch_q4_join(int dtype, int64_t d, const Q4View& c, const Q4AttnArgs& a,
                          hipStream_t st);

}  // namespace thin
