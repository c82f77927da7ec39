// Launch shapes of the gradient of coreset attention (host arithmetic only).
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "attn_plan.hpp"

namespace thin {

// Query rows per step of a workgroup: 32, which the bf16 instruction sums over at a time; float32
// rows of few keys 16, so that the tiles in LDS leave room for several workgroups (40 slices of
// 14251 queries over 2 keys of 128 channels 507 -> 272 us; over 128 keys of 64 channels 16 take
// 239 us where 32 take 214; not measured at 33 to 64 keys of 128 channels, where 32 queries take
// 115,200 bytes and leave one workgroup per compute unit, 16 slices of 4096 over 48 keys 78 us).
constexpr int64_t grad_tile(bool bf16, int64_t waves) { return bf16 || waves > 2 ? 32 : 16; }

struct GradShape {
  int32_t waves, tiles;  // of a workgroup; 16-key tiles of a wave
  int32_t chunks;        // workgroups along the keys
  int32_t parts;         // and along the queries, `run` steps each
  int32_t run;
  bool one;  // a workgroup holds every key: statistics and dQ come from it
  constexpr int64_t keys() const { return 16 * (int64_t)waves * tiles; }
};

// Keys that one workgroup holds at most.  (Their sums of dK and dV are float32, 2 d of them per
// key: 256 of 128 channels take half of a compute unit's registers, and float32 rows' operands
// take twice those of bf16.)
constexpr int64_t grad_most_keys(bool bf16) { return bf16 ? 256 : 128; }

// A wave of more tiles reads a step's rows from LDS for more keys, one of fewer leaves registers
// for a second wave beside it.  Sums of 64 registers per lane (tiles * d = 128) are best where
// there are keys for at least two waves; us for waves x tiles, 64 slices of 8192 queries, bf16:
//   d = 32, 64 keys 4x1 57.8, 2x2 45.7; 128 keys 8x1 107, 4x2 80.3, 2x4 70.4; 256 8x2 148, 4x4 129
//   d = 64, 64 keys 4x1 86.0, 2x2 89.9; 128 keys 8x1 141, 4x2 116, 2x4 318; 256 8x2 191, 4x4 330
// d = 128, 64 slices of 16384 queries: 128 keys 8x1 354, 4x2 500; 192 keys 12x1 495, 8x2 548, 4x3
// 504; 256 keys 8x2 548, 16x1 910, 4x4 855.  float32 rows, 64 slices of 4096 queries over 128
// keys: d = 32 8x1 135, 4x2 118; d = 64 8x1 215, 4x2 232 (with scores to base 2).
// Chunks, d = 128: 8 slices of 2048 queries over 1024 keys 8x1 96, 12x1 96, 8x2 121; 32 of 8192 over
// 512 478, 497, 627; 16 of 4096 over 600 170, 164, 245.
// exact: bf16 rows with all of a float32 dO's three parts, for which the local memory has no room
// beside over 192 keys of 128 channels.
inline GradShape grad_shape(int64_t S, int64_t n_q, int64_t n_out, int64_t d, bool bf16,
                            bool exact) {
  GradShape s{};
  s.one = n_out <= (exact && d == 128 ? 192 : grad_most_keys(bf16));
  auto is = [&](int waves, int tiles) {
    s.waves = waves;
    s.tiles = tiles;
  };
  if (n_out <= 32)
    is(2, 1);
  else if (n_out <= 64)
    d == 32 && bf16 ? is(2, 2) : is(4, 1);
  else if (n_out <= 128)
    d == 32 ? (bf16 ? is(2, 4) : is(4, 2)) : d == 64 && bf16 ? is(4, 2) : is(8, 1);
  else if (s.one && d == 128 && n_out <= 192)
    is(12, 1);
  else if (s.one)
    d == 32 ? is(4, 4) : is(8, 2);
  else  // chunks
    bf16 && d < 128 ? is(8, 2) : is(8, 1);
  s.chunks = (int32_t)((n_out + s.keys() - 1) / s.keys());
  const int64_t tile = grad_tile(bf16, s.waves), steps = (n_q + tile - 1) / tile;
  // (By waves alone.  At 128 channels LDS holds fewer: of float32 rows or a float32 dO two
  // workgroups of two waves instead of four, of float32 rows one of four waves instead of two; the
  // others wait for these.)
  const int64_t slots = s.waves > 8 ? 256 : 256 * (8 / s.waves);
  const StepSplit p = split_steps(S * s.chunks, steps, slots, 2.0, 1.0);
  s.parts = (int32_t)p.parts;
  s.run = (int32_t)p.run;
  return s;
}

// Whether the zeros of dK and dV take a launch of their own (3 us and their bytes at 7 TB/s)
// instead of the workgroups' spare time: where rows are many more than queries and a workgroup
// would have a quarter of a megabyte to write, which takes it 3 to 6 us.  In us, without and with:
//   24 slices of 3 queries, 16370 rows (fp32, d = 128, 17 MB per workgroup) 159, 82
//   84 of 271, 5533 (bf16, d = 128, 0.3 MB) 75, 52; 12 of 113, 7048 (bf16, d = 64, 0.4 MB) 57, 59
//   36 of 3451, 13941 (fp32, d = 64, 1 MB, a fourth as many queries) 79, 83
inline bool grad_zeros(const GradShape& s, int64_t n_q, int64_t n, int64_t row_bytes) {
  return n / 16 >= n_q && n * row_bytes * 2 / s.parts >= (1 << 18);
}

// Waves that share a tile of 16 query rows (and divide its keys) where the rows take a launch of
// their own: as many as leave a workgroup of eight waves for each compute unit.  In us with 1, 2
// and 4: 6 slices of 67 queries, 954 keys (fp32, d = 128) 344, 214, 152; 8 of 2048, 1024 (bf16,
// d = 128) 109, 94, 121; 15 of 2047, 333 (the same) 79, 91, 121.
inline int grad_share(int64_t S, int64_t n_q) {
  auto groups = [&](int64_t tiles) { return S * ((n_q + 16 * tiles - 1) / (16 * tiles)); };
  return groups(2) <= 256 ? 4 : groups(4) <= 256 ? 2 : 1;
}

// Bytes of the workspace: sums of dK and dV, of dlogw, and the statistics.
struct GradBytes {
  size_t part, part_w, stats;
  size_t all() const { return part + part_w + stats; }
};
inline GradBytes grad_bytes(const GradShape& s, int64_t S, int64_t n_q, int64_t d, bool weights) {
  auto up = [](size_t n) { return (n + 255) / 256 * 256; };
  const size_t slots = (size_t)(S * s.chunks * s.parts * s.keys());
  return {up(slots * 2 * (size_t)d * 4), weights ? up(slots * 4) : 0,
          s.one ? 0 : up((size_t)(S * n_q) * 12)};
}

}  // namespace thin
