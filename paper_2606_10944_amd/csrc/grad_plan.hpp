// Launch shapes of the gradient of coreset attention (host arithmetic only).
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "attn_plan.hpp"

namespace thin {

constexpr int64_t kGradTile = 32;  // query rows per step of a workgroup

struct GradShape {
  int32_t waves, tiles;  // of a workgroup; 16-key tiles of a wave
  int32_t chunks;        // workgroups along the keys
  int32_t parts;         // and along the queries, `run` steps each
  int32_t run;
  bool one;  // a workgroup holds every key: statistics and dQ come from it
  constexpr int64_t keys() const { return 16 * (int64_t)waves * tiles; }
};

// Keys that one workgroup holds at most: 32 per wave of eight (bf16), whose sums of dK and dV
// take half of its registers, or 16 (float32).
constexpr int64_t grad_most_keys(bool bf16) { return bf16 ? 256 : 128; }

inline GradShape grad_shape(int64_t S, int64_t n_q, int64_t n_out, int64_t d, bool bf16) {
  GradShape s{};
  s.one = n_out <= grad_most_keys(bf16);
  s.waves = n_out <= 32 ? 2 : n_out <= 64 ? 4 : 8;
  s.tiles = bf16 && n_out > 128 && (s.one || d < 128) ? 2 : 1;
  if (bf16 && n_out > 128 && n_out <= 192 && d == 128) {
    s.waves = 12;
    s.tiles = 1;
  }
  s.chunks = (int32_t)((n_out + s.keys() - 1) / s.keys());
  const int64_t steps = (n_q + kGradTile - 1) / kGradTile;
  const int64_t slots = 256 * (s.waves > 8 ? 1 : 8 / s.waves);
  const StepSplit p = split_steps(S * s.chunks, steps, slots, 2.0, 1.0);
  s.parts = (int32_t)p.parts;
  s.run = (int32_t)p.run;
  return s;
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
          s.one ? 0 : up((size_t)(S * n_q) * 8)};
}

}  // namespace thin
