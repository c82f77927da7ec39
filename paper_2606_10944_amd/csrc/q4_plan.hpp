// Launch shapes of the 4-bit cache's operators (host arithmetic only).
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace thin {

// Tiles of 16 query rows per slice: heads of one token (list), or heads of tokens in a row.
inline int64_t q4_row_tiles(int64_t G, int64_t T, bool list) {
  return list ? T * ((G + 15) / 16) : (T * G + 15) / 16;
}

// Workgroups that share the keys of a tile: enough of them for the device's 256
// compute units to hold four each, with at least 128 keys for each.
inline int64_t q4_splits(int64_t slices, int64_t tiles, int64_t keys) {
  const int64_t groups = slices * tiles, want = groups < 1024 ? 1024 / groups : 1;
  const int64_t most = (keys + 127) / 128;
  return want < most ? want : most;
}

// Bytes of the splits' sums: [tile, split, 16, d] float32, a maximum and a sum per row.
inline size_t q4_attention_bytes(int64_t slices, int64_t tiles, int64_t splits, int64_t d) {
  return splits > 1 ? (size_t)(slices * tiles * splits) * (16 * d + 32) * 4 : 0;
}

// Tokens whose block scores a selection holds at a time: 64 MiB of them, at least one
// token's.
inline int64_t q4_select_tokens(int64_t slices, int64_t blocks, int64_t T) {
  const int64_t n = ((int64_t)64 << 20) / (slices * blocks * 8);
  return n < 1 ? 1 : (n < T ? n : T);
}

}  // namespace thin
