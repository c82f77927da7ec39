// Launch shapes of the 4-bit cache's operators (host arithmetic only).
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace thin {

constexpr int32_t kQ4MaxTokens = 1 << 20;  // per batch entry and call
constexpr int32_t kQ4MaxGroup = 1024;      // query heads per key head
constexpr int32_t kQ4MaxSplits = 512;      // workgroups that share one tile's keys
constexpr int32_t kQ4SharedEntries = 256;  // batch entries whose tiles' keys are shared out
constexpr int32_t kQ4Step = 32;            // keys per step of a wave

// Tiles of 16 query rows per slice: heads of one token (list), or heads of tokens in a row.
inline int64_t q4_row_tiles(int64_t G, int64_t T, bool list) {
  return list ? T * ((G + 15) / 16) : (T * G + 15) / 16;
}

// Query rows of a workgroup of the kernel for many of them.
constexpr int64_t q4_prompt_rows(bool bf16) { return bf16 ? 128 : 64; }

// Workgroups of an attention launch.
struct Q4AttnShape {
  int32_t waves;   // per workgroup; 0: the kernel for many query rows
  int32_t splits;  // workgroups per tile (list), or per tile on average over the sequences
  int32_t least;   // steps of 32 keys that a workgroup takes at least
};

// Few query rows per slice.  A tile's keys go to one workgroup, without a second launch to
// join sums, up to 2048 keys, and up to 4096 where there are workgroups for most compute
// units (d = 128, 4000 rows, one token: 256 workgroups, bf16 25.8 us against 30.0 shared
// out, 22.4 against 23.7 with lengths of 10 to 4000; 160: 22.4, 23.4 and 20.4, 18.8; 128:
// 22.4, 20.7 and 19.7, 17.1).  A compute unit holds one workgroup of eight waves of float32
// rows of 128 (their registers), two of others: four waves where there are more (d = 128,
// 384 workgroups over 1024 rows: float32 22.2 us with eight, 17.7 with four, bf16 18.6,
// 15.0; over 2000 rows 32.4, 27.8 and 27.2, 23.1; d = 64, 320 over lists of 32 blocks: 15.6,
// 16.6).
// Longer keys are shared out to two workgroups of four waves per compute unit (512; 8
// sequences of 3000 to 55000 rows, 8 key heads, d = 128, bf16: 43.7 us, against 51.6 with
// 256, 45.9 with 768, 49.7 with 1024, the last of them run alone), those of more slices in
// two, so that one long sequence among short ones is not left to one workgroup per head.
// Beyond 1024 tiles, several for every compute unit, or kQ4SharedEntries sequences, four of
// them per lane of the wave that shares them out, every tile has one workgroup (160 sequences
// x 8 heads of 3000 to 65536 rows: 1155 us, against 1084 in two; all of 65536: 1872, 1895; of
// 500 to 16000: 292, 287; 300 x 2 of 500 to 16000: 146, 4.6 TB/s).
//
// Many query rows.  The kernel that shares decoded rows pays where each compute unit has a
// workgroup of it (16 sequences x 8 heads x 1024 rows, 256 query rows a head, 256
// workgroups: 32 us against 43; 128 query rows, 128 workgroups: 29 against 24), or where its
// keys are shared out.  Tiles of 16 of 8 key heads, bf16: 192 over 40000 rows 75 us against
// 165, over 16000 44 and 73, over 4500 30 and 31; 128 over 16000 38 and 45, over 4500 28 and
// 24, 64 over 16384 31 and 30.  Up to 4096 rows one workgroup per tile is quicker for longer:
// 512 tiles over 4000 rows 39 against 41, 1024 65 against 54.
inline Q4AttnShape q4_attention_shape(int64_t B, int64_t H, int64_t G, int64_t T, bool list,
                                      int64_t keys, int64_t d, bool bf16) {
  const int64_t groups = B * H * q4_row_tiles(G, T, list);
  if (!list && T * G >= 64) {
    const int64_t per = q4_prompt_rows(bf16), wide = B * H * ((T * G + per - 1) / per);
    if (keys <= 2048 ? wide >= 256 : groups > (keys <= 4096 ? 512 : 127)) {
      if (keys <= 2048 || wide >= 512) return {0, 1, 1};
      const int64_t splits = 512 / wide, most = keys / 512;
      return {0, (int32_t)(splits < most ? splits : most), 1};
    }
  }
  if (keys <= (groups < 192 ? 2048 : 4096) || groups > 1024 || B > kQ4SharedEntries)
    return {groups > (d == 128 ? 256 : 511) ? 4 : 8, 1, 1};
  const int64_t steps = (keys + kQ4Step - 1) / kQ4Step;
  int64_t splits = 512 / groups;
  if (splits < 2) splits = 2;
  if (splits > steps / 4) splits = steps / 4;
  if (splits > kQ4MaxSplits) splits = kQ4MaxSplits;
  int64_t least = (steps + kQ4MaxSplits - 1) / kQ4MaxSplits;
  if (least < 4) least = 4;
  return {4, (int32_t)splits, (int32_t)least};
}

// Bytes of the splits' sums (a slot of [16, d] float32, maxima and sums of 16 rows), and of
// them with the table of slots behind.
inline size_t q4_sums_bytes(int64_t B, int64_t H, int64_t tiles, int64_t splits, int64_t d) {
  return (size_t)(B * H * tiles * splits) * (16 * d + 32) * 4;
}
inline size_t q4_attention_bytes(int64_t B, int64_t H, int64_t tiles, int64_t splits, int64_t d) {
  return splits > 1 ? q4_sums_bytes(B, H, tiles, splits, d) + (size_t)(tiles * B) * 8 : 0;
}

// Whether a selection takes 16 tokens at a time with their scores in LDS, and whether that
// is all of it: tokens that see more blocks than LDS holds are left to a second launch.
constexpr int64_t kQ4SelectBlocks = 2048;  // 16 tokens' float32 scores: 128 KiB
inline bool q4_select_grouped(int64_t slices, int64_t T) {
  return T > 1 && slices * ((T + 15) / 16) >= 64;
}
inline bool q4_select_fused(int64_t slices, int64_t blocks, int64_t T) {
  return blocks <= kQ4SelectBlocks && q4_select_grouped(slices, T);
}

// Workgroups of that second launch, each with a slot for the scores of a token: two per
// compute unit, 64 MiB of slots, at least one.
inline int64_t q4_select_slots(int64_t slices, int64_t blocks, int64_t T) {
  const int64_t hold = ((int64_t)64 << 20) / (blocks * 8), all = slices * T;
  const int64_t n = hold < 512 ? hold : 512;
  return n < 1 ? 1 : (n < all ? n : all);
}

// Tokens of few whose block scores a selection holds at a time: 64 MiB of them, at least
// one token's.
inline int64_t q4_select_tokens(int64_t slices, int64_t blocks, int64_t T) {
  const int64_t n = ((int64_t)64 << 20) / (slices * blocks * 8);
  return n < 1 ? 1 : (n < T ? n : T);
}

}  // namespace thin
