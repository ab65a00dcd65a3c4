// Launch plan of the attention over the 8-bit K/V cache: plain host arithmetic, shared by the
// launcher, the C ABI's workspace size and the context's layout.
#pragma once

#include <algorithm>
#include <cstddef>
#include <cstdint>

namespace ams {

// A split of an attention has at least this many steps of 32 positions: 8 for each wave that shares it.
constexpr int QCACHE_LEAST_STEPS = 32;

// Workgroups of one launch of the 8-bit cache's kernels (of 1,024 threads at most: a grid has fewer than
// 2^32 threads).
constexpr int64_t QCACHE_MAX_BLOCKS = (int64_t)1 << 22;

// keys: a workgroup's four waves share qt tiles of 16 query columns and deal the positions among them;
// otherwise each wave has qt tiles of its own.  tiles: workgroups along a segment's columns; splits: at most
// as many along its positions, `per` steps of 32 each (even: as many as make the pieces of all segments equal),
// leaving partial sums of part_floats in all (0 for one split).  blocks above 2^31 - 1: no launch can
// hold them, and nothing else is planned.
struct QAttendPlan {
  bool keys, even;
  int qt, tiles, splits, per;
  size_t part_floats;
  int64_t blocks;
};

// A call of n_seg segments of at most max_new tokens, n_tok in all, over about max_len positions (n_select > 0:
// over that many pages of 64 for each token); room: floats there are for partial sums; even_below: pairs of a segment and
// a KV head (times its tiles) below which rows are cut into equal pieces.
inline QAttendPlan qcache_attend_plan(int n_seg, int n_heads, int n_kv, int dh, int n_tok, int max_new, int max_len,
                                      int n_select, size_t room = SIZE_MAX, int even_below = 512) {
  QAttendPlan p{};
  const int64_t G = n_heads / n_kv, cols = n_select ? G : max_new * G;
  // Up to 32 columns the waves of a workgroup share them, above that each has its own.  64 rows of 216 to 700 positions, 32
  // heads, 33 new tokens: 104 us, 119 if shared; 48 tokens 105 (119).  Few pairs with 33 to 64 columns would be better off
  // shared, whose rows can be cut: 4 rows of 8,000 to 16,384, 8 x 4 heads, 9 tokens 48.4 us (39.4), 16 tokens 51.2 (41.2).
  p.keys = n_select > 0 || cols <= 32;
  p.qt = p.keys && (cols <= 16 || n_select) ? 1 : 2;
  const int width = p.keys ? 16 * p.qt : 64 * p.qt;
  const int64_t tiles = (cols + width - 1) / width;
  const int64_t blocks = (int64_t)n_seg * n_kv * tiles * (n_select ? max_new : 1);  // (below 2^62 by the calls' limits)
  p.blocks = blocks;
  if (blocks > INT32_MAX) return p;
  p.tiles = (int)tiles;
  // Splits are for launches with too few workgroups; joining them costs a launch (4 us) and a round trip
  // through memory (16 rows of 600 to 656 positions in fp32, 32 heads of 128: 19.5 us in one split, 28 in two).
  const int64_t steps = (n_select ? (int64_t)n_select * 64 : max_len) / 32 + 1;
  const size_t one = (size_t)n_tok * n_heads * (dh + 4);
  const int64_t fit = (int64_t)std::min<size_t>(room / one, 512);
  int64_t s = 1;
  p.even = p.keys && !n_select && blocks < even_below && steps > QCACHE_LEAST_STEPS;
  if (p.even) {
    // 512 equal pieces, two for each CU; from 256 pairs on 1,536, which the CUs take as they get free.  Rows of 8,000 to
    // 32,000 positions, 32 heads of 128, bf16, against splits that are dealt alike: 4 rows 126 us (129), 10 rows 298
    // (325), 12 rows 353 (373); of 1,200 to 2,400: 4 rows 22.2 (20.7), 10 rows 39.6 (38.9), 12 rows 46.5 (42.9).  From 512
    // pairs on pieces lose at every length: 16 rows 487 (471) and 57.2 (46.4), 23 rows 680 (672) and 74.1 (65.1).  768 and
    // 1,024 pieces for 4 rows of 70,000 to 131,000 positions, 8 x 4 heads: 162 and 168 us (157 with 512).
    const int64_t pieces = (blocks <= 256 ? 512 : 1536) - blocks;
    s = std::min(pieces / ((int64_t)n_kv * p.tiles), fit);
    p.even = s > n_seg;
  }
  if (!p.even) {
    const int64_t least = p.keys ? QCACHE_LEAST_STEPS : QCACHE_LEAST_STEPS / 2;
    s = std::min<int64_t>({(512 + blocks - 1) / blocks, (steps + least - 1) / least, fit});
    s = std::max<int64_t>(s, 1);
    p.per = (int)((steps + s - 1) / s);
    s = (steps + p.per - 1) / p.per;
  }
  p.splits = (int)s;
  p.part_floats = s > 1 ? one * s : 0;
  p.blocks = p.even ? (int64_t)n_kv * p.tiles * (s + n_seg) : blocks * s;
  return p;
}

}  // namespace ams
