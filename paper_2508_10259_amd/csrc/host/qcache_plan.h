// Launch plan of the attention over the 8-bit K/V cache: plain host arithmetic, shared by the
// launcher, the C ABI's workspace size and the context's layout.
#pragma once

#include <algorithm>
#include <cstddef>
#include <cstdint>

namespace ams {

// keys: a workgroup's four waves share qt tiles of 16 query columns and deal the positions among them;
// otherwise each wave has qt tiles of its own.  tiles: workgroups along a segment's columns; splits:
// along its positions, `per` steps of 32 each, leaving partial sums of part_floats in all (0 for one split).
struct QAttendPlan {
  bool keys;
  int qt, tiles, splits, per;
  size_t part_floats;
};

// A call of n_seg segments of at most max_new tokens, n_tok in all, over about max_len positions (n_select > 0:
// over that many pages of 64 for each token); room: floats there are for partial sums.
inline QAttendPlan qcache_attend_plan(int n_seg, int n_heads, int n_kv, int dh, int n_tok, int max_new, int max_len,
                                      int n_select, size_t room = SIZE_MAX) {
  QAttendPlan p{};
  const int64_t G = n_heads / n_kv, cols = n_select ? G : max_new * G;
  p.keys = n_select > 0 || cols <= 32;
  p.qt = p.keys && (cols <= 16 || n_select) ? 1 : 2;
  const int per = p.keys ? 16 * p.qt : 64 * p.qt;
  p.tiles = (int)((cols + per - 1) / per);
  // Splits: until there are 512 workgroups (two per CU); a split keeps at least 8 steps of 32 positions for
  // each wave that shares it, since joining splits costs a launch (4 us) and a round trip through memory.
  // Measured: 16 rows of 600 to 656 positions in fp32, 32 heads of 128: 19.5 us in one split, 28 in two; four rows of
  // 70,000 to 131,072, 8 KV heads: 157 us with 512 workgroups, 174 with 768, 183 with 1,024.
  const int64_t blocks = (int64_t)n_seg * n_kv * p.tiles * (n_select ? max_new : 1);
  const int64_t steps = (n_select ? (int64_t)n_select * 64 : max_len) / 32 + 1, least = p.keys ? 32 : 16;
  const size_t one = (size_t)n_tok * n_heads * (dh + 4);
  int64_t s = std::min<int64_t>({(512 + blocks - 1) / blocks, (steps + least - 1) / least, 256});
  s = std::min<int64_t>(s, (int64_t)std::min<size_t>(room / one, 256));
  s = std::max<int64_t>(s, 1);
  p.per = (int)((steps + s - 1) / s);
  p.splits = (int)((steps + p.per - 1) / p.per);
  p.part_floats = p.splits > 1 ? one * p.splits : 0;
  return p;
}

}  // namespace ams
