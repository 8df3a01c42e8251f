// Launch shapes of rope.hip.  Plain C++, which compiles for the host alone too.
#pragma once

#include <stdint.h>

#include "../../include/rs.h"

namespace rs {

constexpr int kRopeThreads = 256;

// log2 of the groups of heads that share a row.  Where a token's heads lie together a workgroup takes one row, a head per
// group, so that it reads and writes long pieces of memory, or two rows where pairs pass through LDS, so that a group has a second
// head to load meanwhile; where a head's tokens lie together, one group with a row per LPR lanes does, split further only until the rows
// fill the chip's 2^19 lanes.  (8192 rows of 32 + 2 x 8 heads of 128 appended to four sequences each: one row 133 us, two 133, four 139;
// 30001 rows of 32 + 8: 96, 97, 101; half of each turned: 131, 104, 105.)  A launch has fewer than 2^32 lanes, which 2^24 rows in groups
// of their own would pass.
inline int head_groups(int64_t rows, int d, int heads, bool tokens, const rs_rope &r) {
  const int most = (d == 128 ? 5 : 6) - (r.layout == RS_ROPE_HALF && r.dim < d);
  int lg = 0;
  while (lg < most && (1 << lg) < heads && rows * (d / 16) << lg < (tokens ? 1ll << 31 : 1ll << 19)) ++lg;
  return lg;
}

// Workgroups of an append: x of `per` rows each, for each of y sequences, or (byrow) of the whole batch.  A sequence takes
// max_rows rows at most, but where only some come near that, most of nseq x max_rows are no rows: then the workgroups are dealt to
// the batch's rows, and find their sequences in `start`, 256 of them at a time.  A step of that search costs about half of what a
// workgroup without rows does, and its barriers 0.3 us of a short call.  (32 + 2 x 8 heads of 128, us by sequence and by row:
// 8192 rows of one sequence and one of 63 more 151 and 33; 512 and 31 8.8 and 5.5, 100 and 15 4.5 and 4.6, 64 and 3 4.3 and 4.6; 16 and
// 4095 113 and 33, 3 and 4095 19 and 33.)  Without queries nothing is done for rows behind the capacity.
struct AppendShape {
  int lg, per;
  int64_t x, y;
  bool byrow;
};
inline AppendShape append_rope_shape(int nseq, int cap, int nrows, int max_rows, bool start, int d, int hkv, int hq, bool tokens, const rs_rope &r) {
  AppendShape s{};
  int most = max_rows < nrows ? max_rows : nrows;  // rows of a sequence at most
  if (hq == 0 && cap < most) most = cap;
  const int64_t all = (int64_t)nseq * most;
  s.lg = head_groups(all < nrows ? all : nrows, d, hkv + hq, tokens, r);
  s.per = kRopeThreads / (d / 16) >> s.lg;
  const int64_t own = (nrows + s.per - 1) / s.per, idle = (all - nrows) / s.per, search = own * ((nseq + kRopeThreads - 1) / kRopeThreads);
  s.byrow = start && idle > 2048 + search / 2;
  s.x = ((s.byrow ? nrows : most) + s.per - 1) / s.per;
  s.y = s.byrow ? 1 : nseq;
  return s;
}

}  // namespace rs
