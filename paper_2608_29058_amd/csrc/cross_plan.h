// Pieces of the kernel of prompts (cross.hip): what the host makes room for, and the groups per piece that every workgroup
// derives from the lengths.  Plain C++, which compiles for the host too.
#pragma once

#include "cache.h"

namespace rs {

constexpr int kTile = 32, kWaves = 4, kGroup = kTile * kWaves;  // rows per wave and step, per workgroup and step
constexpr int kMaxGrid = 1 << 23;  // workgroups of up to 512 threads, of which a launch has fewer than 2^32

// Pieces of a sequence of `tiles` groups at `per` groups a piece.
RS_HD int pieces_of(int tiles, int per) { return tiles > per ? (tiles + per - 1) / per : 1; }
// The same by the product with inv = 1.f / per (quotients of at most 2^11 by at most 2^11: ceil, less half a step).
RS_HD int pieces_by(int tiles, int per, float inv) {
  return tiles > per ? (int)__builtin_ceilf(((float)tiles - 0.5f) * inv) : 1;
}

// Row tiles of all sequences at `trows` rows, `rows` those of a sequence at most: a sequence has those of its own rows, less than
// one of them not full.
inline int64_t cross_tiles(const CacheView &c, const DraftView &q, int rows, int trows) {
  const int64_t all = (int64_t)c.nseq * ((rows + trows - 1) / trows), own = (int64_t)(q.hq / c.hkv) * q.nrows / trows + c.nseq;
  return all < own ? all : own;
}

// What the host plans for `items` of at most `cap` states, with `resident` workgroups at once: workgroups and slots of pieces
// (grid), groups of a piece at least, whether items are split at all.
struct RoundsShape {
  int grid, least;
  bool split;
};
inline RoundsShape rounds_shape(int64_t items, int cap, int resident) {
  RoundsShape s{0, 4, false};
  const int64_t most = items * ((cap + kGroup - 1) / kGroup);
  s.split = cap > s.least * kGroup && items < 8 * resident;
  int64_t n = !s.split ? items : items < resident ? resident : items + 4 * resident;
  n = n < most ? n : most;
  s.grid = n < kMaxGrid ? (int)n : kMaxGrid;
  return s;
}

// Groups per piece.  The chip works in rounds of `resident` workgroups, so that the time is about that of the rounds' longest pieces
// and of what pieces write and the join reads: 132 KB each, at 5 TB/s 1/128 of the time of a round's group (3.9 us; heads of 128, and
// about right for those of 64, which write half and take two thirds).  For each
// number of rounds the shortest pieces that fit are found; of those, and of whole items, the fastest are taken.  (64 rows of 32 heads of
// 128 over 3900 states of 8, 496 groups: 31 us, in one piece per item 83.)
// items, work: items, and their groups in all; longest: groups of the longest; pieces(per): pieces at `per` groups each.
template <typename Pieces>
RS_HD int rounds_groups(int items, int work, int longest, int resident, int grid, int least, Pieces pieces) {
  const int fewest = (items + resident - 1) / resident;
  int best = longest, cost = fewest * longest * 128;
  // (a grid that holds all groups as pieces is room enough for any plan, be it less than a round; more rounds have no more)
  for (int r = fewest > 0 ? fewest : 1, room = 0; r < fewest + 4 && room < grid; ++r) {
    room = r * resident < grid ? r * resident : grid;
    int lo = (work + room - 1) / room;
    lo = lo > least ? lo : least;
    const int few = work / lo;
    if (r * lo * 128 + (items > few ? items : few) >= cost) continue;
    int n = pieces(lo);
    if (n > room) {
      // (an item of n groups has less than n / per + 1 pieces)
      int hi = room > items ? (work + room - items - 1) / (room - items) : longest;
      hi = hi < longest ? hi : longest;
      for (++lo; lo < hi;) {
        const int per = (lo + hi) >> 1;
        if (pieces(per) <= room) hi = per;
        else lo = per + 1;
      }
      n = pieces(lo);
    }
    const int c = r * lo * 128 + n;
    if (n <= room && c < cost) cost = c, best = lo;
  }
  return best;
}

}  // namespace rs
