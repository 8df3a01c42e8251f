// The work of the attention kernels over the key/value cache: what they are given, and how the sequences' lengths, known
// on the device only, become pieces of work.
#pragma once

#include "common.h"
#include "cache.h"
#include "cross_plan.h"

namespace rs {

// What the new rows attend to: the cached rows and their own drafts, the blocks that they select, or the cached rows that
// a key mask leaves (another sequence's states; DraftView.mask is then that mask).
enum { W_ALL = 0, W_SELECT = 1, W_CROSS = 2 };

struct DraftArgs {
  CacheView c;
  DraftView q;
  char *o;
  int64_t so_t, so_h;
  float *lse;
  float *po, *pml;   // pieces: O (unnormalised), then (max, sum) of every row
  int rtiles, trows; // row tiles of a sequence with max_rows rows, rows of one
  int slots, least;  // pieces that all items together may have beyond one each; groups of a piece at least
  const int32_t *list;  // selected blocks [nrows * hkv][nsel], or NULL: all rows
  int nsel, pieces;  // with a list: pieces per item
  int grid;          // workgroups, and slots of pieces
  int resident;      // W_CROSS: workgroups that the chip holds at once, 0: plan by slots alone
  int32_t *plan;     // cross.hip: where it leaves the groups of a piece for the joining kernel; NULL: plan_groups
};

// cross.hip: the matrix-rate kernel of W_CROSS, bf16, row tiles of 128; the join of pieces of more than 32 rows, of at most `items`.
void cross_prompt_launch(const DraftArgs &a, int d, hipStream_t st);
void cross_join_launch(const DraftArgs &a, int d, int items, hipStream_t st);

#if defined(__HIPCC__)
namespace {

// Wave-uniform loads through the scalar cache of arrays that the kernel does not write.
__device__ __forceinline__ int uload(const int32_t *p, int64_t i) {
  typedef const __attribute__((address_space(4))) int32_t cint;
  return ((cint *)p)[i];
}

// ---- the work of a workgroup -------------------------------------------------------------------
// Sequences differ in length, and their lengths are known on the device only.  Every workgroup reads all
// lengths and derives the same plan: the pieces of every item (sequence, head, row tile) in groups of 128
// rows, equal to within one, so that all items together make about `slots` pieces.

// Rows of keys of sequence b that the kernels walk: cached rows, and drafts where they are seen.
template <int WHAT>
__device__ __forceinline__ int walk_len(const DraftArgs &a, int len, int t) {
  if constexpr (WHAT == W_CROSS) return len;
  return len + t < a.c.cap ? len + t : a.c.cap;
}

// What a workgroup works on.
struct Item {
  int b, g, rt, piece, npieces, slot0;  // slot0: the first slot of pieces of the sequence (of the item, with a list)
  int len, t, first;                    // rows held, new rows and the first of them
  int per;                              // items of the sequence: its slots are piece-major
};

// (what lanes agree on, said so: scalar registers, scalar branches)
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ Item uniform(const Item &x) {
  return Item{uniform(x.b), uniform(x.g), uniform(x.rt), uniform(x.piece), uniform(x.npieces), uniform(x.slot0),
              uniform(x.len), uniform(x.t), uniform(x.first), uniform(x.per)};
}

// Sequence of new row r, by the wave; -1: none.
__device__ __forceinline__ int seq_of_row(const CacheView &c, const DraftView &q, int r, int lane) {
  for (int b0 = 0; b0 < c.nseq; b0 += 64) {
    RowRange x{0, 0};
    if (b0 + lane < c.nseq) x = new_rows(q.start, b0 + lane, q.nrows, q.max_rows);
    const unsigned long long hit = __ballot(r >= x.first && r < x.first + x.count);
    if (hit) return b0 + __builtin_ctzll(hit);
  }
  return -1;
}

// What a lane knows of sequence b = b0 + lane; without new rows it has no items.
struct Seq {
  RowRange r;
  int len, groups;
};
template <int WHAT>
__device__ __forceinline__ Seq seq_at(const DraftArgs &a, int b) {
  Seq s{RowRange{0, 0}, 0, 0};
  if (b < a.c.nseq) {
    s.r = new_rows(a.q.start, b, a.q.nrows, a.q.max_rows);
    s.len = cache_len(a.c, b);
    if (s.r.count > 0) s.groups = (walk_len<WHAT>(a, s.len, s.r.count) + kGroup - 1) / kGroup;
  }
  return s;
}

// Items of a sequence, heads x row tiles: those of its own rows (W_ALL: of max_rows).
template <int WHAT>
__device__ __forceinline__ int items_of(const DraftArgs &a, const Seq &q) {
  if constexpr (WHAT == W_CROSS) return a.c.hkv * ((a.q.hq / a.c.hkv * q.r.count + a.trows - 1) / a.trows);
  return a.c.hkv * a.rtiles;
}

// Groups per piece: the same from the lengths alone in every workgroup and in the joining kernel.  first: the
// sequences of the first round of lanes.
template <int WHAT>
__device__ __forceinline__ int plan_groups(const DraftArgs &a, const Seq &first, int lane) {
  if (a.slots == 0) return kMaxN;  // one piece each
  if constexpr (WHAT == W_CROSS) {
    // f's sum over the sequences (the host bounds row tiles by 2^23: tiles x groups pass 32 bits)
    auto all = [&](auto f) {
      long long x = f(first);
      for (int b0 = 64; b0 < a.c.nseq; b0 += 64) x += f(seq_at<WHAT>(a, b0 + lane));
      return wave_sum_long(x);
    };
    const long long work = all([&](const Seq &q) { return (long long)items_of<WHAT>(a, q) * q.groups; });
    long long groups = (work + a.slots - 1) / a.slots;
    groups = groups > a.least ? groups : a.least;
    if (a.resident) {
      // One round of workgroups, each with a piece, unless sequences differ so much that a fifth of the round's time would
      // pass with some of them idle: then pieces of a quarter of a round (32 sequences of 0 to
      // 16384 states, 8 heads: 238 -> 200 us).
      int most = 0;
      for (int b0 = 0; b0 < a.c.nseq; b0 += 64) {
        const Seq q = b0 ? seq_at<WHAT>(a, b0 + lane) : first;
        const int n = q.groups > 0 ? (q.groups + pieces_of(q.groups, (int)groups) - 1) / pieces_of(q.groups, (int)groups) : 0;
        most = larger(most, n);
      }
      most = wave_most(most);
      if (work * 5 < (long long)most * a.resident * 4) groups = (work + 4 * a.resident - 1) / (4 * a.resident);
    }
    return groups > a.least ? (int)groups : a.least;
  }
  int work = first.groups;  // (at most 65535 sequences of 2048 groups)
  for (int b0 = 64; b0 < a.c.nseq; b0 += 64) work += seq_at<WHAT>(a, b0 + lane).groups;
  work = wave_sum(work);
  // with pieces of at most C = ceil(total / slots) groups an item of n groups has less than n / C + 1 of them:
  // all together at most slots + the number of items, which is what the host counts
  const long long total = (long long)work * a.c.hkv * a.rtiles, groups = (total + a.slots - 1) / a.slots;
  return groups > a.least ? (int)groups : a.least;
}

// The id-th piece overall, at `groups` groups a piece; false: there are fewer.  q: the sequences of the first round of lanes.
template <int WHAT>
__device__ __forceinline__ bool find_piece(const DraftArgs &a, Seq q, int groups, int id, int lane, Item &it) {
  int base = 0;
  for (int b0 = 0; b0 < a.c.nseq; b0 += 64) {
    if (b0) q = seq_at<WHAT>(a, b0 + lane);
    const int np = q.r.count > 0 ? pieces_of(q.groups, groups) : 0, per = items_of<WHAT>(a, q);
    const int s = wave_scan(np * per), all = __builtin_amdgcn_readlane(s, 63);
    if (id < base + all) {
      const int l = __builtin_ctzll(__ballot(id < base + s));
      it.b = b0 + l;
      it.npieces = __builtin_amdgcn_readlane(np, l);
      it.first = __builtin_amdgcn_readlane(q.r.first, l);
      it.t = __builtin_amdgcn_readlane(q.r.count, l);
      it.len = __builtin_amdgcn_readlane(q.len, l);
      it.per = WHAT == W_CROSS ? __builtin_amdgcn_readlane(per, l) : per;
      it.slot0 = base + __builtin_amdgcn_readlane(s, l) - it.npieces * it.per;
      const int x = id - it.slot0;  // piece-major: all heads' row tiles of a piece adjacent
      it.piece = x / it.per;
      const int y = x - it.piece * it.per;
      it.rt = y / a.c.hkv;
      it.g = y - it.rt * a.c.hkv;
      return true;
    }
    base += all;
  }
  return false;
}
template <int WHAT>
__device__ bool find_item(const DraftArgs &a, int id, int lane, Item &it) {
  const Seq q = seq_at<WHAT>(a, lane);
  return find_piece<WHAT>(a, q, plan_groups<WHAT>(a, q, lane), id, lane, it);
}

}  // namespace
#endif

}  // namespace rs
