// Attention of new (drafted) rows over the key/value cache: all cached rows (rs_draft_attn), blocks that a
// score selects (rs_select_attn), and the weight that each cached row receives (rs_attn_weights).
//
// For a row r of key/value head g (a query head of a new token) over its visible rows j:
//   l_j = scale q_r . k_j,  p_j = exp(l_j - max l),  O = sum p_j v_j / sum p_j.
// A decode step reads every cached row for at most a few rows r, so memory bounds it: 4 d bytes of K and V
// per row and head against 4 d (hq / hkv) t flops.  The kernels therefore stream K and V from memory
// straight into the registers that the matrix instructions read, without LDS and without barriers:
//   S^T [32 rows x 16] = K Q^T: lane (m = lane % 16, h = lane / 16) holds row m and 8 dimensions of it per
//     instruction (v_mfma_f32_16x16x32_bf16), which is 16 contiguous bytes of K;
//   O^T [d x 16] += V^T P^T: the contraction runs over rows in the order 4h + 0..3, 16 + 4h + 0..3, the rows
//     whose S the lane holds, so P needs no exchange of lanes; and the lane reads dimensions
//     (d / 16) m ... of those 8 rows, a whole row per 16 lanes, whose transposition into the instructions'
//     operands (dimension (d / 16) m + t of the t-th) stays inside the lane: one v_perm per two values.
// Each of the four (short caches: eight) waves takes every fourth (eighth) tile of 32 rows with a running maximum and
// sum of its own and keeps the next tile in flight; the waves are joined once, through LDS, at the end.
#include "common.h"
#include "cache.h"

namespace rs {

namespace {

constexpr int kTile = 32, kWaves = 4, kGroup = kTile * kWaves;  // rows per wave and step, per workgroup and step

__device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(a), as_bf16x8(b), c, 0, 0, 0);
}

// Values of lanes i, i ^ 16, i ^ 32 and i ^ 48 joined, in all four.
// (elements are copied out first: __builtin_bit_cast of a vector's element reads element 0)
__device__ __forceinline__ void halves(u32x2 r, float &a, float &b) {
  const uint32_t x = r[0], y = r[1];
  a = __builtin_bit_cast(float, x);
  b = __builtin_bit_cast(float, y);
}
template <typename F>
__device__ __forceinline__ float join4(float x, F f) {
  float a, b;
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  halves(__builtin_amdgcn_permlane32_swap(u, u, false, false), a, b);
  const uint32_t v = __builtin_bit_cast(uint32_t, f(a, b));
  halves(__builtin_amdgcn_permlane16_swap(v, v, false, false), a, b);
  return f(a, b);
}
__device__ __forceinline__ float max4(float x) { return join4(x, [](float a, float b) { return fmaxf(a, b); }); }
__device__ __forceinline__ float sum4(float x) { return join4(x, [](float a, float b) { return a + b; }); }

// Maximum and sum over the wave.
template <int CTRL, int ROWS>
__device__ __forceinline__ float dpp_or(float other, float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, other), __builtin_bit_cast(int, x), CTRL, ROWS, 0xf, false));
}
template <typename F>
__device__ __forceinline__ float wave_fold(float x, float none, F f) {
  x = f(x, dpp_or<0x111, 0xf>(none, x));
  x = f(x, dpp_or<0x112, 0xf>(none, x));
  x = f(x, dpp_or<0x114, 0xf>(none, x));
  x = f(x, dpp_or<0x118, 0xf>(none, x));
  x = f(x, dpp_or<0x142, 0xa>(none, x));
  x = f(x, dpp_or<0x143, 0xc>(none, x));
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63));
}
__device__ __forceinline__ float wave_max(float x) {
  return wave_fold(x, -__builtin_inff(), [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float wave_total(float x) {
  return wave_fold(x, 0.f, [](float a, float b) { return a + b; });
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// x as hi + lo, both bf16 (8 + 8 bits of its 24).  hi ends at 2^96, so that it is finite, and what is infinite or
// undefined lies in lo alone: the products hi.lo and hi.hi beside it stay finite and keep its sign (a lo that
// subtracts an infinite hi is NaN).  Magnitudes beyond 2^96 have lo's 8 bits.  The clamp is one v_med3 per value: up to
// 6 % of a call's time, 10 % with 17 to 32 rows of Q of d = 128 (16 sequences of 16000 rows, 8 heads: 452 -> 495 us; testing
// the scores and trying again, or walking a piece again, spills registers and takes as long).
constexpr float kSplitMax = 0x1p96f;
__device__ __forceinline__ void split2(float a, float b, uint32_t &hi, uint32_t &lo) {
  hi = pack_bf16x2(__builtin_amdgcn_fmed3f(a, -kSplitMax, kSplitMax), __builtin_amdgcn_fmed3f(b, -kSplitMax, kSplitMax));
  lo = pack_bf16x2(a - __builtin_bit_cast(float, hi << 16), b - __builtin_bit_cast(float, hi & 0xffff0000u));
}

// 8 fp32 values (two 16-byte registers) as two bf16 operands
__device__ __forceinline__ void split8(f32x4 a, f32x4 b, u32x4 &hi, u32x4 &lo) {
  uint32_t h, l;
  split2(a[0], a[1], h, l), hi[0] = h, lo[0] = l;
  split2(a[2], a[3], h, l), hi[1] = h, lo[1] = l;
  split2(b[0], b[1], h, l), hi[2] = h, lo[2] = l;
  split2(b[2], b[3], h, l), hi[3] = h, lo[3] = l;
}

// Wave-uniform loads through the scalar cache of arrays that the kernel does not write.
__device__ __forceinline__ int uload(const int32_t *p, int64_t i) {
  typedef const __attribute__((address_space(4))) int32_t cint;
  return ((cint *)p)[i];
}

// ---- one tile of K and V in registers --------------------------------------------------------
// CH: 16-byte pieces of a lane per K row part of 32 dimensions (1 bf16, 2 fp32).
template <bool F32, int D>
struct Tile {
  static constexpr int KC = D / 32, CH = F32 ? 2 : 1, DT = D / 16;  // DT: output tiles, dimensions per lane of V
  static constexpr int VW = DT * (F32 ? 4 : 2) / 4;                 // words of V per lane and row
  u32x4 k[2][KC][CH];
  uint32_t v[8][VW];
};

template <bool F32, int D>
using VTile = uint32_t[8][Tile<F32, D>::VW];

// The rows of a tile: page and first row in it; rows behind `last` are read as the last (and masked).
struct TileAt {
  const char *k, *v;
  int last;   // last row of the tile that may be read, 0 .. 31
  bool ok;    // the table names a page
};

// The tile from row j of sequence b and head g, whose rows end before `total`.  Without a page: row 0 of page 0,
// to be masked.
__device__ __forceinline__ TileAt tile_at(const CacheView &c, int b, int g, int j, int total) {
  const int p = page_of(c, j);
  const int id = checked_page(c, c.table ? uload(c.table, (int64_t)b * c.max_pages + p) : b * c.max_pages + p);
  TileAt at;
  at.ok = id >= 0;
  at.k = c.k + (at.ok ? k_offset(c, id, p, j, g) : g * c.sk_h);
  at.v = c.v + (at.ok ? v_offset(c, id, p, j, g) : g * c.sv_h);
  at.last = !at.ok ? 0 : total - 1 - j < kTile - 1 ? total - 1 - j : kTile - 1;
  return at;
}

template <bool F32, int D>
__device__ __forceinline__ void load_k(Tile<F32, D> &t, const TileAt &at, int64_t sk, int m, int h) {
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    const int r = 16 * s + m;
    const char *p = at.k + (r < at.last ? r : at.last) * sk + h * (F32 ? 32 : 16);
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
#pragma unroll
      for (int x = 0; x < Tile<F32, D>::CH; ++x) t.k[s][c][x] = *(const u32x4 *)(p + c * (F32 ? 128 : 64) + x * 16);
  }
}

template <bool F32, int D>
__device__ __forceinline__ void load_v(Tile<F32, D> &t, const TileAt &at, int64_t sv, int m, int h) {
  constexpr int VW = Tile<F32, D>::VW;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = (i < 4 ? i : 12 + i) + 4 * h;
    const char *p = at.v + (r < at.last ? r : at.last) * sv + m * (VW * 4);
    if constexpr (VW == 2) {
      const u32x2 x = *(const u32x2 *)p;
      t.v[i][0] = x[0], t.v[i][1] = x[1];
    } else {
#pragma unroll
      for (int w = 0; w < VW / 4; ++w) {
        const u32x4 x = *(const u32x4 *)(p + 16 * w);
#pragma unroll
        for (int e = 0; e < 4; ++e) t.v[i][4 * w + e] = x[e];
      }
    }
  }
}

// The operand V^T of output tile t: dimension DT * m + t of the lane's 8 rows (lo: fp32 only).
template <bool F32, int D>
__device__ __forceinline__ void v_operand(const VTile<F32, D> &v, int t, u32x4 &hi, u32x4 &lo) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (F32) {
      uint32_t x, y;
      split2(__builtin_bit_cast(float, v[2 * i][t]), __builtin_bit_cast(float, v[2 * i + 1][t]), x, y);
      hi[i] = x, lo[i] = y;
    } else {
      hi[i] = __builtin_amdgcn_perm(v[2 * i + 1][t / 2], v[2 * i][t / 2], t % 2 ? 0x07060302u : 0x05040100u);
    }
  }
}

// Barrier after this wave's LDS accesses; loads from memory stay in flight.
__device__ __forceinline__ void stage_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// What the drafted rows of an item are: its sequence's lengths and rows.
struct RowsOf {
  const DraftView *q;
  int len, total, t, first;  // cached rows; with the drafted ones; new rows and the first of them
};

// S^T of 16 cached rows (operand k) and NQ x 16 rows of Q.
template <bool F32, int D, int NQ>
__device__ __forceinline__ void score_rows(const u32x4 (&k)[D / 32][F32 ? 2 : 1], const u32x4 (&q)[NQ][D / 32][F32 ? 2 : 1], f32x4 (&s)[NQ]) {
#pragma unroll
  for (int n = 0; n < NQ; ++n) s[n] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int x = 0; x < D / 32; ++x) {
    if constexpr (F32) {
      u32x4 kh, kl;
      split8(__builtin_bit_cast(f32x4, k[x][0]), __builtin_bit_cast(f32x4, k[x][1]), kh, kl);
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        s[n] = mfma16(kl, q[n][x][0], s[n]);
        s[n] = mfma16(kh, q[n][x][1], s[n]);
        s[n] = mfma16(kh, q[n][x][0], s[n]);
      }
    } else {
#pragma unroll
      for (int n = 0; n < NQ; ++n) s[n] = mfma16(k[x][0], q[n][x][0], s[n]);
    }
  }
}

__device__ __forceinline__ uint32_t low_bits(int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1; }

// Which of the rows j .. j + 31 of its cache the i-th new row of the sequence sees, as bits: the cached ones,
// and of the drafted ones those of its mask row, or up to itself.
__device__ __forceinline__ uint32_t seen_rows(const RowsOf &ro, int i, int j) {
  const int x = j - ro.len;  // drafted row of bit 0, negative: a cached one
  uint32_t drafts = low_bits(i - x + 1);
  if (ro.q->mask) {
    const uint32_t *row = ro.q->mask + (int64_t)(ro.first + i) * ro.q->nwords;
    const int w = x >> 5;
    const uint32_t lo = w >= 0 && w < ro.q->nwords ? row[w] : 0u, hi = w + 1 >= 0 && w + 1 < ro.q->nwords ? row[w + 1] : 0u;
    drafts = (uint32_t)(((uint64_t)hi << 32 | lo) >> (x & 31));
  }
  return low_bits(-x) | (drafts & low_bits(ro.total - j));
}

// An edge: a tile of 32 rows from row j that some row of Q may not see in whole (drafted rows, the end).  Scores
// of rows that are not seen become minus infinity.
template <int NQ>
__device__ __forceinline__ void mask_scores(const RowsOf &ro, const int (&tq)[NQ], int j, int h, f32x4 (&s)[2][NQ]) {
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const uint32_t see = seen_rows(ro, tq[n], j) >> (4 * h);
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[u][n][e] = see >> (16 * u + e) & 1 ? s[u][n][e] : -__builtin_inff();
  }
}

// The weights of NT tiles of 32 rows from their scores: raises the running maxima (and rescales sums and O), adds
// to the sums, and leaves P as the operands of the products with V.
template <int D, int NQ, int NT>
__device__ __forceinline__ void weigh(const f32x4 (&s)[2 * NT][NQ], float c, float (&mx)[NQ], float (&sum)[NQ],
                                      f32x4 (&oacc)[NQ][D / 16], u32x4 (&pb)[NT][NQ]) {
  const float inf = __builtin_inff();
  // maxima and exponents in units of 2^x: c = scale log2(e) > 0 goes into the exponent's one FMA
  float tm[NQ];
  bool raise = false;
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    tm[n] = -inf;
#pragma unroll
    for (int u = 0; u < 2 * NT; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) tm[n] = fmaxf(tm[n], s[u][n][e]);
    tm[n] = fmaxf(max4(tm[n]) * c, mx[n]);
    raise = raise || tm[n] > mx[n];
  }
  if (__any(raise)) {
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      const float al = tm[n] == -inf ? 1.f : exp2_fast(mx[n] - tm[n]);
      mx[n] = tm[n];
      sum[n] *= al;
#pragma unroll
      for (int t = 0; t < D / 16; ++t) oacc[n][t] *= al;
    }
  }
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const float base = mx[n] == -inf ? 0.f : mx[n];
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      float p[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        p[e] = exp2_fast(__builtin_fmaf(s[2 * i + (e >> 2)][n][e & 3], c, -base));
        sum[n] += p[e];
      }
      // P is rounded to bf16 for the product, as in the prefill kernels and for fp32 caches too (half a step of each
      // weight, 2^-8 of sum p |v| at most, as much as the result's own rounding; a second part would be a third more
      // products with V in fp32, twice as many in bf16); its sum is taken before
#pragma unroll
      for (int w = 0; w < 4; ++w) pb[i][n][w] = pack_bf16x2(p[2 * w], p[2 * w + 1]);
    }
  }
}

// A value whose bf16 part is infinite or NaN: a zero weight does not silence it.
__device__ __forceinline__ bool is_special(uint32_t bf) { return (bf & 0x7f80u) == 0x7f80u; }

// Bits 15 and 31: whether the word's bf16 halves are special.
__device__ __forceinline__ uint32_t special_halves(uint32_t w) { return ((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u; }

// A word of two bf16 values without its special ones.
__device__ __forceinline__ uint32_t clean_word(uint32_t w) {
  return w & ((is_special(w) ? 0u : 0xffffu) | (is_special(w >> 16) ? 0u : 0xffff0000u));
}

// Takes infinities and NaN out of an edge's V; whether there were any.
template <bool F32, int D>
__device__ __forceinline__ bool clean_values(VTile<F32, D> &v) {
  constexpr int VW = Tile<F32, D>::VW;
  uint32_t bad = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int w = 0; w < VW; ++w) bad |= special_halves(F32 ? pack_bf16x2(__builtin_bit_cast(float, v[i][w]), 0.f) : v[i][w]);
  if (!__any(bad)) return false;
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int w = 0; w < VW; ++w) {
      if constexpr (F32)
        v[i][w] = is_special(pack_bf16x2(__builtin_bit_cast(float, v[i][w]), 0.f)) ? 0u : v[i][w];
      else
        v[i][w] = clean_word(v[i][w]);
    }
  return true;
}

// O^T += V^T P^T over a tile.
template <bool F32, int D, int NQ>
__device__ __forceinline__ void add_values(const VTile<F32, D> &v, const u32x4 (&pb)[NQ], f32x4 (&oacc)[NQ][D / 16]) {
#pragma unroll
  for (int t = 0; t < D / 16; ++t) {
    u32x4 vh, vl;
    v_operand<F32, D>(v, t, vh, vl);
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      if constexpr (F32) oacc[n][t] = mfma16(vl, pb[n], oacc[n][t]);
      oacc[n][t] = mfma16(vh, pb[n], oacc[n][t]);
    }
  }
}

// ---- the work of a workgroup -------------------------------------------------------------------
// Sequences differ in length, and their lengths are known on the device only.  Every workgroup reads all
// lengths and derives the same plan: the pieces of every item (sequence, head, row tile) in groups of 128
// rows, equal to within one, so that all items together make about `slots` pieces.

// Pieces of a sequence of `tiles` groups at `per` groups a piece.
RS_HD int pieces_of(int tiles, int per) { return tiles > per ? (tiles + per - 1) / per : 1; }

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
};

// Rows of keys of sequence b that the kernels walk: cached rows and drafts.
__device__ __forceinline__ int walk_len(const DraftArgs &a, int len, int t) {
  return len + t < a.c.cap ? len + t : a.c.cap;
}

// What a workgroup works on.
struct Item {
  int b, g, rt, piece, npieces, slot0;  // slot0: the item's first slot of pieces
  int len, t, first;                    // rows held, new rows and the first of them
};

// (what lanes agree on, said so: scalar registers, scalar branches)
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ Item uniform(const Item &x) {
  return Item{uniform(x.b), uniform(x.g), uniform(x.rt), uniform(x.piece), uniform(x.npieces), uniform(x.slot0),
              uniform(x.len), uniform(x.t), uniform(x.first)};
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
__device__ __forceinline__ Seq seq_at(const DraftArgs &a, int b) {
  Seq s{RowRange{0, 0}, 0, 0};
  if (b < a.c.nseq) {
    s.r = new_rows(a.q.start, b, a.q.nrows, a.q.max_rows);
    s.len = cache_len(a.c, b);
    if (s.r.count > 0) s.groups = (walk_len(a, s.len, s.r.count) + kGroup - 1) / kGroup;
  }
  return s;
}

// Groups per piece: the same from the lengths alone in every workgroup and in the joining kernel.  first: the
// sequences of the first round of lanes.
__device__ __forceinline__ int plan_groups(const DraftArgs &a, const Seq &first, int lane) {
  if (a.slots == 0) return kMaxN;  // one piece each
  int work = first.groups;  // (at most 65535 sequences of 2048 groups)
  for (int b0 = 64; b0 < a.c.nseq; b0 += 64) work += seq_at(a, b0 + lane).groups;
  work = wave_sum(work);
  // with pieces of at most C = ceil(total / slots) groups an item of n groups has less than n / C + 1 of them:
  // all together at most slots + the number of items, which is what the host counts
  const long long total = (long long)work * a.c.hkv * a.rtiles, groups = (total + a.slots - 1) / a.slots;
  return groups > a.least ? (int)groups : a.least;
}

// The id-th piece overall; false: there are fewer.
__device__ bool find_item(const DraftArgs &a, int id, int lane, Item &it) {
  Seq q = seq_at(a, lane);
  const int groups = plan_groups(a, q, lane), per = a.c.hkv * a.rtiles;
  int base = 0;
  for (int b0 = 0; b0 < a.c.nseq; b0 += 64) {
    if (b0) q = seq_at(a, b0 + lane);
    const int np = q.r.count > 0 ? pieces_of(q.groups, groups) : 0;
    const int s = wave_scan(np * per), all = __builtin_amdgcn_readlane(s, 63);
    if (id < base + all) {
      const int l = __builtin_ctzll(__ballot(id < base + s));
      it.b = b0 + l;
      it.npieces = __builtin_amdgcn_readlane(np, l);
      it.first = __builtin_amdgcn_readlane(q.r.first, l);
      it.t = __builtin_amdgcn_readlane(q.r.count, l);
      it.len = __builtin_amdgcn_readlane(q.len, l);
      it.slot0 = base + __builtin_amdgcn_readlane(s, l) - it.npieces * per;
      const int x = id - it.slot0;  // piece-major: all heads' row tiles of a piece adjacent
      it.piece = x / per;
      const int y = x - it.piece * per;
      it.rt = y / a.c.hkv;
      it.g = y - it.rt * a.c.hkv;
      return true;
    }
    base += all;
  }
  return false;
}

// ---- the end of a piece ---------------------------------------------------------------------------
template <int D>
constexpr int kLd = D + 4;  // a row of O in LDS, padded

// A wave's O, maximum and sum of 16 rows into LDS (so: rows of kLd, sml: max and sum per row).  Lane (m, h) holds
// dimension 16t + 4h + e (TR: V read transposed) or D / 4 h + D / 16 e + t of row m.
template <int D, bool TR>
__device__ __forceinline__ void store_wave(float *so, float *sml, int m, int h, float mx, float sum, const f32x4 (&oacc)[D / 16]) {
  const float z = sum4(sum);
  if (h == 0) {
    sml[2 * m] = mx;
    sml[2 * m + 1] = z;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e)
#pragma unroll
    for (int t = 0; t < D / 16; ++t) so[m * kLd<D> + (TR ? 16 * t + 4 * h + e : h * (D / 4) + e * (D / 16) + t)] = oacc[t][e];
}

// Infinities and NaN of V count only where they are seen: those that clean_values took out of the edge from row j
// are added, one by one, to the wave's O in LDS (so: `rows` rows of Q from row r0 of the item's nr).
template <bool F32, int D, bool SEL>
__device__ __forceinline__ void add_special(const CacheView &c, const Item &it, const RowsOf &ro, int j, float *so, int rows, int r0,
                                            int nr, int G, int row_t0, int lane) {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  const TileAt at = tile_at(c, it.b, it.g, j, ro.total);
  for (int x = 0; x <= at.last; ++x)
    for (int d = lane; d < D; d += 64) {
      const float v = F32 ? ((const float *)(at.v + x * c.sv_t))[d] : (float)((const bf16 *)(at.v + x * c.sv_t))[d];
      const uint32_t hi = pack_bf16x2(v, 0.f);
      if (!is_special(hi)) continue;
      for (int r = 0; r < rows && r0 + r < nr; ++r)
        if (seen_rows(ro, SEL ? row_t0 : (r0 + r) / G, j) >> x & 1) so[r * kLd<D> + d] += __builtin_bit_cast(float, hi << 16);
    }
}

// Joins KW parts of `rows` rows each (part k at so + k rows kLd) and writes them: as the result where the item
// has one piece, else as the piece `slot`.
template <int D, int KW, int NT, bool SEL>
__device__ __forceinline__ void join_waves(const DraftArgs &a, const Item &it, const float *so, const float *sml, int rows, int r0,
                                           int nr, int G, int row_t0, int slot) {
  for (int x = threadIdx.x; x < rows * (D / 4); x += NT) {
    const int r = x / (D / 4), o4 = x % (D / 4) * 4;
    if (r0 + r >= nr) continue;
    float M = -__builtin_inff(), z = 0.f;
#pragma unroll
    for (int k = 0; k < KW; ++k) M = fmaxf(M, sml[(k * rows + r) * 2]);
    const float base = M == -__builtin_inff() ? 0.f : M;
    f32x4 v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < KW; ++k) {
      const float m = sml[(k * rows + r) * 2], w = exp2_fast(m - base);
      z += w * sml[(k * rows + r) * 2 + 1];
      const f32x4 p = *(const f32x4 *)&so[(k * rows + r) * kLd<D> + o4];
      if (m != -__builtin_inff())
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += w * p[e];
    }
    if (it.npieces == 1) {
      const int t = SEL ? row_t0 : (r0 + r) / G, hh = it.g * G + (SEL ? r0 + r : r0 + r - t * G);
      const float inv = z > 0.f ? 1.f / z : z == 0.f ? 0.f : z;
      u32x2 w2;
      w2[0] = pack_bf16x2(v[0] * inv, v[1] * inv);
      w2[1] = pack_bf16x2(v[2] * inv, v[3] * inv);
      *(u32x2 *)(a.o + ((it.first + t) * a.so_t + hh * a.so_h + o4) * 2) = w2;
      if (a.lse && o4 == 0)
        a.lse[(int64_t)hh * a.q.nrows + it.first + t] = z == 0.f ? -__builtin_inff() : (M + __builtin_amdgcn_logf(z)) * kLn2;
    } else {
      *(f32x4 *)(a.po + ((int64_t)slot * a.trows + r) * D + o4) = v;
      if (o4 == 0) {
        float *ml = a.pml + ((int64_t)slot * a.trows + r) * 2;
        ml[0] = M;
        ml[1] = z;
      }
    }
  }
}

// NQ: 16-row tiles of Q per wave; W: waves (8 only where every item is one piece).
template <bool F32, int D, int NQ, bool SEL, int W = kWaves>
__global__ __launch_bounds__(64 * W, W > kWaves || (D == 128 && (F32 || NQ > 1)) ? 1 : 2) void draft_kernel(const DraftArgs a) {
  using T = Tile<F32, D>;
  constexpr int KC = T::KC, DT = T::DT, E = F32 ? 4 : 2, QP = F32 ? 2 : 1;
  __shared__ float so[W * 16 * NQ * kLd<D>], sml[W * 16 * NQ * 2];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int m = lane & 15, h = lane >> 4;
  Item it;
  int row_t0 = 0;  // with a list: the new row of the item
  if constexpr (SEL) {
    const int r = blockIdx.x / a.pieces;
    it.g = blockIdx.y % a.c.hkv;
    it.rt = blockIdx.y / a.c.hkv;
    it.piece = blockIdx.x - r * a.pieces;
    it.npieces = a.pieces;
    it.b = -1;
    for (int b0 = 0; b0 < a.c.nseq && it.b < 0; b0 += 64) {
      const Seq q = seq_at(a, b0 + lane);
      const unsigned long long hit = __ballot(r >= q.r.first && r < q.r.first + q.r.count);
      if (hit) {
        const int l = __builtin_ctzll(hit);
        it.b = b0 + l;
        it.first = __builtin_amdgcn_readlane(q.r.first, l);
        it.t = __builtin_amdgcn_readlane(q.r.count, l);
        it.len = __builtin_amdgcn_readlane(q.len, l);
      }
    }
    if (it.b < 0) return;  // a row of no sequence
    row_t0 = r - it.first;
    it.slot0 = ((r * a.rtiles + it.rt) * a.c.hkv + it.g) * a.pieces;
  } else {
    if (!find_item(a, blockIdx.x, lane, it)) return;
  }
  it = uniform(it);
  row_t0 = uniform(row_t0);
  const CacheView &c = a.c;
  const int len = it.len;
  const int G = a.q.hq / c.hkv, nr = SEL ? G : G * it.t;  // rows of this sequence (and token) and head
  const int r0 = it.rt * 16 * NQ;
  if (r0 >= nr) return;
  // the walk: rows [0, total), or the selected blocks' rows and then those behind the last complete block
  const int total = walk_len(a, len, it.t), full = len >> 6;
  const int nblk = SEL ? (a.nsel < full ? a.nsel : full) : 0;
  const int steps = SEL ? nblk * 64 + (total - full * 64) : total;
  const int ngroups = (steps + kGroup - 1) / kGroup;
  const int g0 = (int)((long long)ngroups * it.piece / it.npieces), g1 = (int)((long long)ngroups * (it.piece + 1) / it.npieces);
  const int32_t *list = SEL ? a.list + ((int64_t)(it.first + row_t0) * c.hkv + it.g) * a.nsel : nullptr;

  // Q: rows beyond the last are read as the last and not stored
  u32x4 q[NQ][KC][QP];
  int tq[NQ];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    int r = r0 + 16 * n + m;
    r = r < nr ? r : nr - 1;
    tq[n] = SEL ? row_t0 : r / G;
    const int hh = it.g * G + (SEL ? r : r - tq[n] * G);
    const char *p = (const char *)a.q.q + ((it.first + tq[n]) * a.q.sq_t + hh * a.q.sq_h) * E + h * 8 * E;
#pragma unroll
    for (int x = 0; x < KC; ++x) {
      if constexpr (F32)
        split8(*(const f32x4 *)(p + x * 128), *(const f32x4 *)(p + x * 128 + 16), q[n][x][0], q[n][x][1]);
      else
        q[n][x][0] = *(const u32x4 *)(p + x * 64);
    }
  }

  f32x4 oacc[NQ][DT];
  float mx[NQ], sum[NQ];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    mx[n] = -__builtin_inff();
    sum[n] = 0.f;
#pragma unroll
    for (int t = 0; t < DT; ++t) oacc[n][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  // first row of the tile at step s of the walk
  auto row_of = [&](int s) {
    if constexpr (SEL) {
      if (s < nblk * 64) return uload(list, s >> 6) * 64 + (s & 63);
      return full * 64 + s - nblk * 64;
    } else {
      return s;
    }
  };
  auto place = [&](int s, int &j) {
    j = __builtin_amdgcn_readfirstlane(row_of(s));
    return tile_at(c, it.b, it.g, j, total);
  };

  const RowsOf ro{&a.q, len, total, it.t, it.first};
  bool special = false;  // an edge held infinities or NaN
  auto scores = [&](const T &kv, f32x4 (&sc)[2][NQ]) {
#pragma unroll
    for (int u = 0; u < 2; ++u) score_rows<F32, D, NQ>(kv.k[u], q, sc[u]);
  };
  auto use = [&](T &kv, int j, f32x4 (&sc)[2][NQ]) {
    if (j + kTile > len) {
      mask_scores<NQ>(ro, tq, j, h, sc);
      special = clean_values<F32, D>(kv.v) || special;
    }
    u32x4 pb[1][NQ];
    weigh<D, NQ, 1>(sc, a.q.c, mx, sum, oacc, pb);
    add_values<F32, D, NQ>(kv.v, pb[0], oacc);
  };
  auto compute = [&](T &kv, const TileAt &at, int j) {
    if (!at.ok) return;  // no page: nobody sees these rows
    f32x4 sc[2][NQ];
    scores(kv, sc);
    use(kv, j, sc);
  };

  const int s_end = g1 * kGroup < steps ? g1 * kGroup : steps;
  int s = g0 * kGroup + wave * kTile;
  if constexpr (F32 && (D == 128 || NQ > 1)) {
    // two tiles do not fit the registers: the next K is in flight while V is used, and the other way round (16
    // sequences of 16000 rows, 8 heads of 128: one token 410 us, eight 495, at 5.1 and 4.2 TB/s; with two tiles, part of
    // them in scratch, 689 and 1507)
    if (s < s_end) {
      T t;
      int j, jn = 0;
      TileAt at = place(s, j), an{};
      load_k<F32, D>(t, at, c.sk_t, m, h);
      load_v<F32, D>(t, at, c.sv_t, m, h);
      while (true) {
        s += W * kTile;
        const bool more = s < s_end;
        if (more) an = place(s, jn);
        f32x4 sc[2][NQ];
        scores(t, sc);
        if (more) load_k<F32, D>(t, an, c.sk_t, m, h);
        if (at.ok) use(t, j, sc);
        if (!more) break;
        load_v<F32, D>(t, an, c.sv_t, m, h);
        at = an, j = jn;
      }
    }
  } else if (s < s_end) {
    // two tiles take turns: one is in flight while the other is used
    T ta, tb;
    int ja, jb = 0;
    TileAt aa = place(s, ja), ab{};
    load_k<F32, D>(ta, aa, c.sk_t, m, h);
    load_v<F32, D>(ta, aa, c.sv_t, m, h);
    while (true) {
      s += W * kTile;
      const bool more = s < s_end;
      if (more) {
        ab = place(s, jb);
        load_k<F32, D>(tb, ab, c.sk_t, m, h);
        load_v<F32, D>(tb, ab, c.sv_t, m, h);
      }
      compute(ta, aa, ja);
      if (!more) break;
      s += W * kTile;
      const bool again = s < s_end;
      if (again) {
        aa = place(s, ja);
        load_k<F32, D>(ta, aa, c.sk_t, m, h);
        load_v<F32, D>(ta, aa, c.sv_t, m, h);
      }
      compute(tb, ab, jb);
      if (!again) break;
    }
  }

  // join the waves: lane (m, h) holds dimensions [D / 4 h, D / 4 (h + 1)) of row m
#pragma unroll
  for (int n = 0; n < NQ; ++n)
    store_wave<D, false>(&so[(wave * NQ + n) * 16 * kLd<D>], &sml[(wave * NQ + n) * 32], m, h, mx[n], sum[n], oacc[n]);
  if (special)
    for (s = g0 * kGroup + wave * kTile; s < s_end; s += W * kTile) {
      const int j = uniform(row_of(s));
      if (j + kTile > len && tile_at(c, it.b, it.g, j, total).ok)
        add_special<F32, D, SEL>(c, it, ro, j, &so[wave * NQ * 16 * kLd<D>], 16 * NQ, r0, nr, G, row_t0, lane);
    }
  __syncthreads();
  const int slot = SEL ? it.slot0 + it.piece : it.slot0 + it.piece * (c.hkv * a.rtiles) + it.rt * c.hkv + it.g;
  join_waves<D, W, 64 * W, SEL>(a, it, so, sml, 16 * NQ, r0, nr, G, row_t0, slot);
}

// Many rows (a tree: more than 32 per head).  Streaming K and V into each wave's registers would read them once
// per 32 rows; here NW waves share a stage in LDS: NW / KW groups of 32 rows of Q (64, 128 or 256 rows per workgroup),
// KW parts of the stage, one or two tiles of 32 rows per wave and stage.  A stage travels through registers (the
// next one is in flight meanwhile), is written to one of two buffers and read after one barrier.  The 16-byte
// chunks of a row are permuted by an XOR with the row, so that the reads spread over all banks; V is read
// transposed (ds_read_b64_tr_b16).  At 256 rows, per wave and 64 rows of the cache: 64 v_mfma of 16 cycles, 32
// v_exp of 16 and about 190 other vector instructions of 4; LDS passes 32 KB to each wave.
// A stage's barrier keeps its waves in step, so that they wait for the matrix unit together and then for the vector
// unit.  With four waves, two workgroups (d = 64: three) share a CU and fill each other's gaps (16 sequences of 16000
// rows, 8 heads: 64 rows of Q 205 us, 0.67 of what eight waves take; 96 rows 227, 0.60; 256 rows of d = 64 233, 0.59, in
// fp32 461, 0.62).  With d = 128 and 256 rows they would read K and V twice; eight waves stay ahead there (61 rows x 4
// heads per group over 128K rows: 188 us, 0.70 of 1.22 PFLOP/s; 1.07 times that in two tiles of 128).  64 rows per wave
// halve the LDS traffic, but O then lives in accumulation registers and is copied at every rescale test: 2.1 times.

// Chunks of K: 16 rows' equal chunks in different banks; of V: the chunk pairs 2t, 2t + 1 of 8 rows.
template <int D>
__device__ __forceinline__ int chunk_xor(int r) {
  return D == 128 ? (r & 7) << 1 | (r >> 3 & 1) : (r >> 1 & 3) << 1 | (r >> 3 & 1);
}

// F32: values are split into their bf16 parts as they enter LDS, a plane each.
template <bool F32, int D, int KW, int NW>
__global__ __launch_bounds__(64 * NW, D == 64 ? 3 : 2) void draft_wide_kernel(const DraftArgs a) {
  constexpr int NT = KW == 2 || F32 ? 1 : 2;                 // tiles of 32 rows per wave and stage
  constexpr int NQ = 2, RW = NW / KW, SR = 32 * NT * KW;  // SR: rows of a stage
  static_assert(64 % SR == 0, "a stage lies in one page");
  constexpr int E = F32 ? 4 : 2, QP = F32 ? 2 : 1;                // bytes of a value; bf16 parts of it
  constexpr int KC = D / 32, DT = D / 16, CPR = D * E / 16, RPI = 64 / CPR;
  constexpr int NI = 2 * SR / RPI / NW;  // 16-byte loads per lane and stage, K before V
  constexpr int kPlane = SR * D * 2, kBuf = 2 * QP * kPlane;  // a bf16 part of K or V of a stage; all of them
  constexpr int kJoin = NW * 16 * NQ * (kLd<D> + 2) * 4, kLds = 2 * kBuf > kJoin ? 2 * kBuf : kJoin;
  __shared__ __align__(16) char lds[kLds];
  __shared__ int odd;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int m = lane & 15, h = lane >> 4, wk = wave % KW, wr = wave / KW;
  Item it;
  if (!find_item(a, blockIdx.x, lane, it)) return;
  it = uniform(it);
  const CacheView &c = a.c;
  const int len = it.len;
  const int G = a.q.hq / c.hkv, nr = G * it.t, r0 = it.rt * 32 * RW;
  if (r0 >= nr) return;
  const int total = walk_len(a, len, it.t), ngroups = (total + kGroup - 1) / kGroup;
  const int g0 = (int)((long long)ngroups * it.piece / it.npieces), g1 = (int)((long long)ngroups * (it.piece + 1) / it.npieces);
  const int j0 = g0 * kGroup, j1 = g1 * kGroup < total ? g1 * kGroup : total;
  const int nst = (j1 - j0 + SR - 1) / SR;

  u32x4 q[NQ][KC][QP];
  int tq[NQ];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    int r = r0 + 32 * wr + 16 * n + m;
    r = r < nr ? r : nr - 1;
    tq[n] = r / G;
    const char *p = (const char *)a.q.q + ((it.first + tq[n]) * a.q.sq_t + (it.g * G + r - tq[n] * G) * a.q.sq_h) * E + h * 8 * E;
#pragma unroll
    for (int x = 0; x < KC; ++x) {
      if constexpr (F32)
        split8(*(const f32x4 *)(p + x * 128), *(const f32x4 *)(p + x * 128 + 16), q[n][x][0], q[n][x][1]);
      else
        q[n][x][0] = *(const u32x4 *)(p + x * 64);
    }
  }
  f32x4 oacc[NQ][DT];
  float mx[NQ], sum[NQ];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    mx[n] = -__builtin_inff();
    sum[n] = 0.f;
#pragma unroll
    for (int t = 0; t < DT; ++t) oacc[n][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const bool idle = r0 + 32 * wr >= nr;  // a wave without rows only carries its part of the stages

  // Load i of a stage: RPI rows of K or V.  The table's entry is read a stage ahead of its use.
  const int lr = lane / CPR, lc = lane % CPR;
  u32x4 st[NI];
  bool okst;
  int entry;
  auto first_row = [&](int stage) {  // (behind the end: the last row)
    const int j = j0 + stage * SR;
    return __builtin_amdgcn_readfirstlane(j < total ? j : total - 1);
  };
  auto look = [&](int stage) {
    const int p = page_of(c, first_row(stage));
    entry = c.table ? uload(c.table, (int64_t)it.b * c.max_pages + p) : it.b * c.max_pages + p;
  };
  int off[NI];
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int w = (i * NW + wave) % (SR / RPI), isv = (i * NW + wave) / (SR / RPI);
    off[i] = (w * RPI + lr) * (int)(isv ? c.sv_t : c.sk_t) + 16 * lc;
  }
  const char *kg = c.k + it.g * c.sk_h, *vg = c.v + it.g * c.sv_h;
  auto fetch = [&](int stage, u32x4 (&x)[NI], bool &ok) {
    const int j = first_row(stage), id = checked_page(c, entry), in = j - page_of(c, j) * c.page;
    ok = id >= 0;
    const char *kb = kg + (ok ? id * c.sk_p + in * c.sk_t : 0), *vb = vg + (ok ? id * c.sv_p + in * c.sv_t : 0);
    const int most = ok ? total - 1 - j : 0;  // last row that may be read
    look(stage + 1);
    if (most >= SR - 1) {
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const int isv = (i * NW + wave) / (SR / RPI);
        x[i] = *(const u32x4 *)((isv ? vb : kb) + off[i]);
      }
    } else {  // rows behind the end are read as the last, all without a page as its row 0
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const int w = (i * NW + wave) % (SR / RPI), isv = (i * NW + wave) / (SR / RPI), r = w * RPI + lr;
        x[i] = *(const u32x4 *)((isv ? vb : kb) + (r < most ? r : most) * (int)(isv ? c.sv_t : c.sk_t) + 16 * lc);
      }
    }
  };
  // edge: V without infinities and NaN, which `odd` (LDS) then tells of
  auto put = [&](auto edge, char *buf, u32x4 (&x)[NI]) {
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int w = (i * NW + wave) % (SR / RPI), isv = (i * NW + wave) / (SR / RPI), r = w * RPI + lr;
      char *row = buf + isv * QP * kPlane + r * (D * 2);
      if constexpr (decltype(edge)::value)
        if (isv) {
          uint32_t bad = 0;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t y = x[i][e];
            bad |= special_halves(F32 ? pack_bf16x2(__builtin_bit_cast(float, y), 0.f) : y);
          }
          if (__any(bad)) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t y = x[i][e];
              x[i][e] = F32 ? (is_special(pack_bf16x2(__builtin_bit_cast(float, y), 0.f)) ? 0u : y) : clean_word(y);
            }
            odd = 1;
          }
        }
      if constexpr (F32) {
        const f32x4 f = __builtin_bit_cast(f32x4, x[i]);
        uint32_t h0, l0, h1, l1;
        split2(f[0], f[1], h0, l0);
        split2(f[2], f[3], h1, l1);
        row += ((lc >> 1 ^ chunk_xor<D>(r)) << 4) + (lc & 1) * 8;
        *(u32x2 *)row = u32x2{h0, h1};
        *(u32x2 *)(row + kPlane) = u32x2{l0, l1};
      } else {
        *(u32x4 *)(row + ((lc ^ chunk_xor<D>(r)) << 4)) = x[i];
      }
    }
  };
  const RowsOf ro{&a.q, len, total, it.t, it.first};
  // S^T of 16 rows from row r0 of the stage
  auto scores = [&](const char *buf, int r0, f32x4 (&s)[NQ]) {
    const char *row = buf + (r0 + m) * (D * 2);
    u32x4 k[KC][QP];
#pragma unroll
    for (int x = 0; x < KC; ++x)
#pragma unroll
      for (int y = 0; y < QP; ++y) k[x][y] = *(const u32x4 *)(row + y * kPlane + (((4 * x + h) ^ chunk_xor<D>(m)) << 4));
    if constexpr (F32) {
#pragma unroll
      for (int n = 0; n < NQ; ++n) s[n] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int x = 0; x < KC; ++x)
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
          s[n] = mfma16(k[x][1], q[n][x][0], s[n]);
          s[n] = mfma16(k[x][0], q[n][x][1], s[n]);
          s[n] = mfma16(k[x][0], q[n][x][0], s[n]);
        }
    } else {
      score_rows<false, D, NQ>(k, q, s);
    }
  };
  // O^T += V^T P^T over 32 rows: lane (m, h) of a transposing read passes 4 dimensions of row 4h + m / 4 and gets
  // dimension m of rows 4h .. 4h + 3; two of them are the operand of output tile t (dimensions 16t ..)
  typedef short v4i16 __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) v4i16 lds4;
  const int vr = 4 * h + (m >> 2), vf = chunk_xor<D>(vr), vf1 = chunk_xor<D>(vr + 16);
  auto values = [&](const char *buf, int r0, const u32x4 (&p)[NQ]) {
    const char *x0 = buf + QP * kPlane + (r0 + vr) * (D * 2) + (m & 1) * 8, *x1 = x0 + 16 * (D * 2);
#pragma unroll
    for (int t = 0; t < DT; ++t) {
      const int c2 = 2 * t + (m >> 1 & 1);
      u32x4 v[QP];
#pragma unroll
      for (int y = 0; y < QP; ++y) {
        const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(x0 + y * kPlane + ((c2 ^ vf) << 4))));
        const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(x1 + y * kPlane + ((c2 ^ vf1) << 4))));
        v[y] = u32x4{lo[0], lo[1], hi[0], hi[1]};
      }
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        if constexpr (F32) oacc[n][t] = mfma16(v[QP - 1], p[n], oacc[n][t]);
        oacc[n][t] = mfma16(v[0], p[n], oacc[n][t]);
      }
    }
  };

  // stages of cached rows alone, which every row sees (and none what has no page)
  const int nplain = len < j1 ? (len > j0 ? (len - j0) / SR : 0) : (j1 - j0) / SR, wr0 = wk * NT * 32;
  look(0);
  fetch(0, st, okst);
  for (int s = 0; s < nplain; ++s) {
    char *buf = lds + (s & 1) * kBuf;
    put(std::false_type{}, buf, st);
    const bool ok = okst;
    fetch(s + 1, st, okst);  // (behind the last: its last row)
    stage_barrier();
    if (idle || !ok) continue;
    f32x4 sc[2 * NT][NQ];
    __builtin_amdgcn_s_setprio(1);  // matrix instructions first: the other wave's exponents fill their gaps (4 % less)
    u32x4 pb[NT][NQ];
#pragma unroll
    for (int u = 0; u < 2 * NT; ++u) scores(buf, wr0 + 16 * u, sc[u]);
    __builtin_amdgcn_s_setprio(0);
    weigh<D, NQ, NT>(sc, a.q.c, mx, sum, oacc, pb);
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int i = 0; i < NT; ++i) values(buf, wr0 + 32 * i, pb[i]);
    __builtin_amdgcn_s_setprio(0);
  }
  // the few stages of drafted rows and the end
  if (tid == 0) odd = 0;
  for (int s = nplain; s < nst; ++s) {
    __syncthreads();
    put(std::true_type{}, lds, st);
    const bool ok = okst;
    fetch(s + 1, st, okst);
    stage_barrier();
    if (idle || !ok) continue;
    for (int i = 0; i < NT; ++i) {
      const int r = wr0 + 32 * i, j = j0 + s * SR + r;
      if (j >= j1) break;
      f32x4 sc[2][NQ];
      u32x4 pb[1][NQ];
#pragma unroll
      for (int u = 0; u < 2; ++u) scores(lds, r + 16 * u, sc[u]);
      mask_scores<NQ>(ro, tq, j, h, sc);
      weigh<D, NQ, 1>(sc, a.q.c, mx, sum, oacc, pb);
      values(lds, r, pb[0]);
    }
  }
  __syncthreads();
  const bool special = odd;
  const int slot = it.slot0 + it.piece * (c.hkv * a.rtiles) + it.rt * c.hkv + it.g;
  if (KW == 1 && !special) {
    // a wave's rows are its own: lane (m, h) writes dimensions 16t + 4h .. + 3 of row m
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      const float z = sum4(sum[n]);
      const int r = 32 * wr + 16 * n + m;
      if (r0 + r >= nr) continue;
      if (it.npieces == 1) {
        const int t = tq[n], hh = it.g * G + r0 + r - t * G;
        const float inv = z > 0.f ? 1.f / z : z == 0.f ? 0.f : z;
        char *o = a.o + ((it.first + t) * a.so_t + hh * a.so_h + 4 * h) * 2;
#pragma unroll
        for (int x = 0; x < DT; ++x)
          *(u32x2 *)(o + 32 * x) = u32x2{pack_bf16x2(oacc[n][x][0] * inv, oacc[n][x][1] * inv), pack_bf16x2(oacc[n][x][2] * inv, oacc[n][x][3] * inv)};
        if (a.lse && h == 0)
          a.lse[(int64_t)hh * a.q.nrows + it.first + t] = z == 0.f ? -__builtin_inff() : (mx[n] + __builtin_amdgcn_logf(z)) * kLn2;
      } else {
        float *o = a.po + ((int64_t)slot * a.trows + r) * D + 4 * h;
#pragma unroll
        for (int x = 0; x < DT; ++x) *(f32x4 *)(o + 16 * x) = oacc[n][x];
        if (h == 0) {
          float *ml = a.pml + ((int64_t)slot * a.trows + r) * 2;
          ml[0] = mx[n];
          ml[1] = z;
        }
      }
    }
    return;
  }
  float *so = (float *)lds, *sml = so + NW * 16 * NQ * kLd<D>;  // part wk of row group wr at rows 32 wr
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const int at = wk * 32 * RW + 32 * wr + 16 * n;
    store_wave<D, true>(so + at * kLd<D>, sml + at * 2, m, h, mx[n], sum[n], oacc[n]);
  }
  if (special)
    for (int s = nplain; s < nst; ++s)
      for (int i = 0; i < NT; ++i) {
        const int j = j0 + s * SR + wr0 + 32 * i;
        if (j < j1 && tile_at(c, it.b, it.g, j, total).ok)
          add_special<F32, D, false>(c, it, ro, j, so + (wk * 32 * RW + 32 * wr) * kLd<D>, 32, r0 + 32 * wr, nr, G, 0, lane);
      }
  __syncthreads();
  join_waves<D, KW, 64 * NW, false>(a, it, so, sml, 32 * RW, r0, nr, G, 0, slot);
}

// Joins the pieces of every item: WV waves per new row and head (all four of a workgroup, or one where there are so
// many rows that the chip is full of them).  Every wave reads all maxima and sums (a lane per piece), so that each
// knows its weights before its share of the O parts arrives; LDS joins the waves.
template <int D, bool SEL, int WV>
__global__ __launch_bounds__(256) void draft_join_kernel(const DraftArgs a) {
  __shared__ float so[kWaves][D];
  constexpr int PL = D / 64;  // dimensions per lane
  typedef float fv __attribute__((ext_vector_type(PL)));
  const int tid = threadIdx.x, lane = tid & 63, wv = uniform(tid >> 6), wave = WV == 1 ? 0 : wv;
  const CacheView &c = a.c;
  const int G = a.q.hq / c.hkv, r = blockIdx.x, hh = WV == 1 ? blockIdx.y * kWaves + wv : blockIdx.y, g = hh / G;
  if (hh >= a.q.hq) return;
  int slot, np, stride, row;
  bool mine = true;
  if constexpr (SEL) {
    const int rr = hh - g * G, rt = rr / a.trows;
    row = rr - rt * a.trows;
    slot = ((r * a.rtiles + rt) * c.hkv + g) * a.pieces;
    np = a.pieces;
    stride = 1;
  } else {
    Seq q = seq_at(a, lane);
    const int groups = plan_groups(a, q, lane), per = c.hkv * a.rtiles;
    int base = 0, b = -1, first = 0;
    np = 0;
    for (int b0 = 0; b0 < c.nseq && b < 0; b0 += 64) {
      if (b0) q = seq_at(a, b0 + lane);
      const int k = q.r.count > 0 ? pieces_of(q.groups, groups) : 0;
      const int s = wave_scan(k * per);
      const unsigned long long hit = __ballot(r >= q.r.first && r < q.r.first + q.r.count);
      if (hit) {
        const int l = __builtin_ctzll(hit);
        b = b0 + l;
        first = __builtin_amdgcn_readlane(q.r.first, l);
        np = __builtin_amdgcn_readlane(k, l);
        base += __builtin_amdgcn_readlane(s, l) - np * per;
      } else {
        base += __builtin_amdgcn_readlane(s, 63);
      }
    }
    if (b < 0 || np <= 1) return;
    const int rr = (r - first) * G + hh - g * G, rt = rr / a.trows;
    row = rr - rt * a.trows;
    slot = base + rt * c.hkv + g;
    stride = per;
  }
  slot = uniform(slot), np = uniform(np), row = uniform(row);
  const float *po = a.po + ((int64_t)slot * a.trows + row) * D + lane * PL, *pml = a.pml + ((int64_t)slot * a.trows + row) * 2;
  const int64_t step = (int64_t)stride * a.trows;
  float M = -__builtin_inff(), z = 0.f;
  for (int k0 = 0; k0 < np; k0 += 64) {
    const int k = k0 + lane;
    float m = -__builtin_inff(), s = 0.f;
    if (k < np) m = pml[k * step * 2], s = pml[k * step * 2 + 1];
    const float m2 = wave_max(fmaxf(M, m));
    const float base = m2 == -__builtin_inff() ? 0.f : m2;
    s = wave_total(k < np ? s * exp2_fast(m - base) : 0.f);
    z = (z == 0.f ? 0.f : z * exp2_fast(M - base)) + s;
    M = m2;
  }
  const float base = M == -__builtin_inff() ? 0.f : M;
  fv v{};
  constexpr int kAhead = 8;
  for (int k0 = wave; k0 < np; k0 += WV * kAhead) {
    fv p[kAhead];
    float m[kAhead];
#pragma unroll
    for (int x = 0; x < kAhead; ++x) {
      const int k = k0 + x * WV < np ? k0 + x * WV : k0;
      p[x] = *(const fv *)(po + k * step * D);
      m[x] = pml[k * step * 2];
    }
#pragma unroll
    for (int x = 0; x < kAhead; ++x)
      if (k0 + x * WV < np && m[x] != -__builtin_inff()) v += p[x] * exp2_fast(m[x] - base);
  }
  if constexpr (SEL) mine = seq_of_row(c, a.q, r, lane) >= 0;
  *(fv *)&so[wv][lane * PL] = v;
  int at = tid;
  if constexpr (WV == 1) {
    at = lane;
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  } else {
    __syncthreads();
  }
  if (at >= D / 2 || !mine) return;
  float x = 0.f, y = 0.f;
#pragma unroll
  for (int k = 0; k < WV; ++k) {
    x += so[WV == 1 ? wv : k][2 * at];
    y += so[WV == 1 ? wv : k][2 * at + 1];
  }
  const float inv = z > 0.f ? 1.f / z : z == 0.f ? 0.f : z;
  *(uint32_t *)(a.o + (r * a.so_t + hh * a.so_h + 2 * at) * 2) = pack_bf16x2(x * inv, y * inv);
  if (a.lse && at == 0)
    a.lse[(int64_t)hh * a.q.nrows + r] = z == 0.f ? -__builtin_inff() : (M + __builtin_amdgcn_logf(z)) * kLn2;
}

// ---- scores and selection of blocks ------------------------------------------------------------
// score(c) = max over the heads h of g of q_h . mean_c, in fp64.  A product has 16 bits with bf16 q and 32 with fp32 q, a
// sum of 128 of them 7 more: of fp64's 53 that leaves 30 and 14, so sums of terms that lie within 2^30 (2^14) of each
// other are exact and the selection does not depend on their order; others are rounded to 53 bits in the order
// of the instructions, which is always the same.  The products are v_mfma_f64_16x16x4: 16 rows of a
// sequence (tokens and heads) against 16 blocks per wave, both operands straight from memory (a lane holds a
// quarter of a row: the contraction may run in any order), the means converted once for all rows.  The
// vector ALU has the same fp64 rate without padding rows to 16, but its q operands come through LDS: 80 rows x 8
// heads over 36K rows of cache took 114 us so, 25 us with the matrix instructions; what is left is
// latency.
struct SelectArgs {
  CacheView c;
  DraftView q;
  double *score;  // [nrows * hkv][fcap]
  int32_t *list;  // [nrows * hkv][nsel]
  int fcap, nsel, nsink, nlocal;
};

// Rows of a 16-row tile: whole tokens of G heads, or 16 heads of one token.
RS_HD int score_tokens(int G) { return G < 16 ? 16 / G : 1; }

template <bool F32, int D>
__global__ __launch_bounds__(256, 2) void score_kernel(const SelectArgs a) {
  constexpr int DL = D / 4, E = F32 ? 4 : 2;  // dimensions per lane: lane (m, h) holds [DL h, DL (h + 1)) of a row
  __shared__ double ss[kWaves][16][17];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane & 15, h = lane >> 4;
  const int g = blockIdx.y, b = blockIdx.z, c0 = (blockIdx.x * kWaves + wave) * 16;
  const RowRange rr = new_rows(a.q.start, b, a.q.nrows, a.q.max_rows);
  const int F = cache_len(a.c, b) >> 6;
  if (c0 >= F || F <= a.nsel) return;  // (all blocks are taken: no scores)
  const int G = a.q.hq / a.c.hkv, tp = score_tokens(G), parts = (G + 15) >> 4;
  // means of 16 blocks, lane m the m-th; blocks behind the last are read as the last
  const int blk = c0 + m < F ? c0 + m : F - 1, p = page_of(a.c, blk * 64), id = page_id(a.c, b, p);
  double km[DL];
  {
    const u32x4 *x = (const u32x4 *)((const bf16 *)a.c.kmean + mean_offset(a.c, id >= 0 ? id : 0, p, id >= 0 ? blk : p * (a.c.page >> 6), g, D) + DL * h);
#pragma unroll
    for (int i = 0; i < DL / 8; ++i) {
      u32x4 w = x[i];
      if (id < 0) w = u32x4{0, 0, 0, 0};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        km[8 * i + 2 * e] = (double)__builtin_bit_cast(float, w[e] << 16);
        km[8 * i + 2 * e + 1] = (double)__builtin_bit_cast(float, w[e] & 0xffff0000u);
      }
    }
  }
  typedef double f64x4 __attribute__((ext_vector_type(4)));
  for (int t0 = 0; t0 < rr.count; t0 += tp) {
    double best[4] = {-__builtin_inf(), -__builtin_inf(), -__builtin_inf(), -__builtin_inf()};
    for (int part = 0; part < parts; ++part) {
      // the m-th row: head hh of token t; rows beyond the last are read as the last
      int t = t0, hh = part * 16 + m;
      if (parts == 1) {
        t = t0 + m / G;
        hh = m % G;
        if (m >= tp * G || t >= rr.count) t = rr.count - 1;
      }
      hh = hh < G ? hh : G - 1;
      const char *q = (const char *)a.q.q + ((rr.first + t) * a.q.sq_t + (g * G + hh) * a.q.sq_h + DL * h) * E;
      f64x4 s{0., 0., 0., 0.};
#pragma unroll
      for (int i = 0; i < DL / 8; ++i) {
        float f[8];
        if constexpr (F32) {
          const f32x4 x = *(const f32x4 *)(q + 32 * i), y = *(const f32x4 *)(q + 32 * i + 16);
#pragma unroll
          for (int e = 0; e < 4; ++e) f[e] = x[e], f[4 + e] = y[e];
        } else {
          const u32x4 w = *(const u32x4 *)(q + 16 * i);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            f[2 * e] = __builtin_bit_cast(float, w[e] << 16);
            f[2 * e + 1] = __builtin_bit_cast(float, w[e] & 0xffff0000u);
          }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) s = __builtin_amdgcn_mfma_f64_16x16x4f64((double)f[e], km[8 * i + e], s, 0, 0, 0);
      }
      // lane (m, h) holds rows h, 4 + h, ... of block m; the maximum over a token's heads through LDS
#pragma unroll
      for (int e = 0; e < 4; ++e) ss[wave][4 * e + h][m] = s[e];
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
      const int nh = parts == 1 ? G : G - part * 16 < 16 ? G - part * 16 : 16;
#pragma unroll
      for (int e = 0; e < 4; ++e) {  // tokens h, h + 4, ...
        const int tt = h + 4 * e;
        if (tt < tp)
          for (int x = 0; x < nh; ++x) {
            const double v = ss[wave][tt * G + x][m];
            best[e] = v > best[e] ? v : best[e];
          }
      }
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int tt = h + 4 * e;
      if (tt < tp && t0 + tt < rr.count && c0 + m < F)
        a.score[((int64_t)(rr.first + t0 + tt) * a.c.hkv + g) * a.fcap + c0 + m] = best[e];
    }
  }
}

// The selected blocks of a row and head, ascending: a radix selection over the scores as ordered 64-bit keys
// (11 bits a pass, ended as soon as all of the last digit's blocks stay), then their places by a prefix sum.
__device__ __forceinline__ uint64_t double_key(double f) {
  const uint64_t u = __builtin_bit_cast(uint64_t, f + 0.0);  // -0.0 equals 0.0
  return u >> 63 ? ~u : u | 1ull << 63;
}

constexpr int kSelThreads = 256, kSelPer = kMaxN / 64 / kSelThreads;

__global__ __launch_bounds__(kSelThreads) void select_kernel(const SelectArgs a) {
  constexpr int kBins = 2048;
  __shared__ int hist[kBins], sw[kSelThreads / 64], pick[3];
  const int tid = threadIdx.x, r = blockIdx.x, g = blockIdx.y;
  int F = -1;
  for (int b0 = 0; b0 < a.c.nseq && F < 0; b0 += 64) {
    const int b = b0 + (tid & 63);
    RowRange q{0, 0};
    int len = 0;
    if (b < a.c.nseq) {
      q = new_rows(a.q.start, b, a.q.nrows, a.q.max_rows);
      len = cache_len(a.c, b);
    }
    const unsigned long long hit = __ballot(r >= q.first && r < q.first + q.count);
    if (hit) F = __builtin_amdgcn_readlane(len, __builtin_ctzll(hit)) >> 6;
  }
  if (F < 0) return;  // a row of no sequence
  const int64_t item = (int64_t)r * a.c.hkv + g;
  int32_t *list = a.list + item * a.nsel;
  const int nb = a.nsel < F ? a.nsel : F;
  for (int x = nb + tid; x < a.nsel; x += kSelThreads) list[x] = -1;
  if (F <= a.nsel) {
    for (int x = tid; x < F; x += kSelThreads) list[x] = x;
    return;
  }
  const int per = (F + kSelThreads - 1) / kSelThreads, c0 = tid * per;
  uint64_t key[kSelPer];
#pragma unroll
  for (int x = 0; x < kSelPer; ++x) {
    const int c = c0 + x;
    key[x] = 0;  // (below every key)
    if (x < per && c < F) key[x] = c < a.nsink || c >= F - a.nlocal ? ~0ull : double_key(a.score[item * a.fcap + c]);
  }
  uint64_t prefix = 0, have = 0;
  int need = nb, equal = F, all;
  for (int sh = 53; need < equal; sh -= 11) {
    const int low = sh > 0 ? sh : 0, bins = sh > 0 ? kBins : kBins >> -sh;  // the last digit has 9 bits
    for (int x = tid; x < bins; x += kSelThreads) hist[x] = 0;
    __syncthreads();
#pragma unroll
    for (int x = 0; x < kSelPer; ++x)
      if (x < per && c0 + x < F && (key[x] & have) == prefix) atomicAdd(&hist[(key[x] >> low) & (bins - 1)], 1);
    __syncthreads();
    const int pb = bins / kSelThreads, top = bins - 1 - tid * pb;
    int sum = 0;
    for (int x = 0; x < pb; ++x) sum += hist[top - x];
    int before = block_scan<kSelThreads>(sum, sw, &all);
    if (before < need && before + sum >= need) {
      int x = top;
      while (before + hist[x] < need) before += hist[x--];
      pick[0] = x;
      pick[1] = need - before;
      pick[2] = hist[x];
    }
    __syncthreads();
    prefix |= (uint64_t)pick[0] << low;
    have |= (uint64_t)(bins - 1) << low;
    need = pick[1];
    equal = pick[2];
    __syncthreads();
    if (low == 0) break;
  }
  int e = 0, above = 0;
#pragma unroll
  for (int x = 0; x < kSelPer; ++x)
    if (x < per && c0 + x < F) {
      e += (key[x] & have) == prefix;
      above += (key[x] & have) > prefix;
    }
  // blocks before this thread's that equal the border: the first `need` of them stay, so the thread's place
  // is known from both counts
  const int both = block_scan<kSelThreads>(above | e << 16, sw, &all);
  int eq = both >> 16, at = (both & 0xffff) + (eq < need ? eq : need);
#pragma unroll
  for (int x = 0; x < kSelPer; ++x)
    if (x < per && c0 + x < F) {
      const uint64_t k = key[x] & have;
      if (k > prefix || (k == prefix && eq < need)) list[at++] = c0 + x;
      eq += k == prefix;
    }
}

// ---- accumulated weights -------------------------------------------------------------------------
// acc_j += sum over rows r of w_r exp(l_rj - lse_r).  K once, acc in and out once: memory bounds it while a head
// has few rows.  The products are S = Q K^T here, Q as the first operand: lane (m, h) then holds row m of the
// cache and 4 of the 16 rows of Q, so the sum over rows stays in one register per 16 cached rows until two
// exchanges at the end (with S^T, as in the attention, 16 lanes hold each sum apart: 128 exchanges per 128 rows).
// A row of the cache belongs to one wave, so nothing is added in an order that varies.
struct WeightArgs {
  CacheView c;
  DraftView q;
  const float *lse, *row_w, *acc_in;
  float *acc_out;
  int rows;  // cached rows per workgroup
};

// NQ: 16-row tiles of Q kept in registers; 0: more rows than that, 128 at a time in LDS (in the order and parts in
// which the instructions take them), and K once for each of these.  16 sequences of 16000 rows, 8 heads of 128: 64
// rows of Q 129 us in bf16 (158 with Q read from memory for every 64 cached rows, 181 from registers) and 217 in
// fp32 (535; floor 206); 256 rows 291 and 533.
template <bool F32, int D, int NQ>
__global__ __launch_bounds__(256, 2) void weights_kernel(const WeightArgs a) {
  constexpr int KC = D / 32, E = F32 ? 4 : 2, QP = F32 ? 2 : 1, NK = NQ ? NQ : 1;
  constexpr int NU = F32 && (D == 128 || NQ == 0) ? 2 : 4, RW = 16 * NU;  // 16-row pieces of K in a wave's step (registers)
  constexpr int kRowsLds = NQ ? 16 * NQ : 128;  // rows of Q whose factors (and values) LDS holds
  __shared__ float sl[kRowsLds], sw[kRowsLds];
  __shared__ int st[kRowsLds];
  __shared__ u32x4 sq[NQ ? 1 : kRowsLds / 16][KC][QP][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int m = lane & 15, h = lane >> 4, g = blockIdx.y, b = blockIdx.z;
  const CacheView &c = a.c;
  const RowRange rr = new_rows(a.q.start, b, a.q.nrows, a.q.max_rows);
  const int len = cache_len(c, b), total = len + rr.count < c.cap ? len + rr.count : c.cap;
  const int first = blockIdx.x * a.rows;
  if (first >= total || rr.count == 0) return;
  const int G = a.q.hq / c.hkv, nr = G * rr.count;
  const int64_t at = ((int64_t)b * c.hkv + g) * c.cap;

  auto load_q = [&](int r0, u32x4 (&q)[KC][QP]) {
    const int r = r0 + m < nr ? r0 + m : nr - 1, t = r / G, hh = g * G + r - t * G;
    const char *p = (const char *)a.q.q + ((rr.first + t) * a.q.sq_t + hh * a.q.sq_h) * E + h * 8 * E;
#pragma unroll
    for (int x = 0; x < KC; ++x) {
      if constexpr (F32)
        split8(*(const f32x4 *)(p + x * 128), *(const f32x4 *)(p + x * 128 + 16), q[x][0], q[x][1]);
      else
        q[x][0] = *(const u32x4 *)(p + x * 64);
    }
  };
  // 16 cached rows, lane m the m-th: rows behind the end are read as the last, without a page as row 0 of page 0
  auto load_k = [&](int j0, u32x4 (&k)[KC][QP], bool &ok) {
    const int p = page_of(c, j0), id = checked_page(c, c.table ? uload(c.table, (int64_t)b * c.max_pages + p) : b * c.max_pages + p);
    ok = id >= 0;
    const int r = j0 + m < total ? m : total - 1 - j0;
    const char *x = (ok ? c.k + k_offset(c, id, p, j0, g) + r * c.sk_t : c.k + g * c.sk_h) + h * 8 * E;
#pragma unroll
    for (int i = 0; i < KC; ++i)
#pragma unroll
      for (int y = 0; y < QP; ++y) k[i][y] = *(const u32x4 *)(x + i * 32 * E + 16 * y);
  };

  // fp32: the values of 16 rows become their bf16 parts, once for all tiles of Q (one tile: as it uses them)
  auto split = [&](u32x4 (&k)[KC][QP]) {
    if constexpr (F32 && NQ != 1)
#pragma unroll
      for (int i = 0; i < KC; ++i) {
        const f32x4 x = __builtin_bit_cast(f32x4, k[i][0]), y = __builtin_bit_cast(f32x4, k[i][1]);
        split8(x, y, k[i][0], k[i][1]);
      }
  };
  u32x4 q[NK][KC][QP];
  if constexpr (NQ > 0)
#pragma unroll
    for (int n = 0; n < NQ; ++n) load_q(16 * n, q[n]);

  // one tile of 16 rows of Q (factors at r0 of LDS) against 16 cached rows; `plain`: every row counts and
  // sees all of them
  auto add = [&](const u32x4 (&qq)[KC][QP], const u32x4 (&kk)[KC][QP], int r0, int j0, float &sum) {
    f32x4 s{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int x = 0; x < KC; ++x) {
      if constexpr (F32) {
        u32x4 kh = kk[x][0], kl = kk[x][1];
        if constexpr (NQ == 1) split8(__builtin_bit_cast(f32x4, kk[x][0]), __builtin_bit_cast(f32x4, kk[x][1]), kh, kl);
        s = mfma16(qq[x][0], kl, s);
        s = mfma16(qq[x][1], kh, s);
        s = mfma16(qq[x][0], kh, s);
      } else {
        s = mfma16(qq[x][0], kk[x][0], s);
      }
    }
    const f32x4 l2 = *(const f32x4 *)&sl[r0 + 4 * h], w = *(const f32x4 *)&sw[r0 + 4 * h];
    const int i = j0 + m - len;  // drafted row, negative: a cached one
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      bool see = w[e] != 0.f;
      if (j0 + 16 > len) {
        const int t = st[r0 + 4 * h + e];
        if (i >= 0) {
          bool v = i < rr.count && i <= t;
          if (i < rr.count && a.q.mask) v = a.q.mask[(int64_t)(rr.first + t) * a.q.nwords + (i >> 5)] >> (i & 31) & 1;
          see = see && v;
        }
      }
      sum += see ? w[e] * exp2_fast(s[e] * a.q.c - l2[e]) : 0.f;
    }
  };

  for (int base = 0; base < nr; base += kRowsLds) {  // (once, but for more rows than LDS holds)
    __syncthreads();
    if constexpr (NQ == 0)
      for (int x = wave; x < kRowsLds / 16 && base + 16 * x < nr; x += 4) {
        load_q(base + 16 * x, q[0]);
#pragma unroll
        for (int i = 0; i < KC; ++i)
#pragma unroll
          for (int y = 0; y < QP; ++y) sq[x][i][y][lane] = q[0][i][y];
      }
    for (int x = tid; x < kRowsLds; x += 256) {
      const int r = base + x, t = r < nr ? r / G : 0;
      const float l = r < nr ? a.lse[(int64_t)(g * G + r - t * G) * a.q.nrows + rr.first + t] * kLog2e : 0.f;
      const float w = r < nr ? (a.row_w ? a.row_w[rr.first + t] : 1.f) : 0.f;
      sl[x] = l;
      sw[x] = l == -__builtin_inff() ? 0.f : w;  // a row that sees nothing weighs nothing
      st[x] = t;
    }
    __syncthreads();
    const int rows = nr - base < kRowsLds ? nr - base : kRowsLds;
    const int end = total - first < a.rows ? total : first + a.rows;
    u32x4 k[NU][KC][QP], kn[NU][KC][QP];
    bool ok[NU], okn[NU];
    // RW cached rows per wave and step, the next in flight
    auto fetch = [&](int j0, u32x4 (&x)[NU][KC][QP], bool (&o)[NU]) {
#pragma unroll
      for (int u = 0; u < NU; ++u) load_k(j0 + 16 * u < end ? j0 + 16 * u : j0, x[u], o[u]);
    };
    // lane (m, h) writes row 16 h + m
    auto finish = [&](int j0, float (&sum)[NU], const bool (&o)[NU]) {
#pragma unroll
      for (int u = 0; u < NU; ++u) sum[u] = sum4(sum[u]);
      float x0 = sum[0];
      bool has = o[0];
#pragma unroll
      for (int u = 1; u < NU; ++u) {
        x0 = h == u ? sum[u] : x0;
        has = h == u ? o[u] : has;
      }
      const int j = j0 + lane;
      if (lane < RW && j < end && has) {
        const float in = base ? a.acc_out[at + j] : a.acc_in ? a.acc_in[at + j] : 0.f;
        a.acc_out[at + j] = in + x0;
      }
    };
    auto step = [&](int j0, u32x4 (&x)[NU][KC][QP], const bool (&o)[NU]) {
      float sum[NU] = {};
      if constexpr (NQ > 0) {
#pragma unroll
        for (int n = 0; n < NQ; ++n)
#pragma unroll
          for (int u = 0; u < NU; ++u) add(q[n], x[u], 16 * n, j0 + 16 * u, sum[u]);
      } else {
#pragma unroll
        for (int u = 0; u < NU; ++u) split(x[u]);
        for (int r0 = 0; r0 < rows; r0 += 16) {
#pragma unroll
          for (int i = 0; i < KC; ++i)
#pragma unroll
            for (int y = 0; y < QP; ++y) q[0][i][y] = sq[r0 / 16][i][y][lane];
#pragma unroll
          for (int u = 0; u < NU; ++u) add(q[0], x[u], r0, j0 + 16 * u, sum[u]);
        }
      }
      finish(j0, sum, o);
    };
    int j = first + wave * RW;
    if (j >= end) continue;
    fetch(j, k, ok);
    if constexpr (F32 && NQ > 1) {
      // two steps do not fit the registers: 16 rows at a time become bf16 parts and make room for the next step's
      // (16 sequences of 16000 rows, 8 heads of 128, 32 rows of Q: 209 us; 378 with Q read again for every 16 rows)
      while (true) {
        const int jn = j + 4 * RW;
        float sum[NU] = {};
#pragma unroll
        for (int u = 0; u < NU; ++u) {
          split(k[u]);
          u32x4 x[KC][QP];
#pragma unroll
          for (int i = 0; i < KC; ++i)
#pragma unroll
            for (int y = 0; y < QP; ++y) x[i][y] = k[u][i][y];
          if (jn < end) load_k(jn + 16 * u < end ? jn + 16 * u : jn, k[u], okn[u]);
#pragma unroll
          for (int n = 0; n < NQ; ++n) add(q[n], x, 16 * n, j + 16 * u, sum[u]);
        }
        finish(j, sum, ok);
        if (jn >= end) break;
        j = jn;
#pragma unroll
        for (int u = 0; u < NU; ++u) ok[u] = okn[u];
      }
      continue;
    }
    if constexpr (F32 && NQ == 0 && D == 128) {
      // (the steps are long: the SIMD's other wave covers their loads, and nothing goes to scratch)
      while (true) {
        step(j, k, ok);
        j += 4 * RW;
        if (j >= end) break;
        fetch(j, k, ok);
      }
      continue;
    }
    while (true) {
      if (j + 4 * RW < end) fetch(j + 4 * RW, kn, okn);
      step(j, k, ok);
      j += 4 * RW;
      if (j >= end) break;
      if (j + 4 * RW < end) fetch(j + 4 * RW, k, ok);
      step(j, kn, okn);
      j += 4 * RW;
      if (j >= end) break;
    }
  }
}

// ---- launches --------------------------------------------------------------------------------------
// Rows of an item: up to 32 are held by every wave (16 or 32); more of them share stages, in tiles of 64 or 128 rows (four
// waves, two workgroups per CU; fp32 and d = 64 only gain from 128), or of 256 where that pads less: up to 192 rows
// of d = 128 take three tiles of 64 (16 x 16000 rows, 132 rows of Q: 370 us, 520 in one tile of 256), an odd number of
// 128s those (44 sequences of 1 to 1599 rows, 264 rows of Q: 88 us, 133 in two of 256).  Selections belong to one
// token, whose heads rarely are that many: row tiles of 32.
int tile_rows(bool f32, int d, bool sel, int rows) {
  if (rows <= 32 || sel) return rows <= 16 ? 16 : 32;
  if (!f32 && (rows <= 64 || (d == 128 && rows > 128 && rows <= 192))) return 64;
  return f32 || d == 64 || (rows + 127) / 128 % 2 ? 128 : 256;
}

struct DraftShape {
  int trows, rtiles, slots, least, grid, pieces, waves;
};

constexpr int kShort = 256;
constexpr int kMaxGrid = 1 << 23;  // workgroups of up to 512 threads, of which a launch has fewer than 2^32

DraftShape draft_shape(const CacheView &c, const DraftView &q, bool f32, int d, int nsel) {
  DraftShape s{};
  s.waves = kWaves;
  const int G = q.hq / c.hkv, rows = nsel ? G : G * q.max_rows;
  s.trows = tile_rows(f32, d, nsel > 0, rows);
  s.rtiles = (rows + s.trows - 1) / s.trows;
  // workgroups that the chip holds at once: with stages three per CU (d = 64: 16 sequences of 16000 rows, 256 rows of Q,
  // 233 us, planned for two 295), two (d = 128, four waves) or one; else two with d = 64 or 16 rows of bf16, or one
  const bool two = d == 64 || (!f32 && s.trows == 16), wide = s.trows > 32;
  const int resident = 256 * (!wide ? 1 + two : d == 64 ? 3 : s.trows < 256 ? 2 : 1);
  if (nsel) {
    const int64_t items = (int64_t)q.nrows * c.hkv * s.rtiles;
    const int most = (int)(((int64_t)nsel * 64 + 63 + q.max_rows + kGroup - 1) / kGroup);
    int64_t p = items ? resident / items : 1;
    p = p < most ? p : most;
    s.pieces = p > 1 ? (int)p : 1;
    s.grid = (int)(items * s.pieces);
    return s;
  }
  const int64_t items = (int64_t)c.nseq * c.hkv * s.rtiles, most = items * ((c.cap + kGroup - 1) / kGroup);
  // A short cache stays in one piece and needs no joining launch (4 us): up to kShort rows in four waves, twice that in
  // eight where a CU holds two waves per SIMD (8 heads over 500 rows: one sequence 12.6 -> 10.0 us, 64 of them 36.7 ->
  // 27.5).  Longer ones gain from pieces (one token over 1001 rows: 14.7 us in one piece, 12.3 in several): few items
  // make one round of workgroups; many, pieces of a quarter of a round, so that the last round is short.
  if (c.cap <= (two && !wide ? 2 * kShort : kShort)) {
    s.waves = c.cap > kShort ? 8 : kWaves;
    s.slots = 0;
    s.grid = (int)items;
    return s;
  }
  // A piece of many rows writes, and the join reads, as much as 2 trows rows of fp32: where the items alone fill
  // the chip, it walks so many groups that this stays small beside K and V (49 sequences of 0 to 433 rows, 448 rows
  // of Q per head: 215 us in pieces of one group, 53 us in one piece each; 33 sequences of 2000 to 8000 rows, 132 rows
  // in tiles of 128: 448 us from 8 groups on, 347 from 16).
  s.slots = items <= resident / 2 ? resident - (int)items : 4 * resident;
  s.least = items <= resident / 2 ? 1 : s.trows >= 128 ? 16 : s.trows / 16;
  if (c.cap <= s.least * kGroup) s.slots = 0;  // no sequence is long enough for two pieces
  const int64_t grid = items + s.slots;
  s.grid = (int)(grid < most && s.slots ? grid : s.slots ? most : items);
  return s;
}

template <typename F>
void by_tiles(bool f32, int d, int trows, F f) {
  using N1 = std::integral_constant<int, 1>;
  using N2 = std::integral_constant<int, 2>;
  auto with_d = [&](auto x, auto dd) { trows == 16 ? f(x, dd, N1{}) : f(x, dd, N2{}); };
  auto with_t = [&](auto x) {
    d == 128 ? with_d(x, std::integral_constant<int, 128>{}) : with_d(x, std::integral_constant<int, 64>{});
  };
  f32 ? with_t(std::true_type{}) : with_t(std::false_type{});
}

template <bool F32, int D>
void wide_launch(const DraftArgs &a, const DraftShape &s, hipStream_t st) {
  if (s.trows == 128) return draft_wide_kernel<F32, D, 1, 4><<<s.grid, 256, 0, st>>>(a);
  if constexpr (!F32) {
    if (s.trows == 64) return draft_wide_kernel<F32, D, 2, 4><<<s.grid, 256, 0, st>>>(a);
    if constexpr (D == 128) draft_wide_kernel<F32, D, 1, 8><<<s.grid, 512, 0, st>>>(a);
  }
}

DraftArgs draft_parts(Arena &ar, const CacheView &c, const DraftView &q, const DraftShape &s, int d) {
  DraftArgs a{};
  a.c = c;
  a.q = q;
  a.rtiles = s.rtiles;
  a.trows = s.trows;
  a.slots = s.slots;
  a.least = s.least;
  a.pieces = s.pieces;
  // (a single piece is the result itself; its call asks for one line all the same, so that no caller does without one)
  const size_t rows = s.slots > 0 || s.pieces > 1 ? (size_t)s.grid * s.trows : 0;
  a.po = ar.take<float>(rows ? rows * d : 64);
  a.pml = ar.take<float>(rows * 2);
  return a;
}

SelectArgs select_parts(Arena &ar, const CacheView &c, const DraftView &q, int nsel) {
  SelectArgs s{};
  s.c = c;
  s.q = q;
  s.nsel = nsel;
  s.fcap = c.cap >> 6;
  s.list = ar.take<int32_t>((size_t)q.nrows * c.hkv * nsel);
  s.score = ar.take<double>((size_t)q.nrows * c.hkv * s.fcap);
  return s;
}

template <bool SEL>
rs_status attend(const DraftArgs &a, const DraftShape &s, bool f32, int d, hipStream_t st) {
  if (s.trows > 32)
    f32 ? (d == 128 ? wide_launch<true, 128>(a, s, st) : wide_launch<true, 64>(a, s, st))
        : (d == 128 ? wide_launch<false, 128>(a, s, st) : wide_launch<false, 64>(a, s, st));
  else
    by_tiles(f32, d, s.trows, [&](auto x, auto dd, auto nn) {
      constexpr bool F = decltype(x)::value;
      constexpr int D = decltype(dd)::value, NQ = decltype(nn)::value;
      if constexpr (SEL)
        draft_kernel<F, D, NQ, true><<<dim3(a.q.nrows * s.pieces, a.c.hkv * s.rtiles), 256, 0, st>>>(a);
      else {
        if constexpr (D == 64 || (!F && NQ == 1))
          if (s.waves > kWaves) return draft_kernel<F, D, NQ, false, 8><<<s.grid, 512, 0, st>>>(a);
        draft_kernel<F, D, NQ, false><<<s.grid, 256, 0, st>>>(a);
      }
    });
  if (SEL ? s.pieces > 1 : s.slots > 0) {
    if ((int64_t)a.q.nrows * a.q.hq >= 4096) {
      const dim3 grid(a.q.nrows, (a.q.hq + kWaves - 1) / kWaves);
      d == 128 ? draft_join_kernel<128, SEL, 1><<<grid, 256, 0, st>>>(a) : draft_join_kernel<64, SEL, 1><<<grid, 256, 0, st>>>(a);
    } else {
      const dim3 grid(a.q.nrows, a.q.hq);
      d == 128 ? draft_join_kernel<128, SEL, kWaves><<<grid, 256, 0, st>>>(a) : draft_join_kernel<64, SEL, kWaves><<<grid, 256, 0, st>>>(a);
    }
  }
  RS_HIP(hipGetLastError());
  return RS_OK;
}

}  // namespace

size_t draft_ws_bytes(const CacheView &c, const DraftView &q, bool f32, int d, int nsel) {
  Arena ar(nullptr, 0);
  const DraftShape s = draft_shape(c, q, f32, d, nsel);
  if (!nsel && s.grid >= kMaxGrid) return 0;
  if (nsel) select_parts(ar, c, q, nsel);
  draft_parts(ar, c, q, s, d);
  return ar.off + 256;
}

rs_status draft_launch(const CacheView &c, const DraftView &q, bool f32, int d, void *o, int64_t so_t, int64_t so_h, float *lse,
                       void *ws, size_t ws_bytes, hipStream_t st) {
  const DraftShape s = draft_shape(c, q, f32, d, 0);
  if (s.grid >= kMaxGrid) return fail(RS_ERR_UNSUPPORTED, "draft: at most 2^23 - 1 workgroups (nseq x hkv x row tiles)");
  Arena ar(ws, ws_bytes);
  DraftArgs a = draft_parts(ar, c, q, s, d);
  if (!ws || !ar.ok())
    return fail(RS_ERR_WORKSPACE, "draft attention workspace too small: need " + std::to_string(draft_ws_bytes(c, q, f32, d, 0)));
  a.o = (char *)o, a.so_t = so_t, a.so_h = so_h, a.lse = lse;
  return attend<false>(a, s, f32, d, st);
}

rs_status select_launch(const CacheView &c, const DraftView &q, bool f32, int d, int nsel, int nsink, int nlocal, void *o,
                        int64_t so_t, int64_t so_h, float *lse, int32_t *blocks, void *ws, size_t ws_bytes, hipStream_t st) {
  const DraftShape s = draft_shape(c, q, f32, d, nsel);
  Arena ar(ws, ws_bytes);
  SelectArgs sel = select_parts(ar, c, q, nsel);
  DraftArgs a = draft_parts(ar, c, q, s, d);
  if (!ws || !ar.ok())
    return fail(RS_ERR_WORKSPACE, "selected attention workspace too small: need " + std::to_string(draft_ws_bytes(c, q, f32, d, nsel)));
  if (blocks) sel.list = blocks;
  sel.nsink = nsink, sel.nlocal = nlocal;
  a.o = (char *)o, a.so_t = so_t, a.so_h = so_h, a.lse = lse;
  a.list = sel.list, a.nsel = nsel;
  if (sel.fcap > nsel) {
    const dim3 grid((sel.fcap + 63) / 64, c.hkv, c.nseq);
    f32 ? (d == 128 ? score_kernel<true, 128><<<grid, 256, 0, st>>>(sel) : score_kernel<true, 64><<<grid, 256, 0, st>>>(sel))
        : (d == 128 ? score_kernel<false, 128><<<grid, 256, 0, st>>>(sel) : score_kernel<false, 64><<<grid, 256, 0, st>>>(sel));
  }
  const dim3 rows(q.nrows, c.hkv);
  select_kernel<<<rows, kSelThreads, 0, st>>>(sel);
  return attend<true>(a, s, f32, d, st);
}

rs_status weights_launch(const CacheView &c, const DraftView &q, bool f32, int d, const float *lse, const float *row_w,
                         const float *acc_in, float *acc_out, hipStream_t st) {
  // four steps of every wave, so that loads run ahead; one where that would leave CUs idle
  const int per = (int64_t)((c.cap + 1023) / 1024) * c.hkv * c.nseq >= 512 ? 1024 : 256;
  const WeightArgs a{c, q, lse, row_w, acc_in, acc_out, per};
  const dim3 grid((c.cap + per - 1) / per, c.hkv, c.nseq);
  const int rows = q.hq / c.hkv * q.max_rows;
  auto run = [&](auto x, auto dd) {
    constexpr bool F = decltype(x)::value;
    constexpr int DD = decltype(dd)::value;
    if (rows <= 16) return weights_kernel<F, DD, 1><<<grid, 256, 0, st>>>(a);
    if (rows <= 32) return weights_kernel<F, DD, 2><<<grid, 256, 0, st>>>(a);
    weights_kernel<F, DD, 0><<<grid, 256, 0, st>>>(a);
  };
  auto with_d = [&](auto x) { d == 128 ? run(x, std::integral_constant<int, 128>{}) : run(x, std::integral_constant<int, 64>{}); };
  f32 ? with_d(std::true_type{}) : with_d(std::false_type{});
  RS_HIP(hipGetLastError());
  return RS_OK;
}

}  // namespace rs
