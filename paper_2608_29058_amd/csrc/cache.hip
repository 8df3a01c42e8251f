// The key/value cache between the attention calls: new rows in, accepted rows kept, rows of least
// accumulated weight out.  All of it is copying: what bounds these kernels is memory and, for the
// short calls, the launch itself, so each call is one launch where its parts allow that.
#include "common.h"
#include "cache.h"

namespace rs {

namespace {

// ---- append --------------------------------------------------------------------------------
// A workgroup writes up to kAppendRows rows of one sequence, all heads, in pieces of 16 bytes; K and V of
// a piece by the same thread, so that both loads are in flight before either store.
constexpr int kAppendRows = 16;

__global__ __launch_bounds__(256) void append_kernel(CacheView c, const char *kn, const char *vn, int64_t skt, int64_t skh,
                                                     int64_t svt, int64_t svh, const int32_t *start, int nrows,
                                                     int max_rows, int lp) {  // 1 << lp pieces per row
  const int b = blockIdx.y, r0 = blockIdx.x * kAppendRows;
  const RowRange rr = new_rows(start, b, nrows, max_rows);
  const int len = cache_len(c, b);
  const int most = rr.count < c.cap - len ? rr.count : c.cap - len;
  const int rows = most - r0 < kAppendRows ? most - r0 : kAppendRows;
  if (rows <= 0) return;
  const int per_row = c.hkv << lp, total = rows * per_row;
  for (int x = threadIdx.x; x < total; x += 256) {
    const int i = x / per_row, y = x - i * per_row, g = y >> lp, o = (y & ((1 << lp) - 1)) * 16;
    const int j = len + r0 + i, p = page_of(c, j), id = page_id(c, b, p);
    if (id < 0) continue;
    const int64_t row = rr.first + r0 + i;
    const u32x4 kk = *(const u32x4 *)(kn + row * skt + g * skh + o), vv = *(const u32x4 *)(vn + row * svt + g * svh + o);
    *(u32x4 *)(c.k + k_offset(c, id, p, j, g) + o) = kk;
    *(u32x4 *)(c.v + v_offset(c, id, p, j, g) + o) = vv;
    if (c.acc && o == 0) c.acc[((int64_t)b * c.hkv + g) * c.cap + j] = 0.f;
  }
}

// ---- block means ---------------------------------------------------------------------------
// Mean of the 64 K rows of block blk, by one wave: lane l sums rows l / (D / 8), ... of its 8 dimensions in
// fp64, then the lanes of equal dimensions add up (in one order; exact while values lie within 2^39 of each other in
// bf16, 53 bits less 8 and 6 of carry, or 2^23 in fp32).  The mean is rounded to fp32 and that to bf16, so what lies
// within 2^-25 of the middle of two bf16 values counts as the middle: it is a score's factor, and 8 bits of it rank
// blocks as well as 24.
template <typename T, int D>
__device__ void block_mean(const CacheView &c, int b, int g, int blk, int lane) {
  constexpr int LPR = D / 8, RPI = 64 / LPR;  // lanes per row, rows per step
  const int p = page_of(c, blk * 64), id = page_id(c, b, p);
  if (id < 0) return;
  const char *base = c.k + k_offset(c, id, p, blk * 64, g);
  const int dl = lane % LPR, r0 = lane / LPR;
  double s[8] = {};
  for (int r = r0; r < 64; r += RPI) {
    const T *x = (const T *)(base + r * c.sk_t) + dl * 8;
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] += (double)(float)x[e];
  }
#pragma unroll
  for (int m = LPR; m < 64; m <<= 1)
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] += __shfl_xor(s[e], m);
  if (r0 == 0) {
    u32x4 w;
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = pack_bf16x2((float)(s[2 * e] * 0.015625), (float)(s[2 * e + 1] * 0.015625));
    *(u32x4 *)((bf16 *)c.kmean + mean_offset(c, id, p, blk, g, D) + dl * 8) = w;
  }
}

// ---- commit --------------------------------------------------------------------------------
// Few rows: one workgroup per sequence moves the rows of the path, then writes positions, means and the
// new length, in one launch.  The path ascends, so row i comes from a row at or behind it: what a step
// reads before its barrier lies behind everything that earlier steps wrote, and its own writes follow the
// barrier.
constexpr int kCommitThreads = 1024, kCommitPieces = 4;

template <typename T, int D>
__global__ __launch_bounds__(kCommitThreads) void commit_kernel(CacheView c, const int32_t *naccept, const int32_t *path,
                                                                int max_new) {
  __shared__ int sp[kMaxDraft];
  constexpr int NP = D * (int)sizeof(T) / 16;
  const int b = blockIdx.x, tid = threadIdx.x;
  const int len = cache_len(c, b);
  int na = clampi(naccept[b], 0, max_new);
  na = na < c.cap - len ? na : c.cap - len;
  const int seen = c.seen ? c.seen[b] : 0;
  if (path) {
    for (int i = tid; i < na; i += kCommitThreads) {
      int x = path[(int64_t)b * max_new + i];
      if (x < i || x >= max_new || len + x >= c.cap) x = i;
      sp[i] = x;
    }
    __syncthreads();
    const int per_row = c.hkv * NP, total = na * per_row;  // a piece: 16 bytes of K and the same of V
    for (int x0 = 0; x0 < total; x0 += kCommitThreads * kCommitPieces) {
      u32x4 kk[kCommitPieces], vv[kCommitPieces];
      float a[kCommitPieces];
      int64_t ko[kCommitPieces], vo[kCommitPieces], ao[kCommitPieces];
#pragma unroll
      for (int u = 0; u < kCommitPieces; ++u) {
        const int x = x0 + u * kCommitThreads + tid;
        ko[u] = -1;
        if (x >= total) continue;
        const int i = x / per_row, y = x - i * per_row, g = y / NP, o = (y % NP) * 16;
        if (sp[i] == i) continue;
        const int js = len + sp[i], jd = len + i, ps = page_of(c, js), pd = page_of(c, jd);
        const int is = page_id(c, b, ps), id = page_id(c, b, pd);
        if (is < 0 || id < 0) continue;
        kk[u] = *(const u32x4 *)(c.k + k_offset(c, is, ps, js, g) + o);
        vv[u] = *(const u32x4 *)(c.v + v_offset(c, is, ps, js, g) + o);
        ko[u] = k_offset(c, id, pd, jd, g) + o;
        vo[u] = v_offset(c, id, pd, jd, g) + o;
        ao[u] = -1;
        if (c.acc && o == 0) {
          const int64_t h = ((int64_t)b * c.hkv + g) * c.cap;
          a[u] = c.acc[h + js];
          ao[u] = h + jd;
        }
      }
      __syncthreads();
#pragma unroll
      for (int u = 0; u < kCommitPieces; ++u)
        if (ko[u] >= 0) {
          *(u32x4 *)(c.k + ko[u]) = kk[u];
          *(u32x4 *)(c.v + vo[u]) = vv[u];
          if (ao[u] >= 0) c.acc[ao[u]] = a[u];
        }
      __syncthreads();
    }
  }
  if (c.pos)
    for (int x = tid; x < na * c.hkv; x += kCommitThreads) {
      const int g = x / na, i = x - g * na;
      c.pos[((int64_t)b * c.hkv + g) * c.cap + len + i] = seen + i;
    }
  if (c.kmean) {
    const int b0 = len >> 6, nb = ((len + na) >> 6) - b0;
    for (int x = tid >> 6; x < nb * c.hkv; x += kCommitThreads / 64) block_mean<T, D>(c, b, x / nb, b0 + x % nb, tid & 63);
  }
  // every wave of this workgroup has read len by now; no other workgroup reads this sequence's
  __syncthreads();
  if (tid == 0) {
    c.len[b] = len + na;
    if (c.seen) c.seen[b] = seen + na;
  }
}

// Many rows (a prompt, a chunk): a wave per block of 64 rows and head; the lengths follow in a launch of
// their own, since all workgroups of this one read them.
template <typename T, int D>
__global__ __launch_bounds__(256) void commit_rows_kernel(CacheView c, const int32_t *naccept, int max_new) {
  const int b = blockIdx.z, g = blockIdx.y, lane = threadIdx.x & 63;
  const int len = cache_len(c, b);
  int na = clampi(naccept[b], 0, max_new);
  na = na < c.cap - len ? na : c.cap - len;
  const int blk = (len >> 6) + blockIdx.x * 4 + (threadIdx.x >> 6), j = blk * 64 + lane;
  if (blk * 64 >= len + na) return;
  if (c.pos && j >= len && j < len + na) c.pos[((int64_t)b * c.hkv + g) * c.cap + j] = (c.seen ? c.seen[b] : 0) + j - len;
  if (c.kmean && blk * 64 + 64 <= len + na) block_mean<T, D>(c, b, g, blk, lane);
}

__global__ void commit_len_kernel(CacheView c, const int32_t *naccept, int max_new) {
  const int b = blockIdx.x * 64 + threadIdx.x;
  if (b >= c.nseq) return;
  const int len = cache_len(c, b);
  int na = clampi(naccept[b], 0, max_new);
  na = na < c.cap - len ? na : c.cap - len;
  c.len[b] = len + na;
  if (c.seen) c.seen[b] += na;
}

// ---- eviction ------------------------------------------------------------------------------
// Plan, one workgroup per sequence and head (or several, below): the `budget` first rows of the order (firm
// rows, then acc descending, then row ascending) are found by a radix selection over 32-bit keys with the counts
// in LDS.  The first digit has 12 bits: weights lie in a few
// octaves, and with 8 bits nearly all of a wave's counts would go to the same word.  One more pass lists,
// in row order, the places before the budget whose row goes and the rows behind it that stay.
struct EvictPlan {
  int32_t *count;  // [nseq * hkv] rows that move; -1: the sequence is not over its budget
  int32_t *hole;   // [nseq * hkv][most]
  int32_t *mover;  // [nseq * hkv][most]
  int most;
};

constexpr int kPlanThreads = 1024;

// Key of a row in the order of the selection: firm rows share the highest, which no other row has (a NaN with all
// bits set would).
__device__ __forceinline__ uint32_t evict_key(float a, int pos, int nsink, int firm_from) {
  const uint32_t k = float_key(a);
  return pos < nsink || pos >= firm_from ? 0xffffffffu : k < 0xfffffffeu ? k : 0xfffffffeu;
}

// The bin in which the count from the highest key down reaches `need`: pick = {bin, rows of it that still
// stay, rows in it}.  Thread t counts the t-th highest group of bins.
__device__ __forceinline__ void pick_bin(const int *hist, int bins, int need, int *sw, int *pick) {
  const int per = bins / kPlanThreads, top = bins - 1 - (int)threadIdx.x * per;
  int sum = 0, all;
  for (int x = 0; x < per; ++x) sum += hist[top - x];
  int before = block_scan<kPlanThreads>(sum, sw, &all);
  if (before < need && before + sum >= need) {
    int x = top;
    while (before + hist[x] < need) before += hist[x--];
    pick[0] = x;
    pick[1] = need - before;
    pick[2] = hist[x];
  }
  __syncthreads();
}

// Counts of the digit (key >> sh) & (bins - 1) of the rows [lo, hi) whose leading digits are `prefix`.
__device__ __forceinline__ void count_digit(const float *acc, const int *pos, int lo, int hi, int nsink, int firm_from,
                                            uint32_t prefix, uint32_t have, int sh, int bins, int *hist) {
  constexpr int kPer = 8;
  const int tid = threadIdx.x;
  for (int x = tid; x < bins; x += kPlanThreads) hist[x] = 0;
  __syncthreads();
  for (int j0 = lo + tid; j0 < hi; j0 += kPlanThreads * kPer) {
    float x[kPer];
    int y[kPer];
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
      const int j = j0 + u * kPlanThreads < hi ? j0 + u * kPlanThreads : j0;
      x[u] = acc[j];
      y[u] = pos[j];
    }
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
      const uint32_t key = evict_key(x[u], y[u], nsink, firm_from);
      if (j0 + u * kPlanThreads < hi && (key & have) == prefix) atomicAdd(&hist[(key >> sh) & (bins - 1)], 1);
    }
  }
  __syncthreads();
}

// What is known of the budget-th largest key: its digits (those under `have`), how many rows share them
// and how many of these still stay.
struct Border {
  uint32_t prefix, have;
  int need, equal;
};
constexpr int kBins = 4096;  // bins of a digit at most
__device__ __forceinline__ int digit_bins(int pass) { return pass ? 1024 : 4096; }
__device__ __forceinline__ int digit_shift(int pass) { return pass == 0 ? 20 : pass == 1 ? 10 : 0; }

// Rows of a step: `PER` pieces of 64 consecutive rows per wave, the waves one after the other; thread (wave, lane)
// holds rows j0 + wave 64 PER + 64 x + lane.
template <int PER>
__device__ __forceinline__ void load_keys(const float *acc, const int *pos, int j0, int hi, int nsink, int firm_from, uint32_t (&key)[PER]) {
  const int jw = j0 + (threadIdx.x >> 6) * 64 * PER + (threadIdx.x & 63);
  float a[PER];
  int q[PER];
#pragma unroll
  for (int x = 0; x < PER; ++x) {
    const int j = jw + 64 * x < hi ? jw + 64 * x : hi - 1;
    a[x] = acc[j];
    q[x] = pos[j];
  }
#pragma unroll
  for (int x = 0; x < PER; ++x) key[x] = evict_key(a[x], q[x], nsink, firm_from);
}

// Lists, in row order, the places before the budget whose row goes and the rows behind it that stay, of a step
// from row j0 of [.., hi).  Before it: `ranked` rows equal to the border's, `holes` such places and `movers` such
// rows.
template <int PER>
__device__ __forceinline__ void list_moves(const uint32_t (&key)[PER], int j0, int hi, int budget, const Border &bd, int &ranked,
                                           int &holes, int &movers, int *hole_out, int *mover_out, int *sw) {
  const bool ties = bd.need < bd.equal;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, jw = j0 + wave * 64 * PER + lane;
  const uint64_t below = (1ull << lane) - 1;
  // x of the waves before this one, and of all
  auto scan = [&](int x, int &all) {
    if (lane == 0) sw[wave] = x;
    __syncthreads();
    int before = 0;
    all = 0;
#pragma unroll
    for (int k = 0; k < kPlanThreads / 64; ++k) {
      const int y = sw[k];
      before += k < wave ? y : 0;
      all += y;
    }
    __syncthreads();
    return before;
  };
  int all, at = 0;
  uint64_t eq[PER];
  int e = 0;
#pragma unroll
  for (int x = 0; x < PER; ++x) {
    eq[x] = __ballot(jw + 64 * x < hi && (key[x] & bd.have) == bd.prefix);
    e += __popcll(eq[x]);
  }
  if (ties) {
    at = ranked + scan(e, all);
    ranked += all;
  }
  uint64_t hole[PER], mover[PER];
  int hm = 0;
#pragma unroll
  for (int x = 0; x < PER; ++x) {
    const int j = jw + 64 * x;
    const uint32_t k = key[x] & bd.have;
    const bool stay = k > bd.prefix || (k == bd.prefix && (!ties || at + __popcll(eq[x] & below) < bd.need));
    at += __popcll(eq[x]);
    hole[x] = __ballot(j < hi && j < budget && !stay);
    mover[x] = __ballot(j < hi && j >= budget && stay);
    hm += __popcll(hole[x]) | __popcll(mover[x]) << 16;  // at most 1024 PER of each in a step
  }
  const int before = scan(hm, all);
  int h = holes + (before & 0xffff), m = movers + (before >> 16);
#pragma unroll
  for (int x = 0; x < PER; ++x) {
    if (hole[x] >> lane & 1) hole_out[h + __popcll(hole[x] & below)] = jw + 64 * x;
    if (mover[x] >> lane & 1) mover_out[m + __popcll(mover[x] & below)] = jw + 64 * x;
    h += __popcll(hole[x]);
    m += __popcll(mover[x]);
  }
  holes += all & 0xffff;
  movers += all >> 16;
}

// Caches of up to 1024 PER rows: read once, their keys in registers.
template <int PER>
__global__ __launch_bounds__(kPlanThreads) void evict_plan_kernel(CacheView c, int budget, int nsink, int nrecent, EvictPlan pl) {
  __shared__ int hist[kBins], sw[kPlanThreads / 64], pick[3];
  const int b = blockIdx.y, g = blockIdx.x;
  const int64_t item = (int64_t)b * c.hkv + g;
  const int n = cache_len(c, b);
  if (n <= budget) {
    if (threadIdx.x == 0) pl.count[item] = -1;
    return;
  }
  const float *acc = c.acc + item * c.cap;
  const int *pos = c.pos + item * c.cap;
  const int seen = c.seen[b], firm_from = (seen > 0 ? seen : 0) - nrecent;
  uint32_t key[PER];
  load_keys<PER>(acc, pos, 0, n, nsink, firm_from, key);
  const int jw = (threadIdx.x >> 6) * 64 * PER + (threadIdx.x & 63);
  Border bd{0, 0, budget, n};
  for (int pass = 0; pass < 3 && bd.need < bd.equal; ++pass) {
    const int bins = digit_bins(pass), sh = digit_shift(pass);
    for (int x = threadIdx.x; x < bins; x += kPlanThreads) hist[x] = 0;
    __syncthreads();
#pragma unroll
    for (int x = 0; x < PER; ++x)
      if (jw + 64 * x < n && (key[x] & bd.have) == bd.prefix) atomicAdd(&hist[(key[x] >> sh) & (bins - 1)], 1);
    __syncthreads();
    pick_bin(hist, bins, bd.need, sw, pick);
    bd = Border{bd.prefix | (uint32_t)pick[0] << sh, bd.have | (uint32_t)(bins - 1) << sh, pick[1], pick[2]};
    __syncthreads();
  }
  int ranked = 0, holes = 0, movers = 0;
  list_moves<PER>(key, 0, n, budget, bd, ranked, holes, movers, pl.hole + item * pl.most, pl.mover + item * pl.most, sw);
  if (threadIdx.x == 0) pl.count[item] = movers;
}

// The same with the rows of an item cut into slices, a workgroup each: one workgroup reads 8 bytes per row and
// pass at the rate of one CU (two sequences of 128K rows and 8 heads: 197 us).  Slices do not cross the budget,
// so that one has either places or movers.  A launch per digit: it adds up the slices' counts of the digit
// before (every workgroup for itself), finds the border's next bin, notes how many of the rows above and in it
// lie in earlier slices, and counts its own slice's next digit.  The last launch lists.
struct EvictSlices {
  uint16_t *hist;   // [item][slice][3 digits: 4096, 1024, 1024]
  Border *border;   // [item][3], after each digit
  int *above;       // [2][item][slice + 1][2] after the first and second digit: rows above the border so far, and
                    // equal to it, in earlier slices; last those of all slices before the budget
  int nslice, n1, rows;  // slices per item, those before the budget, rows of a slice
};
constexpr int kSliceBins = 4096 + 1024 + 1024;
__device__ __forceinline__ int digit_first(int pass) { return pass == 0 ? 0 : pass == 1 ? 4096 : 5120; }

// PASS 0, 1, 2: counts that digit; 3: lists.
template <int PASS>
__global__ __launch_bounds__(kPlanThreads) void evict_slice_kernel(CacheView c, int budget, int nsink, int nrecent, EvictPlan pl,
                                                                   EvictSlices sl) {
  __shared__ int hist[kBins], sw[kPlanThreads / 64], pick[3], part[4];
  const int s = blockIdx.x, g = blockIdx.y, b = blockIdx.z, tid = threadIdx.x;
  const int64_t item = (int64_t)b * c.hkv + g;
  const int n = cache_len(c, b);
  if (n <= budget) {
    if (PASS == 3 && s == 0 && tid == 0) pl.count[item] = -1;
    return;
  }
  const float *acc = c.acc + item * c.cap;
  const int *pos = c.pos + item * c.cap;
  const int seen = c.seen[b], firm_from = (seen > 0 ? seen : 0) - nrecent;
  const int lo = s < sl.n1 ? s * sl.rows : budget + (s - sl.n1) * sl.rows;
  int hi = lo + sl.rows;
  hi = s < sl.n1 ? (hi < budget ? hi : budget) : (hi < n ? hi : n);
  Border bd{0, 0, budget, n};
  const int64_t items = (int64_t)c.nseq * c.hkv;
  auto above_at = [&](int pass, int x) { return sl.above + ((pass * items + item) * (sl.nslice + 1) + x) * 2; };
  int above[2] = {0, 0}, equal[2] = {0, 0};  // of earlier slices, and of all slices before the budget
  if constexpr (PASS > 1) {
    bd = sl.border[item * 3 + PASS - 2];
    const int *w = above_at(PASS - 2, s), *w1 = above_at(PASS - 2, sl.nslice);
    above[0] = w[0], equal[0] = w[1];
    above[1] = w1[0], equal[1] = w1[1];
  }
  if constexpr (PASS > 0) {
    if (PASS == 1 || bd.need < bd.equal) {
      constexpr int bins = PASS == 1 ? 4096 : 1024, sh = PASS == 1 ? 20 : PASS == 2 ? 10 : 0, per = bins / kPlanThreads;
      const uint16_t *h = sl.hist + item * sl.nslice * kSliceBins + digit_first(PASS - 1);
      int before[4] = {0, 0, 0, 0}, first[4] = {0, 0, 0, 0}, all[4] = {0, 0, 0, 0};  // of bins tid, tid + 1024, ...
#pragma unroll 6
      for (int x = 0; x < sl.nslice; ++x)
#pragma unroll
        for (int u = 0; u < per; ++u) {
          const int v = h[(int64_t)x * kSliceBins + tid + u * kPlanThreads];
          all[u] += v;
          before[u] += x < s ? v : 0;
          first[u] += x < sl.n1 ? v : 0;
        }
      for (int u = 0; u < per; ++u) hist[tid + u * kPlanThreads] = all[u];
      if (tid < 4) part[tid] = 0;
      __syncthreads();
      pick_bin(hist, bins, bd.need, sw, pick);
      int p0 = 0, p1 = 0;
      for (int u = 0; u < per; ++u) {
        const int x = tid + u * kPlanThreads;
        p0 += x > pick[0] ? before[u] : 0;
        p1 += x > pick[0] ? first[u] : 0;
        if (x == pick[0]) part[2] = before[u], part[3] = first[u];
      }
      if (p0) atomicAdd(&part[0], p0);
      if (p1) atomicAdd(&part[1], p1);
      __syncthreads();
      bd = Border{bd.prefix | (uint32_t)pick[0] << sh, bd.have | (uint32_t)(bins - 1) << sh, pick[1], pick[2]};
      for (int k = 0; k < 2; ++k) above[k] += part[k], equal[k] = part[2 + k];
      __syncthreads();
    }
    if constexpr (PASS < 3)
      if (tid == 0) {
        int *w = above_at(PASS - 1, s);
        w[0] = above[0], w[1] = equal[0];
        if (s == 0) {
          sl.border[item * 3 + PASS - 1] = bd;
          w = above_at(PASS - 1, sl.nslice);
          w[0] = above[1], w[1] = equal[1];
        }
      }
  }
  if constexpr (PASS < 3) {
    if (PASS > 0 && bd.need == bd.equal) return;  // the border is known
    const int bins = digit_bins(PASS), sh = digit_shift(PASS);
    count_digit(acc, pos, lo, hi, nsink, firm_from, bd.prefix, bd.have, sh, bins, hist);
    uint16_t *h = sl.hist + (item * sl.nslice + s) * kSliceBins + digit_first(PASS);
    for (int x = tid; x < bins; x += kPlanThreads) h[x] = (uint16_t)hist[x];
  } else {
    const int kept = above[0] + (equal[0] < bd.need ? equal[0] : bd.need);    // rows that stay in earlier slices,
    const int kept1 = above[1] + (equal[1] < bd.need ? equal[1] : bd.need);   // and before the budget
    int holes = s < sl.n1 ? lo - kept : 0, movers = s < sl.n1 ? 0 : kept - kept1;
    int ranked = equal[0];
    for (int j0 = lo; j0 < hi; j0 += kPlanThreads * 8) {
      uint32_t key[8];
      load_keys<8>(acc, pos, j0, hi, nsink, firm_from, key);
      list_moves<8>(key, j0, hi, budget, bd, ranked, holes, movers, pl.hole + item * pl.most, pl.mover + item * pl.most, sw);
    }
    if (s == 0 && tid == 0) pl.count[item] = budget - kept1;
  }
}

// The planned moves: places before the budget receive rows behind it, so nothing is read that is written.
// The lengths change here, where only the plan is read.
constexpr int kMoveRows = 64;

__global__ __launch_bounds__(256) void evict_move_kernel(CacheView c, int budget, EvictPlan pl, int lp) {
  const int b = blockIdx.z, g = blockIdx.y;
  const int64_t item = (int64_t)b * c.hkv + g;
  const int count = pl.count[item];
  if (count < 0) return;
  if (blockIdx.x == 0 && g == 0 && threadIdx.x == 0) c.len[b] = budget;
  const int i0 = blockIdx.x * kMoveRows;
  const int rows = count - i0 < kMoveRows ? count - i0 : kMoveRows;
  for (int x = threadIdx.x; x < rows << lp; x += 256) {
    const int i = i0 + (x >> lp), o = (x & ((1 << lp) - 1)) * 16;
    const int js = pl.mover[item * pl.most + i], jd = pl.hole[item * pl.most + i];
    if (o == 0) {
      c.acc[item * c.cap + jd] = c.acc[item * c.cap + js];
      c.pos[item * c.cap + jd] = c.pos[item * c.cap + js];
    }
    const int ps = page_of(c, js), pd = page_of(c, jd), is = page_id(c, b, ps), id = page_id(c, b, pd);
    if (is < 0 || id < 0) continue;
    const u32x4 kk = *(const u32x4 *)(c.k + k_offset(c, is, ps, js, g) + o), vv = *(const u32x4 *)(c.v + v_offset(c, is, ps, js, g) + o);
    *(u32x4 *)(c.k + k_offset(c, id, pd, jd, g) + o) = kk;
    *(u32x4 *)(c.v + v_offset(c, id, pd, jd, g) + o) = vv;
  }
}

// Means of the complete blocks that received rows, a wave each.
template <typename T, int D>
__global__ __launch_bounds__(256) void evict_means_kernel(CacheView c, int budget, EvictPlan pl) {
  const int b = blockIdx.z, g = blockIdx.y, blk = blockIdx.x * 4 + (threadIdx.x >> 6);
  const int64_t item = (int64_t)b * c.hkv + g;
  const int count = pl.count[item];
  if (count < 0 || blk * 64 + 64 > budget) return;
  const int *hole = pl.hole + item * pl.most;  // ascending: the first at or behind the block's first row
  int lo = 0, hi = count;
  while (lo < hi) {
    const int m = (lo + hi) >> 1;
    if (hole[m] < blk * 64)
      lo = m + 1;
    else
      hi = m;
  }
  if (lo < count && hole[lo] < blk * 64 + 64) block_mean<T, D>(c, b, g, blk, threadIdx.x & 63);
}

EvictPlan plan_at(Arena &a, int64_t items, int budget, int cap) {
  EvictPlan pl{};
  pl.most = budget < cap - budget ? budget : cap - budget;
  if (pl.most < 0) pl.most = 0;
  pl.count = a.take<int32_t>((size_t)items);
  pl.hole = a.take<int32_t>((size_t)items * pl.most);
  pl.mover = a.take<int32_t>((size_t)items * pl.most);
  return pl;
}

// Slices of 8K rows or more (their counts fit 16 bits), about 16 of them, where a cache holds more than one
// workgroup keeps in registers: at 19K rows of 2 x 2 to 16 x 8 heads one workgroup per head takes 28 to 32 us, slices
// 37; at 43K rows 50 to 68 (its registers spill) against 37.
constexpr int kSliceRows = 8192;
EvictSlices slices_at(Arena &a, int64_t items, int budget, int cap) {
  EvictSlices sl{};
  if (cap <= 32 * kPlanThreads) return sl;
  const int r = (cap + 15) / 16;
  sl.rows = r > kSliceRows ? r : kSliceRows;
  sl.n1 = (budget + sl.rows - 1) / sl.rows;
  sl.nslice = sl.n1 + (cap - budget + sl.rows - 1) / sl.rows;
  sl.hist = a.take<uint16_t>((size_t)items * sl.nslice * kSliceBins);
  sl.border = a.take<Border>((size_t)items * 3);
  sl.above = a.take<int>((size_t)items * (sl.nslice + 1) * 4);
  return sl;
}

int log2i(int x) { return 31 - __builtin_clz((unsigned)x); }

template <typename F>
void by_type(int dtype, int d, F f) {
  if (dtype == RS_BF16)
    d == 128 ? f(bf16{}, std::integral_constant<int, 128>{}) : f(bf16{}, std::integral_constant<int, 64>{});
  else
    d == 128 ? f(float{}, std::integral_constant<int, 128>{}) : f(float{}, std::integral_constant<int, 64>{});
}

}  // namespace

rs_status append_launch(const CacheView &c, int dtype, int d, const void *kn, const void *vn, int64_t skt, int64_t skh,
                        int64_t svt, int64_t svh, const int32_t *start, int nrows, int max_rows, hipStream_t st) {
  // max_rows is also the distance of the sequences' rows without `start`; no sequence takes more than cap of them
  const int e = dtype == RS_BF16 ? 2 : 4, most = max_rows < c.cap ? max_rows : c.cap;
  append_kernel<<<dim3((most + kAppendRows - 1) / kAppendRows, c.nseq), 256, 0, st>>>(
      c, (const char *)kn, (const char *)vn, skt * e, skh * e, svt * e, svh * e, start, nrows, max_rows, log2i(d * e / 16));
  RS_HIP(hipGetLastError());
  return RS_OK;
}

rs_status commit_launch(const CacheView &c, int dtype, int d, const int32_t *naccept, const int32_t *path, int max_new,
                        hipStream_t st) {
  by_type(dtype, d, [&](auto t, auto dd) {
    using T = decltype(t);
    constexpr int D = decltype(dd)::value;
    if (max_new <= kMaxDraft) {
      commit_kernel<T, D><<<c.nseq, kCommitThreads, 0, st>>>(c, naccept, path, max_new);
      return;
    }
    if (c.pos || c.kmean)
      commit_rows_kernel<T, D><<<dim3((max_new / 64 + 2 + 3) / 4, c.hkv, c.nseq), 256, 0, st>>>(c, naccept, max_new);
    commit_len_kernel<<<(c.nseq + 63) / 64, 64, 0, st>>>(c, naccept, max_new);
  });
  RS_HIP(hipGetLastError());
  return RS_OK;
}

size_t evict_ws_bytes(int64_t items, int budget, int cap) {
  Arena a(nullptr, 0);
  plan_at(a, items, budget, cap);
  if (budget < cap) slices_at(a, items, budget, cap);
  return a.off + 256;
}

rs_status evict_launch(const CacheView &c, int dtype, int d, int budget, int nsink, int nrecent, void *ws, size_t ws_bytes,
                       hipStream_t st) {
  if (budget >= c.cap) return RS_OK;  // no sequence can hold more
  Arena a(ws, ws_bytes);
  const EvictPlan pl = plan_at(a, (int64_t)c.nseq * c.hkv, budget, c.cap);
  const EvictSlices sl = slices_at(a, (int64_t)c.nseq * c.hkv, budget, c.cap);
  if (!ws || !a.ok())
    return fail(RS_ERR_WORKSPACE, "eviction workspace too small: need " + std::to_string(evict_ws_bytes((int64_t)c.nseq * c.hkv, budget, c.cap)));
  if (sl.nslice) {
    const dim3 grid(sl.nslice, c.hkv, c.nseq);
    evict_slice_kernel<0><<<grid, kPlanThreads, 0, st>>>(c, budget, nsink, nrecent, pl, sl);
    evict_slice_kernel<1><<<grid, kPlanThreads, 0, st>>>(c, budget, nsink, nrecent, pl, sl);
    evict_slice_kernel<2><<<grid, kPlanThreads, 0, st>>>(c, budget, nsink, nrecent, pl, sl);
    evict_slice_kernel<3><<<grid, kPlanThreads, 0, st>>>(c, budget, nsink, nrecent, pl, sl);
  } else {
    const dim3 grid(c.hkv, c.nseq);
    if (c.cap <= 4 * kPlanThreads)
      evict_plan_kernel<4><<<grid, kPlanThreads, 0, st>>>(c, budget, nsink, nrecent, pl);
    else if (c.cap <= 16 * kPlanThreads)
      evict_plan_kernel<16><<<grid, kPlanThreads, 0, st>>>(c, budget, nsink, nrecent, pl);
    else
      evict_plan_kernel<32><<<grid, kPlanThreads, 0, st>>>(c, budget, nsink, nrecent, pl);
  }
  const int e = dtype == RS_BF16 ? 2 : 4;
  evict_move_kernel<<<dim3((pl.most + kMoveRows - 1) / kMoveRows, c.hkv, c.nseq), 256, 0, st>>>(c, budget, pl, log2i(d * e / 16));
  if (c.kmean && budget >= 64)
    by_type(dtype, d, [&](auto t, auto dd) {
      evict_means_kernel<decltype(t), decltype(dd)::value><<<dim3((budget / 64 + 3) / 4, c.hkv, c.nseq), 256, 0, st>>>(c, budget, pl);
    });
  RS_HIP(hipGetLastError());
  return RS_OK;
}

}  // namespace rs
