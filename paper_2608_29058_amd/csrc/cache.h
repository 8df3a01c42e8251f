// The key/value cache as the decoding kernels see it: addresses of rows, the rows of a sequence.
// The address arithmetic is plain C++ and compiles for the host too.
#pragma once

#include <stdint.h>

#if defined(__HIPCC__)
#define RS_HD __host__ __device__ __forceinline__
#else
#define RS_HD inline
#endif

namespace rs {

constexpr int kMaxDraft = 256;  // drafted rows of one sequence

// rs_cache by value: strides in bytes.
struct CacheView {
  char *k, *v;
  int64_t sk_p, sk_h, sk_t, sv_p, sv_h, sv_t;
  const int32_t *table;
  int32_t *len;
  int32_t nseq, hkv, page;
  uint32_t pmul;                   // ceil(2^31 / (page / 64)), 0 where a sequence has one page: see page_of
  int32_t npages, max_pages, cap, kblocks;  // kblocks: blocks of 64 rows per page (the last may be partial)
  void *kmean;
  float *acc;
  int32_t *pos, *seen;
};

RS_HD int clampi(int x, int lo, int hi) { return x < lo ? lo : x > hi ? hi : x; }

// Rows that sequence b holds.
RS_HD int cache_len(const CacheView &c, int b) { return clampi(c.len[b], 0, c.cap); }

// j / page by a multiplication: with B = page / 64 and M = ceil(2^31 / B), 2 (j / 64) M / 2^32 lies above
// (j / 64) / B by less than (j / 64) B / (2^31 B) < 2^-19 < 1 / B, since j / 64 and B are at most 2^12.
RS_HD int page_of(const CacheView &c, int j) { return (int)(((uint64_t)((uint32_t)(j >> 6) * 2u) * c.pmul) >> 32); }
RS_HD uint32_t page_mul(int page, int max_pages) {
  return max_pages == 1 ? 0u : (uint32_t)(((1ull << 31) + (uint64_t)(page / 64) - 1) / (uint64_t)(page / 64));
}

// The page that `entry` of the table names; -1: none.
RS_HD int checked_page(const CacheView &c, int entry) { return entry >= 0 && entry < c.npages ? entry : -1; }

// Page id of page p of sequence b, -1 where the table names none.
RS_HD int page_id(const CacheView &c, int b, int p) {
  const int64_t at = (int64_t)b * c.max_pages + p;
  return checked_page(c, c.table ? c.table[at] : (int)at);
}

// Byte offset of row j (in page p with id `id`) of head g in K and V.
RS_HD int64_t k_offset(const CacheView &c, int id, int p, int j, int g) {
  return id * c.sk_p + g * c.sk_h + (int64_t)(j - p * c.page) * c.sk_t;
}
RS_HD int64_t v_offset(const CacheView &c, int id, int p, int j, int g) {
  return id * c.sv_p + g * c.sv_h + (int64_t)(j - p * c.page) * c.sv_t;
}

// Element offset of the mean of block `blk` (64 rows) of head g, in page p with id `id`.
RS_HD int64_t mean_offset(const CacheView &c, int id, int p, int blk, int g, int d) {
  return (((int64_t)id * c.hkv + g) * c.kblocks + (blk - p * (c.page >> 6))) * d;
}

// First row and number of rows of sequence b in a batch of new rows, whatever `start` holds.
struct RowRange {
  int first, count;
};
RS_HD RowRange new_rows(const int32_t *start, int b, int nrows, int max_rows) {
  const int64_t s0 = start ? start[b] : (int64_t)b * max_rows, s1 = start ? start[b + 1] : s0 + max_rows;
  const int f = s0 < 0 ? 0 : s0 > nrows ? nrows : (int)s0, e = s1 < f ? f : s1 > nrows ? nrows : (int)s1;
  return RowRange{f, e - f < max_rows ? e - f : max_rows};
}

// rs_draft by value: strides in elements.
struct DraftView {
  const void *q;
  int32_t hq, nrows, max_rows, nwords;
  int64_t sq_t, sq_h;
  const int32_t *start;
  const uint32_t *mask;
  float c;  // logit scale times log2(e)
};

#if defined(__HIPCC__)
// Inclusive prefix sum over the wave: DPP row shifts, then the rows' last lanes broadcast (six adds; __shfl_up
// goes through LDS, 100 cycles a step).
template <int CTRL, int ROWS>
__device__ __forceinline__ int dpp_or_0(int x) {
  return __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false);
}
__device__ __forceinline__ int wave_scan(int x) {
  x += dpp_or_0<0x111, 0xf>(x);
  x += dpp_or_0<0x112, 0xf>(x);
  x += dpp_or_0<0x114, 0xf>(x);
  x += dpp_or_0<0x118, 0xf>(x);
  x += dpp_or_0<0x142, 0xa>(x);
  x += dpp_or_0<0x143, 0xc>(x);
  return x;
}
__device__ __forceinline__ int wave_sum(int x) { return __builtin_amdgcn_readlane(wave_scan(x), 63); }

// Exclusive prefix sum of x over the NT threads of a workgroup, and the total; sw: NT / 64 words of LDS.
template <int NT>
__device__ __forceinline__ int block_scan(int x, int *sw, int *total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int s = wave_scan(x);
  if (lane == 63) sw[w] = s;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int k = 0; k < NT / 64; ++k) {
    const int y = sw[k];
    before += k < w ? y : 0;
    all += y;
  }
  __syncthreads();
  *total = all;
  return before + s - x;
}
#endif

}  // namespace rs
