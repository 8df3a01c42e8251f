// C entry points of the key/value cache and of the attention over it: argument checks and dispatch.
#include <hip/hip_runtime.h>

#include <cmath>
#include <string>

#include "common.h"
#include "draft_plan.h"
#include "rope.h"

namespace rs {

rs_status append_launch(const CacheView &c, int dtype, int d, const void *kn, const void *vn, int64_t skt, int64_t skh,
                        int64_t svt, int64_t svh, const int32_t *start, int nrows, int max_rows, hipStream_t st);
rs_status commit_launch(const CacheView &c, int dtype, int d, const int32_t *naccept, const int32_t *path, int max_new,
                        hipStream_t st);
size_t evict_ws_bytes(int64_t items, int budget, int cap);
rs_status evict_launch(const CacheView &c, int dtype, int d, int budget, int nsink, int nrecent, void *ws, size_t ws_bytes,
                       hipStream_t st);
size_t draft_ws_bytes(const CacheView &c, const DraftView &q, bool f32, int d, int nsel, int what);
rs_status draft_launch(const CacheView &c, const DraftView &q, bool f32, int d, int what, void *o, int64_t so_t, int64_t so_h,
                       float *lse, void *ws, size_t ws_bytes, hipStream_t st);
rs_status select_launch(const CacheView &c, const DraftView &q, bool f32, int d, int nsel, int nsink, int nlocal, void *o,
                        int64_t so_t, int64_t so_h, float *lse, int32_t *blocks, void *ws, size_t ws_bytes, hipStream_t st);
rs_status weights_launch(const CacheView &c, const DraftView &q, bool f32, int d, const float *lse, const float *row_w,
                         const float *acc_in, float *acc_out, hipStream_t st);

static bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }

static rs_status check_cache(const rs_cache *x, CacheView *c) {
  if (!x) return fail(RS_ERR_INVALID_ARG, "cache is NULL");
  if (!x->k || !x->v || !x->len) return fail(RS_ERR_INVALID_ARG, "cache: k, v or len is NULL");
  if (x->dtype != RS_BF16 && x->dtype != RS_F32) return fail(RS_ERR_INVALID_ARG, "cache: unknown dtype");
  if (x->d != 64 && x->d != 128) return fail(RS_ERR_UNSUPPORTED, "cache: head dim must be 64 or 128");
  if (x->nseq < 1 || x->nseq > 65535 || x->hkv < 1 || x->hkv > 4096)
    return fail(RS_ERR_INVALID_ARG, "cache: need 1 <= nseq <= 65535 and 1 <= hkv <= 4096");
  if (x->page < 1 || x->npages < 1 || x->max_pages < 1) return fail(RS_ERR_INVALID_ARG, "cache: page, npages and max_pages must be positive");
  if ((int64_t)x->page * x->max_pages > kMaxN) return fail(RS_ERR_UNSUPPORTED, "cache: at most 262144 rows per sequence");
  if (x->page % 64 != 0 && x->max_pages != 1)
    return fail(RS_ERR_UNSUPPORTED, "cache: a page holds a multiple of 64 rows, unless a sequence has only one");
  if (!x->table && (int64_t)x->nseq * x->max_pages > x->npages)
    return fail(RS_ERR_INVALID_ARG, "cache: without a table every sequence needs max_pages pages of its own");
  const int vec = x->dtype == RS_BF16 ? 8 : 4, e = x->dtype == RS_BF16 ? 2 : 4;
  const int64_t s[6] = {x->sk_p, x->sk_h, x->sk_t, x->sv_p, x->sv_h, x->sv_t};
  for (int i = 0; i < 6; ++i)
    if (s[i] < 0 || s[i] % vec != 0) return fail(RS_ERR_INVALID_ARG, "cache: strides must be non-negative multiples of 16 bytes");
  if (x->sk_t < x->d || x->sv_t < x->d) return fail(RS_ERR_INVALID_ARG, "cache: row stride smaller than head dim");
  if (x->sk_t * e > (1 << 24) || x->sv_t * e > (1 << 24)) return fail(RS_ERR_UNSUPPORTED, "cache: rows at most 16 MiB apart");
  if (!aligned16(x->k) || !aligned16(x->v) || !aligned16(x->kmean)) return fail(RS_ERR_INVALID_ARG, "cache: k, v and kmean must be 16-byte aligned");
  c->k = (char *)x->k;
  c->v = (char *)x->v;
  c->sk_p = x->sk_p * e, c->sk_h = x->sk_h * e, c->sk_t = x->sk_t * e;
  c->sv_p = x->sv_p * e, c->sv_h = x->sv_h * e, c->sv_t = x->sv_t * e;
  c->table = x->table;
  c->len = x->len;
  c->nseq = x->nseq, c->hkv = x->hkv, c->page = x->page;
  c->pmul = page_mul(x->page, x->max_pages);
  c->npages = x->npages, c->max_pages = x->max_pages, c->cap = x->page * x->max_pages;
  c->kblocks = (x->page + 63) / 64;
  c->kmean = x->kmean, c->acc = x->acc, c->pos = x->pos, c->seen = x->seen;
  return RS_OK;
}

// What rs_draft and rs_cross have in common: queries of new rows.
template <typename Y>
static rs_status check_queries(const rs_cache *x, const Y *y, int most_rows, const std::string &name, DraftView *q) {
  if (!y) return fail(RS_ERR_INVALID_ARG, name + " is NULL");
  if ((!y->q && y->nrows != 0) || !aligned16(y->q)) return fail(RS_ERR_INVALID_ARG, name + ": q must be a 16-byte aligned device pointer");
  if (y->hq < 1 || y->hq > 65535 || y->hq % x->hkv != 0) return fail(RS_ERR_INVALID_ARG, name + ": hq must be a positive multiple of hkv");
  if (y->nrows < 0 || y->max_rows < 1) return fail(RS_ERR_INVALID_ARG, name + ": nrows < 0 or max_rows < 1");
  if (y->max_rows > most_rows) return fail(RS_ERR_UNSUPPORTED, name + ": at most " + std::to_string(most_rows) + " new rows per sequence");
  if (y->nrows > (1 << 20)) return fail(RS_ERR_UNSUPPORTED, name + ": at most 1048576 new rows");
  if ((int64_t)x->nseq * y->hq * y->max_rows > (1 << 28))
    return fail(RS_ERR_UNSUPPORTED, name + ": at most 2^28 rows of queries (nseq x hq x max_rows)");
  if ((int64_t)y->nrows * x->hkv > (1 << 24)) return fail(RS_ERR_UNSUPPORTED, name + ": at most 2^24 new rows x key/value heads");
  if (!y->start && (int64_t)x->nseq * y->max_rows > y->nrows)
    return fail(RS_ERR_INVALID_ARG, name + ": without start every sequence has max_rows rows");
  const int vec = x->dtype == RS_BF16 ? 8 : 4;
  if (y->sq_t < 0 || y->sq_h < 0 || y->sq_t % vec || y->sq_h % vec) return fail(RS_ERR_INVALID_ARG, name + ": strides must be non-negative multiples of 16 bytes");
  float sc = y->scale;
  if (sc == 0.f) sc = 1.f / std::sqrt((float)x->d);
  if (!(sc > 0.f) || !std::isfinite(sc)) return fail(RS_ERR_INVALID_ARG, name + ": scale must be positive and finite");
  q->q = y->q;
  q->hq = y->hq, q->nrows = y->nrows, q->max_rows = y->max_rows, q->nwords = y->nwords;
  q->sq_t = y->sq_t, q->sq_h = y->sq_h;
  q->start = y->start;
  q->c = sc * kLog2e;
  return RS_OK;
}

static rs_status check_draft(const rs_cache *x, const rs_draft *y, DraftView *q) {
  rs_status st;
  if ((st = check_queries(x, y, kMaxDraft, "draft", q)) != RS_OK) return st;
  if (y->mask && (y->nwords < 1 || (int64_t)y->nwords * 32 < y->max_rows)) return fail(RS_ERR_INVALID_ARG, "draft: mask rows shorter than max_rows");
  q->mask = y->mask;
  return RS_OK;
}

static rs_status check_cross(const rs_cache *x, const rs_cross *y, DraftView *q) {
  rs_status st;
  if ((st = check_queries(x, y, 1 << 28, "cross", q)) != RS_OK) return st;
  if (y->kmask && (y->nwords < 1 || (int64_t)y->nwords * 32 < (int64_t)x->page * x->max_pages))
    return fail(RS_ERR_INVALID_ARG, "cross: key mask shorter than the cache's capacity");
  if ((uintptr_t)y->kmask & 3) return fail(RS_ERR_INVALID_ARG, "cross: kmask must be 4-byte aligned");
  q->mask = y->kmask;
  return RS_OK;
}

static rs_status check_rows_out(const void *o, int64_t so_t, int64_t so_h, int d) {
  if (!o) return fail(RS_ERR_INVALID_ARG, "output is NULL");
  if (((uintptr_t)o & 7) || so_t % 4 != 0 || so_h % 4 != 0 || so_t < d || so_h < d)
    return fail(RS_ERR_INVALID_ARG, "output must be 8-byte aligned with strides of at least d, multiples of 4 elements");
  return RS_OK;
}

// The new rows of an append.
static rs_status check_append(const rs_cache *cache, CacheView *c, const void *k_new, const void *v_new, int64_t sk_t, int64_t sk_h,
                              int64_t sv_t, int64_t sv_h, const int32_t *start, int32_t nrows, int32_t max_rows) {
  rs_status st;
  if ((st = check_cache(cache, c)) != RS_OK) return st;
  if (((!k_new || !v_new) && nrows != 0) || !aligned16(k_new) || !aligned16(v_new)) return fail(RS_ERR_INVALID_ARG, "append: k_new and v_new must be 16-byte aligned device pointers");
  const int vec = cache->dtype == RS_BF16 ? 8 : 4;
  const int64_t s[4] = {sk_t, sk_h, sv_t, sv_h};
  for (int i = 0; i < 4; ++i)
    if (s[i] < 0 || s[i] % vec != 0) return fail(RS_ERR_INVALID_ARG, "append: strides must be non-negative multiples of 16 bytes");
  if (nrows < 0 || max_rows < 1) return fail(RS_ERR_INVALID_ARG, "append: nrows < 0 or max_rows < 1");
  if (!start && (int64_t)c->nseq * max_rows > nrows) return fail(RS_ERR_INVALID_ARG, "append: without start every sequence has max_rows rows");
  return RS_OK;
}

static rs_status check_select(const rs_cache *x, int32_t nsel, int32_t nsink, int32_t nlocal) {
  if (!x->kmean) return fail(RS_ERR_INVALID_ARG, "select: the cache has no block means");
  if (nsel < 1 || nsink < 0 || nlocal < 0 || (int64_t)nsink + nlocal > nsel)
    return fail(RS_ERR_INVALID_ARG, "select: need nsel >= 1 and 0 <= nsink + nlocal <= nsel");
  if (nsel > kMaxN / 64) return fail(RS_ERR_UNSUPPORTED, "select: at most 4096 blocks");
  return RS_OK;
}

}  // namespace rs

using namespace rs;

extern "C" {

rs_status rs_cache_append(const rs_cache *cache, const void *k_new, const void *v_new, int64_t sk_t, int64_t sk_h,
                          int64_t sv_t, int64_t sv_h, const int32_t *start, int32_t nrows, int32_t max_rows,
                          rs_stream stream) {
  set_error("");
  CacheView c;
  rs_status st;
  if ((st = check_append(cache, &c, k_new, v_new, sk_t, sk_h, sv_t, sv_h, start, nrows, max_rows)) != RS_OK) return st;
  if (nrows == 0) return RS_OK;
  return append_launch(c, cache->dtype, cache->d, k_new, v_new, sk_t, sk_h, sv_t, sv_h, start, nrows, max_rows, (hipStream_t)stream);
}

rs_status rs_cache_append_rope(const rs_cache *cache, const rs_rope *rope, const void *k_new, const void *v_new, int64_t sk_t,
                               int64_t sk_h, int64_t sv_t, int64_t sv_h, const rs_rope_part *q, const int32_t *pos,
                               const int32_t *start, int32_t nrows, int32_t max_rows, rs_stream stream) {
  set_error("");
  CacheView c;
  rs_status st;
  if ((st = check_append(cache, &c, k_new, v_new, sk_t, sk_h, sv_t, sv_h, start, nrows, max_rows)) != RS_OK) return st;
  if ((st = check_rope(rope, cache->d)) != RS_OK) return st;
  if (nrows > 1 << 24) return fail(RS_ERR_UNSUPPORTED, "append: at most 16777216 rows to rotate");
  if (nrows == 0) return RS_OK;
  if (q && (st = check_rope_part(q, cache->dtype, cache->d, nrows, "append: q")) != RS_OK) return st;
  return append_rope_launch(c, cache->dtype, cache->d, *rope, k_new, v_new, sk_t, sk_h, sv_t, sv_h, q, pos, start, nrows, max_rows,
                            (hipStream_t)stream);
}

rs_status rs_cache_commit(const rs_cache *cache, const int32_t *naccept, const int32_t *path, int32_t max_new, rs_stream stream) {
  set_error("");
  CacheView c;
  rs_status st;
  if ((st = check_cache(cache, &c)) != RS_OK) return st;
  if (!naccept) return fail(RS_ERR_INVALID_ARG, "commit: naccept is NULL");
  if (max_new < 1 || max_new > kMaxN) return fail(RS_ERR_INVALID_ARG, "commit: need 1 <= max_new <= 262144");
  if (path && max_new > kMaxDraft) return fail(RS_ERR_UNSUPPORTED, "commit: a path has at most 256 rows");
  if (c.pos && !c.seen) return fail(RS_ERR_INVALID_ARG, "commit: positions need the cache's seen");
  return commit_launch(c, cache->dtype, cache->d, naccept, path, max_new, (hipStream_t)stream);
}

size_t rs_draft_attn_workspace_size(const rs_cache *cache, const rs_draft *draft) {
  CacheView c;
  DraftView q;
  if (check_cache(cache, &c) != RS_OK || check_draft(cache, draft, &q) != RS_OK) return 0;
  return draft_ws_bytes(c, q, cache->dtype == RS_F32, cache->d, 0, W_ALL);
}

rs_status rs_draft_attn(const rs_cache *cache, const rs_draft *draft, void *o, int64_t so_t, int64_t so_h, float *lse, void *ws,
                        size_t ws_bytes, rs_stream stream) {
  set_error("");
  CacheView c;
  DraftView q;
  rs_status st;
  if ((st = check_cache(cache, &c)) != RS_OK) return st;
  if ((st = check_draft(cache, draft, &q)) != RS_OK) return st;
  if (q.nrows == 0) return RS_OK;
  if ((st = check_rows_out(o, so_t, so_h, cache->d)) != RS_OK) return st;
  if (!aligned16(ws)) return fail(RS_ERR_WORKSPACE, "workspace must be 16-byte aligned");
  return draft_launch(c, q, cache->dtype == RS_F32, cache->d, W_ALL, o, so_t, so_h, lse, ws, ws_bytes, (hipStream_t)stream);
}

size_t rs_cross_attn_workspace_size(const rs_cache *cache, const rs_cross *cross) {
  CacheView c;
  DraftView q;
  if (check_cache(cache, &c) != RS_OK || check_cross(cache, cross, &q) != RS_OK) return 0;
  return draft_ws_bytes(c, q, cache->dtype == RS_F32, cache->d, 0, W_CROSS);
}

rs_status rs_cross_attn(const rs_cache *cache, const rs_cross *cross, void *o, int64_t so_t, int64_t so_h, float *lse, void *ws,
                        size_t ws_bytes, rs_stream stream) {
  set_error("");
  CacheView c;
  DraftView q;
  rs_status st;
  if ((st = check_cache(cache, &c)) != RS_OK) return st;
  if ((st = check_cross(cache, cross, &q)) != RS_OK) return st;
  if (q.nrows == 0) return RS_OK;
  if ((st = check_rows_out(o, so_t, so_h, cache->d)) != RS_OK) return st;
  if (!aligned16(ws)) return fail(RS_ERR_WORKSPACE, "workspace must be 16-byte aligned");
  return draft_launch(c, q, cache->dtype == RS_F32, cache->d, W_CROSS, o, so_t, so_h, lse, ws, ws_bytes, (hipStream_t)stream);
}

size_t rs_select_attn_workspace_size(const rs_cache *cache, const rs_draft *draft, int32_t nsel) {
  CacheView c;
  DraftView q;
  if (check_cache(cache, &c) != RS_OK || check_draft(cache, draft, &q) != RS_OK || nsel < 1 || nsel > kMaxN / 64) return 0;
  return draft_ws_bytes(c, q, cache->dtype == RS_F32, cache->d, nsel, W_SELECT);
}

rs_status rs_select_attn(const rs_cache *cache, const rs_draft *draft, int32_t nsel, int32_t nsink, int32_t nlocal, void *o,
                         int64_t so_t, int64_t so_h, float *lse, int32_t *blocks, void *ws, size_t ws_bytes, rs_stream stream) {
  set_error("");
  CacheView c;
  DraftView q;
  rs_status st;
  if ((st = check_cache(cache, &c)) != RS_OK) return st;
  if ((st = check_draft(cache, draft, &q)) != RS_OK) return st;
  if ((st = check_select(cache, nsel, nsink, nlocal)) != RS_OK) return st;
  if (q.nrows == 0) return RS_OK;
  if ((st = check_rows_out(o, so_t, so_h, cache->d)) != RS_OK) return st;
  if (!aligned16(ws)) return fail(RS_ERR_WORKSPACE, "workspace must be 16-byte aligned");
  return select_launch(c, q, cache->dtype == RS_F32, cache->d, nsel, nsink, nlocal, o, so_t, so_h, lse, blocks, ws, ws_bytes,
                       (hipStream_t)stream);
}

rs_status rs_attn_weights(const rs_cache *cache, const rs_draft *draft, const float *lse, const float *row_w, const float *acc_in,
                          float *acc_out, rs_stream stream) {
  set_error("");
  CacheView c;
  DraftView q;
  rs_status st;
  if ((st = check_cache(cache, &c)) != RS_OK) return st;
  if ((st = check_draft(cache, draft, &q)) != RS_OK) return st;
  if (q.nrows == 0) return RS_OK;
  if (!lse || !acc_out) return fail(RS_ERR_INVALID_ARG, "weights: lse or acc_out is NULL");
  return weights_launch(c, q, cache->dtype == RS_F32, cache->d, lse, row_w, acc_in, acc_out, (hipStream_t)stream);
}

size_t rs_cache_evict_workspace_size(const rs_cache *cache, int32_t budget) {
  CacheView c;
  if (check_cache(cache, &c) != RS_OK || budget < 1) return 0;
  return evict_ws_bytes((int64_t)c.nseq * c.hkv, budget, c.cap);
}

rs_status rs_cache_evict(const rs_cache *cache, int32_t budget, int32_t nsink, int32_t nrecent, void *ws, size_t ws_bytes,
                         rs_stream stream) {
  set_error("");
  CacheView c;
  rs_status st;
  if ((st = check_cache(cache, &c)) != RS_OK) return st;
  if (!c.acc || !c.pos || !c.seen) return fail(RS_ERR_INVALID_ARG, "evict: the cache needs acc, pos and seen");
  if (budget < 1 || nsink < 0 || nrecent < 0 || (int64_t)nsink + nrecent > budget)
    return fail(RS_ERR_INVALID_ARG, "evict: need budget >= 1 and 0 <= nsink + nrecent <= budget");
  if (!aligned16(ws)) return fail(RS_ERR_WORKSPACE, "workspace must be 16-byte aligned");
  return evict_launch(c, cache->dtype, cache->d, budget, nsink, nrecent, ws, ws_bytes, (hipStream_t)stream);
}

}  // extern "C"
