"""fp64 reference of decoding over a key/value cache: pages, drafted rows, selected blocks, accumulated
weights, eviction and cache updates.  Plain loops over sequences, heads and rows."""
import numpy as np


def cache_rows(x, table, page, b, g, n):
    """Rows 0 .. n - 1 of sequence b, head g of pages x [npages, hkv, page, d], and which of them lie in a page."""
    out = np.zeros((n, x.shape[3]), np.float64)
    ok = np.zeros(n, bool)
    for j in range(n):
        p = int(table[b, j // page])
        if 0 <= p < x.shape[0]:
            out[j] = x[p, g, j % page]
            ok[j] = True
    return out, ok


def row_ranges(start, nseq, nrows, max_rows):
    """(first, count) of every sequence's new rows, whatever start holds."""
    if start is None:
        start = [b * max_rows for b in range(nseq + 1)]
    out = []
    for b in range(nseq):
        f = min(max(int(start[b]), 0), nrows)
        e = min(max(int(start[b + 1]), f), nrows)
        out.append((f, min(e - f, max_rows)))
    return out


def seen_drafts(mask, row, i, count):
    """Which of the `count` drafted rows the i-th one (row `row` of the batch) sees."""
    if mask is None:
        return np.arange(count) <= i
    words = np.ascontiguousarray(mask[row]).view(np.uint32)
    return np.array([bool(int(words[j >> 5]) >> (j & 31) & 1) for j in range(count)], bool)


def softmax_row(q, k, v, see, scale):
    """O, lse, the weights, sum p |v| and the largest sum |q_d k_d| scale of one row; k, v: its seen rows."""
    if not see.any():
        return np.zeros(v.shape[1]), -np.inf, np.zeros(len(see)), np.zeros(v.shape[1]), 0.0
    l = np.full(len(see), -np.inf)
    l[see] = k[see] @ q * scale
    m = l.max()
    p = np.exp(l - m)
    z = p.sum()
    p /= z
    span = float((np.abs(k[see]) @ np.abs(q)).max() * scale)
    return p[see] @ v[see], m + np.log(z), p, p[see] @ np.abs(v[see]), span


def draft(q, k, v, lens, table, page, rows, mask, cap, scale, blocks=None):
    """Attention of the drafted rows: dict of o [nrows, hq, d], lse [hq, nrows], abs (sum p |v|), span, and
    weights {(b, g): [nrows of b][heads of g][rows]}.  blocks: {(row, g): selected blocks}."""
    nrows, hq, d = q.shape
    hkv = k.shape[1]
    G = hq // hkv
    o = np.full((nrows, hq, d), np.nan)
    lse = np.full((hq, nrows), np.nan)
    ab = np.zeros((nrows, hq, d))
    span = 0.0
    W = {}
    for b, (f, t) in enumerate(rows):
        n = min(max(int(lens[b]), 0), cap)
        total = min(n + t, cap)
        for g in range(hkv):
            if t == 0:
                continue
            kk, ok = cache_rows(k, table, page, b, g, total)
            vv, _ = cache_rows(v, table, page, b, g, total)
            for i in range(t):
                see = ok.copy()
                see[n:total] &= seen_drafts(mask, f + i, i, t)[:total - n]
                if blocks is not None:
                    on = np.zeros(total, bool)
                    on[n // 64 * 64:] = True
                    for c in blocks[f + i, g]:
                        on[c * 64:c * 64 + 64] = True
                    see &= on
                for h in range(g * G, g * G + G):
                    r = softmax_row(q[f + i, h], kk, vv, see, scale)
                    o[f + i, h], lse[h, f + i], ab[f + i, h] = r[0], r[1], r[3]
                    W.setdefault((b, g), {})[i, h] = r[2]
                    span = max(span, r[4])
    return dict(o=o, lse=lse, abs=ab, span=span, weights=W)


def block_means(k):
    """[npages, hkv, page // 64, d] means of complete blocks in fp64."""
    n, h, page, d = k.shape
    m = page // 64
    return k[:, :, :m * 64].reshape(n, h, m, 64, d).mean(3)


def select(q, kmean, lens, table, page, rows, nsel, nsink, nlocal, cap):
    """{(row, g): selected blocks, ascending}; kmean [npages, hkv, blocks, d]."""
    hq, hkv = q.shape[1], kmean.shape[1]
    G = hq // hkv
    out = {}
    for b, (f, t) in enumerate(rows):
        F = min(max(int(lens[b]), 0), cap) // 64
        for i in range(t):
            for g in range(hkv):
                sc = np.zeros(F)
                for c in range(F):
                    p = int(table[b, c * 64 // page])
                    m = kmean[p, g, c * 64 % page // 64] if 0 <= p < kmean.shape[0] else np.zeros(q.shape[2])
                    sc[c] = max(float(m @ q[f + i, h]) for h in range(g * G, g * G + G))
                c = np.arange(F)
                must = (c < nsink) | (c >= F - nlocal)
                out[f + i, g] = np.sort(np.lexsort((c, -sc, ~must))[:nsel])
    return out


def evict(acc, pos, seen, n, budget, nsink, nrecent):
    """(places that become free, rows that move there) of one sequence and head, in order."""
    if n <= budget:
        return np.zeros(0, int), np.zeros(0, int)
    must = (pos[:n] < nsink) | (pos[:n] >= seen - nrecent)
    key = np.where(must, np.inf, acc[:n].astype(np.float64))  # firm rows rank alike: more than the budget, the lower ones
    neg = np.signbit(acc[:n]) & ~must  # -0.0 comes after +0.0
    stay = np.lexsort((np.arange(n), neg, -key, ~must))[:budget]
    return np.setdiff1d(np.arange(budget), stay), np.sort(stay[stay >= budget])


def cross(q, k, v, lens, table, page, rows, kmask, cap, scale):
    """Attention of a decoder's rows over the cached rows that kmask [nseq, words] (or None) leaves: dict of o, lse,
    abs and span as of draft()."""
    nrows, hq, d = q.shape
    hkv = k.shape[1]
    G = hq // hkv
    o, lse, ab, span = np.full((nrows, hq, d), np.nan), np.full((hq, nrows), np.nan), np.zeros((nrows, hq, d)), 0.0
    for b, (f, t) in enumerate(rows):
        n = min(max(int(lens[b]), 0), cap)
        bits = np.ones(n, bool) if kmask is None else seen_drafts(kmask, b, 0, n)
        for g in range(hkv):
            if t == 0:
                continue
            kk, ok = cache_rows(k, table, page, b, g, n)
            vv, _ = cache_rows(v, table, page, b, g, n)
            for i in range(t):
                for h in range(g * G, g * G + G):
                    r = softmax_row(q[f + i, h], kk, vv, ok & bits, scale)
                    o[f + i, h], lse[h, f + i], ab[f + i, h] = r[0], r[1], r[3]
                    span = max(span, r[4])
    return dict(o=o, lse=lse, abs=ab, span=span)
