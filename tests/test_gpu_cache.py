"""The cache around the attention: rows written and kept (rs_cache_append, rs_cache_commit), accumulated
weights (rs_attn_weights) and eviction (rs_cache_evict) against the fp64 oracle; copies are exact."""
import numpy as np
import pytest

from oracle import decode as OD
from paper_2608_29058_amd import _rs
from decode_helpers import Setup, check_rows, logit_error

pytestmark = pytest.mark.gpu


class Book:
    """acc, pos, seen and block means of a Setup, as numpy and on the device."""

    def __init__(self, s, seed=0, seen=None):
        import torch
        r = np.random.default_rng(seed)
        n = len(s.lens)
        self.acc = r.random((n, s.hkv, s.cap)).astype(np.float32)
        self.pos = np.stack([[r.permutation(s.cap) for _ in range(s.hkv)] for _ in range(n)]).astype(np.int32)
        self.seen = np.array(s.lens if seen is None else seen, np.int32)
        self.kmean, self.dmean = s.means()
        up = lambda x: torch.from_numpy(x.copy()).cuda()
        self.dacc, self.dpos, self.dseen = up(self.acc), up(self.pos), up(self.seen)

    def args(self):
        return dict(kmean=self.dmean, acc=self.dacc, pos=self.dpos, seen=self.dseen)


def place(s, b, j):
    return int(s.table[b, j // s.page]), j % s.page


def same_rows(s, k, v):
    """Whole pools, bit for bit (numpy against the device)."""
    assert np.array_equal(s.dk.float().cpu().numpy(), k) and np.array_equal(s.dv.float().cpu().numpy(), v)


@pytest.mark.parametrize("dtype,d,page,layout,lens,rows,max_new,path", [
    ("bf16", 128, 64, "head", [0, 63, 64, 100, 127], [1, 1, 1, 1, 1], 1, False),
    ("bf16", 64, 128, "token", [0, 5, 127, 60], [3, 16, 9, 70], 70, True),
    ("f32", 128, 64, "head", [10, 0], [256, 130], 256, True),
    ("f32", 64, 64, "token", [0, 700, 63], [300, 1000, 2], 1000, False),   # a prompt's worth of rows
    ("bf16", 128, 192, "head", [100, 0], [600, 0], 600, False),
])
def test_append_then_commit(dtype, d, page, layout, lens, rows, max_new, path):
    import torch
    s = Setup(sum(rows) + d, lens, rows, d=d, dtype=dtype, page=page, layout=layout, extra=2)
    bk = Book(s, 1, seen=[7 * i + l for i, l in enumerate(lens)])
    c = s.cache(**bk.args())
    r = np.random.default_rng(5)
    td = s.dk.dtype
    new = [torch.from_numpy(r.standard_normal((s.nrows, s.hkv, d + 8)).astype(np.float32)).to(td).cuda()[..., :d] for _ in range(2)]
    _rs.rs_cache_append(c, new[0], new[1], max_rows=max(rows), start=s.dstart)
    k, v, acc, pos = s.k.copy(), s.v.copy(), bk.acc.copy(), bk.pos.copy()
    nk, nv = (x.float().cpu().numpy() for x in new)
    for b, (f, t) in enumerate(OD.row_ranges(s.start, len(lens), s.nrows, max(rows))):
        for i in range(t):
            p, j = place(s, b, lens[b] + i)
            k[p, :, j], v[p, :, j] = nk[f + i], nv[f + i]
            acc[b, :, lens[b] + i] = 0
    same_rows(s, k, v)
    assert np.array_equal(bk.dacc.cpu().numpy(), acc) and np.array_equal(s.dlen.cpu().numpy(), s.lens)
    # accepted: about half of the rows, or all
    bk.dacc.add_(1.0)
    acc = bk.dacc.cpu().numpy()
    na = np.array([t - t // 2 if path else t for t in rows], np.int32)
    pt = np.zeros((len(lens), max_new), np.int32)
    for b, t in enumerate(rows):
        pt[b, :na[b]] = np.sort(r.choice(t, na[b], replace=False))
    dpath = torch.from_numpy(pt).cuda() if path else None
    _rs.rs_cache_commit(c, torch.from_numpy(na).cuda(), max_new, path=dpath)
    kmean = bk.kmean.copy()
    for b, n in enumerate(lens):
        src = [int(x) if path else i for i, x in enumerate(pt[b, :na[b]])]
        rk = [k[place(s, b, n + x)[0], :, place(s, b, n + x)[1]].copy() for x in src]
        rv = [v[place(s, b, n + x)[0], :, place(s, b, n + x)[1]].copy() for x in src]
        acc[b][:, n:n + na[b]] = acc[b][:, [n + x for x in src]]
        for i in range(na[b]):
            p, j = place(s, b, n + i)
            k[p, :, j], v[p, :, j] = rk[i], rv[i]
            pos[b, :, n + i] = bk.seen[b] + i
        for blk in range(n // 64, (n + na[b]) // 64):
            p, j = place(s, b, blk * 64)
            m = k[p, :, j:j + 64].astype(np.float64).mean(1)
            kmean[p, :, j // 64] = torch.from_numpy(m).to(torch.bfloat16).double().numpy()
    same_rows(s, k, v)
    assert np.array_equal(bk.dacc.cpu().numpy(), acc) and np.array_equal(bk.dpos.cpu().numpy(), pos)
    assert np.array_equal(s.dlen.cpu().numpy(), s.lens + na) and np.array_equal(bk.dseen.cpu().numpy(), bk.seen + na)
    assert np.array_equal(bk.dmean.double().cpu().numpy(), kmean)


def test_append_and_commit_stop_at_the_capacity_and_at_missing_pages():
    import torch
    s = Setup(3, [60, 50], [2, 2], d=64, page=64)
    s.table[1, 0] = s.k.shape[0]                    # names no page
    s.dtable.copy_(torch.from_numpy(s.table))
    c = s.cache(seen=torch.zeros(2, dtype=torch.int32, device="cuda"))
    assert c.cap == 64
    new = torch.ones((20, s.hkv, 64), dtype=torch.bfloat16, device="cuda")
    start = torch.tensor([0, 10, 20], dtype=torch.int32, device="cuda")
    _rs.rs_cache_append(c, new, new, max_rows=10, start=start)
    k, v = s.k.copy(), s.v.copy()
    p = int(s.table[0, 0])
    k[p, :, 60:], v[p, :, 60:] = 1, 1
    same_rows(s, k, v)
    # path entries that do not ascend or lie outside are read as the row's own
    path = torch.tensor([[0, -4, 99, 1, 2, 0, 0, 0, 0, 0]] * 2, dtype=torch.int32, device="cuda")
    na = torch.tensor([99, -1], dtype=torch.int32, device="cuda")
    _rs.rs_cache_commit(c, na, 10, path=path)
    same_rows(s, k, v)
    assert s.dlen.tolist() == [64, 50] and c.seen.tolist() == [4, 0]
    _rs.rs_cache_commit(c, na, 400)
    assert s.dlen.tolist() == [64, 50]


@pytest.mark.parametrize("hq,hkv,d,dtype,lens,rows,kind,page", [
    (8, 2, 128, "bf16", [0, 1, 70, 600], [1, 1, 1, 1], None, 64),
    (28, 4, 64, "bf16", [300, 33], [3, 5], None, 128),
    (8, 1, 128, "f32", [130, 64], [9, 20], "tree", 64),
    (16, 16, 64, "f32", [90], [4], "random", 64),
    (4, 2, 128, "bf16", [700, 0, 40], [40, 3, 0], "random", 64),
    (24, 2, 64, "bf16", [200, 3], [90, 40], "tree", 64),      # 1080 rows of Q per head: in parts
    (12, 1, 128, "f32", [70], [50], None, 128),
    (4, 2, 64, "bf16", [9, 2100] * 40, [1] * 80, None, 64),   # more sequences than a wave has lanes
    (8, 2, 128, "f32", [2000, 1, 500], [8, 2, 5], "tree", 64),       # 32 rows of Q
    (14, 2, 64, "f32", [1111, 64], [3, 4], None, 64),                # 28
    (16, 2, 128, "f32", [1500, 0, 77], [8, 3, 6], "random", 128),    # 64
    (7, 1, 64, "f32", [2049, 31], [9, 8], "tree", 64),               # 63
])
def test_weights(hq, hkv, d, dtype, lens, rows, kind, page):
    import torch
    s = Setup(hq + d, lens, rows, hq=hq, hkv=hkv, d=d, dtype=dtype, kind=kind, page=page, extra=1, spread=2.0)
    ref = s.oracle()
    r = np.random.default_rng(1)
    w = (r.random(s.nrows) * (r.random(s.nrows) < 0.7)).astype(np.float32)
    lse = torch.from_numpy(ref["lse"].astype(np.float32)).cuda()
    s.dq[w == 0] = float("nan") if dtype == "bf16" else float("inf")    # rows of weight 0 may hold anything
    acc = r.random((len(lens), hkv, s.cap)).astype(np.float32)
    dw, c = torch.from_numpy(w).cuda(), s.cache()
    for use_in in (True, False):
        out = torch.from_numpy(acc.copy()).cuda()
        _rs.rs_attn_weights(c, s.draft, lse, out if use_in else None, out, row_w=dw)
        got = out.cpu().numpy().astype(np.float64)
        dl = logit_error(dtype, d, ref["span"])
        for b, (f, t) in enumerate(s.rows):
            n = min(lens[b] + t, s.cap) if t else 0
            for g in range(hkv):
                add = np.zeros(n)
                for (i, h), p in ref["weights"].get((b, g), {}).items():
                    add += w[f + i] * p[:n]
                want = add + (acc[b, g, :n] if use_in else 0)
                # per term: the logit's error, the given lse's rounding (2^-24 |lse|) and the exponent's; then
                # the sum's steps
                lim = (dl + 2.0 ** -22 * (8 + np.abs(ref["lse"][np.isfinite(ref["lse"])]).max())) * add + \
                    2.0 ** -24 * (len(ref["weights"].get((b, g), {})) + 4) * want
                assert (np.abs(got[b, g, :n] - want) <= lim + 1e-37).all(), (b, g)
                assert np.array_equal(got[b, g, n:], acc[b, g, n:].astype(np.float64))


@pytest.mark.parametrize("dtype,d,page,layout,lens,budget,nsink,nrecent", [
    ("bf16", 128, 64, "head", [129, 128, 127, 0, 300], 128, 4, 16),
    ("f32", 64, 128, "token", [500, 90], 65, 0, 0),
    ("bf16", 64, 64, "head", [9000, 8193], 700, 10, 100),
    ("bf16", 64, 64, "head", [1000], 999, 0, 999),          # one row goes; all that stay are recent
    ("bf16", 128, 64, "head", [64, 200], 1, 1, 0),
])
def test_evict(dtype, d, page, layout, lens, budget, nsink, nrecent):
    s = Setup(d + budget, lens, [0] * len(lens), d=d, dtype=dtype, page=page, layout=layout)
    bk = Book(s, 2, seen=[x + 5 for x in lens])
    c = s.cache(**bk.args())
    _rs.rs_cache_evict(c, budget, nsink, nrecent, _rs.workspace(_rs.rs_cache_evict_workspace_size(c, budget)))
    check_evicted(s, bk, lens, budget, nsink, nrecent)


def check_evicted(s, bk, lens, budget, nsink, nrecent):
    import torch
    k, v, acc, pos, kmean = s.k.copy(), s.v.copy(), bk.acc.copy(), bk.pos.copy(), bk.kmean.copy()
    for b, n in enumerate(lens):
        for g in range(s.hkv):
            free, come = OD.evict(bk.acc[b, g], bk.pos[b, g], int(bk.seen[b]), n, budget, nsink, nrecent)
            assert len(free) == len(come)
            for to, fr in zip(free, come):
                (pt, jt), (pf, jf) = place(s, b, to), place(s, b, fr)
                k[pt, g, jt], v[pt, g, jt] = k[pf, g, jf], v[pf, g, jf]
                acc[b, g, to], pos[b, g, to] = acc[b, g, fr], pos[b, g, fr]
            for blk in set((free // 64).tolist()):
                if blk * 64 + 64 <= budget:
                    p, j = place(s, b, blk * 64)
                    m = torch.from_numpy(k[p, g, j:j + 64].astype(np.float64).mean(0))
                    kmean[p, g, j // 64] = m.to(torch.bfloat16).double().numpy()
    same_rows(s, k, v)
    assert np.array_equal(bk.dacc.cpu().numpy().view(np.int32), acc.view(np.int32)) and np.array_equal(bk.dpos.cpu().numpy(), pos)
    assert np.array_equal(s.dlen.cpu().numpy(), np.minimum(lens, budget))
    assert np.array_equal(bk.dmean.double().cpu().numpy(), kmean)


@pytest.mark.parametrize("kind", ["equal", "few", "zeros", "tiny"])
def test_evict_with_equal_weights(kind):
    """Ties go to the lower row, -0.0 comes after +0.0, and weights that share their leading bits are told apart."""
    import torch
    s = Setup(4, [5000, 700], [0, 0], d=64)
    bk = Book(s, 3)
    r = np.random.default_rng(9)
    n = bk.acc.shape
    bk.acc = {"equal": np.full(n, 0.25, np.float32),
              "few": r.choice(np.array([0.5, 0.25, 3.0], np.float32), n),
              "zeros": r.choice(np.array([0.0, -0.0], np.float32), n),
              "tiny": (1.0 + r.integers(0, 900, n) * 2.0 ** -23).astype(np.float32)}[kind].astype(np.float32)
    bk.dacc.copy_(torch.from_numpy(bk.acc))
    c = s.cache(**bk.args())
    _rs.rs_cache_evict(c, 600, 3, 50, _rs.workspace(_rs.rs_cache_evict_workspace_size(c, 600)))
    check_evicted(s, bk, [5000, 700], 600, 3, 50)


@pytest.mark.parametrize("lens,budget,nsink,nrecent,kind", [
    ([70001, 8193], 8192, 100, 1000, "random"),
    ([40000, 17000], 20001, 0, 7, "few"),        # ties across slices of rows, on both sides of the budget
    ([33333], 33332, 5, 300, "tiny"),
    ([32000, 9000], 15000, 5, 300, "few"),
    ([20000, 100, 16500], 100, 4, 10, "equal"),
    ([150000], 60000, 0, 0, "random"),           # slices longer than 8K rows
])
def test_long_caches(lens, budget, nsink, nrecent, kind):
    import torch
    s = Setup(4, lens, [0] * len(lens), hq=1, hkv=1, d=64, page=1024)
    bk = Book(s, 3)
    r = np.random.default_rng(9)
    n = bk.acc.shape
    if kind != "random":
        bk.acc = {"equal": np.full(n, 0.25), "few": r.choice([0.5, 0.25, 3.0], n),
                  "tiny": 1.0 + r.integers(0, 900, n) * 2.0 ** -23}[kind].astype(np.float32)
        bk.dacc.copy_(torch.from_numpy(bk.acc))
    c = s.cache(**bk.args())
    _rs.rs_cache_evict(c, budget, nsink, nrecent, _rs.workspace(_rs.rs_cache_evict_workspace_size(c, budget)))
    check_evicted(s, bk, lens, budget, nsink, nrecent)


def test_evict_skips_rows_without_a_page_and_replays():
    import torch
    s = Setup(4, [400, 64], [0, 0], d=64)
    bk = Book(s, 3)
    s.table[0, 1] = -1
    s.dtable.copy_(torch.from_numpy(s.table))
    c = s.cache(**bk.args())
    ws = _rs.workspace(_rs.rs_cache_evict_workspace_size(c, 100))
    _rs.rs_cache_evict(c, 100, 0, 0, ws)
    k = s.k.copy()
    got = s.dk.float().cpu().numpy()
    used = {int(x) for x in s.table[0] if x >= 0}
    for p in range(k.shape[0]):
        if p not in used:
            assert np.array_equal(got[p], k[p])
    assert s.dlen.tolist() == [100, 64]
    # a captured eviction, with new weights and lengths between the replays
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        _rs.rs_cache_evict(c, 100, 4, 10, ws)
    r = torch.Generator(device="cuda").manual_seed(3)
    for n in (400, 101, 333):
        bk.dacc.copy_(torch.rand(bk.acc.shape, device="cuda", generator=r))
        state = (s.dk, s.dv, bk.dacc, bk.dpos, s.dlen, bk.dmean)
        s.dlen[0] = n
        before = [x.clone() for x in state]
        _rs.rs_cache_evict(c, 100, 4, 10, ws)
        want = [x.clone() for x in state]
        for x, y in zip(state, before):
            x.copy_(y)
        g.replay()
        torch.cuda.synchronize()
        for x, y in zip(state, want):
            assert torch.equal(x, y)


def test_decoding_after_a_prefill():
    """One program: a prompt prefilled into the cache, drafted rows attended, accepted and kept (each row equal to
    the prefill's row of the same tokens), weights accumulated, the cache evicted, decoding over blocks."""
    import torch
    from oracle import attention as A
    hq, hkv, d, n, total = 4, 2, 128, 300, 330
    r = np.random.default_rng(0)
    from synth import gen as G
    q, k, v = (G.bf16_round(r.standard_normal((h, total, d)).astype(np.float32)) for h in (hq, hkv, hkv))
    bf = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16).cuda()
    cap = 384
    pk, pv = (torch.zeros((1, hkv, cap, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    pk[0, :, :n], pv[0, :, :n] = bf(k[:, :n]), bf(v[:, :n])
    # the prefill reads the cache's page as its K and V
    qd = bf(q)
    qkv = _rs.make_qkv(qd[:, :n], pk[0, :, :n], pv[0, :, :n])
    o = torch.zeros((hq, n, d), dtype=torch.bfloat16, device="cuda")
    units = _rs.make_units([(h, 0, n) for h in range(hq)])
    _rs.rs_dense_attn_prefill(qkv, units, hq, o, None, _rs.workspace(_rs.rs_attn_workspace_size(qkv, units, hq)))
    i32 = dict(dtype=torch.int32, device="cuda")
    length, seen = torch.zeros(1, **i32), torch.zeros(1, **i32)
    acc, pos = torch.zeros((1, hkv, cap), device="cuda"), torch.full((1, hkv, cap), -1, **i32)
    kmean = torch.zeros((1, hkv, cap // 64, d), dtype=torch.bfloat16, device="cuda")
    c = _rs.KvCache(pk, pv, length, kmean=kmean, acc=acc, pos=pos, seen=seen)
    _rs.rs_cache_commit(c, torch.tensor([n], **i32), n)
    assert length.item() == n and torch.equal(pos[0, 0, :n], torch.arange(n, **i32))
    ref = np.stack([A.dense_attention(q[h], k[h // 2], v[h // 2]) for h in range(hq)])   # [hq, total, d]
    at, step = n, 0
    while at < total:
        # two branches of up to three tokens: the true continuation at the odd rows, noise at the even ones
        m = min(3, total - at)
        rows = 2 * m
        mask = np.zeros((rows, 32), bool)
        for i in range(m):
            for b in (0, 1):
                mask[2 * i + b, [2 * x + b for x in range(i + 1)]] = True
        words = torch.from_numpy(np.packbits(mask, axis=1, bitorder="little").view(np.int32)).cuda()
        rep = lambda x: bf(np.repeat(x[:, at:at + m], 2, axis=1).transpose(1, 0, 2))
        qn, kn, vn = rep(q), rep(k), rep(v)
        kn[0::2].normal_(), vn[0::2].normal_()
        start = torch.tensor([0, rows], **i32)
        dr = _rs.Draft(qn, max_rows=rows, start=start, mask=words)
        _rs.rs_cache_append(c, kn, vn, max_rows=rows, start=start)
        out, lse = torch.zeros_like(qn), torch.zeros((hq, rows), device="cuda")
        _rs.rs_draft_attn(c, dr, out, lse, _rs.workspace(_rs.rs_draft_attn_workspace_size(c, dr)))
        got = out[1::2].float().cpu().numpy().transpose(1, 0, 2)
        assert np.abs(got - ref[:, at:at + m]).max() <= 2e-2
        _rs.rs_attn_weights(c, dr, lse, acc, acc, row_w=torch.tensor([0.0, 1.0] * m, device="cuda"))
        path = torch.arange(1, rows, 2, **i32)[None].contiguous()
        pad = torch.zeros((1, rows), **i32)
        pad[:, :m] = path
        _rs.rs_cache_commit(c, torch.tensor([m], **i32), rows, path=pad)
        at += m
        step += 1
    assert length.item() == total == seen.item()
    assert torch.equal(pk[0, :, :total], bf(k)) and torch.equal(pv[0, :, :total], bf(v))
    want = kmean.clone()
    want[0, :, :total // 64] = pk[0, :, :total // 64 * 64].view(hkv, -1, 64, d).double().mean(2).to(torch.bfloat16)
    assert torch.equal(kmean, want)
    # every drafted row that was accepted spread a weight of 1 per query head over the rows it saw
    assert torch.allclose(acc[0, :, :total].sum(1), torch.full((hkv,), float((total - n) * hq // hkv), device="cuda"), rtol=1e-4)
    stay = [set(pos[0, g, :total][torch.argsort(acc[0, g, :total], descending=True, stable=True)].tolist()[:1]) for g in range(hkv)]
    _rs.rs_cache_evict(c, 200, 4, 64, _rs.workspace(_rs.rs_cache_evict_workspace_size(c, 200)))
    assert length.item() == 200 and seen.item() == total
    p = pos[0, :, :200].long()
    for g in range(hkv):
        have = set(p[g].tolist())
        assert len(have) == 200 and set(range(4)) <= have and set(range(total - 64, total)) <= have and stay[g] <= have
        assert torch.equal(pk[0, g, :200], bf(k)[g, p[g]]) and torch.equal(pv[0, g, :200], bf(v)[g, p[g]])
    # all blocks selected: the same as attention over everything that is left
    qn = bf(r.standard_normal((1, hq, d)))
    dr = _rs.Draft(qn)
    _rs.rs_cache_append(c, qn[:, :hkv].contiguous(), qn[:, :hkv].contiguous())
    a, b = torch.zeros_like(qn), torch.zeros_like(qn)
    _rs.rs_draft_attn(c, dr, a, None, _rs.workspace(_rs.rs_draft_attn_workspace_size(c, dr)))
    _rs.rs_select_attn(c, dr, 3, 0, 0, b, None, _rs.workspace(_rs.rs_select_attn_workspace_size(c, dr, 3)))
    assert (a.float() - b.float()).abs().max() <= 2.0 ** -7 * a.float().abs().max()
