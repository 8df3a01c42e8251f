"""Rotated rows entering the cache (rs_cache_append_rope): K against the fp64 oracle and, bit for bit, against a rotation
followed by a plain append; pages, strides and positions of every kind; what lies elsewhere stays."""
import numpy as np
import pytest

from paper_2608_29058_amd import _rs
from decode_helpers import Setup, check_rows
from oracle import decode as OD
from oracle import rope as OR
from rope_helpers import Rot, bits, check, rows

pytestmark = pytest.mark.gpu


def append(s, rot, k, v, q=None, q_out=None, pos=None, seen=None, acc=None, **kw):
    c = s.cache(seen=seen, acc=acc)
    _rs.rs_cache_append_rope(c, rot.rope, k, v, q=q, q_out=q_out, pos=pos, max_rows=s.max_rows, start=s.dstart, **kw)
    return c


@pytest.mark.parametrize("hq,hkv,d,dtype,page,layout,lens,counts,dim,inter", [
    (8, 2, 128, "bf16", 64, "head", [0, 1, 63, 64, 200], [1, 1, 1, 1, 1], 128, False),
    (32, 8, 128, "bf16", 128, "token", [0, 100, 511], [3, 60, 1], 64, False),
    (28, 4, 64, "f32", 64, "token", [5, 0, 130], [13, 0, 7], 48, True),
    (4, 4, 64, "bf16", 192, "head", [190, 0], [5, 300], 64, True),
    (7, 1, 128, "f32", 64, "head", [64, 10], [70, 1], 10, False),
    (40, 40, 128, "bf16", 64, "head", [3], [2], 128, True),
    (2, 1, 64, "f32", 64, "token", [0, 900], [1000, 33], 62, False),
])
def test_rows_against_the_oracle(hq, hkv, d, dtype, page, layout, lens, counts, dim, inter):
    import torch
    s = Setup(sum(lens) + d, lens, counts, hq=hq, hkv=hkv, d=d, dtype=dtype, page=page, layout=layout, extra=3)
    rot = Rot(dim, inter, base=500000.0, mscale=1.1)
    k, kv = rows(1, s.nrows, hkv, d, dtype, "wide")
    v, vv = rows(2, s.nrows, hkv, d, dtype, "head")
    q, qv = rows(3, s.nrows, hq, d, dtype, "wide")
    r = np.random.default_rng(0)
    seen = s.lens + r.integers(0, 5000, len(lens)).astype(np.int32)
    own = r.integers(0, 200000, s.nrows).astype(np.int32)
    was_k, was_v = s.dk.clone(), s.dv.clone()
    for mode in ("pos", "seen", "len"):
        s.dk.copy_(was_k)
        s.dv.copy_(was_v)
        out = torch.full((s.nrows, hq, d), -7.0, dtype=q.dtype, device="cuda")
        acc = torch.full((len(lens), hkv, s.cap), 5.0, device="cuda")
        append(s, rot, k, v, q, out, pos=torch.from_numpy(own).cuda() if mode == "pos" else None,
               seen=torch.from_numpy(seen).cuda() if mode != "len" else None, acc=acc)
        pos = own.astype(np.int64)
        want_k, want_v, want_acc = s.k.astype(np.float64), s.v.astype(np.float64), np.full(acc.shape, 5.0)
        abk = np.zeros_like(want_k)
        used = np.zeros(s.nrows, bool)
        for b, (f, t) in enumerate(s.rows):
            if mode != "pos":
                pos[f:f + t] = (seen if mode == "seen" else s.lens)[b] + np.arange(t)
            used[f:f + t] = True
        y, ab = rot.oracle(kv, pos)
        for b, (f, t) in enumerate(s.rows):
            for i in range(t):
                j = int(s.lens[b]) + i
                at = s.table[b, j // page]
                want_k[at, :, j % page], abk[at, :, j % page], want_v[at, :, j % page] = y[f + i], ab[f + i], vv[f + i]
                want_acc[b, :, j] = 0.0
        check(s.dk.double().cpu().numpy(), want_k, abk, dtype, rot, pos)
        still = abk == 0  # other rows, and what does not turn, to the bit
        assert np.array_equal(s.dk.double().cpu().numpy()[still], want_k[still])
        assert np.array_equal(s.dv.double().cpu().numpy(), want_v)
        assert np.array_equal(acc.cpu().numpy(), want_acc)
        yq, abq = rot.oracle(qv, pos)
        got = out.double().cpu().numpy()
        check(got[used], yq[used], abq[used], dtype, rot, pos)
        assert (got[~used] == -7.0).all() and s.dlen.tolist() == list(lens)


@pytest.mark.parametrize("dtype,dim,inter", [("bf16", 128, False), ("f32", 64, True), ("bf16", 34, False)])
@pytest.mark.parametrize("lens,counts", [([0, 50, 127], [1, 1, 1]), ([10, 0], [300, 500])])
def test_as_a_rotation_and_a_plain_append(dtype, dim, inter, lens, counts):
    import torch
    s = Setup(7, lens, counts, hq=4, hkv=2, d=128, dtype=dtype, page=128)
    rot = Rot(dim, inter)
    k, v, q = (rows(i, s.nrows, h, 128, dtype)[0] for i, h in enumerate((2, 2, 4)))
    was = s.dk.clone(), s.dv.clone()
    pos = torch.cat([a + torch.arange(t, dtype=torch.int32, device="cuda") for a, t in zip(lens, counts)]).int()
    rk, rq = torch.empty_like(k), torch.empty_like(q)
    _rs.rs_rope_apply(rot.rope, _rs.RopeRows([(k, rk), (q, rq)], pos=pos))
    _rs.rs_cache_append(s.cache(), rk, v, max_rows=s.max_rows, start=s.dstart)
    want = s.dk.clone(), s.dv.clone()
    s.dk.copy_(was[0])
    s.dv.copy_(was[1])
    append(s, rot, k, v, q)  # q in place
    assert torch.equal(bits(s.dk), bits(want[0])) and torch.equal(bits(s.dv), bits(want[1])) and torch.equal(bits(q), bits(rq))
    s.dk.copy_(was[0])
    append(s, rot, k, v)     # no queries
    assert torch.equal(bits(s.dk), bits(want[0]))


def test_rows_behind_the_capacity_or_in_no_page_are_left_out():
    import torch
    s = Setup(1, [60, 120, 10], [10, 10, 10], hq=2, hkv=2, d=64, page=64)
    table = s.dtable.clone()
    table[0, 1] = -1                    # rows 64 .. of the first
    table[2, 0] = s.dk.shape[0]         # the third has no page at all
    lens = torch.tensor([60, 125, 10], dtype=torch.int32, device="cuda")   # the second ends at 128
    rot = Rot(64)
    k, v, q = (rows(i, 30, 2, 64, "bf16")[0] for i in range(3))
    was = s.dk.clone()
    c = _rs.KvCache(s.dk, s.dv, lens, table=table[:, :2].contiguous())
    out = torch.full_like(q, -7.0)
    _rs.rs_cache_append_rope(c, rot.rope, k, v, q=q, q_out=out, max_rows=10, start=s.dstart)
    pos = torch.tensor([a + i for a in (60, 125, 10) for i in range(10)], dtype=torch.int32, device="cuda")
    rk, rq = torch.empty_like(k), torch.empty_like(q)
    _rs.rs_rope_apply(rot.rope, _rs.RopeRows([(k, rk), (q, rq)], pos=pos))
    assert torch.equal(bits(out), bits(rq))  # queries of all of them
    want = was.clone()
    want[s.table[0, 0], :, 60:64] = rk[0:4].transpose(0, 1)
    want[s.table[1, 1], :, 61:64] = rk[10:13].transpose(0, 1)
    assert torch.equal(bits(s.dk), bits(want))


def test_absurd_starts_and_lengths_stay_in_bounds():
    """Clamped as in rs_cache_append: the same rows land in the same places."""
    import torch
    for start, lens in (([5, 2, 90], [3, 1]), ([-4, 3, 4], [-9, 1 << 30]), ([0, 1 << 30, -1], [100, 5])):
        res = []
        for rotated in (False, True):
            s = Setup(2, [70, 20], [8, 8], hq=2, hkv=2, d=64, page=64)
            s.dlen.copy_(torch.tensor(lens))
            st = torch.tensor(start, dtype=torch.int32, device="cuda")
            k, v = (rows(i, 16, 2, 64, "bf16")[0] for i in range(2))
            if rotated:
                _rs.rs_cache_append_rope(s.cache(), _rs.Rope(64, turns=[0.0] * 32), k, v, max_rows=6, start=st)
            else:
                _rs.rs_cache_append(s.cache(), k, v, max_rows=6, start=st)
            res.append((s.dk.clone(), s.dv.clone()))
        assert torch.equal(bits(res[0][0]), bits(res[1][0])) and torch.equal(bits(res[0][1]), bits(res[1][1]))


def test_without_starts_a_replayed_graph_of_steps():
    """A captured decode step, append and commit, replayed: every step's keys land behind the last with their own positions."""
    import torch
    nseq, hkv, d = 3, 2, 128
    s = Setup(4, [0, 30, 63], [1, 1, 1], hq=4, hkv=hkv, d=d, page=64, room=20)
    rot = Rot(128)
    seen = torch.tensor([0, 1030, 63], dtype=torch.int32, device="cuda")
    pos = torch.zeros((nseq, hkv, s.cap), dtype=torch.int32, device="cuda")
    c = s.cache(seen=seen, pos=pos)
    one = torch.ones(nseq, dtype=torch.int32, device="cuda")
    k, v, q = (rows(i, nseq, h, d, "bf16")[0] for i, h in enumerate((hkv, hkv, 4)))
    out = torch.empty_like(q)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _rs.rs_cache_append_rope(c, rot.rope, k, v, q=q, q_out=out)
        _rs.rs_cache_commit(c, one, 1)
    want = s.dk.clone()
    for step in range(5):
        k.copy_(rows(100 + step, nseq, hkv, d, "bf16")[0])
        q.copy_(rows(200 + step, nseq, 4, d, "bf16")[0])
        at = torch.tensor([step, 1030 + step, 63 + step], dtype=torch.int32, device="cuda")
        rk, rq = torch.empty_like(k), torch.empty_like(q)
        _rs.rs_rope_apply(rot.rope, _rs.RopeRows([(k, rk), (q, rq)], pos=at))
        for b, j in enumerate((step, 30 + step, 63 + step)):
            want[s.table[b, j // 64], :, j % 64] = rk[b]
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(bits(s.dk), bits(want)) and torch.equal(bits(out), bits(rq))
        assert seen.tolist() == [step + 1, 1031 + step, 64 + step]


def test_the_most_rows():
    """2^24 rows of 64 heads, of which the cache has room for 128; heads share their rows."""
    import torch
    n, d, hkv, cap = 1 << 24, 64, 64, 128
    k = torch.zeros(n, 1, d, dtype=torch.bfloat16, device="cuda")
    k[:200] = torch.randn(200, 1, d, generator=torch.Generator().manual_seed(0)).to(torch.bfloat16).cuda()
    rot = Rot(64)
    got = []
    for m in (n, 200):
        x = k[:m].expand(m, hkv, d)
        dk, dv = (torch.full((1, hkv, cap, d), 3.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        c = _rs.KvCache(dk, dv, torch.full((1,), 7, dtype=torch.int32, device="cuda"))
        _rs.rs_cache_append_rope(c, rot.rope, x, x, max_rows=m)
        assert torch.equal(dv[0, :, 7:], k[:cap - 7, 0].expand(hkv, cap - 7, d)) and (dk[0, :, :7] == 3).all()
        got.append(dk)
    assert torch.equal(*got)
    want, ab = rot.oracle(k[:cap - 7].double().cpu().numpy(), 7 + np.arange(cap - 7))
    check(got[0][0, 5, 7:, None].double().cpu().numpy(), want, ab, "bf16", rot, [cap])
