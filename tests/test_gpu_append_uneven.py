"""Rotated appends of batches whose sequences differ much in new rows (rs_cache_append_rope deals its workgroups to the batch's
rows): bit for bit a rotation followed by a plain append; what belongs to no sequence or lies elsewhere stays."""
import numpy as np
import pytest

from append_shapes import ABSURD, BEHIND, BOUNDS, MANY, REPLAY, UNEVEN
from decode_helpers import Setup
from oracle import decode as OD
from paper_2608_29058_amd import _rs
from rope_helpers import Rot, bits, rows

pytestmark = pytest.mark.gpu


def batch(seed, s, layout="token"):
    return tuple(rows(seed + i, s.nrows, h, s.d, s.dtype, layout)[0] for i, h in enumerate((s.hkv, s.hkv, s.hq)))


def compare(s, rot, k, v, q, start, max_rows, pos=None, seen=None, inplace=False):
    """Both ways from the same state."""
    import torch
    lens = np.clip(s.dlen.cpu().numpy(), 0, s.cap)
    ranges = OD.row_ranges(start.cpu().numpy(), len(lens), s.nrows, max_rows)
    at, used = np.zeros(s.nrows, np.int32), np.zeros(s.nrows, bool)
    for b, (f, t) in enumerate(ranges):
        at[f:f + t] = (lens[b] if seen is None else int(seen[b])) + np.arange(t)
        used[f:f + t] = True
    at = torch.from_numpy(at).cuda() if pos is None else pos
    used = torch.from_numpy(used).cuda()
    was = s.dk.clone(), s.dv.clone()
    acc = [torch.full((len(lens), s.hkv, s.cap), 5.0, device="cuda") for _ in range(2)]
    rk, rq = torch.empty_like(k), torch.empty_like(q)
    _rs.rs_rope_apply(rot.rope, _rs.RopeRows([(k, rk), (q, rq)], pos=at))
    _rs.rs_cache_append(s.cache(acc=acc[0]), rk, v, max_rows=max_rows, start=start)
    want = s.dk.clone(), s.dv.clone()
    s.dk.copy_(was[0])
    s.dv.copy_(was[1])
    x = q.clone() if inplace else q
    out = x if inplace else torch.full_like(q, -7.0)
    _rs.rs_cache_append_rope(s.cache(acc=acc[1], seen=seen), rot.rope, k, v, q=x, q_out=out, pos=pos, max_rows=max_rows, start=start)
    assert torch.equal(bits(s.dk), bits(want[0])) and torch.equal(bits(s.dv), bits(want[1])) and torch.equal(acc[0], acc[1])
    assert torch.equal(bits(out[used]), bits(rq[used]))
    rest = q[~used] if inplace else torch.full_like(q[~used], -7.0)
    assert torch.equal(bits(out[~used]), bits(rest))  # of no sequence: neither read nor written
    s.dk.copy_(was[0])
    s.dv.copy_(was[1])
    _rs.rs_cache_append_rope(s.cache(seen=seen), rot.rope, k, v, pos=pos, max_rows=max_rows, start=start)  # without queries
    assert torch.equal(bits(s.dk), bits(want[0])) and torch.equal(bits(s.dv), bits(want[1]))


@pytest.mark.parametrize("hq,hkv,d,dtype,page,dim,inter,layout,counts", UNEVEN)
def test_as_a_rotation_and_a_plain_append(hq, hkv, d, dtype, page, dim, inter, layout, counts):
    import torch
    r = np.random.default_rng(sum(counts))
    lens = r.integers(0, 200, len(counts)).tolist()
    s = Setup(1, lens, counts, hq=hq, hkv=hkv, d=d, dtype=dtype, page=page, layout="head" if layout == "head" else "token", extra=3)
    rot = Rot(dim, inter, base=500000.0, mscale=1.1)
    k, v, q = batch(5, s, layout)
    seen = torch.from_numpy(s.lens + r.integers(0, 5000, len(lens)).astype(np.int32)).cuda()
    pos = torch.from_numpy(r.integers(0, 200000, s.nrows).astype(np.int32)).cuda()
    for inplace in (False, True):
        compare(s, rot, k, v, q, s.dstart, s.max_rows, inplace=inplace)
    compare(s, rot, k, v, q, s.dstart, s.max_rows, seen=seen)
    compare(s, rot, k, v, q, s.dstart, s.max_rows, seen=seen, pos=pos)


def setup(seed, of, lens, counts, **kw):
    hq, hkv, d, nseq, nrows, _ = of
    s = Setup(seed, (lens + [0] * nseq)[:nseq], (counts + [0] * nseq)[:nseq], hq=hq, hkv=hkv, d=d, **kw)
    assert s.nrows == nrows
    return s


def test_more_rows_than_a_sequence_may_have_and_a_bound_that_bounds_nothing():
    s = setup(2, BOUNDS, [10] * 300, [400] + [1] * 299, extra=2)
    k, v, q = batch(9, s)
    for most in BOUNDS[5]:  # with the first, rows 170 .. 399 are of no sequence
        compare(s, Rot(64), k, v, q, s.dstart, most)


def test_more_sequences_than_a_workgroup_has_lanes():
    counts = [0, 1, 0, 1, 0, 0, 0, 1, 0, 0] * 70
    counts[255:257] = 60, 70
    counts[600] = 80
    s = setup(3, MANY, np.random.default_rng(3).integers(0, 70, 700).tolist(), counts)
    compare(s, Rot(64), *batch(4, s), s.dstart, MANY[5][0])


def test_rows_behind_the_capacity_and_without_a_page():
    import torch
    s = setup(4, BEHIND, [60, 120, 10, 0, 0, 5], [90, 2, 1, 0, 0, 1], room=130)
    s.dlen[:6] = torch.tensor([s.cap - 11, s.cap + 5, 10, 0, 0, -4])
    s.dtable[0, -1] = -1
    s.dtable[2, 0] = s.dk.shape[0]
    compare(s, Rot(64), *batch(6, s), s.dstart, s.max_rows)


def test_absurd_starts_stay_in_bounds():
    """Clamped as in rs_cache_append, in no order: of 300 sequences a few have rows, up to 12 of the 40."""
    import torch
    some = [38, 30, 1 << 30, -1, 12] + [12] * 200 + [24, 24, 29, 3, -7] + [-7] * 91
    for start in (some, [-5, -4, -3, -2, -1, 0] + [1 << 30] * 295, [1 << 30] * 301, list(range(301)), [20, 8, 8, 8, 8] + [50, 50, 44, 41] * 74):
        s = setup(2, ABSURD, [70, 20, 0, 5, 64, 1] + [3] * 294, [40], page=64, room=20)
        compare(s, Rot(128), *batch(8, s), torch.tensor(start, dtype=torch.int32, device="cuda"), ABSURD[5][0])


def test_rows_that_several_sequences_claim_enter_the_first():
    """A start that descends, which the call does not allow: in bounds, and the same every time."""
    import torch
    start = [0, 12, 6, 18] + [18, 14] * 148 + [40]
    assert len(start) == ABSURD[3] + 1
    s = setup(3, ABSURD, [10, 20, 30, 0, 5], [40], room=20)
    k, v, q = batch(3, s)
    rot = Rot(128)
    st = torch.tensor(start, dtype=torch.int32, device="cuda")
    rk = torch.empty_like(k)
    at = torch.arange(s.nrows, dtype=torch.int32, device="cuda") + 10
    _rs.rs_rope_apply(rot.rope, _rs.RopeRows([(k, rk)], pos=at))
    was, got = (s.dk.clone(), s.dv.clone()), []
    for _ in range(5):
        s.dk.copy_(was[0])
        s.dv.copy_(was[1])
        out = torch.full_like(q, -7.0)
        _rs.rs_cache_append_rope(s.cache(), rot.rope, k, v, q=q, q_out=out, max_rows=ABSURD[5][0], start=st)
        got.append((s.dk.clone(), s.dv.clone(), out))
        page = s.table[0, 0]
        assert torch.equal(bits(s.dk[page, :, 10:22]), bits(rk[:12].transpose(0, 1))) and torch.equal(bits(s.dv[page, :, 10:22]), bits(v[:12].transpose(0, 1)))
        for a, b in zip(got[0], got[-1]):
            assert torch.equal(bits(a), bits(b))


def test_a_replayed_graph():
    """Starts and lengths as they are at each replay."""
    import torch
    n = REPLAY[3]
    s = setup(5, REPLAY, [0, 30, 63, 7, 100] + [1] * (n - 5), [40] + [1] * (n - 1), room=40)
    rot = Rot(128)
    k, v, q = batch(2, s)
    out = torch.empty_like(q)
    was = s.dk.clone(), s.dv.clone()
    c = s.cache()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _rs.rs_cache_append_rope(c, rot.rope, k, v, q=q, q_out=out, max_rows=40, start=s.dstart)
    r = np.random.default_rng(7)
    for step in range(4):
        counts = np.ones(n, int)
        counts[r.integers(0, n)] = 40
        start = np.concatenate([[0], np.cumsum(counts)])
        s.dstart.copy_(torch.from_numpy(start))
        s.dlen[:5] = torch.tensor([step, 30, 63 - step, 7, 90 + step])
        s.dk.copy_(was[0])
        s.dv.copy_(was[1])
        graph.replay()
        torch.cuda.synchronize()
        got = s.dk.clone(), s.dv.clone(), out.clone()
        s.dk.copy_(was[0])
        s.dv.copy_(was[1])
        rk, rq = torch.empty_like(k), torch.empty_like(q)
        at = np.zeros(s.nrows, np.int32)
        for b, (f, t) in enumerate(OD.row_ranges(start, n, s.nrows, 40)):
            at[f:f + t] = int(s.dlen[b]) + np.arange(t)
        _rs.rs_rope_apply(rot.rope, _rs.RopeRows([(k, rk), (q, rq)], pos=torch.from_numpy(at).cuda()))
        _rs.rs_cache_append(c, rk, v, max_rows=40, start=s.dstart)
        assert torch.equal(bits(got[0]), bits(s.dk)) and torch.equal(bits(got[1]), bits(s.dv)) and torch.equal(bits(got[2]), bits(rq))
