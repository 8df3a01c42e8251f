"""Attention over selected blocks (rs_select_attn): the selected blocks equal those of the definition in 64
bits, block by block, and the rows equal the fp64 attention over them."""
import numpy as np
import pytest

from oracle import decode as OD
from paper_2608_29058_amd import _rs
from decode_helpers import Setup, check_rows

pytestmark = pytest.mark.gpu


def run(s, c, nsel, nsink=0, nlocal=0, blocks=True):
    import torch
    o, l = s.outputs()
    bl = torch.full((s.nrows, s.hkv, nsel), -7, dtype=torch.int32, device="cuda") if blocks else None
    ws = _rs.workspace(_rs.rs_select_attn_workspace_size(c, s.draft, nsel))
    _rs.rs_select_attn(c, s.draft, nsel, nsink, nlocal, o, l, ws, blocks=bl)
    return o, l, bl


def check(s, kmean, got, nsel, nsink=0, nlocal=0):
    o, l, bl = got
    sel = OD.select(s.q.astype(np.float64), kmean, s.lens, s.table, s.page, s.rows, nsel, nsink, nlocal, s.cap)
    if bl is not None:
        b = bl.cpu().numpy()
        for (r, g), want in sel.items():
            assert np.array_equal(b[r, g, :len(want)], want) and (b[r, g, len(want):] == -1).all(), (r, g, b[r, g], want)
    check_rows(s, s.oracle(blocks=sel), o, l)
    return sel


@pytest.mark.parametrize("hq,hkv,d,dtype,page,layout,lens,rows,kind,nsel,nsink,nlocal", [
    (8, 2, 128, "bf16", 64, "head", [0, 63, 64, 700, 1000], [1] * 5, None, 4, 1, 1),
    (4, 4, 64, "bf16", 128, "token", [2000, 190], [3, 2], None, 7, 0, 0),
    (14, 2, 128, "f32", 64, "head", [900, 1300], [1, 4], "tree", 3, 2, 1),
    (20, 1, 64, "bf16", 256, "head", [5000], [1], None, 40, 1, 4),        # 20 heads of one group, several pieces
    (8, 2, 64, "bf16", 64, "head", [640, 641, 700], [2, 1, 5], "random", 50, 3, 5),  # every block is taken
    (40, 1, 128, "f32", 64, "head", [1200], [2], None, 1, 0, 1),          # the forced block alone; two row tiles
    (4, 2, 64, "bf16", 64, "head", [300, 0, 777] * 30, [1, 2, 1] * 30, None, 3, 1, 1),  # more sequences than lanes
])
def test_selected_blocks(hq, hkv, d, dtype, page, layout, lens, rows, kind, nsel, nsink, nlocal):
    s = Setup(len(lens) + hq, lens, rows, hq=hq, hkv=hkv, d=d, dtype=dtype, page=page, layout=layout, kind=kind, extra=2, spread=2.0)
    kmean, dm = s.means()
    c = s.cache(kmean=dm)
    got = run(s, c, nsel, nsink, nlocal)
    check(s, kmean, got, nsel, nsink, nlocal)
    used = int(s.start[-1])
    assert (got[0][used:] == -7).all() and (got[1][:, used:] == -7).all() and (got[2][used:] == -7).all()
    o, l, _ = run(s, c, nsel, nsink, nlocal, blocks=False)
    assert (o == got[0]).all() and (l == got[1]).all()


def test_equal_scores_take_the_lower_blocks():
    s = Setup(2, [64 * 40, 64 * 300], [1, 1], hq=4, hkv=2, d=64, page=64)
    kmean, dm = s.means()
    kmean[:] = kmean[:1, :1, :1]                   # one mean everywhere ...
    for b, c, x in ((0, 30, 1.0), (0, 35, 1.0), (1, 257, 1.0), (1, 5, -1.0)):
        kmean[s.table[b, c]] = x * s.q[b, 0] * 2   # ... but for a few blocks of known order
    dm.copy_(__import__("torch").from_numpy(kmean))
    kmean = dm.double().cpu().numpy()
    got = run(s, s.cache(kmean=dm), 9, 0, 0)
    sel = check(s, kmean, got, 9)
    assert {30, 35} <= set(sel[0, 0].tolist()) and 257 in sel[1, 0]


def test_scores_one_step_apart_are_told_apart():
    """Scores that differ in their last of 40 bits: fp32 sums would call them equal."""
    import torch
    s = Setup(4, [64 * 64], [1], hq=1, hkv=1, d=128, page=64)
    q = np.zeros((s.nrows, 1, 128), np.float32)
    q[0, 0, 0], q[0, 0, 1] = 1.0, 2.0 ** -20
    s.q = q
    s.dq.copy_(torch.from_numpy(q))
    kmean, dm = s.means()
    kmean[:] = 0
    order = np.random.default_rng(0).permutation(64)
    for c in range(64):
        kmean[s.table[0, c], 0, 0, 0] = 1.0
        kmean[s.table[0, c], 0, 0, 1] = (order[c] - 30) * 2.0 ** -12    # score 1 + rank 2^-32
    dm.copy_(torch.from_numpy(kmean))
    got = run(s, s.cache(kmean=dm), 5)
    check(s, kmean, got, 5)
    assert set(got[2][0, 0].tolist()) == set(np.argsort(-order)[:5].tolist())


def test_missing_pages_and_odd_means():
    import torch
    s = Setup(6, [64 * 20 + 7], [2], hq=4, hkv=2, d=64, page=64)
    s.table[0, 3] = -1                             # scores 0, sees nothing there
    s.dtable.copy_(torch.from_numpy(s.table))
    kmean, dm = s.means()
    dm[int(s.table[0, 5])] = float("nan")          # NaN scores: after everything else
    dm[int(s.table[0, 6])] = float("inf")
    kmean = dm.double().cpu().numpy()
    o, l, bl = run(s, s.cache(kmean=dm), 6, 1, 1)
    b = bl.cpu().numpy()
    assert not (b == 5).any()
    sel = {(r, g): b[r, g] for r in range(2) for g in range(2)}
    check_rows(s, s.oracle(blocks=sel), o, l)


def test_graph_replays_follow_lengths_and_queries():
    import torch
    s = Setup(8, [3000, 64 * 9, 200], [1, 3, 2], hq=8, hkv=2, d=128, page=64)
    _, dm = s.means()
    c = s.cache(kmean=dm)
    ws = _rs.workspace(_rs.rs_select_attn_workspace_size(c, s.draft, 6))
    o, l = s.outputs()
    bl = torch.full((s.nrows, 2, 6), -7, dtype=torch.int32, device="cuda")
    _rs.rs_select_attn(c, s.draft, 6, 1, 1, o, l, ws, blocks=bl)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        _rs.rs_select_attn(c, s.draft, 6, 1, 1, o, l, ws, blocks=bl)
    for n in (3000, 64, 1999):
        s.dlen[0] = n
        s.dq.mul_(-1.5)
        want = run(s, c, 6, 1, 1)
        o.fill_(-7), bl.fill_(-7)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, want[0]) and torch.equal(l, want[1]) and torch.equal(bl, want[2])
