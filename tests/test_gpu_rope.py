"""Rotary positions (rs_rope_apply) against the fp64 oracle: both layouts, any part of the head, every scaling, far and negative
positions, strides, in place, several parts, the transposed rotation as inverse and as gradient, streams and graphs."""
import numpy as np
import pytest

from oracle import rope as OR
from paper_2608_29058_amd import _rs
from rope_helpers import Rot, bits, check, rows

pytestmark = pytest.mark.gpu


def turn(rot, x, pos=None, pos0=0, transpose=False, y=None):
    import torch
    y = torch.full_like(x, -7.0) if y is None else y
    p = None if pos is None else torch.from_numpy(np.asarray(pos, np.int32)).cuda()
    _rs.rs_rope_apply(rot.rope, _rs.RopeRows([(x, y)], pos=p, pos0=pos0), transpose=transpose)
    return y


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,dim", [(128, 128), (128, 64), (128, 16), (128, 10), (128, 126), (64, 64), (64, 32), (64, 2), (64, 48), (64, 62)])
@pytest.mark.parametrize("inter", [False, True])
def test_layouts_and_parts_of_the_head(dtype, d, dim, inter):
    rot = Rot(dim, inter)
    for n, heads, layout in ((1, 1, "token"), (3, 5, "head"), (67, 7, "wide"), (300, 3, "head")):
        x, xv = rows(n + dim, n, heads, d, dtype, layout)
        pos = np.random.default_rng(n).integers(0, 131072, n)
        got = turn(rot, x, pos)
        want, ab = rot.oracle(xv, pos)
        check(got.double().cpu().numpy(), want, ab, dtype, rot, pos)
        import torch
        assert torch.equal(bits(got[..., dim:]), bits(x[..., dim:]))  # what does not turn keeps its bits


@pytest.mark.parametrize("kw", [
    dict(base=500000.0), dict(scaling=OR.LINEAR, factor=4.0), dict(scaling=OR.TURNS, factor=8.0, context=8192.0, mscale=1.2079),
    dict(scaling=OR.PAIRS, factor=8.0, context=4096.0, mscale=0.75), dict(mscale=-2.0),
])
def test_scalings(kw):
    rot = Rot(128, **kw)
    x, xv = rows(5, 200, 4, 128, "f32")
    for transpose in (False, True):
        got = turn(rot, x, pos0=1000, transpose=transpose)
        want, ab = rot.oracle(xv, 1000 + np.arange(200), transpose)
        check(got.cpu().numpy(), want, ab, "f32", rot, [1200])


@pytest.mark.parametrize("pos,pos0", [
    ([0, 1, 2, 3], 0), ([-1, -5, -100000, 7], 0), ([262143, 262144, 16777217, 2 ** 31 - 1], 0), ([-2 ** 31, 2 ** 30 + 1, -2 ** 24 - 1, 0], 0),
    (None, 2 ** 31 - 2), (None, -2 ** 31), (None, -2),
])
def test_far_and_negative_positions(pos, pos0):
    rot = Rot(64, base=10000.0)
    x, xv = rows(9, 4, 2, 64, "f32")
    at = np.array(pos if pos is not None else pos0 + np.arange(4), np.int64)
    got = turn(rot, x, pos, pos0)
    want, ab = rot.oracle(xv, at)
    check(got.cpu().numpy(), want, ab, "f32", rot, at)


def test_frequencies_of_the_callers_own():
    per = [0.5, 0.25, 0.125, 0.0, -0.25, 3.0, 1e-9, 0.3]
    rot = Rot(16)
    rot.rope, rot.per = _rs.Rope(16, turns=per), np.array(per)
    x, xv = rows(2, 9, 2, 64, "f32")
    got = turn(rot, x, pos0=-4).cpu().numpy()
    want, ab = rot.oracle(xv, np.arange(-4, 5))
    check(got, want, ab, "f32", rot, [5])
    # quarter turns are exact
    assert np.array_equal(got[:, :, 3], xv[:, :, 3]) and np.array_equal(got[3, :, 0], -xv[3, :, 0])  # no turn; half a turn


@pytest.mark.parametrize("n", [1, 2, 31, 33, 1000, 20000])
def test_parts_share_positions_and_rows_are_left_alone(n):
    """Four parts of one launch, as four launches; nothing but their rows is written."""
    import torch
    rot = Rot(128)
    pos = torch.arange(n, dtype=torch.int32, device="cuda") * 3
    xs = [rows(i, n, h, 128, "bf16", lay)[0] for i, (h, lay) in enumerate(((1, "head"), (8, "wide"), (33, "token"), (2, "head")))]
    frames = [torch.full((n + 2, x.shape[1] + 2, 128), -7.0, dtype=x.dtype, device="cuda") for x in xs]
    ys = [f[1:-1, 1:-1] for f in frames]
    _rs.rs_rope_apply(rot.rope, _rs.RopeRows(list(zip(xs, ys)), pos=pos))
    for x, y, f in zip(xs, ys, frames):
        one = torch.empty_like(x)
        _rs.rs_rope_apply(rot.rope, _rs.RopeRows([(x, one)], pos=pos))
        assert torch.equal(bits(y), bits(one))
        f[1:-1, 1:-1] = -7.0
        assert (f == -7.0).all()


@pytest.mark.parametrize("dim,inter", [(128, False), (128, True), (64, False), (10, False), (24, True)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [3, 5000])
def test_in_place(dim, inter, dtype, n):
    import torch
    rot = Rot(dim, inter)
    x, _ = rows(1, n, 6, 128, dtype, "wide")
    want = turn(rot, x, pos0=7)
    turn(rot, x, pos0=7, y=x)
    assert torch.equal(bits(x), bits(want))


@pytest.mark.parametrize("inter", [False, True])
def test_the_transposed_rotation_is_the_gradient_and_undoes(inter):
    """L = <w, y(x)>: its gradient is the transposed rotation of w, by the formula and by differences of L."""
    rot = Rot(48, inter, mscale=1.25)
    n, d = 41, 64
    x, xv = rows(3, n, 3, d, "f32")
    w, wv = rows(4, n, 3, d, "f32")
    pos = np.random.default_rng(0).integers(0, 9000, n)
    grad = turn(rot, w, pos, transpose=True).cpu().numpy().astype(np.float64)
    want, ab = rot.oracle(wv, pos, True)
    check(grad, want, ab, "f32", rot, pos)
    # L is linear: the difference quotient is exact but for the roundings of y, 2^-20 of the terms at most
    for seed in range(3):
        step, sv = rows(10 + seed, n, 3, d, "f32")
        up, down = (turn(rot, v.contiguous(), pos).double().cpu().numpy() for v in (x + step, x - step))
        moved = ((x + step).double() - (x - step).double()).cpu().numpy()
        diff = (wv * (up - down)).sum()
        terms = (np.abs(wv) * 1.25 * 2 * (np.abs(xv) + np.abs(sv)) * 2).sum()
        assert abs(diff - (grad * moved).sum()) <= 2.0 ** -20 * terms
    one = Rot(48, inter)
    back = turn(one, turn(one, x, pos), pos, transpose=True)
    # two rotations: each within 2^-21 (|x_1| + |x_2|) and its rounding
    a, ab1 = one.oracle(xv, pos)
    _, ab2 = one.oracle(a, pos)
    assert (np.abs(back.cpu().numpy() - xv) <= (2.0 ** -21 + 2.0 ** -23) * (ab1 + 2 * ab2) + 2.0 ** -23 * np.abs(xv)).all()


def test_infinities_stay_in_their_pairs():
    import torch
    rot = Rot(32)
    x, _ = rows(8, 4, 2, 64, "bf16")
    clean = turn(rot, x, pos0=5)
    x = x.clone()
    x[1, 0, 3] = float("inf")      # pair (3, 19)
    x[2, 1, 40] = float("nan")     # behind dim
    x[3, 1, 33] = float("-inf")
    got = turn(rot, x, pos0=5)
    odd = ~torch.isfinite(got)
    want = torch.zeros_like(odd)
    want[1, 0, 3] = want[1, 0, 19] = want[2, 1, 40] = want[3, 1, 33] = True
    assert torch.equal(odd, want) and got[3, 1, 33] == float("-inf")
    assert torch.equal(got[~want], clean[~want])


def test_a_prompts_rows_and_offsets_behind_2_gib():
    """[heads, n, d] of a prompt as it is, 2.1 GB of fp32 a tensor: offsets pass 31 bits."""
    import torch
    n, heads = 131072, 34
    rot = Rot(128, base=500000.0)
    q = torch.randn(heads, n, 128, device="cuda")
    y = torch.empty_like(q)
    _rs.rs_rope_apply(rot.rope, _rs.RopeRows([(q.transpose(0, 1), y.transpose(0, 1))]))
    at = np.array([0, 1, 63, 70000, 131071])
    for h in (0, 15, 33):
        want, ab = rot.oracle(q[h, at].double().cpu().numpy()[:, None], at)
        check(y[h, at].cpu().numpy()[:, None], want, ab, "f32", rot, at)
    # every row: lengths of pairs stay
    a, b = q[..., :64].double().square() + q[..., 64:].double().square(), y[..., :64].double().square() + y[..., 64:].double().square()
    assert float(((a - b).abs() / a.clamp(min=1e-3)).max()) < 2.0 ** -19


def test_no_rows_another_stream_and_a_replayed_graph():
    import torch
    rot = Rot(128)
    e = torch.empty(0, 4, 128, dtype=torch.bfloat16, device="cuda")
    _rs.rs_rope_apply(rot.rope, _rs.RopeRows([(e, e)]))
    x, _ = rows(6, 500, 8, 128, "bf16")
    want = turn(rot, x, pos0=3)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    y = torch.zeros_like(x)
    _rs.rs_rope_apply(rot.rope, _rs.RopeRows([(x, y)], pos0=3), stream=st)
    st.synchronize()
    assert torch.equal(bits(y), bits(want))
    pos = torch.arange(500, dtype=torch.int32, device="cuda")
    r = _rs.RopeRows([(x, y)], pos=pos)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _rs.rs_rope_apply(rot.rope, r)
    for k in range(4):
        pos.copy_(torch.arange(500, device="cuda") + 11 * k)
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(bits(y), bits(turn(rot, x, pos0=11 * k)))


@pytest.mark.parametrize("d,dim", [(128, 2), (128, 10), (128, 126), (64, 20), (64, 62)])
@pytest.mark.parametrize("inter", [False, True])
def test_what_does_not_turn_keeps_the_bits_of_any_nan(d, dim, inter):
    import torch
    x, _ = rows(dim, 9, 3, d, "bf16")
    bits(x)[..., dim::2] = 0x7f81  # a NaN that an arithmetic instruction would change
    bits(x)[..., dim + 1::2] = -(1 << 15) + 0x7fa5
    rot = Rot(dim, inter)
    got = turn(rot, x, pos0=5)
    assert torch.equal(bits(got[..., dim:]), bits(x[..., dim:])) and not got[..., :dim].isnan().any()
    same = x.clone()
    assert torch.equal(bits(turn(rot, same, pos0=5, y=same)), bits(got))
