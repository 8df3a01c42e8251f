"""Branches of the decoding calls that only larger batches take, tight checks of long sums, and graph replays of the
calls that change the cache."""
import numpy as np
import pytest

from oracle import decode as OD
from paper_2608_29058_amd import _rs
from decode_helpers import Setup, check_rows, logit_error

pytestmark = pytest.mark.gpu


def torch_attention(s, see_blocks=None):
    """The batch's attention on the device in fp64, sequence by sequence: o, lse, sum p |v| and the weights."""
    import torch
    G = s.hq // s.hkv
    f64 = dict(dtype=torch.float64, device="cuda")
    o, ab = torch.zeros(s.nrows, s.hq, s.d, **f64), torch.zeros(s.nrows, s.hq, s.d, **f64)
    lse, span, weights = torch.full((s.hq, s.nrows), -np.inf, **f64), 0.0, {}
    for b, (f, t) in enumerate(s.rows):
        n = int(s.lens[b])
        if not t:
            continue
        j = np.arange(n + t)
        p, i = (torch.from_numpy(x).cuda() for x in (s.table[b, j // s.page].astype(np.int64), j % s.page))
        see = torch.ones(t, n + t, dtype=torch.bool)
        see[:, n:] = torch.from_numpy(np.stack([OD.seen_drafts(s.mask, f + r, r, t) for r in range(t)]))
        see = see.cuda()
        for g in range(s.hkv):
            k, v = s.dk[p, g, i].double(), s.dv[p, g, i].double()
            q = s.dq[f:f + t, g * G:(g + 1) * G].double()
            on = see[:, None].expand(t, G, n + t)
            if see_blocks is not None:
                sel = torch.zeros(t, n + t, dtype=torch.bool, device="cuda")
                sel[:, n // 64 * 64:] = True
                for r in range(t):
                    for c in see_blocks[f + r, g]:
                        sel[r, c * 64:c * 64 + 64] = True
                on = on & sel[:, None]
            l = (q.reshape(t * G, -1) @ k.t() * s.scale).view(t, G, -1).masked_fill(~on, -np.inf)
            span = max(span, float((q.abs().reshape(t * G, -1) @ k.abs().t()).max() * s.scale))
            z = torch.logsumexp(l, 2)
            w = torch.where(on, torch.exp(l - z[..., None].clamp(min=-1e300)), torch.zeros((), **f64))
            o[f:f + t, g * G:(g + 1) * G] = (w.view(t * G, -1) @ v).view(t, G, -1)
            ab[f:f + t, g * G:(g + 1) * G] = (w.view(t * G, -1) @ v.abs()).view(t, G, -1)
            lse[g * G:(g + 1) * G, f:f + t] = z.t()
            weights[b, g] = w
    return dict(o=o.cpu().numpy(), lse=lse.cpu().numpy(), abs=ab.cpu().numpy(), span=span, weights=weights)


def attend(s):
    o, l = s.outputs()
    c = s.cache()
    _rs.rs_draft_attn(c, s.draft, o, l, _rs.workspace(_rs.rs_draft_attn_workspace_size(c, s.draft)))
    return o, l


# 32 sequences of 8 heads with more than 1024 rows fill the chip: 1024 cached rows per workgroup, up to four steps of each wave
@pytest.mark.parametrize("hq,d,dtype,t,kind", [
    (16, 128, "bf16", 3, "tree"),      # up to 16 rows of Q
    (32, 64, "bf16", 6, "random"),     # 17 to 32
    (32, 128, "bf16", 11, "tree"),     # more: parts of 128 rows in LDS
    (64, 64, "bf16", 20, None),        # 160: two parts
    (24, 64, "f32", 4, "tree"), (32, 64, "f32", 8, None), (16, 64, "f32", 20, "random"),
    (16, 128, "f32", 7, None), (32, 128, "f32", 7, "tree"), (16, 128, "f32", 30, "tree"),
])
def test_weights_of_large_batches(hq, d, dtype, t, kind):
    import torch
    top = 1100
    lens = [(37 * i * i + 61 * i) % top for i in range(32)]
    lens[:12] = [top, 0, 1, 63, 64, 65, 255, 256, 257, 511, 768, 1023]
    rows = [1 + (5 * i + t - 1) % t for i in range(32)]
    s = Setup(hq + t, lens, rows, hq=hq, hkv=8, d=d, dtype=dtype, kind=kind, spread=2.0)
    assert -(-s.cap // 1024) * 8 * 32 >= 512
    ref = torch_attention(s)
    r = np.random.default_rng(1)
    w = (r.random(s.nrows) * (r.random(s.nrows) < 0.8)).astype(np.float32)
    lse = torch.from_numpy(ref["lse"].astype(np.float32)).cuda()
    acc = torch.from_numpy(r.random((32, 8, s.cap)).astype(np.float32)).cuda()
    out = torch.full_like(acc, -3.0)
    _rs.rs_attn_weights(s.cache(), s.draft, lse, acc, out, row_w=torch.from_numpy(w).cuda())
    top_lse = np.abs(ref["lse"][np.isfinite(ref["lse"])]).max()
    dl = logit_error(dtype, d, ref["span"])
    dw = torch.from_numpy(w).cuda().double()
    for b, (f, n_new) in enumerate(s.rows):
        n = lens[b] + n_new
        assert (out[b, :, n:] == -3.0).all()
        for g in range(8):
            p = ref["weights"][b, g]
            add = (p * dw[f:f + n_new, None, None]).sum((0, 1))
            want = acc[b, g, :n].double() + add
            # per term: the logit's error, the given lse's rounding (2^-24 |lse|) and the exponent's; then the sum's steps
            lim = (dl + 2.0 ** -22 * (8 + top_lse)) * add + 2.0 ** -24 * (p.shape[0] * p.shape[1] + 4) * want + 1e-37
            assert ((out[b, g, :n].double() - want).abs() <= lim).all(), (b, g)


@pytest.mark.parametrize("hq,hkv,d,dtype,lens,t,kind", [
    (64, 8, 64, "bf16", [700, 1500, 0, 90] * 16, 1, None),    # 4096 rows to join: a wave each
    (64, 8, 128, "bf16", [700, 1500, 0, 90] * 16, 1, None),
    (32, 8, 64, "f32", [600, 0, 2000, 64] * 8, 4, "tree"),
    (16, 4, 64, "bf16", [3000, 17, 900] * 2, 60, "tree"),
])
def test_joins_of_many_rows(hq, hkv, d, dtype, lens, t, kind):
    rows = [1 + (3 * i + t - 1) % t for i in range(len(lens))] if kind is None else [t] * len(lens)
    s = Setup(hq + d, lens, rows, hq=hq, hkv=hkv, d=d, dtype=dtype, kind=kind, spread=2.0)
    assert s.nrows * hq >= 4096
    o, l = attend(s)
    check_rows(s, torch_attention(s), o, l)


@pytest.mark.parametrize("hq,hkv,d,dtype,lens,t,nsel", [
    (64, 1, 64, "bf16", [3000, 1200], 32, 20),       # 64 heads of one group in four pieces: joins of many rows
    (128, 1, 128, "bf16", [2600, 900], 16, 12),
    (8, 4, 64, "f32", [1500, 40, 640], 3, 7),        # fp32, d = 64
    (48, 2, 64, "f32", [1500, 333], 2, 9),           # 24 rows
])
def test_selections_in_pieces(hq, hkv, d, dtype, lens, t, nsel):
    import torch
    s = Setup(hq + nsel, lens, [t] * len(lens), hq=hq, hkv=hkv, d=d, dtype=dtype, spread=2.0)
    kmean, dm = s.means()
    c = s.cache(kmean=dm)
    o, l = s.outputs()
    bl = torch.full((s.nrows, hkv, nsel), -7, dtype=torch.int32, device="cuda")
    _rs.rs_select_attn(c, s.draft, nsel, 1, 2, o, l, _rs.workspace(_rs.rs_select_attn_workspace_size(c, s.draft, nsel)), blocks=bl)
    sel = OD.select(s.q.astype(np.float64), kmean, s.lens, s.table, s.page, s.rows, nsel, 1, 2, s.cap)
    b = bl.cpu().numpy()
    for (r, g), want in sel.items():
        assert np.array_equal(b[r, g, :len(want)], want) and (b[r, g, len(want):] == -1).all()
    check_rows(s, torch_attention(s, sel), o, l)


@pytest.mark.parametrize("hq,hkv,d,dtype,lens,t", [
    (8, 2, 128, "bf16", [30000, 5000], 1), (32, 4, 64, "bf16", [20000, 300], 3), (16, 2, 128, "bf16", [17000, 900], 12),
    (8, 1, 128, "bf16", [9000, 4000], 30), (8, 2, 64, "bf16", [9000, 60], 40), (8, 2, 128, "f32", [12000, 700], 1),
    (8, 2, 128, "f32", [9000, 5000], 7), (8, 2, 64, "f32", [9000, 100], 30),
])
def test_long_sums_of_positive_values(hq, hkv, d, dtype, lens, t):
    """With V >= 0 nothing cancels: sum p |v| is the result itself, and its bound is 2^-7 of it at any length."""
    import torch
    s = Setup(hq + t, lens, [t] * len(lens), hq=hq, hkv=hkv, d=d, dtype=dtype, page=256, spread=2.0)
    s.dv.abs_()
    s.dv.mul_(0.25 + torch.arange(d, device="cuda") % 5 / 4)   # (dimensions differ)
    ref = torch_attention(s)
    o, l = attend(s)
    check_rows(s, ref, o, l)
    got, want = o.double().cpu().numpy(), ref["o"]
    assert (np.abs(got / want - 1) <= 1.01 * (2 * 2.0 ** -8 + 2 * logit_error(dtype, d, ref["span"]) + 2.0 ** -15)).all()


def test_updates_and_weights_replay():
    """append, commit along a path and weights captured together, with other rows, counts and lengths per replay."""
    import torch
    for max_new, path in ((5, True), (300, False)):
        s = Setup(3, [100, 0, 640], [min(max_new, 5)] * 3, hq=8, hkv=2, d=64, page=64, room=2 * max_new)
        r = torch.Generator(device="cuda").manual_seed(5)
        _, km = s.means()
        acc = torch.rand((3, 2, s.cap), device="cuda", generator=r)
        pos, seen = torch.zeros((3, 2, s.cap), dtype=torch.int32, device="cuda"), s.dlen.clone()
        c = s.cache(kmean=km, acc=acc, pos=pos, seen=seen)
        n = 3 * max_new
        new = [torch.randn((n, 2, 64), device="cuda", generator=r).to(torch.bfloat16) for _ in range(2)]
        na = torch.tensor([2, 1, 4], dtype=torch.int32, device="cuda")
        way = torch.tensor([[0, 2, 4, 0, 0], [3, 0, 0, 0, 0], [0, 1, 3, 4, 0]], dtype=torch.int32, device="cuda")
        lse = torch.full((8, s.nrows), 3.0, device="cuda")

        def step():
            _rs.rs_cache_append(c, new[0], new[1], max_rows=max_new)
            _rs.rs_attn_weights(c, s.draft, lse, acc, acc)
            _rs.rs_cache_commit(c, na, max_new, path=way if path else None)

        state = (s.dk, s.dv, km, acc, pos, seen, s.dlen)
        start = [x.clone() for x in state]
        step()                                     # (eager first: nothing is set up inside the capture)
        for x, y in zip(state, start):
            x.copy_(y)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        for i in range(4):
            for x in new:
                x.normal_(generator=r)
            na.copy_(torch.tensor([[2, 1, 4], [0, 5, 1], [3, 3, 3], [5, 0, 2]][i], dtype=torch.int32) * (1 if path else max_new // 5))
            s.dlen.copy_(torch.tensor([[100, 0, 640], [63, 64, 1], [127, 500, 0], [0, 0, 0]][i], dtype=torch.int32))
            before = [x.clone() for x in state]
            step()
            torch.cuda.synchronize()
            want = [x.clone() for x in state]
            for x, y in zip(state, before):
                x.copy_(y)
            g.replay()
            torch.cuda.synchronize()
            for x, y in zip(state, want):
                assert torch.equal(x, y)
            for x, y in zip(state, start):
                x.copy_(y)
