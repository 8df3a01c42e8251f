"""Rotations and rotated appends of more bytes than the memory-side cache holds, whose loads bypass it: every layout and part of the
head, bit for bit as the same rows in calls of fewer."""
import numpy as np
import pytest

from paper_2608_29058_amd import _rs
from rope_helpers import Rot, bits, check

pytestmark = pytest.mark.gpu

SIDE_CACHE = 256 << 20
PARTS = [(128, False), (128, True), (64, False), (24, True), (10, False), (126, False)]


def randn(seed, n, heads, dtype, layout):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    shape = (heads, n, 128) if layout == "head" else (n, heads, 128)
    x = torch.randn(*shape, generator=g, device="cuda", dtype=torch.bfloat16 if dtype == "bf16" else torch.float32)
    return x.transpose(0, 1) if layout == "head" else x


@pytest.mark.parametrize("dim,inter", PARTS)
@pytest.mark.parametrize("layout", ["token", "head"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rotations(dim, inter, layout, dtype):
    import torch
    n, hq, hkv = 40001 if dtype == "bf16" else 20001, 24, 4
    rot = Rot(dim, inter, base=500000.0)
    q, k = randn(1, n, hq, dtype, layout), randn(2, n, hkv, dtype, layout)
    assert (q.numel() + k.numel()) * q.element_size() > SIDE_CACHE
    yq, yk = torch.empty_like(q), torch.empty_like(k)
    _rs.rs_rope_apply(rot.rope, _rs.RopeRows([(q, yq), (k, yk)], pos0=3))
    for r0 in range(0, n, 10007):
        a, b = q[r0:r0 + 10007], k[r0:r0 + 10007]
        wq, wk = torch.empty_like(a), torch.empty_like(b)
        _rs.rs_rope_apply(rot.rope, _rs.RopeRows([(a, wq), (b, wk)], pos0=3 + r0))
        assert torch.equal(bits(yq[r0:r0 + 10007]), bits(wq)) and torch.equal(bits(yk[r0:r0 + 10007]), bits(wk))
    at = [0, 1, n // 2, n - 1]
    want, ab = rot.oracle(q[at].double().cpu().numpy(), 3 + np.array(at))
    check(yq[at].double().cpu().numpy(), want, ab, dtype, rot, [n])
    both = torch.cat([q, k], 1) if layout == "token" else torch.cat([q.transpose(0, 1), k.transpose(0, 1)]).transpose(0, 1)
    _rs.rs_rope_apply(rot.rope, _rs.RopeRows([(both, both)], pos0=3))  # in place
    assert torch.equal(bits(both[:, :hq]), bits(yq)) and torch.equal(bits(both[:, hq:]), bits(yk))


@pytest.mark.parametrize("dim,inter", PARTS)
@pytest.mark.parametrize("layout", ["token", "head"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("uneven", [False, True])
def test_appends(dim, inter, layout, dtype, uneven):
    import torch
    n, hq, hkv, page = 40001 if dtype == "bf16" else 20001, 20, 4, 256
    counts = [n - 60] + [1] * 60 if uneven else [n - n // 3, n // 3]
    rot = Rot(dim, inter, base=500000.0)
    q, k, v = (randn(i, n, h, dtype, layout) for i, h in enumerate((hq, hkv, hkv)))
    assert (q.numel() + 2 * k.numel()) * q.element_size() > SIDE_CACHE
    lens = torch.arange(len(counts), dtype=torch.int32, device="cuda") * 7
    used = [-(-(7 * b + c) // page) for b, c in enumerate(counts)]
    table, at = torch.full((len(counts), max(used)), -1, dtype=torch.int32), 0
    for b, m in enumerate(used):
        table[b, :m] = torch.arange(at, at + m, dtype=torch.int32).flip(0)
        at += m
    table = table.cuda()
    start = torch.tensor([0] + counts, device="cuda").cumsum(0).int()
    pos = torch.cat([7 * b + torch.arange(c, dtype=torch.int32, device="cuda") for b, c in enumerate(counts)]).int()
    got = []
    for fused in (True, False):
        dk, dv = (torch.full((at, hkv, page, 128), 3.0, dtype=q.dtype, device="cuda") for _ in range(2))
        c = _rs.KvCache(dk, dv, lens, table=table)
        yq = torch.empty_like(q)
        if fused:
            _rs.rs_cache_append_rope(c, rot.rope, k, v, q=q, q_out=yq, max_rows=max(counts), start=start)
        else:
            yk = torch.empty_like(k)
            for r0 in range(0, n, 10007):
                r = slice(r0, r0 + 10007)
                _rs.rs_rope_apply(rot.rope, _rs.RopeRows([(q[r], yq[r]), (k[r], yk[r])], pos=pos[r]))
            _rs.rs_cache_append(c, yk, v, max_rows=max(counts), start=start)
        got.append((dk, dv, yq))
    for a, b in zip(*got):
        assert torch.equal(bits(a), bits(b))
