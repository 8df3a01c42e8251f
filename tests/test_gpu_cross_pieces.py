"""Cross attention whose items are several pieces (rs_cross_attn): joins per item and per row, more than 64 sequences, tiles of every
kind, against the fp64 oracle; hidden infinities and NaN in prompts of heads of 64."""
import numpy as np
import pytest

from cross_helpers import Encoded
from cross_shapes import ITEMS, ROWS, STAGES
from decode_helpers import check_rows
from oracle import decode as OD

pytestmark = pytest.mark.gpu


def oracle(s):
    """As oracle.decode.cross, a product per sequence and head."""
    G = s.hq // s.hkv
    o, ab = np.full((s.nrows, s.hq, s.d), np.nan), np.zeros((s.nrows, s.hq, s.d))
    lse, span = np.full((s.hq, s.nrows), np.nan), 0.0
    for b, (f, t) in enumerate(s.rows):
        n = min(max(int(s.lens[b]), 0), s.cap)
        see = np.ones(n, bool) if s.kmask is None else OD.seen_drafts(s.kmask, b, 0, n)
        for g in range(s.hkv):
            kk, ok = OD.cache_rows(s.k, s.table, s.page, b, g, n)
            vv, _ = OD.cache_rows(s.v, s.table, s.page, b, g, n)
            on = ok & see
            h = slice(g * G, g * G + G)
            if t == 0 or not on.any():
                o[f:f + t, h], lse[h, f:f + t] = 0.0, -np.inf
                continue
            kk, vv, q = kk[on], vv[on], s.q[f:f + t, h].astype(np.float64).reshape(t * G, s.d)
            lg = q @ kk.T * s.scale
            m = lg.max(1, keepdims=True)
            p = np.exp(lg - m)
            z = p.sum(1, keepdims=True)
            p /= z
            o[f:f + t, h] = (p @ vv).reshape(t, G, s.d)
            ab[f:f + t, h] = (p @ np.abs(vv)).reshape(t, G, s.d)
            lse[h, f:f + t] = (m + np.log(z)).reshape(t, G).T
            span = max(span, float((np.abs(q) @ np.abs(kk).T).max() * s.scale))
    return dict(o=o, lse=lse, abs=ab, span=span)


def untouched(s, o, l):
    own = np.zeros(s.nrows, bool)
    for f, t in s.rows:
        own[f:f + t] = True
    assert (o.float().cpu().numpy()[~own] == -7.0).all() and (l.cpu().numpy()[:, ~own] == -7.0).all()


def test_the_oracle_by_products_is_the_oracle():
    s = Encoded(1, [70, 0, 130], [3, 2, 1], hq=4, hkv=2, d=64, hide=0.3, all_hidden=(2,), extra=1)
    a, b = oracle(s), s.oracle()
    for x in ("o", "lse", "abs"):
        assert np.allclose(a[x], b[x], rtol=1e-12, atol=1e-12, equal_nan=True)
    assert abs(a["span"] - b["span"]) <= 1e-12 * b["span"]


@pytest.mark.parametrize("hq,hkv,d,dtype,lens,rows,extra,hide", ITEMS + ROWS + STAGES)
def test_joined_pieces(hq, hkv, d, dtype, lens, rows, extra, hide):
    import torch
    s = Encoded(sum(lens) + hq, lens, rows, hq=hq, hkv=hkv, d=d, dtype=dtype, hide=hide, all_hidden=(1,) if len(lens) > 1 else (), extra=extra,
                spread=1.5)
    o, l = s.run()
    check_rows(s, oracle(s), o, l)
    untouched(s, o, l)
    again, l2 = s.run()
    assert torch.equal(o, again) and torch.equal(l, l2)  # to the bit
    only, l3 = s.run(lse=False)
    assert torch.equal(o, only) and (l3 == -7.0).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,rows", [([70, 129, 200], [300, 5, 130]), ([2100, 700, 64], [300, 5, 130])])
def test_hidden_infinities_and_nan_in_prompts(lens, rows, d):
    """In one piece and in several: no bit changes with what hidden states, states behind the end and unnamed pages hold."""
    import torch
    s = Encoded(5, lens, rows, hq=4, hkv=2, d=d, hide=0.3, all_hidden=(2,))
    o, l = s.run()
    check_rows(s, oracle(s), o, l)
    see = np.unpackbits(s.kmask.view(np.uint8), axis=1, bitorder="little").astype(bool)
    live = np.zeros(s.k.shape[:1] + s.k.shape[2:3], bool)
    for b, n in enumerate(s.lens):
        for j in np.flatnonzero(see[b, :n]):
            live[s.table[b, j // 64], j % 64] = True
    for bad in (np.nan, np.inf, -np.inf):
        for x in (s.k, s.v):
            x[:] = np.where(live[:, None, :, None], x, bad)
        s.upload()
        o2, l2 = s.run()
        assert torch.equal(o, o2) and torch.equal(l, l2)
    assert (o[s.start[2]:] == 0).all() and torch.isneginf(l[:, s.start[2]:]).all()
