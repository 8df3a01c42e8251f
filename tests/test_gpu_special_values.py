"""Infinities and NaN in cached rows, in bf16 and fp32 caches and in every form of the kernels: a key of minus
infinity takes its row's weight away and nothing else, an infinite value is infinite in its own dimension, and NaN
reaches the rows and dimensions that read it."""
import numpy as np
import pytest

from paper_2608_29058_amd import _rs
from decode_helpers import Setup, check_rows, logit_error

pytestmark = [pytest.mark.gpu, pytest.mark.filterwarnings("ignore:invalid value encountered")]

# heads, key/value heads, d, new rows: 16 and 32 rows of Q per head in registers, then stages of 64, 128 and 256
FORMS = [(8, 2, 128, [1, 1]), (12, 2, 64, [2, 1]), (8, 2, 128, [6, 8]), (10, 2, 64, [5, 6]), (8, 2, 128, [12, 16]),
         (8, 2, 64, [30, 20]), (8, 2, 128, [64, 50])]
LENS = [300, 900]


def make(form, dtype):
    import torch
    hq, hkv, d, rows = form
    s = Setup(hq + d + rows[0], LENS, rows, hq=hq, hkv=hkv, d=d, dtype=dtype, kind="tree" if rows[0] > 1 else None)
    s.q[..., 0] = np.abs(s.q[..., 0]) + 0.5       # (a step of bf16 may be lost: read back)
    s.dq.copy_(torch.from_numpy(s.q))
    s.q = s.dq.float().cpu().numpy()
    return s


def attend(s, select):
    import torch
    o, l = s.outputs()
    if select:
        _, km = s.means()
        c = s.cache(kmean=km)
        ws = _rs.workspace(_rs.rs_select_attn_workspace_size(c, s.draft, 20))
        _rs.rs_select_attn(c, s.draft, 20, 0, 0, o, l, ws)     # (20 blocks: all of them)
    else:
        c = s.cache()
        _rs.rs_draft_attn(c, s.draft, o, l, _rs.workspace(_rs.rs_draft_attn_workspace_size(c, s.draft)))
    torch.cuda.synchronize()
    return o, l


@pytest.mark.parametrize("select", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("form", FORMS)
def test_keys_of_minus_infinity(form, dtype, select):
    """Two whole pages of such rows: the rest is what it is without these pages."""
    import torch
    s = make(form, dtype)
    lost = [(0, 1), (1, 5)]
    for b, p in lost:
        s.dk[int(s.table[b, p]), :, :, 0] = -float("inf")
    o, l = attend(s, select)
    c = s.cache()
    acc = torch.full((2, s.hkv, s.cap), 0.5, device="cuda")
    _rs.rs_attn_weights(c, s.draft, l, acc, acc)
    for b, p in lost:
        s.table[b, p] = -1
    ref = s.oracle()
    check_rows(s, ref, o, l)
    got = acc.cpu().numpy().astype(np.float64)
    dl = logit_error(dtype, s.d, ref["span"])
    for b, (f, t) in enumerate(s.rows):
        n = LENS[b] + t
        for g in range(s.hkv):
            w = ref["weights"][b, g]
            add = sum(x[:n] for x in w.values())
            # as for the weights of finite rows, once more for the lse that the kernel itself has computed
            lim = (2 * dl + 2.0 ** -20 * (n / 16 + 64)) * add + 2.0 ** -24 * (len(w) + 4) * (0.5 + add)
            assert (np.abs(got[b, g, :n] - 0.5 - add) <= lim).all()


@pytest.mark.parametrize("select", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("form", FORMS)
def test_infinite_and_undefined_values(form, dtype, select):
    """In a cached row's V, dimension by dimension; a key of NaN in the other sequence's last head."""
    s = make(form, dtype)
    at = lambda b, j: (int(s.table[b, j // 64]), j % 64)
    for (b, j, g, d), x in {(0, 70, 0, 3): np.inf, (0, 70, 0, 7): -np.inf, (0, 201, 0, 9): np.nan, (0, 255, 1, 0): np.inf,
                            (1, 640, 0, 5): -np.inf, (1, 641, 0, 6): np.inf, (1, 3, 0, 6): -np.inf}.items():
        p, i = at(b, j)
        s.v[p, g, i, d] = s.dv[p, g, i, d] = x
    p, i = at(1, 100)
    s.k[p, s.hkv - 1, i, 2] = s.dk[p, s.hkv - 1, i, 2] = np.nan
    o, l = attend(s, select)
    ref = s.oracle()
    ref["span"] = logit_span(s)                    # (of the rows without NaN)
    G = s.hq // s.hkv
    used, bad = int(s.start[-1]), slice(s.hq - G, s.hq)
    got, gl = o.float().cpu().numpy()[:used], l.cpu().numpy()[:, :used]
    want, r1 = ref["o"][:used], slice(s.rows[1][0], used)
    assert np.isnan(got[r1, bad]).all() and np.isnan(gl[bad, r1]).all()
    for x in (ref["o"], ref["abs"]):
        x[r1, bad] = 0.0
    ref["lse"][bad, r1] = 0.0
    o[r1, bad], l[bad, r1] = 0.0, 0.0
    check_rows(s, ref, o, l)
    inf = np.isinf(ref["o"][:used])
    assert inf.any() and np.array_equal(o.float().cpu().numpy()[:used][inf], want[inf])
    assert np.array_equal(np.isinf(o.float().cpu().numpy()[:used]), inf)


def logit_span(s):
    k = np.abs(np.nan_to_num(s.k.astype(np.float64))).max(axis=(0, 1, 2))
    return float((np.abs(s.q.astype(np.float64)) @ k).max() * s.scale)


@pytest.mark.parametrize("d", [64, 128])
def test_large_fp32_values_are_finite(d):
    """Magnitudes up to the largest bf16 keep at least eight bits and stay finite, whatever the form."""
    for form in [f for f in FORMS if f[2] == d]:
        s = make(form, "f32")
        s.v[..., 1] *= np.float32(2.0 ** 110)
        s.v[..., 2] *= np.float32(2.0 ** 90)
        import torch
        s.dv.copy_(torch.from_numpy(s.v))
        o, _ = attend(s, False)
        ref = s.oracle()
        got = o.float().cpu().numpy().astype(np.float64)[:int(s.start[-1])]
        want, ab = ref["o"][:int(s.start[-1])], ref["abs"][:int(s.start[-1])]
        dl = logit_error("f32", d, ref["span"])
        # half a bf16 step of the result, of every weight, and of values from 2^96 on
        tol = 1.01 * (2.0 ** -8 * np.abs(want) + (2 * 2.0 ** -8 + 2 * dl + 2.0 ** -15) * ab)
        assert np.isfinite(got).all() and (np.abs(got - want) <= tol).all()
