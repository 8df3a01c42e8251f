"""CPU checks of rotary positions and cross attention: frequencies of every scaling against the oracle, struct layouts,
and refusals of what the calls cannot do before anything is launched."""
import ctypes as C
import math
import os
import shutil
import subprocess

import numpy as np
import pytest

from oracle import rope as OR
from paper_2608_29058_amd import _rs
from test_decode_host import cache

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INV, UNS, WSP = _rs.RS_ERR_INVALID_ARG, _rs.RS_ERR_UNSUPPORTED, _rs.RS_ERR_WORKSPACE


@pytest.mark.parametrize("dim", [2, 10, 48, 64, 126, 128])
@pytest.mark.parametrize("kw", [
    dict(), dict(base=500000.0), dict(scaling=OR.LINEAR, factor=4.0), dict(scaling=OR.LINEAR, factor=1.0),
    dict(scaling=OR.TURNS, factor=8.0, context=8192.0), dict(scaling=OR.TURNS, factor=4.0, context=32768.0, low=1.0, high=4.0),
    dict(scaling=OR.PAIRS, factor=8.0, context=4096.0), dict(scaling=OR.PAIRS, factor=5.5, context=32768.0, base=500000.0),
    dict(scaling=OR.PAIRS, factor=2.0, context=1.0),  # no pair turns once: all divided but the first
    dict(scaling=OR.TURNS, factor=2.0, context=1e9),  # all turn more than that: none divided
])
def test_frequencies_follow_their_rule(dim, kw):
    want = OR.turns(dim, **kw)
    got = np.array(_rs.Rope(dim, **kw).c.turns)
    # pow, a log and a few products in fp64: some steps of 2^-53, and the ramp's ends are integers or plain turns
    assert np.allclose(got[:dim // 2], want, rtol=2.0 ** -46, atol=0)
    assert (got[dim // 2:] == 0).all()


def test_scalings_at_their_ends():
    plain = np.array(_rs.Rope(128, base=10000.0).c.turns)
    assert plain[0] == 1 / (2 * math.pi)
    ramp = np.array(_rs.Rope(128, base=10000.0, scaling=_rs.RS_ROPE_TURNS, factor=8.0, context=8192.0).c.turns)
    n = plain * 8192
    assert np.array_equal(ramp[n >= 32], plain[n >= 32]) and np.allclose(ramp[n <= 1], plain[n <= 1] / 8, rtol=2.0 ** -50)
    mid = (n > 1) & (n < 32)
    assert mid.any() and ((ramp < plain) & (ramp > plain / 8))[mid].all()
    r = _rs.Rope(8, turns=[0.5, 0.25, 0.125, 0.0])
    assert list(r.c.turns)[:5] == [0.5, 0.25, 0.125, 0.0, 0.0] and r.c.mscale == 1.0
    with pytest.raises(ValueError):
        _rs.Rope(8, turns=[0.5])


@pytest.mark.parametrize("kw", [
    dict(dim=0), dict(dim=3), dict(dim=130), dict(dim=-2), dict(layout=2), dict(layout=-1), dict(scaling=4), dict(scaling=-1),
    dict(base=1.0), dict(base=float("nan")), dict(base=float("inf")), dict(scaling=1, factor=0.5), dict(scaling=1, factor=float("nan")),
    dict(scaling=2, factor=2.0), dict(scaling=2, factor=2.0, context=float("inf")), dict(scaling=3, factor=2.0, context=100.0, low=0.0),
    dict(scaling=3, factor=2.0, context=100.0, low=4.0, high=4.0), dict(scaling=2, factor=2.0, context=100.0, high=float("nan")),
    dict(mscale=float("inf")), dict(mscale=1e300),
])
def test_bad_frequencies_are_refused(kw):
    with pytest.raises(_rs.RsError) as e:
        _rs.Rope(**dict(dict(dim=64), **kw))
    assert e.value.status == INV
    assert _rs.lib().rs_rope_init(None, None) == INV


def test_struct_layouts_match_the_c_compiler(tmp_path):
    if not shutil.which("gcc"):
        pytest.skip("gcc not available")
    structs = dict(rs_rope_cfg=_rs.RsRopeCfg, rs_rope=_rs.RsRope, rs_rope_part=_rs.RsRopePart, rs_rope_rows=_rs.RsRopeRows,
                   rs_cross=_rs.RsCross)
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "rs.h"', "int main(void) {"]
    for name, py in structs.items():
        lines.append(f'printf("{name} size %zu\\n", sizeof({name}));')
        lines += [f'printf("{name} {f[0]} %zu\\n", offsetof({name}, {f[0]}));' for f in py._fields_ if not f[0].startswith("_pad")]
    src = tmp_path / "layout.c"
    src.write_text("\n".join(lines + ["return 0; }"]))
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    for line in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split("\n"):
        if line:
            name, field, val = line.split()
            assert (C.sizeof(structs[name]) if field == "size" else getattr(structs[name], field).offset) == int(val), line


def rope(**kw):
    r = _rs.RsRope(dim=64, layout=0, mscale=1.0)
    for k, v in kw.items():
        if k == "turn":
            r.turns[v[0]] = v[1]
        else:
            setattr(r, k, v)
    return r


def rows(part=None, **kw):
    a = dict(dtype=0, n=4, d=128, nparts=1, pos=4096, pos0=0)
    a.update(kw)
    r = _rs.RsRopeRows(**a)
    for i in range(min(max(a["nparts"], 0), 4)):
        r.part[i] = _rs.RsRopePart(**dict(dict(x=4096, y=8192, heads=8, sx_t=1024, sx_h=128, sy_t=1024, sy_h=128), **(part or {})))
    return r


BAD_ROPES = [dict(dim=0), dict(dim=5), dict(dim=130), dict(layout=2), dict(mscale=float("nan")), dict(turn=(0, float("inf"))),
             dict(turn=(31, float("nan")))]
BAD_PARTS = [dict(x=None), dict(y=None), dict(x=4104), dict(y=4100), dict(heads=0), dict(heads=70000), dict(sx_t=4), dict(sy_h=12),
             dict(sx_h=-8), dict(sy_t=64), dict(sy_h=64), dict(sy_t=0), dict(sy_h=0), dict(sy_t=128),
             dict(sy_t=512, sy_h=256), dict(y=4096, sy_t=2048)]


def test_rotations_are_refused():
    L = _rs.lib()
    call = lambda r, x, back=0: L.rs_rope_apply(C.byref(r) if r is not None else None, C.byref(x) if x is not None else None, back, None)
    assert call(None, rows()) == INV and call(rope(), None) == INV
    for kw in BAD_ROPES:
        assert call(rope(**kw), rows()) == INV, kw
        assert L.rs_last_error().startswith(b"rope")
    for kw, want in ((dict(dtype=2), INV), (dict(d=96), UNS), (dict(d=256), UNS), (dict(n=-1), INV), (dict(n=(1 << 24) + 1), UNS),
                     (dict(nparts=0), INV), (dict(nparts=5), INV), (dict(pos0=1 << 40), INV), (dict(pos0=-(1 << 32)), INV)):
        assert call(rope(), rows(**kw)) == want, kw
    for kw in BAD_PARTS:
        assert call(rope(), rows(part=kw)) == INV, kw
    assert call(rope(dim=128), rows(d=64)) == INV       # more than the head
    assert call(rope(turn=(40, float("nan"))), rows(n=0)) == _rs.RS_OK  # (a pair that dim leaves out)
    assert call(rope(), rows(n=0, part=dict(x=None))) == _rs.RS_OK      # nothing to do


def test_rotated_appends_are_refused():
    L = _rs.lib()

    def call(c=None, r=rope(), q=None, none_q=False, kn=4096, vn=4096, a=256, b=128, cc=256, d=128, st=4096, n=2, m=1):
        part = None if none_q else C.byref(_rs.RsRopePart(**dict(dict(x=4096, y=8192, heads=8, sx_t=1024, sx_h=128, sy_t=1024, sy_h=128), **(q or {}))))
        return L.rs_cache_append_rope(C.byref(c or cache()), C.byref(r) if r is not None else None, kn, vn, a, b, cc, d, part, 4096, st, n, m, None)

    for kw, want in ((dict(k=None), INV), (dict(d=96), UNS), (dict(page=100), UNS), (dict(sk_t=64), INV)):
        assert call(c=cache(**kw)) == want
        assert L.rs_last_error().startswith(b"cache")
    for kw in (dict(kn=None), dict(vn=4100), dict(a=4), dict(n=-1), dict(m=0), dict(st=None, n=1)):
        assert call(**kw) == INV
        assert L.rs_last_error().startswith(b"append")
    for kw in BAD_ROPES:
        assert call(r=rope(**kw)) == INV, kw
    assert call(r=None) == INV
    for kw in BAD_PARTS:
        assert call(q=kw) == INV, kw
    assert call(n=0) == _rs.RS_OK and call(n=0, kn=None, q=dict(x=None)) == _rs.RS_OK
    assert call(n=(1 << 24) + 1) == UNS


def cross(**kw):
    a = dict(q=4096, hq=8, nrows=2, max_rows=1, nwords=8, sq_t=8 * 128, sq_h=128, start=4096, kmask=None, scale=0.0)
    a.update(kw)
    return _rs.RsCross(**a)


def attend(c, x, o=4096, so_t=1024, so_h=128, ws=4096, nbytes=1 << 34):
    return _rs.lib().rs_cross_attn(C.byref(c), C.byref(x) if x is not None else None, o, so_t, so_h, None, ws, nbytes, None)


@pytest.mark.parametrize("kw,want", [
    (dict(q=None), INV), (dict(q=4104), INV), (dict(hq=7), INV), (dict(hq=0), INV), (dict(nrows=-1), INV), (dict(max_rows=0), INV),
    (dict(start=None, nrows=1), INV), (dict(kmask=4096, nwords=7), INV), (dict(kmask=4098), INV), (dict(sq_t=4), INV), (dict(sq_h=-8), INV),
    (dict(scale=-1.0), INV), (dict(scale=float("nan")), INV), (dict(nrows=(1 << 20) + 1), UNS), (dict(max_rows=1 << 26), UNS),
])
def test_bad_cross_queries_are_refused(kw, want):
    L = _rs.lib()
    c, x = cache(), cross(**kw)
    assert attend(c, x) == want
    assert L.rs_last_error().startswith(b"cross")
    assert L.rs_cross_attn_workspace_size(C.byref(c), C.byref(x)) == 0


def test_cross_outputs_and_workspaces_are_checked():
    L = _rs.lib()
    c, x = cache(), cross()
    need = L.rs_cross_attn_workspace_size(C.byref(c), C.byref(x))
    assert need > 0 and attend(c, None) == INV
    assert attend(c, x, o=None) == INV and attend(c, x, o=4100) == INV and attend(c, x, so_h=64) == INV and attend(c, x, so_t=1023) == INV
    assert attend(c, x, ws=None) == WSP and attend(c, x, nbytes=need - 512) == WSP and attend(c, x, ws=4104) == WSP
    assert attend(c, cross(nrows=0, q=None)) == _rs.RS_OK
    for kw, want in ((dict(k=None), INV), (dict(len=None), INV), (dict(d=96), UNS), (dict(page=100), UNS)):
        assert attend(cache(**kw), x) == want
        assert L.rs_cross_attn_workspace_size(C.byref(cache(**kw)), C.byref(x)) == 0
    # more workgroups than a launch holds: refused, and no workspace would do
    many = dict(nseq=65535, hkv=256, npages=1 << 20)
    big = cross(hq=256, nrows=1 << 16, max_rows=1, start=4096)
    assert attend(cache(**many), big) == UNS
    assert L.rs_cross_attn_workspace_size(C.byref(cache(**many)), C.byref(big)) == 0


def test_bindings_refuse_what_does_not_fit():
    import torch
    x = torch.zeros(4, 2, 64)
    with pytest.raises(ValueError):
        _rs.RopeRows([(x, x[:, :1])])
    with pytest.raises(ValueError):
        _rs.RopeRows([(x, x.bfloat16())])
    with pytest.raises(ValueError):
        _rs.RopeRows([(x, x), (x[:3], x[:3])])
    with pytest.raises(ValueError):
        _rs.RopeRows([])
    with pytest.raises(ValueError):
        _rs.RopeRows([(x.half(), x.half())])
    with pytest.raises(ValueError):
        _rs.RopeRows([(x.transpose(1, 2), x.transpose(1, 2))])
    with pytest.raises(ValueError):
        _rs.RopeRows([(x, x)], pos=torch.zeros(4, dtype=torch.int64))
    with pytest.raises(ValueError):
        _rs.RopeRows([(x, x)], pos=torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError):
        _rs.rs_rope_apply(_rs.Rope(64), _rs.RopeRows([(x, x)]))  # not on a GPU
    one = _rs.RopeRows([(x[:1].transpose(0, 1).contiguous().transpose(0, 1), torch.zeros(1, 2, 64))])
    assert one.c.part[0].sx_t == 64                           # a dimension of one entry has any stride
    k = torch.zeros(2, 2, 64, 64)
    c = _rs.KvCache(k, k.clone(), torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError):
        _rs.rs_cache_append_rope(c, _rs.Rope(64), x, x, q=x[:2])
    with pytest.raises(ValueError):
        _rs.rs_cache_append_rope(c, _rs.Rope(64), x, x, pos=torch.zeros(5, dtype=torch.int32))
    with pytest.raises(ValueError):
        _rs.Cross(x, kmask=torch.zeros(2, 2))
    with pytest.raises(ValueError):
        _rs.Cross(x[0])
    m = _rs.Cross(x, max_rows=2, kmask=torch.zeros(3, 2, dtype=torch.int32))
    with pytest.raises(ValueError):
        _rs.rs_cross_attn(c, m, torch.zeros(4, 2, 64, dtype=torch.bfloat16), None, None)
