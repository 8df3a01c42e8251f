"""The calls of a decoder layer together: a rotated prompt through the dense prefill and into the cache, decode steps whose rows
are rotated on their way into it, self-attention over it, and cross attention over an encoder's states - against the fp64 oracle."""
import numpy as np
import pytest

from oracle import decode as OD
from paper_2608_29058_amd import _rs
from cross_helpers import Encoded
from decode_helpers import check_rows
from rope_helpers import Rot, bits, rows
from synth import gen as G

pytestmark = pytest.mark.gpu


def test_prompt_then_steps():
    import torch
    hq, hkv, d, n, page, steps = 8, 2, 128, 200, 64, 4
    rot = Rot(64, base=10000.0)
    q, qv = rows(1, n + steps, hq, d, "bf16")
    k, kv = rows(2, n + steps, hkv, d, "bf16")
    v, vv = rows(3, n + steps, hkv, d, "bf16")
    enc = Encoded(4, [90], [1], hq=hq, hkv=hkv, d=d, hide=0.2)
    npages = (n + steps + page - 1) // page
    pk = torch.zeros(npages, hkv, page, d, dtype=torch.bfloat16, device="cuda")
    pv = torch.zeros_like(pk)
    ln, seen = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    cache = _rs.KvCache(pk, pv, ln, seen=seen)
    # the prompt: Q and K [heads, n, d] turned in one launch, the dense prefill, the rows into the cache
    qr, kr = (torch.empty(h, n, d, dtype=torch.bfloat16, device="cuda") for h in (hq, hkv))
    _rs.rs_rope_apply(rot.rope, _rs.RopeRows([(q[:n], qr.transpose(0, 1)), (k[:n], kr.transpose(0, 1))]))
    vt = v[:n].transpose(0, 1).contiguous()
    layer = _rs.make_qkv(qr, kr, vt)
    units = _rs.make_units([(h, 0, n) for h in range(hq)])
    po, plse = torch.empty(hq, n, d, dtype=torch.bfloat16, device="cuda"), torch.empty(hq, n, device="cuda")
    ws = _rs.workspace(_rs.rs_attn_workspace_size(layer, units, hq))
    _rs.rs_dense_attn_prefill(layer, units, hq, po, plse, ws)
    _rs.rs_cache_append_rope(cache, rot.rope, k[:n], v[:n], max_rows=n)
    _rs.rs_cache_commit(cache, torch.full((1,), n, dtype=torch.int32, device="cuda"), n)
    assert torch.equal(bits(pk.transpose(1, 2).reshape(-1, hkv, d)[:n]), bits(kr.transpose(0, 1)))
    # the oracle goes on with the rotated rows as the library rounded them
    assert ln.tolist() == seen.tolist() == [n]
    one = torch.ones(1, dtype=torch.int32, device="cuda")
    for i in range(steps):
        r = slice(n + i, n + i + 1)
        qi = torch.empty(1, hq, d, dtype=torch.bfloat16, device="cuda")
        _rs.rs_cache_append_rope(cache, rot.rope, k[r], v[r], q=q[r], q_out=qi)
        draft = _rs.Draft(qi)
        o, l = torch.empty_like(qi), torch.empty(hq, 1, device="cuda")
        _rs.rs_draft_attn(cache, draft, o, l, _rs.workspace(_rs.rs_draft_attn_workspace_size(cache, draft)))
        want_q, ab = rot.oracle(qv[r], [n + i])
        assert (np.abs(qi.double().cpu().numpy() - want_q) <= 2.0 ** -8 * np.abs(want_q) * 1.01 + 2.0 ** -21 * ab * 1.01).all()

        class Step:  # what check_rows reads
            dtype, lens, max_rows, rows = "bf16", np.array([n + i], np.int32), 1, [(0, 1)]
        Step.d = d
        ref = OD.draft(qi.double().cpu().numpy(), pk.double().cpu().numpy(), pv.double().cpu().numpy(), [n + i],
                       np.arange(npages, dtype=np.int32)[None], page, [(0, 1)], None, npages * page, 1 / np.sqrt(d))
        check_rows(Step, ref, o, l)
        # then the other attention, its queries the rows as they come
        enc.dq.copy_(o)
        enc.q = o.float().cpu().numpy()
        co, cl = enc.run()
        check_rows(enc, enc.oracle(), co, cl)
        _rs.rs_cache_commit(cache, one, 1)
    assert ln.tolist() == [n + steps]
    # keys in the cache are those of their positions
    got = pk.transpose(1, 2).reshape(-1, hkv, d)[:n + steps].double().cpu().numpy()
    want, ab = rot.oracle(kv, np.arange(n + steps))
    assert (np.abs(got - want) <= 2.0 ** -8 * np.abs(want) * 1.01 + 2.0 ** -21 * ab * 1.01).all()


def test_an_evicted_cache_goes_on_at_its_tokens_positions():
    """After an eviction rows are fewer than tokens: new keys are turned by the tokens' positions, not the rows'."""
    import torch
    hkv, d, page = 2, 64, 64
    rot = Rot(64)
    pk = torch.zeros(2, hkv, page, d, dtype=torch.bfloat16, device="cuda")
    pv, ln, seen = torch.zeros_like(pk), torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    acc, pos = torch.zeros(1, hkv, 128, device="cuda"), torch.zeros(1, hkv, 128, dtype=torch.int32, device="cuda")
    c = _rs.KvCache(pk, pv, ln, acc=acc, pos=pos, seen=seen)
    k, _ = rows(1, 100, hkv, d, "bf16")
    _rs.rs_cache_append_rope(c, rot.rope, k, k, max_rows=100)
    _rs.rs_cache_commit(c, torch.full((1,), 100, dtype=torch.int32, device="cuda"), 100)
    ws = _rs.workspace(_rs.rs_cache_evict_workspace_size(c, 40))
    _rs.rs_cache_evict(c, 40, 4, 8, ws)
    new, nv = rows(2, 3, hkv, d, "bf16")
    _rs.rs_cache_append_rope(c, rot.rope, new, new, max_rows=3)
    _rs.rs_cache_commit(c, torch.full((1,), 3, dtype=torch.int32, device="cuda"), 3)
    want = torch.empty_like(new)
    _rs.rs_rope_apply(rot.rope, _rs.RopeRows([(new, want)], pos0=100))
    assert ln.tolist() == [43] and seen.tolist() == [103] and pos[0, 0, 40:43].tolist() == [100, 101, 102]
    assert torch.equal(bits(pk[0, :, 40:43].transpose(0, 1)), bits(want))
