"""What the decoding calls do at the edges of their definitions: roundings, untouched rows, refusals beside valid
arguments."""
import pytest

from paper_2608_29058_amd import _rs
from decode_helpers import Setup

pytestmark = pytest.mark.gpu


def test_means_round_to_fp32_and_then_to_bf16():
    """A mean just above the middle of two bf16 values whose fp32 rounding is the middle: to the even one."""
    import torch
    k = torch.zeros((2, 1, 64, 64), device="cuda")
    mid = 1.0 + 2.0 ** -8
    k[0] = mid
    k[0, 0, 0, 0] = mid + 2.0 ** -23               # mean mid + 2^-29: fp32 has 2^-23 there
    k[0, 0, :, 1] = mid + 2.0 ** -23               # mean mid + 2^-23 is one of fp32: up
    k[1] = -k[0]
    n = torch.zeros(2, dtype=torch.int32, device="cuda")
    km = torch.zeros((2, 1, 1, 64), dtype=torch.bfloat16, device="cuda")
    c = _rs.KvCache(k, k.clone(), n, kmean=km)
    _rs.rs_cache_commit(c, torch.tensor([64, 64], dtype=torch.int32, device="cuda"), 64)
    want = torch.full((64,), 1.0)
    want[1] = 1.0 + 2.0 ** -7
    assert torch.equal(km[0, 0, 0].float().cpu(), want) and torch.equal(km[1, 0, 0].float().cpu(), -want)


def test_weights_of_sequences_without_new_rows_are_left():
    """acc_in and acc_out apart: rows that nobody sees are carried over, sequences without new rows are not touched."""
    import torch
    s = Setup(6, [200, 130, 64], [2, 0, 3], hq=4, hkv=2, d=64, kind="random")
    s.table[2, 0] = -1
    s.dtable.copy_(torch.from_numpy(s.table))
    o, l = s.outputs()
    _rs.rs_draft_attn(s.cache(), s.draft, o, l, _rs.workspace(_rs.rs_draft_attn_workspace_size(s.cache(), s.draft)))
    acc = torch.rand((3, 2, s.cap), device="cuda")
    out = torch.full_like(acc, -3.0)
    _rs.rs_attn_weights(s.cache(), s.draft, l, acc, out)
    assert (out[1] == -3.0).all() and (out[0, :, 202:] == -3.0).all() and (out[0, :, :202] >= acc[0, :, :202]).all()
    assert (out[2, :, :64] == -3.0).all() and (out[2, :, 64:67] >= acc[2, :, 64:67]).all()
    alone = torch.zeros(s.nrows, device="cuda")    # no row counts: what is written is what was there
    _rs.rs_attn_weights(s.cache(), s.draft, l, acc, out, row_w=alone)
    assert torch.equal(out[0, :, :202], acc[0, :, :202]) and torch.equal(out[2, :, 64:67], acc[2, :, 64:67])
