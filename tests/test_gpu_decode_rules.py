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
