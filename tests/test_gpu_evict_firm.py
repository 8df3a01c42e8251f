"""Firm rows stay whatever the others' weights hold, NaN of any sign and payload among them."""
import numpy as np
import pytest

from paper_2608_29058_amd import _rs
from decode_helpers import Setup

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [0x7fffffff, 0x7fc00000, 0x7f800001, 0xffffffff, 0xffc00000])
@pytest.mark.parametrize("n", [700, 5000, 40000])
def test_undefined_weights_do_not_displace_firm_rows(n, bits):
    import torch
    s = Setup(3, [n], [0], hq=1, hkv=1, d=64, page=1024 if n > 1024 else 64)
    budget, nsink, nrecent = 90, 10, 70            # ten places for others
    acc = np.full((1, 1, s.cap), bits, np.uint32)
    acc[0, 0, 1::2] = np.float32(0.5).view(np.uint32)
    pos = np.full((1, 1, s.cap), 5000, np.int32)
    firm = np.random.default_rng(2).permutation(np.arange(n // 2, n))[:80]
    pos[0, 0, firm] = np.concatenate([np.arange(10), 100000 - 70 + np.arange(70)])
    dacc, dpos = torch.from_numpy(acc.view(np.float32)).cuda(), torch.from_numpy(pos).cuda()
    c = s.cache(acc=dacc, pos=dpos, seen=torch.tensor([100000], dtype=torch.int32, device="cuda"))
    _rs.rs_cache_evict(c, budget, nsink, nrecent, _rs.workspace(_rs.rs_cache_evict_workspace_size(c, budget)))
    assert s.dlen.item() == budget
    kept = dpos[0, 0, :budget].tolist()
    assert sorted(x for x in kept if x != 5000) == list(range(10)) + list(range(100000 - 70, 100000))
    src = {int(pos[0, 0, j]): j for j in firm}     # and each brings its own row
    for at, x in enumerate(kept):
        if x != 5000:
            j = src[x]
            assert np.array_equal(s.dk[int(s.table[0, at // s.page]), 0, at % s.page].float().cpu().numpy(),
                                  s.k[int(s.table[0, j // s.page]), 0, j % s.page])
