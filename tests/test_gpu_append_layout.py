"""New rows without row starts: sequence b's are [b max_rows, (b + 1) max_rows) whatever a sequence can hold."""
import numpy as np
import pytest

from paper_2608_29058_amd import _rs
from decode_helpers import Setup

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens", [[0, 0, 0], [100, 0, 127], [128, 3, 64]])
@pytest.mark.parametrize("max_rows", [100, 128, 150, 1000])
def test_sequences_keep_their_rows_beyond_the_capacity(lens, max_rows):
    import torch
    s = Setup(max_rows, lens, [1, 1, 1], d=64, page=128)
    cap = 128
    s.dtable = s.dtable[:, :1].contiguous()        # (one page each)
    s.table = s.table[:, :1]
    c = s.cache()
    assert c.cap == cap
    r = np.random.default_rng(1)
    new = [torch.from_numpy(r.standard_normal((3 * max_rows, s.hkv, 64)).astype(np.float32)).to(torch.bfloat16).cuda()
           for _ in range(2)]
    _rs.rs_cache_append(c, new[0], new[1], max_rows=max_rows)
    k, v = s.k.copy(), s.v.copy()
    for b, n in enumerate(lens):
        p, m = int(s.table[b, 0]), min(max_rows, cap - n)
        f = b * max_rows
        k[p, :, n:n + m] = new[0][f:f + m].float().cpu().numpy().transpose(1, 0, 2)
        v[p, :, n:n + m] = new[1][f:f + m].float().cpu().numpy().transpose(1, 0, 2)
    assert np.array_equal(s.dk.float().cpu().numpy(), k) and np.array_equal(s.dv.float().cpu().numpy(), v)
