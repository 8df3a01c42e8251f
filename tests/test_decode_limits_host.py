"""CPU checks of what the decoding calls ask for and refuse before anything is launched."""
import ctypes as C

from paper_2608_29058_amd import _rs
from test_decode_host import INV, cache


def test_new_rows_without_starts_are_max_rows_apart_beyond_the_capacity_too():
    """Two sequences of 300 rows each are 600 rows, though a sequence holds 256."""
    L = _rs.lib()
    c = cache()
    assert c.page * c.max_pages == 256
    assert L.rs_cache_append(C.byref(c), 4096, 4096, 256, 128, 256, 128, None, 512, 300, None) == INV
    assert L.rs_cache_append(C.byref(c), 4096, 4096, 256, 128, 256, 128, None, 599, 300, None) == INV


def test_workspaces_elsewhere_or_with_gaps_are_refused():
    """Every call that takes one, with arguments that fit otherwise (the device of the cache is not the host's here)."""
    import pytest
    import torch
    for device, ws in (("meta", torch.zeros(1 << 16, dtype=torch.uint8)),
                       ("cpu", torch.zeros(1 << 17, dtype=torch.uint8)[::2]),
                       ("cpu", torch.zeros(1, dtype=torch.uint8).expand(1 << 16)),
                       ("cpu", torch.zeros(1 << 16, dtype=torch.uint8, device="meta"))):
        z = lambda *s, dt=torch.bfloat16: torch.zeros(*s, dtype=dt, device=device)
        k, n = z(2, 2, 64, 64), z(2, dt=torch.int32)
        acc, pos = z(2, 2, 64, dt=torch.float32), z(2, 2, 64, dt=torch.int32)
        c = _rs.KvCache(k, k, n, kmean=z(2, 2, 1, 64), acc=acc, pos=pos, seen=n)
        d, o, lse = _rs.Draft(z(2, 2, 64)), z(2, 2, 64), z(2, 2, dt=torch.float32)
        for f in (lambda: _rs.rs_draft_attn(c, d, o, lse, ws), lambda: _rs.rs_select_attn(c, d, 1, 0, 0, o, lse, ws),
                  lambda: _rs.rs_cache_evict(c, 8, 0, 0, ws)):
            with pytest.raises(ValueError, match="workspace"):
                f()
