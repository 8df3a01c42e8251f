"""CPU checks of what the decoding calls ask for and refuse before anything is launched."""
import ctypes as C

from paper_2608_29058_amd import _rs
from test_decode_host import INV, UNS, attend, cache, draft


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


def test_workspaces_hold_pieces_only_where_there_are_several():
    """Caches of one piece, and selections whose rows fill the chip, write their results themselves."""
    L = _rs.lib()
    size = lambda c, d, nsel=None: (L.rs_draft_attn_workspace_size(C.byref(c), C.byref(d)) if nsel is None
                                    else L.rs_select_attn_workspace_size(C.byref(c), C.byref(d), nsel))
    many = dict(nseq=500, npages=5000)
    assert 256 <= size(cache(**many), draft(nrows=500 * 64, max_rows=64)) <= 4096          # 256 rows per sequence
    assert size(cache(**many, max_pages=40), draft(nrows=500 * 64, max_rows=64)) > 500 * 2 * 256 * 128 * 4
    c, d, nsel = cache(**many, max_pages=400, page=64), draft(nrows=500), 10
    blocks, scores = 500 * 2 * nsel * 4, 500 * 2 * 400 * 8
    assert blocks + scores <= size(c, d, nsel) <= blocks + scores + 4096                    # 1000 items
    few = draft(nrows=3)
    assert size(c, few, nsel) > 3 * 2 * (nsel * 4 + 400 * 8) + 6 * 2 * 16 * 130 * 4


def test_more_workgroups_than_a_launch_has_are_refused():
    c = cache(nseq=65535, hkv=256, npages=1 << 18)
    d = draft(hq=256, nrows=65535)
    assert attend(c, d, nbytes=1 << 40) == UNS
    assert _rs.lib().rs_draft_attn_workspace_size(C.byref(c), C.byref(d)) == 0
    fits = draft(hq=256, nrows=32767)              # a launch of 2^23 - 256
    assert _rs.lib().rs_draft_attn_workspace_size(C.byref(cache(nseq=32767, hkv=256, npages=1 << 17)), C.byref(fits)) > 0


def test_tables_of_other_than_two_dimensions_are_refused():
    import pytest
    import torch
    k, n = torch.zeros(4, 2, 64, 64, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    for table in (torch.zeros(4, dtype=torch.int32), torch.zeros((), dtype=torch.int32), torch.zeros(2, 2, 1, dtype=torch.int32)):
        with pytest.raises(ValueError, match="table"):
            _rs.KvCache(k, k, n, table=table)
