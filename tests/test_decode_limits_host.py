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
