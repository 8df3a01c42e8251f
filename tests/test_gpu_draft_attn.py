"""Attention of drafted rows over the paged cache (rs_draft_attn) against the fp64 oracle: lengths from none
to several pieces, head groups of 1 to 64, chains, trees and arbitrary masks with rows that see nothing,
pages in any order and missing, strides, non-finite values in places that nobody sees."""
import numpy as np
import pytest

from paper_2608_29058_amd import _rs
from decode_helpers import Setup, check_rows

pytestmark = pytest.mark.gpu


def run(s, cache=None, lse=True):
    c = cache or s.cache()
    o, l = s.outputs()
    ws = _rs.workspace(_rs.rs_draft_attn_workspace_size(c, s.draft))
    _rs.rs_draft_attn(c, s.draft, o, l if lse else None, ws)
    return o, l


LENS = [0, 1, 31, 32, 33, 63, 64, 127, 128, 129, 300, 1000]


@pytest.mark.parametrize("hq,hkv,d,dtype,page,layout", [
    (8, 2, 128, "bf16", 64, "head"),
    (4, 4, 64, "bf16", 128, "token"),
    (7, 1, 128, "f32", 64, "token"),
    (20, 4, 64, "f32", 192, "head"),
    (40, 2, 128, "bf16", 64, "head"),    # 20 rows: two row tiles of a wave
    (64, 1, 64, "bf16", 256, "head"),    # 64 rows: four
    (48, 1, 128, "f32", 64, "head"),     # 48 rows in fp32: row tiles of their own
])
def test_one_token_per_sequence(hq, hkv, d, dtype, page, layout):
    s = Setup(hq * d, LENS, [1] * len(LENS), hq=hq, hkv=hkv, d=d, dtype=dtype, page=page, layout=layout, spread=2.0)
    o, l = run(s)
    check_rows(s, s.oracle(), o, l)


@pytest.mark.parametrize("hq,hkv,d,dtype,lens,rows,kind", [
    (8, 2, 128, "bf16", [0, 5, 200, 64], [3, 1, 4, 2], None),
    (8, 2, 64, "bf16", [0, 37, 127], [33, 64, 1], "tree"),
    (4, 1, 128, "bf16", [0, 0, 90, 31], [9, 2, 40, 64], "random"),
    (28, 4, 64, "f32", [0, 61, 130], [13, 5, 13], "tree"),
    (4, 4, 128, "f32", [0, 100], [7, 70], "random"),
    (8, 2, 128, "bf16", [40, 3], [256, 100], "tree"),       # the most rows
    (8, 2, 64, "f32", [300, 45], [70, 256], "tree"),
    (14, 2, 128, "f32", [700, 0, 64], [10, 16, 1], None),   # 70 to 112 rows
    (8, 2, 128, "f32", [1000, 0], [200, 60], "random"),
    (12, 1, 128, "bf16", [333, 20], [5, 3], None),          # 36 to 60 rows
    (20, 2, 64, "bf16", [1200], [12], "tree"),              # 120 rows
    (8, 2, 64, "bf16", [63, 500], [2, 0], None),            # a sequence without new rows
    (8, 2, 128, "bf16", [2500, 0, 130], [40, 48, 33], "tree"),    # up to 192 rows: three tiles of 64
    (12, 2, 128, "bf16", [1500, 64, 7], [50, 64, 1], "random"),   # up to 384: three of 128
    (16, 4, 128, "bf16", [900, 4000], [64, 50], "tree"),          # up to 256: one
    (6, 2, 64, "bf16", [3000, 1], [33, 64], "random"),            # 192 of d = 64: two of 128
    (5, 1, 128, "f32", [2100, 31], [64, 52], "tree"),             # 320 in fp32: three of 128
])
def test_drafted_rows(hq, hkv, d, dtype, lens, rows, kind):
    s = Setup(sum(lens) + hq, lens, rows, hq=hq, hkv=hkv, d=d, dtype=dtype, kind=kind, extra=3)
    o, l = run(s)
    ref = s.oracle()
    check_rows(s, ref, o, l)
    used = int(s.start[-1])
    assert (o[used:] == -7).all() and (l[:, used:] == -7).all()
    if kind == "random" and 0 in lens:   # (rows without a draft to see, and nothing cached)
        empty = np.isneginf(ref["lse"][:, :used])
        assert empty.any() and (o[:used].cpu().float().numpy()[empty.T] == 0).all()


@pytest.mark.parametrize("hq,hkv,d,dtype,t", [
    (8, 2, 128, "bf16", 3), (28, 4, 64, "bf16", 4), (4, 4, 64, "f32", 2), (10, 2, 64, "f32", 5), (8, 2, 128, "f32", 7)])
@pytest.mark.parametrize("top", [250, 300, 505])
def test_caches_of_one_piece(hq, hkv, d, dtype, t, top):
    """Capacities around those that are attended in one piece, with infinities and NaN behind the ends."""
    lens = [top, 0, 1, 31, 32, 127, 128, 224, 225, 249, top - 32]
    rows = [1 + (3 * i) % t for i in range(len(lens))]
    s = Setup(top + hq, lens, rows, hq=hq, hkv=hkv, d=d, dtype=dtype, kind="tree" if t > 2 else None, spread=2.0)
    for b, n in enumerate(s.lens + s.counts):
        p, j = divmod(int(n), 64)
        if p < s.table.shape[1] and s.table[b, p] >= 0:
            s.dk[int(s.table[b, p]), :, j:], s.dv[int(s.table[b, p]), :, j:] = float("inf"), float("nan")
    o, l = run(s)
    check_rows(s, s.oracle(), o, l)


@pytest.mark.parametrize("hq,hkv,d,lens,rows,kind", [
    (8, 2, 128, [2500, 40, 700], [8, 5, 2], "tree"),     # 32 rows of Q
    (5, 1, 128, [5000], [5], None),                      # 25
    (3, 1, 128, [3001, 0, 900], [5, 1, 3], "tree"),      # 15
    (12, 2, 64, [4100, 333], [4, 5], "random"),          # 30
])
def test_long_fp32_caches(hq, hkv, d, lens, rows, kind):
    s = Setup(hq * d, lens, rows, hq=hq, hkv=hkv, d=d, dtype="f32", kind=kind, page=128, spread=2.0)
    o, l = run(s)
    check_rows(s, s.oracle(), o, l)


@pytest.mark.parametrize("lens,rows,hq,hkv,kind", [
    ([20011], [1], 8, 2, None),                 # one item per head, many pieces
    ([9000, 1, 0, 4097], [16, 1, 1, 3], 4, 1, "tree"),
    ([3000] * 5 + [17] * 90, [1] * 95, 4, 2, None),   # more sequences than a wave has lanes
    ([500, 0, 2100] * 20, [40, 7, 64] * 20, 8, 2, "tree"),   # items that fill the chip, of many rows
])
def test_split_sequences(lens, rows, hq, hkv, kind):
    s = Setup(7, lens, rows, hq=hq, hkv=hkv, d=128, page=128, kind=kind, spread=3.0)
    o, l = run(s)
    check_rows(s, s.oracle(), o, l)
    again, _ = run(s)
    assert (again == o).all()


def test_without_table_start_and_lse_on_an_odd_buffer():
    import torch
    s = Setup(3, [37, 100, 0], [2, 2, 2], page=103, table=False)
    s.lens[1] = s.dlen[1] = 102                     # capacity 103: the second drafted row has no place
    s.draft = _rs.Draft(s.dq, max_rows=2)
    c = s.cache()
    assert c.cap == 103
    o, l = run(s, c, lse=False)
    check_rows(s, s.oracle(), o, None)
    assert (l == -7).all()
    # strided queries and outputs: heads of a wider projection
    wide = torch.zeros((s.nrows, s.hq + 4, s.d + 16), dtype=torch.bfloat16, device="cuda")
    wide[:, 2:2 + s.hq, 8:8 + s.d] = s.dq
    out = torch.full_like(wide, -7)
    dr = _rs.Draft(wide[:, 2:2 + s.hq, 8:8 + s.d], max_rows=2)
    ws = _rs.workspace(_rs.rs_draft_attn_workspace_size(c, dr))
    _rs.rs_draft_attn(c, dr, out[:, 2:2 + s.hq, 8:8 + s.d], None, ws)
    assert (out[:, 2:2 + s.hq, 8:8 + s.d] == o).all()
    out[:, 2:2 + s.hq, 8:8 + s.d] = -7
    assert (out == -7).all()


def test_lengths_and_starts_out_of_range_are_clamped():
    import torch
    from oracle import decode as OD
    s = Setup(11, [70, 64, 50, 30], [2, 3, 1, 2], page=64, room=64)
    s.lens[0], s.lens[1] = -5, 10 ** 6            # none; the whole capacity, no room for drafts
    s.start[:] = [-3, 2, 4, 4, 99]                # the fourth sequence's rows run past max_rows and the end
    s.dlen.copy_(torch.from_numpy(s.lens))
    s.dstart.copy_(torch.from_numpy(s.start))
    s.table[1] = s.table[2]                        # (a full table for the overlong sequence)
    s.dtable.copy_(torch.from_numpy(s.table))
    s.rows = OD.row_ranges(s.start, 4, s.nrows, s.max_rows)
    o, l = run(s)
    ref = s.oracle()
    assert s.rows == [(0, 2), (2, 2), (4, 0), (4, 3)]
    check_rows(s, ref, o, l)


@pytest.mark.parametrize("dtype,bad", [("bf16", -1), ("f32", 10 ** 6), ("bf16", -2 ** 31)])
def test_rows_without_a_page_are_not_seen(dtype, bad):
    import torch
    s = Setup(5, [300, 40], [3, 1], dtype=dtype)
    s.table[0, 1] = s.table[0, 4] = bad            # cached rows, and the page of the drafted ones
    s.table[1, 0] = bad                            # a sequence that has nothing left
    spare = (set(range(s.k.shape[0])) - set(s.table.ravel().tolist()) - {0}).pop()
    s.table[s.table == 0] = spare                  # page 0 belongs to nobody, and holds nothing good
    s.dtable.copy_(torch.from_numpy(s.table))
    s.dk[0], s.dv[0] = float("nan"), float("nan")
    o, l = run(s)
    ref = s.oracle()
    assert np.isneginf(ref["lse"][:, 3]).all()
    check_rows(s, ref, o, l)


@pytest.mark.parametrize("dtype,hq", [("bf16", 8), ("f32", 8), ("bf16", 24), ("f32", 24), ("bf16", 40), ("bf16", 80), ("f32", 80)])
def test_values_that_nobody_sees_do_no_harm(dtype, hq):
    """Drafted rows of other branches, and whatever lies behind a sequence, hold infinities and NaN."""
    import torch
    s = Setup(9, [50, 131], [5, 4], dtype=dtype, kind="tree", hq=hq)
    m = np.zeros((s.nrows, 32), bool)
    for f, t in s.rows:
        m[f:f + t, :t] = np.eye(t, dtype=bool)
    s.mask = np.packbits(m, axis=1, bitorder="little").view(np.int32)
    s.dmask.copy_(torch.from_numpy(s.mask))
    at = lambda b, j: (int(s.table[b, j // 64]), slice(None), j % 64)
    plain, _ = run(s)
    for b, j, kv, x in ((0, 52, s.dv, float("nan")), (0, 53, s.dv, float("inf")), (1, 132, s.dk, float("nan")),
                        (1, 133, s.dk, -float("inf")), (0, 55, s.dv, float("nan")), (1, 140, s.dk, float("inf"))):
        kv[at(b, j)] = x
    o, l = run(s)
    for r in range(9):
        if r in (2, 3, 6, 7):
            continue
        assert torch.equal(o[r], plain[r]), r
    assert o[2].isnan().all() and (o[3] == float("inf")).all() and o[6].isnan().all()


def test_scale_and_large_logits():
    s = Setup(21, [400, 3], [2, 2], d=128, scale=0.5, spread=40.0)
    o, l = run(s)
    check_rows(s, s.oracle(), o, l)


def test_cache_beyond_32_bit_offsets():
    """Pages 5 GiB into the buffers (element offsets beyond 2^31, byte offsets beyond 2^32)."""
    import torch
    s = Setup(13, [150, 90], [1, 2], hq=4, hkv=2, d=128, page=64)
    big = torch.zeros((5 << 30) // (2 * 64 * 128 * 2) + 8, 2, 64, 128, dtype=torch.bfloat16, device="cuda")
    base = big.shape[0] - s.dk.shape[0]
    big[base:] = s.dk
    keep = big[base:].clone()
    c = _rs.KvCache(big, big, s.dlen, table=s.dtable + base)
    s.v = s.k
    o, l = run(s, c)
    check_rows(s, s.oracle(), o, l)
    assert torch.equal(big[base:], keep)


def test_two_streams_and_graph_replays():
    import torch
    s = Setup(17, [700, 5000, 3], [1, 4, 2], hq=8, hkv=2, d=128, page=128, kind="tree")
    c = s.cache()
    want, wl = run(s)
    o, l = s.outputs()
    ws = [_rs.workspace(_rs.rs_draft_attn_workspace_size(c, s.draft)) for _ in range(2)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    o2, l2 = s.outputs()
    side.wait_stream(torch.cuda.current_stream())
    _rs.rs_draft_attn(c, s.draft, o2, l2, ws[1], stream=side)
    _rs.rs_draft_attn(c, s.draft, o, l, ws[0])
    torch.cuda.synchronize()
    assert torch.equal(o, want) and torch.equal(o2, want) and torch.equal(l2, wl)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        _rs.rs_draft_attn(c, s.draft, o, l, ws[0])
    for n in (700, 2, 640):
        s.dlen[0] = n
        eager, el = run(s)
        o.fill_(-7)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, eager) and torch.equal(l, el)


def test_shared_pages_and_head_major_outputs():
    """Sequences that share the pages of their beginning; O as [hq][nrows][d]."""
    import torch
    s = Setup(23, [200, 330, 64], [2, 1, 3], hq=8, hkv=2, d=128, page=64)
    s.table[1, :3] = s.table[0, :3]
    s.table[2, 0] = s.table[0, 0]
    s.dtable.copy_(torch.from_numpy(s.table))
    c = s.cache()
    o = torch.full((s.hq, s.nrows, s.d), -7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.empty(s.hq, s.nrows, device="cuda")
    _rs.rs_draft_attn(c, s.draft, o.transpose(0, 1), lse, _rs.workspace(_rs.rs_draft_attn_workspace_size(c, s.draft)))
    check_rows(s, s.oracle(), o.transpose(0, 1), lse)
