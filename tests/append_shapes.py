"""Batches of new rows whose sequences differ so much that appends deal their workgroups to the rows, with queries and without:
(hq, hkv, d, dtype, page, dim, interleaved, layout, new rows of each sequence)."""

UNEVEN = [
    (32, 8, 128, "bf16", 64, 128, False, "token", [300] + [1] * 39),
    (8, 2, 128, "bf16", 64, 64, False, "token", [1, 0, 0, 700, 1, 1, 0, 3] + [0] * 48),
    (4, 2, 128, "bf16", 128, 10, False, "wide", [0] * 65 + [600]),
    (4, 4, 64, "f32", 64, 48, True, "head", [1] * 60 + [600, 1, 0]),
    (6, 2, 64, "bf16", 64, 64, False, "head", [700, 2, 1, 1, 0, 1, 257] + [0, 1] * 50),
    (7, 1, 128, "f32", 192, 128, True, "token", [5, 900, 0, 0, 0, 0, 1, 2] + [0] * 72),
    (2, 1, 64, "f32", 64, 62, False, "token", [900] + [1] * 149),
    (40, 40, 128, "bf16", 64, 128, False, "head", [700] + [0, 1] * 200),
]

# the same of the other tests, with queries: (hq, hkv, d, sequences, rows, rows of a sequence at most)
BOUNDS = (4, 2, 64, 300, 701, (170, 400, 1000, 1 << 30))
MANY = (4, 2, 64, 700, 420, (70,))
BEHIND = (30, 2, 64, 100, 94, (90,))
ABSURD = (30, 2, 128, 300, 40, (12,))
REPLAY = (30, 2, 128, 120, 159, (40,))
