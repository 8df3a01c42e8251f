"""Batches of prompts whose plans have several pieces per item, joined per item or per row: (hq, hkv, d, dtype, lens, rows, extra, hide).
extra: rows of no sequence; hide: share of the states that the key mask hides."""
import numpy as np


def _spread(seed, n, lo, hi):
    return np.random.default_rng(seed).integers(lo, hi + 1, n).tolist()


# the kernel of prompts (bf16, 128 rows), its pieces joined per item
ITEMS = [
    (32, 8, 128, "bf16", [2000, 0, 700, 1500], [200, 130, 3, 181], 0, None),
    (32, 8, 128, "bf16", [1300, 640, 700, 2050], [200, 0, 140, 175], 2, 0.2),
    (16, 4, 64, "bf16", [1800, 901, 33], [600, 430, 5], 0, None),
    (16, 4, 64, "bf16", [1025, 1800], [430, 600], 1, 0.4),
    (8, 2, 64, "bf16", _spread(1, 70, 0, 1600), _spread(2, 70, 0, 70), 0, None),       # more than 64 sequences, less than a round of items
    (8, 8, 128, "bf16", _spread(3, 80, 200, 1500), _spread(4, 80, 20, 45), 0, 0.1),    # more than a round of them
]
# the same kernel, joined per row
ROWS = [
    (2, 1, 128, "bf16", _spread(5, 80, 0, 1800), _spread(6, 80, 30, 70), 0, None),
    (4, 1, 64, "bf16", [9000, 513], [100, 3], 0, None),
    (8, 2, 128, "bf16", [4100], [64], 0, 0.3),
]
# tiles of 64 (bf16) and of 128 rows (fp32) that share stages, their pieces joined per item
STAGES = [
    (4, 1, 128, "bf16", [5000], [15], 4100, None),
    (4, 1, 64, "bf16", [3000, 77], [13, 16], 4100, 0.3),
    (28, 4, 64, "f32", [1500, 40], [400, 200], 0, None),
    (16, 4, 128, "f32", [1300, 0, 900], [500, 90, 440], 0, 0.3),
    (4, 4, 64, "f32", _spread(7, 70, 0, 900), _spread(8, 70, 40, 80), 0, None),
]
