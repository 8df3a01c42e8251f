"""The plan of pieces of prompts in cross attention (cross_plan.h) compiled for the host: what fits is split, whatever the capacity
rounds to, and no plan has more pieces than there is room for."""
import os
import shutil
import subprocess

import numpy as np
import pytest

from cross_shapes import ITEMS, ROWS

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SOURCE = r'''
#include <cstdio>
#include <vector>
#include "cross_plan.h"
using namespace rs;
// cases: hq hkv nseq cap max_rows nrows, then len and rows of each sequence -> grid, items (host), items, groups per piece, pieces
int main() {
  for (int t = 1; t <= 2048; ++t)
    for (int per = 1; per <= 2048; ++per)
      if (pieces_by(t, per, 1.f / (float)per) != pieces_of(t, per)) return printf("pieces_by %d %d\n", t, per), 1;
  int hq, hkv, nseq, cap, max_rows, nrows;
  while (scanf("%d %d %d %d %d %d", &hq, &hkv, &nseq, &cap, &max_rows, &nrows) == 6) {
    std::vector<int> items, groups;
    const int G = hq / hkv;
    int all = 0, work = 0, longest = 0;
    for (int b = 0; b < nseq; ++b) {
      int len, t;
      if (scanf("%d %d", &len, &t) != 2) return 2;
      items.push_back(hkv * ((G * t + 127) / 128));
      groups.push_back(t > 0 ? (len + kGroup - 1) / kGroup : 0);
      all += items[b], work += items[b] * groups[b];
      longest = longest > groups[b] ? longest : groups[b];
    }
    CacheView c{};
    DraftView q{};
    c.nseq = nseq, c.hkv = hkv, q.hq = hq, q.nrows = nrows;
    const int64_t most = cross_tiles(c, q, G * (nrows < max_rows ? nrows : max_rows), 128) * hkv;
    const RoundsShape s = rounds_shape(most, cap, 512);
    auto pieces = [&](int per) {
      int n = 0;
      for (int b = 0; b < nseq; ++b) n += items[b] * pieces_of(groups[b], per);
      return n;
    };
    const int per = s.split ? rounds_groups(all, work, longest, 512, s.grid, s.least, pieces) : longest;
    printf("%d %lld %d %d %d\n", s.grid, (long long)most, all, per, pieces(per));
  }
  return 0;
}
'''


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    if not shutil.which("g++"):
        pytest.skip("g++ not available")
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-O1", "-std=c++17", "-fsanitize=undefined", "-fno-sanitize-recover", "-I",
                    os.path.join(ROOT, "paper_2608_29058_amd", "csrc"), str(d / "plan.cpp"), "-o", str(d / "plan")], check=True)

    def run(cases):
        """[(hq, hkv, lens, rows)] -> [(grid, items at most, items, groups per piece, pieces)]"""
        text = []
        for hq, hkv, lens, rows in cases:
            cap = max(1, -(-max(lens) // 64)) * 64
            text.append(" ".join(map(str, [hq, hkv, len(lens), cap, max(rows), sum(rows)] + [int(x) for p in zip(lens, rows) for x in p])))
        out = subprocess.run([str(d / "plan")], input="\n".join(text), capture_output=True, text=True)
        assert out.returncode == 0, out.stdout + out.stderr
        return [tuple(map(int, line.split())) for line in out.stdout.splitlines()]

    return run


@pytest.mark.parametrize("hq,hkv,lens,rows,want", [
    # few items: pieces of four groups, as long as one round has room for them
    (32, 8, [4000], [64], 128), (32, 8, [3900], [64], 128), (32, 8, [2000], [64], 64),
    (8, 2, [16000], [64], 128), (32, 8, [1500], [100], 96), (16, 16, [1500], [200], 96),
    (12, 12, [1500], [300], 108), (4, 1, [20000], [50], 80),
    (4, 1, [20000, 100], [50, 3], 81), (4, 1, [9000], [100], 72),
    (2, 2, [5000, 0, 700, 64], [70, 130, 1, 200], 2 * (10 + 2 + 2 + 2)),
    (4, 4, [512], [64], 4),            # no sequence is long enough for two pieces
    (1, 1, [0, 0], [64, 200], 3),      # nor is there one at all
])
def test_few_prompts_are_split(plan, hq, hkv, lens, rows, want):
    (grid, most, items, per, pieces), = plan([(hq, hkv, lens, rows)])
    assert pieces == want and items <= most and pieces <= grid


def batches(seed, n):
    r = np.random.default_rng(seed)
    for _ in range(n):
        nseq = int(2 ** r.uniform(0, 8))
        hkv = int(r.choice([1, 2, 4, 8, 16]))
        hq = hkv * int(r.choice([1, 2, 4, 7, 16]))
        hi = int(2 ** r.uniform(6, 16))
        yield hq, hkv, r.integers(r.choice([0, hi // 2, hi]), hi + 1, nseq).tolist(), r.integers(r.choice([0, 1]), 2 + int(2 ** r.uniform(0, 9)), nseq).tolist()


def test_plans_fit_their_room(plan):
    cases = [c for c in batches(1, 4000) if max(c[3]) > 0]
    for (hq, hkv, lens, rows), (grid, most, items, per, pieces) in zip(cases, plan(cases)):
        assert items <= most and pieces <= grid, (hq, hkv, lens, rows)


def test_one_round_is_shared_among_its_workgroups(plan):
    """Fewer items than workgroups: at P groups a piece, P the larger of four and all groups over the room that the items leave,
    they fit, so that no piece is longer than that."""
    cases = [c for c in batches(2, 4000) if max(c[3]) > 0]
    checked = 0
    for (hq, hkv, lens, rows), (grid, most, items, per, pieces) in zip(cases, plan(cases)):
        if not 0 < items < 256 or max(lens) <= 512:
            continue
        tiles = [hkv * -(-hq // hkv * t // 128) for t in rows]
        work = sum(a * -(-n // 128) for a, n in zip(tiles, lens))
        longest = max(-(-n // 128) if t else 0 for n, t in zip(lens, rows))
        bound = max(4, -(-work // (512 - items)))
        # (more rounds of shorter pieces, or whole items where pieces cost more than they save, may be estimated as faster)
        if longest * 128 > bound * 128 + 512:
            checked += 1
            assert per <= bound, (hq, hkv, lens, rows, per, bound)
    assert checked > 100


def test_the_batches_of_the_value_tests_have_several_pieces(plan):
    """Those that the kernel of prompts takes in tests of the joins."""
    shapes = ITEMS + ROWS
    for x, (grid, most, items, per, pieces) in zip(shapes, plan([(hq, hkv, lens, rows) for hq, hkv, d, dtype, lens, rows, extra, hide in shapes])):
        assert items < pieces <= grid, x
