"""The launch shape of rotated appends (rope_plan.h) compiled for the host: workgroups as there are rows, however uneven the
sequences are."""
import os
import shutil
import subprocess

import pytest

from append_shapes import ABSURD, BEHIND, BOUNDS, MANY, REPLAY, UNEVEN

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SOURCE = r'''
#include <cstdio>
#include "rope_plan.h"
using namespace rs;
int main() {
  int nseq, cap, nrows, max_rows, start, d, hkv, hq, tokens, dim;
  while (scanf("%d %d %d %d %d %d %d %d %d %d", &nseq, &cap, &nrows, &max_rows, &start, &d, &hkv, &hq, &tokens, &dim) == 10) {
    rs_rope r{};
    r.dim = dim, r.layout = RS_ROPE_HALF;
    const AppendShape s = append_rope_shape(nseq, cap, nrows, max_rows, start, d, hkv, hq, tokens, r);
    printf("%d %lld %d\n", s.per, (long long)s.x * s.y, s.byrow);
  }
}
'''


@pytest.fixture(scope="module")
def shape(tmp_path_factory):
    if not shutil.which("g++"):
        pytest.skip("g++ not available")
    d = tmp_path_factory.mktemp("append")
    (d / "s.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-fsanitize=undefined", "-fno-sanitize-recover", "-I",
                    os.path.join(ROOT, "paper_2608_29058_amd", "csrc"), str(d / "s.cpp"), "-o", str(d / "s")], check=True)

    def run(**kw):
        """(rows of a workgroup, workgroups, whether they are dealt to rows)"""
        x = dict(nseq=1, cap=1 << 18, nrows=1, max_rows=1, start=1, d=128, hkv=8, hq=32, tokens=1, dim=128)
        assert set(kw) <= set(x)
        x.update(kw)
        out = subprocess.run([str(d / "s")], input=" ".join(str(int(v)) for v in x.values()), capture_output=True, text=True)
        assert out.returncode == 0, out.stdout + out.stderr
        return tuple(map(int, out.stdout.split()))

    return run


@pytest.mark.parametrize("kw", [
    dict(nseq=64, nrows=8192 + 63, max_rows=8192),                           # a chunk of a prompt among decode steps
    dict(nseq=64, nrows=8192 + 63, max_rows=8192, dim=64),
    dict(nseq=64, nrows=8192 + 63, max_rows=8192, tokens=0),
    dict(nseq=256, nrows=2048 + 255, max_rows=2048, d=64, dim=64),
    dict(nseq=65535, nrows=1 << 20, max_rows=1 << 20),
    dict(nseq=64, nrows=64, max_rows=1 << 30),                               # a bound that bounds nothing
    dict(nseq=3, nrows=1 << 24, max_rows=1 << 24, hq=0),
    dict(nseq=64, nrows=64, max_rows=1), dict(nseq=64, nrows=500, max_rows=16), dict(nseq=4, nrows=4 * 8192, max_rows=8192),
    dict(nseq=4, nrows=4 * 8192, max_rows=8192, start=0), dict(nseq=5, nrows=3, max_rows=1),
])
def test_workgroups_are_as_many_as_the_rows_need(shape, kw):
    """But for those that take less time than the search for the rows' sequences."""
    per, n, byrow = shape(**kw)
    own = -(-kw["nrows"] // per)
    assert n <= own + kw["nseq"] + 2048 + own * -(-kw["nseq"] // 256) // 2


@pytest.mark.parametrize("nseq,cap,nrows", [(1, 128, 1 << 24), (4, 1024, 1 << 20), (1, 64, 65536)])
def test_without_queries_rows_behind_the_capacity_have_no_workgroups(shape, nseq, cap, nrows):
    per, n, byrow = shape(nseq=nseq, cap=cap, nrows=nrows, max_rows=nrows // nseq, hq=0, start=0)
    assert n <= nseq * -(-cap // per)
    per, n, byrow = shape(nseq=nseq, cap=cap, nrows=nrows, max_rows=nrows, hq=0)
    assert n <= nseq * -(-cap // per)


@pytest.mark.parametrize("hq,hkv,d,dtype,page,dim,inter,layout,counts", UNEVEN)
def test_the_batches_of_the_value_tests_are_dealt_by_row(shape, hq, hkv, d, dtype, page, dim, inter, layout, counts):
    # (the interleaved layout of a part of a head does not pass through LDS: as many groups as the whole head has)
    for heads in (0, hq):
        assert shape(nseq=len(counts), nrows=sum(counts) + 3, max_rows=max(counts), d=d, hkv=hkv, hq=heads, tokens=layout != "head",
                     dim=d if inter else dim)[2] == 1


@pytest.mark.parametrize("hq,hkv,d,nseq,nrows,bounds", [ABSURD, BEHIND, BOUNDS, MANY, REPLAY])
def test_so_are_those_of_the_other_tests(shape, hq, hkv, d, nseq, nrows, bounds):
    for most in bounds:
        assert shape(nseq=nseq, nrows=nrows, max_rows=most, d=d, hkv=hkv, hq=hq, dim=d)[2] == 1


@pytest.mark.parametrize("kw", [
    dict(nseq=64, nrows=64, max_rows=1), dict(nseq=64, nrows=69, max_rows=6), dict(nseq=8, nrows=23, max_rows=16), dict(nseq=4, nrows=67, max_rows=64),
    dict(nseq=4096, nrows=4098, max_rows=3), dict(nseq=4, nrows=4 * 8192, max_rows=8192), dict(nseq=64, nrows=8192 + 63, max_rows=129, start=0),
])
def test_short_and_even_batches_are_dealt_by_sequence(shape, kw):
    assert shape(**kw)[2] == 0
