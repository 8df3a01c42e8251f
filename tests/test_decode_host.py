"""CPU checks of decoding: the calls refuse what they cannot do before anything is launched, and the
kernels' address arithmetic (pages, lengths, row ranges) stays in bounds for any table, length and start."""
import ctypes as C
import os
import shutil
import subprocess

import numpy as np
import pytest

from paper_2608_29058_amd import _rs

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INV, UNS, WSP = _rs.RS_ERR_INVALID_ARG, _rs.RS_ERR_UNSUPPORTED, _rs.RS_ERR_WORKSPACE


def cache(**kw):
    a = dict(k=4096, v=4096, dtype=0, nseq=2, hkv=2, d=128, page=64, npages=8, max_pages=4, table=4096, len=4096,
             sk_p=2 * 64 * 128, sk_h=64 * 128, sk_t=128, sv_p=2 * 64 * 128, sv_h=64 * 128, sv_t=128, kmean=4096, acc=4096,
             pos=4096, seen=4096)
    a.update(kw)
    return _rs.RsCache(**a)


def draft(**kw):
    a = dict(q=4096, hq=8, nrows=2, max_rows=1, nwords=1, sq_t=8 * 128, sq_h=128, start=4096, mask=None, scale=0.0)
    a.update(kw)
    return _rs.RsDraft(**a)


def attend(c, d, o=4096, so_t=1024, so_h=128, ws=4096, nbytes=1 << 30, nsel=None, nsink=0, nlocal=0):
    L = _rs.lib()
    if nsel is None:
        return L.rs_draft_attn(C.byref(c), C.byref(d), o, so_t, so_h, None, ws, nbytes, None)
    return L.rs_select_attn(C.byref(c), C.byref(d), nsel, nsink, nlocal, o, so_t, so_h, None, None, ws, nbytes, None)


@pytest.mark.parametrize("kw,want", [
    (dict(k=None), INV), (dict(len=None), INV), (dict(dtype=2), INV), (dict(d=96), UNS), (dict(nseq=0), INV),
    (dict(hkv=0), INV), (dict(page=0), INV), (dict(page=32), UNS), (dict(page=100), UNS), (dict(max_pages=1 << 20), UNS),
    (dict(table=None, npages=7), INV), (dict(sk_t=64), INV), (dict(sv_h=4), INV), (dict(sk_p=-8), INV), (dict(k=4100), INV),
    (dict(kmean=4104), INV), (dict(sk_t=1 << 24), UNS),
])
def test_bad_caches_are_refused(kw, want):
    L = _rs.lib()
    c, d = cache(**kw), draft()
    calls = [lambda: attend(c, d), lambda: attend(c, d, nsel=4),
             lambda: L.rs_attn_weights(C.byref(c), C.byref(d), 4096, None, None, 4096, None),
             lambda: L.rs_cache_append(C.byref(c), 4096, 4096, 256, 128, 256, 128, 4096, 2, 1, None),
             lambda: L.rs_cache_commit(C.byref(c), 4096, None, 1, None),
             lambda: L.rs_cache_evict(C.byref(c), 64, 0, 0, 4096, 1 << 30, None)]
    for f in calls:
        assert f() == want, L.rs_last_error()
        assert L.rs_last_error().startswith(b"cache")
    assert L.rs_draft_attn_workspace_size(C.byref(c), C.byref(d)) == 0
    assert L.rs_select_attn_workspace_size(C.byref(c), C.byref(d), 4) == 0
    assert L.rs_cache_evict_workspace_size(C.byref(c), 64) == 0


@pytest.mark.parametrize("kw,want", [
    (dict(q=None), INV), (dict(q=4104), INV), (dict(hq=7), INV), (dict(nrows=-1), INV), (dict(max_rows=0), INV),
    (dict(max_rows=257), UNS), (dict(start=None, nrows=1), INV), (dict(mask=4096, max_rows=33), INV), (dict(sq_t=4), INV),
    (dict(scale=-1.0), INV), (dict(scale=float("nan")), INV), (dict(nrows=1 << 21), UNS),
    (dict(hq=0), INV),
])
def test_bad_drafts_are_refused(kw, want):
    L = _rs.lib()
    c, d = cache(), draft(**kw)
    assert attend(c, d) == want and attend(c, d, nsel=4) == want
    assert L.rs_attn_weights(C.byref(c), C.byref(d), 4096, None, None, 4096, None) == want
    assert L.rs_draft_attn_workspace_size(C.byref(c), C.byref(d)) == 0


def test_outputs_workspaces_and_budgets_are_checked():
    L = _rs.lib()
    c, d = cache(), draft()
    need = L.rs_draft_attn_workspace_size(C.byref(c), C.byref(d))
    assert need > 0
    assert attend(c, d, o=None) == INV and attend(c, d, o=4100) == INV and attend(c, d, so_h=64) == INV
    assert attend(c, d, so_t=1023) == INV
    assert attend(c, d, ws=None) == WSP and attend(c, d, nbytes=need - 512) == WSP and attend(c, d, ws=4104) == WSP
    for nsel, a, b, want in ((0, 0, 0, INV), (4, 3, 2, INV), (4, -1, 0, INV), (5000, 0, 0, UNS)):
        assert attend(c, d, nsel=nsel, nsink=a, nlocal=b) == want
    assert attend(cache(kmean=None), d, nsel=4) == INV
    need = L.rs_select_attn_workspace_size(C.byref(c), C.byref(d), 2)
    assert attend(c, d, nsel=2, nbytes=need - 512) == WSP
    w = lambda lse, out: L.rs_attn_weights(C.byref(c), C.byref(d), lse, None, None, out, None)
    assert w(None, 4096) == INV and w(4096, None) == INV
    a = lambda **k: L.rs_cache_append(C.byref(c), *[dict(dict(kn=4096, vn=4096, a=256, b=128, c=256, d=128, st=4096, n=2, m=1), **k)[x]
                                                    for x in ("kn", "vn", "a", "b", "c", "d", "st", "n", "m")], None)
    assert a(kn=None) == INV and a(vn=4100) == INV and a(a=4) == INV and a(n=-1) == INV and a(m=0) == INV
    assert a(st=None, n=1) == INV and a(n=0) == _rs.RS_OK
    m = lambda cc, na=4096, path=None, mx=1: L.rs_cache_commit(C.byref(cc), na, path, mx, None)
    assert m(c, na=None) == INV and m(c, mx=0) == INV and m(c, mx=1 << 19) == INV
    assert m(c, path=4096, mx=257) == UNS and m(cache(seen=None)) == INV
    e = lambda cc, *b, ws=4096, n=1 << 30: L.rs_cache_evict(C.byref(cc), *b, ws, n, None)
    assert e(c, 0, 0, 0) == INV and e(c, 64, 60, 5) == INV and e(c, 64, -1, 0) == INV
    for name in ("acc", "pos", "seen"):
        assert e(cache(**{name: None}), 64, 0, 0) == INV
    assert e(c, 64, 0, 0, n=100) == WSP and e(c, 64, 0, 0, ws=None) == WSP
    assert e(c, 256, 0, 0, ws=None) == _rs.RS_OK   # the capacity: nothing can be over it


def test_addresses_stay_in_bounds_whatever_the_device_arrays_hold(tmp_path):
    """cache.h compiled for the host, with tables, lengths and starts from plain to absurd."""
    if not shutil.which("g++"):
        pytest.skip("g++ not available")
    src = tmp_path / "walk.cpp"
    src.write_text(r'''
#include <cstdio>
#include <cstdlib>
#include <climits>
#include <initializer_list>
#include "cache.h"
using namespace rs;
static int bad(const char *what) { printf("%s\n", what); return 1; }
int main() {
  for (int blocks = 1; blocks <= 4096; ++blocks) {  // page numbers of every row block, for every page size
    CacheView c{};
    c.page = 64 * blocks; c.pmul = page_mul(c.page, 2);
    for (int j = 0; j < 4096; ++j) if (page_of(c, j * 64 + j % 64) != j / blocks) return bad("page_of");
  }
  const int odd[] = {0, 1, -1, 5, 6, 7, INT_MAX, INT_MIN, 64, 63, 255, 256, 257, 1 << 20};
  const int N = sizeof(odd) / sizeof(odd[0]);
  for (int page : {64, 128, 192, 100}) for (int with_table = 0; with_table < 2; ++with_table) {
    CacheView c{};
    int table[12], len[3], start[4];
    c.nseq = 3; c.hkv = 2; c.page = page;     c.max_pages = page == 100 ? 1 : 4; c.npages = 3 * c.max_pages; c.cap = page * c.max_pages; c.kblocks = (page + 63) / 64;
    c.pmul = page_mul(page, c.max_pages);
    c.sk_t = 256; c.sk_h = page * 256; c.sk_p = 2 * c.sk_h; c.sv_t = 512; c.sv_h = page * 512; c.sv_p = 2 * c.sv_h;
    c.table = with_table ? table : nullptr; c.len = len;
    for (int a = 0; a < N; ++a) for (int b = 0; b < N; ++b) {
      for (int i = 0; i < 12; ++i) table[i] = odd[(a + i * b) % N];
      for (int i = 0; i < 3; ++i) len[i] = odd[(b + i) % N];
      for (int i = 0; i < 4; ++i) start[i] = odd[(a * 3 + i * b) % N];
      for (int s = 0; s < 3; ++s) {
        const int n = cache_len(c, s);
        if (n < 0 || n > c.cap) return bad("length");
        for (int j = 0; j < n; ++j) {
          const int p = page_of(c, j), id = page_id(c, s, p);
          if (p < 0 || p >= c.max_pages) return bad("page");
          if (id < 0) continue;
          if (id >= c.npages) return bad("id");
          for (int g = 0; g < 2; ++g) {
            if (k_offset(c, id, p, j, g) < 0 || k_offset(c, id, p, j, g) + 256 > c.npages * c.sk_p) return bad("k");
            if (v_offset(c, id, p, j, g) < 0 || v_offset(c, id, p, j, g) + 512 > c.npages * c.sv_p) return bad("v");
            const int64_t m = mean_offset(c, id, p, j / 64, g, 128);
            if (m < 0 || m + 128 > (int64_t)c.npages * 2 * c.kblocks * 128) return bad("mean");
          }
        }
        for (int nrows : {0, 1, 5, 100}) for (int most : {1, 4, 256}) {
          const RowRange r = new_rows(start, s, nrows, most);
          if (r.first < 0 || r.count < 0 || r.count > most || r.first + r.count > nrows) return bad("rows");
        }
      }
    }
  }
  printf("ok\n");
  return 0;
}
''')
    exe = tmp_path / "walk"
    subprocess.run(["g++", "-std=c++17", "-fsanitize=undefined", "-fno-sanitize-recover", "-I",
                    os.path.join(ROOT, "paper_2608_29058_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0 and out.stdout.strip() == "ok", out.stdout + out.stderr


def test_struct_layouts_match_the_c_compiler(tmp_path):
    if not shutil.which("gcc"):
        pytest.skip("gcc not available")
    structs = {"rs_cache": _rs.RsCache, "rs_draft": _rs.RsDraft}
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "rs.h"', 'int main(void) {']
    for name, py in structs.items():
        lines.append(f'printf("{name} size %zu\\n", sizeof({name}));')
        lines += [f'printf("{name} {f[0]} %zu\\n", offsetof({name}, {f[0]}));' for f in py._fields_]
    src, exe = tmp_path / "l.c", tmp_path / "l"
    src.write_text("\n".join(lines + ["return 0; }"]))
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    for line in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split("\n"):
        if line:
            name, field, val = line.split()
            py = structs[name]
            assert (C.sizeof(py) if field == "size" else getattr(py, field).offset) == int(val), line


def test_bindings_refuse_tensors_that_do_not_fit():
    import torch
    z = lambda *s, dt=torch.bfloat16: torch.zeros(*s, dtype=dt)
    k, n = z(4, 2, 64, 64), z(2, dt=torch.int32)
    ok = _rs.KvCache(k, k, n)
    assert ok.cap == 128
    for bad in (lambda: _rs.KvCache(k, z(4, 2, 64, 128), n), lambda: _rs.KvCache(k, k.float(), n),
                lambda: _rs.KvCache(k.transpose(2, 3), k.transpose(2, 3), n), lambda: _rs.KvCache(k, k, z(3, dt=torch.int32)),
                lambda: _rs.KvCache(k, k, n.long()), lambda: _rs.KvCache(k, k, n, table=z(3, 2, dt=torch.int32)),
                lambda: _rs.KvCache(k, k, n, acc=z(2, 2, 100, dt=torch.float32)), lambda: _rs.Draft(z(2, 4, 64).transpose(1, 2)),
                lambda: _rs.Draft(z(2, 4, 64), mask=z(1, 1, dt=torch.int32)), lambda: _rs.Draft(z(2, 4, 64), start=n.long())):
        with pytest.raises(ValueError):
            bad()
    d = _rs.Draft(z(2, 4, 64))
    o, lse = z(2, 4, 64), z(4, 2, dt=torch.float32)
    for bad in (lambda: _rs.rs_draft_attn(ok, d, o.float(), lse, None), lambda: _rs.rs_draft_attn(ok, d, z(2, 4, 32), lse, None),
                lambda: _rs.rs_draft_attn(ok, d, o, lse.t(), None), lambda: _rs.rs_draft_attn(ok, _rs.Draft(o.float()), o, lse, None),
                lambda: _rs.rs_select_attn(ok, d, 3, 0, 0, o, lse, None, blocks=z(2, 2, 4, dt=torch.int32)),
                lambda: _rs.rs_attn_weights(ok, d, lse, None, z(2, 2, 64, dt=torch.float32)),
                lambda: _rs.rs_cache_append(ok, z(2, 2, 32), z(2, 2, 32)), lambda: _rs.rs_cache_commit(ok, n.long(), 1),
                lambda: _rs.rs_cache_commit(ok, n, 3, path=z(2, 2, dt=torch.int32))):
        with pytest.raises(ValueError):
            bad()


def test_no_new_rows_are_nothing_to_do():
    L = _rs.lib()
    c, d = cache(), draft(q=None, nrows=0)
    assert attend(c, d, o=None, ws=None) == _rs.RS_OK and attend(c, d, o=None, ws=None, nsel=4) == _rs.RS_OK
    assert L.rs_attn_weights(C.byref(c), C.byref(d), None, None, None, None, None) == _rs.RS_OK
    assert L.rs_cache_append(C.byref(c), None, None, 0, 0, 0, 0, 4096, 0, 1, None) == _rs.RS_OK


def test_batches_beyond_the_index_range_are_refused():
    c = cache(nseq=60000, npages=8)
    assert attend(c, draft(hq=64, max_rows=256)) == UNS
    assert attend(cache(nseq=60000, hkv=64), draft(hq=64, nrows=1 << 19)) == UNS


def test_tensors_in_host_memory_are_refused():
    import torch
    k, n = torch.zeros(2, 2, 64, 64, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    c, d = _rs.KvCache(k, k, n, kmean=torch.zeros(2, 2, 1, 64, dtype=torch.bfloat16)), _rs.Draft(k[:, :, 0].contiguous())
    o, acc = torch.zeros(2, 2, 64, dtype=torch.bfloat16), torch.zeros(2, 2, 64)
    for f in (lambda: _rs.rs_draft_attn(c, d, o, None, None), lambda: _rs.rs_select_attn(c, d, 1, 0, 0, o, None, None),
              lambda: _rs.rs_attn_weights(c, d, torch.zeros(2, 2), None, acc), lambda: _rs.rs_cache_append(c, o, o),
              lambda: _rs.rs_cache_commit(c, n, 1), lambda: _rs.rs_cache_evict(c, 1, 0, 0, None)):
        with pytest.raises(ValueError, match="GPU"):
            f()
