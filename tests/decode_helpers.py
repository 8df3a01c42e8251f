"""Caches and drafts for the decoding tests: seeded inputs in numpy and on the device."""
import numpy as np

from oracle import decode as OD
from paper_2608_29058_amd import _rs
from synth import gen as G


class Setup:
    """A batch with a cache: numpy values (rounded as the device holds them) and device tensors.
    lens: cached rows per sequence; rows: new rows per sequence; kind: None (chain), "tree", "random"
    (any mask, some rows empty); extra: rows of q behind the last sequence."""

    def __init__(self, seed, lens, rows, hq=8, hkv=2, d=64, dtype="bf16", page=64, layout="head", kind=None, extra=0,
                 table=True, scale=0.0, spread=1.0, room=0, max_rows=None):
        import torch
        r = np.random.default_rng(seed)
        self.hq, self.hkv, self.d, self.page, self.dtype = hq, hkv, d, page, dtype
        self.lens, self.counts = np.array(lens, np.int32), np.array(rows, np.int32)
        nseq = len(lens)
        need = [max(1, -(-(int(a) + int(c) + room) // page)) for a, c in zip(lens, rows)]
        max_pages = max(need)
        rnd = G.bf16_round if dtype == "bf16" else (lambda x: np.asarray(x, np.float32))
        npages = sum(need) + 2 if table else nseq * max_pages
        shape = (npages, hkv, page, d)
        self.k, self.v = (rnd(r.standard_normal(shape).astype(np.float32)) for _ in range(2))
        if table:
            ids = r.permutation(npages)[:sum(need)]
            self.table = np.full((nseq, max_pages), -1, np.int32)
            at = 0
            for b, m in enumerate(need):
                self.table[b, :m] = ids[at:at + m]
                at += m
        else:
            self.table = np.arange(npages, dtype=np.int32).reshape(nseq, max_pages)
        self.cap = max_pages * page
        self.max_rows = max_rows or max(1, int(max(rows)))
        self.start = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
        self.nrows = int(self.start[-1]) + extra
        self.q = rnd((spread * r.standard_normal((self.nrows, hq, d))).astype(np.float32))
        self.rows = OD.row_ranges(self.start, nseq, self.nrows, self.max_rows)
        self.scale = scale or 1 / np.sqrt(d)
        self.mask = None
        if kind:
            words = (self.max_rows + 31) // 32
            m = np.zeros((self.nrows, words * 32), bool)
            for f, t in self.rows:
                for i in range(t):
                    if kind == "random":
                        m[f + i, :t] = r.random(t) < 0.4 if i % 3 else False
                        continue
                    p = int(r.integers(-1, i)) if i else -1
                    if p >= 0:
                        m[f + i] = m[f + p]
                    m[f + i, i] = True
            self.mask = np.packbits(m, axis=1, bitorder="little").view(np.int32)
        td = torch.bfloat16 if dtype == "bf16" else torch.float32

        def put(x):
            t = torch.from_numpy(x).to(td)
            if layout == "token":
                return t.transpose(1, 2).contiguous().cuda().transpose(1, 2)
            return t.cuda()

        i32 = lambda x: None if x is None else torch.from_numpy(np.ascontiguousarray(x)).cuda()
        self.dk, self.dv = put(self.k), put(self.v)
        self.dq = torch.from_numpy(self.q).to(td).cuda()
        self.dlen, self.dtable = i32(self.lens), i32(self.table) if table else None
        self.dstart, self.dmask = i32(self.start), i32(self.mask)
        self.draft = _rs.Draft(self.dq, max_rows=self.max_rows, start=self.dstart, mask=self.dmask, scale=scale)

    def cache(self, **kw):
        return _rs.KvCache(self.dk, self.dv, self.dlen, table=self.dtable, **kw)

    def outputs(self):
        import torch
        return (torch.full((self.nrows, self.hq, self.d), -7.0, dtype=torch.bfloat16, device="cuda"),
                torch.full((self.hq, self.nrows), -7.0, device="cuda"))

    def means(self):
        """Block means as the cache holds them, as numpy and on the device."""
        import torch
        m = torch.from_numpy(OD.block_means(self.k.astype(np.float64))).to(torch.bfloat16)
        full = torch.zeros((self.k.shape[0], self.hkv, (self.page + 63) // 64, self.d), dtype=torch.bfloat16)
        full[:, :, :m.shape[2]] = m
        return full.double().numpy(), full.cuda()

    def oracle(self, blocks=None):
        return OD.draft(self.q.astype(np.float64), self.k, self.v, self.lens, self.table, self.page, self.rows, self.mask,
                        self.cap, self.scale, blocks=blocks)


def logit_error(dtype, d, span):
    """Bound of a logit's error: fp32 sums of d exact products (d steps of 2^-24 of sum |q k|), the scale's
    and the exponent's roundings; fp32 inputs as two bf16 parts each add 2^-16 (x = hi + lo leaves 2^-17 of
    each factor, lo.lo 2^-16 x 2^-2 of the product)."""
    return span * ((d + 8) * 2.0 ** -24 + (2.0 ** -15 if dtype == "f32" else 0))


def check_rows(s, ref, o, lse, rows=None):
    """O and lse of the batch's rows against the oracle.  O: half a bf16 step of the result (2^-8) and of every
    weight (2^-8 of sum p |v|), the weights' error 2 dl, V's two parts 2^-16; 1 % for second-order terms.
    lse: dl, and the fp32 sum of n terms in steps of 2^-24, exp2 and log2 to an ulp each."""
    got, gl = o.float().cpu().numpy().astype(np.float64), None if lse is None else lse.cpu().numpy().astype(np.float64)
    dl = logit_error(s.dtype, s.d, ref["span"])
    n = int(max(s.lens.max(), 0)) + s.max_rows
    for f, t in (s.rows if rows is None else rows):
        r = slice(f, f + t)
        want, ab = ref["o"][r], ref["abs"][r]
        assert np.array_equal(np.isnan(got[r]), np.isnan(want))
        tol = 1.01 * (2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2 * dl + 2.0 ** -15) * ab) + 1e-30
        bad = np.abs(got[r] - want) > tol
        assert not bad.any(), (np.argwhere(bad)[:4], got[r][bad][:4], want[bad][:4])
        if gl is not None:
            w = ref["lse"][:, r]
            assert np.array_equal(np.isneginf(gl[:, r]), np.isneginf(w))
            fin = np.isfinite(w)
            off = np.abs(gl[:, r][fin] - w[fin])
            lim = dl + 2.0 ** -24 * (n / 16 + 64) + 2.0 ** -21 * np.abs(w[fin])
            assert (off <= lim).all(), (off.max(), lim.min())
