"""Encoder states in a cache and a decoder's rows, for the tests of cross attention."""
import numpy as np

from oracle import decode as OD
from paper_2608_29058_amd import _rs
from synth import gen as G


class Encoded:
    """lens: states per sequence; rows: queries per sequence; hide: share of the states that the key mask hides (None: no
    mask), all_hidden: sequences of which it hides every state."""

    def __init__(self, seed, lens, rows, hq=8, hkv=2, d=64, dtype="bf16", page=64, layout="head", hide=None, all_hidden=(), extra=0,
                 scale=0.0, spread=1.0, max_rows=None, start=True, max_pages=None):
        import torch
        r = np.random.default_rng(seed)
        self.hq, self.hkv, self.d, self.page, self.dtype = hq, hkv, d, page, dtype
        self.lens, self.counts = np.array(lens, np.int32), np.array(rows, np.int32)
        nseq = len(lens)
        need = [max(1, -(-int(n) // page)) for n in lens]
        mp = max_pages or max(need)
        rnd = G.bf16_round if dtype == "bf16" else (lambda x: np.asarray(x, np.float32))
        npages = sum(need) + 2
        self.k, self.v = (rnd(r.standard_normal((npages, hkv, page, d)).astype(np.float32)) for _ in range(2))
        ids, at = r.permutation(npages), 0
        self.table = np.full((nseq, mp), -1, np.int32)
        for b, m in enumerate(need):
            self.table[b, :m] = ids[at:at + m]
            at += m
        self.cap = mp * page
        self.max_rows = max_rows or max(1, int(max(rows)))
        self.start = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32) if start else None
        self.nrows = (int(self.start[-1]) if start else nseq * self.max_rows) + extra
        self.q = rnd((spread * r.standard_normal((self.nrows, hq, d))).astype(np.float32))
        self.rows = OD.row_ranges(self.start, nseq, self.nrows, self.max_rows)
        self.scale = scale or 1 / np.sqrt(d)
        self.kmask = None
        if hide is not None:
            see = r.random((nseq, (self.cap + 31) // 32 * 32)) >= hide
            for b in (b for b in all_hidden if b < nseq):
                see[b] = False
            self.kmask = np.packbits(see, axis=1, bitorder="little").view(np.int32)
        self.td = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.layout, self.arg = layout, scale
        self.upload()

    def put(self, x):
        import torch
        t = torch.from_numpy(x).to(self.td)
        return t.transpose(1, 2).contiguous().cuda().transpose(1, 2) if self.layout == "token" else t.cuda()

    def upload(self):
        import torch
        i32 = lambda x: None if x is None else torch.from_numpy(np.ascontiguousarray(x)).cuda()
        self.dk, self.dv, self.dq = self.put(self.k), self.put(self.v), torch.from_numpy(self.q).to(self.td).cuda()
        self.dlen, self.dtable, self.dstart, self.dmask = i32(self.lens), i32(self.table), i32(self.start), i32(self.kmask)
        self.cross = _rs.Cross(self.dq, max_rows=self.max_rows, start=self.dstart, kmask=self.dmask, scale=self.arg)

    def cache(self):
        return _rs.KvCache(self.dk, self.dv, self.dlen, table=self.dtable)

    def outputs(self):
        import torch
        return (torch.full((self.nrows, self.hq, self.d), -7.0, dtype=torch.bfloat16, device="cuda"),
                torch.full((self.hq, self.nrows), -7.0, device="cuda"))

    def run(self, lse=True):
        c = self.cache()
        o, l = self.outputs()
        ws = _rs.workspace(_rs.rs_cross_attn_workspace_size(c, self.cross))
        _rs.rs_cross_attn(c, self.cross, o, l if lse else None, ws)
        return o, l

    def oracle(self):
        return OD.cross(self.q.astype(np.float64), self.k, self.v, self.lens, self.table, self.page, self.rows, self.kmask, self.cap,
                        self.scale)
