"""The operators of decoding over a key/value cache, as cases that can be timed and compared.

A case is a dict of plain values:

  op          "draft": attention of drafted tokens (one row: a plain decode step) over the cache;
              "select": the same over the blocks that each query's scores select;
              "weights": attention weight accumulated per cached row;
              "evict": rows of least accumulated weight leave the cache;
              "update": new rows written and the accepted ones kept;
  nseq, lo, hi   sequences and the range of their lengths (spread evenly, the first is lo, the second hi);
  t, ragged   new rows per sequence: t, or 1 .. t;
  tree        a mask names the drafted rows that a row sees (else those up to itself);
  hq, hkv, d, dtype   heads, head dimension, "bf16" or "f32";
  page, layout        rows per page; pages are [heads, rows, d] ("head") or [rows, heads, d] ("token");
  nsel, nsink, nlocal blocks of 64 that a query reads, how many of them always from the front and the end;
  budget, nsink, nrecent   rows that stay, how many of them always the oldest and the newest.

Inputs are drawn on the GPU from the seed alone; lengths and row counts from the case alone.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False
DEV = "cuda"


def _case(name, op, nseq, lo, hi, t=1, ragged=False, tree=False, hq=32, hkv=8, d=128, dtype="bf16", page=64,
          layout="head", nsel=0, nsink=0, nlocal=0, budget=0, nrecent=0):
    c = dict(op=op, nseq=nseq, lo=lo, hi=hi, t=t, ragged=ragged, tree=tree, hq=hq, hkv=hkv, d=d, dtype=dtype,
             page=page, layout=layout, nsel=nsel, nsink=nsink, nlocal=nlocal, budget=budget, nrecent=nrecent)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token of one short conversation: latency
        _case("draft_1_1k", "draft", 1, 1001, 1001),
        # a serving batch of plain decode steps, lengths from nothing to 16K
        _case("draft_64_ragged", "draft", 64, 0, 16384, page=128),
        # a tree of 61 drafted tokens at the end of a 128K prompt
        _case("draft_tree_128k", "draft", 1, 131000, 131000, t=61, tree=True, page=256),
        # fp32, d = 64, an odd group, ragged drafts on token-major pages
        _case("draft_f32_tree", "draft", 6, 1, 5003, t=13, ragged=True, tree=True, hq=28, hkv=4, d=64, dtype="f32",
              layout="token"),
        # one token at the end of a 128K prompt, 50 blocks of 64
        _case("select_1_128k", "select", 1, 131001, 131001, nsel=50, nsink=1, nlocal=4, page=256),
        # a batch of chains of up to four tokens over 8K to 64K, 100 blocks of 64 each
        _case("select_32_64k", "select", 32, 8000, 65536, t=4, ragged=True, nsel=100, nsink=2, nlocal=8, page=128),
        # weights of one decode step of a small batch
        _case("weights_4_4k", "weights", 4, 3000, 4099),
        # weights of the last drafted rows of long contexts
        _case("weights_16_32k", "weights", 16, 16000, 32768, t=8, ragged=True, tree=True, page=128),
        # a batch held at 2K rows that has outgrown them by one block
        _case("evict_32_2k", "evict", 32, 2048, 2112, budget=2048, nsink=4, nrecent=256),
        # two 128K prompts cut to 16K rows after the prefill
        _case("evict_2_128k", "evict", 2, 131072, 131072, budget=16384, nsink=128, nrecent=1024, page=256),
        # drafted rows of a batch written, the accepted path kept
        _case("update_64_tree", "update", 64, 100, 9000, t=16, ragged=True, tree=True),
        # chunks of 8K rows of four prefills enter the cache
        _case("update_4_chunk", "update", 4, 0, 57344, t=8192, page=256),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    """One more case of the ranges above."""
    op = rng.choice(["draft", "draft", "draft", "select", "select", "weights", "evict", "update"])
    hq, hkv = rng.choice([(32, 8), (32, 8), (16, 16), (8, 2), (28, 4), (40, 8), (64, 8)])
    d = rng.choice([128, 128, 128, 64])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    page = rng.choice([64, 128, 256, 1024])
    nseq = _log_int(rng, 1, 64)
    cap = int(min(131072, 500000 * 8 / hkv / nseq / (2 if dtype == "f32" else 1)))
    more = {}
    if op == "draft":
        t = rng.choice([1, 1, 1, 2, 5, 16, 33, 64])
        hi = _log_int(rng, 200, max(400, min(cap, int(131072 * 64 * 32 / (nseq * t * hq)))))
        lo = rng.choice([0, 1, hi // 2, hi])
        more = dict(t=t, ragged=rng.random() < 0.5, tree=rng.random() < 0.5)
    elif op == "select":
        hi = _log_int(rng, 1000, max(2000, cap // 2))
        lo = rng.choice([50, hi // 2, hi])
        more = dict(t=rng.choice([1, 1, 2, 4]), ragged=rng.random() < 0.5, tree=rng.random() < 0.3,
                    nsel=rng.choice([8, 16, 50, 100]), nsink=rng.choice([0, 1, 2]), nlocal=rng.choice([0, 2, 4]))
        if nseq * more["t"] * more["nsel"] * hkv > 64000:  # as many rows as the largest batch reads
            more.update(t=1, nsel=max(8, min(more["nsel"], 64000 // (nseq * hkv))))
    elif op == "weights":
        t = rng.choice([1, 1, 4, 8])
        hi = _log_int(rng, 200, max(400, min(cap // 2, int(32768 * 16 * 8 * 32 / (nseq * t * hq)))))
        lo = rng.choice([0, 1, hi // 2, hi])
        more = dict(t=t, ragged=rng.random() < 0.5, tree=rng.random() < 0.5)
    elif op == "evict":
        hi = _log_int(rng, 300, max(400, min(cap, 131072 * 16 // (hkv * nseq))))
        lo = rng.choice([hi // 2, hi])
        budget = max(128, int(hi * rng.choice([0.1, 0.5, 0.97])))
        more = dict(budget=budget, nsink=rng.choice([0, 4]), nrecent=min(budget - 8, rng.choice([0, 64, 256])))
    else:
        t = rng.choice([1, 2, 7, 16, 64, 1000])
        hi = _log_int(rng, 200, max(400, cap // 2))
        lo = rng.choice([0, 1, hi // 2])
        more = dict(t=t, ragged=t <= 64 and rng.random() < 0.5, tree=t <= 64 and rng.random() < 0.7)
    return _case(None, op, nseq, lo, hi, hq=hq, hkv=hkv, d=d, dtype=dtype, page=page,
                 layout=rng.choice(["head", "head", "token"]), **more)


# ---- sizes that follow from a case ---------------------------------------------------------

def _lens(case):
    n, lo, hi = case["nseq"], case["lo"], case["hi"]
    x = lo + np.round((hi - lo) * np.mod(np.arange(n) * 0.6180339887498949, 1.0)).astype(np.int64)
    if n > 1:
        x[1] = hi
    return x


def _rows(case):
    n, t = case["nseq"], case["t"]
    return 1 + (np.arange(n) * 7 + t - 1) % t if case["ragged"] else np.full(n, t, np.int64)


def _accept(case):
    r = _rows(case)
    return (r + 1) // 2 if case["tree"] else r


def _kept(case):
    return np.minimum(_lens(case), case["budget"])


def _full_blocks(case):
    return _lens(case) // 64


def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    hq, hkv, d, op = case["hq"], case["hkv"], case["d"], case["op"]
    L, T = _lens(case).astype(float), _rows(case).astype(float)
    row = 2.0 * e * d * hkv
    if op == "draft":
        return dict(bytes=float((row * (L + T)).sum() + (T * hq * (d * (e + 2) + 4)).sum()),
                    flops=float((4.0 * d * hq * T * (L + T)).sum()))
    if op == "select":
        F = _full_blocks(case).astype(float)
        # rows that the queries of a sequence read: each its own blocks, at most the whole cache
        keys = np.minimum(np.minimum(F, case["nsel"]) * 64 * T, L) + (L - 64 * F) + T
        return dict(bytes=float((row * keys + 2.0 * d * hkv * F + T * hq * (d * (e + 2) + 4) +
                                 T * hkv * case["nsel"] * 4).sum()),
                    flops=float((4.0 * d * hq * T * (np.minimum(F, case["nsel"]) * 64 + L - 64 * F + T) +
                                 2.0 * d * hq * T * F).sum()))
    if op == "weights":
        return dict(bytes=float(((row / 2 + 8.0 * hkv) * (L + T) + T * hq * (d * e + 4)).sum()),
                    flops=float((2.0 * d * hq * T * (L + T)).sum()))
    if op == "evict":
        gone = np.maximum(L - case["budget"], 0)
        moved = gone * case["budget"] / np.maximum(L, 1)  # places before the budget that lose their row
        # the bookkeeping is put back before each pass: read and written once more
        return dict(bytes=float((8.0 * hkv * (2 * L + L * (gone > 0)) + moved * 2 * row).sum()), flops=float((L * hkv).sum()))
    n = _accept(case).astype(float)
    blocks = np.floor((L + n) / 64) - np.floor(L / 64)
    return dict(bytes=float((2 * row * T + (2 * row * n if case["tree"] else 0 * n) + 8.0 * hkv * n +
                             blocks * (2.0 * d * hkv)).sum()), flops=float((row / e * n).sum()))


# ---- inputs --------------------------------------------------------------------------------

def _means(k):
    """Means of 64 rows of [npages, hkv, page, d], in bf16."""
    out = torch.empty((k.shape[0], k.shape[1], k.shape[2] // 64, k.shape[3]), dtype=torch.bfloat16, device=DEV)
    for i in range(0, k.shape[0], 256):
        x = k[i:i + 256]
        out[i:i + 256] = (x.reshape(x.shape[0], x.shape[1], -1, 64, x.shape[3]).double().sum(3) / 64).to(torch.bfloat16)
    return out


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed * 7919 + 11)
    rs = np.random.RandomState((seed * 104729 + 17) % (1 << 31))
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    nseq, hq, hkv, d, page, op = (case[x] for x in ("nseq", "hq", "hkv", "d", "page", "op"))
    lens, rows = _lens(case), _rows(case)
    used = np.maximum(1, -(-(lens + (rows if op != "evict" else 0)) // page))
    max_pages, npages = int(used.max()), int(used.sum())

    def randn(*s, dtype=dt):
        return torch.randn(*s, generator=g, device=DEV, dtype=dtype)

    # a direction per key/value head that some blocks of 64 rows and all queries share
    u = randn(hkv, d, dtype=torch.float32)

    def pool():
        x = randn(npages, page, hkv, d) if case["layout"] == "token" else randn(npages, hkv, page, d)
        return x.transpose(1, 2) if case["layout"] == "token" else x

    k, v = pool(), pool()
    blocks = torch.rand(npages, hkv, page // 64, generator=g, device=DEV) < 0.04
    near = (0.8 * blocks.repeat_interleave(64, 2)).to(dt)
    k.addcmul_(near[..., None], u.to(dt)[None, :, None])
    table = np.full((nseq, max_pages), -1, np.int32)
    ids, at = rs.permutation(npages).astype(np.int32), 0
    for b in range(nseq):
        table[b, :used[b]] = ids[at:at + used[b]]
        at += used[b]
    s = dict(case=case, k=k, v=v, table=torch.from_numpy(table).to(DEV),
             start=torch.from_numpy(np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)).to(DEV))
    nrows, t = int(rows.sum()), int(rows.max())
    cap = max_pages * page
    s["nrows"], s["t"], s["cap"] = nrows, t, cap
    i32 = torch.int32
    lens_d = torch.from_numpy(lens.astype(np.int32)).to(DEV)
    s["q"] = (randn(nrows, hq, d, dtype=torch.float32) +
              0.6 * u.repeat_interleave(hq // hkv, 0)).to(dt) if op in ("draft", "select", "weights") else None
    s["mask"] = None
    if case["tree"]:  # each drafted row continues an earlier one or the cached text
        words = (t + 31) // 32
        m = np.zeros((nrows, words * 32), bool)
        path = np.zeros((nseq, t), np.int32)
        r0 = 0
        for b in range(nseq):
            for i in range(int(rows[b])):
                p = int(rs.randint(max(-1, i - 4), i)) if i else -1
                if p >= 0:
                    m[r0 + i] = m[r0 + p]
                m[r0 + i, i] = True
            r0 += int(rows[b])
            n = int(_accept(case)[b])
            path[b, :n] = np.sort(rs.choice(int(rows[b]), n, replace=False))
        s["mask"] = torch.from_numpy(np.packbits(m, axis=1, bitorder="little").view(np.int32)).to(DEV)
        s["path"] = torch.from_numpy(path).to(DEV)
    if op == "select":
        s["kmean"] = _means(k)
    if op == "weights":
        s["len"] = lens_d
        s["lse"] = _plain_attention(s)[1]
        s["row_w"] = torch.from_numpy((rs.rand(nrows) < 0.6).astype(np.float32)).to(DEV)
        s["acc_in"] = torch.rand(nseq, hkv, cap, generator=g, device=DEV)
        s["acc"] = s["acc_in"].clone()
    if op in ("evict", "update"):
        # bookkeeping of a pass in one block, so that one copy puts it back: len, seen, acc, pos
        n = nseq * hkv * cap
        keep = torch.empty(2 * nseq + 2 * n, dtype=i32, device=DEV)
        keep[:nseq] = lens_d
        seen = lens.astype(np.int32) + (rs.randint(0, 1000, nseq).astype(np.int32) if op == "evict" else 0)
        keep[nseq:2 * nseq] = torch.from_numpy(seen).to(DEV)
        acc = torch.rand(nseq, hkv, cap, generator=g, device=DEV).pow_(8)  # few rows carry most of the weight
        keep[2 * nseq:2 * nseq + n] = acc.reshape(-1).view(i32)
        # rows of an evicted cache are not in the order of their positions
        pos = torch.arange(cap, device=DEV, dtype=i32).expand(nseq, hkv, cap)
        old = torch.from_numpy(seen).to(DEV)[:, None, None] - lens_d[:, None, None]
        turn = (pos + torch.from_numpy(rs.randint(0, 1 << 20, (nseq, hkv, 1)).astype(np.int32)).to(DEV)) % \
            lens_d.clamp(min=1)[:, None, None] if op == "evict" else pos
        keep[2 * nseq + n:] = (turn + old).reshape(-1)
        work_ = keep.clone()
        s["keep"], s["work"] = keep, work_
        s["len"], s["seen"] = work_[:nseq], work_[nseq:2 * nseq]
        s["acc"] = work_[2 * nseq:2 * nseq + n].view(torch.float32).view(nseq, hkv, cap)
        s["pos"] = work_[2 * nseq + n:].view(nseq, hkv, cap)
        s["kmean"] = _means(k)
        s["head"] = 2 * nseq  # an update puts back the lengths alone
        if op == "update":
            s["naccept"] = torch.from_numpy(_accept(case).astype(np.int32)).to(DEV)
            s["k_new"], s["v_new"] = randn(nrows, hkv, d), randn(nrows, hkv, d)
    s.setdefault("len", lens_d)
    if op in ("draft", "select"):
        s["o"] = torch.empty(nrows, hq, d, dtype=torch.bfloat16, device=DEV)
        s["lse"] = torch.empty(hq, nrows, device=DEV)
        if op == "select":
            s["blocks"] = torch.empty(nrows, hkv, case["nsel"], dtype=i32, device=DEV)
    if own:  # the descriptors and the workspace that a serving loop keeps
        from paper_2608_29058_amd import _rs
        s["cache"] = _rs.KvCache(k, v, s["len"], table=s["table"], kmean=s.get("kmean"), acc=s.get("acc"),
                                 pos=s.get("pos"), seen=s.get("seen"))
        if s["q"] is not None:
            s["draft"] = _rs.Draft(s["q"], max_rows=t, start=s["start"], mask=s["mask"])
        size = {"draft": lambda: _rs.rs_draft_attn_workspace_size(s["cache"], s["draft"]),
                "select": lambda: _rs.rs_select_attn_workspace_size(s["cache"], s["draft"], case["nsel"]),
                "evict": lambda: _rs.rs_cache_evict_workspace_size(s["cache"], case["budget"])}.get(op)
        s["ws"] = _rs.workspace(size()) if size else None
    return s


# ---- the plain forms -----------------------------------------------------------------------

def _row_places(s):
    """Sequence of each new row and its place in it."""
    i = torch.arange(s["nrows"], device=DEV)
    b = torch.searchsorted(s["start"].long(), i, right=True) - 1
    return b, i - s["start"].long()[b]


def _whole(s, x):
    """Pages of x as [nseq, hkv, cap, d] in 32 bits (rows behind a sequence's end are any page's)."""
    y = x[s["table"].long().clamp(min=0)].float()  # [nseq, max_pages, hkv, page, d]
    return y.transpose(1, 2).reshape(y.shape[0], y.shape[2], -1, y.shape[4])


def _seen_draft(s, b, off):
    """[nrows, t]: drafted row j of a row's sequence is one it sees."""
    j = torch.arange(s["t"], device=DEV)
    if s["mask"] is None:
        bits = j <= off[:, None]
    else:
        w = s["mask"][:, :, None] >> torch.arange(32, device=DEV, dtype=torch.int32)
        bits = (w & 1).bool().reshape(s["nrows"], -1)[:, :s["t"]]
    return bits & (j < (s["start"][1:] - s["start"][:-1]).long()[b][:, None])


def _logits(s):
    """Logits of every new row over its sequence's rows, minus infinity where it does not see one:
    [nseq, hkv, t, G, cap], and the rows' places."""
    c = s["case"]
    b, off = _row_places(s)
    hq, hkv, d, t, nseq, cap = c["hq"], c["hkv"], c["d"], s["t"], c["nseq"], s["cap"]
    q = torch.zeros(nseq, t, hq, d, device=DEV)
    q[b, off] = s["q"].float()
    q = q.view(nseq, t, hkv, hq // hkv, d).transpose(1, 2).reshape(nseq, hkv, -1, d)
    l = torch.matmul(q, _whole(s, s["k"]).transpose(2, 3)).mul_(1 / math.sqrt(d)).view(nseq, hkv, t, -1, cap)
    seen = torch.zeros(nseq, t, cap + t, dtype=torch.bool, device=DEV)
    n = s["len"].long()
    seen[b, off] = torch.arange(cap + t, device=DEV) < n[b][:, None]
    cols = n[b][:, None] + torch.arange(t, device=DEV)
    seen[b[:, None], off[:, None], cols] = _seen_draft(s, b, off)
    return l.masked_fill_(~seen[:, None, :, None, :cap], -math.inf), b, off


def _plain_softmax(l):
    m = l.amax(-1, keepdim=True)
    p = torch.exp(l - torch.where(m == -math.inf, torch.zeros_like(m), m))
    z = p.sum(-1, keepdim=True)
    return p, z, torch.where(z > 0, m + torch.log(z), m)[..., 0]


def _plain_attention(s):
    c = s["case"]
    l, b, off = _logits(s)
    p, z, lse = _plain_softmax(l)
    nseq, hkv, t, G, cap = l.shape
    o = torch.matmul(p.view(nseq, hkv, t * G, cap), _whole(s, s["v"])).view(nseq, hkv, t, G, -1)
    o = torch.where(z > 0, o / z, torch.zeros_like(o)).permute(0, 2, 1, 3, 4).reshape(nseq, t, c["hq"], c["d"])
    return o[b, off].to(torch.bfloat16), lse.permute(0, 2, 1, 3).reshape(nseq, t, c["hq"])[b, off].t().contiguous()


def _plain_select(s):
    c = s["case"]
    b, off = _row_places(s)
    hq, hkv, d, t, page, nsel = c["hq"], c["hkv"], c["d"], s["t"], c["page"], c["nsel"]
    G, nrows, n = hq // hkv, s["nrows"], s["len"].long()
    # scores in 64 bits: two blocks next to the border must not change places
    km = s["kmean"][s["table"].long().clamp(min=0)].double()  # [nseq, max_pages, hkv, page / 64, d]
    km = km.transpose(1, 2).reshape(km.shape[0], hkv, -1, d)
    q = torch.zeros(c["nseq"], t, hq, d, device=DEV, dtype=torch.float64)
    q[b, off] = s["q"].double()
    q = q.view(-1, t, hkv, G, d).transpose(1, 2).reshape(-1, hkv, t * G, d)
    sc = torch.matmul(q, km.transpose(2, 3)).view(-1, hkv, t, G, km.shape[2]).amax(3)  # [nseq, hkv, t, F]
    sc = sc.transpose(1, 2)[b, off]  # [nrows, hkv, F]
    F = (n // 64)[b][:, None, None]
    at = torch.arange(sc.shape[2], device=DEV)
    sc = sc.masked_fill((at < c["nsink"]) | (at >= F - c["nlocal"]), math.inf).masked_fill_(at >= F, -math.inf)
    top = torch.sort(sc, dim=2, descending=True, stable=True)[1][:, :, :nsel]
    wide = torch.nn.functional.pad(top, (0, nsel - top.shape[2]), value=0)
    some = torch.arange(nsel, device=DEV) < F
    none = 1 << 30
    blocks = torch.sort(torch.where(some, wide, torch.full_like(wide, none)), dim=2)[0]
    some = blocks < none
    # keys of the selected blocks, then those behind the last complete block
    first = torch.where(some, blocks, torch.zeros_like(blocks)) * 64
    j = (first[..., None] + torch.arange(64, device=DEV)).reshape(nrows, hkv, -1)
    tail = (F * 64 + torch.arange(64 + t, device=DEV)).expand(nrows, hkv, -1)
    see = _seen_draft(s, b, off)
    place = (tail - n[b][:, None, None])[:, 0]
    see = torch.gather(see, 1, place.clamp(0, t - 1)) & (place >= 0) & (place < t) | (place < 0)
    live = torch.cat([some.repeat_interleave(64, 2), see[:, None].expand(-1, hkv, -1)], 2)
    j = torch.cat([j, tail], 2).clamp(max=s["cap"] - 1)
    pg = s["table"].long().clamp(min=0)[b[:, None, None], j // page]
    head = torch.arange(hkv, device=DEV)[None, :, None]
    K, V = s["k"][pg, head, j % page].float(), s["v"][pg, head, j % page].float()
    l = torch.matmul(s["q"].float().view(nrows, hkv, G, d), K.transpose(2, 3)) * (1 / math.sqrt(d))
    p, z, lse = _plain_softmax(l.masked_fill_(~live[:, :, None], -math.inf))
    o = torch.where(z > 0, torch.matmul(p, V) / z, torch.zeros((), device=DEV))
    return (o.reshape(nrows, hq, d).to(torch.bfloat16), lse.reshape(nrows, hq).t().contiguous(),
            torch.where(some, blocks, torch.full_like(blocks, -1)).int())


def _plain_weights(s):
    l, b, off = _logits(s)
    nseq, hkv, t, G, cap = l.shape
    lse = torch.full((nseq, t, hkv * G), math.inf, device=DEV)
    lse[b, off] = torch.where(s["row_w"][:, None] > 0, s["lse"].t(), torch.full_like(s["lse"].t(), math.inf))
    w = torch.zeros(nseq, t, device=DEV)
    w[b, off] = s["row_w"]
    lse = lse.view(nseq, t, hkv, G).transpose(1, 2)[..., None]
    p = torch.exp(l - torch.where(lse == -math.inf, torch.full_like(lse, math.inf), lse)) * w[:, None, :, None, None]
    live = torch.arange(cap, device=DEV) < (s["len"] + s["start"][1:] - s["start"][:-1])[:, None, None]
    s["acc"].copy_(torch.where(live, s["acc_in"] + p.sum((2, 3)), s["acc"]))
    return s["acc"]


def _plain_evict(s):
    c, page, B = s["case"], s["case"]["page"], min(s["case"]["budget"], s["cap"])
    nseq, hkv, cap = s["acc"].shape
    n, at = s["len"][:, None, None], torch.arange(cap, device=DEV)
    live = at < n
    firm = (s["pos"] < c["nsink"]) | (s["pos"] >= s["seen"][:, None, None] - c["nrecent"])
    key = torch.where(firm, math.inf, s["acc"]).masked_fill_(~live, -math.inf)
    order = torch.sort(key, dim=2, descending=True, stable=True)[1]
    kept = torch.zeros(nseq, hkv, cap, dtype=torch.bool, device=DEV).scatter_(2, order[:, :, :B], True) & live
    over = n > B
    hole, mover = ~kept & (at < B) & over, kept & (at >= B) & over
    # the i-th row that stays behind the budget goes to the i-th place that is free before it
    place = torch.where(mover, mover.cumsum(2) - 1, torch.full_like(order, cap))
    src = torch.zeros(nseq, hkv, cap + 1, dtype=torch.int64, device=DEV).scatter_(2, place, at.expand_as(place))
    src = torch.where(hole, torch.gather(src, 2, (hole.cumsum(2) - 1).clamp(min=0)), at)[:, :, :B]
    s["acc"][:, :, :B] = torch.gather(s["acc"], 2, src)
    s["pos"][:, :, :B] = torch.gather(s["pos"], 2, src)
    seq, head = torch.arange(nseq, device=DEV)[:, None, None], torch.arange(hkv, device=DEV)[None, :, None]
    to = at[:B].expand_as(src)
    # places behind a short sequence's own pages name its first row, which then receives itself
    fine = to < n
    to, src = torch.where(fine, to, torch.zeros_like(to)), torch.where(fine, src, src[:, :, :1])
    pages = s["table"].long().clamp(min=0)
    s["k"][pages[seq, to // page], head, to % page] = s["k"][pages[seq, src // page], head, src % page]
    s["v"][pages[seq, to // page], head, to % page] = s["v"][pages[seq, src // page], head, src % page]
    m = B // 64
    rows = s["k"][pages[seq, to[:, :, :m * 64] // page], head, to[:, :, :m * 64] % page]
    mean = (rows.view(nseq, hkv, m, 64, -1).double().sum(3) / 64).to(torch.bfloat16)
    blk = torch.arange(m, device=DEV).expand(nseq, hkv, m)
    ok = (blk * 64 < n - 63) & over
    blk = torch.where(ok, blk, torch.zeros_like(blk))
    old = s["kmean"][pages[seq, blk * 64 // page], head, blk * 64 % page // 64]
    first = torch.where(ok[:, :, :1, None], mean[:, :, :1], old[:, :, :1])
    s["kmean"][pages[seq, blk * 64 // page], head, blk * 64 % page // 64] = torch.where(ok[..., None], mean, first)
    s["len"].clamp_(max=B)
    return s["k"], s["v"], s["kmean"], s["acc"], s["pos"], s["len"]


def _plain_update(s):
    c, page = s["case"], s["case"]["page"]
    nseq, hkv, cap = s["acc"].shape
    b, off = _row_places(s)
    pages, head = s["table"].long().clamp(min=0), torch.arange(hkv, device=DEV)[None, :]
    at = s["len"].long()[b] + off
    s["k"][pages[b, at // page][:, None], head, (at % page)[:, None]] = s["k_new"]
    s["v"][pages[b, at // page][:, None], head, (at % page)[:, None]] = s["v_new"]
    s["acc"][b, :, at] = 0.0
    # the i-th accepted row moves to the i-th place; the places of rows that go keep what they hold
    n, na = s["len"].long(), s["naccept"].long()
    ok = off < na[b]
    src = n[b] + (torch.where(ok, s["path"].long()[b, off], off) if c["tree"] else off)
    pt, ps = pages[b, at // page][:, None], pages[b, src // page][:, None]
    for x in (s["k"], s["v"]):
        x[pt, head, (at % page)[:, None]] = x[ps, head, (src % page)[:, None]]
    s["acc"][b, :, at] = s["acc"][b, :, src]
    s["pos"][b, :, at] = torch.where(ok[:, None], (s["seen"].long()[b] + off)[:, None].int(), s["pos"][b, :, at])
    # blocks that these rows complete; in the place of those that stay incomplete the first, as it then is
    seq = torch.arange(nseq, device=DEV)[:, None]
    m = s["t"] // 64 + 1
    blk = (n // 64)[:, None] + torch.arange(m, device=DEV)
    full = (blk + 1) * 64 <= (n + na)[:, None]
    blk = torch.where(full, blk, blk[:, :1].clamp(max=cap // 64 - 1))
    j = (blk[..., None] * 64 + torch.arange(64, device=DEV)).view(nseq, 1, -1)
    rows = s["k"][pages[seq[..., None], j // page], head[..., None], j % page]
    mean = (rows.view(nseq, hkv, m, 64, -1).double().sum(3) / 64).to(torch.bfloat16).transpose(1, 2)
    place = pages[seq, blk * 64 // page][..., None], head[None], (blk * 64 % page // 64)[..., None]
    first = torch.where(full[:, :1, None, None], mean[:, :1], s["kmean"][place][:, :1])
    s["kmean"][place] = torch.where(full[..., None, None], mean, first)
    s["len"].add_(s["naccept"])
    s["seen"].add_(s["naccept"])
    return s["k"], s["v"], s["kmean"], s["acc"], s["pos"], s["len"], s["seen"]


def run(s):
    c, op = s["case"], s["case"]["op"]
    if op == "evict":  # a pass starts from the same bookkeeping; rows that moved are still where they came from
        s["work"].copy_(s["keep"])
    elif op == "update":
        s["work"][:s["head"]].copy_(s["keep"][:s["head"]])
    if not own:
        if op == "draft":
            return _plain_attention(s)
        return {"select": _plain_select, "weights": _plain_weights, "evict": _plain_evict, "update": _plain_update}[op](s)
    from paper_2608_29058_amd import _rs
    if op == "draft":
        _rs.rs_draft_attn(s["cache"], s["draft"], s["o"], s["lse"], s["ws"])
        return s["o"], s["lse"]
    if op == "select":
        _rs.rs_select_attn(s["cache"], s["draft"], c["nsel"], c["nsink"], c["nlocal"], s["o"], s["lse"], s["ws"],
                           blocks=s["blocks"])
        return s["o"], s["lse"], s["blocks"]
    if op == "weights":
        _rs.rs_attn_weights(s["cache"], s["draft"], s["lse"], s["acc_in"], s["acc"], row_w=s["row_w"])
        return s["acc"]
    if op == "evict":
        _rs.rs_cache_evict(s["cache"], c["budget"], c["nsink"], c["nrecent"], s["ws"])
        return s["k"], s["v"], s["kmean"], s["acc"], s["pos"], s["len"]
    _rs.rs_cache_append(s["cache"], s["k_new"], s["v_new"], max_rows=s["t"], start=s["start"])
    _rs.rs_cache_commit(s["cache"], s["naccept"], s["t"], path=s["path"] if c["tree"] else None)
    return s["k"], s["v"], s["kmean"], s["acc"], s["pos"], s["len"], s["seen"]


# ---- from the definitions, one sequence at a time, in 64 bits ------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    op, page, hq, hkv, d = (case[x] for x in ("op", "page", "hq", "hkv", "d"))
    G = hq // hkv
    lens, rows = _lens(case), _rows(case)
    first = np.concatenate([[0], np.cumsum(rows)])
    table = s["table"].cpu().numpy()

    def places(b, n):
        """(page, row in it) of rows 0 .. n - 1 of a sequence."""
        j = np.arange(n)
        return torch.from_numpy(table[b, j // page].astype(np.int64)).to(DEV), torch.from_numpy(j % page).to(DEV)

    def keys(x, b, n, h):
        p, i = places(b, n)
        return x[p, h, i]

    def allowed(b, i, n):
        """Whether row i of sequence b sees each of the rows 0 .. n + rows[b] - 1."""
        a = np.ones(n + int(rows[b]), bool)
        if s["mask"] is None:
            a[n + i + 1:] = False
        else:
            bits = np.unpackbits(s["mask"][int(first[b]) + i].cpu().numpy().view(np.uint8), bitorder="little")
            a[n:] = bits[:int(rows[b])] > 0
        return torch.from_numpy(a).to(DEV)

    if op in ("draft", "weights"):
        o = torch.zeros(s["nrows"], hq, d, dtype=torch.float64, device=DEV)
        lse = torch.zeros(hq, s["nrows"], dtype=torch.float64, device=DEV)
        acc = s["acc_in"].double() if op == "weights" else None
        if op == "weights":
            keep = s["acc"].double()
        for b in range(case["nseq"]):
            n, t = int(lens[b]), int(rows[b])
            r = slice(int(first[b]), int(first[b]) + t)
            see = torch.stack([allowed(b, i, n) for i in range(t)])
            for h in range(hkv):
                k = keys(s["k"], b, n + t, h).double()
                q = s["q"][r, h * G:(h + 1) * G].double().reshape(t * G, d)
                l = (q @ k.t() / math.sqrt(d)).view(t, G, n + t).masked_fill(~see[:, None], -math.inf)
                if op == "draft":
                    lse[h * G:(h + 1) * G, r] = torch.logsumexp(l, 2).t()
                    o[r, h * G:(h + 1) * G] = (torch.softmax(l, 2).view(t * G, -1) @ keys(s["v"], b, n + t, h).double()).view(t, G, d)
                else:
                    p = torch.exp(l - s["lse"][h * G:(h + 1) * G, r].t().double()[..., None])
                    keep[b, h, :n + t] = acc[b, h, :n + t] + (p * s["row_w"][r].double()[:, None, None]).sum((0, 1))
        return (o, lse) if op == "draft" else keep
    if op == "select":
        o = torch.zeros(s["nrows"], hq, d, dtype=torch.float64, device=DEV)
        lse = torch.zeros(hq, s["nrows"], dtype=torch.float64, device=DEV)
        blocks = torch.full((s["nrows"], hkv, case["nsel"]), -1, dtype=torch.int32, device=DEV)
        for b in range(case["nseq"]):
            n, t = int(lens[b]), int(rows[b])
            F = n // 64
            c = np.arange(F)
            pg = torch.from_numpy(table[b, c * 64 // page].astype(np.int64)).to(DEV)
            for h in range(hkv):
                km = s["kmean"][pg, h, torch.from_numpy(c * 64 % page // 64).to(DEV)].double()
                kk, vv = keys(s["k"], b, n + t, h), keys(s["v"], b, n + t, h)
                for i in range(t):
                    q = s["q"][int(first[b]) + i, h * G:(h + 1) * G].double()
                    sc = (km @ q.t()).amax(1).cpu().numpy() if F else np.zeros(0)
                    must = (c < case["nsink"]) | (c >= F - case["nlocal"])
                    sel = np.sort(np.lexsort((c, -sc, ~must))[:case["nsel"]])
                    blocks[int(first[b]) + i, h, :len(sel)] = torch.from_numpy(sel.astype(np.int32)).to(DEV)
                    on = np.zeros(n + t, bool)
                    on[:F * 64] = np.isin(np.arange(F * 64) // 64, sel)
                    on[F * 64:] = True
                    j = (torch.from_numpy(on).to(DEV) & allowed(b, i, n)).nonzero()[:, 0]
                    l = q @ kk[j].double().t() / math.sqrt(d)
                    lse[h * G:(h + 1) * G, int(first[b]) + i] = torch.logsumexp(l, 1)
                    o[int(first[b]) + i, h * G:(h + 1) * G] = torch.softmax(l, 1) @ vv[j].double()
        return o, lse, blocks
    k, v, km = s["k"].clone(), s["v"].clone(), s["kmean"].clone()
    acc, pos, ln, seen = s["acc"].clone(), s["pos"].clone(), s["len"].clone(), s["seen"].clone()

    def mean(b, blk):
        p, i = int(table[b, blk * 64 // page]), blk * 64 % page
        km[p, :, i // 64] = k[p, :, i:i + 64].double().mean(1).to(torch.bfloat16)

    if op == "evict":
        B = case["budget"]
        for b in range(case["nseq"]):
            n = int(lens[b])
            if n <= B:
                continue
            pg, at = places(b, n)
            for h in range(hkv):
                a, p = acc[b, h, :n].cpu().numpy(), pos[b, h, :n].cpu().numpy()
                must = (p < case["nsink"]) | (p >= int(seen[b]) - case["nrecent"])
                stay = np.lexsort((np.arange(n), -a.astype(np.float64), ~must))[:B]
                free = torch.from_numpy(np.setdiff1d(np.arange(B), stay)).to(DEV)
                come = torch.from_numpy(np.sort(stay[stay >= B])).to(DEV)
                for x in (k, v):
                    x[pg[free], h, at[free]] = x[pg[come], h, at[come]]
                acc[b, h, free], pos[b, h, free] = acc[b, h, come], pos[b, h, come]
            ln[b] = B
            for blk in range(B // 64):
                mean(b, blk)
        return k, v, km, acc, pos, ln
    for b in range(case["nseq"]):
        n, t, na = int(lens[b]), int(rows[b]), int(s["naccept"][b])
        pg, at = places(b, n + t)
        r = slice(int(first[b]), int(first[b]) + t)
        new = s["k_new"][r].clone(), s["v_new"][r].clone()
        take = s["path"][b, :na].long() if case["tree"] else torch.arange(na, device=DEV)
        for x, y in zip((k, v), new):
            y[:na] = y[take]
            x[pg[n:], :, at[n:]] = y
        acc[b, :, n:n + t] = 0
        pos[b, :, n:n + na] = int(seen[b]) + torch.arange(na, device=DEV, dtype=torch.int32)
        ln[b] += na
        seen[b] += na
        for blk in range(n // 64, (n + na) // 64):
            mean(b, blk)
    return k, v, km, acc, pos, ln, seen
