"""Timed and compared workloads of the paged-cache operators: attention of a chunk of new tokens over a cache
(`chunk_attn`, `chunk_attn_paged`, with the score modifiers), appending the chunk's rows to the pages
(`append_paged`) and keeping the pages themselves (`pages_fork`, `pages_reserve`, `pages_free`, `pages_compact`,
`pages_copy`).

`run` computes each operator in its plain form (elementary torch operations in 32 bits) unless `own` is true, in which
case it makes the calls of `paper_2412_04652_b200.binding`.  Lengths, page assignments and row counts follow from a
case's sizes alone; values follow from the seed.
"""
import math

import numpy as np
import torch

own = False

NEG = -1.0e30


# ------------------------------------------------------------------------------------------------ cases

def _attn(name, batch, n_q, n_kv, d, lens, new, page_rows=128, softcap=0.0, bias=False, gaps=False, docs=0, prefix=0,
          spread=0, n=1.0, lse=True):
    """lens, new: (shortest, longest) over the batch; page_rows 0: a dense cache; spread: how far the heads' row counts
    differ (a pruned cache keeps another number of rows per head); gaps: positions of a pruned cache (not 0, 1, 2, ...);
    docs: documents packed one after the other; prefix: leading rows that every query sees."""
    return {"name": name, "op": "attn", "batch": batch, "n_q": n_q, "n_kv": n_kv, "d": d, "len_lo": lens[0], "len_hi": lens[1],
            "new_lo": new[0], "new_hi": new[1], "page_rows": page_rows, "softcap": softcap, "bias": bias, "gaps": gaps,
            "docs": docs, "prefix": prefix, "spread": spread, "n": n, "lse": lse}


def _append(name, batch, n_kv, d, lens, new, page_rows=128, spread=0):
    return {"name": name, "op": "append", "batch": batch, "n_kv": n_kv, "d": d, "len_lo": lens[0], "len_hi": lens[1],
            "new_lo": new[0], "new_hi": new[1], "page_rows": page_rows, "spread": spread}


def _fork(name, parents, ways, n_kv, d, lens, page_rows=128, whole=False):
    """Every parent gets `ways` children that share its pages; reserve room for one more token in all of them (or, whole:
    give every sequence pages of its own, as a prune in place needs), copy, drop the children again."""
    return {"name": name, "op": "fork", "parents": parents, "ways": ways, "n_kv": n_kv, "d": d, "len_lo": lens[0],
            "len_hi": lens[1], "page_rows": page_rows, "whole": whole}


def _trim(name, batch, n_kv, d, lens, keep_pct, page_rows=128):
    """After a prune in place: hand back the pages behind the kept rows, move the live pages together."""
    return {"name": name, "op": "trim", "batch": batch, "n_kv": n_kv, "d": d, "len_lo": lens[0], "len_hi": lens[1],
            "keep_pct": keep_pct, "page_rows": page_rows}


def listed():
    return [
        # the smallest call: one sequence in its first steps of decoding, few heads; latency is all there is
        _attn("one token, short cache", 1, 8, 4, 64, (100, 100), (1, 1)),
        # a serving batch of 32 sequences decoding over pruned caches (20 % of 2 K - 8 K positions, 32 heads, each
        # head with its own row count)
        _attn("one token, serving batch", 32, 32, 32, 128, (410, 1640), (1, 1), spread=30, lse=False),
        # long multi-image caches, 28 query heads on 4 KV heads, pruned (positions with gaps), distance bias
        _attn("one token, long GQA, bias", 4, 28, 4, 128, (8192, 32768), (1, 1), bias=True, gaps=True, spread=100),
        # the last chunk of a six-image prompt of 4 K positions, 32 heads: what a prefill in chunks runs
        _attn("512 tokens over 4 K", 1, 32, 32, 128, (4096, 4096), (512, 512)),
        # the largest: chunks of up to 1 K tokens over 8 K - 32 K positions, grouped heads, ragged
        _attn("1 K tokens, long GQA", 4, 28, 4, 128, (8192, 32768), (513, 1024)),
        # scores capped by a tanh and a bias by distance, odd sizes, dense cache, narrow heads
        _attn("capped, bias, dense", 3, 16, 8, 64, (701, 2311), (97, 333), page_rows=0, softcap=30.0, bias=True),
        # four documents packed into each row of the batch, the first 576 rows (an image) visible to all of them
        _attn("documents and prefix", 2, 32, 32, 128, (1500, 2048), (1500, 2048), docs=4, prefix=576, page_rows=256),
        # the rows of one decoded token of a serving batch go to its pages
        _append("append one token", 32, 32, 128, (410, 1640), (1, 1), spread=30),
        # the rows of prompt chunks
        _append("append 1 K tokens", 4, 32, 128, (3001, 9000), (513, 1024)),
        # two parallel answers for each of four short prompts: bookkeeping and a handful of pages
        _fork("two-way fork", 4, 2, 4, 64, (100, 1000)),
        # sixteen prompts, four answers each, every answer given pages of its own before it is pruned in place
        _fork("four-way fork, own pages", 16, 4, 8, 128, (2048, 8192), whole=True),
        # a serving batch after a prune to 20 %: four fifths of the pages go back, the rest moves together
        _trim("free and compact", 32, 8, 128, (2048, 8192), 20),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attn"] * 6 + ["append"] * 2 + ["fork"] * 2 + ["trim"] * 2)
    d = rng.choice([64, 128, 128])
    n_kv = rng.choice([1, 2, 4, 8, 16, 32])
    batch = _log(rng, 1, 32)
    page_rows = rng.choice([128, 128, 256, 512])
    hi = _log(rng, 64, 32768)
    while batch * n_kv * hi * d > 1 << 28:      # the cache of a case stays around a gigabyte
        batch, hi = max(1, batch * 2 // 3), max(64, hi * 3 // 4)
    lo = max(1, int(hi * rng.uniform(0.2, 1.0)))
    if op == "attn":
        group = rng.choice([1, 1, 2, 3, 4, 5, 6, 7, 8])
        top = 1 if rng.random() < 0.4 else _log(rng, 2, 1024)
        top = min(top, lo)
        while batch * n_kv * group * top * hi > 17 * 10 ** 8:
            top = max(1, top * 2 // 3)
        new = (max(1, int(top * rng.uniform(0.3, 1.0))), top)
        kind = rng.choice(["plain", "plain", "bias", "cap", "cap and bias", "docs", "prefix"])
        return _attn("", batch, n_kv * group, n_kv, d, (lo, hi), new, rng.choice([0, page_rows]),
                     softcap=rng.choice([15.0, 30.0, 50.0]) if "cap" in kind else 0.0, bias="bias" in kind,
                     gaps=rng.random() < 0.5, docs=rng.randint(2, 6) if kind == "docs" else 0,
                     prefix=rng.randint(1, hi) if kind == "prefix" else 0, spread=rng.choice([0, min(20, lo - new[1])]),
                     n=rng.choice([0.0, 1.0, 1.0]), lse=rng.random() < 0.7)
    if op == "append":
        top = min(lo, rng.choice([1, _log(rng, 2, 1024)]))
        return _append("", batch, n_kv, d, (lo, hi), (max(1, top // 2), top), page_rows, spread=rng.choice([0, min(20, lo - top)]))
    if op == "fork":
        ways = rng.randint(1, 6)
        whole = rng.random() < 0.4
        while batch * (1 + (ways if whole else 0)) * n_kv * hi * d > 1 << 28:
            batch, hi = max(1, batch * 2 // 3), max(64, hi * 3 // 4)
        return _fork("", batch, ways, n_kv, d, (min(lo, hi), hi), page_rows, whole)
    return _trim("", batch, n_kv, d, (lo, hi), rng.choice([5, 10, 20, 40]), page_rows)


# ------------------------------------------------------------------------------------------------ sizes

def _between(lo, hi, count, step=7):
    """`count` whole numbers spread over [lo, hi], the longest among them, not in order."""
    at = [(k * step + count - 1) % count for k in range(count)] if math.gcd(step, count) == 1 else list(range(count))[::-1]
    return np.array([hi if count == 1 else lo + (hi - lo) * a // (count - 1) for a in at], np.int64)


def _row_counts(c):
    """(rows per head [B, Hkv], new tokens [B], rows of the longest cache)."""
    lens = _between(c["len_lo"], c["len_hi"], c["batch"])
    new = np.minimum(_between(c["new_lo"], c["new_hi"], c["batch"], 5), lens)
    h = np.arange(c["n_kv"])
    rows = np.maximum(lens[:, None] - (h * 37 % (c["spread"] + 1))[None, :], new[:, None])
    return rows, new, int(lens.max())


def _scatter_pages(held, n_pages):
    """Which page each table entry names: a fixed shuffle of the pool."""
    B, mp = len(held), int(held.max())
    order = np.random.RandomState(7919 + n_pages).permutation(n_pages)
    table = np.full((B, mp), -1, np.int32)
    inside = np.arange(mp)[None, :] < held[:, None]
    table[inside] = order[:int(held.sum())]
    return table


def _page_sizes(c):
    """Page numbers of a fork or trim case."""
    R = c["page_rows"]
    if c["op"] == "fork":
        lens = _between(c["len_lo"], c["len_hi"], c["parents"])
        held = -(-lens // R)
        kids = c["parents"] * c["ways"]
        mp = int(max(held.max(), (lens.max() + 1 + R - 1) // R))
        extra = int((-(-(lens + 1) // R)).sum()) * (1 + c["ways"]) if c["whole"] else c["parents"] * (1 + c["ways"])
        return lens, held, kids, mp, int(held.sum()) + extra
    lens = _between(c["len_lo"], c["len_hi"], c["batch"])
    held = -(-lens // R)
    kept = np.maximum(lens * c["keep_pct"] // 100, 1)
    return lens, held, kept, int(held.max()), int(held.sum()) + 8


def _moved_pages(c):
    """How many pages a fork or trim case copies."""
    R = c["page_rows"]
    if c["op"] == "fork":
        lens, held, _, _, _ = _page_sizes(c)
        shared = held if c["whole"] else held - lens // R            # 0 where the next token opens a page of its own
        return int(shared.sum()) * c["ways"]
    _, held, kept, _, n_pages = _page_sizes(c)
    table = _scatter_pages(held, n_pages)
    live = -(-kept // R)
    pages = table[np.arange(table.shape[1])[None, :] < live[:, None]]
    return int((pages >= live.sum()).sum())


def _visible_pairs(c):
    """Sum over sequences, KV heads and new tokens of the rows that the token sees."""
    rows, new, _ = _row_counts(c)
    lens = _between(c["len_lo"], c["len_hi"], c["batch"])
    total = 0
    for b in range(c["batch"]):
        for L, times in zip(*np.unique(rows[b], return_counts=True)):
            r = L - new[b] + np.arange(new[b])
            lim = np.minimum(np.maximum(r, c["prefix"] - 1), L - 1)
            first = np.zeros_like(r)
            if c["docs"]:
                doc = r * c["docs"] // lens[b]
                first = -(-doc * lens[b] // c["docs"])
                lim = np.minimum(lim, -(-(doc + 1) * lens[b] // c["docs"]) - 1)
            total += int(np.maximum(lim - first + 1, 0).sum()) * int(times)
    return total


def work(case):
    c = case
    if c["op"] == "attn":
        rows, new, _ = _row_counts(c)
        G = c["n_q"] // c["n_kv"]
        tokens = int(new.sum()) * c["n_q"]
        meta = (4 * int(rows.sum()) if c["gaps"] and c["bias"] else 0) + (4 * c["batch"] * c["len_hi"] if c["docs"] else 0)
        return {"bytes": int(rows.sum()) * c["d"] * 4 + tokens * c["d"] * 4 + (4 * tokens if c["lse"] else 0) + meta,
                "flops": 4.0 * c["d"] * G * _visible_pairs(c)}
    if c["op"] == "append":
        _, new, _ = _row_counts(c)
        return {"bytes": int(new.sum()) * c["n_kv"] * c["d"] * 8 + 8 * c["batch"] * c["n_kv"], "flops": 0.0}
    lens, held, _, mp, n_pages = _page_sizes(c)
    seqs = len(lens) * (1 + c["ways"]) if c["op"] == "fork" else len(lens)
    tables = 4 * (2 * n_pages + 2 * seqs * mp + 2 * seqs + seqs * c["n_kv"])
    return {"bytes": _moved_pages(c) * c["page_rows"] * c["n_kv"] * c["d"] * 8 + tables, "flops": 0.0}


# ------------------------------------------------------------------------------------------------ inputs

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(shape, g, gain=1.0):
    return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * gain).to(torch.bfloat16)


def _cuda(a, dtype=torch.int32):
    return torch.as_tensor(np.ascontiguousarray(a), dtype=dtype).cuda()


def prepare(case, seed):
    c, g = dict(case), _gen(seed)
    s = {"c": c}
    if c["op"] in ("attn", "append"):
        rows, new, cap = _row_counts(c)
        B, H, d, R = c["batch"], c["n_kv"], c["d"], c["page_rows"]
        T = int(new.max())
        s.update(rows=_cuda(rows), new=_cuda(new), cap=cap, T=T)
        if R:
            mp = -(-cap // R)
            held = np.full(B, mp) if c["op"] == "append" else -(-rows.max(1) // R)
            n_pages = int(held.sum()) + 2
            s["table"] = _cuda(_scatter_pages(held, n_pages))
            shape = (n_pages, H, R, d)
        else:
            shape = (B, H, cap, d)
        s["k"], s["v"] = _normal(shape, g), _normal(shape, g)
        if c["op"] == "append":
            s["before"] = s["rows"] - s["new"][:, None]
            s["k_new"], s["v_new"] = _normal((B, T, H, d), g).transpose(1, 2), _normal((B, T, H, d), g).transpose(1, 2)
            s["after"] = torch.zeros_like(s["before"])
        else:
            s["q"] = _normal((B, T, c["n_q"], d), g, 1.5).transpose(1, 2)
            s["out"] = torch.zeros((B, T, c["n_q"], d), dtype=torch.bfloat16, device="cuda").transpose(1, 2)
            s["lse"] = torch.zeros((B, c["n_q"], T), device="cuda") if c["lse"] else None
            s["slopes"] = torch.exp2(-8.0 * torch.arange(1, c["n_q"] + 1, device="cuda") / c["n_q"]) if c["bias"] else None
            s["positions"] = s["documents"] = s["prefix"] = None
            if c["bias"] and c["gaps"]:
                s["positions"] = torch.randint(1, 6, (B, H, cap), generator=g, device="cuda").cumsum(2).to(torch.int32)
            if c["docs"]:
                lens = _between(c["len_lo"], c["len_hi"], B)
                s["documents"] = _cuda(np.arange(cap)[None, :] * c["docs"] // lens[:, None])
            if c["prefix"]:
                s["prefix"] = _cuda(np.full((B, 1), c["prefix"]))
        if own:
            from paper_2412_04652_b200 import binding as csp
            p = csp.Params(B, c.get("n_q", H), H, d, 1, 0, cap, cap, n=c.get("n", 1.0))
            s["p"] = p
            if c["op"] == "append":
                s["ws"] = csp.new_append_workspace(p)
            else:
                s["ws"] = csp.new_chunk_workspace(p, T)
                s["mods"] = None
                if c["softcap"] or c["bias"] or c["docs"] or c["prefix"]:
                    s["mods"] = csp.ScoreMods(softcap=c["softcap"], slopes=s["slopes"], positions=s["positions"],
                                              documents=s["documents"], prefix=s["prefix"])
        return s
    H, d, R = c["n_kv"], c["d"], c["page_rows"]
    lens, held, third, mp, n_pages = _page_sizes(c)
    table = np.full((len(lens), mp), -1, np.int32)
    scattered = _scatter_pages(held, n_pages)
    table[:, :scattered.shape[1]] = scattered
    refs = np.zeros(n_pages, np.int32)
    refs[table[table >= 0]] = 1
    if c["op"] == "fork":
        P, kids = c["parents"], third
        table = np.concatenate([table, np.full((kids, mp), -1, np.int32)])
        held = np.concatenate([held, np.zeros(kids, np.int64)])
        rows = np.concatenate([np.repeat(lens[:, None], H, 1), np.zeros((kids, H), np.int64)])
        s.update(src=_cuda(np.repeat(np.arange(P), c["ways"])), dst=_cuda(P + np.arange(kids)))
    else:
        rows = np.maximum(third[:, None] - (np.arange(H) * 5 % 7)[None, :], 1)
    s.update(table=_cuda(table), held=_cuda(held), refs=_cuda(refs), rows=_cuda(rows),
             k=_normal((n_pages, H, R, d), g), v=_normal((n_pages, H, R, d), g),
             moves=torch.full((n_pages, 2), -1, dtype=torch.int32, device="cuda"),
             n_moves=torch.zeros(1, dtype=torch.int32, device="cuda"))
    if c["op"] == "trim":
        s.update(table0=s["table"].clone(), held0=s["held"].clone(), refs0=s["refs"].clone())
    else:
        s["more"] = torch.ones(len(held), dtype=torch.int32, device="cuda")
    if own:
        from paper_2412_04652_b200 import binding as csp
        s["p"] = csp.Params(len(held), H, H, d, 1, 0, mp * R, mp * R)
        s["pages"] = csp.PageState(s["table"], s["held"], s["refs"], s["rows"], R)
        s["ws"] = csp.new_pages_workspace(s["pages"])
    return s


# ------------------------------------------------------------------------------------------------ one pass

def run(s):
    op = s["c"]["op"]
    if own:
        from paper_2412_04652_b200 import binding as csp
        return {"attn": _attn_own, "append": _append_own, "fork": _fork_own, "trim": _trim_own}[op](csp, s)
    return {"attn": _attn_plain, "append": _append_plain, "fork": _fork_plain, "trim": _trim_plain}[op](s)


def _attn_own(csp, s):
    if s["c"]["page_rows"]:
        csp.chunk_attn_paged(s["p"], s["q"], s["k"], s["v"], s["table"], s["rows"], s["out"], s["ws"], n_new=s["new"],
                             mods=s["mods"], lse=s["lse"])
    else:
        csp.chunk_attn(s["p"], s["q"], s["k"], s["v"], s["rows"], s["out"], s["ws"], n_new=s["new"], mods=s["mods"],
                       lse=s["lse"])
    return {"out": s["out"], "lse": s["lse"]} if s["lse"] is not None else {"out": s["out"]}


def _append_own(csp, s):
    csp.append_paged(s["p"], s["k_new"], s["v_new"], s["k"], s["v"], s["table"], s["before"], s["after"], s["ws"],
                     n_new=s["new"])
    return {"k": s["k"], "v": s["v"], "rows": s["after"]}


def _page_outputs(s):
    return {k: s[k] for k in ("table", "held", "refs", "rows", "n_moves", "k", "v")}


def _fork_own(csp, s):
    csp.pages_fork(s["pages"], s["src"], s["dst"], s["ws"])
    csp.pages_reserve(s["pages"], s["moves"], s["n_moves"], s["ws"], n_new=s["more"], whole=s["c"]["whole"])
    csp.pages_copy(s["p"], s["k"], s["v"], s["moves"], s["n_moves"], s["ws"])
    forked = s["table"].clone()
    s["rows"][s["c"]["parents"]:].zero_()
    csp.pages_free(s["pages"], s["ws"])
    return {"forked": forked, **_page_outputs(s)}


def _trim_own(csp, s):
    s["table"].copy_(s["table0"])
    s["held"].copy_(s["held0"])
    s["refs"].copy_(s["refs0"])
    csp.pages_free(s["pages"], s["ws"])
    csp.pages_compact(s["pages"], s["moves"], s["n_moves"], s["ws"])
    csp.pages_copy(s["p"], s["k"], s["v"], s["moves"], s["n_moves"], s["ws"])
    return _page_outputs(s)


# ---- plain forms

def _dense(pool, s):
    """[B, H, rows, d] in 32 bits of a dense cache, or of a pool read through the page table."""
    if not s["c"]["page_rows"]:
        return pool.float()
    rows = pool[s["table"].clamp(min=0).long()]                     # [B, pages, H, R, d]
    B, mp, H, R, d = rows.shape
    return rows.transpose(1, 2).reshape(B, H, mp * R, d)[:, :, :s["cap"]].float()


def _attn_plain(s):
    c = s["c"]
    B, H, d, T, cap = c["batch"], c["n_kv"], c["d"], s["T"], s["cap"]
    G = c["n_q"] // H
    k, v = _dense(s["k"], s), _dense(s["v"], s)
    t = torch.arange(k.shape[2], device="cuda")
    i = torch.arange(T, device="cuda")
    rows, new = s["rows"].long(), s["new"].long()
    there = (t < rows[:, :, None])[..., None]
    v = torch.where(there, v, 0.0)
    r = rows[:, :, None] - new[:, None, None] + i                   # row of each query's own token [B, H, T]
    at = r.clamp(0, t.numel() - 1)
    o = torch.matmul(s["q"].float().reshape(B, H, G * T, d), k.transpose(2, 3)).reshape(B, H, G, T, -1)
    o *= 1.0 / math.sqrt(d)
    if c["softcap"]:
        o = c["softcap"] * torch.tanh(o / c["softcap"])
    if c["bias"]:
        pos = t.expand(B, H, -1) if s["positions"] is None else s["positions"].long()
        far = (pos.gather(2, at)[..., None] - pos[:, :, None, :]).abs().float()
        o -= s["slopes"].reshape(1, H, G, 1, 1) * far[:, :, None]
    lim = r if s["prefix"] is None else torch.maximum(r, s["prefix"].long()[:, :, None] - 1)
    sees = (t <= lim[..., None]) & (t < rows[:, :, None, None])
    if c["docs"]:
        doc = s["documents"][:, None, :].expand(B, H, -1)
        sees &= doc.gather(2, at)[..., None] == doc[:, :, None, :]
    o.masked_fill_(~sees[:, :, None], NEG)
    m = o.amax(-1, keepdim=True)
    e = torch.exp(o - m) * sees[:, :, None]
    l = e.sum(-1, keepdim=True)
    out = torch.matmul(e.reshape(B, H, G * T, -1), v).reshape(B, H, G, T, d)
    share = c["n"] * torch.exp(-m) + l if c["n"] else l
    out = torch.where(l > 0, out / share, 0.0).reshape(B, H * G, T, d)
    live = (i < new[:, None])[:, None, :]
    s["out"].copy_(torch.where(live[..., None], out.to(torch.bfloat16), s["out"]))
    if s["lse"] is None:
        return {"out": s["out"]}
    s["lse"].copy_(torch.where(live, (m + torch.log(l)).reshape(B, H * G, T), s["lse"]))
    return {"out": s["out"], "lse": s["lse"]}


def _append_plain(s):
    c = s["c"]
    B, H, R, T, d = c["batch"], c["n_kv"], c["page_rows"], s["T"], c["d"]
    i = torch.arange(T, device="cuda")
    before, new = s["before"].long(), s["new"].long()
    there = (i < new[:, None])[:, None, :].expand(B, H, T)
    t = torch.where(there, before[:, :, None] + i, before[:, :, None] + new[:, None, None] - 1)     # spare slots repeat the last row
    page = s["table"].long()[torch.arange(B, device="cuda")[:, None, None], t // R]
    slot = (page * H + torch.arange(H, device="cuda")[None, :, None]) * R + t % R
    last = torch.where(there, i, new[:, None, None] - 1)[..., None].expand(B, H, T, d)
    s["k"].view(-1, d)[slot.reshape(-1)] = s["k_new"].gather(2, last).reshape(-1, d)
    s["v"].view(-1, d)[slot.reshape(-1)] = s["v_new"].gather(2, last).reshape(-1, d)
    s["after"].copy_(before + new[:, None])
    return {"k": s["k"], "v": s["v"], "rows": s["after"]}


def _copy_plain(s):
    n = torch.arange(s["moves"].shape[0], device="cuda") < s["n_moves"]
    spare = (s["refs"] == 0).int().argmax()                         # moves that are none copy a free page onto itself
    src = torch.where(n, s["moves"][:, 0], spare).long()
    dst = torch.where(n, s["moves"][:, 1], spare).long()
    for pool in (s["k"], s["v"]):
        pool[dst] = pool[src]


def _free_plain(s):
    R, table, held = s["c"]["page_rows"], s["table"], s["held"]
    i = torch.arange(table.shape[1], device="cuda")
    need = torch.minimum((s["rows"].amax(1) + R - 1) // R, held)
    gone = (i >= need[:, None]) & (i < held[:, None])
    s["refs"].scatter_add_(0, table.clamp(min=0).long().reshape(-1), -gone.int().reshape(-1))
    table.masked_fill_(gone, -1)
    held.copy_(need)


def _fork_plain(s):
    c, table, held, refs, rows = s["c"], s["table"], s["held"], s["refs"], s["rows"]
    R = c["page_rows"]
    i = torch.arange(table.shape[1], device="cuda")
    src, dst = s["src"].long(), s["dst"].long()
    # fork: the children name their parent's pages
    table[dst], held[dst], rows[dst] = table[src], held[src], rows[src]
    named = (i < held[src][:, None]).int()
    refs.scatter_add_(0, table[src].clamp(min=0).long().reshape(-1), named.reshape(-1))
    # reserve: a free page for every shared page that will be written and for every page that is missing
    first = torch.zeros_like(held) if c["whole"] else rows.amin(1) // R
    need = (rows.amax(1) + s["more"] + R - 1) // R
    page = table.clamp(min=0).long()
    inside = (i >= first[:, None]) & (i < held[:, None]) & (i < need[:, None])
    claim = (inside & (refs[page] > 1)).reshape(-1)
    flat, order = page.reshape(-1), torch.arange(table.numel(), device="cuda")
    claims = torch.zeros_like(refs).scatter_add_(0, flat, claim.int())
    last = torch.full(refs.shape, -1, device="cuda").scatter_reduce_(0, flat, torch.where(claim, order, -1), "amax")
    copy = claim & ~((claims[flat] == refs[flat]) & (last[flat] == order))
    fresh = ((i >= held[:, None]) & (i < need[:, None])).reshape(-1)
    want = copy | fresh
    free = torch.sort((refs != 0).int(), stable=True).indices
    to = free[(want.cumsum(0) - 1).clamp(min=0)]
    rank = torch.where(copy, copy.cumsum(0) - 1, s["moves"].shape[0])
    moves = torch.full((s["moves"].shape[0] + 1, 2), -1, dtype=torch.int32, device="cuda")
    moves[rank] = torch.stack([flat, to], 1).int()
    s["moves"].copy_(moves[:-1])
    s["n_moves"].copy_(copy.sum().reshape(1))
    refs.scatter_add_(0, flat, -copy.int())
    refs.scatter_add_(0, to, want.int())
    table.copy_(torch.where(want, to, table.reshape(-1)).reshape(table.shape))
    held.copy_(torch.maximum(held, need))
    _copy_plain(s)
    forked = table.clone()
    rows[c["parents"]:].zero_()
    _free_plain(s)
    return {"forked": forked, **_page_outputs(s)}


def _trim_plain(s):
    table, refs = s["table"], s["refs"]
    table.copy_(s["table0"])
    s["held"].copy_(s["held0"])
    refs.copy_(s["refs0"])
    _free_plain(s)
    # compact: the live pages behind the first n_live go to the holes in front, both in ascending order
    n = torch.arange(refs.shape[0], device="cuda")
    used = refs > 0
    n_live = used.sum()
    hole, mover = ~used & (n < n_live), used & (n >= n_live)
    holes = torch.sort((~hole).int(), stable=True).indices
    to = torch.where(mover, holes[(mover.cumsum(0) - 1).clamp(min=0)], n)
    rank = torch.where(mover, mover.cumsum(0) - 1, s["moves"].shape[0])
    moves = torch.full((s["moves"].shape[0] + 1, 2), -1, dtype=torch.int32, device="cuda")
    moves[rank] = torch.stack([n, to], 1).int()
    s["moves"].copy_(moves[:-1])
    s["n_moves"].copy_(mover.sum().reshape(1))
    table.copy_(torch.where(table >= 0, to[table.clamp(min=0).long()].int(), table))
    moved = torch.where(mover, 0, refs)
    refs.copy_(moved.scatter_add(0, to, torch.where(mover, refs, 0)))
    _copy_plain(s)
    return _page_outputs(s)


# ------------------------------------------------------------------------------------------------ 64 bits

def exact(case, seed):
    """The definition, in 64 bits, one KV head of one sequence at a time; None for the operators that only move rows."""
    if case["op"] != "attn":
        return None
    s = prepare(case, seed)
    c = s["c"]
    G, R, scale = c["n_q"] // c["n_kv"], c["page_rows"], 1.0 / math.sqrt(c["d"])
    rows, new = s["rows"].tolist(), s["new"].tolist()
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros((c["batch"], c["n_q"], s["T"]), dtype=torch.float64, device="cuda")
    for b in range(c["batch"]):
        for h in range(c["n_kv"]):
            L, n = rows[b][h], new[b]
            if R:
                pages = s["table"][b, :-(-L // R)].long()
                K, V = (x[pages, h].reshape(-1, c["d"])[:L].double() for x in (s["k"], s["v"]))
            else:
                K, V = s["k"][b, h, :L].double(), s["v"][b, h, :L].double()
            where = torch.arange(L, device="cuda") if s["positions"] is None else s["positions"][b, h, :L]
            limit = torch.arange(L - n, L, device="cuda")
            hidden = torch.arange(L, device="cuda")[None, :] > torch.clamp(limit, min=c["prefix"] - 1)[:, None]
            if c["docs"]:
                doc = s["documents"][b, :L]
                hidden |= doc[L - n:, None] != doc[None, :]
            for hq in range(h * G, h * G + G):
                x = s["q"][b, hq, :n].double() @ K.T * scale
                if c["softcap"]:
                    e2 = torch.exp(-2.0 * x.abs() / c["softcap"])
                    x = x.sign() * c["softcap"] * (1.0 - e2) / (1.0 + e2)
                if c["bias"]:
                    x -= s["slopes"][hq].double() * (where[L - n:, None] - where[None, :]).abs().double()
                x[hidden] = -math.inf
                z = torch.logsumexp(x, 1)
                total = torch.logaddexp(z, torch.full_like(z, math.log(c["n"]))) if c["n"] else z
                out[b, hq, :n] = torch.exp(x - total[:, None]) @ V
                lse[b, hq, :n] = z
    return {"out": out, "lse": lse} if c["lse"] else {"out": out}
