"""Timed and compared workloads of the paged cache in 4 bits and of the rotated append: attention of new tokens over pages
held in 4 bits (`chunk_attn_q4_paged`), appending rows to such pages (`append_q4_paged`), reading rows back
(`load_q4_paged`), and appending to pages in bf16 or fp32 with the position rotation applied on the way
(`append_rope_paged`).

`run` computes each operator in its plain form (elementary torch operations in 32 bits) unless `own` is true, in which
case it makes the calls of `paper_2412_04652_b200.binding`.  Lengths, page assignments and row counts follow from a
case's sizes alone; values follow from the seed.

A row of d values in 4 bits: byte i holds the codes of values 2 i (low half) and 2 i + 1; beside the codes stand two bf16
numbers, scale and base; the value is base + scale * code.  base is the smallest value of the row, scale the row's
spread divided by 15, rounded to bf16 (0 where that is no normal number: a constant row), and a code the whole number
nearest to (value - base) / scale, the upper one where two are.
"""
import math

import numpy as np
import torch

own = False

NEG = -1.0e30
SMALLEST = 2.0 ** -126
UP = 1.0 + 2.0 ** -21       # a quotient halfway between two codes stays above the middle, whatever its factors were rounded to


# ------------------------------------------------------------------------------------------------ cases

def _attn(name, batch, n_q, n_kv, d, lens, new, page_rows=128, softcap=0.0, bias=False, docs=0, prefix=0, spread=0, n=1.0,
          lse=True):
    """lens, new: (shortest, longest) over the batch; spread: how far the heads' row counts differ (a pruned cache keeps
    another number of rows per head); bias: by distance, between the positions of a pruned cache; docs: documents packed one
    after the other; prefix: leading rows that every query sees."""
    return {"name": name, "op": "attn", "batch": batch, "n_q": n_q, "n_kv": n_kv, "d": d, "len_lo": lens[0], "len_hi": lens[1],
            "new_lo": new[0], "new_hi": new[1], "page_rows": page_rows, "softcap": softcap, "bias": bias, "docs": docs,
            "prefix": prefix, "spread": spread, "n": n, "lse": lse}


def _append(name, bits, batch, n_q, n_kv, d, lens, new, rope, page_rows=128, interleaved=False, per_head=False,
            positions=True):
    """bits: 4, or 16 / 32 for pages in bf16 / fp32; n_q: query heads rotated in the same call (0: none); rope: rotated leading
    dimensions (0: none); per_head: another number of new rows per head, as a prune leaves them; positions: given, or those
    of the rows."""
    return {"name": name, "op": "append", "bits": bits, "batch": batch, "n_q": n_q, "n_kv": n_kv, "d": d, "len_lo": lens[0],
            "len_hi": lens[1], "new_lo": new[0], "new_hi": new[1], "rope": rope, "page_rows": page_rows,
            "interleaved": interleaved, "per_head": per_head, "positions": positions}


def _load(name, batch, n_kv, d, lens, page_rows=128, f32=False, spread=0, first=0, values=True):
    """first: rows in front that are not read; values: V as well as K."""
    return {"name": name, "op": "load", "batch": batch, "n_kv": n_kv, "d": d, "len_lo": lens[0], "len_hi": lens[1],
            "page_rows": page_rows, "f32": f32, "spread": spread, "first": first, "values": values}


def listed():
    return [
        # the smallest call: one sequence in its first steps of decoding, few heads; latency is all there is
        _attn("q4 token, short cache", 1, 8, 4, 64, (100, 100), (1, 1)),
        # a serving batch of 32 sequences decoding over pruned caches (20 % of 2 K - 8 K positions, 32 heads, each head
        # with its own row count)
        _attn("q4 token, serving batch", 32, 32, 32, 128, (410, 1640), (1, 1), spread=30, lse=False),
        # long multi-image caches, 28 query heads on 4 KV heads, pruned (positions with gaps), distance bias
        _attn("q4 token, long GQA, bias", 4, 28, 4, 128, (8192, 32768), (1, 1), bias=True, spread=100),
        # five drafted tokens at once over the caches of eight sequences, scores capped by a tanh
        _attn("q4 five tokens, capped", 8, 32, 8, 128, (2049, 8191), (5, 5), softcap=30.0, page_rows=256),
        # the largest: chunks of up to 1 K tokens over 8 K - 32 K positions, grouped heads, ragged
        _attn("q4 1 K tokens, long GQA", 4, 28, 4, 128, (8192, 32768), (513, 1024)),
        # one decoded token of a serving batch: its keys and queries are rotated, its rows go to their pages
        _append("rotated token", 16, 32, 32, 32, 128, (410, 1640), (1, 1), 128),
        # the rows of prompt chunks, grouped heads
        _append("rotated 1 K tokens", 16, 4, 32, 8, 128, (3001, 9000), (513, 1024), 128),
        # fp32 pages, neighbouring pairs, half of the dimensions rotated, odd sizes
        _append("rotated fp32, interleaved", 32, 3, 0, 5, 64, (700, 2311), (97, 333), 32, interleaved=True, positions=False),
        # one decoded token of a serving batch goes to pages in 4 bits
        _append("q4 append, rotated token", 4, 32, 32, 8, 128, (410, 1640), (1, 1), 128),
        # what a prune left of six-image prompts (another number of rows per head) goes to pages in 4 bits
        _append("q4 append, pruned prompts", 4, 8, 0, 32, 128, (1640, 1640), (410, 1640), 0, per_head=True),
        # the keys and values of a serving batch read back for a prune
        _load("q4 read back", 16, 8, 128, (2048, 8192)),
        # the keys behind a shared prefix, as a check of a few heads reads them
        _load("q4 read back, fp32", 2, 3, 64, (257, 901), f32=True, spread=9, first=64, values=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attn"] * 5 + ["rope"] * 2 + ["q4"] * 2 + ["load"])
    d = rng.choice([64, 128, 128])
    n_kv = rng.choice([1, 2, 3, 4, 8, 16, 32])
    batch = _log(rng, 1, 32)
    page_rows = rng.choice([128, 128, 256, 512])
    hi = _log(rng, 64, 32768)
    while batch * n_kv * hi * d > 1 << 27:      # (a cache in 4 bits of a quarter of a gigabyte with K and V)
        batch, hi = max(1, batch * 2 // 3), max(64, hi * 3 // 4)
    lo = max(1, int(hi * rng.uniform(0.2, 1.0)))
    group = rng.choice([1, 1, 2, 3, 4, 5, 6, 7, 8])
    if op == "attn":
        top = 1 if rng.random() < 0.4 else _log(rng, 2, 1024)
        top = min(top, lo)
        while batch * n_kv * group * top * hi > 17 * 10 ** 8:
            top = max(1, top * 2 // 3)
        new = (max(1, int(top * rng.uniform(0.3, 1.0))), top)
        kind = rng.choice(["plain", "plain", "bias", "cap", "cap and bias", "docs", "prefix"])
        return _attn("", batch, n_kv * group, n_kv, d, (lo, hi), new, page_rows,
                     softcap=rng.choice([15.0, 30.0, 50.0]) if "cap" in kind else 0.0, bias="bias" in kind,
                     docs=rng.randint(2, 6) if kind == "docs" else 0, prefix=rng.randint(1, hi) if kind == "prefix" else 0,
                     spread=rng.choice([0, min(20, lo - new[1])]), n=rng.choice([0.0, 1.0, 1.0]), lse=rng.random() < 0.7)
    if op == "load":
        return _load("", batch, n_kv, d, (lo, hi), page_rows, f32=rng.random() < 0.4, spread=rng.choice([0, min(20, lo - 1)]),
                     first=rng.choice([0, 0, rng.randint(0, lo // 2)]), values=rng.random() < 0.6)
    top = min(lo, rng.choice([1, _log(rng, 2, 1024)]))
    new = (max(1, top // 2), top)
    rope = 16 * rng.randint(1, d // 16) if rng.random() < 0.5 else d
    if op == "q4":
        per_head = rng.random() < 0.3
        rope = 0 if per_head or rng.random() < 0.3 else rope
        return _append("", 4, batch, n_kv * group if rope and rng.random() < 0.6 else 0, n_kv, d, (lo, hi), new, rope, page_rows,
                       rng.random() < 0.3, per_head=per_head, positions=rng.random() < 0.7)
    return _append("", rng.choice([16, 16, 32]), batch, n_kv * group if rng.random() < 0.6 else 0, n_kv, d, (lo, hi), new, rope,
                   page_rows, rng.random() < 0.3, positions=rng.random() < 0.7)


# ------------------------------------------------------------------------------------------------ sizes

def _between(lo, hi, count, step=7):
    """`count` whole numbers spread over [lo, hi], the longest among them, not in order."""
    at = [(k * step + count - 1) % count for k in range(count)] if math.gcd(step, count) == 1 else list(range(count))[::-1]
    return np.array([hi if count == 1 else lo + (hi - lo) * a // (count - 1) for a in at], np.int64)


def _row_counts(c):
    """(rows per head [B, Hkv], new tokens [B] or [B, Hkv], rows of the longest cache)."""
    B, H = c["batch"], c["n_kv"]
    lens = _between(c["len_lo"], c["len_hi"], B)
    h = np.arange(H)
    if c["op"] == "load":
        return np.maximum(lens[:, None] - (h * 37 % (c["spread"] + 1))[None, :], 0), None, int(lens.max())
    new = np.minimum(_between(c["new_lo"], c["new_hi"], B, 5), lens)
    if c["op"] == "append":
        if c["per_head"]:
            new = np.maximum(new[:, None] - (h * 31 % 61)[None, :], 1)
            return np.maximum(lens[:, None], new), new, int(lens.max())
        return np.repeat(lens[:, None], H, 1), new, int(lens.max())
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
    rows, new, cap = _row_counts(c)
    d, H = c["d"], c["n_kv"]
    row4 = d // 2 + 4                           # bytes of a row in 4 bits
    if c["op"] == "attn":
        tokens = int(new.sum()) * c["n_q"]
        meta = (4 * int(rows.sum()) if c["bias"] else 0) + (4 * c["batch"] * c["len_hi"] if c["docs"] else 0)
        return {"bytes": int(rows.sum()) * 2 * row4 + tokens * d * 4 + (4 * tokens if c["lse"] else 0) + meta,
                "flops": 4.0 * d * (c["n_q"] // H) * _visible_pairs(c)}
    if c["op"] == "load":
        count = int(np.maximum(rows - c["first"], 0).sum()) * (2 if c["values"] else 1)
        return {"bytes": count * (row4 + d * (4 if c["f32"] else 2)), "flops": 2.0 * count * d}
    count = int(new.sum()) * (1 if c["per_head"] else H)              # rows of K
    size = 4 if c["bits"] == 32 else 2
    tokens = 0 if c["per_head"] else int(new.sum())
    moved = count * 2 * d * size + tokens * c["n_q"] * d * 2 * size + tokens * c["rope"] * 4 + 8 * c["batch"] * H
    # in 4 bits: the codes are written, and the values that they stand for are what comes back
    moved += count * 2 * (row4 + d * size) if c["bits"] == 4 else count * 2 * d * size
    return {"bytes": moved, "flops": 3.0 * c["rope"] * (count + tokens * c["n_q"]) + (8.0 * count * d if c["bits"] == 4 else 0.0)}


# ------------------------------------------------------------------------------------------------ inputs

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(shape, g, gain=1.0, dtype=torch.bfloat16):
    return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * gain).to(dtype)


def _channels(d, g):
    """Channels of keys and values differ in size, a few of them by much."""
    return torch.exp(0.4 * torch.randn(d, generator=g, device="cuda"))


def _cuda(a, dtype=torch.int32):
    return torch.as_tensor(np.ascontiguousarray(a), dtype=dtype).cuda()


def _pack(x):
    """bf16 rows -> (codes uint8 [..., d / 2], scale and base bf16 [..., 2])."""
    x = x.float()
    lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    scale = ((hi - lo) * (1.0 / 15.0)).to(torch.bfloat16)
    scale = torch.where(scale.float() < SMALLEST, 0.0, scale)
    s = scale.float()
    code = torch.round((x - lo) * torch.where(s > 0, 1.0 / s * UP, 0.0)).clamp(max=15.0).to(torch.uint8)
    return code[..., 0::2] | (code[..., 1::2] << 4), torch.cat([scale, lo.to(torch.bfloat16)], -1)


def _unpack(codes, scales):
    """The values in 32 bits."""
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).float()
    return scales[..., 1:].float() + scales[..., :1].float() * c


def _pages4(n_pages, H, R, d, g):
    """A pool in 4 bits with rows in all of its pages."""
    gain = _channels(d, g)
    codes = torch.empty((n_pages, H, R, d // 2), dtype=torch.uint8, device="cuda")
    scales = torch.empty((n_pages, H, R, 2), dtype=torch.bfloat16, device="cuda")
    step = max(1, (1 << 26) // (H * R * d))
    for p in range(0, n_pages, step):
        part = slice(p, min(p + step, n_pages))
        codes[part], scales[part] = _pack(_normal((part.stop - p, H, R, d), g, gain))
    return codes, scales


def prepare(case, seed):
    c, g = dict(case), _gen(seed)
    s = {"c": c}
    rows, new, cap = _row_counts(c)
    B, H, d, R = c["batch"], c["n_kv"], c["d"], c["page_rows"]
    mp = -(-cap // R)
    held = np.full(B, mp) if c["op"] == "append" else np.maximum(-(-rows.max(1) // R), 1)
    n_pages = int(held.sum()) + 2
    s.update(rows=_cuda(rows), cap=cap, table=_cuda(_scatter_pages(held, n_pages)))
    in4 = c["op"] != "append" or c["bits"] == 4
    f32 = c.get("f32", False) or c.get("bits") == 32
    dtype = torch.float32 if f32 else torch.bfloat16
    if in4:
        s["k"], s["k_scales"] = _pages4(n_pages, H, R, d, g)
        s["v"], s["v_scales"] = _pages4(n_pages, H, R, d, g)
    else:
        s["k"], s["v"] = _normal((n_pages, H, R, d), g, 1.0, dtype), _normal((n_pages, H, R, d), g, 1.0, dtype)
    if c["op"] == "load":
        s["from"] = torch.full((B, H), c["first"], dtype=torch.int32, device="cuda")
        s["span"] = max(cap - c["first"], 1)
        s["k_out"] = torch.zeros((B, H, s["span"], d), dtype=dtype, device="cuda")
        s["v_out"] = torch.zeros_like(s["k_out"]) if c["values"] else None
    else:
        T = int(new.max())
        s.update(new=_cuda(new), T=T)
    if c["op"] == "append":
        per = new if c["per_head"] else np.repeat(new[:, None], H, 1)
        s["before"] = _cuda(rows - per)
        s["after"] = torch.zeros_like(s["before"])
        gain = _channels(d, g)
        s["k_new"] = _normal((B, T, H, d), g, gain, dtype).transpose(1, 2)
        s["v_new"] = _normal((B, T, H, d), g, gain, dtype).transpose(1, 2)
        s["q"] = _normal((B, T, c["n_q"], d), g, 1.5, dtype).transpose(1, 2) if c["n_q"] else None
        s["q_out"] = torch.zeros((B, T, c["n_q"], d), dtype=dtype, device="cuda").transpose(1, 2) if c["n_q"] else None
        s["cos_sin"] = s["positions"] = None
        if c["rope"]:
            reach = cap
            if c["positions"]:                  # a pruned cache: the tokens stand farther on than the rows
                first = torch.randint(0, 4 * cap, (B, 1), generator=g, device="cuda")
                s["positions"] = (first + torch.arange(T, device="cuda")).to(torch.int32)
                reach = 4 * cap + T
            turn = 10000.0 ** (-2.0 * torch.arange(c["rope"] // 2, device="cuda", dtype=torch.float64) / c["rope"])
            angle = torch.arange(reach, device="cuda", dtype=torch.float64)[:, None] * turn
            s["cos_sin"] = torch.cat([angle.cos(), angle.sin()], 1).float()
        if in4:                                 # the new rows read back: how many at most, and where to
            s["k_out"] = torch.zeros((B, H, T, d), dtype=torch.bfloat16, device="cuda")
            s["v_out"] = torch.zeros_like(s["k_out"])
    if c["op"] == "attn":
        s["q"] = _normal((B, T, c["n_q"], d), g, 1.5).transpose(1, 2)
        s["out"] = torch.zeros((B, T, c["n_q"], d), dtype=torch.bfloat16, device="cuda").transpose(1, 2)
        s["lse"] = torch.zeros((B, c["n_q"], T), device="cuda") if c["lse"] else None
        s["slopes"] = torch.exp2(-8.0 * torch.arange(1, c["n_q"] + 1, device="cuda") / c["n_q"]) if c["bias"] else None
        s["positions"] = s["documents"] = s["prefix"] = None
        if c["bias"]:
            s["positions"] = torch.randint(1, 6, (B, H, cap), generator=g, device="cuda").cumsum(2).to(torch.int32)
        if c["docs"]:
            lens = _between(c["len_lo"], c["len_hi"], B)
            s["documents"] = _cuda(np.arange(cap)[None, :] * c["docs"] // lens[:, None])
        if c["prefix"]:
            s["prefix"] = _cuda(np.full((B, 1), c["prefix"]))
    if own:
        from paper_2412_04652_b200 import binding as csp
        n_q = c.get("n_q") or H
        s["p"] = csp.Params(B, n_q, H, d, 1, 0, cap, cap, dtype=csp.F32 if f32 else csp.BF16, n=c.get("n", 1.0))
        if in4:
            s["K"], s["V"] = csp.Q4Cache(s["k"], s["k_scales"]), csp.Q4Cache(s["v"], s["v_scales"])
        if c["op"] == "attn":
            s["ws"] = csp.new_chunk_q4_workspace(s["p"], T)
            s["mods"] = None
            if c["softcap"] or c["bias"] or c["docs"] or c["prefix"]:
                s["mods"] = csp.ScoreMods(softcap=c["softcap"], slopes=s["slopes"], positions=s["positions"],
                                          documents=s["documents"], prefix=s["prefix"])
        else:
            s["ws"] = csp.new_append_workspace(s["p"])
            if c["op"] == "append":
                s["rope"] = csp.Rope(s["cos_sin"], positions=s["positions"], interleaved=c["interleaved"]) if c["rope"] else None
    return s


# ------------------------------------------------------------------------------------------------ one pass

def run(s):
    op = s["c"]["op"]
    if own:
        from paper_2412_04652_b200 import binding as csp
        return {"attn": _attn_own, "append": _append_own, "load": _load_own}[op](csp, s)
    return {"attn": _attn_plain, "append": _append_plain, "load": _load_plain}[op](s)


def _attn_own(csp, s):
    csp.chunk_attn_q4_paged(s["p"], s["q"], s["K"], s["V"], s["table"], s["rows"], s["out"], s["ws"], n_new=s["new"],
                            mods=s["mods"], lse=s["lse"])
    return {"out": s["out"], "lse": s["lse"]} if s["lse"] is not None else {"out": s["out"]}


def _append_own(csp, s):
    if s["c"]["bits"] == 4:
        csp.append_q4_paged(s["p"], s["k_new"], s["v_new"], s["K"], s["V"], s["table"], s["before"], s["after"], s["ws"],
                            n_new=s["new"], rope=s["rope"], q=s["q"], q_out=s["q_out"])
        # what is held in 4 bits comes back as the values that it stands for
        csp.load_q4_paged(s["p"], s["K"], s["V"], s["table"], s["after"], s["k_out"], s["v_out"], s["ws"], first=s["before"])
    else:
        csp.append_rope_paged(s["p"], s["k_new"], s["v_new"], s["k"], s["v"], s["table"], s["before"], s["after"], s["ws"],
                              s["rope"], n_new=s["new"], q=s["q"], q_out=s["q_out"])
    return _append_outputs(s)


def _append_outputs(s):
    k, v = ("k_out", "v_out") if s["c"]["bits"] == 4 else ("k", "v")
    return {name: s[at] for name, at in (("k", k), ("v", v), ("rows", "after"), ("q", "q_out")) if s[at] is not None}


def _load_own(csp, s):
    csp.load_q4_paged(s["p"], s["K"], s["V"] if s["c"]["values"] else None, s["table"], s["rows"], s["k_out"], s["v_out"], s["ws"],
                      first=s["from"])
    return _load_outputs(s)


def _load_outputs(s):
    return {"k": s["k_out"], "v": s["v_out"]} if s["c"]["values"] else {"k": s["k_out"]}


# ---- plain forms

def _by_table(pool, s):
    """[B, H, rows, ...] of a pool read through the page table."""
    rows = pool[s["table"].clamp(min=0).long()].transpose(1, 2)    # [B, H, pages, R, ...]
    return rows.flatten(2, 3)[:, :, :s["cap"]]


def _attn_plain(s):
    c = s["c"]
    B, H, d, T = c["batch"], c["n_kv"], c["d"], s["T"]
    G = c["n_q"] // H
    k = _unpack(_by_table(s["k"], s), _by_table(s["k_scales"], s))
    v = _unpack(_by_table(s["v"], s), _by_table(s["v_scales"], s))
    t = torch.arange(k.shape[2], device="cuda")
    i = torch.arange(T, device="cuda")
    rows, new = s["rows"].long(), s["new"].long()
    v = torch.where((t < rows[:, :, None])[..., None], v, 0.0)
    r = rows[:, :, None] - new[:, None, None] + i                   # row of each query's own token [B, H, T]
    at = r.clamp(0, t.numel() - 1)
    o = torch.matmul(s["q"].float().reshape(B, H, G * T, d), k.transpose(2, 3)).reshape(B, H, G, T, -1)
    o *= 1.0 / math.sqrt(d)
    if c["softcap"]:
        o = c["softcap"] * torch.tanh(o / c["softcap"])
    if c["bias"]:
        pos = s["positions"].long()
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


def _rotate(x, s, heads_at):
    """x [B, h, T, d] in 32 bits, the leading dimensions rotated; heads_at: rows in front of the new ones [B, h]."""
    c = s["c"]
    if not c["rope"]:
        return x
    at = s["positions"].long()[:, None, :] if c["positions"] else heads_at.long()[:, :, None] + torch.arange(x.shape[2], device="cuda")
    cos, sin = s["cos_sin"][at.clamp(max=s["cos_sin"].shape[0] - 1)].chunk(2, -1)
    turned, rest = x[..., :c["rope"]], x[..., c["rope"]:]
    if c["interleaved"]:
        a, b = turned[..., 0::2], turned[..., 1::2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = turned.chunk(2, -1)
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, rest], -1)


def _append_plain(s):
    c = s["c"]
    B, H, R, T, d = c["batch"], c["n_kv"], c["page_rows"], s["T"], c["d"]
    i = torch.arange(T, device="cuda")
    before = s["before"].long()
    new = s["new"].long() if c["per_head"] else s["new"].long()[:, None].expand(B, H)
    live = i < new[:, :, None]                                     # [B, H, T]
    k = _rotate(s["k_new"].float(), s, s["before"]).to(s["k_new"].dtype)
    # spare slots repeat the last row
    last = torch.where(live, i, new[:, :, None] - 1)[..., None].expand(B, H, T, d)
    k, v = k.gather(2, last), s["v_new"].gather(2, last)
    t = before[:, :, None] + last[..., 0]
    page = s["table"].long()[torch.arange(B, device="cuda")[:, None, None], t // R]
    slot = ((page * H + torch.arange(H, device="cuda")[None, :, None]) * R + t % R).reshape(-1)
    s["after"].copy_(before + new)
    if c["bits"] == 4:
        for name, x in (("k", k), ("v", v)):
            codes, scales = _pack(x)
            s[name].view(-1, d // 2)[slot] = codes.reshape(-1, d // 2)
            s[name + "_scales"].view(-1, 2)[slot] = scales.reshape(-1, 2)
            back = _unpack(s[name].view(-1, d // 2)[slot], s[name + "_scales"].view(-1, 2)[slot]).to(torch.bfloat16)
            s[name + "_out"].copy_(torch.where(live[..., None], back.reshape(B, H, T, d), s[name + "_out"]))
    else:
        s["k"].view(-1, d)[slot] = k.reshape(-1, d)
        s["v"].view(-1, d)[slot] = v.reshape(-1, d)
    if s["q"] is not None:
        G = c["n_q"] // H
        q = _rotate(s["q"].float(), s, s["before"].repeat_interleave(G, 1)).to(s["q"].dtype)
        s["q_out"].copy_(torch.where(live.repeat_interleave(G, 1)[..., None], q, s["q_out"]))
    return _append_outputs(s)


def _load_plain(s):
    c = s["c"]
    i = torch.arange(s["span"], device="cuda")
    t = s["from"].long()[:, :, None] + i
    live = (t < s["rows"][:, :, None])[..., None]
    for name in ("k", "v") if c["values"] else ("k",):
        codes, scales = _by_table(s[name], s), _by_table(s[name + "_scales"], s)
        at = t.clamp(max=codes.shape[2] - 1)[..., None]
        back = _unpack(codes.gather(2, at.expand(*t.shape, codes.shape[3])), scales.gather(2, at.expand(*t.shape, 2)))
        s[name + "_out"].copy_(torch.where(live, back.to(s[name + "_out"].dtype), s[name + "_out"]))
    return _load_outputs(s)


# ------------------------------------------------------------------------------------------------ 64 bits

def _values64(s, name, b, h, first, last):
    """Rows [first, last) of one head as the values that the format gives them."""
    R = s["c"]["page_rows"]
    t = torch.arange(first, last, device="cuda")
    page, at = s["table"][b].long()[t // R], t % R
    codes, pair = s[name][page, h, at].long(), s[name + "_scales"][page, h, at].double()
    out = torch.empty((last - first, 2 * codes.shape[1]), dtype=torch.float64, device="cuda")
    out[:, 0::2] = pair[:, 1:] + pair[:, :1] * (codes % 16)
    out[:, 1::2] = pair[:, 1:] + pair[:, :1] * (codes // 16)
    return out


def exact(case, seed):
    """The definition, in 64 bits, one head of one sequence at a time."""
    s = prepare(case, seed)
    return {"attn": _attn_exact, "append": _append_exact, "load": _load_exact}[case["op"]](s)


def _attn_exact(s):
    c = s["c"]
    G, scale = c["n_q"] // c["n_kv"], 1.0 / math.sqrt(c["d"])
    rows, new = s["rows"].tolist(), s["new"].tolist()
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros((c["batch"], c["n_q"], s["T"]), dtype=torch.float64, device="cuda")
    for b in range(c["batch"]):
        for h in range(c["n_kv"]):
            L, n = rows[b][h], new[b]
            K, V = _values64(s, "k", b, h, 0, L), _values64(s, "v", b, h, 0, L)
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
                    where = s["positions"][b, h, :L]
                    x -= s["slopes"][hq].double() * (where[L - n:, None] - where[None, :]).abs().double()
                x[hidden] = -math.inf
                z = torch.logsumexp(x, 1)
                total = torch.logaddexp(z, torch.full_like(z, math.log(c["n"]))) if c["n"] else z
                out[b, hq, :n] = torch.exp(x - total[:, None]) @ V
                lse[b, hq, :n] = z
    return {"out": out, "lse": lse} if c["lse"] else {"out": out}


def _turned64(s, x, at):
    """Rows x [n, d] of tokens at positions `at`, each pair turned by the table's angle."""
    c = s["c"]
    y = x.double().clone()
    half = c["rope"] // 2
    table = s["cos_sin"][at].double()
    one, two = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if c["interleaved"] else (slice(0, half), slice(half, 2 * half))
    z = torch.complex(y[:, one].contiguous(), y[:, two].contiguous()) * torch.complex(table[:, :half], table[:, half:])
    y[:, one], y[:, two] = z.real, z.imag
    return y


def _held64(x):
    """bf16 rows -> what 4 bits, a bf16 scale and a bf16 base keep of them."""
    x = x.double()
    low = x.min(1, keepdim=True).values
    step = ((x.max(1, keepdim=True).values - low) / 15).to(torch.bfloat16).double()
    code = torch.where(step >= SMALLEST, (x - low) / step + 0.5, 0.0).floor().clamp(max=15)
    return low + step * code


def _append_exact(s):
    c = s["c"]
    B, H, R = c["batch"], c["n_kv"], c["page_rows"]
    before, new, table = s["before"].tolist(), s["new"].tolist(), s["table"].tolist()
    in4 = c["bits"] == 4
    got = {"k": (s["k_out"] if in4 else s["k"]).double(), "v": (s["v_out"] if in4 else s["v"]).double(), "rows": None}
    if s["q"] is not None:
        got["q"] = torch.zeros(s["q_out"].shape, dtype=torch.float64, device="cuda")
    if max(x.numel() for x in got.values() if x is not None) > 1 << 28:
        return None

    def at(b, first, n):
        return s["positions"][b, :n].long() if c["positions"] else torch.arange(first, first + n, device="cuda")

    for b in range(B):
        for h in range(H):
            n = new[b][h] if c["per_head"] else new[b]
            first = before[b][h]
            k, v = s["k_new"][b, h, :n], s["v_new"][b, h, :n]
            if c["rope"]:
                k = _turned64(s, k, at(b, first, n))
            if in4:
                got["k"][b, h, :n], got["v"][b, h, :n] = _held64(k.to(torch.bfloat16)), _held64(v)
            else:
                t = torch.arange(first, first + n, device="cuda")
                page = s["table"][b].long()[t // R]
                got["k"][page, h, t % R], got["v"][page, h, t % R] = k.double(), v.double()
        for hq in range(c["n_q"]):
            n = new[b]
            got["q"][b, hq, :n] = _turned64(s, s["q"][b, hq, :n], at(b, before[b][hq * H // c["n_q"]], n))
    return got


def _load_exact(s):
    c = s["c"]
    rows = s["rows"].tolist()
    got = {}
    for name in ("k", "v") if c["values"] else ("k",):
        out = torch.zeros(s["k_out"].shape, dtype=torch.float64, device="cuda")
        for b in range(c["batch"]):
            for h in range(c["n_kv"]):
                n = rows[b][h] - c["first"]
                if n > 0:
                    out[b, h, :n] = _values64(s, name, b, h, c["first"], rows[b][h])
        got[name] = out
    return got
