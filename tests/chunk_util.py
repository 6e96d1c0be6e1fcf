"""Shared by the tests of chunk attention and of the page operators: the definition in 64 bits on the CPU, the tolerance
that follows from the arithmetic, and small paged caches."""
from __future__ import annotations

import math

import numpy as np
import torch


def paged_copy(k, v, rows, page_rows, seed, spare=2, fill=float("nan")):
    """Scatters dense [B, H, cap, d] caches into a shuffled pool; rows [B, H].  Everything behind a sequence's longest
    head is `fill`, unused table entries point outside the pool."""
    B, H, cap, d = k.shape
    per_seq = [-(-int(r.max()) // page_rows) for r in rows]
    max_pages = max(1, -(-cap // page_rows))
    n_pages = sum(per_seq) + spare
    order = np.random.RandomState(seed).permutation(n_pages)
    table = np.full((B, max_pages), 10 ** 6, np.int32)
    k_pool = torch.full((n_pages, H, page_rows, d), fill, dtype=k.dtype, device=k.device)
    v_pool = torch.full((n_pages, H, page_rows, d), fill, dtype=k.dtype, device=k.device)
    nxt = 0
    for b in range(B):
        for i in range(per_seq[b]):
            pg = int(order[nxt])
            nxt += 1
            table[b, i] = pg
            r0, r1 = i * page_rows, min((i + 1) * page_rows, int(rows[b].max()))
            k_pool[pg, :, :r1 - r0] = k[b, :, r0:r1]
            v_pool[pg, :, :r1 - r0] = v[b, :, r0:r1]
    return k_pool, v_pool, torch.from_numpy(table).to(k.device)


def reference(q, k, v, rows, new, n=1.0, scale=0.0, softcap=0.0, slopes=None, positions=None, documents=None, prefix=None):
    """The definition, one query at a time, in 64 bits.  q [B, Hq, T, d], k, v [B, Hkv, cap, d] (CPU); rows [B, Hkv], new [B].
    Returns out, lse, and what the tolerance needs per query: sum of weight * |v| (same shape as out) and the bound
    on the error of a logit."""
    B, Hq, T, d = q.shape
    Hkv, cap = k.shape[1], k.shape[2]
    G = Hq // Hkv
    scale = scale or 1.0 / math.sqrt(d)
    out = torch.zeros(B, Hq, T, d, dtype=torch.float64)
    lse = torch.full((B, Hq, T), -math.inf, dtype=torch.float64)
    mass = torch.zeros_like(out)
    logit_err = torch.zeros(B, Hq, T, dtype=torch.float64)
    for b in range(B):
        for h in range(Hkv):
            L, N = int(rows[b, h]), int(new[b])
            if L == 0 or N == 0:
                continue
            K, V = k[b, h, :L].double(), v[b, h, :L].double()
            t = torch.arange(L)
            pos = t if positions is None else (positions[b, h] if positions.dim() == 3 else positions[b])[:L].long()
            doc = None if documents is None else (documents[b, h] if documents.dim() == 3 else documents[b])[:L]
            pre = 0 if prefix is None else int(prefix[b, h % prefix.shape[1]])
            for i in range(N):
                r = L - N + i
                if r < 0:
                    continue
                see = t <= max(r, pre - 1)
                if doc is not None:
                    see &= doc == doc[r]
                for hq in range(h * G, (h + 1) * G):
                    qv = q[b, hq, i].double()
                    o = (K @ qv) * scale
                    # fp32: d exact products summed (d roundings of the running sum of magnitudes), scaled (one more),
                    # then the cap (its argument, a base-2 exponential, a quotient: below 2^-20 of the cap) and the
                    # bias (one rounding of the distance, one of the product, one of the difference)
                    err = 2.0 ** -24 * (d + 4) * float(((K.abs() @ qv.abs()) * scale)[see].max())
                    if softcap:
                        o = softcap * torch.tanh(o / softcap)
                        err += 2.0 ** -20 * softcap
                    if slopes is not None:
                        far = (pos[r] - pos).abs().double()
                        o = o - float(slopes[hq]) * far
                        w_err = 3 * 2.0 ** -24 * float(slopes[hq]) * far
                        w = torch.exp(torch.where(see, o, torch.tensor(-math.inf, dtype=torch.float64)) - o[see].max())
                        # a bias that is large enough to round badly has a weight that is small enough not to matter
                        err += float((w_err * torch.where(w > 2.0 ** -40, 1.0, 0.0)).max())
                    o = torch.where(see, o, torch.tensor(-math.inf, dtype=torch.float64))
                    z = torch.logsumexp(o, 0)
                    total = torch.logaddexp(z, torch.tensor(math.log(n), dtype=torch.float64)) if n else z
                    w = torch.exp(o - total)
                    out[b, hq, i] = w @ V
                    mass[b, hq, i] = w @ V.abs()
                    lse[b, hq, i] = z
                    # exponentials (2^-22 from the instruction, a rounding of its argument of up to 2^-24 times that)
                    logit_err[b, hq, i] = err + 2.0 ** -21 + 2.0 ** -23 * float(o[see].abs().max())
    return out, lse, mass, logit_err


def assert_chunk_close(got_out, got_lse, ref, new, what=""):
    """|out - want| <= 2^-8 |want|                  the result is rounded to bf16 once (half a step of 2^-7)
                      + (2^-8 + 4 e) sum w |v|       each weight is rounded to bf16 once; e bounds a logit's error, which a
                                                     weight and its normaliser both carry (twice e each, to first order)
                      + 2^-126                       results below the smallest normal number are flushed
       |lse - want| <= e + 2^-22 (1 + |want|)        the logarithm and two roundings of the result"""
    out, lse, mass, err = ref
    got = got_out.detach().cpu().double()
    for b in range(out.shape[0]):
        N = int(new[b])
        o, g, m, e = out[b, :, :N], got[b, :, :N], mass[b, :, :N], err[b, :, :N]
        tol = 2.0 ** -8 * o.abs() * (1 + 2.0 ** -8) + (2.0 ** -8 + 4 * e[..., None]) * m + 2.0 ** -126
        assert torch.isfinite(g).all(), f"{what}: sequence {b}: non-finite outputs"
        bad = (g - o).abs() > tol
        assert not bad.any(), (f"{what}: sequence {b}: {int(bad.sum())} of {bad.numel()} outputs off, first at {bad.nonzero()[0].tolist()}, "
                               f"worst {float(((g - o).abs() / tol).max()):.2f} of the tolerance")
        if got_lse is None:
            continue
        z, y = lse[b, :, :N], got_lse[b, :, :N].detach().cpu().double()
        empty = torch.isinf(z)
        assert torch.equal(torch.isinf(y) & (y < 0), empty), f"{what}: sequence {b}: rows that see nothing"
        diff = (y - z).abs()[~empty]
        bound = (e + 2.0 ** -22 * (1 + z.abs()))[~empty]
        assert (diff <= bound).all(), f"{what}: sequence {b}: lse off by up to {float((diff / bound).max()):.2f} of the tolerance"
