"""Shared by the tests of the cache in 4 bits: the format in 64 bits, caches and their pages, and the attention's tolerance."""
from __future__ import annotations

import math

import numpy as np
import torch

from chunk_util import reference

SMALLEST = 2.0 ** -126


def quantise(x):
    """bf16 rows [..., d] -> (codes [..., d] whole numbers, scale, base [...], how far every quotient is from the middle
    between two codes), in 64 bits."""
    x = x.double()
    base, top = x.amin(-1), x.amax(-1)
    scale = ((top - base) / 15).to(torch.bfloat16).double()
    scale = torch.where(scale < SMALLEST, 0.0, scale)
    y = torch.where(scale[..., None] > 0, (x - base[..., None]) / scale[..., None], 0.0)
    return (y + 0.5).floor().clamp(0, 15), scale, base, ((y - y.floor()) - 0.5).abs()


def values(codes, scales):
    """uint8 [..., d / 2], bf16 [..., 2] -> the rows' values in 64 bits (exact)."""
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).double()
    return scales[..., 1:].double() + scales[..., :1].double() * c


def random_rows(shape, gen, gain=1.0):
    """Codes and scales of rows as they come out of quantising normal values."""
    x = (torch.randn(*shape, generator=gen) * gain).to(torch.bfloat16)
    codes, scale, base, _ = quantise(x)
    c = codes.to(torch.uint8)
    return c[..., 0::2] | (c[..., 1::2] << 4), torch.stack([scale, base], -1).to(torch.bfloat16)


def to_pages(dense, rows, page_rows, order, n_pages, fill):
    """[B, H, cap, w] -> pool [n_pages, H, page_rows, w] and table; rows behind the last one, and spare pages, are `fill`."""
    B, H, cap, w = dense.shape
    pool = torch.full((n_pages, H, page_rows, w), fill, dtype=dense.dtype)
    table = np.full((B, max(1, -(-cap // page_rows))), 10 ** 6, np.int32)
    nxt = 0
    for b in range(B):
        for i in range(-(-int(rows[b].max()) // page_rows)):
            pg = int(order[nxt])
            nxt += 1
            table[b, i] = pg
            for h in range(H):
                r1 = min((i + 1) * page_rows, int(rows[b, h]))
                if r1 > i * page_rows:
                    pool[pg, h, :r1 - i * page_rows] = dense[b, h, i * page_rows:r1]
    return pool, torch.from_numpy(table)


def paged_cache(rows, cap, H, d, page_rows, seed, gain=1.0):
    """K and V in 4 bits, dense on the CPU and paged on the GPU: (dense pairs, pool pairs, table).  What no row fills is
    garbage: codes of 15, scales that are no number."""
    gen = torch.Generator().manual_seed(seed)
    B = rows.shape[0]
    n_pages = int(sum(-(-int(r.max()) // page_rows) for r in rows)) + 2
    order = np.random.RandomState(seed).permutation(n_pages)
    dense, pools, table = [], [], None
    for _ in range(2):
        codes, scales = random_rows((B, H, cap, d), gen, gain)
        dense.append((codes, scales))
        pc, table = to_pages(codes, rows, page_rows, order, n_pages, 255)
        ps, _ = to_pages(scales, rows, page_rows, order, n_pages, float("nan"))
        pools.append((pc.cuda(), ps.cuda()))
    return dense, pools, table.cuda()


def check(got_out, got_lse, q, dense, rows, new, what="", n=1.0, scale=0.0, **mods):
    """Against the definition in 64 bits of the values base + scale code.

    A logit is scale' (s <q, c> + b sum q): d products of a half and a whole number, added up in fp32 by the tensor cores (a
    unit in the last place of the running sum each, 2^-23), three operations more for the row's numbers and its factor; relative to the
    magnitudes s <|q|, c> + |b| sum |q|.  A query's value is a half after scaling to a largest value in [1, 2): exact
    down to 2^-14 of it, below that off by 2^-25 of the power of two that is at most the largest value.  Modifiers and exponentials as in
    `reference`, which bounds them by e.
    |out - want| <= 2^-8 |want|                             rounded to bf16 once
                  + (r 2^-11 + 4 e + 2^-23 L) sum w (s c + |b|) r = 1: weights times scales are rounded to halves; r = 2, with more than
                                                            sixteen query rows per KV head: weights are, and the values of V; e as
                                                            there; L rows added up
                  + L 2^-25 15 max s                            weights times scales below 2^-14 of the largest scale; r = 2: weights
                                                            below 2^-14, of the largest values
                  + (r = 2) 2^-17 max (15 s + |b|)              the values of V are halves times 2^7 of a power of two that is at most
                                                            the largest of them: base and sum, each rounded by up to 2^-25 where
                                                            they are below 2^-14, and the weights add up to one at most
                  + 2^-126"""
    (kc, ks), (vc, vs) = dense
    K, V = values(kc, ks), values(vc, vs)
    out, lse, mass, err = reference(q.cpu(), K, V, rows, new, n=n, scale=scale, **mods)
    mag_k = (K - ks[..., 1:].double()) + ks[..., 1:].double().abs()
    mag_v = (V - vs[..., 1:].double()) + vs[..., 1:].double().abs()
    B, Hq, T, d = q.shape
    G = Hq // K.shape[1]
    sc = scale or 1.0 / math.sqrt(d)
    _, _, mass, _ = reference(q.cpu(), K, mag_v, rows, new, n=n, scale=scale, **mods)
    got = got_out.detach().cpu().double()
    rounds = 2 if T * G > 16 else 1
    for b in range(B):
        N = int(new[b])
        for hq in range(Hq):
            L = int(rows[b, hq // G])
            if L == 0 or N == 0:
                assert (got[b, hq, :N] == 0).all(), f"{what}: nothing seen, but not zero"
                continue
            qa = q[b, hq, :N].cpu().double().abs()
            mk = mag_k[b, hq // G, :L]
            e = err[b, hq, :N] + sc * (2.0 ** -23 * (d + 4) * (qa @ mk.T).amax(1) + 2.0 ** -25 * qa.amax(1) * (K - ks[..., 1:].double())[b, hq // G, :L].sum(1).max())
            o, g, m = out[b, hq, :N], got[b, hq, :N], mass[b, hq, :N]
            s_max = 15 * float(vs[b, hq // G, :L, 0].double().max())
            v_max = float((15 * vs[b, hq // G, :L, 0].double() + vs[b, hq // G, :L, 1].double().abs()).max())
            small = L * 2.0 ** -25 * s_max if rounds == 1 else (L * 2.0 ** -25 + 2.0 ** -17) * v_max
            tol = 2.0 ** -8 * o.abs() * (1 + 2.0 ** -8) + (rounds * 2.0 ** -11 + 4 * e[:, None] + 2.0 ** -23 * L) * m + small + 2.0 ** -126
            assert torch.isfinite(g).all(), f"{what}: sequence {b}, head {hq}: non-finite outputs"
            bad = (g - o).abs() > tol
            assert not bad.any(), (f"{what}: sequence {b}, head {hq}: {int(bad.sum())} of {bad.numel()} outputs off, first at "
                                   f"{bad.nonzero()[0].tolist()}, worst {float(((g - o).abs() / tol).max()):.2f} of the tolerance")
            if got_lse is None:
                continue
            z, y = lse[b, hq, :N], got_lse[b, hq, :N].detach().cpu().double()
            empty = torch.isinf(z)
            assert torch.equal(torch.isinf(y) & (y < 0), empty), f"{what}: sequence {b}, head {hq}: rows that see nothing"
            bound = (e + 2.0 ** -22 * (1 + z.abs()) + 2.0 ** -23 * L)[~empty]
            diff = (y - z).abs()[~empty]
            assert (diff <= bound).all(), f"{what}: sequence {b}, head {hq}: lse off by up to {float((diff / bound).max()):.2f} of the tolerance"
