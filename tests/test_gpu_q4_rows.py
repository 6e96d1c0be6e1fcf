"""Rows on their way into 4 bits and back where other tests do not reach: scales that lie in the middle between two bf16 numbers, reads
and appends of the size where blocks go round more than once."""
import math
from fractions import Fraction

import pytest
import torch

from q4_util import random_rows, values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def csp():
    from paper_2412_04652_b200 import binding
    binding.lib()
    return binding


def _rounded(x):
    """A positive fraction as the bf16 number next to it, the even one of two."""
    e = math.floor(math.log2(float(x)))
    e += (Fraction(2) ** (e + 1) <= x) - (Fraction(2) ** e > x)
    unit = Fraction(2) ** (e - 7)
    n, rest = divmod(x, unit)
    return float((n + (2 * rest > unit or (2 * rest == unit and n % 2 == 1))) * unit)


def test_scales_between_two_numbers(csp):
    """Rows whose spread is 15 times the middle between two bf16 numbers, or next to that: the scale is what (max - min) / 15 rounds to."""
    gen = torch.Generator().manual_seed(1)
    n, d = 6000, 64
    middle = (2 * torch.randint(128, 256, (n,), generator=gen) + 1) * torch.exp2(torch.randint(-90, 90, (n,), generator=gen).float())
    lo = (torch.randn(n, generator=gen) * middle * torch.exp2(torch.randint(-20, 6, (n,), generator=gen).float())).to(torch.bfloat16)
    hi = (15 * middle + lo.float()).to(torch.bfloat16)
    lo[0], hi[0] = 25.0, 4480.0                          # 4455 / 15 = 297, between 296 and 298
    x = lo[:, None].repeat(1, d)
    x[:, 17] = hi
    x = x[None, None].cuda()
    cap = -(-n // 128) * 128
    p = csp.Params(1, 1, 1, d, 1, 0, cap, cap)
    K, V = csp.new_q4_cache(cap // 128, 1, 128, d), csp.new_q4_cache(cap // 128, 1, 128, d)
    table = torch.arange(cap // 128, dtype=torch.int32, device="cuda")[None]
    rows, ws = torch.zeros(1, 1, dtype=torch.int32, device="cuda"), csp.new_append_workspace(p)
    csp.append_q4_paged(p, x, x, K, V, table, rows, rows, ws)
    assert csp.device_status(ws) == 0
    got = K.scales.flatten(0, 2)[:n].cpu().double()
    want = torch.tensor([_rounded((Fraction(float(b)) - Fraction(float(a))) / 15) for a, b in zip(lo, hi)], dtype=torch.float64)
    off = got[:, 0] != want
    assert float(want[0]) == 296.0
    assert not off.any(), f"{int(off.sum())} of {n} scales, first at {int(off.nonzero()[0])}: {float(got[off][0, 0])} for {float(want[off][0])}"
    assert torch.equal(got[:, 1], lo.double())


def _pool(n_pages, H, d, seed, R=128):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randint(0, 256, (n_pages, H, R, d // 2), generator=gen, dtype=torch.uint8, device="cuda"),
            torch.randn(n_pages, H, R, 2, generator=gen, device="cuda").to(torch.bfloat16))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d,cap", [(64, 6500), (128, 4100)])
@pytest.mark.parametrize("with_v", [True, False])
def test_large_reads(csp, dtype, d, cap, with_v):
    """So many rows that a lane has four of them under way: whole caches, parts of them, heads without rows, and a page that is none."""
    B, H, R = 2, 4, 128
    mp = -(-cap // R)
    n_pages = B * mp + 1
    table = torch.randperm(n_pages, generator=torch.Generator().manual_seed(d))[:B * mp].reshape(B, mp).to(torch.int32).cuda()
    table[1, 2] = n_pages
    rows = torch.tensor([[cap, 0, cap - 1, 257], [cap - 130, cap, 1, cap]], dtype=torch.int32, device="cuda")
    first = torch.tensor([[0, 0, 77, 256], [0, cap - 1, 0, 300]], dtype=torch.int32, device="cuda")
    pools = [_pool(n_pages, H, d, d + i) for i in range(2)]
    K, V = (csp.Q4Cache(*x) for x in pools)
    p = csp.Params(B, H, H, d, 1, 0, cap, cap, dtype=csp.F32 if dtype == torch.float32 else csp.BF16)
    ws = csp.new_append_workspace(p)
    outs = [torch.full((B, cap + 3, H, d), 9.0, dtype=dtype, device="cuda").transpose(1, 2) for _ in range(2)]
    csp.load_q4_paged(p, K, V if with_v else None, table, rows, outs[0], outs[1] if with_v else None, ws, first=first)
    assert csp.device_status(ws) == csp.DEV_BAD_LEN      # the page that is none
    for out, pool in zip(outs, pools[:2 if with_v else 1]):
        for b in range(B):
            for h in range(H):
                t = torch.arange(int(first[b, h]), int(rows[b, h]), device="cuda")
                page = table[b].long()[t // R]
                at = page.clamp(max=n_pages - 1), h, t % R
                want = values(pool[0][at], pool[1][at]).float().to(dtype)
                want[page == n_pages] = 0
                assert torch.equal(out[b, h, :len(t)], want) and (out[b, h, len(t):] == 9.0).all(), (b, h)


@pytest.mark.parametrize("cap", [200, 6500])
def test_flags_of_reads(csp, cap):
    """Rows that do not fit are left out, a negative first row counts as none, counts past the capacity are cut."""
    B, H, d, R = 2, 4, 64, 128
    mp = -(-cap // R)
    table = torch.arange(B * mp, dtype=torch.int32, device="cuda").reshape(B, mp)
    pool = _pool(B * mp, H, d, 5)
    K = csp.Q4Cache(*pool)
    p = csp.Params(B, H, H, d, 1, 0, cap, cap)
    whole = values(pool[0], pool[1]).float().to(torch.bfloat16).reshape(B, mp, H, R, d).transpose(1, 2).reshape(B, H, mp * R, d)

    def call(rows, first, slots):
        ws = csp.new_append_workspace(p)
        out = torch.full((B, H, slots, d), 9.0, dtype=torch.bfloat16, device="cuda")
        as_int = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda").expand(B, H).contiguous()  # noqa: E731
        csp.load_q4_paged(p, K, None, table, as_int(rows), out, None, ws, first=as_int(first))
        return csp.device_status(ws), out
    status, out = call(cap, 0, cap - 9)
    assert status == csp.DEV_CAPACITY and torch.equal(out, whole[:, :, :cap - 9])
    status, out = call(cap, -5, cap + 2)
    assert status == csp.DEV_BAD_LEN and torch.equal(out[:, :, :cap], whole[:, :, :cap]) and (out[:, :, cap:] == 9.0).all()
    status, out = call(cap + 1, 3, cap + 2)
    assert status == csp.DEV_BAD_LEN and torch.equal(out[:, :, :cap - 3], whole[:, :, 3:cap]) and (out[:, :, cap - 3:] == 9.0).all()
    status, out = call(-1, 0, cap)
    assert status == csp.DEV_BAD_LEN and (out == 9.0).all()
    status, out = call([[cap, 1, 7, 0]], [[cap, 5, 7, 0]], cap)
    assert status == 0 and (out == 9.0).all()


@pytest.mark.parametrize("kind,d,rope", [("q4", 64, 64), ("q4", 128, 128), ("bf16", 64, 32), ("bf16", 128, 128), ("bf16", 256, 256), ("fp32", 128, 64)])
@pytest.mark.parametrize("positions", [False, True])
def test_groups_of_lanes_go_over_several_heads(csp, kind, d, rope, positions):
    """Batches of prompt chunks, for which a block goes over the heads more than once with one set of cosines (each head with its own
    rows, so that positions that are row numbers differ): the same bits as calls of a hundred tokens of one sequence, for which it does not."""
    B, H, G, T, R = 8, 8, 4, 603, 128
    dtype = torch.float32 if kind == "fp32" else torch.bfloat16
    gen = torch.Generator(device="cuda").manual_seed(d)
    k, v, q = (torch.randn(B, T, h, d, generator=gen, device="cuda").to(dtype).transpose(1, 2) for h in (H, H, H * G))
    first = torch.randint(0, 60, (B, H), generator=gen, device="cuda", dtype=torch.int32)
    new = torch.tensor([T, T - 1, 0, T, 500, T, 1, T], dtype=torch.int32, device="cuda")
    cap, mp = 768, 6
    table = torch.randperm(B * mp, generator=gen, device="cuda").reshape(B, mp).to(torch.int32)
    angle = torch.arange(1000, device="cuda")[:, None] * torch.exp2(-torch.arange(rope // 2, device="cuda") / 4.0)
    cos_sin = torch.cat([angle.cos(), angle.sin()], 1)
    pos = torch.randint(0, 1000, (B, T), generator=gen, device="cuda", dtype=torch.int32) if positions else None
    both = []
    for small in (False, True):
        if kind == "q4":
            K, V = csp.new_q4_cache(B * mp, H, R, d), csp.new_q4_cache(B * mp, H, R, d)
        else:
            K, V = (torch.zeros(B * mp, H, R, d, dtype=dtype, device="cuda") for _ in range(2))
        q_out, rows = torch.zeros_like(q), first.clone()

        def call(b0, b1, i0, i1):
            n = (new[b0:b1] - i0).clamp(0, i1 - i0)
            p = csp.Params(b1 - b0, H * G, H, d, 1, 0, cap, cap, dtype=csp.F32 if kind == "fp32" else csp.BF16)
            ws = csp.new_append_workspace(p)
            at = rows[b0:b1].clone()
            r = csp.Rope(cos_sin, positions=None if pos is None else pos[b0:b1, i0:i1], interleaved=d == 128)
            f = csp.append_q4_paged if kind == "q4" else csp.append_rope_paged
            f(p, k[b0:b1, :, i0:i1], v[b0:b1, :, i0:i1], K, V, table[b0:b1].contiguous(), at, at, ws, rope=r, n_new=n, q=q[b0:b1, :, i0:i1], q_out=q_out[b0:b1, :, i0:i1])
            assert csp.device_status(ws) == 0
            rows[b0:b1] = at
        if small:
            for b in range(B):
                for i in range(0, T, 100):
                    call(b, b + 1, i, min(i + 100, T))
        else:
            call(0, B, 0, T)
        assert torch.equal(rows, first + new[:, None])
        both.append((K.codes, K.scales, V.codes, V.scales, q_out) if kind == "q4" else (K, V, q_out))
    for a, b in zip(*both):
        assert torch.equal(a, b)
    # ... and those of a query are what the definition says
    at = pos[0, :T] if positions else first[0, 0] + torch.arange(T, device="cuda")
    c, s = cos_sin.double()[at.long()].chunk(2, -1)
    x, got = q[0, 1].double(), both[0][-1][0, 1].double()
    one, two = (slice(0, rope, 2), slice(1, rope, 2)) if d == 128 else (slice(0, rope // 2), slice(rope // 2, rope))
    half = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    for want, mag, y in ((x[:, one] * c - x[:, two] * s, (x[:, one] * c).abs() + (x[:, two] * s).abs(), got[:, one]),
                         (x[:, two] * c + x[:, one] * s, (x[:, two] * c).abs() + (x[:, one] * s).abs(), got[:, two])):
        assert ((y - want).abs() <= 3 * 2.0 ** -24 * mag * (1 + half) + half * want.abs() + 2.0 ** -126).all()
    assert torch.equal(got[:, rope:], x[:, rope:])
