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
