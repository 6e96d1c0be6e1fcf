"""Attention over pages in 4 bits against the definition in 64 bits."""
import pytest
import torch

from q4_util import check, paged_cache

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def csp():
    from paper_2412_04652_b200 import binding
    binding.lib()
    return binding


def _case(csp, rows, new, G=1, d=128, page_rows=128, n=1.0, scale=0.0, seed=1, cap=None, lse=True, gain=1.0, q_gain=1.5, mods=None, dense_edit=None):
    rows, new = torch.tensor(rows, dtype=torch.int32), torch.tensor(new, dtype=torch.int32)
    B, H = rows.shape
    T = max(int(new.max()), 1)
    cap = cap or max(int(rows.max()), 1)
    dense, pools, table = paged_cache(rows, cap, H, d, page_rows, seed, gain)
    gen = torch.Generator().manual_seed(seed + 1)
    q = (torch.randn(B, T, H * G, d, generator=gen) * q_gain).to(torch.bfloat16).cuda().transpose(1, 2)
    out = torch.full((B, T, H * G, d), 7.0, dtype=torch.bfloat16, device="cuda").transpose(1, 2)
    z = torch.full((B, H * G, T), 7.0, device="cuda") if lse else None
    p = csp.Params(B, H * G, H, d, 1, 0, cap, cap, n=n, scale=scale)
    ws = csp.new_chunk_q4_workspace(p, T)
    kw = mods(B, H, G, cap) if mods else {}
    sm = csp.ScoreMods(**{k: v.cuda() if torch.is_tensor(v) else v for k, v in kw.items()}) if kw else None
    K, V = (csp.Q4Cache(*x) for x in pools)
    csp.chunk_attn_q4_paged(p, q, K, V, table, rows.cuda(), out, ws, n_new=new.cuda(), mods=sm, lse=z)
    assert csp.device_status(ws) == 0
    for b in range(B):                                   # tokens that nobody brought are left as they were
        assert (out[b, :, int(new[b]):] == 7.0).all() and (z is None or (z[b, :, int(new[b]):] == 7.0).all())
    check(out, z, q, dense, rows, new, n=n, scale=scale, **kw)
    return p, q, K, V, table, rows, out, z, ws


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows", [1, 2, 15, 17, 31, 33, 63, 64, 65, 127, 128, 129, 300, 1000])
def test_one_token_lengths(csp, rows, d):
    _case(csp, [[rows, max(rows - 1, 1)]], [1], d=d)


@pytest.mark.parametrize("G", [1, 2, 3, 5, 7, 8])
def test_one_token_groups(csp, G):
    _case(csp, [[400, 77, 129], [1, 650, 64]], [1, 1], G=G, seed=G)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,T", [(1, 2), (1, 8), (1, 9), (1, 16), (1, 17), (2, 9), (4, 5), (7, 2), (7, 3), (8, 33), (3, 100), (1, 130), (1, 257), (5, 70)])
def test_chunks(csp, G, T, d):
    _case(csp, [[T + 200, T], [T + 3, 333 + T]], [T, max(T - 3, 1)], G=G, d=d, seed=T)


def test_nothing_to_see(csp):
    """Sequences without tokens, heads without rows, more tokens than rows (flagged elsewhere): zeros and -infinity."""
    rows = torch.tensor([[5, 0], [0, 0], [200, 130]])
    p, q, K, V, table, rows, out, z, ws = _case(csp, [[200, 130], [5, 9], [64, 65]], [2, 0, 3], G=2)
    new = torch.tensor([4, 1, 3], dtype=torch.int32, device="cuda")
    few = torch.tensor([[2, 0], [0, 1], [64, 65]], dtype=torch.int32, device="cuda")
    T = 4
    p = csp.Params(3, 4, 2, 128, 1, 0, 200, 200)
    q = torch.randn(3, 4, T, 128, device="cuda").to(torch.bfloat16)
    out = torch.full_like(q, 7.0)
    z = torch.full((3, 4, T), 7.0, device="cuda")
    ws = csp.new_chunk_q4_workspace(p, T)
    csp.chunk_attn_q4_paged(p, q, K, V, table, few, out, ws, n_new=new, lse=z)
    assert csp.device_status(ws) == csp.DEV_BAD_LEN      # more tokens than rows
    assert (out[0, :2, :2] == 0).all() and torch.isinf(z[0, :2, :2]).all()
    assert torch.isfinite(z[0, :2, 2:]).all()
    assert (out[0, 2:, :4] == 0).all() and torch.isinf(z[0, 2:, :4]).all()
    assert (out[1, :2, :1] == 0).all() and (out[1, :, 1:] == 7.0).all()


@pytest.mark.parametrize("T", [1, 4, 40])
@pytest.mark.parametrize("kind", ["cap", "bias", "positions", "docs", "prefix", "all"])
def test_modifiers(csp, kind, T):
    def mods(B, H, G, cap):
        gen = torch.Generator().manual_seed(5)
        m = {}
        if kind in ("cap", "all"):
            m["softcap"] = 15.0
        if kind in ("bias", "positions", "all"):
            m["slopes"] = torch.exp2(-torch.arange(1, H * G + 1).float())
        if kind in ("positions", "all"):
            m["positions"] = torch.randint(1, 9, (B, H, cap), generator=gen).cumsum(2).to(torch.int32)
        if kind in ("docs", "all"):
            m["documents"] = (torch.arange(cap)[None] * 4 // torch.tensor([[400], [300]])).to(torch.int32)
        if kind in ("prefix", "all"):
            m["prefix"] = torch.tensor([[390, 10], [0, 1000]], dtype=torch.int32)
        return m
    _case(csp, [[400, 390], [222, 300]], [T, max(T - 1, 1)], G=3, mods=mods, seed=T)


@pytest.mark.parametrize("T", [1, 30])
@pytest.mark.parametrize("n", [0.0, 1.0, 2.5])
def test_normaliser(csp, n, T):
    _case(csp, [[300, 40]], [T], n=n, seed=3)
    _case(csp, [[300, 40]], [T], n=n, scale=0.01, seed=3)


@pytest.mark.parametrize("T", [1, 30])
def test_large_and_small_values(csp, T):
    """Scales of V that differ by many powers of two between the rows, queries far from one."""
    _case(csp, [[500, 129]], [T], gain=torch.exp2(torch.randint(-12, 12, (1, 2, 500, 1)).float()), q_gain=0.02, seed=9)
    _case(csp, [[500, 129]], [T], gain=1e-20, q_gain=1e20, seed=9)
    _case(csp, [[500, 129]], [T], gain=1e18, q_gain=1e-18, seed=9)


@pytest.mark.parametrize("T", [1, 40])
def test_many_units_and_long_caches(csp, T):
    """More items than blocks, and caches that are cut between blocks."""
    _case(csp, [[70 + 13 * (b * 8 + h) % 500 + T for h in range(8)] for b in range(24)], [T] * 24, d=64, lse=False)
    _case(csp, [[9000, 5000]], [T], G=4, page_rows=256)
