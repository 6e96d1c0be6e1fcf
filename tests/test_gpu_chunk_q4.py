"""Attention over pages in 4 bits against the definition in 64 bits."""
import pytest
import torch

from q4_util import check, paged_cache, random_rows, values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def csp():
    from paper_2412_04652_b200 import binding
    binding.lib()
    return binding


def _case(csp, rows, new, G=1, d=128, page_rows=128, n=1.0, scale=0.0, seed=1, cap=None, lse=True, gain=1.0, q_gain=1.5, mods=None, capacity=None):
    rows, new = torch.tensor(rows, dtype=torch.int32), torch.tensor(new, dtype=torch.int32)
    B, H = rows.shape
    T = max(int(new.max()), 1)
    cap = cap or max(int(rows.max()), 1)
    dense, pools, table = paged_cache(rows, cap, H, d, page_rows, seed, gain)
    gen = torch.Generator().manual_seed(seed + 1)
    q = (torch.randn(B, T, H * G, d, generator=gen) * q_gain).to(torch.bfloat16).cuda().transpose(1, 2)
    out = torch.full((B, T, H * G, d), 7.0, dtype=torch.bfloat16, device="cuda").transpose(1, 2)
    z = torch.full((B, H * G, T), 7.0, device="cuda") if lse else None
    if capacity:                                         # more than the rows need
        wide = torch.full((B, -(-capacity // page_rows)), 10 ** 6, dtype=torch.int32, device="cuda")
        wide[:, :table.shape[1]] = table
        table = wide
    p = csp.Params(B, H * G, H, d, 1, 0, capacity or cap, capacity or cap, n=n, scale=scale)
    ws = csp.new_chunk_q4_workspace(p, T)
    kw = mods(B, H, G, capacity or cap) if mods else {}
    sm = csp.ScoreMods(**{k: v.cuda() if torch.is_tensor(v) else v for k, v in kw.items()}) if kw else None
    K, V = (csp.Q4Cache(*x) for x in pools)
    csp.chunk_attn_q4_paged(p, q, K, V, table, rows.cuda(), out, ws, n_new=new.cuda(), mods=sm, lse=z)
    assert csp.device_status(ws) == 0
    for b in range(B):                                   # tokens that nobody brought are left as they were
        assert (out[b, :, int(new[b]):] == 7.0).all() and (z is None or (z[b, :, int(new[b]):] == 7.0).all())
    for k in ("positions", "documents"):
        if k in kw:
            kw[k] = kw[k][..., :cap]
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
@pytest.mark.parametrize("G,T", [(1, 2), (1, 8), (1, 9), (1, 16), (1, 17), (2, 9), (4, 5), (7, 2), (7, 3), (7, 6), (7, 7), (1, 48), (1, 49), (4, 12), (4, 13), (3, 15), (8, 33), (3, 100), (1, 130), (1, 257), (5, 70)])
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


def _mods(kind):
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
    return mods


@pytest.mark.parametrize("T", [1, 4, 40])
@pytest.mark.parametrize("kind", ["cap", "bias", "positions", "docs", "prefix", "all"])
def test_modifiers(csp, kind, T):
    _case(csp, [[400, 390], [222, 300]], [T, max(T - 1, 1)], G=3, mods=_mods(kind), seed=T)


WIDE = 1 << 18                                           # a capacity for which items of sixteen rows are taken where rows allow it


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,T", [(1, 9), (1, 16), (1, 31), (2, 8), (3, 4), (4, 4), (4, 8), (5, 3), (5, 5), (7, 2), (7, 4), (8, 2), (8, 5)])
def test_items_of_sixteen_rows(csp, G, T, d):
    _case(csp, [[T + 200, T], [T + 3, 333 + T]], [T, max(T - 3, 1)], G=G, d=d, seed=T, capacity=WIDE)
    _case(csp, [[9000, 5000]], [T], G=G, d=d, capacity=2 * WIDE, lse=False)


@pytest.mark.parametrize("kind", ["cap", "bias", "positions", "docs", "prefix", "all"])
def test_modifiers_of_sixteen_rows(csp, kind):
    _case(csp, [[400, 390], [222, 300]], [5, 4], G=3, mods=_mods(kind), capacity=WIDE)
    _case(csp, [[400, 390], [222, 300]], [9, 10], G=3, d=64, mods=_mods(kind), capacity=WIDE)


def test_numbers_of_sixteen_rows(csp):
    """Normalisers, large and small values, NaN behind the last row and in front of it."""
    for n in (0.0, 1.0, 2.5):
        _case(csp, [[300, 40]], [12], n=n, seed=3, capacity=2 * WIDE)
    _case(csp, [[500, 129]], [12], gain=torch.exp2(torch.randint(-12, 12, (1, 2, 500, 1)).float()), q_gain=0.02, seed=9, capacity=2 * WIDE)
    _case(csp, [[500, 129]], [12], gain=2.0 ** -100, q_gain=2.0 ** 100, seed=9, capacity=2 * WIDE)
    p, q, K, V, table, rows, out, z, ws = _case(csp, [[200, 150]], [6], G=2, capacity=2 * WIDE)
    good = out.clone()
    for x in (K, V):
        keep = x.scales.clone()
        x.scales[table[0, 0].long(), 0, 5, 0] = float("nan")
        csp.chunk_attn_q4_paged(p, q, K, V, table, rows.cuda(), out, ws)
        assert csp.device_status(ws) == 0 and torch.isnan(out[0, :2]).all() and torch.equal(out[0, 2:], good[0, 2:])
        x.scales.copy_(keep)
    q[0, 0, 0] = 0
    csp.chunk_attn_q4_paged(p, q, K, V, table, rows.cuda(), out, ws)
    assert torch.isfinite(out).all() and torch.equal(out[0, 1:], good[0, 1:])


@pytest.mark.parametrize("G,T", [(1, 1), (1, 30), (2, 30)])
@pytest.mark.parametrize("n", [0.0, 1.0, 2.5])
def test_normaliser(csp, n, G, T):
    _case(csp, [[300, 40]], [T], G=G, n=n, seed=3)
    _case(csp, [[300, 40]], [T], G=G, n=n, scale=0.01, seed=3)


@pytest.mark.parametrize("T", [1, 30, 60])
def test_large_and_small_values(csp, T):
    """Scales of V that differ by many powers of two between the rows, queries far from one."""
    _case(csp, [[500, 129]], [T], gain=torch.exp2(torch.randint(-12, 12, (1, 2, 500, 1)).float()), q_gain=0.02, seed=9)
    _case(csp, [[500, 129]], [T], gain=1e-20, q_gain=1e20, seed=9)
    _case(csp, [[500, 129]], [T], gain=1e18, q_gain=1e-18, seed=9)
    _case(csp, [[500, 129]], [T], gain=2.0 ** -100, q_gain=2.0 ** 100, seed=9)
    _case(csp, [[500, 129]], [T], gain=2.0 ** 110, q_gain=2.0 ** -118, seed=9)


@pytest.mark.parametrize("T", [1, 40, 60])
def test_many_units_and_long_caches(csp, T):
    """More items than blocks, and caches that are cut between blocks."""
    _case(csp, [[70 + 13 * (b * 8 + h) % 500 + T for h in range(8)] for b in range(24)], [T] * 24, d=64, lse=False)
    _case(csp, [[9000, 5000]], [T], G=4, page_rows=256)


# ---- what may be wrong with the inputs

@pytest.mark.parametrize("T", [1, 40, 60])
def test_a_page_outside_the_pool_reads_as_zeros(csp, T):
    p, q, K, V, table, rows, out, z, ws = _case(csp, [[384, 300]], [T])
    (kc, ks), (vc, vs) = [(c.cpu(), s.cpu()) for c, s in ((K.codes, K.scales), (V.codes, V.scales))]
    n_pages = kc.shape[0]
    for bad in (-1, n_pages, 2 ** 31 - 1):
        t = table.clone()
        t[0, 1] = bad
        csp.chunk_attn_q4_paged(p, q, K, V, t, rows.cuda(), out, ws, lse=z)
        assert csp.device_status(ws) == csp.DEV_BAD_LEN
        dense = []
        for c, s in ((kc, ks), (vc, vs)):
            pages = table[0].cpu().long()
            pair = [x[pages].transpose(0, 1).flatten(1, 2)[None].clone() for x in (c, s)]
            for x in pair:
                x[:, :, 128:256] = 0
            for h in range(2):
                pair[1][0, h, int(rows[0, h]):] = 0      # (what no row fills is not compared either)
            dense.append(pair)
        check(out, z, q, dense, rows, torch.tensor([T]), what=str(bad))
    csp.chunk_attn_q4_paged(p, q, K, V, table, rows.cuda(), out, ws)
    assert csp.device_status(ws) == 0


@pytest.mark.parametrize("T", [1, 40])
def test_bad_counts_are_clamped_and_flagged(csp, T):
    p, q, K, V, table, rows, out, z, ws = _case(csp, [[128, 100], [90, 128]], [T, T], cap=128, G=2)
    good_out, good_z = out.clone(), z.clone()
    csp.chunk_attn_q4_paged(p, q, K, V, table, torch.tensor([[1000, 100], [90, 128]], dtype=torch.int32, device="cuda"), out, ws,
                            n_new=torch.tensor([T + 5, T], dtype=torch.int32, device="cuda"), lse=z)
    assert csp.device_status(ws) == csp.DEV_BAD_LEN and torch.equal(out, good_out) and torch.equal(z, good_z)
    out.fill_(7.0)
    csp.chunk_attn_q4_paged(p, q, K, V, table, torch.tensor([[128, -4], [90, 128]], dtype=torch.int32, device="cuda"), out, ws,
                            n_new=torch.tensor([T, -1], dtype=torch.int32, device="cuda"), lse=z)
    assert csp.device_status(ws) == csp.DEV_BAD_LEN
    assert torch.equal(out[0, :2], good_out[0, :2]) and (out[0, 2:] == 0).all() and (out[1] == 7.0).all()


@pytest.mark.parametrize("T", [1, 3, 40])
@pytest.mark.parametrize("d", [64, 128])
def test_rows_that_are_no_numbers(csp, T, d):
    """Behind the last row anything may stand, infinities as well as NaN; a visible row that is none makes no number, for its own
    head; one whose key nobody sees does nothing."""
    p, q, K, V, table, rows, out, z, ws = _case(csp, [[200, 150]], [T], d=d, G=2)
    good = out.clone()
    for x in (K, V):
        pages = table[0].long()
        x.scales[pages[1], 0, 200 - 128:] = float("inf")
        x.scales[pages[1], 1, 150 - 128:] = float("-inf")
    csp.chunk_attn_q4_paged(p, q, K, V, table, rows.cuda(), out, ws)
    assert csp.device_status(ws) == 0 and torch.equal(out, good)
    for x, y in ((K, V), (V, K)):
        keep = x.scales.clone()
        x.scales[table[0, 0].long(), 0, 5, 0] = float("nan")
        csp.chunk_attn_q4_paged(p, q, K, V, table, rows.cuda(), out, ws)
        assert csp.device_status(ws) == 0 and torch.isnan(out[0, :2]).all() and torch.equal(out[0, 2:], good[0, 2:])
        x.scales.copy_(keep)
    docs = torch.zeros(1, 200, dtype=torch.int32, device="cuda")
    docs[0, :20] = 1
    csp.chunk_attn_q4_paged(p, q, K, V, table, rows.cuda(), out, ws, mods=csp.ScoreMods(documents=docs))
    good = out.clone()
    K.scales[table[0, 0].long(), 0, 5, 0] = float("nan")
    csp.chunk_attn_q4_paged(p, q, K, V, table, rows.cuda(), out, ws, mods=csp.ScoreMods(documents=docs))
    assert torch.equal(out, good)


@pytest.mark.parametrize("T", [1, 40])
def test_queries_out_of_the_ordinary(csp, T):
    """Zeros weigh every row alike; an infinity or NaN makes no number, for its own row."""
    p, q, K, V, table, rows, out, z, ws = _case(csp, [[200, 150]], [T], G=2)
    good = out.clone()
    q[0, 0, 0] = 0
    csp.chunk_attn_q4_paged(p, q, K, V, table, rows.cuda(), out, ws, lse=z)
    dense = [tuple(x.cpu()[table[0].cpu().long()].transpose(0, 1).flatten(1, 2)[None].clone() for x in (c.codes, c.scales)) for c in (K, V)]
    for _, s in dense:
        s[torch.isnan(s)] = 0
    check(out, z, q, dense, rows, torch.tensor([T]))
    assert torch.equal(out[0, 1:], good[0, 1:]) and torch.equal(out[0, 0, 1:], good[0, 0, 1:])
    for bad in (float("nan"), float("inf"), float("-inf")):
        q[0, 0, 0] = 1.0
        q[0, 0, 0, 77] = bad
        csp.chunk_attn_q4_paged(p, q, K, V, table, rows.cuda(), out, ws, lse=z)
        assert torch.isnan(out[0, 0, 0]).all() and torch.equal(out[0, 1:], good[0, 1:]) and torch.equal(out[0, 0, 1:], good[0, 0, 1:])


@pytest.mark.parametrize("T", [3, 200])
@pytest.mark.parametrize("gap", [2 ** 23 - 400, 2 ** 24, 2 ** 30])
def test_tokens_far_apart(csp, T, gap):
    """A chunk whose first tokens lie `gap` positions in front of the others: exact distances up to 2^23, flagged beyond."""
    cap = 300
    rows = torch.tensor([[300, 299]], dtype=torch.int32)
    dense, pools, table = paged_cache(rows, cap, 2, 64, 128, 5)
    pos = torch.arange(cap, dtype=torch.int32)[None].clone()
    pos[:, cap - T // 2 - 2:] += gap
    mods = dict(slopes=torch.exp2(-torch.arange(1, 5).float()), positions=pos)
    q = torch.randn(1, 4, T, 64, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
    p = csp.Params(1, 4, 2, 64, 1, 0, cap, cap)
    out, z, ws = torch.zeros_like(q), torch.zeros(1, 4, T, device="cuda"), csp.new_chunk_q4_workspace(p, T)
    csp.chunk_attn_q4_paged(p, q, csp.Q4Cache(*pools[0]), csp.Q4Cache(*pools[1]), table, rows.cuda(), out, ws, lse=z,
                            mods=csp.ScoreMods(**{k: v.cuda() for k, v in mods.items()}))
    if gap < 2 ** 23:
        assert csp.device_status(ws) == 0
        check(out, z, q, dense, rows, torch.tensor([T]), **mods)
    else:
        assert csp.device_status(ws) == csp.DEV_BAD_LEN


# ---- how it is called

def _pool(csp, shape, wide, dtype, data):
    """A pool whose pages and heads lie in gaps of a larger one: [n_pages, H, R, w], heads outermost."""
    n, H, R, w = shape
    big = torch.zeros(H, n + 1, R * w + wide, dtype=dtype, device="cuda")
    view = big.as_strided(shape, (big.stride(1), big.stride(0), w, 1))
    view.copy_(data)
    return view


@pytest.mark.parametrize("T", [1, 40])
@pytest.mark.parametrize("d", [64, 128])
def test_strided_pools_queries_and_outputs(csp, T, d):
    p, q, K, V, table, rows, out, z, ws = _case(csp, [[300, 40], [129, 256]], [T, T], G=2, d=d)
    a, b = (csp.Q4Cache(_pool(csp, tuple(x.codes.shape), 48, torch.uint8, x.codes), _pool(csp, tuple(x.scales.shape), 24, torch.bfloat16, x.scales)) for x in (K, V))
    qkv = torch.full((2, T, 9, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    qkv[:, :, 2:6] = q.transpose(1, 2)
    wide = torch.full((2, T, 4, d + 8), 3.0, dtype=torch.bfloat16, device="cuda")
    o2 = wide[..., :d].transpose(1, 2)
    csp.chunk_attn_q4_paged(p, qkv[:, :, 2:6].transpose(1, 2), a, b, table, rows.cuda(), o2, ws)        # (without counts of new tokens)
    assert csp.device_status(ws) == 0 and torch.equal(o2, out) and (wide[..., d:] == 3.0).all()


def test_offsets_past_32_bits(csp):
    """Pools of more than 2^32 bytes of codes, the sequence on their last pages."""
    H, d, R = 8, 128, 128
    n_pages = 2 ** 32 // (H * R * d // 2) + 40
    rows = torch.full((1, H), 300, dtype=torch.int32)
    gen = torch.Generator().manual_seed(3)
    table = torch.tensor([[n_pages - 1, 0, n_pages - 3]], dtype=torch.int32, device="cuda")
    dense, caches = [], []
    for _ in range(2):
        codes, scales = random_rows((1, H, 384, d), gen)
        c = csp.Q4Cache(torch.empty(n_pages, H, R, d // 2, dtype=torch.uint8, device="cuda"), torch.empty(n_pages, H, R, 2, dtype=torch.bfloat16, device="cuda"))
        for i in range(3):
            c.codes[int(table[0, i])] = codes[0, :, 128 * i:128 * i + 128].cuda()
            c.scales[int(table[0, i])] = scales[0, :, 128 * i:128 * i + 128].cuda()
        dense.append((codes, scales))
        caches.append(c)
    p = csp.Params(1, H, H, d, 1, 0, 300, 300)
    for T in (1, 20, 60):
        q = torch.randn(1, H, T, d, generator=gen).to(torch.bfloat16).cuda()
        out, ws = torch.zeros_like(q), csp.new_chunk_q4_workspace(p, T)
        csp.chunk_attn_q4_paged(p, q, *caches, table, rows.cuda(), out, ws)
        assert csp.device_status(ws) == 0
        check(out, None, q, dense, rows, torch.tensor([T]))
    # rows are appended there, and read back
    k, v = (torch.randn(1, H, 7, d, generator=gen).to(torch.bfloat16).cuda() for _ in range(2))
    p = csp.Params(1, H, H, d, 1, 0, 384, 384)
    at, ws = rows.cuda(), csp.new_append_workspace(p)
    csp.append_q4_paged(p, k, v, *caches, table, at, at, ws)
    back = [torch.zeros(1, H, 20, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    csp.load_q4_paged(p, *caches, table, at, *back, ws, first=torch.full((1, H), 298, dtype=torch.int32, device="cuda"))
    assert csp.device_status(ws) == 0 and (at == 307).all()
    for x, got, c, (codes, scales) in zip((k, v), back, caches, dense):
        assert torch.equal(got[:, :, :2].cpu(), values(codes, scales)[:, :, 298:300].float().to(torch.bfloat16))
        step = c.scales[n_pages - 3, :, 44:51, 0].double()
        assert ((got[0, :, 2:9].double() - x[0].double()).abs().amax(-1) <= step * (0.5 + 16 * 2.0 ** -8) + 2.0 ** -8 * 8).all()


SHAPES = [(2, 2, 2, 6000), (1, 3, 4, 2500), (40, 1, 2, 6000), (20, 4, 80, 250), (30, 4, 80, 250), (5, 2, 4, 890)]


@pytest.mark.parametrize("T,B,H,cap", SHAPES)
def test_captured_calls_replay_on_new_inputs(csp, T, B, H, cap):
    """Cut items and their joining, few rows and many, and items drawn from a counter: replays, and calls on a workspace that others
    have used, give the same bits."""
    doc = (torch.arange(cap, dtype=torch.int32) * 4 // cap)[None, :].expand(B, cap).contiguous()
    both = []
    for i in range(2):
        rows = torch.full((B, H), cap - 7 * i, dtype=torch.int32)
        dense, pools, table = paged_cache(rows, cap, H, 64, 128, 60 + i)
        q = torch.randn(B, 2 * H, T, 64, generator=torch.Generator().manual_seed(i)).to(torch.bfloat16)
        both.append((dense, [pools[0][0], pools[0][1], pools[1][0], pools[1][1], table, rows.cuda(), q.cuda()]))
    p = csp.Params(B, 2 * H, H, 64, 1, 0, cap, cap)
    dev = [x.clone() for x in both[0][1]]
    ws, out = csp.new_chunk_q4_workspace(p, T), torch.zeros(B, 2 * H, T, 64, dtype=torch.bfloat16, device="cuda")
    for mods in (csp.ScoreMods(documents=doc.cuda()), None):
        def call():
            csp.chunk_attn_q4_paged(p, dev[6], csp.Q4Cache(dev[0], dev[1]), csp.Q4Cache(dev[2], dev[3]), dev[4], dev[5], out, ws, mods=mods)
        call()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        for dense, src in both[::-1]:
            for x, y in zip(dev, src):
                x.copy_(y)
            seen = []
            for _ in range(2):
                out.zero_()
                graph.replay()
                seen.append(out.clone())
            call()
            assert csp.device_status(ws) == 0 and int(ws[:256].sum()) == 0
            assert torch.equal(seen[0], out) and torch.equal(seen[1], out)
            one = [tuple(x[:1, :1] for x in pair) for pair in dense]
            check(out[:1, :2], None, dev[6][:1, :2], one, dev[5][:1, :1].cpu(), torch.tensor([T]), **({"documents": doc[:1]} if mods else {}))


def test_two_streams_at_once(csp):
    """Calls on two streams with a workspace each, while the default stream does something else."""
    for T in (1, 30):
        work = []
        for i in range(2):
            rows = torch.tensor([[1200 - 100 * i, 900], [77, 1100]], dtype=torch.int32)
            dense, pools, table = paged_cache(rows, 1200, 2, 128, 128, 70 + i)
            q = torch.randn(2, 8, T, 128, generator=torch.Generator().manual_seed(i)).to(torch.bfloat16).cuda()
            p = csp.Params(2, 8, 2, 128, 1, 0, 1200, 1200)
            work.append((torch.cuda.Stream(), p, q, csp.Q4Cache(*pools[0]), csp.Q4Cache(*pools[1]), table, rows.cuda(), torch.zeros_like(q),
                         csp.new_chunk_q4_workspace(p, T), dense))
        torch.cuda.synchronize()
        for _ in range(3):
            for st, p, q, K, V, table, rows, out, ws, _ in work:
                with torch.cuda.stream(st):
                    csp.chunk_attn_q4_paged(p, q, K, V, table, rows, out, ws)
        torch.cuda.synchronize()
        for _, p, q, K, V, table, rows, out, ws, dense in work:
            assert csp.device_status(ws) == 0
            check(out, None, q, dense, rows.cpu(), torch.tensor([T, T]))


def test_one_workspace_for_chunks_of_all_lengths(csp):
    """Made for the longest chunk, used for that one, for the lengths around a change of kernel and for single tokens."""
    for G, H, longest in ((7, 2, 5), (1, 3, 40), (8, 2, 300), (3, 2, 20)):
        rows = torch.tensor([[1500 - 3 * h for h in range(H)]], dtype=torch.int32)
        dense, pools, table = paged_cache(rows, 1500, H, 128, 128, G)
        p = csp.Params(1, G * H, H, 128, 1, 0, 1500, 1500)
        ws = csp.new_chunk_q4_workspace(p, longest)
        for T in sorted({longest, 1, 2, min(longest, 4), min(longest, 6), min(longest, 17), min(longest, 33)}, reverse=True):
            q = torch.randn(1, G * H, T, 128, generator=torch.Generator().manual_seed(T)).to(torch.bfloat16).cuda()
            out = torch.zeros_like(q)
            csp.chunk_attn_q4_paged(p, q, csp.Q4Cache(*pools[0]), csp.Q4Cache(*pools[1]), table, rows.cuda(), out, ws)
            assert csp.device_status(ws) == 0
            check(out, None, q, dense, rows, torch.tensor([T]), what=f"T={T}")


@pytest.mark.parametrize("B,T", [(2, 0), (0, 3), (0, 0)])
def test_nothing_to_do(csp, B, T):
    p = csp.Params(B, 4, 2, 64, 1, 0, 256, 256)
    q = torch.zeros(B, 4, T, 64, dtype=torch.bfloat16, device="cuda")
    K, V = csp.new_q4_cache(5, 2, 128, 64), csp.new_q4_cache(5, 2, 128, 64)
    rows, new = torch.full((B, 2), 7, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    table = torch.zeros(B, 2, dtype=torch.int32, device="cuda")
    ws = csp.new_chunk_q4_workspace(p, T)
    csp.chunk_attn_q4_paged(p, q, K, V, table, rows, torch.zeros_like(q), ws, n_new=new, mods=csp.ScoreMods(prefix=new), lse=torch.zeros(B, 4, T, device="cuda"))
    assert csp.device_status(ws) == 0
    x = torch.zeros(B, 2, T, 64, dtype=torch.bfloat16, device="cuda")
    after, aws = torch.zeros_like(rows), csp.new_append_workspace(p)
    csp.append_q4_paged(p, x, x, K, V, table, rows, after, aws)
    csp.load_q4_paged(p, K, V, table, torch.full_like(rows, T), x, x.clone(), aws)
    assert csp.device_status(aws) == 0 and torch.equal(after, rows + T)


def test_tensors_on_another_device_are_refused(csp):
    p, q, K, V, table, rows, out, z, ws = _case(csp, [[100, 90]], [3], d=64)
    good = dict(q=q, K=K, V=V, table=table, rows=rows.cuda(), out=out, ws=ws)

    def call(**kw):
        a = dict(good, **kw)
        csp.chunk_attn_q4_paged(p, a["q"], a["K"], a["V"], a["table"], a["rows"], a["out"], a["ws"], **{k: a[k] for k in ("n_new", "lse", "mods") if k in a})
    half = csp.Q4Cache(K.codes, K.scales.cpu())
    for kw in (dict(q=q.cpu()), dict(K=half), dict(V=half), dict(table=table.cpu()), dict(rows=rows), dict(out=out.cpu()), dict(ws=ws.cpu()),
               dict(n_new=torch.tensor([3], dtype=torch.int32)), dict(lse=z.cpu()), dict(mods=csp.ScoreMods(slopes=torch.ones(2)))):
        with pytest.raises(ValueError):
            call(**kw)
    call()


def test_random_launches(csp):
    """Seeded shapes over the whole range."""
    import numpy as np
    rng = np.random.RandomState(78)
    for trial in range(24):
        d, H, G, B = int(rng.choice([64, 128])), int(rng.choice([1, 2, 3])), int(rng.randint(1, 9)), int(rng.randint(1, 4))
        cap = int(rng.randint(1, 900))
        rows = rng.randint(0, cap + 1, size=(B, H))
        T = int(rng.choice([1, 2, 8, 40, 130]))
        new = [int(rng.randint(0, min(T, int(r.min())) + 1)) for r in rows]

        def mods(B, H, G, cap):
            m = {}
            if rng.rand() < 0.4:
                m["softcap"] = float(rng.uniform(2, 60))
            if rng.rand() < 0.4:
                m["slopes"] = torch.exp2(-torch.arange(1, H * G + 1).float())
                if rng.rand() < 0.5:
                    m["positions"] = torch.from_numpy(np.cumsum(rng.randint(1, 5, size=(B, H, cap)), 2).astype(np.int32))
            if rng.rand() < 0.4:
                m["documents"] = torch.from_numpy(np.sort(rng.randint(0, 4, size=(B, cap)), 1).astype(np.int32))
            if rng.rand() < 0.4:
                m["prefix"] = torch.from_numpy(rng.randint(0, cap + 1, size=(B, H)).astype(np.int32))
            return m
        _case(csp, rows.tolist(), new, G=G, d=d, page_rows=int(rng.choice([128, 256])), n=float(rng.choice([0.0, 1.0])), seed=trial, cap=cap,
              q_gain=float(rng.choice([0.5, 1.5, 4.0])), mods=mods)


def test_a_querys_sum_keeps_32_bits(csp):
    """Keys that are all -8 (scale 0): every logit is -8 scale sum q, all weights are one, and the log-sum-exp shows what the sum is off
    by.  Twelve roundings of partial sums at most (the scaling is exact), each by 2^-24 of what has the size |q| for random signs; the
    logarithm and the last steps 2^-22 (1 + |lse|)."""
    for T in (1, 3, 60):
        rows = torch.full((4, 4), 512, dtype=torch.int32)
        _, pools, table = paged_cache(rows, 512, 4, 128, 128, 31)
        pools[0][1][..., 0], pools[0][1][..., 1] = 0, -8
        q = torch.randn(4, 16, T, 128, generator=torch.Generator().manual_seed(T)).to(torch.bfloat16)
        p = csp.Params(4, 16, 4, 128, 1, 0, 512, 512)
        out, z, ws = torch.zeros_like(q).cuda(), torch.zeros(4, 16, T, device="cuda"), csp.new_chunk_q4_workspace(p, T)
        csp.chunk_attn_q4_paged(p, q.cuda(), csp.Q4Cache(*pools[0]), csp.Q4Cache(*pools[1]), table, rows.cuda(), out, ws, lse=z)
        sc = 128 ** -0.5
        want = -8 * sc * q.double().sum(-1) + (512 - T + 1 + torch.arange(T)).double().log()
        rms = (z.cpu().double() - want).square().mean().sqrt()
        size = q.double().norm(dim=-1).square().mean().sqrt()
        assert rms <= 12 * 2.0 ** -24 * 8 * sc * size + 2.0 ** -22 * (1 + want.square().mean().sqrt()), (T, float(rms))


# ---- together

@pytest.mark.parametrize("interleaved", [False, True])
def test_a_serving_round(csp, interleaved):
    """Two prompts enter in chunks, rotated and in 4 bits (reserve, append, attention), each is forked, the forks decode a few tokens
    (pages are copied on write), all are pruned: read back as numbers, scored and compacted, and the rows that stay go back to other
    pages in 4 bits.  Decoding goes on with positions that are no row numbers any more.  At every step the rows read back are
    what the pages say, and the attention equals the definition on them."""
    import numpy as np
    from test_gpu_pages import Pages
    torch.manual_seed(0)
    B, Hq, H, d, R, mp, n_pages = 4, 6, 2, 64, 128, 6, 60
    cap = mp * R
    x = Pages(csp, B, H, mp, R, n_pages)
    p = csp.Params(B, Hq, H, d, 1, 0, cap, cap)
    K, V = csp.new_q4_cache(n_pages, H, R, d), csp.new_q4_cache(n_pages, H, R, d)
    for c in (K, V):
        c.codes.fill_(0xa5)
        c.scales.fill_(float("nan"))
    angle = torch.arange(2000)[:, None] * torch.exp2(-torch.arange(d // 2) / 4.0)
    rope_table = torch.cat([angle.cos(), angle.sin()], 1).cuda()
    aws, cws = csp.new_append_workspace(p), csp.new_chunk_q4_workspace(p, 150)
    seen = [0] * B                                       # tokens so far: positions
    rows_before = None

    def step(new):
        nonlocal rows_before
        T = max(max(new), 1)
        n = torch.tensor(new, dtype=torch.int32, device="cuda")
        before = x.m.rows.copy()
        x.reserve(new)
        csp.pages_copy_q4(p, K, V, x.moves, x.n, aws)
        pos = torch.tensor([[seen[b] + i for i in range(T)] for b in range(B)], dtype=torch.int32, device="cuda")
        rope = csp.Rope(rope_table, positions=pos, interleaved=interleaved)
        kn, vn, q = (torch.randn(B, T, h, d, device="cuda").to(torch.bfloat16).transpose(1, 2) for h in (H, H, Hq))
        out, lse = torch.zeros_like(q), torch.zeros(B, Hq, T, device="cuda")
        csp.append_q4_paged(p, kn, vn, K, V, x.s.page_table, x.s.n_rows, x.s.n_rows, aws, n_new=n, rope=rope, q=q, q_out=q)
        x.m.rows += np.asarray(new, np.int32)[:, None]
        csp.chunk_attn_q4_paged(p, q, K, V, x.s.page_table, x.s.n_rows, out, cws, n_new=n, lse=lse)
        k_back, v_back = (torch.zeros(B, H, cap, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        csp.load_q4_paged(p, K, V, x.s.page_table, x.s.n_rows, k_back, v_back, aws)
        x.same()
        assert csp.device_status(aws) == 0 and csp.device_status(cws) == 0
        rows = torch.from_numpy(x.m.rows.astype(np.int32))
        dense, table = [], x.s.page_table.cpu().long().clamp(0, n_pages - 1)
        for c, back in ((K, k_back), (V, v_back)):
            codes, scales = (y.cpu()[table].transpose(1, 2).flatten(2, 3).contiguous() for y in (c.codes, c.scales))
            for b in range(B):
                for h in range(H):
                    scales[b, h, int(rows[b, h]):] = 0
                    codes[b, h, int(rows[b, h]):] = 0
            assert torch.equal(back.cpu(), values(codes, scales).float().to(torch.bfloat16))
            dense.append((codes, scales))
        # what was there is there, new values are near what was brought
        if rows_before is not None:
            for b in range(B):
                for h in range(H):
                    L = int(before[b, h])
                    assert torch.equal(k_back[b, h, :L], rows_before[0][b, h, :L]) and torch.equal(v_back[b, h, :L], rows_before[1][b, h, :L])
        for b in range(B):
            for h in range(H):
                L, N = int(rows[b, h]), new[b]
                far = (v_back[b, h, L - N:L].double() - vn[b, h, :N].double()).abs()
                assert (far.cpu() <= dense[1][1][b, h, L - N:L, :1].double() * 0.6 + 2.0 ** -8 * 8).all()
            seen[b] += new[b]
        rows_before = (k_back, v_back)
        check(out, lse, q, dense, rows, torch.tensor(new))

    step([150, 100, 0, 0])
    step([150, 28, 0, 0])
    x.fork([0, 1], [2, 3])
    for y in rows_before:
        y[2], y[3] = y[0], y[1]
    seen[2], seen[3] = seen[0], seen[1]
    step([1, 1, 1, 1])
    step([2, 0, 1, 3])
    # the prune: numbers again, the rows that stay to pages of their own
    pp = csp.Params(B, Hq, H, d, 32, 32, cap, cap)
    mod = torch.zeros(B, cap, dtype=torch.uint8, device="cuda")
    bud = torch.tensor([[40, 0, 0, 0], [20, 0, 0, 0], [60, 0, 0, 0], [10, 0, 0, 0]], dtype=torch.int32, device="cuda")
    k_out, v_out = (torch.zeros(B, H, cap, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    mod_out, n_out = torch.zeros(B, H, cap, dtype=torch.uint8, device="cuda"), torch.zeros(B, H, dtype=torch.int32, device="cuda")
    qw, pws = torch.randn(B, Hq, 32, d, device="cuda").to(torch.bfloat16), csp.new_workspace(pp)
    csp.prune_layer(pp, qw, *rows_before, mod, x.s.n_rows[:, 0].contiguous(), bud, k_out, v_out, mod_out, n_out, pws)
    assert csp.device_status(pws) == 0
    x.set_rows(np.zeros((B, H), np.int32))
    x.free()
    kept = n_out.cpu().numpy()
    x.reserve([int(r.max()) for r in kept])
    csp.append_q4_paged(p, k_out, v_out, K, V, x.s.page_table, x.s.n_rows, x.s.n_rows, aws, n_new=n_out)
    assert csp.device_status(aws) == 0 and torch.equal(x.s.n_rows, n_out)
    x.set_rows(kept)
    rows_before = None
    step([1, 1, 1, 1])
    step([130, 1, 0, 60])
