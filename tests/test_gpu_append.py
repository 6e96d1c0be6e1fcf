"""Appending rows with the rotation on the way, appending to pages in 4 bits, reading 4-bit rows back."""
import math

import pytest
import torch

from q4_util import quantise, values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def csp():
    from paper_2412_04652_b200 import binding
    binding.lib()
    return binding


def _table(rope_dim, n, seed=0):
    gen = torch.Generator().manual_seed(seed)
    freq = torch.exp2(-torch.rand(rope_dim // 2, generator=gen, dtype=torch.float64) * 12)
    a = torch.arange(n, dtype=torch.float64)[:, None] * freq
    return torch.cat([a.cos(), a.sin()], 1).float()


def _rotated(x, cos_sin, pos, interleaved):
    """x [..., T, d] (any type), pos [..., T] -> in 64 bits, and the magnitudes that were added up."""
    r = cos_sin.shape[1]
    c, s = cos_sin.double()[pos.long()].chunk(2, -1)
    y, m = x.double().clone(), x.double().abs()
    one, two = (slice(0, r, 2), slice(1, r, 2)) if interleaved else (slice(0, r // 2), slice(r // 2, r))
    a, b = x.double()[..., one], x.double()[..., two]
    y[..., one], y[..., two] = a * c - b * s, b * c + a * s
    m[..., one], m[..., two] = (a * c).abs() + (b * s).abs(), (b * c).abs() + (a * s).abs()
    return y, m


def _close(got, want, mag, dtype):
    """Two products and a sum, each off by 2^-24 of what it yields (3 2^-24 of the magnitudes covers them), then one rounding to
    the type; the smallest normal number for what is flushed."""
    half = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    tol = 3 * 2.0 ** -24 * mag * (1 + half) + half * want.abs() + 2.0 ** -126
    bad = (got.double() - want).abs() > tol
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} off, first at {bad.nonzero()[0].tolist()}"


def _setup(csp, first, new, H, G, d, dtype, page_rows=128, per_head=False, seed=1, cap=None):
    B = len(first)
    first = torch.tensor(first, dtype=torch.int32)
    new_t = torch.tensor(new, dtype=torch.int32)
    T = max(int(new_t.max()), 1) + 2                     # more slots than any sequence brings
    per = new_t if per_head else new_t[:, None].expand(B, H)
    rows = first + per
    cap = cap or int(rows.max())
    mp = -(-cap // page_rows)
    gen = torch.Generator().manual_seed(seed)
    table = torch.randperm(B * mp + 2, generator=gen)[:B * mp].reshape(B, mp).to(torch.int32)
    x = [torch.randn(B, T, h, d, generator=gen).to(dtype).transpose(1, 2) for h in (H, H, H * G)]
    p = csp.Params(B, H * G, H, d, 1, 0, cap, cap, dtype=csp.F32 if dtype == torch.float32 else csp.BF16)
    return p, first, new_t, per, table, x, B * mp + 2


def _where(table, b, t, page_rows):
    return table[b].long()[t // page_rows], t % page_rows


@pytest.mark.parametrize("dtype,d,rope", [(torch.bfloat16, 64, 64), (torch.bfloat16, 128, 128), (torch.bfloat16, 128, 48), (torch.bfloat16, 256, 256),
                                          (torch.bfloat16, 256, 16), (torch.float32, 32, 16), (torch.float32, 64, 64), (torch.float32, 128, 96)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("new", [[1, 1, 1], [3, 0, 9], [140, 33, 7]])
def test_rotated_append(csp, dtype, d, rope, interleaved, new):
    H, G, R = 3, 2, 128
    first = [[5, 5, 5], [0, 127, 126], [300, 301, 255]]
    p, first, new_t, per, table, (k, v, q), n_pages = _setup(csp, first, new, H, G, d, dtype)
    T = k.shape[2]
    use_positions = new[0] != 3
    pos = torch.randint(0, 900, (3, T), generator=torch.Generator().manual_seed(3), dtype=torch.int32)
    cs = _table(rope, 1000)
    pools = [torch.full((n_pages, H, R, d), 9.0, dtype=dtype) for _ in range(2)]
    kp, vp = (x.cuda() for x in pools)
    qd, q_out = q.cuda(), torch.full((3, H * G, T, d), 9.0, dtype=dtype, device="cuda")
    counts = first.cuda()
    ws = csp.new_append_workspace(p)
    r = csp.Rope(cs.cuda(), positions=pos.cuda() if use_positions else None, interleaved=interleaved)
    csp.append_rope_paged(p, k.cuda(), v.cuda(), kp, vp, table.cuda(), counts, counts, ws, r, n_new=new_t.cuda(), q=qd, q_out=q_out)
    assert csp.device_status(ws) == 0
    assert torch.equal(counts.cpu(), first + per)
    i = torch.arange(T)
    at = pos[:, None].expand(3, H, T) if use_positions else (first[:, :, None] + i).clamp(max=999)
    want, mag = _rotated(k, cs, at, interleaved)
    left_k, left_v = kp.cpu(), vp.cpu()
    for b in range(3):
        for h in range(H):
            n = int(per[b, h])
            page, slot = _where(table, b, first[b, h] + torch.arange(n), R)
            _close(left_k[page, h, slot], want[b, h, :n], mag[b, h, :n], dtype)
            assert torch.equal(left_v[page, h, slot], v[b, h, :n])
            left_k[page, h, slot], left_v[page, h, slot] = 9.0, 9.0
    assert torch.equal(left_k, pools[0]) and torch.equal(left_v, pools[1])          # nothing else was written
    want, mag = _rotated(q, cs, at.repeat_interleave(G, 1), interleaved)
    for b in range(3):
        n = new[b]
        _close(q_out[b, :, :n].cpu(), want[b, :, :n], mag[b, :, :n], dtype)
        assert (q_out[b, :, n:] == 9.0).all()
    # queries in place, from tensors of the other layout
    ws2 = csp.new_append_workspace(p)
    again, after = first.cuda(), torch.zeros_like(first).cuda()
    csp.append_rope_paged(p, k.contiguous().cuda(), v.contiguous().cuda(), kp, vp, table.cuda(), again, after, ws2, r, n_new=new_t.cuda(), q=qd, q_out=qd)
    for b in range(3):
        assert torch.equal(qd[b, :, :new[b]], q_out[b, :, :new[b]]) and torch.equal(qd[b, :, new[b]:].cpu(), q[b, :, new[b]:])
    assert torch.equal(after.cpu(), first + per) and torch.equal(again.cpu(), first)


def _codes(pool, page, h, slot):
    c, s = pool.codes.cpu()[page, h, slot], pool.scales.cpu()[page, h, slot]
    return torch.stack([c & 15, c >> 4], -1).flatten(-2).double(), s[..., 0].double(), s[..., 1].double()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("per_head", [False, True])
@pytest.mark.parametrize("rope", [0, 1])
def test_append_in_4_bits(csp, d, per_head, rope):
    H, G, R = 3, 2, 128
    first = [[5, 5, 5], [0, 127, 126], [300, 301, 255]]
    new = [[3, 0, 140], [1, 9, 2], [33, 7, 8]] if per_head else [140, 1, 33]
    p, first, new_t, per, table, (k, v, q), n_pages = _setup(csp, first, new, H, G, d, torch.bfloat16, per_head=per_head, seed=d)
    T = k.shape[2]
    v[:, :, 0] = 2.5                                     # a constant row
    v[:, :, 1, 3] = 1000.0                               # one far out
    K, V = csp.new_q4_cache(n_pages, H, R, d), csp.new_q4_cache(n_pages, H, R, d)
    K.codes.fill_(0x5a), V.codes.fill_(0x5a)
    after = torch.zeros_like(first).cuda()
    ws = csp.new_append_workspace(p)
    kw = {}
    rotated = k
    if rope:
        cs = _table(d, 600)
        r = csp.Rope(cs.cuda(), interleaved=per_head)
        q_out = torch.zeros(3, H * G, T, d, dtype=torch.bfloat16, device="cuda")
        kw = dict(rope=r, q=q.cuda(), q_out=q_out)
        # the rotated row as a bf16 cache holds it
        kp, vp = (torch.zeros(n_pages, H, R, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        q2 = torch.zeros_like(q_out)
        csp.append_rope_paged(p, k.cuda(), v.cuda(), kp, vp, table.cuda(), first.cuda(), after, ws, r, n_new=new_t.cuda(), q=kw["q"], q_out=q2)
        rotated = torch.zeros(3, H, T, d, dtype=torch.bfloat16)
        for b in range(3):
            for h in range(H):
                n = int(per[b, h])
                page, slot = _where(table, b, first[b, h] + torch.arange(n), R)
                rotated[b, h, :n] = kp.cpu()[page, h, slot]
    csp.append_q4_paged(p, k.cuda(), v.cuda(), K, V, table.cuda(), first.cuda(), after, ws, n_new=new_t.cuda(), **kw)
    assert csp.device_status(ws) == 0
    assert torch.equal(after.cpu(), first + per)
    if rope:
        assert torch.equal(q_out, q2)
    k_out, v_out = (torch.full((3, H, T, d), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    csp.load_q4_paged(p, K, V, table.cuda(), after, k_out, v_out, ws, first=first.cuda())
    assert csp.device_status(ws) == 0
    touched = torch.zeros(n_pages, H, R, dtype=torch.bool)
    for x, pool, back in ((rotated, K, k_out), (v, V, v_out)):
        for b in range(3):
            for h in range(H):
                n = int(per[b, h])
                page, slot = _where(table, b, first[b, h] + torch.arange(n), R)
                touched[page, h, slot] = True
                code, scale, base = _codes(pool, page, h, slot)
                want_code, want_scale, want_base, off = quantise(x[b, h, :n])
                assert torch.equal(scale, want_scale) and torch.equal(base, want_base)
                sure = (off > 2.0 ** -20) | (off == 0)   # exactly in the middle: the upper one
                if n:
                    assert torch.equal(code[sure], want_code[sure]) and float((code - want_code).abs().max()) <= 1
                    exact = base[:, None] + scale[:, None] * code
                    # within half a step (and what rounding the step to bf16 takes at the upper end: 15 steps of 2^-8)
                    assert ((exact - x[b, h, :n].double()).abs() <= scale[:, None] * (0.5 + 15 * 2.0 ** -8) + 2.0 ** -126).all()
                    assert torch.equal(back[b, h, :n].cpu(), exact.float().to(torch.bfloat16))
                assert (back[b, h, n:] == 9.0).all()
    assert (K.codes.cpu()[~touched] == 0x5a).all() and (V.codes.cpu()[~touched] == 0x5a).all()
    assert (K.scales.cpu()[~touched] == 0).all() and (V.scales.cpu()[~touched] == 0).all()


@pytest.mark.parametrize("d", [64, 128])
def test_rows_out_of_the_ordinary(csp, d):
    """Infinities, NaN, spreads that are no number or almost nothing."""
    x = torch.randn(1, 1, 10, d).to(torch.bfloat16)
    x[0, 0, 0, 7] = float("inf")
    x[0, 0, 1, 3] = float("-inf")
    x[0, 0, 2, d - 1] = float("nan")
    x[0, 0, 3, 0], x[0, 0, 3, 1] = 3.3e38, -3.3e38
    x[0, 0, 4] = 0.0
    x[0, 0, 5] = float("inf")
    x[0, 0, 6] = -1.5
    x[0, 0, 7] *= 1e-38                                  # the step is no normal number: the row reads as its smallest value
    x[0, 0, 8] *= 1e36
    x[0, 0, 9, 1:] = -7.0
    p = csp.Params(1, 1, 1, d, 1, 0, 128, 128)
    K, V = csp.new_q4_cache(1, 1, 128, d), csp.new_q4_cache(1, 1, 128, d)
    table = torch.zeros(1, 1, dtype=torch.int32, device="cuda")
    rows = torch.zeros(1, 1, dtype=torch.int32, device="cuda")
    ws = csp.new_append_workspace(p)
    csp.append_q4_paged(p, x.cuda(), x.cuda(), K, V, table, rows, rows, ws)
    back = torch.zeros(1, 1, 10, d, dtype=torch.bfloat16, device="cuda")
    csp.load_q4_paged(p, K, None, table, rows, back, None, ws)
    assert csp.device_status(ws) == 0 and int(rows) == 10
    got = back[0, 0].cpu()
    for i in (0, 1, 2, 3, 5):
        assert torch.isnan(got[i]).all(), i
    assert (got[4] == 0).all() and (got[6] == -1.5).all()
    assert (got[7] == x[0, 0, 7].amin()).all()
    for i in (8, 9):
        code, scale, base, _ = quantise(x[0, 0, i])
        assert torch.equal(got[i], (base + scale * code).float().to(torch.bfloat16))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("with_v", [True, False])
def test_read_back(csp, dtype, d, with_v):
    B, H, R, cap = 3, 2, 256, 700
    gen = torch.Generator().manual_seed(d)
    mp, n_pages = 3, 12
    pools = []
    for _ in range(2):
        codes = torch.randint(0, 256, (n_pages, H, R, d // 2), generator=gen, dtype=torch.uint8)
        scales = torch.randn(n_pages, H, R, 2, generator=gen).to(torch.bfloat16)
        pools.append((codes, scales))
    table = torch.randperm(n_pages, generator=gen)[:B * mp].reshape(B, mp).to(torch.int32)
    table[1, 1] = 99                                     # no page
    rows = torch.tensor([[700, 0], [513, 300], [256, 5]], dtype=torch.int32)
    first = torch.tensor([[0, 0], [200, 299], [256, 4]], dtype=torch.int32)
    p = csp.Params(B, H, H, d, 1, 0, cap, cap, dtype=csp.F32 if dtype == torch.float32 else csp.BF16)
    outs = [torch.full((B, cap, H, d), 9.0, dtype=dtype, device="cuda").transpose(1, 2) for _ in range(2)]
    ws = csp.new_append_workspace(p)
    K, V = (csp.Q4Cache(c.cuda(), s.cuda()) for c, s in pools)
    csp.load_q4_paged(p, K, V if with_v else None, table.cuda(), rows.cuda(), outs[0], outs[1] if with_v else None, ws, first=first.cuda())
    assert csp.device_status(ws) == csp.DEV_BAD_LEN      # the page that is none
    for which in range(2 if with_v else 1):
        full = values(*pools[which]).float().to(dtype)
        for b in range(B):
            for h in range(H):
                n = int(rows[b, h]) - int(first[b, h])
                got = outs[which][b, h].cpu()
                assert (got[n:] == 9.0).all()
                t = int(first[b, h]) + torch.arange(n)
                page = table[b].long()[t // R]
                want = full[page.clamp(max=n_pages - 1), h, t % R]
                want[page >= n_pages] = 0
                assert torch.equal(got[:n], want), (b, h)


def test_flags(csp):
    """Rows that do not fit, counts and positions that are none, pages outside the pool: flagged, nothing is written astray."""
    d, H = 64, 2
    k = torch.randn(2, H, 4, d).to(torch.bfloat16).cuda()
    cs = _table(d, 10).cuda()

    def call(first, new, table, pos=None, cap=256):
        p = csp.Params(2, H, H, d, 1, 0, cap, cap)
        K, V = csp.new_q4_cache(4, H, 128, d), csp.new_q4_cache(4, H, 128, d)
        rows = torch.tensor(first, dtype=torch.int32, device="cuda")
        pos = None if pos is None else torch.tensor(pos, dtype=torch.int32, device="cuda")
        ws = csp.new_append_workspace(p)
        csp.append_q4_paged(p, k, k, K, V, torch.tensor(table, dtype=torch.int32, device="cuda"), rows, rows, ws, rope=csp.Rope(cs, positions=pos),
                            n_new=None if new is None else torch.tensor(new, dtype=torch.int32, device="cuda"))
        status = csp.device_status(ws)
        assert int(ws[:256].sum()) == 0                  # counters are left at zero
        return status, rows.cpu().tolist(), int((K.scales != 0).any(-1).sum())

    ok = [[0, 1], [2, 3]]
    assert call([[0, 1], [2, 3]], None, ok) == (0, [[4, 5], [6, 7]], 16)
    assert call([[0, 1], [2, 253]], None, ok, pos=[[0, 1, 2, 3]] * 2) == (csp.DEV_CAPACITY, [[4, 5], [6, 253]], 12)
    assert call([[0, 1], [2, -3]], None, ok, pos=[[0, 1, 2, 3]] * 2) == (csp.DEV_BAD_LEN, [[4, 5], [6, -3]], 12)
    assert call([[0, 1], [2, 3]], [5, -1], ok) == (csp.DEV_BAD_LEN, [[4, 5], [2, 3]], 8)
    assert call([[0, 1], [2, 3]], None, [[0, 1], [4, 3]]) == (csp.DEV_BAD_LEN, [[4, 5], [6, 7]], 8)
    assert call([[0, 1], [2, 3]], None, [[0, 1], [-1, 3]]) == (csp.DEV_BAD_LEN, [[4, 5], [6, 7]], 8)
    assert call([[0, 1], [2, 3]], None, ok, pos=[[0, 1, 10, 3], [0, 1, 2, -5]]) == (csp.DEV_BAD_LEN, [[4, 5], [6, 7]], 16)
    assert call([[0, 1], [2, 3]], [0, 0], ok) == (0, [[0, 1], [2, 3]], 0)


@pytest.mark.parametrize("H,G", [(1, 1), (3, 1), (1, 7), (5, 3), (2, 8), (8, 5)])
@pytest.mark.parametrize("T", [1, 6, 70])
@pytest.mark.parametrize("four", [False, True])
def test_heads_of_all_counts(csp, H, G, T, four):
    """Odd numbers of query heads, more heads than a block has groups of lanes for, a batch of several sequences."""
    B, d, R = 5, 64, 128
    p, first, new, per, table, (k, v, q), n_pages = _setup(csp, [[3 + 40 * b] * H for b in range(B)], [T, max(T - 1, 0), T, 0, 1], H, G, d, torch.bfloat16, seed=H + G + T)
    cs = _table(48, 400)
    slots = k.shape[2]
    q_out = torch.full((B, H * G, slots, d), 9.0, dtype=torch.bfloat16, device="cuda")
    K, V = (csp.new_q4_cache(n_pages, H, R, d) if four else torch.zeros(n_pages, H, R, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    rows, ws = first.cuda(), csp.new_append_workspace(p)
    call = csp.append_q4_paged if four else csp.append_rope_paged
    call(p, k.cuda(), v.cuda(), K, V, table.cuda(), rows, rows, ws, rope=csp.Rope(cs.cuda(), interleaved=bool(G % 2)), n_new=new.cuda(), q=q.cuda(), q_out=q_out)
    assert csp.device_status(ws) == 0 and torch.equal(rows.cpu(), first + per)
    at = first[:, :1, None] + torch.arange(slots)
    for x, got_all, heads in ((q, q_out.cpu(), H * G), (k, None, H)):
        want, mag = _rotated(x, cs, at.expand(B, heads, slots).clamp(max=399), bool(G % 2))
        for b in range(B):
            n = int(new[b])
            if got_all is not None:
                _close(got_all[b, :, :n], want[b, :, :n], mag[b, :, :n], torch.bfloat16)
                assert (got_all[b, :, n:] == 9.0).all()
            elif n:
                page, slot = _where(table, b, first[b, 0] + torch.arange(n), R)
                if four:
                    c, s = K.codes.cpu()[page, :, slot], K.scales.cpu()[page, :, slot]
                    step = s[..., :1].double().transpose(0, 1)
                    # half a step, fifteen roundings of the step, and the rotated row's rounding to bf16 (the largest value's)
                    slack = step * (0.5 + 15 * 2.0 ** -8) + 2.0 ** -7 * mag[b, :, :n].amax(-1, keepdim=True)
                    assert ((values(c, s).transpose(0, 1) - want[b, :, :n]).abs() <= slack).all()
                else:
                    _close(K.cpu()[page, :, slot].transpose(0, 1), want[b, :, :n], mag[b, :, :n], torch.bfloat16)


def test_captured_appends_replay(csp):
    """Two appends in one graph, the counts updated in place: every replay goes on where the last one ended, and lands
    where calls outside of a graph do."""
    B, H, G, d, R = 2, 2, 2, 128, 128
    p = csp.Params(B, H * G, H, d, 1, 0, 512, 512)
    gen = torch.Generator().manual_seed(2)
    k, v, q = (torch.randn(B, h, 40, d, generator=gen).to(torch.bfloat16).cuda() for h in (H, H, H * G))
    table = torch.randperm(8, generator=gen).reshape(B, 4).to(torch.int32).cuda()
    rope = csp.Rope(_table(d, 512).cuda())
    ends = []
    for captured in (False, True):
        K, V = csp.new_q4_cache(8, H, R, d), csp.new_q4_cache(8, H, R, d)
        rows, ws, new = torch.zeros(B, H, dtype=torch.int32, device="cuda"), csp.new_append_workspace(p), torch.tensor([40, 7], dtype=torch.int32, device="cuda")
        q_out = torch.zeros_like(q)

        def two():
            csp.append_q4_paged(p, k, v, K, V, table, rows, rows, ws, n_new=new, rope=rope, q=q, q_out=q_out)
            csp.append_q4_paged(p, v[:, :, :1], k[:, :, :1], K, V, table, rows, rows, ws)
        two()
        if captured:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                two()
            for _ in range(3):
                graph.replay()
        else:
            for _ in range(3):
                two()
        assert csp.device_status(ws) == 0
        assert rows.cpu().tolist() == [[164, 164], [32, 32]]
        ends.append((K.codes, K.scales, V.codes, V.scales, q_out))
    assert all(torch.equal(a, b) for a, b in zip(*ends))


def test_strided_pools_and_another_stream(csp):
    B, H, d, R = 2, 3, 64, 128
    p = csp.Params(B, H, H, d, 1, 0, 256, 256)
    gen = torch.Generator().manual_seed(4)
    k, v = (torch.randn(B, 33, H, d + 8, generator=gen).to(torch.bfloat16).cuda()[..., :d].transpose(1, 2) for _ in range(2))
    table = torch.tensor([[3, 0], [2, 1]], dtype=torch.int32, device="cuda")
    plain = [csp.new_q4_cache(4, H, R, d) for _ in range(2)]
    codes = torch.full((2, H, 5, R * d // 2 + 16), 0x77, dtype=torch.uint8, device="cuda")
    scales = torch.full((2, H, 5, R * 2 + 8), 3.0, dtype=torch.bfloat16, device="cuda")
    gaps = [csp.Q4Cache(codes[i].as_strided((4, H, R, d // 2), (codes.stride(2), codes.stride(1), d // 2, 1), codes[i].storage_offset()),
                        scales[i].as_strided((4, H, R, 2), (scales.stride(2), scales.stride(1), 2, 1), scales[i].storage_offset())) for i in range(2)]
    for c in gaps:
        c.codes.zero_(), c.scales.zero_()
    before = [int((codes == 0x77).sum()), int((scales == 3.0).sum())]
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    outs = []
    for pools in (plain, gaps):
        rows, after, ws = (torch.full((B, H), 111, dtype=torch.int32, device="cuda"), torch.zeros(B, H, dtype=torch.int32, device="cuda"), csp.new_append_workspace(p))
        back = [torch.zeros(B, 40, H, d + 8, dtype=torch.bfloat16, device="cuda")[..., :d].transpose(1, 2) for _ in range(2)]
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            csp.append_q4_paged(p, k, v, *pools, table, rows, after, ws)
            csp.load_q4_paged(p, *pools, table, after, *back, ws, first=rows)
        stream.synchronize()
        assert csp.device_status(ws) == 0 and (after == 144).all()
        outs.append(back)
    for i in range(2):
        assert torch.equal(plain[i].codes, gaps[i].codes) and torch.equal(plain[i].scales, gaps[i].scales) and torch.equal(outs[0][i], outs[1][i])
    gone = sum(int((c.codes == 0x77).sum()) for c in gaps)
    assert int((codes == 0x77).sum()) - gone == before[0] and int((scales == 3.0).sum()) - sum(int((c.scales == 3.0).sum()) for c in gaps) == before[1]


def test_tensors_on_another_device_are_refused(csp):
    B, H, d = 1, 2, 64
    p = csp.Params(B, H, H, d, 1, 0, 128, 128)
    bf = dict(dtype=torch.bfloat16, device="cuda")
    k, pool = torch.zeros(B, H, 3, d, **bf), torch.zeros(1, H, 128, d, **bf)
    K = csp.new_q4_cache(1, H, 128, d)
    rows, table = torch.zeros(B, H, dtype=torch.int32, device="cuda"), torch.zeros(B, 1, dtype=torch.int32, device="cuda")
    ws, cs = csp.new_append_workspace(p), _table(d, 200).cuda()
    pos = torch.zeros(B, 3, dtype=torch.int32)
    half = csp.Q4Cache(K.codes, K.scales.cpu())
    ropes = (csp.Rope(cs.cpu()), csp.Rope(cs, positions=pos))
    good = dict(k=k, v=k, K=K, V=K, rows=rows, out=rows, table=table, ws=ws, rope=csp.Rope(cs), q=k, q_out=k.clone(), n_new=None)

    def call(four, **kw):
        a = dict(good, **kw)
        if not four:
            a["K"] = a["V"] = kw.get("pool", pool)
        f = csp.append_q4_paged if four else csp.append_rope_paged
        f(p, a["k"], a["v"], a["K"], a["V"], a["table"], a["rows"], a["out"], a["ws"], rope=a["rope"], n_new=a["n_new"], q=a["q"], q_out=a["q_out"])
    for four in (True, False):
        for kw in (dict(k=k.cpu()), dict(v=k.cpu()), dict(rows=rows.cpu()), dict(out=rows.cpu()), dict(table=table.cpu()), dict(ws=ws.cpu()),
                   dict(rope=ropes[0]), dict(rope=ropes[1]), dict(q=k.cpu()), dict(q_out=k.cpu()), dict(n_new=torch.zeros(1, dtype=torch.int32)),
                   dict(K=half) if four else dict(pool=pool.cpu())):
            with pytest.raises(ValueError):
                call(four, **kw)
    for kw in (dict(a=half), dict(a=K, rows=rows.cpu()), dict(a=K, first=rows.cpu()), dict(a=K, table=table.cpu()), dict(a=K, out=k.cpu()), dict(a=K, ws=ws.cpu())):
        with pytest.raises(ValueError):
            csp.load_q4_paged(p, kw["a"], None, kw.get("table", table), kw.get("rows", rows), kw.get("out", k), None, kw.get("ws", ws), first=kw.get("first"))
