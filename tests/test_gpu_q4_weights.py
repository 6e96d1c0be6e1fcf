"""What the weights of the 4-bit attention are held by: rows that a query does not see, rows that weigh nearly nothing and rows whose
values are far from the others' do not cost those that it sees their bits."""
import math

import pytest
import torch

from q4_util import random_rows, to_pages, values

pytestmark = pytest.mark.gpu

WIDE = 1 << 18                                           # a capacity for which items of sixteen rows are taken where rows allow it
# query heads per KV head, tokens, capacity or None, head_dim: one item of eight query rows, several, of sixteen, several ...
FEW = [(1, 1, None, 128), (2, 3, None, 64), (4, 5, None, 128), (3, 5, WIDE, 128), (1, 40, 2 * WIDE, 64), (8, 6, 2 * WIDE, 128)]
# ... and of row tiles of 128: one item, several, of 7 heads
MANY = [(1, 60, None, 64), (4, 13, None, 128), (2, 200, None, 128), (7, 45, None, 64)]


@pytest.fixture(scope="module")
def csp():
    from paper_2412_04652_b200 import binding
    binding.lib()
    return binding


def definition(q, dense, rows, documents=None, prefix=0, item=None):
    """The attention of the last T rows' tokens in 64 bits on the GPU, and how far it may be off.  q [B, Hq, T, d]; rows [B, H];
    documents [cap] of every sequence; item: tokens that share the power of two that values of V are relative to (None: the
    kernel of few query rows).

    A logit is off by e: d products and three steps more in fp32, twice (the magnitudes of codes and base apart, then of the sum),
    what a query's value loses below 2^-14 of the largest (2^-25 of that), the exponential and the rounding of its argument.
    |out - want| <= 2^-8 |want|                           rounded to bf16 once
                  + (r 2^-11 + 4 e + 2^-23 (L / 8 + 16)) sum w (s c + |b|)   weights (times scales; or weights and values: r = 2)
                                                          rounded to halves; a running sum takes one addition in eight rows
      few rows    + 15 L 2^-33 max w s                    a query's products w s are held by a factor that brings the largest to 2^8
                                                          at least; below 2^-14 they are off by 2^-25
      row tiles   + L 2^-32 max w max v                   weights likewise, the largest 2^7
                  + 2^-17 max v sum w [|v| or |b| < 2^-6 max v]    and values, base and sum each 2^-18 of the largest that the item
                                                          sees where they are small beside it
                  + 2^-126"""
    (kc, ks), (vc, vs) = [tuple(x.cuda() for x in pair) for pair in dense]
    B, Hq, T, d = q.shape
    G, sc = Hq // kc.shape[1], 1.0 / math.sqrt(d)
    want, tol = (torch.zeros(B, Hq, T, d, dtype=torch.float64, device="cuda") for _ in range(2))
    for b in range(B):
        for h in range(kc.shape[1]):
            L = int(rows[b, h])
            K, V = values(kc[b, h, :L], ks[b, h, :L]), values(vc[b, h, :L], vs[b, h, :L])
            kb, vb, s = ks[b, h, :L, 1:].double(), vs[b, h, :L, 1:].double(), vs[b, h, :L, 0].double()
            mk, mv = (K - kb) + kb.abs(), (V - vb) + vb.abs()
            t, r = torch.arange(L, device="cuda"), L - T + torch.arange(T, device="cuda")
            see = t[None] <= r.clamp(min=prefix - 1)[:, None]
            if documents is not None:
                see &= documents.cuda()[:L][None] == documents.cuda()[r][:, None]
            top = torch.full((T,), math.inf, dtype=torch.float64, device="cuda")
            if item:                                     # the largest value of the rows that the item's tokens see
                for i in range(0, T, item):
                    top[i:i + item] = mv[see[i:i + item].any(0)].max()
            for hq in range(h * G, h * G + G):
                x = q[b, hq].cuda().double()
                o = torch.where(see, x @ K.T * sc, -math.inf)
                e = sc * (2.0 ** -23 * (d + 4) * torch.where(see, x.abs() @ mk.T, 0.0).amax(1) + 2.0 ** -24 * (d + 4) * torch.where(see, x.abs() @ K.abs().T, 0.0).amax(1) +
                          2.0 ** -25 * x.abs().amax(1) * (K - kb).sum(1).max()) + 2.0 ** -21 + 2.0 ** -23 * torch.where(see, o.abs(), 0.0).amax(1)
                w = torch.exp(o - torch.logaddexp(torch.logsumexp(o, 1), torch.zeros(1, dtype=torch.float64, device="cuda"))[:, None])
                want[b, hq] = w @ V
                small = (15 * L * 2.0 ** -33 * (w * s).amax(1))[:, None]
                if item:
                    few = (w.amax(1) * L * 2.0 ** -32 * top)[:, None].expand(T, d).clone()
                    for i in range(0, T, item):
                        tiny = (mv > 0) & ((V.abs() < 2.0 ** -6 * top[i]) | (vb.abs() < 2.0 ** -6 * top[i]))
                        few[i:i + item] += 2.0 ** -17 * top[i] * (w[i:i + item] @ tiny.double())
                    small = few
                tol[b, hq] = 2.0 ** -8 * (1 + 2.0 ** -8) * want[b, hq].abs() + ((2 if item else 1) * 2.0 ** -11 + 4 * e + 2.0 ** -23 * (L / 8 + 16))[:, None] * (w @ mv) + small + 2.0 ** -126
    return want, tol


def _item(G, T):
    """Tokens of an item of the row-tile kernel; None for up to three items of sixteen query rows, which are not its."""
    return None if -(-T // (16 // G)) <= 3 else 2 * (128 // G)


def _holds(out, want, tol, what=""):
    far = (out.double() - want).abs()
    assert torch.isfinite(out).all(), what
    assert (far <= tol).all(), f"{what}: {int((far > tol).sum())} of {far.numel()} outputs off, worst {float((far / tol).max()):.2f} of the tolerance"


def _attend(csp, q, dense, rows, G, T, capacity, d, page_rows=128, documents=None, prefix=0, what=""):
    """Pages of dense pairs of codes and scales, the call, and the comparison."""
    B, H = rows.shape
    cap = int(rows.max())
    n_pages = int(sum(-(-int(r.max()) // page_rows) for r in rows)) + 2
    order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(cap)).numpy()
    pools, table = [], None
    for codes, scales in dense:
        pc, table = to_pages(codes, rows, page_rows, order, n_pages, 255)
        ps, _ = to_pages(scales, rows, page_rows, order, n_pages, float("nan"))
        pools.append(csp.Q4Cache(pc.cuda(), ps.cuda()))
    capacity = max(capacity or cap, cap)
    wide = torch.full((B, -(-capacity // page_rows)), 10 ** 6, dtype=torch.int32)
    wide[:, :table.shape[1]] = table
    p = csp.Params(B, H * G, H, d, 1, 0, capacity, capacity)
    mods = {}
    if documents is not None:
        mods["documents"] = torch.cat([documents, torch.zeros(capacity - documents.shape[0], dtype=torch.int32)])[None].expand(B, -1).contiguous().cuda()
    if prefix:
        mods["prefix"] = torch.full((B,), prefix, dtype=torch.int32, device="cuda")
    q, out, ws = q.cuda(), torch.zeros(B, H * G, T, d, dtype=torch.bfloat16, device="cuda"), csp.new_chunk_q4_workspace(p, T)
    again = torch.zeros_like(out)
    for o in (out, again):
        csp.chunk_attn_q4_paged(p, q, *pools, wide.cuda(), rows.cuda(), o, ws, mods=csp.ScoreMods(**mods) if mods else None)
    assert csp.device_status(ws) == 0 and torch.equal(out, again)        # (the same bits every time)
    want, tol = definition(q, dense, rows, documents, prefix, _item(G, T))
    _holds(out, want, tol, what)
    return out


def _cache(shape, seed, gain=1.0):
    gen = torch.Generator().manual_seed(seed)
    return [random_rows(shape, gen, gain) for _ in range(2)]


def _queries(B, Hq, T, d, seed, gain=1.0):
    return (torch.randn(B, Hq, T, d, generator=torch.Generator().manual_seed(seed)) * gain).to(torch.bfloat16)


@pytest.mark.parametrize("G,T,capacity,d", FEW + MANY)
def test_ordinary_values(csp, G, T, capacity, d):
    rows = torch.tensor([[700, 433], [T, T + 130]], dtype=torch.int32)
    _attend(csp, _queries(2, 2 * G, T, d, 1, 1.5), _cache((2, 2, 700, d), 2), rows, G, T, capacity, d)


@pytest.mark.parametrize("power", [116, -116])
@pytest.mark.parametrize("G,T,capacity,d", FEW + MANY)
def test_values_far_from_one(csp, G, T, capacity, d, power):
    rows = torch.tensor([[500, 222]], dtype=torch.int32)
    dense = _cache((1, 2, 500, d), 12)
    dense[1][1].mul_(2.0 ** power)
    _attend(csp, _queries(1, 2 * G, T, d, 13), dense, rows, G, T, capacity, d)


@pytest.mark.parametrize("power", [26, 100])
@pytest.mark.parametrize("G,T,capacity,d", FEW + MANY)
def test_large_values_of_other_documents(csp, G, T, capacity, d, power):
    """Every third row is another document's, in the same tiles as the visible ones, with V 2^26 and 2^100 times as large."""
    L = 500
    rows = torch.tensor([[L, L - 70]], dtype=torch.int32)
    doc = torch.where(torch.arange(L) % 3 == 1, 5, 0).to(torch.int32)
    doc[L - 70 - T:] = 0
    dense = _cache((1, 2, L, d), 3)
    dense[1][1][:, :, doc == 5] *= 2.0 ** power
    _attend(csp, _queries(1, 2 * G, T, d, 4), dense, rows, G, T, capacity, d, documents=doc)


@pytest.mark.parametrize("power", [26, 100])
@pytest.mark.parametrize("G,T,capacity,d", [x for x in FEW if x[1] > 1])
def test_large_values_behind_a_token(csp, G, T, capacity, d, power):
    """The last row, which only the last token sees, has V 2^26 and 2^100 times as large as the others."""
    rows = torch.tensor([[333, T]], dtype=torch.int32)
    dense = _cache((1, 2, 333, d), 5)
    for h in range(2):
        dense[1][1][0, h, int(rows[0, h]) - 1] *= 2.0 ** power
    _attend(csp, _queries(1, 2 * G, T, d, 6), dense, rows, G, T, capacity, d)


@pytest.mark.parametrize("power", [26, 100])
@pytest.mark.parametrize("G,T,d", [(1, 300, 64), (2, 300, 128), (5, 90, 64)])
def test_large_values_behind_an_item(csp, G, T, d, power):
    """Row tiles: the first items' tokens do not see the last rows, some of which lie in tiles that they do see."""
    item = _item(G, T)
    first = T // item * item if T % item else T - item   # tokens of the items in front of the last one
    rows = torch.tensor([[T + 20, T]], dtype=torch.int32)
    dense = _cache((1, 2, T + 20, d), 5)
    for h in range(2):
        dense[1][1][0, h, int(rows[0, h]) - T + first:] *= 2.0 ** power
    _attend(csp, _queries(1, 2 * G, T, d, 6), dense, rows, G, T, None, d)


@pytest.mark.parametrize("G,T,capacity,d", FEW)
def test_large_values_of_rows_that_weigh_nothing(csp, G, T, capacity, d):
    """A row in the middle with V 2^26 times as large and a weight of some 2^-100."""
    rows = torch.tensor([[400, 333]], dtype=torch.int32)
    dense = _cache((1, 2, 400, d), 7, 0.1)
    dense[0][1][:, :, 77, 0], dense[0][1][:, :, 77, 1] = 0, -70.0 / math.sqrt(d)
    dense[1][1][:, :, 77] *= 2.0 ** 26
    _attend(csp, 1 + _queries(1, 2 * G, T, d, 8, 0.1), dense, rows, G, T, capacity, d)


def _faint(L, d, seed, nats):
    """K and V: row 0 with logits and values of zero, the others with logits of some -nats and values from 1 to 4."""
    gen = torch.Generator().manual_seed(seed)
    out = []
    for scale, base in ((0.01, -nats / math.sqrt(d) - 0.075), (0.2, 1.0)):
        codes = torch.randint(0, 256, (1, 2, L, d // 2), generator=gen, dtype=torch.uint8)
        scales = torch.empty(1, 2, L, 2, dtype=torch.bfloat16)
        scales[..., 0], scales[..., 1] = scale, base
        scales[:, :, 0] = 0
        out.append((codes, scales))
    return out


@pytest.mark.parametrize("G,T,capacity,d", FEW + MANY)
def test_one_row_weighs_more_than_all_others(csp, G, T, capacity, d):
    """Weights of some 2^-26 beside one of one, whose values are zero: the others' are the result."""
    rows = torch.tensor([[2000, 1999]], dtype=torch.int32)
    _attend(csp, 1 + _queries(1, 2 * G, T, d, 10, 0.05), _faint(2000, d, 9, 18.0), rows, G, T, capacity, d)


@pytest.mark.parametrize("G,T,capacity,d", [FEW[0], FEW[3], MANY[0]])
def test_a_million_faint_rows(csp, G, T, capacity, d):
    rows = torch.tensor([[1 << 20, 900000]], dtype=torch.int32)
    _attend(csp, 1 + _queries(1, 2 * G, T, d, 10, 0.05), _faint(1 << 20, d, 9, 17.7), rows, G, T, capacity, d, page_rows=1024)


@pytest.mark.parametrize("G,T,capacity,d", [(1, 1, None, 64), (2, 3, None, 64), (2, 8, 2 * WIDE, 64), (1, 1, None, 128)])
def test_more_items_than_a_block_looks_at_at_once(csp, G, T, capacity, d):
    """Some five thousand short caches, more than 32 to a block, some of them without rows or with fewer than there are tokens."""
    B, H = 165, 32
    gen = torch.Generator().manual_seed(3)
    rows = torch.randint(T, 120, (B, H), generator=gen, dtype=torch.int32)
    rows[::7, 3] = 0
    rows[::5, 4:9] = T
    cap = 128
    pools, dense = [], []
    for i in range(2):
        codes, scales = random_rows((B, H, cap, d), gen)
        dense.append((codes, scales))
        pools.append(csp.Q4Cache(codes.cuda(), scales.cuda()))
    wide = max(capacity or cap, cap)
    table = torch.full((B, -(-wide // 128)), 10 ** 6, dtype=torch.int32, device="cuda")
    table[:, 0] = torch.arange(B, device="cuda")         # (a cache that is not paged: a page per sequence)
    p = csp.Params(B, H * G, H, d, 1, 0, wide, wide)
    q, ws = _queries(B, H * G, T, d, 4), csp.new_chunk_q4_workspace(p, T)
    out = torch.full((B, H * G, T, d), 7.0, dtype=torch.bfloat16, device="cuda")
    csp.chunk_attn_q4_paged(p, q.cuda(), *pools, table, rows.cuda(), out, ws)
    assert csp.device_status(ws) == csp.DEV_BAD_LEN      # (rows without tokens: more tokens than rows)
    empty = (rows == 0).repeat_interleave(G, 1).cuda()
    assert (out[empty] == 0).all() and torch.isfinite(out).all() and not (out == 7.0).all(-1).any()
    for b in range(0, B, 8):
        heads = [h for h in range(H) if rows[b, h] > 0]
        of_q = [h * G + g for h in heads for g in range(G)]
        want, tol = definition(q[b:b + 1, of_q], [(c[b:b + 1, heads], s[b:b + 1, heads]) for c, s in dense], rows[b:b + 1, heads])
        _holds(out[b:b + 1, of_q], want, tol, f"sequence {b}")
