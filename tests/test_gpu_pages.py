"""The csp_pages_* calls and csp_append_paged against a plain model on the host (exact: integers and copied bits), and a
whole serving round: prompts in chunks, forks, prune in place, pages given back, decoding, compaction."""
import numpy as np
import pytest
import torch

from chunk_util import assert_chunk_close, reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def csp():
    from paper_2412_04652_b200 import binding
    binding.lib()
    return binding


class Model:
    """What the header says, entry by entry."""

    def __init__(self, table, held, refs, rows, R):
        self.table, self.held, self.refs, self.rows, self.R = table.copy(), held.copy(), refs.copy(), rows.copy(), R

    def fork(self, src, dst):
        bad = False
        named = [d for d in dst]
        held0 = self.held.copy()
        for i, (s, d) in enumerate(zip(src, dst)):
            B = len(self.held)
            if not (0 <= s < B and 0 <= d < B) or named.index(d) != i or s in named or held0[d] != 0:
                bad = True
                continue
            h = self.held[s]
            self.table[d, :h] = self.table[s, :h]
            self.held[d] = h
            self.rows[d] = self.rows[s]
            for p in self.table[s, :h]:
                self.refs[p] += 1
        return bad

    def reserve(self, new, whole):
        """The moves, or None if the pool or a table row is too small."""
        B, mp = self.table.shape
        first = [0 if whole else int(self.rows[b].min()) // self.R for b in range(B)]
        need = [-(-(int(self.rows[b].max()) + int(new[b])) // self.R) for b in range(B)]
        if max(need) > mp:
            return None
        entries = [(b, i) for b in range(B) for i in range(mp)]
        claims = {}
        for b, i in entries:
            if first[b] <= i < min(self.held[b], need[b]) and self.refs[self.table[b, i]] > 1:
                claims.setdefault(int(self.table[b, i]), []).append((b, i))
        copy = set()
        for page, who in claims.items():
            copy |= set(who[:-1] if len(who) == self.refs[page] else who)
        fresh = {(b, i) for b, i in entries if self.held[b] <= i < need[b]}
        free = [p for p in range(len(self.refs)) if self.refs[p] == 0]
        if len(copy | fresh) > len(free):
            return None
        moves = []
        for e in entries:
            if e in copy or e in fresh:
                to = free.pop(0)
                if e in copy:
                    moves.append((int(self.table[e]), to))
                    self.refs[self.table[e]] -= 1
                self.table[e] = to
                self.refs[to] = 1
        self.held = np.maximum(self.held, need).astype(np.int32)
        return moves

    def free(self):
        bad = False
        for b in range(len(self.held)):
            need = -(-int(self.rows[b].max()) // self.R)
            if self.rows[b].min() < 0 or need > self.held[b]:
                bad = True
                continue
            for i in range(need, self.held[b]):
                self.refs[self.table[b, i]] -= 1
                self.table[b, i] = -1
            self.held[b] = need
        return bad

    def compact(self):
        live = int((self.refs > 0).sum())
        holes = [p for p in range(live) if self.refs[p] == 0]
        movers = [p for p in range(live, len(self.refs)) if self.refs[p] > 0]
        to = dict(zip(movers, holes))
        for b in range(len(self.held)):
            for i in range(self.held[b]):
                self.table[b, i] = to.get(int(self.table[b, i]), self.table[b, i])
        for p, q in to.items():
            self.refs[q], self.refs[p] = self.refs[p], 0
        return list(to.items())


class Pages:
    """A state on the GPU with its model."""

    def __init__(self, csp, batch, heads, max_pages, R, n_pages):
        self.csp = csp
        self.s = csp.new_page_state(batch, heads, max_pages, R, n_pages)
        self.ws = csp.new_pages_workspace(self.s)
        self.ws[256:] = 0xff
        self.moves = torch.full((batch * max_pages + n_pages, 2), -7, dtype=torch.int32, device="cuda")
        self.n = torch.full((1,), -7, dtype=torch.int32, device="cuda")
        self.m = Model(*(t.cpu().numpy() for t in (self.s.page_table, self.s.held, self.s.refs, self.s.n_rows)), R)

    def set_rows(self, rows):
        self.m.rows[:] = rows
        self.s.n_rows.copy_(torch.as_tensor(self.m.rows))

    def same(self, status=0):
        assert self.csp.device_status(self.ws) == status
        for b in range(len(self.m.held)):
            h = self.m.held[b]
            np.testing.assert_array_equal(self.s.page_table[b, :h].cpu().numpy(), self.m.table[b, :h])
        np.testing.assert_array_equal(self.s.held.cpu().numpy(), self.m.held)
        np.testing.assert_array_equal(self.s.refs.cpu().numpy(), self.m.refs)
        np.testing.assert_array_equal(self.s.n_rows.cpu().numpy(), self.m.rows)
        # and the two views agree: refs count the table's entries
        count = np.zeros_like(self.m.refs)
        for b in range(len(self.m.held)):
            for p in self.m.table[b, :self.m.held[b]]:
                count[p] += 1
        np.testing.assert_array_equal(count, self.m.refs)

    def got_moves(self):
        return [tuple(x) for x in self.moves[:int(self.n)].cpu().tolist()]

    def fork(self, src, dst, status=None):
        bad = self.m.fork(src, dst)
        t = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        self.csp.pages_fork(self.s, t(src), t(dst), self.ws)
        self.same(self.csp.DEV_BAD_LEN if bad else 0)

    def reserve(self, new, whole=False):
        want = self.m.reserve(new, whole)
        t = torch.as_tensor(np.asarray(new, np.int32)).cuda()
        self.csp.pages_reserve(self.s, self.moves, self.n, self.ws, n_new=t, whole=whole)
        assert self.got_moves() == (want or [])
        self.same(0 if want is not None else self.csp.DEV_CAPACITY)
        return want

    def free(self):
        bad = self.m.free()
        self.csp.pages_free(self.s, self.ws)
        self.same(self.csp.DEV_BAD_LEN if bad else 0)

    def compact(self):
        want = self.m.compact()
        self.csp.pages_compact(self.s, self.moves, self.n, self.ws)
        assert self.got_moves() == want
        self.same()
        return want


def test_reserve_takes_the_lowest_free_pages_in_order(csp):
    x = Pages(csp, 3, 2, 6, 128, 16)
    assert x.reserve([300, 0, 128]) == []
    assert x.s.page_table[0, :3].tolist() == [0, 1, 2] and x.s.page_table[2, 0].item() == 3
    x.set_rows([[300, 200], [0, 0], [128, 1]])
    x.reserve([84, 1, 0])                               # exactly full; first page; nothing
    x.reserve([85, 0, 1])
    x.reserve([0, 0, 0])


def test_fork_shares_and_reserve_copies_on_write(csp):
    x = Pages(csp, 6, 2, 4, 128, 20)
    x.reserve([300, 256, 0, 0, 0, 0])
    x.set_rows([[300, 290], [256, 256], [0, 0], [0, 0], [0, 0], [0, 0]])
    x.fork([0, 0, 1], [2, 3, 4])
    moves = x.reserve([1] * 6)                          # page 2 of three sequences: two copies, the last one keeps it
    assert len(moves) == 2
    x.fork([3], [5])
    x.reserve([0, 0, 0, 0, 0, 200])                     # without new rows the owners of a shared last page claim it as well
    x.reserve([1] * 6, whole=True)
    assert (x.s.refs.cpu() <= 1).all()
    x.set_rows([[0, 0]] * 6)
    x.free()
    assert (x.s.refs.cpu() == 0).all() and (x.s.held.cpu() == 0).all()


def test_a_head_that_kept_fewer_rows_decides_from_where_pages_are_owned(csp):
    x = Pages(csp, 2, 3, 5, 128, 12)
    x.reserve([500, 0])
    x.set_rows([[500, 130, 400], [0, 0, 0]])
    x.fork([0], [1])
    assert len(x.reserve([1, 0])) == 3                  # pages 1, 2, 3 hold rows from 130 on


def test_forks_that_break_the_rules_are_skipped_and_flagged(csp):
    x = Pages(csp, 8, 1, 3, 128, 30)
    x.reserve([200, 200, 100, 0, 0, 0, 0, 0])
    x.set_rows([[200], [200], [100], [0], [0], [0], [0], [0]])
    x.fork([0, 1], [3, 3])                              # one dst twice: the first is done
    x.fork([0], [1])                                    # a dst that holds pages
    x.fork([0, 4], [4, 5])                              # a dst that is a src
    x.fork([0], [0])
    x.fork([-1, 8, 0, 0], [4, 5, -2, 99])               # sequences that do not exist
    x.fork([0], [6])
    x.fork([7], [5])                                    # an empty sequence can be forked: nothing to share


def test_reserve_is_all_or_nothing(csp):
    x = Pages(csp, 3, 1, 4, 128, 5)
    assert x.reserve([300, 200, 1]) is None             # 6 pages wanted
    assert x.reserve([300, 200, 0]) == []
    x.set_rows([[300], [200], [0]])
    x.fork([0], [2])
    assert x.reserve([1, 0, 1]) is None                 # the pool is empty
    assert x.reserve([400, 0, 0]) is None               # the table row is too short
    x.s.n_rows[1] = -1
    csp.pages_reserve(x.s, x.moves, x.n, x.ws)
    assert csp.device_status(x.ws) == csp.DEV_BAD_LEN and int(x.n) == 0
    x.s.n_rows[1] = 200
    csp.pages_reserve(x.s, x.moves, x.n, x.ws, n_new=torch.tensor([0, -1, 0], dtype=torch.int32, device="cuda"))
    assert csp.device_status(x.ws) == csp.DEV_BAD_LEN
    x.same()


def test_a_move_list_that_is_too_short_changes_nothing(csp):
    x = Pages(csp, 4, 1, 2, 128, 12)
    x.reserve([200, 0, 0, 0])
    x.set_rows([[200], [0], [0], [0]])
    x.fork([0, 0, 0], [1, 2, 3])
    short = torch.full((2, 2), -7, dtype=torch.int32, device="cuda")
    csp.pages_reserve(x.s, short, x.n, x.ws, n_new=torch.ones(4, dtype=torch.int32, device="cuda"))
    assert csp.device_status(x.ws) == csp.DEV_CAPACITY and int(x.n) == 0 and (short == -7).all()
    x.same()
    x.reserve([1] * 4)
    x.set_rows([[0], [0], [201], [0]])                  # its own copy lies behind pages that are free now: one move
    x.free()
    csp.pages_compact(x.s, short[:0], x.n, x.ws)
    assert csp.device_status(x.ws) == csp.DEV_CAPACITY and int(x.n) == 0
    x.same()
    assert len(x.compact()) == 1


def test_free_after_a_prune_and_of_failed_prunes(csp):
    x = Pages(csp, 4, 2, 6, 128, 30)
    x.reserve([700, 700, 700, 100])
    x.set_rows([[700, 700]] * 3 + [[100, 100]])
    x.set_rows([[128, 129], [-1, 60], [256, 0], [100, 90]])     # -1: a prune that did not fit
    x.free()
    x.set_rows([[400, 0], [0, 0], [1, 0], [0, 0]])               # 400 rows in two pages: contradicts itself
    x.free()


def test_entries_outside_the_pool_are_flagged_and_left_alone(csp):
    x = Pages(csp, 2, 1, 4, 128, 10)
    x.reserve([500, 0])
    x.set_rows([[500], [0]])
    x.s.page_table[0, 2] = 77
    x.s.n_rows[0] = 100
    csp.pages_free(x.s, x.ws)
    assert csp.device_status(x.ws) == csp.DEV_BAD_LEN
    assert x.s.refs.tolist()[:4] == [1, 0, 1, 0] and x.s.held.tolist() == [1, 0]
    x.s.page_table[0, 0] = -4
    csp.pages_compact(x.s, x.moves, x.n, x.ws)
    assert csp.device_status(x.ws) == csp.DEV_BAD_LEN
    csp.pages_reserve(x.s, x.moves, x.n, x.ws, whole=True)
    assert csp.device_status(x.ws) == csp.DEV_BAD_LEN and int(x.n) == 0
    csp.pages_fork(x.s, torch.tensor([0], dtype=torch.int32, device="cuda"), torch.tensor([1], dtype=torch.int32, device="cuda"), x.ws)
    assert csp.device_status(x.ws) == csp.DEV_BAD_LEN


@pytest.mark.parametrize("batch,max_pages,n_pages", [(5, 3, 20), (40, 70, 2500), (300, 40, 9000), (3, 5000, 12000)])
def test_random_rounds(csp, batch, max_pages, n_pages):
    """Seeded sequences of calls, sizes beyond one block-wide step of the scans among them."""
    rng = np.random.RandomState(batch)
    x = Pages(csp, batch, 3, max_pages, 128, n_pages)
    top = min(max_pages * 128 - 1, n_pages * 128 // batch)
    for _ in range(6):
        rows = x.m.rows.copy()
        empty = [b for b in range(batch) if x.m.held[b] == 0]
        full = [b for b in range(batch) if x.m.held[b] > 0]
        if empty and full:
            dst = list(rng.permutation(empty)[:max(1, len(empty) // 2)])
            x.fork([int(rng.choice(full)) for _ in dst], [int(d) for d in dst])
        new = rng.randint(0, max(2, top // 3), size=batch)
        if x.reserve(new, whole=bool(rng.rand() < 0.3)) is not None:
            x.set_rows(np.minimum(x.m.rows + np.minimum(new[:, None], rng.randint(0, top, size=(batch, 3))), x.m.held[:, None] * 128))
        keep = rng.rand(batch, 1) * (rng.rand(batch, 1) < 0.8)
        x.set_rows((x.m.rows * keep).astype(np.int32))
        x.free()
        x.compact()
        del rows


# ---- rows

def _pool(n_pages, H, R, d, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(n_pages, H, R, d, generator=g, device="cuda").to(dtype)


@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 64), (torch.bfloat16, 128), (torch.float32, 64), (torch.float32, 128), (torch.bfloat16, 256)])
@pytest.mark.parametrize("R", [128, 384, 7])
def test_copy_moves_whole_pages(csp, dtype, d, R):
    H, n = 3, 11
    k, v = _pool(n, H, R, d, dtype), _pool(n, H, R, d, dtype, 1)
    wk, wv = k.clone(), v.clone()
    p = csp.Params(1, H, H, d, 1, 0, R, R, dtype=csp.F32 if dtype == torch.float32 else csp.BF16)
    ws = csp.new_append_workspace(p)
    pairs = [(3, 0), (10, 5), (3, 9), (7, 1)]
    moves = torch.tensor(pairs + [(-1, -1)], dtype=torch.int32, device="cuda")
    count = torch.tensor([4], dtype=torch.int32, device="cuda")
    csp.pages_copy(p, k, v, moves, count, ws)
    for a, b in pairs:
        wk[b], wv[b] = wk[a], wv[a]
    assert csp.device_status(ws) == 0 and torch.equal(k, wk) and torch.equal(v, wv)
    count.fill_(0)
    csp.pages_copy(p, k, v, moves, count, ws)
    assert csp.device_status(ws) == 0 and torch.equal(k, wk)
    count.fill_(9)                                      # more than the list holds: clamped; (-1, -1) is no page
    csp.pages_copy(p, k, v, moves, count, ws)
    assert csp.device_status(ws) == csp.DEV_BAD_LEN and torch.equal(k, wk) and torch.equal(v, wv)


def test_copy_of_strided_pools_and_past_32_bits(csp):
    """Pools whose pages hold several layers (a wide page stride), K and V strided differently, and a pool of more than
    2^32 bytes."""
    H, R, d = 2, 128, 128
    wide = torch.zeros(9, 3, H, R, d, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(4)
    wide[:] = torch.randn(wide.shape, generator=g, device="cuda").to(torch.bfloat16)
    rows_first = torch.randn(9, R, H, d, generator=g, device="cuda").to(torch.bfloat16)
    k, v = wide[:, 1], rows_first.transpose(1, 2)
    want_wide, want_v = wide.clone(), v.clone()
    want_wide[8, 1], want_wide[0, 1] = wide[2, 1], wide[5, 1]
    want_v[8], want_v[0] = v[2].clone(), v[5].clone()
    p = csp.Params(1, H, H, d, 1, 0, R, R)
    ws = csp.new_append_workspace(p)
    moves = torch.tensor([(2, 8), (5, 0)], dtype=torch.int32, device="cuda")
    count = torch.tensor([2], dtype=torch.int32, device="cuda")
    csp.pages_copy(p, k, v, moves, count, ws)
    assert csp.device_status(ws) == 0 and torch.equal(wide, want_wide) and torch.equal(v, want_v)
    n = 2 ** 31 // (H * R * d) + 5
    big_k = torch.empty(n, H, R, d, dtype=torch.bfloat16, device="cuda")
    big_v = torch.empty_like(big_k)
    big_k[n - 1], big_v[n - 1] = k[2], v[2]
    big_k[4], big_v[4] = k[5], v[5]
    moves = torch.tensor([(n - 1, 1), (4, n - 2)], dtype=torch.int32, device="cuda")
    csp.pages_copy(p, big_k, big_v, moves, count, ws)
    assert csp.device_status(ws) == 0
    assert torch.equal(big_k[1], k[2]) and torch.equal(big_v[1], v[2]) and torch.equal(big_k[n - 2], k[5]) and torch.equal(big_v[n - 2], v[5])


@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 64), (torch.bfloat16, 128), (torch.float32, 64)])
@pytest.mark.parametrize("T", [1, 3, 130])
@pytest.mark.parametrize("in_place", [False, True])
def test_append(csp, dtype, d, T, in_place):
    B, H, R, mp = 3, 4, 128, 4
    k, v = _pool(13, H, R, d, dtype), _pool(13, H, R, d, dtype, 1)
    g = torch.Generator(device="cuda").manual_seed(2)
    kn = torch.randn(B, T, H, d, generator=g, device="cuda").to(dtype).transpose(1, 2)
    vn = torch.randn(B, H, T, d, generator=g, device="cuda").to(dtype)
    table = torch.tensor([[3, 1, 12, 7], [0, 9, 4, 2], [5, 6, 8, 10]], dtype=torch.int32, device="cuda")
    rows = torch.tensor([[0, 127, 128, 300], [5, 5, 255, 256], [511 - T, 512 - T, 1, 2]], dtype=torch.int32, device="cuda")
    new = torch.tensor([T, max(0, T - 2), T], dtype=torch.int32, device="cuda")
    p = csp.Params(B, H, H, d, 1, 0, mp * R, mp * R, dtype=csp.F32 if dtype == torch.float32 else csp.BF16)
    ws = csp.new_append_workspace(p)
    wk, wv, before = k.clone(), v.clone(), rows.clone()
    for b in range(B):
        for h in range(H):
            for i in range(int(new[b])):
                t = int(before[b, h]) + i
                wk[int(table[b, t // R]), h, t % R] = kn[b, h, i]
                wv[int(table[b, t // R]), h, t % R] = vn[b, h, i]
    after = rows if in_place else torch.full_like(rows, -9)
    csp.append_paged(p, kn, vn, k, v, table, rows, after, ws, n_new=new)
    assert csp.device_status(ws) == 0
    assert torch.equal(k, wk) and torch.equal(v, wv) and torch.equal(after, before + new[:, None])
    assert in_place or torch.equal(rows, before)


def test_append_flags_what_it_cannot_write(csp):
    H, R, d = 2, 128, 64
    k, v = _pool(4, H, R, d, torch.bfloat16), _pool(4, H, R, d, torch.bfloat16, 1)
    k0, v0 = k.clone(), v.clone()
    new_rows = torch.ones(1, H, 3, d, dtype=torch.bfloat16, device="cuda")
    p = csp.Params(1, H, H, d, 1, 0, 256, 256)
    ws = csp.new_append_workspace(p)
    out = torch.zeros(1, H, dtype=torch.int32, device="cuda")
    table = torch.tensor([[1, 2]], dtype=torch.int32, device="cuda")

    def call(rows, n_new, tab=table):
        csp.append_paged(p, new_rows, new_rows, k, v, tab, torch.tensor([rows], dtype=torch.int32, device="cuda"), out, ws,
                         n_new=torch.tensor([n_new], dtype=torch.int32, device="cuda"))
        return csp.device_status(ws), out.tolist()[0]
    assert call([254, 300], 3) == (csp.DEV_CAPACITY, [254, 300]) and torch.equal(k, k0)
    assert call([-1, 10], 0) == (csp.DEV_BAD_LEN, [-1, 10]) and torch.equal(k, k0)
    assert call([5, 10], -2) == (csp.DEV_BAD_LEN, [5, 10]) and torch.equal(k, k0)
    # a page outside the pool: its rows are dropped, the others written
    assert call([126, 126], 3, torch.tensor([[1, 9]], dtype=torch.int32, device="cuda")) == (csp.DEV_BAD_LEN, [129, 129])
    k0[1, :, 126:128] = 1
    v0[1, :, 126:128] = 1
    assert torch.equal(k, k0) and torch.equal(v, v0)
    assert call([0, 0], 99) == (csp.DEV_BAD_LEN, [3, 3])         # more tokens than the chunk has


# ---- together

def test_a_serving_round(csp):
    """Two prompts enter in chunks (reserve, append, chunk attention), each is forked, the forks decode a few tokens, all
    are pruned in place to different row counts, pages go back and are moved together, and decoding goes on: at every
    step the attention equals the definition on the rows that a plain program would hold."""
    torch.manual_seed(0)
    B, Hq, H, d, R, mp, n_pages = 4, 6, 2, 64, 128, 6, 30
    x = Pages(csp, B, H, mp, R, n_pages)
    p = csp.Params(B, Hq, H, d, 1, 0, mp * R, mp * R)
    k = torch.full((n_pages, H, R, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    v = torch.full_like(k, float("inf"))
    mine = [[(torch.zeros(0, d), torch.zeros(0, d)) for _ in range(H)] for _ in range(B)]       # the plain program's rows
    aws, cws = csp.new_append_workspace(p), csp.new_chunk_workspace(p, 150)

    def step(new):
        T = max(max(new), 1)
        n = torch.tensor(new, dtype=torch.int32, device="cuda")
        x.reserve(new)
        csp.pages_copy(p, k, v, x.moves, x.n, aws)
        kn, vn = torch.randn(B, H, T, d).to(torch.bfloat16), torch.randn(B, H, T, d).to(torch.bfloat16)
        q = torch.randn(B, Hq, T, d).to(torch.bfloat16)
        csp.append_paged(p, kn.cuda(), vn.cuda(), k, v, x.s.page_table, x.s.n_rows, x.s.n_rows, aws, n_new=n)
        x.m.rows += np.asarray(new, np.int32)[:, None]
        out = torch.zeros(B, Hq, T, d, dtype=torch.bfloat16, device="cuda")
        lse = torch.zeros(B, Hq, T, device="cuda")
        csp.chunk_attn_paged(p, q.cuda(), k, v, x.s.page_table, x.s.n_rows, out, cws, n_new=n, lse=lse)
        x.same()
        assert csp.device_status(aws) == 0 and csp.device_status(cws) == 0
        cap = mp * R
        dk, dv = torch.zeros(B, H, cap, d), torch.zeros(B, H, cap, d)
        for b in range(B):
            for h in range(H):
                mine[b][h] = (torch.cat([mine[b][h][0], kn[b, h, :new[b]].float()]), torch.cat([mine[b][h][1], vn[b, h, :new[b]].float()]))
                L = mine[b][h][0].shape[0]
                assert L == x.m.rows[b, h]
                dk[b, h, :L], dv[b, h, :L] = mine[b][h]
        assert_chunk_close(out, lse, reference(q, dk, dv, x.m.rows, new), new)

    step([150, 100, 0, 0])
    step([150, 28, 0, 0])
    x.fork([0, 1], [2, 3])
    for b in (0, 1):
        mine[b + 2] = [tuple(t.clone() for t in mine[b][h]) for h in range(H)]
    step([1, 1, 1, 1])
    step([2, 0, 1, 3])
    # prune in place: every sequence gets pages of its own, a kept subset moves down, per head another number of rows
    x.reserve([0] * B, whole=True)
    csp.pages_copy(p, k, v, x.moves, x.n, aws)
    cap = mp * R
    pp = csp.Params(B, Hq, H, d, 32, 32, cap, cap)
    mod = torch.zeros(B, H, cap, dtype=torch.uint8, device="cuda")
    lens = x.s.n_rows[:, 0].contiguous()
    bud = torch.tensor([[40, 0, 0, 0], [20, 0, 0, 0], [60, 0, 0, 0], [10, 0, 0, 0]], dtype=torch.int32, device="cuda")
    idx = torch.full((B, H, cap), -1, dtype=torch.int32, device="cuda")
    mod_out = torch.zeros_like(mod)
    qw = torch.randn(B, Hq, 32, d, device="cuda").to(torch.bfloat16)
    pws = csp.new_workspace(pp)
    n_out = torch.zeros(B, H, dtype=torch.int32, device="cuda")
    csp.prune_layer_paged(pp, qw, k, v, x.s.page_table, mod, lens, bud, k, v, mod_out, n_out, pws, keep_idx=idx)
    assert csp.device_status(pws) == 0
    for b in range(B):
        for h in range(H):
            keep = idx[b, h, :int(n_out[b, h])].cpu().long()
            mine[b][h] = tuple(t[keep] for t in mine[b][h])
    x.set_rows(n_out.cpu().numpy())
    x.free()
    x.compact()
    csp.pages_copy(p, k, v, x.moves, x.n, aws)
    step([1, 1, 1, 1])
    step([130, 1, 0, 60])


def test_a_captured_round_replays(csp):
    """Fork, reserve, copy, append, attention and free in one graph: replays do what the first run did."""
    B, Hq, H, d, R, mp, n_pages = 4, 4, 2, 128, 128, 4, 16
    x = Pages(csp, B, H, mp, R, n_pages)
    x.reserve([200, 130, 0, 0])
    x.set_rows([[200, 200], [130, 120], [0, 0], [0, 0]])
    p = csp.Params(B, Hq, H, d, 1, 0, mp * R, mp * R)
    k, v = _pool(n_pages, H, R, d, torch.bfloat16), _pool(n_pages, H, R, d, torch.bfloat16, 1)
    kn, vn = torch.randn(2, B, H, 1, d, device="cuda").to(torch.bfloat16).unbind(0)
    q = torch.randn(B, Hq, 1, d, device="cuda").to(torch.bfloat16)
    out = torch.zeros(B, Hq, 1, d, dtype=torch.bfloat16, device="cuda")
    aws, cws = csp.new_append_workspace(p), csp.new_chunk_workspace(p, 1)
    src, dst = (torch.tensor(t, dtype=torch.int32, device="cuda") for t in ([0, 1], [2, 3]))
    one, none = torch.ones(B, dtype=torch.int32, device="cuda"), torch.zeros(2, H, dtype=torch.int32, device="cuda")
    after = torch.zeros(B, H, dtype=torch.int32, device="cuda")

    def round_trip():
        csp.pages_fork(x.s, src, dst, x.ws)
        csp.pages_reserve(x.s, x.moves, x.n, x.ws, n_new=one)
        csp.pages_copy(p, k, v, x.moves, x.n, aws)
        csp.append_paged(p, kn, vn, k, v, x.s.page_table, x.s.n_rows, after, aws)
        csp.chunk_attn_paged(p, q, k, v, x.s.page_table, after, out, cws)
        x.s.n_rows[2:].copy_(none)
        csp.pages_free(x.s, x.ws)
    buffers = (k, v, x.s.page_table, x.s.held, x.s.refs)
    start = [t.clone() for t in buffers]
    round_trip()
    torch.cuda.synchronize()
    want, state = out.clone(), [t.clone() for t in (x.s.held, x.s.refs, x.s.page_table[:2, :2])]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        round_trip()
    for _ in range(3):
        out.zero_()
        for t, t0 in zip(buffers, start):               # who keeps a shared page and who gets a copy moves the rows about
            t.copy_(t0)
        graph.replay()
        torch.cuda.synchronize()
        assert csp.device_status(x.ws) == 0 and csp.device_status(aws) == 0 and csp.device_status(cws) == 0
        assert torch.equal(out, want)
        for a, b in zip(state, (x.s.held, x.s.refs, x.s.page_table[:2, :2])):
            assert torch.equal(a, b)


# ---- a state that contradicts itself

def test_reserve_leaves_a_page_that_is_named_more_often_than_counted(csp):
    x = Pages(csp, 5, 1, 4, 128, 12)
    x.reserve([200, 0, 0, 0, 100])
    x.set_rows([[200], [0], [0], [0], [100]])
    x.fork([0, 0], [1, 2])                              # page 1 is the last one of three sequences
    x.s.refs[1] = 2
    table, held, refs = (t.clone() for t in (x.s.page_table, x.s.held, x.s.refs))
    csp.pages_reserve(x.s, x.moves, x.n, x.ws, n_new=torch.tensor([1, 1, 1, 1, 100], dtype=torch.int32, device="cuda"))
    assert csp.device_status(x.ws) == csp.DEV_BAD_LEN and int(x.n) == 0
    table[3, 0], table[4, 1] = 3, 4                     # the others get what they asked for
    refs[3] = refs[4] = 1
    held[3], held[4] = 1, 2
    assert torch.equal(x.s.page_table, table) and torch.equal(x.s.refs, refs) and torch.equal(x.s.held, held)
    # fewer ask than it is counted for: as far as this call sees nothing is wrong
    x.s.n_rows[1:3] = 128
    csp.pages_reserve(x.s, x.moves, x.n, x.ws)
    assert csp.device_status(x.ws) == 0 and x.got_moves() == [(1, 5)]
    assert x.s.refs.tolist() == [3, 1, 1, 1, 1, 1, 0, 0, 0, 0, 0, 0]


@pytest.mark.parametrize("batch,max_pages", [(3, 4), (3, 5000)])
def test_reserve_does_not_give_away_a_page_that_is_named(csp, batch, max_pages):
    """A page that a table entry names, but that is counted free; also with more entries than one step of the scan has."""
    x = Pages(csp, batch, 1, max_pages, 128, 9)
    x.reserve([300, 0, 0])
    x.set_rows([[300], [0], [0]])
    x.s.refs[2] = 0
    csp.pages_reserve(x.s, x.moves, x.n, x.ws, n_new=torch.tensor([1, 100, 300], dtype=torch.int32, device="cuda"))
    assert csp.device_status(x.ws) == csp.DEV_BAD_LEN and int(x.n) == 0
    assert x.s.page_table[:, :4].tolist() == [[0, 1, 2, -1], [3, -1, -1, -1], [4, 5, 6, -1]]
    assert x.s.refs.tolist() == [1, 1, 0, 1, 1, 1, 1, 0, 0] and x.s.held.tolist() == [3, 1, 3]
    # it counts as taken when the pool runs short
    csp.pages_reserve(x.s, x.moves, x.n, x.ws, n_new=torch.tensor([1, 0, 700], dtype=torch.int32, device="cuda"))
    assert csp.device_status(x.ws) & csp.DEV_CAPACITY and int(x.n) == 0
    assert x.s.held.tolist() == [3, 1, 3]


@pytest.mark.parametrize("page", [1, 6])
def test_compact_moves_nothing_where_a_free_page_is_named(csp, page):
    """In front of the last live page, where another page would move in, and behind it."""
    x = Pages(csp, 3, 1, 3, 128, 10)
    x.reserve([300, 300, 300])
    x.set_rows([[300], [0], [300]])
    x.free()                                            # pages 0, 1, 2 and 6, 7, 8 are in use
    keep = [t.clone() for t in (x.s.page_table, x.s.held, x.s.refs)]
    x.s.refs[page] = 0
    keep[2][page] = 0
    csp.pages_compact(x.s, x.moves, x.n, x.ws)
    assert csp.device_status(x.ws) == csp.DEV_BAD_LEN and int(x.n) == 0
    for a, b in zip(keep, (x.s.page_table, x.s.held, x.s.refs)):
        assert torch.equal(a, b)
    x.s.refs[page] = 1
    assert x.compact() == [(6, 3), (7, 4), (8, 5)]


def test_free_leaves_entries_that_contradict_the_counts(csp):
    x = Pages(csp, 2, 1, 4, 128, 10)
    x.reserve([500, 300])
    x.set_rows([[0], [300]])
    x.s.page_table[0, 1] = 77
    x.s.refs[2] = 0
    csp.pages_free(x.s, x.ws)
    assert csp.device_status(x.ws) == csp.DEV_BAD_LEN
    assert x.s.page_table.tolist() == [[-1, 77, 2, -1], [4, 5, 6, -1]]
    assert x.s.held.tolist() == [0, 3] and x.s.refs.tolist() == [0, 1, 0, 0, 1, 1, 1, 0, 0, 0]


def test_forks_of_sequences_that_contradict_the_counts_are_skipped(csp):
    x = Pages(csp, 7, 1, 50, 128, 120)
    x.reserve([5000, 5000, 300, 0, 0, 0, 0])
    x.set_rows([[5000], [5000], [300], [0], [0], [0], [0]])
    x.s.page_table[0, 39] = 200
    x.s.refs[int(x.s.page_table[1, 33])] = 0
    table, held, refs, rows = (t.clone() for t in (x.s.page_table, x.s.held, x.s.refs, x.s.n_rows))
    t = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    csp.pages_fork(x.s, t(0, 1, 2, 1), t(3, 4, 5, 6), x.ws)
    assert csp.device_status(x.ws) == csp.DEV_BAD_LEN
    table[5], held[5], rows[5] = table[2], held[2], rows[2]
    refs[table[2, :3].long()] = 2
    for a, b in zip((table, held, refs, rows), (x.s.page_table, x.s.held, x.s.refs, x.s.n_rows)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("B,T", [(2, 0), (0, 3), (0, 0)])
@pytest.mark.parametrize("in_place", [False, True])
def test_nothing_to_append(csp, B, T, in_place):
    p = csp.Params(B, 2, 2, 64, 1, 0, 256, 256)
    pool = _pool(5, 2, 128, 64, torch.bfloat16)
    before, rows = pool.clone(), torch.arange(2 * B, dtype=torch.int32, device="cuda").reshape(B, 2)
    after = rows if in_place else torch.full_like(rows, -9)
    new, ws = torch.zeros(B, 2, T, 64, dtype=torch.bfloat16, device="cuda"), csp.new_append_workspace(p)
    csp.append_paged(p, new, new, pool, pool, torch.zeros(B, 2, dtype=torch.int32, device="cuda"), rows, after, ws)
    assert csp.device_status(ws) == 0 and torch.equal(pool, before)
    assert after.tolist() == [[2 * b, 2 * b + 1] for b in range(B)]


def test_a_pool_without_sequences(csp):
    x = Pages(csp, 0, 2, 3, 128, 6)
    x.ws[:256] = 0
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    csp.pages_fork(x.s, none, none, x.ws)
    csp.pages_reserve(x.s, x.moves, x.n, x.ws, n_new=none)
    assert int(x.n) == 0
    csp.pages_free(x.s, x.ws)
    csp.pages_compact(x.s, x.moves, x.n, x.ws)
    assert int(x.n) == 0 and csp.device_status(x.ws) == 0
