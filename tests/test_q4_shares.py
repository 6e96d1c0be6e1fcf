"""The arithmetic by which the 4-bit attention's work is shared out, and its divisions by multiplication, said again in Python: every tile
of every item is taken once, and the blocks that an item is cut between are those that its count names."""
import random

import pytest

COST = MIN_TILES = 4                                     # of few query rows: what an item costs besides its tiles, tiles that a part has at least


def cut(weights, tiles, at, share, snap):
    """Where the cut at `at` falls: item and tile, and of an item that is cut the block it begins in and in how many its parts are."""
    s = 0
    for i, w in enumerate(weights):
        if at < s + w:
            t = at - s - COST
            if at - s <= snap or t < MIN_TILES:
                return i, 0, None
            if s + w - at <= snap or tiles[i] - t < MIN_TILES:
                return i + 1, 0, None
            first = (s + max(snap, COST + MIN_TILES - 1)) // share + 1
            last = (s + w - max(snap, MIN_TILES - 1) - 1) // share
            return i, t, (first - 1, last - first + 2)
        s += w
    return len(weights), 0, None


def block_shares(tiles, grid):
    """tiles: of every item, None where it has no tokens."""
    weights = [0 if t is None else t + COST for t in tiles]
    share = max(-(-sum(weights) // grid), COST + MIN_TILES)
    snap = share // 8
    cuts = [cut(weights, tiles, share * c, share, snap) for c in range(grid + 1)]
    return [(cuts[c], cuts[c + 1]) for c in range(grid)]


def warp_parts(tiles, begin, end, warps):
    """What the warps of a block have: lists of (item, lo, hi)."""
    (item0, tile0, _), (item1, tile1, _) = begin, end
    n = len(tiles)
    last = min(item1, n - 1)

    def low(i):
        return tile0 if i == item0 else 0

    weights = []
    for i in range(item0, last + 1):
        if tiles[i] is None or (i == item1 and tile1 == 0):
            weights.append(0)
        else:
            weights.append(max((tile1 if i == item1 else tiles[i]) - low(i), 0) + 1)
    part = max(-(-sum(weights) // warps), 2)
    got = []
    for warp in range(warps):
        ends = [(n, 0), (n, 0)]
        for k in range(2):
            p, at = 0, (warp + k) * part
            for i, w in zip(range(item0, last + 1), weights):
                if p <= at < p + w:
                    ends[k] = (i, low(i) + max(at - p - 1, 0))
                p += w
        (b, b_tile), (e, e_tile) = ends
        mine = []
        for i in range(b, min(e, item1, n - 1) + 1):
            if (i == e and e_tile == low(i)) or (i == item1 and tile1 == 0):
                break
            if tiles[i] is None:
                continue
            mine.append((i, b_tile if i == b else low(i), e_tile if i == e else tile1 if i == item1 else tiles[i]))
        got.append(mine)
    return got


@pytest.mark.parametrize("warps", [8, 12])
def test_every_tile_is_taken_once(warps):
    rng = random.Random(warps)
    for trial in range(250):
        n, grid = rng.choice([1, 2, 5, 40, 150, 400]), rng.choice([1, 2, 7, 30, 148])
        longest = rng.choice([1, 8, 60, 400])
        tiles = [None if rng.random() < 0.1 else rng.randint(0, longest) if rng.random() < 0.8 else rng.randint(0, 8 * longest) for _ in range(n)]
        shares = block_shares(tiles, grid)
        taken = [[] for _ in range(n)]                   # (block, lo, hi)
        for c, (begin, end) in enumerate(shares):
            for parts in warp_parts(tiles, begin, end, warps):
                for item, lo, hi in parts:
                    taken[item].append((c, lo, hi))
        for i, t in enumerate(tiles):
            if t is None:
                assert not taken[i]
                continue
            at = 0
            for _, lo, hi in taken[i]:                   # one behind the other
                assert lo == at and hi >= lo
                at = hi
            assert at == t and taken[i], (trial, i)      # (an item without tiles is somebody's as well: its outputs are zeros)
            blocks = sorted({c for c, _, _ in taken[i]})
            if len(blocks) == 1:
                assert not any(s[1][0] == i and s[1][1] > 0 for s in shares)
                continue
            # the parts: what a block says of the item that it goes on with, and of the one that goes on in the next
            names = {shares[c][0][2] for c in blocks[1:]} | {shares[c][1][2] for c in blocks[:-1]}
            assert names == {(blocks[0], len(blocks))} and blocks == list(range(blocks[0], blocks[-1] + 1)) and len(blocks) < 256


EDGES = [0, 1, 2, 127, 128, 129, 2 ** 16 - 1, 2 ** 16, 2 ** 30 - 1, 2 ** 30, 2 ** 31 - 2, 2 ** 31 - 1]


def test_divisions_by_multiplication():
    """Whole numbers below 2^31: m = 2^(31 + l) / n rounded up with 2^(l - 1) < n <= 2^l, and 2^32 / n + 1 with a correction by one."""
    rng = random.Random(1)
    divisors = list(range(1, 70)) + [128 * i for i in range(1, 40)] + [2 ** i + j for i in range(7, 31) for j in (-1, 0, 1)] + [2 ** 31 - 1]
    for n in divisors:
        bits = (n - 1).bit_length()
        m = (2 ** (31 + bits) + n - 1) // n
        inverse = 2 ** 32 // n + 1
        assert m < 2 ** 32
        for t in EDGES + [k * n + j for k in (1, 7, (2 ** 31 - 1) // n) for j in (-1, 0, 1)] + [rng.randrange(2 ** 31) for _ in range(50)]:
            if not 0 <= t < 2 ** 31:
                continue
            assert t * m >> 31 + bits == t // n, (t, n)
            if n > 1:                                    # (2^32 + 1 does not fit)
                q = t * inverse >> 32
                rest = t - q * n
                assert (q, rest) == divmod(t, n) or (rest < 0 and (q - 1, rest + n) == divmod(t, n)), (t, n)
