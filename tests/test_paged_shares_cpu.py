"""The split of the attention's work over a fixed number of blocks, restated:
tiles laid end to end, equal shares, short tiles whole, boundaries moved to
key blocks.  Every tile's key blocks are covered once and in order, a tile in
one share leaves no partial, and the partials' kinds let the join find them."""
import random

import pytest

NONE, FIRST, MIDDLE, LAST = range(4)


def tiles_of(reqs, tq, heads, extra):
    """(start on the axis, keys) of every tile in order, and the axis' length."""
    at, tiles = 0, []
    for n, kv in reqs:
        for _ in range(heads):
            for t in range(-(-n // tq)):
                keys = max(1, kv - n + min((t + 1) * tq, n))
                tiles.append((at, keys))
                at += keys + extra
    return tiles, at


def before(n, kv, t, tq, extra):
    """The closed form of the tiles' lengths before tile t of a request."""
    c = kv - n
    flat = min(t, (-c) // tq) if c < 0 else 0
    m = t - flat
    return flat + m * c + tq * (m * flat + m * (m + 1) // 2) + t * extra


def walk(tiles, total, share, c, kb, extra):
    """Share c's visits: (tile, first block, end block, blocks, kind, slot)."""
    lo, hi = share * c, min(total, share * (c + 1))
    left, visits, first = hi - lo, [], True
    if left <= 0:
        return visits
    i = max(k for k, (start, _) in enumerate(tiles) if start <= lo)
    off = lo - tiles[i][0]
    while left > 0:
        keys = tiles[i][1]
        length, whole = keys + extra, keys <= 2 * extra
        if whole and off > 0:
            left, off, i = left - (length - off), 0, i + 1
            continue
        take = length if whole else min(left, length - off)
        blocks = -(-keys // kb)
        j0, j1 = min(blocks, -(-off // kb)), min(blocks, -(-(off + take) // kb))
        slot, first, tile = (0 if first else 1), False, i
        left, off = left - take, off + take
        if off >= length:
            off, i = 0, i + 1
        if j0 < j1:
            kind = (NONE if j1 == blocks else FIRST) if j0 == 0 else \
                (LAST if j1 == blocks else MIDDLE)
            visits.append((tile, j0, j1, blocks, kind, slot))
    return visits


@pytest.mark.parametrize("seed", range(40))
def test_every_block_is_covered_once_and_partials_are_found(seed):
    rng = random.Random(seed)
    for _ in range(40):
        reqs = []
        for _ in range(rng.randint(1, 12)):
            n = rng.choice([0, 1, 1, rng.randint(1, 700)])
            reqs.append((n, rng.choice([0, n, n + rng.randint(0, 3000), rng.randint(0, 50)])))
        if not any(n for n, _ in reqs):
            continue
        tq, kb, extra, least = rng.choice([(64, 128, 384, 256), (32, 128, 256, 256),
                                           (4, 64, 64, 128), (16, 32, 32, 128)])
        shares, heads = rng.choice([3, 16, 152]), rng.randint(1, 4)
        tiles, total = tiles_of(reqs, tq, heads, extra)
        at = 0
        for n, kv in reqs:    # the closed form agrees with the tiles laid out
            for t in range(-(-n // tq)):
                assert before(n, kv, t, tq, extra) == tiles[at + t][0] - tiles[at][0]
            at += heads * -(-n // tq)
        share = -(-max(-(-total // shares), least) // kb) * kb
        cover, kinds = {}, []
        for c in range(shares):
            kinds.append([NONE, NONE])
            for tile, j0, j1, blocks, kind, slot in walk(tiles, total, share, c, kb, extra):
                cover.setdefault(tile, []).append((c, j0, j1, blocks, kind, slot))
                if kind != NONE:
                    assert kinds[c][slot] == NONE
                    kinds[c][slot] = kind
        for tile in range(len(tiles)):
            v = cover[tile]
            assert v[0][1] == 0 and v[-1][2] == v[-1][3]
            assert all(x[2] == y[1] and x[0] < y[0] for x, y in zip(v, v[1:]))
            if len(v) == 1:
                assert v[0][4] == NONE
                continue
            assert [x[4] for x in v] == [FIRST] + [MIDDLE] * (len(v) - 2) + [LAST]
            assert all(x[5] == 0 for x in v[1:])
            # the join: the first share after the tile's that ends a tile
            c = v[0][0]
            assert kinds[c].count(FIRST) == 1
            end = next(i for i in range(c + 1, shares) if kinds[i][0] == LAST)
            assert end == v[-1][0]
            visited = {x[0] for x in v}
            assert all((kinds[i][0] == MIDDLE) == (i in visited) for i in range(c + 1, end))
