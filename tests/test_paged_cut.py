"""The cut of the paged attention's line, restated on the CPU: every tile of every portion belongs to exactly one part,
the parts of a portion are neighbours and are the ones that the join counts, and no part is without a tile."""
import random

import pytest


def part_begin(total, parts, i):
    return total // parts * i + min(i, total % parts)


def part_of(total, parts, u):
    size, longer = total // parts, total % parts
    return u // (size + 1) if u < longer * (size + 1) else longer + (u - longer * (size + 1)) // size


def tiles_of_part(heads, subs, per_tile, total, parts, i):
    """What a CTA walks: (head, portion, tile) of its part, from the head that its first box is in."""
    unit, end = part_begin(total, parts, i), part_begin(total, parts, i + 1)
    before, h = 0, 0
    while before + heads[h] * subs <= unit:
        before += heads[h] * subs
        h += 1
    sub, k = (unit - before) // heads[h], (unit - before) % heads[h]
    at, t0, walked = before + sub * heads[h], -(-k // per_tile), []
    while at < end and h < len(heads):
        n = -(-heads[h] // per_tile)
        while sub < subs and at < end and n:
            walked += [(h, sub, t) for t in range(t0, min(n, -(-(end - at) // per_tile)))]
            sub, t0, at = sub + 1, 0, at + heads[h]
        h, sub = h + 1, 0
    return walked


@pytest.mark.parametrize("seed", range(8))
def test_every_tile_is_in_one_part(seed):
    rng = random.Random(seed)
    for _ in range(400):
        per_tile, subs = rng.choice([2, 4]), rng.choice([1, 1, 2, 3])
        heads = [rng.choice([0, 1, 2, 3, 5, 7, 8, 13, 40]) for _ in range(rng.randint(1, 30))]
        total = sum(heads) * subs
        if total == 0:
            continue
        parts = min(rng.choice([1, 2, 5, 17, 60]), max(min(total, 1), total // per_tile))
        owner = {}
        for i in range(parts):
            walked = tiles_of_part(heads, subs, per_tile, total, parts, i)
            assert walked
            for tile in walked:
                assert tile not in owner
                owner[tile] = i
        at = 0
        for h, boxes in enumerate(heads):
            for sub in range(subs):
                n = -(-boxes // per_tile)
                if n:
                    own = [owner.pop((h, sub, t)) for t in range(n)]
                    first, last = part_of(total, parts, at), part_of(total, parts, at + (n - 1) * per_tile)
                    assert own == sorted(own) and set(own) == set(range(first, last + 1))
                at += boxes
        assert not owner


def test_parts_of_a_line():
    for total in range(1, 60):
        for parts in range(1, total + 1):
            begins = [part_begin(total, parts, i) for i in range(parts + 1)]
            assert begins[0] == 0 and begins[-1] == total
            for i in range(parts):
                assert all(part_of(total, parts, u) == i for u in range(begins[i], begins[i + 1]))


def find_unit(units, seg_heads, u):
    """The head that unit u is in and the units before it, searched in segments of heads, then in 32 heads at a time; reads
    of heads that are not there fail."""
    at, seg, heads = 0, 0, len(units)
    while True:
        sums = [sum(units[i * seg_heads: (i + 1) * seg_heads]) if i * seg_heads < heads else 0 for i in range(seg, seg + 32)]
        upto = [sum(sums[: i + 1]) for i in range(32)]
        past = [i for i in range(32) if at + upto[i] > u]
        if past:
            at += upto[past[0]] - sums[past[0]]
            seg += past[0]
            break
        at += upto[31]
        if (seg + 32) * seg_heads >= heads:
            return heads, at
        seg += 32
    h = seg * seg_heads
    while h < heads:
        mine = [units[h + i] if h + i < heads else 0 for i in range(32)]
        upto = [sum(mine[: i + 1]) for i in range(32)]
        past = [i for i in range(32) if at + upto[i] > u]
        if past:
            return h + past[0], at + upto[past[0]] - mine[past[0]]
        at += upto[31]
        h += 32
    return heads, at


@pytest.mark.parametrize("heads,seg_heads", [(1, 32), (4, 32), (32, 32), (33, 32), (1024, 32), (1025, 32), (3000, 64)])
def test_the_search_for_a_unit_ends_and_finds_it(heads, seg_heads):
    rng = random.Random(heads)
    for units in ([0] * heads, [1] * heads, [rng.choice([0, 0, 1, 5]) for _ in range(heads)]):
        total = sum(units)
        for u in {0, total // 3, total - 1, total, total + 7}:
            h, before = find_unit(units, seg_heads, u)
            if 0 <= u < total:
                assert before <= u < before + units[h] and before == sum(units[:h])
            elif u >= total:
                assert (h, before) == (heads, total)
