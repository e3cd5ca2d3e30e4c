"""The check of stored codes (codes_check.py) without a GPU: it passes what the 64-bit
form stores and finds one code, scale or earlier row that is off.  And the turns in which
two warps that share a block exchange their maxima, in every order that they can run in."""
from __future__ import annotations

import pytest
import torch

from . import codes_check as check
from . import codes_ref as ref


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("page,r", [(16, 4), (24, 3), (100, 100), (8, 1)])
def test_stored_rows_pass_and_mistakes_do_not(fmt, page, r):
    g = torch.Generator().manual_seed(page)
    lens, counts = [0, 1, r - 1, 2 * r, 77, r // 2], [3 * r + 1, 2, 1, 130, 0, 1]
    B, n = len(lens), max(counts)
    cols = -(-(max(lens) + n) // page) + 1
    table = torch.randperm(B * cols + 3, generator=g)[:B * cols].view(B, cols).to(torch.int32)
    codes = ref.nearest(torch.randint(-100, 100, (B * cols + 3, 2, page, 64), generator=g).double(), fmt)
    scales = torch.exp2(torch.randint(-12, 2, (B * cols + 3, 2, page // r), generator=g).double())
    x = torch.randn(B, n, 2, 64, generator=g, dtype=torch.float64) * check.interleaved_sizes(g, B, n, 2, r)
    before = codes.clone(), scales.clone()
    ref.store(codes, scales, table, lens, x, counts, fmt)
    rows = [(x[b, :c], torch.zeros_like(x[b, :c])) for b, c in enumerate(counts)]
    check.check_stored(before, (codes, scales), table, lens, rows, counts, fmt, "stored")
    step = 1 if fmt == "int8" else 32

    def spoilt(change):
        c, s = codes.clone(), scales.clone()
        change(c, s)
        with pytest.raises(AssertionError):
            check.check_stored(before, (c, s), table, lens, rows, counts, fmt, "spoilt")

    spoilt(lambda c, s: c[int(table[0, 0]), 0, 0, 5].add_(step))
    spoilt(lambda c, s: s[int(table[0, 0]), 1, 0].mul_(2))
    spoilt(lambda c, s: s[int(table[3, 2 * r // page]), 0, 2 * r % page // r].div_(2))
    spoilt(lambda c, s: c[int(table[4, 0]), 0, 0, 1].add_(step))                  # a sequence without new rows
    spoilt(lambda c, s: s[int(table[4, 0]), 1, 0].mul_(2))
    if r > 1:
        spoilt(lambda c, s: c[int(table[5, 0]), 0, 0, 1].add_(step))              # a row before the new one in its block


def foreign_reads(turns, tiles, passes_without_a_head):
    """Two warps of a team with a head in all but the last of a tile's turns, values (no barrier of the CTA at a tile's
    start): each turn writes its maximum to the turn's place, meets the other at the team's barrier, reads both.  In how
    many states that some order of their steps reaches does a warp read a maximum of another turn?"""
    steps, place = [], 0
    for tile in range(tiles):
        for turn in range(turns):
            if turn < turns - 1:
                steps += [("write", place, (tile, turn)), ("meet",), ("read", place, (tile, turn))]
            elif passes_without_a_head:
                steps += [("meet",)]
            place ^= 1
    seen, found = set(), 0
    states = [((0, 0), ((None, None), (None, None)), (False, False))]
    while states:
        state = states.pop()
        if state in seen:
            continue
        seen.add(state)
        at, places, waits = state
        if all(waits):
            states.append(((at[0] + 1, at[1] + 1), places, (False, False)))
            continue
        for w in (0, 1):
            if waits[w] or at[w] == len(steps):
                continue
            what, *rest = steps[at[w]]
            if what == "meet":
                states.append((at, places, tuple(waits[i] or i == w for i in (0, 1))))
                continue
            now = [list(p) for p in places]
            if what == "write":
                now[rest[0]][w] = rest[1]
            elif any(x != rest[1] for x in places[rest[0]]):
                found += 1
                continue
            states.append((tuple(at[i] + (i == w) for i in (0, 1)), tuple(map(tuple, now)), waits))
    assert any(s[0] == (len(steps), len(steps)) for s in seen) or found        # the warps reach the end: nothing waits for good
    return found


@pytest.mark.parametrize("turns", [2, 3, 4, 5])
def test_a_team_meets_in_every_turn(turns):
    assert foreign_reads(turns, 4, True) == 0
    assert foreign_reads(turns, 4, False) > 0    # what a team that does not meet without a head could do
