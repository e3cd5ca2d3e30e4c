"""Blocks that two warps share, an odd number of heads to the CTA's two teams, and tiles
one after the other: the team without a head in a tile's last turn starts the next tile
while its warps may be a turn apart, and each still has to take its own block's maximum."""
from __future__ import annotations

import pytest

from .test_gpu_paged_codes_angles import append_and_check, chained

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("turns", [2, 3, 4])
@pytest.mark.parametrize("dtype,D,Hkv,page,r", [("f32", 128, 3, 16, 16), ("f32", 128, 7, 24, 12), ("f32", 64, 5, 32, 32), ("f32", 64, 3, 40, 20)])
def test_a_team_without_a_head_in_the_last_turn(dtype, D, Hkv, page, r, turns):
    """The halves of a block, which the two warps hold, and neighbouring blocks differ by up to 2^9 in size."""
    n = chained(r, dtype, D, turns)
    for seed in range(3):
        append_and_check(dtype=dtype, D=D, fmt="e4m3" if seed else "int8", Hkv=Hkv, Hq=Hkv, page=page, r=r, lens=[0, r // 2, 5, 3 * r - 1],
                         counts=[n, n - r - 1, n // 2, n - 3 * r], gains=seed == 1, seed=10 * r + seed)
