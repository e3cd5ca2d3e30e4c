"""Attention with accumulated weights where the groups and the block table's rows
are odd: scores that start at odd places of their workspace."""
from __future__ import annotations

import pytest

from .test_gpu_paged import check_attend, pkg  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,D,page,lens", [
    (71, 1, 64, 1, [14, 3, 9, 0]),           # 15 columns of one row
    (71, 1, 64, 5, [310, 1, 299, 17, 33]),   # 63 columns of five
    (34, 2, 128, 3, [16, 7, 0, 15]),         # 7 of three, two KV heads of 17
    (51, 3, 64, 15, [400, 29, 411]),         # 29 of 15, three KV heads of 17
    (25, 1, 128, 1, [70, 70, 2]),            # 71 of one
    (18, 1, 64, 5, [67, 9, 41]),             # an even group over odd rows
    (9, 3, 128, 7, [95, 3, 92]),            # 15 of seven, three heads each
])
def test_attend_odd_groups_over_odd_rows(pkg, dtype, Hq, Hkv, D, page, lens):  # noqa: F811
    assert page * (-(-max(lens) // page) + 1) % 2 == 1
    check_attend(pkg, Hq=Hq, Hkv=Hkv, D=D, dtype=dtype, page=page, lens=lens, track=True, seed=Hq)
