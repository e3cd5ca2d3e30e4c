"""Where the paged attention keeps its scores (csrc/paged_scores.h, compiled here
without CUDA): every eight-byte store that the rule allows is aligned, and no
score lies outside the workspace."""
from __future__ import annotations

import ctypes
import itertools
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SHIM = """
#include "paged_scores.h"
extern "C" long long place(int b, int kvh, int h0, int Hkv, int G, long long rows) { return prism::score_place(b, kvh, h0, Hkv, G, rows); }
extern "C" int pairs(unsigned long long first, int heads) { return prism::score_pairs((const float *)first, heads); }
"""
BASE = 1 << 20                            # the workspace's parts start at multiples of 256 bytes


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    d = tmp_path_factory.mktemp("scores")
    (d / "shim.cpp").write_text(SHIM)
    so = str(d / "shim.so")
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2602_01762_gb300", "csrc"),
                    str(d / "shim.cpp"), "-o", so], check=True)
    lib = ctypes.CDLL(so)
    lib.place.restype = ctypes.c_longlong
    lib.place.argtypes = [ctypes.c_int] * 5 + [ctypes.c_longlong]
    lib.pairs.argtypes = [ctypes.c_ulonglong, ctypes.c_int]
    return lib


def test_pair_stores_are_aligned(rule):
    for G, Hkv, rows in itertools.product([*range(1, 40), 71, 79, 128], (1, 2, 3), (1, 2, 15, 16, 75, 64)):
        B, tile = 3, 4 if G <= 4 else 8 if G <= 8 else 16
        taken = set()
        for b, kvh, h0 in itertools.product(range(B), range(Hkv), range(0, G, tile)):
            heads, first = min(tile, G - h0), rule.place(b, kvh, h0, Hkv, G, rows)
            where = (G, Hkv, rows, b, kvh, h0)
            places = range(first, first + rows * heads)
            assert 0 <= first and places.stop <= B * Hkv * G * rows and not taken.intersection(places), where
            taken.update(places)
            allowed = rule.pairs(BASE + 4 * first, heads)
            if allowed:
                assert all((BASE + 4 * (first + j * heads + h)) % 8 == 0 for j in range(min(rows, 4)) for h in range(0, heads, 2)), where
            assert bool(allowed) == (heads % 2 == 0 and first % 2 == 0), where
        assert len(taken) == B * Hkv * G * rows


def test_an_odd_group_over_odd_rows_starts_at_odd_scores(rule):
    """71 query heads on one KV head, pages of one row, 15 columns: the second sequence's first tile holds 16 heads and starts
    four bytes off."""
    first = rule.place(1, 0, 0, 1, 71, 15)
    assert first == 71 * 15 and not rule.pairs(BASE + 4 * first, 16)
    assert rule.pairs(BASE, 16)
