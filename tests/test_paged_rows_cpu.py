"""Divisions and seen rows of the paged operators (csrc/paged_rows.h, compiled here
without CUDA)."""
from __future__ import annotations

import ctypes
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SHIM = """
#include "paged_rows.h"
using namespace prism;
extern "C" int quotient(int n, unsigned d) { return Divisor(d).of(n); }
extern "C" long long wrong(unsigned d, int from, int n) {
    const Divisor by(d);
    for (int i = 0; i < n; ++i) if (by.of(from + i) != (int)((unsigned)(from + i) / d)) return from + i;
    return -1;
}
// places that are seen, in order, into out; -1: a place past the rows, or a row that is seen but not by its tile
extern "C" int seen(int len, int window, int sinks, int tile, int *out) {
    SeenRows r;
    r.set(len, window, sinks);
    int n = 0;
    for (int t = 0; t < r.count(); t += tile) {
        const int first = r.key(t);
        int here = 0;
        for (int i = 0; i < tile; ++i) {
            if (t + i < r.count() && r.key(t + i) != first + i) return -1;
            if (r.sees(first + i)) out[n++] = first + i, ++here;
        }
        if (r.sees_all(first, tile) != (here == tile) || r.sees_any(first, tile) != (here > 0)) return -1;
    }
    return n;
}
extern "C" int blocks(int len, int window, int sinks) {
    SeenRows r;
    r.set(len, window, sinks);
    return (r.count() + kAttendUnit - 1) / kAttendUnit;
}
"""
TOP = 2 ** 31 - 1


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    d = tmp_path_factory.mktemp("rows")
    (d / "shim.cpp").write_text(SHIM)
    so = str(d / "shim.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2602_01762_gb300", "csrc"),
                    str(d / "shim.cpp"), "-o", so], check=True)
    lib = ctypes.CDLL(so)
    lib.wrong.restype = ctypes.c_longlong
    lib.wrong.argtypes = [ctypes.c_uint, ctypes.c_int, ctypes.c_int]
    lib.quotient.argtypes = [ctypes.c_int, ctypes.c_uint]
    return lib


def test_quotients(rule):
    rng = random.Random(1)
    divisors = [*range(1, 300), 1000, 4096, 65535, 65537, 10 ** 6 + 3, 2 ** 30 - 1, 2 ** 30, 2 ** 30 + 1, TOP - 1, TOP]
    divisors += [rng.randint(1, TOP) for _ in range(60)]
    for d in divisors:
        assert rule.wrong(d, 0, 2000) == -1 and rule.wrong(d, TOP - 2000, 2000) == -1, d
        for _ in range(20):
            n = rng.randint(0, TOP)
            k = min(TOP, n // d * d)
            for m in {n, k, max(0, k - 1)}:
                assert rule.quotient(m, d) == m // d, (m, d)


def test_seen_rows_once_each_and_few_blocks(rule):
    out = (ctypes.c_int * 4096)()
    for n in (0, 1, 16, 63, 64, 65, 129, 333):
        for window in (0, 1, 16, 17, 63, 64, 65, 128, 332, 333, TOP):
            for sinks in (0, 1, 16, 63, 64, 65, 130, TOP):
                want = [j for j in range(n) if j < sinks or j >= n - window]
                for tile in (8, 16, 32):
                    count = rule.seen(n, window, sinks, tile, out)
                    assert list(out[:max(count, 0)]) == want and count >= 0, (n, window, sinks, tile)
                assert rule.blocks(n, window, sinks) <= -(-min(sinks, n) // 64) + -(-min(window, n) // 64) + 1
