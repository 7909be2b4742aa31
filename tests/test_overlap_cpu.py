"""Which matrices share memory: the library's own rule, compiled for the host, against the bytes themselves."""
import ctypes
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = """
#include "%s"
using namespace bmgdk;
extern "C" int share(long long a, long long ra, long long wa, long long la, long long b, long long rb, long long wb, long long lb) {
    return share_memory(Region{(void*)a, ra, wa, la}, Region{(void*)b, rb, wb, lb});
}
extern "C" int alike(long long a, long long ra, long long wa, long long la, long long b, long long rb, long long wb, long long lb) {
    return same_or_apart(Region{(void*)a, ra, wa, la}, Region{(void*)b, rb, wb, lb});
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("overlap")
    (d / "overlap.cpp").write_text(SOURCE % os.path.join(ROOT, "paper_2312_08728_b200", "csrc", "overlap.cuh"))
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-ftrapv", "-shared", "-fPIC", "-o", str(d / "overlap.so"), str(d / "overlap.cpp")])
    L = ctypes.CDLL(str(d / "overlap.so"))
    for f in (L.share, L.alike):
        f.argtypes = [ctypes.c_longlong] * 8
    return L


def cells(base, rows, width, ld):
    return {base + i * ld + k for i in range(rows) for k in range(width)}


def test_against_the_bytes(lib):
    rng, seen = random.Random(1), [0, 0]
    for _ in range(40_000):
        both = []
        for _ in range(2):
            width = rng.randint(1, 9)
            both.append((1000 + rng.randint(0, 60), rng.randint(1, 9), width, width + rng.choice([0, 0, 1, 2, 5, 8, 11, 20])))
        if rng.random() < 0.3:      # the same stride, as parts of one buffer have it
            ld = max(both[0][2], both[1][2]) + rng.randint(0, 12)
            both = [(*m[:3], ld) for m in both]
        want = bool(cells(*both[0]) & cells(*both[1]))
        seen[want] += 1
        assert lib.share(*both[0], *both[1]) == want and lib.share(*both[1], *both[0]) == want, both
        x, y = both
        same = x[0] == y[0] and x[1:3] == y[1:3] and (x[3] == y[3] or x[1] == 1)
        assert lib.alike(*x, *y) == (same or not want), both
    assert min(seen) > 5000


def test_nothing_shares_nothing(lib):
    for x in ((0, 3, 4, 8), (1000, 0, 4, 8), (1000, 3, 0, 8)):
        assert not lib.share(*x, 1000, 3, 4, 8) and not lib.share(1000, 3, 4, 8, *x)


def test_large(lib):
    """Halves of rows 2^31 rows long and as far apart as 64 bits go; one value more, and they meet."""
    at, rows = 1 << 40, 2 ** 31 - 1
    for half in (64, 4098, 1 << 24):
        assert not lib.share(at, rows, half, 2 * half, at + half, rows, half, 2 * half)
        assert lib.share(at, rows, half + 1, 2 * half, at + half, rows, half, 2 * half)
        assert lib.share(at, rows, half, 2 * half, at + half + 1, rows, half, 2 * half)     # (the last byte of a row, the first of the next)
        assert not lib.share(at, rows, half, 2 * half, at + half + 1, rows, half - 1, 2 * half)
    # strides without a common measure meet somewhere; two that are multiples of one another need not
    assert lib.share(at, rows, 8, 1001, at + 500, rows, 8, 997)
    assert not lib.share(at, rows, 8, 48, at + 8, rows, 8, 16 * 3 * 7)
    far = 2 ** 62
    assert not lib.share(at, rows, 8, far, at + 8, rows, 8, far) and lib.share(at, rows, 8, far, at + 4, rows, 8, far)
