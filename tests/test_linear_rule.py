"""The rule that cuts a linear layer's columns into ranges, compiled for the host."""
import ctypes as C
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_21604_b200", "csrc")


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("rule")
    (d / "rule.cpp").write_text("""#include "linear_rule.h"
extern "C" int ranges(int64_t u, int p, const int* f) { return lq_ranges(u, p, f); }
extern "C" int cluster_ranges(int64_t u, int g, int two) { return lq_cluster_ranges(u, g, two ? LQ_FIT_TWO : LQ_FIT_ONE); }
extern "C" int tensor(int m, int n, int g) { return lq_prefers_tensor(m, n, g); }
""")
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-I" + CSRC, str(d / "rule.cpp"), "-o", str(d / "rule.so")], check=True)
    x = C.CDLL(str(d / "rule.so"))
    x.ranges.argtypes = [C.c_int64, C.c_int, C.POINTER(C.c_int)]
    x.cluster_ranges.argtypes = [C.c_int64, C.c_int, C.c_int]
    return x


@pytest.fixture
def ranges(lib):
    return lambda units, pairs, fit: lib.ranges(units, pairs, (C.c_int * 9)(0, *fit))


WHOLE = [148, 74, 45, 33, 26, 22, 15, 15]


def test_sizes_that_do_not_fit_are_passed_over(ranges):
    assert ranges(20, 216, WHOLE) > 1
    small = [20, 10, 6, 5, 4, 3, 2, 0]                # a part of the GPU without room for eight CTAs side by side
    for units in (1, 2, 3, 20, 500):
        for pairs in (1, 4, 40, 216):
            best = ranges(units, pairs, small)
            assert 1 <= best <= 7
            assert ranges(units, pairs, small[:best - 1] + [0] * (9 - best)) < best       # the next best of the rest
    assert ranges(1, 216, [0, 0, 3, 0, 0, 0, 0, 0]) == 3
    assert ranges(1, 216, [1, 0, 0, 0, 0, 0, 0, 0]) == 1
    assert ranges(1, 216, [0] * 8) == 0


def test_shortest_run(ranges):
    """Rounds of clusters times steps; four pairs of groups a range at least."""
    for units in (1, 5, 20, 112, 216, 10 ** 7):
        for pairs in (1, 3, 4, 8, 15, 16, 32, 112, 216):
            cost = {k: -(-units // WHOLE[k - 1]) * (2 * -(-pairs // k) + 20) for k in range(1, 9) if k == 1 or pairs // k >= 4}
            k = ranges(units, pairs, WHOLE)
            assert cost[k] == min(cost.values()) and k == min(x for x in cost if cost[x] == cost[k])


def test_clusters_run_at_once(lib):
    """More than one range only where every cluster has its place, in ranges of 512 columns or more."""
    two, one = {1: 296, 2: 148, 4: 71, 8: 33}, {1: 148, 2: 74, 4: 33, 8: 15}
    for fit, which in ((two, 1), (one, 0)):
        for units in (1, 15, 16, 33, 34, 71, 72, 74, 75, 148, 149, 10 ** 6):
            for groups in (1, 15, 16, 63, 64, 432):
                best = max(k for k in fit if k == 1 or (units <= fit[k] and -(-groups // k) >= 8))
                assert lib.cluster_ranges(units, groups, which) == best


# features, columns, us on mma.sync and on tcgen05 of 12 rows, and of 8 whose x is too long for one CTA
MEASURED = {12: [(1024, 4096, 5.1, 10.0), (2048, 20480, 19.2, 21.9), (4096, 4096, 7.4, 12.2), (4096, 14336, 17.4, 21.3), (4096, 27648, 27.5, 32.4),
                 (5120, 5120, 13.7, 13.9), (5120, 11008, 23.8, 19.2), (5120, 27648, 50.1, 32.8), (8192, 8192, 17.5, 19.0),
                 (8192, 20480, 37.0, 35.3), (10240, 4096, 17.5, 15.4), (10240, 8192, 31.0, 23.1), (12288, 4096, 17.8, 18.1),
                 (14336, 4096, 17.3, 18.4), (14336, 14336, 49.9, 45.0), (16384, 5120, 21.2, 22.1), (20480, 4096, 31.3, 27.6),
                 (24576, 2560, 21.2, 20.4), (28672, 1024, 11.4, 13.1), (28672, 8192, 56.8, 49.2), (40960, 2560, 34.3, 38.1),
                 (40960, 8192, 94.0, 78.8), (65536, 1024, 22.3, 24.7), (65536, 5120, 73.0, 66.3)],
            8: [(2048, 27648, 19.4, 25.9), (4096, 14336, 13.6, 21.1), (5120, 14336, 20.7, 21.7), (5120, 27648, 36.9, 32.6), (8192, 27648, 37.2, 44.2),
                (10240, 9600, 27.1, 25.0), (10240, 27648, 67.8, 55.8), (14336, 14336, 37.1, 44.8), (20480, 14336, 70.4, 63.5), (28672, 9600, 48.5, 56.7)]}


def test_choice_of_the_kernel(lib):
    for rows, sizes in MEASURED.items():
        for n, k, mma, tensor in sizes:
            assert (tensor if lib.tensor(rows, n, k // 64) else mma) <= 1.05 * min(mma, tensor), (rows, n, k)


def test_choice_of_the_kernel_is_kept(lib):
    """A layer with more columns, or a call with more rows, never leaves tcgen05 again: its scratch does not shrink."""
    for n in list(range(64, 4000, 320)) + list(range(4096, 70000, 1300)):
        last = {4: 0, 12: 0}
        for g in range(1, 600):
            now = {m: lib.tensor(m, n, g) for m in last}
            assert now[12] >= now[4] and all(now[m] >= last[m] for m in now), (n, g)
            last = now
