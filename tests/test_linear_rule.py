"""The rule that cuts a linear layer's columns into ranges, compiled for the host."""
import ctypes as C
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_21604_b200", "csrc")


@pytest.fixture(scope="module")
def ranges(tmp_path_factory):
    d = tmp_path_factory.mktemp("rule")
    (d / "rule.cpp").write_text('#include "linear_rule.h"\nextern "C" int ranges(int64_t u, int p, const int* f) { return lq_ranges(u, p, f); }\n')
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-I" + CSRC, str(d / "rule.cpp"), "-o", str(d / "rule.so")], check=True)
    f = C.CDLL(str(d / "rule.so")).ranges
    f.argtypes = [C.c_int64, C.c_int, C.POINTER(C.c_int)]
    return lambda units, pairs, fit: f(units, pairs, (C.c_int * 9)(0, *fit))


WHOLE = [148, 74, 49, 36, 28, 22, 20, 16]


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
