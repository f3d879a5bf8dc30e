"""The scratch of the attention over a shared context, on the host: a server allocates it once for its
largest batch, so the size may not shrink when a call grows.  Nothing is launched: the calls below name an
output that overlaps an input, which is refused after the scratch has been looked at."""
import random

import pytest

from test_context_op_refusals import INVALID, SHARED, TOO_LARGE, WORKSPACE, b  # noqa: F401

ROW = dict(nkv=8, nq=32, hd=128)


def size(b, c):
    return b.lib.akvs_op_attention_shared_scratch_bytes(c["dtype"], c["R"], c["P"], c["S"], c["cap"], c["nq"], c["nkv"], c["hd"])


def enough(b, c, nbytes, ragged):
    """Whether the call takes a scratch of nbytes."""
    row = c["nkv"] * c["hd"]
    args = {**SHARED, **c, "q_ld": c["nq"] * c["hd"], "c_ld": row, "o_ld": row, "o_seq": row * c["cap"], "scratch_bytes": nbytes,
            "out": SHARED["q"], "off": SHARED["lens"] if ragged else None}
    code = b.lib.akvs_op_attention_shared(*args.values())
    assert code in (INVALID, WORKSPACE)
    return code == INVALID


@pytest.mark.parametrize("R", range(1, 70))
def test_a_scratch_for_the_largest_batch_serves_a_smaller_one(b, R):  # noqa: F811
    """One row each, 32 over 8 heads, 32768 tokens of context: sequences come and go."""
    top = dict(dtype=1, R=70, S=70, P=32768, cap=1024, **ROW)
    assert enough(b, {**top, "R": R, "S": R}, size(b, top), False)
    assert size(b, {**top, "R": R, "S": R}) <= size(b, top)


def test_scratch_grows_with_every_size(b):  # noqa: F811
    rng = random.Random(5)

    def log(hi):
        return int(round(2 ** rng.uniform(0, hi))) - 1

    for _ in range(12000):
        nkv = rng.choice((1, 2, 3, 8, 40))
        c = dict(dtype=rng.choice((0, 1, 2)), R=1 + log(9), S=log(9), P=log(17), cap=log(13), nkv=nkv,
                 nq=nkv * rng.choice((1, 2, 4, 5, 8, 16, 17, 100, 128)), hd=rng.choice((64, 128)))
        small = dict(c, R=rng.randint(1, c["R"]), S=rng.randint(0, c["S"]), P=rng.randint(0, c["P"]), cap=rng.randint(0, c["cap"]))
        have = size(b, c)
        assert size(b, small) <= have, (small, c)
        for ragged in (False, True):
            if small["S"] > 0 and (ragged or small["R"] >= small["S"]):
                assert enough(b, small, have, ragged), (small, c, ragged)


@pytest.mark.parametrize("dtype,nkv", [(0, 8), (1, 8), (2, 1), (0, 1)])
def test_scratch_of_many_rows_is_in_proportion(b, dtype, nkv):  # noqa: F811
    """Many rows need few splits: two parts of each row, or up to five of a single float head."""
    c = dict(dtype=dtype, R=8192, S=1, P=32768, cap=8192, nkv=nkv, nq=4 * nkv, hd=128)
    parts = 5 if dtype == 0 and nkv == 1 else 2
    assert size(b, c) <= parts * 1.05 * 8192 * 4 * nkv * 130 * 4 + 40e6


def test_scratch_of_calls_that_are_too_large(b):  # noqa: F811
    c = dict(dtype=1, R=1 << 30, S=1, P=1 << 20, cap=64, **ROW)
    assert size(b, c) == -1
    assert b.lib.akvs_op_attention_shared(*{**SHARED, **c, "q_ld": 4096, "c_ld": 1024, "o_ld": 1024, "o_seq": 65536}.values()) == TOO_LARGE
