"""The operators that answer from a context cache at the ends of their types.  Expected values follow
from the definitions by hand."""
import math

import pytest
import torch

from test_gpu_context_ops import TYPES, gen, mass_case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def akvs():
    import paper_2607_21604_b200 as a
    return a


# ------------------------------------------------------------------------- infinite keys that rows see

@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("hd,nq,nkv,R", [(128, 1, 1, 1), (64, 5, 1, 3), (128, 8, 2, 17), (128, 10, 2, 60), (64, 3, 1, 100),
                                         (128, 64, 1, 2), (128, 128, 1, 3)])
def test_mass_of_infinite_keys_that_all_rows_see(akvs, dt, hd, nq, nkv, R):
    """A key whose scores are all -inf has no weight, one that some row scores +inf has an infinite one, a NaN
    stays NaN; the other keys keep their bits.  Stacked rows both fill whole tiles and leave them ragged."""
    q, k, lse, lo, hi = mass_case(nq + R, dt, hd, nq, nkv, R, 300, "all")
    q[..., 0] = -q[..., 0].abs() - 0.5                        # every row scores the same sign on the first value
    old = torch.rand((nkv, 300), generator=gen(2), device="cuda")
    clean = akvs.op_attention_mass(q, k, lse, lo, hi, old)
    kinds = {math.inf: slice(3, None, 13), -math.inf: slice(5, None, 17), math.nan: slice(7, None, 101)}
    for kind, at in kinds.items():
        bad = k.clone()
        bad[at, :, 0] = kind
        got = akvs.op_attention_mass(q, bad, lse, lo, hi, old)
        if kind == math.inf:                                  # q < 0: scores of -inf
            assert torch.equal(got[:, at], old[:, at])
        elif kind == -math.inf:
            assert (got[:, at] == math.inf).all()
        else:
            assert got[:, at].isnan().all()
        rest = torch.ones(300, dtype=torch.bool, device="cuda")
        rest[at] = False
        assert torch.equal(got[:, rest], clean[:, rest])
