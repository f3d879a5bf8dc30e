"""The operators that answer from a context cache where a CTA or a warp does more than one piece of work,
and how close they come to their 64-bit forms on the whole."""
import math

import pytest
import torch

from test_gpu_context_ops import (BF16, F16, F32, TYPES, check_mass, check_norm, check_shared, gen, ints, mass_case, rnd,
                                  shared_case, shared_ref)

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def akvs():
    import paper_2607_21604_b200 as a
    return a


# ------------------------------------------------------------------------- more work than SMs

@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("hd,nq,nkv,R,T,kind", [
    (128, 32, 8, 17, 9001, "ragged"), (128, 16, 8, 60, 20011, "causal"), (64, 8, 8, 3, 12000, "all"), (64, 15, 5, 40, 25000, "ragged"),
    (128, 40, 8, 100, 9001, "ragged"), (64, 16, 8, 70, 9001, "causal"), (128, 8, 8, 400, 6000, "all"), (128, 14, 2, 150, 40003, "ragged")])
def test_mass_of_more_keys_than_the_device_holds_at_once(akvs, dt, hd, nq, nkv, R, T, kind):
    """Up to 128 stacked rows and more: CTAs walk several stretches of 256 keys, and several heads."""
    assert -(-T // 256) * nkv > 148
    q, k, lse, lo, hi = mass_case(R + T, dt, hd, nq, nkv, R, T, kind)
    old = torch.rand((nkv, T), generator=gen(1), device="cuda")
    got = akvs.op_attention_mass(q, k, lse, lo, hi, old)
    check_mass(got, q, k, lse, lo, hi, old)
    akvs.op_attention_mass(q, k, lse, lo, hi, old, old)
    assert torch.equal(got, old)


@pytest.mark.parametrize("dt,hd,n,nq,nkv", [
    (F16, 128, 12000, 40, 8), (BF16, 128, 5000, 40, 8), (BF16, 64, 5000, 37, 4), (F32, 128, 5000, 21, 2), (F16, 32, 9500, 33, 1),
    (F32, 256, 9500, 5, 0), (BF16, 256, 9501, 0, 7)])
def test_norm_rope_of_many_rows(akvs, dt, hd, n, nq, nkv):
    """Warps that walk several groups of heads, the last of them ragged; in place, in the columns of one
    tensor."""
    per = 32 // (hd // 2 // (4 if dt == F32 else 8))
    assert n * -(-(-(-(nq + nkv) // per)) // 2) >= 148 * 64
    g = gen(n + hd)
    qkv = rnd(g, n, nq + 2 * nkv + 1, hd, dt=dt, scale=3.0)
    q, k = qkv[:, :nq], qkv[:, nq:nq + nkv]
    gq, gk = rnd(g, hd) + 1, rnd(g, hd) * 0.1 + 1
    pos = torch.randint(0, 2 ** 31 - 1, (n,), generator=g, device="cuda", dtype=torch.int32)
    before = qkv.clone()
    oq, ok = akvs.op_qk_norm_rope(q, k, gq, gk, pos, 1e-6, 1e4)
    assert torch.equal(qkv, before)
    for got, x, gain in ((oq, q, gq), (ok, k, gk)):
        for h in range(x.shape[1]):                           # a head at a time: the 64-bit form is large
            check_norm(got[:, h:h + 1], x[:, h:h + 1], gain, pos, 1e-6, 1e4)
    akvs.op_qk_norm_rope(q, k, gq, gk, pos, 1e-6, 1e4, q, k)
    assert torch.equal(q, oq) and torch.equal(k, ok) and torch.equal(qkv[:, nq + nkv:], before[:, nq + nkv:])


# ------------------------------------------------------------------------- clamped lengths and offsets

@pytest.mark.parametrize("dt", TYPES)
def test_shared_clamped_offsets_give_the_rows_that_are_left(akvs, dt):
    """Sequences of rows [0, 2), [2, 4), none and [3, 8) after clamping: row 3 belongs to two of them, all
    others have one result."""
    q, ck, cv, sk, sv, _, _ = shared_case(5, dt, 128, 4, 2, 60, 32, [32, 32, 32, 32], [2, 2, 2, 2])
    sk, sv = torch.nan_to_num(sk), torch.nan_to_num(sv)
    got = akvs.op_attention_shared(q, ck, cv, sk, sv, ints([99, -4, 32, 2 ** 31 - 1]), ints([-3, 2, 4, 3, 400]))
    lens, off = [32, 0, 32, 32], [0, 2, 4, 4, 8]
    want = akvs.op_attention_shared(q, ck, cv, sk, sv, ints(lens), ints(off))
    for x, y in zip(got, want):
        x[3] = y[3]
    check_shared(got, q, ck, cv, sk, sv, lens, off)


# ------------------------------------------------------------------------- error on the whole

@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("S", [1, 4, 40])
def test_shared_error_on_the_whole(akvs, dt, hd, S):
    """Root mean squares, which no single worst case hides.  Float: a score is a sum of hd products whose
    partial sums stay below 2 sqrt(hd); their roundings of 2^-24 add up like independent ones to 2^-19.5, the
    exponent's argument (below 16) adds 2^-20 and exp2 2^-22: 2^-19 of the output, and a factor of 2 for the
    sums.  16 bits, up to 16 stacked rows: probabilities carry their remainder, so that only the output's own
    rounding is left (5 % more).  More rows: probabilities are rounded like the output is, independently:
    sqrt(2) times the output's rounding (6 % more)."""
    lens = [(17 * s) % 60 + 3 for s in range(S)]
    c = shared_case(S + hd, dt, hd, 16, 4, 3000, 64, lens, [1] * S)
    out, lse = akvs.op_attention_shared(*c[:5], ints(lens))
    again = akvs.op_attention_shared(*c[:5], ints(lens))
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
    ref = shared_ref(*c)[0]

    def rms(x):
        return float(x.square().mean().sqrt())

    err, rounding = rms(out.double() - ref), rms(ref.to(dt).double() - ref)
    bound = 2.0 ** -18 * rms(ref) if dt == F32 else (1.05 if 4 * S <= 16 else 1.5) * rounding
    assert err <= bound, (err, bound, math.log2(err / rms(ref)))


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("S,behind", [(1, 1), (2, 40), (50, 10), (50, 300)])
def test_shared_rows_behind_the_last_sequence(akvs, dt, S, behind):
    """One row each and rows that belong to no sequence, NaN here: those stay as they were, and the others
    are what they are without them, to the bit."""
    lens = [(7 * s) % 30 + 1 for s in range(S)]
    q, ck, cv, sk, sv, _, _ = shared_case(S, dt, 128, 8, 2, 2000, 600, lens, [1] * S)
    more = torch.cat([q, torch.full((behind, 8, 128), math.nan, device="cuda", dtype=dt)])
    out, lse = torch.full_like(more, 9.0), torch.full(more.shape[:2], 9.0, device="cuda")
    scratch = akvs.op_attention_shared_scratch(dt, S + behind + 5, 2500, S + 2, 700, 8, 2, 128)       # of a larger call
    akvs.op_attention_shared(more, ck, cv, sk, sv, ints(lens), None, out, lse, scratch)
    want = akvs.op_attention_shared(q, ck, cv, sk, sv, ints(lens))
    assert torch.equal(out[:S], want[0]) and torch.equal(lse[:S], want[1])
    assert (out[S:] == 9).all() and (lse[S:] == 9).all()


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("rows,cap", [([16], 2500), ([30, 2], 1300), ([64], 900), ([1, 1, 70, 1, 1, 1], 400)])
def test_shared_many_new_rows_over_long_slots(akvs, dt, rows, cap):
    """Few sequences of many rows each over many own tokens, or one such among single rows."""
    lens = [cap - 3 * s for s in range(len(rows))]
    c = shared_case(cap, dt, 128, 8, 2, 40, cap, lens, rows)
    check_shared(akvs.op_attention_shared(*c[:5], ints(lens), ints(c[6])), *c)
