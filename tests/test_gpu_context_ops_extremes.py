"""The operators that answer from a context cache at the ends of their types.  Expected values follow
from the definitions by hand."""
import math

import pytest
import torch

from test_gpu_context_ops import BF16, F16, F32, TINY, TYPES, gen, half, ints, mass_case, rnd, shared_case

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


# ------------------------------------------------------------------------- scores far from zero

# (type, values of q and k): sums of their products are exact, and the scores are about -2e33, +-1.5e12 and
# +-1.5e9 in units of log2
FAR = [(F32, 2.0 ** 50, -1.375 * 2.0 ** 60), (BF16, 2.0 ** 50, -1.375 * 2.0 ** 60), (F32, 2.0 ** 20, 1.375 * 2.0 ** 20),
       (BF16, 2.0 ** 20, 1.375 * 2.0 ** 20), (BF16, 2.0 ** 20, -1.375 * 2.0 ** 20), (F16, 2.0 ** 15, 1.375 * 2.0 ** 15),
       (F16, 2.0 ** 15, -1.375 * 2.0 ** 15)]
WIDTH = 8                                                     # values of a row that are not zero


def far_keys(n, nkv, hd, dt, kv):
    """Keys of one score, but every third of a score so much lower that it has no weight."""
    k = torch.zeros((n, nkv, hd), dtype=dt, device="cuda")
    k[..., :WIDTH] = kv
    k[::3, :, :WIDTH] = kv / 2 if kv > 0 else max(2 * kv, torch.finfo(dt).min)
    return k


def check_far(o, v, dt):
    """The mean of the values that the rows see: v [n][n_kv][hd] with no weight on every third of each part."""
    ref = v.double().mean(0).repeat_interleave(o.shape[1] // v.shape[1], 0)
    mag = v.double().abs().mean(0).repeat_interleave(o.shape[1] // v.shape[1], 0)
    # equal weights, which may be rounded once to the 16-bit type; sums of n terms in float
    tol = half(dt) * ref.abs() + (2.0 ** -16 + (0.0 if dt == F32 else half(dt))) * mag + TINY[dt]
    assert ((o.double() - ref).abs() <= tol).all(), (o.double() - ref).abs().max()


def weighty(x):
    keep = torch.ones(x.shape[0], dtype=torch.bool, device="cuda")
    keep[::3] = False
    return x[keep]


@pytest.mark.parametrize("dt,qv,kv", FAR)
@pytest.mark.parametrize("S", [1, 3, 9, 40])
@pytest.mark.parametrize("hd", [64, 128])
def test_shared_attention_of_far_scores(akvs, dt, qv, kv, S, hd):
    """The softmax depends on differences of scores alone, however far they are from zero."""
    g = gen(S + hd)
    nq, nkv, P, cap = 8, 2, 600, 45
    q = torch.zeros((S, nq, hd), dtype=dt, device="cuda")
    q[..., :WIDTH] = qv
    ck, cv = far_keys(P, nkv, hd, dt, kv), rnd(g, P, nkv, hd, dt=dt)
    one = far_keys(cap, nkv, hd, dt, kv)
    sk, sv = one.expand(S, cap, nkv, hd).contiguous(), rnd(g, 1, cap, nkv, hd, dt=dt).expand(S, cap, nkv, hd).contiguous()
    out, lse = akvs.op_attention_shared(q, ck, cv, sk, sv, ints([cap] * S))
    v = torch.cat([weighty(cv), weighty(sv[0])])
    check_far(out, v, dt)
    top = qv * kv * WIDTH / math.sqrt(hd)
    want = top + math.log(v.shape[0])
    # seven roundings of up to 2^-24: log2(e), the root and its quotient, the product with the score, the sum
    # with log2 of the row's sum, log(2) and its product
    assert ((lse.double() - want).abs() <= 2.0 ** -21 * abs(want)).all()


@pytest.mark.parametrize("dt,qv,kv", FAR)
def test_attention_of_far_scores(akvs, dt, qv, kv):
    g = gen(3)
    nq, nkv, hd, n = 8, 2, 128, 400
    q = torch.zeros((50, nq, hd), dtype=dt, device="cuda")
    q[..., :WIDTH] = qv
    k, v = far_keys(n, nkv, hd, dt, kv), rnd(g, n, nkv, hd, dt=dt)
    lo, hi = ints([0] * 50), ints([n - 1] * 50)
    check_far(akvs.op_attention(q, k, v, lo, hi), weighty(v), dt)


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("S", [1, 40])
@pytest.mark.parametrize("where", ["context", "own"])
def test_shared_infinite_values_show(akvs, dt, hd, S, where):
    """An infinity in a V that a row sees gives infinity or NaN in its column, and leaves the others alone."""
    c = shared_case(S + hd, dt, hd, 8, 2, 700, 40, [40] * S, [1] * S)
    q, ck, cv, sk, sv, lens, off = c
    clean = akvs.op_attention_shared(q, ck, cv, sk, sv, ints(lens))
    for bad in (math.inf, -math.inf):
        (cv[300] if where == "context" else sv[:, 7])[..., 5] = bad
        out, lse = akvs.op_attention_shared(q, ck, cv, sk, sv, ints(lens))
        assert not out[..., 5].isfinite().any()
        out[..., 5] = clean[0][..., 5]
        assert torch.equal(out, clean[0]) and torch.equal(lse, clean[1])


@pytest.mark.parametrize("S", [1, 40])
def test_shared_largest_float16_values_stay_finite(akvs, S):
    """The mean of the type's largest value is that value, give or take a rounding of the weights."""
    q, ck, cv, sk, sv, lens, _ = shared_case(S, F16, 128, 8, 2, 700, 40, [40] * S, [1] * S)
    cv.fill_(65504), sv.fill_(65504)
    out, _ = akvs.op_attention_shared(q, ck, cv, sk, sv, ints(lens))
    assert out.isfinite().all() and (out >= 65504 * (1 - 2.0 ** -10)).all()


LIGHT = -26                                                   # log2 of a light key's weight


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("hd,S,P,cap", [(64, 1000, 30000, 0), (128, 1000, 30000, 0), (128, 3, 30000, 0), (64, 200, 0, 4000), (128, 40, 20, 15000)])
def test_shared_one_key_above_many_light_ones(akvs, dt, hd, S, P, cap):
    """A key that draws nearly all weight and whose V is zero: what remains are the small weights of all
    others.  float16 holds a weight to 2^-32 of the row's largest."""
    nq, nkv = 16, 4
    light = round(LIGHT * math.log(2) * math.sqrt(hd)) / 4    # exact in every type

    def keys(n, first, heavy):
        k, v = torch.zeros((n, nkv, hd), dtype=dt, device="cuda"), rnd(gen(n), n, nkv, hd, dt=dt).abs()
        k[..., 0] = light
        if heavy:
            k[first], v[first] = 0, 0
        return k, v

    q = torch.zeros((S, nq, hd), dtype=dt, device="cuda")
    q[..., 0] = 4
    ck, cv = keys(P, 40, P > 20)
    k1, v1 = keys(cap, 40, P <= 20)
    sk, sv = (x[None].expand(S, cap, nkv, hd).contiguous() for x in (k1, v1))
    out, lse = akvs.op_attention_shared(q, ck, cv, sk, sv, ints([cap] * S))
    w = math.exp(4 * light / math.sqrt(hd))
    total, v = 1 + (P + cap - 1) * w, torch.cat([cv, v1]).double()
    ref = (v.sum(0) * w / total).repeat_interleave(nq // nkv, 0)
    held = 2.0 ** -32 * v.abs().sum(0).repeat_interleave(nq // nkv, 0) if dt == F16 else 0.0
    # scores of 18 are right to 2^-19; a weight may be rounded once to the 16-bit type; n additions to the
    # row's sum and n to the output, each rounded by up to 2^-24 of the sum
    n = P + cap
    tol = half(dt) * ref + (2.0 ** -18 + 2 * n * 2.0 ** -24 + (0 if dt == F32 else half(dt))) * ref + held + TINY[dt]
    assert ((out.double() - ref).abs() <= tol).all(), ((out.double() - ref).abs() / ref).max()
    assert (lse.double() - math.log(total)).abs().max() <= n * 2.0 ** -24 + 2.0 ** -20
