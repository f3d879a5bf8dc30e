"""The operators that answer from a context cache against plain forms in 64 bits.

Tolerances count roundings.  eps / 2 of the output type is one rounding of a result.  A float dot
product of n terms is off by at most n * 2^-23 of the sum of its terms' magnitudes (an addition
rounds by 2^-24 and the tensor cores may truncate, which doubles it); a score that is off by d
changes its weight by a factor of at most 1 + 2d for small d; exp2 and its argument's rounding add
under 2^-17 for scores below 64.  On the tensor cores a probability may be rounded once to the
16-bit type: eps / 2 of the sum of p |v|.
"""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]
TINY = {F32: 0.0, BF16: 0.0, F16: 2.0 ** -25}        # half a step of the smallest float16 numbers


@pytest.fixture(scope="module")
def akvs():
    import paper_2607_21604_b200 as a
    return a


def half(dt):
    return torch.finfo(dt).eps / 2


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def rnd(g, *shape, dt=F32, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dt)


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


# ------------------------------------------------------------------------- norm and rotation

def norm_rope_ref(x, gain, pos, eps, base):
    hd = x.shape[-1]
    x = x.double()
    y = x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * gain.double()
    a = pos.double()[:, None, None] * base ** (-2.0 * torch.arange(hd // 2, device=x.device, dtype=torch.float64) / hd)
    u, v = y[..., :hd // 2], y[..., hd // 2:]
    c, s = a.cos(), a.sin()
    both = (u.abs() + v.abs()).repeat(1, 1, 2)
    return torch.cat([u * c - v * s, v * c + u * s], -1), both


def check_norm(got, x, gain, pos, eps, base):
    ref, both = norm_rope_ref(x, gain, pos, eps, base)
    # the mean of squares: 16 roundings of 2^-24, halved by the root; rsqrt, two gains, two products and
    # a sum: under 2^-20 of |u| + |v| with the cosine's own 2^-23; angles are right to 2^-22 up to 2^31
    tol = half(got.dtype) * ref.abs() + 2.0 ** -20 * both + TINY[got.dtype]
    assert ((got.double() - ref).abs() <= tol).all(), ((got.double() - ref).abs() - tol).max()


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("hd", [32, 64, 128, 256])
@pytest.mark.parametrize("n,nq,nkv", [(1, 32, 8), (1, 1, 1), (37, 5, 1), (300, 40, 8), (2, 3, 0), (2, 0, 3)])
def test_norm_rope(akvs, dt, hd, n, nq, nkv):
    g = gen(n + hd)
    qkv = rnd(g, n, nq + 2 * nkv, hd, dt=dt, scale=3.0)
    q, k = qkv[:, :nq], qkv[:, nq:nq + nkv]
    if n > 2:
        q[1, 0] = 0                                           # a head of zeros: eps keeps it zero
        q[2] *= 1e-3
    gq, gk = rnd(g, hd) + 1, rnd(g, hd) * 0.1 + 1
    pos = torch.randint(0, 20000, (n,), generator=g, device="cuda", dtype=torch.int32)
    pos[0] = [0, 2 ** 31 - 1, -5, 1000003][(n + hd // 32) % 4]
    before = qkv.clone()
    oq, ok = akvs.op_qk_norm_rope(q, k, gq, gk, pos, 1e-6, 1e4)
    assert torch.equal(qkv, before)
    check_norm(oq, q, gq, pos, 1e-6, 1e4)
    check_norm(ok, k, gk, pos, 1e-6, 1e4)
    # in place, in the columns of one tensor: the same bits, and the third range untouched
    akvs.op_qk_norm_rope(q, k, gq, gk, pos, 1e-6, 1e4, q, k)
    assert torch.equal(q, oq) and torch.equal(k, ok)
    assert torch.equal(qkv[:, nq + nkv:], before[:, nq + nkv:])


def test_norm_rope_agrees_with_rope_and_other_bases(akvs):
    """Unit gains on unit-norm heads leave the rotation alone, at another base."""
    g = gen(4)
    x = rnd(g, 50, 4, 128)
    x = x / x.double().square().mean(-1, keepdim=True).sqrt().float()
    pos = torch.arange(50, device="cuda", dtype=torch.int32) * 241
    one = torch.ones(128, device="cuda")
    q, _ = akvs.op_qk_norm_rope(x, x[:, :1], one, one, pos, 0.0, 5e5)
    want = akvs.op_rope(x.clone(), pos, 5e5)
    assert (q - want).abs().max() <= 2.0 ** -20 * 2 * x.abs().max()


# ------------------------------------------------------------------------- shared attention

def shared_ref(q, ck, cv, sk, sv, lens, off):
    """out, lse, sum of p |v|, and the largest error a score of the row may have."""
    R, nq, hd = q.shape
    nkv, P = ck.shape[1], ck.shape[0]
    gr, f64 = nq // nkv, torch.float64
    out, lse = torch.zeros((R, nq, hd), dtype=f64, device="cuda"), torch.full((R, nq), -math.inf, dtype=f64, device="cuda")
    mag, err = torch.zeros_like(out), torch.zeros_like(lse)
    for s in range(len(lens)):
        for r in range(off[s], off[s + 1]):
            own = min(max(lens[s] - (off[s + 1] - 1 - r), 0), sk.shape[1])
            k, v = torch.cat([ck, sk[s, :own]]).double(), torch.cat([cv, sv[s, :own]]).double()
            if k.shape[0] == 0:
                continue
            for h in range(nkv):
                x = q[r, h * gr:(h + 1) * gr].double()
                y = x @ k[:, h].T / math.sqrt(hd)
                z = torch.logsumexp(y, -1)
                p = (y - z[:, None]).exp()
                out[r, h * gr:(h + 1) * gr] = p @ v[:, h]
                mag[r, h * gr:(h + 1) * gr] = p @ v[:, h].abs()
                lse[r, h * gr:(h + 1) * gr] = z
                err[r, h * gr:(h + 1) * gr] = (x.abs() @ k[:, h].abs().T).amax(-1) / math.sqrt(hd) * hd * 2.0 ** -23
    return out, lse, mag, err


def check_shared(got, q, ck, cv, sk, sv, lens, off):
    (o, l), dt = got, q.dtype
    ref, lse, mag, err = shared_ref(q, ck, cv, sk, sv, lens, off)
    used = slice(off[0], off[-1])
    o, l, ref, lse, mag, err = (x[used] for x in (o, l, ref, lse, mag, err))
    none = lse == -math.inf
    assert torch.equal(l == -math.inf, none) and (o[none] == 0).all()
    rounded = 0.0 if dt == F32 else half(dt)
    tol = half(dt) * ref.abs() + (2 * err[..., None] + 2.0 ** -16 + rounded) * mag + TINY[dt]
    assert ((o.double() - ref).abs() <= tol).all(), ((o.double() - ref).abs() / tol).max()
    d = (l.double() - lse)[~none].abs()
    assert (d <= (err + 2.0 ** -18 + 2.0 ** -22 * lse.abs())[~none]).all()


def shared_case(seed, dt, hd, nq, nkv, P, cap, lens, rows, behind=0):
    g = gen(seed)
    off = [0] + list(np.cumsum(rows))
    R, S = off[-1] + behind, len(lens)
    q = rnd(g, R, nq, hd, dt=dt, scale=2.0)
    ck, cv = rnd(g, P, nkv, hd, dt=dt), rnd(g, P, nkv, hd, dt=dt)
    sk, sv = rnd(g, S, cap, nkv, hd, dt=dt), rnd(g, S, cap, nkv, hd, dt=dt)
    for s, n in enumerate(lens):                              # what is not filled is anything
        sk[s, max(n, 0):] = math.nan
        sv[s, max(n, 0):] = math.inf if s % 2 else math.nan
    return q, ck, cv, sk, sv, lens, [int(x) for x in off]


HEADS = [(4, 2), (5, 1), (8, 1), (16, 2), (3, 3), (40, 2)]


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("nq,nkv", HEADS)
@pytest.mark.parametrize("P", [0, 1, 129, 700])
def test_shared_one_row_each(akvs, dt, hd, nq, nkv, P):
    lens = [0, 1, 15, 16, 17, 40, 64, 65, 100]
    c = shared_case(P + nq, dt, hd, nq, nkv, P, 100, lens, [1] * len(lens))
    got = akvs.op_attention_shared(*c[:5], ints(lens))
    check_shared(got, *c)
    again = akvs.op_attention_shared(*c[:5], ints(lens))
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("hd,nq", [(128, 128), (64, 100), (128, 65)])
def test_shared_many_heads_per_kv_head(akvs, dt, hd, nq):
    """One query row alone fills a tile or leaves it ragged."""
    lens = [9, 0, 33]
    c = shared_case(nq, dt, hd, nq, 1, 300, 40, lens, [1, 1, 1])
    check_shared(akvs.op_attention_shared(*c[:5], ints(lens)), *c)
    c = shared_case(nq + 1, dt, hd, nq, 1, 0, 40, lens, [2, 1, 4], behind=1)
    check_shared(akvs.op_attention_shared(*c[:5], ints(lens), ints(c[6])), *c)


@pytest.mark.parametrize("dt", TYPES)
def test_shared_without_any_key(akvs, dt):
    """Neither context nor room for own tokens: zeros, and a log-sum-exp of -inf."""
    g = gen(1)
    q, none, room = rnd(g, 4, 8, 128, dt=dt), rnd(g, 0, 2, 128, dt=dt), rnd(g, 3, 0, 2, 128, dt=dt)
    out, lse = torch.full_like(q, 5.0), torch.full((4, 8), 5.0, device="cuda")
    akvs.op_attention_shared(q, none, none, room, room, ints([0, 0, 0]), None, out, lse)
    assert (out[:3] == 0).all() and (lse[:3] == -math.inf).all() and (out[3] == 5).all() and (lse[3] == 5).all()
    # a context alone
    ctx = rnd(g, 70, 2, 128, dt=dt)
    got = akvs.op_attention_shared(q[:3], ctx, ctx.flip(0), room, room, ints([0, 0, 0]))
    check_shared(got, q[:3], ctx, ctx.flip(0), room, room, [0, 0, 0], [0, 1, 2, 3])


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("hd,nq,nkv", [(128, 8, 2), (64, 5, 1), (128, 16, 1)])
@pytest.mark.parametrize("P", [0, 50, 1000])
def test_shared_ragged_rows(akvs, dt, hd, nq, nkv, P):
    """Sequences of several new rows, of none, with fewer own tokens than rows, and rows behind the
    last sequence, which stay as they were."""
    rows, lens = [3, 0, 1, 20, 7, 2], [3, 5, 60, 33, 4, 0]
    c = shared_case(7 * P + nq, dt, hd, nq, nkv, P, 64, lens, rows, behind=4)
    q, ck, cv, sk, sv, _, off = c
    out, lse = torch.full_like(q, 77.0), torch.full(q.shape[:2], 55.0, device="cuda")
    got = akvs.op_attention_shared(q, ck, cv, sk, sv, ints(lens), ints(off), out, lse)
    assert got[0] is out
    check_shared(got, *c)
    assert (out[off[-1]:] == 77).all() and (lse[off[-1]:] == 55).all()


@pytest.mark.parametrize("dt", [F32, BF16, F16])
@pytest.mark.parametrize("hd", [64, 128])
def test_shared_later_tokens_never_reach_a_row(akvs, dt, hd):
    """The K and V of a sequence's later rows may be NaN or infinite: the rows before do not see them."""
    n, length = 21, 53
    c = shared_case(3, dt, hd, 6, 2, 40, 64, [length], [n])
    q, ck, cv, sk, sv, lens, off = c
    clean = akvs.op_attention_shared(q, ck, cv, sk, sv, ints(lens), ints(off))
    for bad in (math.nan, math.inf):
        for first in (length - n + 1, length - 3, length - 1):
            k2, v2 = sk.clone(), sv.clone()
            k2[0, first:length], v2[0, first:length] = bad, bad
            got = akvs.op_attention_shared(q, ck, cv, k2, v2, ints(lens), ints(off))
            seen = first - (length - n)                       # rows that see none of the bad tokens
            assert torch.equal(got[0][:seen], clean[0][:seen]) and torch.equal(got[1][:seen], clean[1][:seen])
            assert not got[0][seen:].isfinite().any()


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("S,cap", [(1, 3000), (2, 1500), (3, 700)])
def test_shared_long_own_tokens(akvs, dt, S, cap):
    """Few sequences with long slots: a cluster shares each sequence's tokens."""
    lens = [cap - 1 - 600 * s for s in range(S)]
    c = shared_case(S, dt, 128, 8, 2, 300, cap, lens, [1] * S)
    check_shared(akvs.op_attention_shared(*c[:5], ints(lens)), *c)
    rows = [4, 1, 9][:S]
    c = shared_case(S + 9, dt, 64, 4, 1, 0, cap, lens, rows)
    check_shared(akvs.op_attention_shared(*c[:5], ints(lens), ints(c[6])), *c)


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("hd,nq,nkv,S,P", [(128, 8, 2, 90, 2100), (64, 8, 2, 150, 515), (128, 5, 1, 40, 900), (128, 4, 4, 200, 257)])
def test_shared_many_rows(akvs, dt, hd, nq, nkv, S, P):
    lens = [(7 * s) % 33 for s in range(S)]
    c = shared_case(S, dt, hd, nq, nkv, P, 32, lens, [1] * S)
    check_shared(akvs.op_attention_shared(*c[:5], ints(lens)), *c)


@pytest.mark.parametrize("dt,hd,P", [(BF16, 64, 6090), (F16, 128, 6144), (F16, 64, 6018)])
def test_shared_key_ranges_of_unequal_length(akvs, dt, hd, P):
    """80 blocks of rows and heads, more than half of the SMs: a long and a short range of the context."""
    rows = [60] * 5
    c = shared_case(P, dt, hd, 32, 8, P, 70, [64, 70, 61, 60, 3], rows)
    check_shared(akvs.op_attention_shared(*c[:5], ints(c[5]), ints(c[6])), *c)


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("S", [2, 70])
@pytest.mark.parametrize("shape", ["rising", "falling", "spiky"])
def test_shared_moving_maximum(akvs, dt, S, shape):
    """Scores whose maximum moves by far more than any single step along the context."""
    c = shared_case(11, dt, 128, 8, 2, 1500, 40, [40] * S, [1] * S)
    q, ck, cv, sk, sv, lens, off = c
    ramp = torch.linspace(0.05, 6.0, 1500, device="cuda")
    if shape == "spiky":
        ramp = torch.where(torch.rand(1500, generator=gen(1), device="cuda") < 0.02, 8.0, 0.2)
    ck.copy_((ck.float() * (ramp.flip(0) if shape == "falling" else ramp)[:, None, None]).to(dt))
    check_shared(akvs.op_attention_shared(q, ck, cv, sk, sv, ints(lens)), *c)


def test_shared_bad_offsets_stay_inside(akvs):
    """Lengths and offsets outside their range are clamped; a range that runs backwards is empty."""
    c = shared_case(5, BF16, 128, 4, 2, 60, 32, [32, 32, 32, 32], [2, 2, 2, 2])
    q, ck, cv, sk, sv, _, _ = c
    sk, sv = torch.nan_to_num(sk), torch.nan_to_num(sv)
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
    akvs.op_attention_shared(q, ck, cv, sk, sv, ints([99, -4, 32, 2 ** 31 - 1]), ints([-3, 2, 4, 3, 400]), out, lse)
    # the sequences own rows [0, 2), [2, 4), none, [3, 8): row 3 belongs to two, which write it in turn
    want = akvs.op_attention_shared(q, ck, cv, sk, sv, ints([32, 0, 32, 32]), ints([0, 2, 4, 4, 8]))
    keep = [0, 1, 2, 4, 5, 6, 7]
    assert torch.equal(out[[0, 1, 2]], want[0][[0, 1, 2]])
    assert torch.isfinite(out[keep].float()).all()


def test_shared_strides_and_far_offsets(akvs):
    """Token strides beyond the packed ones, a slice of a larger cache, slots interleaved by token, and
    caches that reach past 2^31 elements."""
    g = gen(8)
    big = torch.zeros(2_400_000_000, dtype=BF16, device="cuda")
    P, S, nkv, hd = 600, 5, 2, 128
    lens = [3, 0, 17, 20, 9]
    c = shared_case(1, BF16, hd, 8, nkv, P, 20, lens, [1] * S)
    q, ck, cv, sk, sv, _, off = c
    step = (2_400_000_000 - 1024) // (P - 1) // 8 * 8
    fk = big.as_strided((P, nkv, hd), (step, hd, 1))
    fv = big.as_strided((P, nkv, hd), (step, hd, 1), storage_offset=512)
    fk.copy_(ck), fv.copy_(cv)
    base = akvs.op_attention_shared(q, ck, cv, sk, sv, ints(lens))
    wide = torch.zeros((S, 12, hd), dtype=BF16, device="cuda")
    wide[:, 2:10] = q
    inter = [x.transpose(0, 1).contiguous().transpose(0, 1) for x in (sk, sv)]     # [cap][S] in memory
    got = akvs.op_attention_shared(wide[:, 2:10], fk, fv, *inter, ints(lens))
    assert torch.equal(got[0], base[0]) and torch.equal(got[1], base[1])
    check_shared(got, *c)
    # far slots of own tokens
    far = (2_400_000_000 - 20 * nkv * hd * 2) // (S - 1) // 8 * 8
    for t, x, o in ((0, sk, 0), (1, sv, 20 * nkv * hd)):
        big.as_strided((S, 20, nkv, hd), (far, nkv * hd, hd, 1), storage_offset=o).copy_(x)
    ok, ov = (big.as_strided((S, 20, nkv, hd), (far, nkv * hd, hd, 1), storage_offset=o) for o in (0, 20 * nkv * hd))
    got = akvs.op_attention_shared(q, ck, cv, ok, ov, ints(lens))
    assert torch.equal(got[0], base[0]) and torch.equal(got[1], base[1])


def test_shared_replayed_graph_follows_lengths(akvs):
    """A captured step reads lengths and tokens when it is replayed, with two graphs on one scratch."""
    lens = [5, 0, 30, 11]
    c = shared_case(2, F16, 128, 8, 2, 400, 40, lens, [1] * 4)
    q, ck, cv, sk, sv, _, off = c
    sk, sv = torch.nan_to_num(sk, 0.5, 0.5), torch.nan_to_num(sv, 0.5, 0.5)
    dl = ints(lens)
    scratch = akvs.op_attention_shared_scratch(F16, 4, 400, 4, 40, 8, 2, 128)
    outs = [(torch.zeros_like(q), torch.zeros(4, 8, device="cuda")) for _ in range(2)]
    akvs.op_attention_shared(q, ck, cv, sk, sv, dl, None, *outs[0], scratch)
    graphs = []
    for o in outs:
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            akvs.op_attention_shared(q, ck, cv, sk, sv, dl, None, *o, scratch)
        graphs.append(gr)
    for step in range(3):
        lens = [x + 2 for x in lens]
        dl.copy_(ints(lens))
        q.mul_(0.9)
        for gr, o in zip(graphs, outs):
            o[0].zero_()
            gr.replay()
        torch.cuda.synchronize()
        check_shared(outs[0], q, ck, cv, sk, sv, lens, off)
        assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])


def test_shared_streams(akvs):
    """Calls on another stream than the default one, with their own scratch, at the same time."""
    cs = [shared_case(20 + i, BF16, 128, 8, 2, 900 + i, 40, [7, 40, 1], [1] * 3) for i in range(2)]
    torch.cuda.synchronize()
    got = []
    streams = [torch.cuda.Stream() for _ in cs]
    for _ in range(5):
        got = []
        for st, c in zip(streams, cs):
            with torch.cuda.stream(st):
                got.append(akvs.op_attention_shared(*c[:5], ints([7, 40, 1])))
    torch.cuda.synchronize()
    for x, c in zip(got, cs):
        check_shared(x, *c)


# ------------------------------------------------------------------------- attention mass

def mass_ref(q, k, lse, lo, hi):
    R, nq, hd = q.shape
    T, nkv = k.shape[:2]
    t = torch.arange(T, device="cuda")
    seen = (t >= lo[:, None]) & (t <= hi[:, None])
    out, err = torch.zeros((nkv, T), dtype=torch.float64, device="cuda"), 0.0
    for i in range(nq if R else 0):
        h = i // (nq // nkv)
        x = q[:, i].double() @ k[:, h].double().T / math.sqrt(hd)
        e = (q[:, i].double().abs() @ k[:, h].double().abs().T).max() / math.sqrt(hd) * hd * 2.0 ** -23
        err = max(err, float(e))
        p = (x - lse[:, i, None].double()).exp() * seen
        out[h] += torch.where(seen & (lse[:, i, None] > -math.inf), p, torch.zeros_like(p)).sum(0)
    return out, err


def check_mass(got, q, k, lse, lo, hi, mass=None):
    ref, err = mass_ref(q, k, lse, lo, hi)
    total = ref if mass is None else ref + mass.double()
    n = q.shape[0] * q.shape[1] // k.shape[1]
    # every weight: its score, the exponent's rounding; the sums: n additions of positive terms
    tol = (2 * err + 2.0 ** -17 + n * 2.0 ** -24) * ref + 2.0 ** -24 * total.abs()
    assert ((got.double() - total).abs() <= tol).all(), ((got.double() - total).abs() / tol.clamp_min(1e-300)).max()


def mass_case(seed, dt, hd, nq, nkv, R, T, kind):
    g = gen(seed)
    q, k = rnd(g, R, nq, hd, dt=dt, scale=1.5), rnd(g, T, nkv, hd, dt=dt)
    lo = torch.zeros(R, dtype=torch.int32, device="cuda")
    hi = torch.full((R,), T - 1, dtype=torch.int32, device="cuda")
    if kind == "causal":
        hi = (T - R + torch.arange(R, device="cuda")).int()
    elif kind == "ragged":                                   # empty, single, far outside, in no order
        lo = torch.randint(-5, T + 5, (R,), generator=g, device="cuda", dtype=torch.int32)
        hi = lo + torch.randint(-3, max(2, T // 2), (R,), generator=g, device="cuda", dtype=torch.int32)
    t = torch.arange(T, device="cuda")
    seen = (t >= lo[:, None]) & (t <= hi[:, None])
    x = torch.stack([q[:, i].double() @ k[:, i // (nq // nkv)].double().T for i in range(nq)], 1) / math.sqrt(hd)
    lse = torch.logsumexp(x.masked_fill(~seen[:, None], -math.inf), -1).float() if R else torch.zeros((0, nq), device="cuda")
    return q, k, lse, lo, hi


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("hd,nq,nkv", [(128, 8, 2), (64, 5, 1), (128, 40, 8), (64, 2, 2), (128, 16, 1)])
@pytest.mark.parametrize("R,T,kind", [(1, 1, "all"), (1, 700, "all"), (16, 300, "all"), (90, 257, "causal"), (130, 1000, "ragged"),
                                      (0, 64, "all")])
def test_mass(akvs, dt, hd, nq, nkv, R, T, kind):
    q, k, lse, lo, hi = mass_case(R + T, dt, hd, nq, nkv, R, T, kind)
    got = akvs.op_attention_mass(q, k, lse, lo, hi)
    check_mass(got, q, k, lse, lo, hi)
    old = torch.rand((nkv, T), generator=gen(1), device="cuda")
    more = akvs.op_attention_mass(q, k, lse, lo, hi, old)
    check_mass(more, q, k, lse, lo, hi, old)
    want = old + got
    akvs.op_attention_mass(q, k, lse, lo, hi, old, old)      # in place, and the same bits again
    assert torch.equal(old, more) and torch.equal(want, more)


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("hd,nq,nkv", [(128, 128, 1), (64, 100, 1), (128, 65, 1), (64, 14, 2), (128, 6, 2)])
@pytest.mark.parametrize("R", [1, 3, 150])
def test_mass_many_heads_per_kv_head(akvs, dt, hd, nq, nkv, R):
    """Groups that fill a tile of rows, leave it ragged, or need several of them, with ragged ranges."""
    q, k, lse, lo, hi = mass_case(nq + R, dt, hd, nq, nkv, R, 530, "ragged")
    check_mass(akvs.op_attention_mass(q, k, lse, lo, hi), q, k, lse, lo, hi)


def test_mass_hidden_keys_and_blind_rows(akvs):
    """NaN or infinite keys outside a row's range add nothing, and neither does a row with lse = -inf."""
    for dt in TYPES:
        q, k, lse, lo, hi = mass_case(6, dt, 128, 8, 2, 40, 500, "all")
        lo.fill_(130), hi.fill_(400)
        want = akvs.op_attention_mass(q, k, lse, lo, hi)
        k[:130], k[401:] = math.nan, math.inf
        got = akvs.op_attention_mass(q, k, lse, lo, hi)
        assert torch.equal(got, want) and (got[:, :130] == 0).all() and (got[:, 401:] == 0).all()
        lse[3:] = -math.inf
        few = akvs.op_attention_mass(q, k, lse, lo, hi)
        only = akvs.op_attention_mass(q[:3], k, lse[:3], lo[:3], hi[:3])
        assert torch.allclose(few, only, rtol=2.0 ** -20, atol=0)


def test_mass_strides_and_far_keys(akvs):
    q, k, lse, lo, hi = mass_case(9, F16, 128, 8, 2, 20, 500, "causal")
    want = akvs.op_attention_mass(q, k, lse, lo, hi)
    big = torch.zeros(2_400_000_000, dtype=F16, device="cuda")
    far = big.as_strided((500, 2, 128), ((2_400_000_000 - 512) // 499 // 8 * 8, 128, 1))
    far.copy_(k)
    wide = torch.zeros((20, 11, 128), dtype=F16, device="cuda")
    wide[:, 1:9] = q
    assert torch.equal(akvs.op_attention_mass(wide[:, 1:9], far, lse, lo, hi), want)


# ------------------------------------------------------------------------- eviction

def evict_ref(mass, budget, sink, recent):
    m = np.where(np.isnan(mass), -np.inf, mass.astype(np.float64))
    L, H, T = m.shape
    idx = np.empty((L, H, budget), np.int64)
    always = np.concatenate([np.arange(sink), np.arange(T - recent, T)])
    nan = np.isnan(mass)
    for l in range(L):
        for h in range(H):
            order = np.lexsort((np.arange(T), -m[l, h], nan[l, h]))
            free = order[(order >= sink) & (order < T - recent)][:budget - len(always)]
            idx[l, h] = np.sort(np.concatenate([always, free]))
    return idx


def check_evict(akvs, mass, k, v, budget, sink, recent):
    idx, ko, vo, mo = akvs.op_evict(mass, k, v, budget, sink, recent)
    ref = torch.from_numpy(evict_ref(mass.cpu().numpy(), budget, sink, recent)).cuda()
    assert torch.equal(idx.long(), ref)
    at = ref.transpose(1, 2)[..., None].expand(-1, -1, -1, k.shape[-1])
    assert torch.equal(ko, torch.gather(k, 1, at)) and torch.equal(vo, torch.gather(v, 1, at))
    assert torch.equal(mo.nan_to_num(-1.0), torch.gather(mass, 2, ref).nan_to_num(-1.0))


@pytest.mark.parametrize("dt,hd", [(F32, 64), (F32, 128), (BF16, 64), (F16, 128)])
@pytest.mark.parametrize("L,T,nkv", [(1, 1, 1), (3, 31, 2), (1, 700, 8), (2, 5003, 1), (40, 129, 5)])
def test_evict(akvs, dt, hd, L, T, nkv):
    g = gen(T + L)
    k, v = rnd(g, L, T, nkv, hd, dt=dt), rnd(g, L, T, nkv, hd, dt=dt)
    mass = torch.rand((L, nkv, T), generator=g, device="cuda").pow(8)
    tied = (mass * 8).round() / 8                             # heavy ties, most at zero
    odd = torch.where(tied == 0, -0.0, tied)
    odd[..., ::3] = 0.0
    if T > 8:
        odd[..., 4], odd[..., 6], odd[..., 7] = math.nan, math.inf, -math.inf
    for m in (mass, tied, odd):
        for budget, sink, recent in {(T, 0, 0), (max(1, T // 3), 0, 0), (max(1, T // 2), min(2, T // 4), T // 5), (T // 2, 0, T // 2),
                                     (1, 0, 0), (0, 0, 0), (T - T // 9, min(4, T // 8), 1 if T > 8 else 0)}:
            check_evict(akvs, m, k, v, budget, sink, recent)


@pytest.mark.parametrize("T", [40_000, 500_000])              # clusters; more keys than their shared memory holds
def test_evict_long(akvs, T):
    g = gen(3)
    k, v = rnd(g, 1, T, 1, 64, dt=BF16), rnd(g, 1, T, 1, 64, dt=BF16)
    mass = (torch.rand((1, 1, T), generator=g, device="cuda") * 5000).round() / 16
    check_evict(akvs, mass, k, v, T // 3 + 7, 4, 1001)
    check_evict(akvs, torch.zeros_like(mass), k, v, T // 3 + 7, 0, 0)


def test_evict_slice_of_a_cache_and_far_offsets(akvs):
    g = gen(5)
    full = rnd(g, 3, 300, 2, 128, dt=F16)
    other = rnd(g, 3, 300, 2, 128, dt=F16)
    mass = torch.rand((3, 2, 250), generator=g, device="cuda")
    check_evict(akvs, mass, full[:, 20:270], other[:, 20:270], 90, 3, 20)
    big = torch.zeros(2_400_000_000, dtype=F16, device="cuda")
    tok = (2_400_000_000 - 1024) // 249 // 8 * 8
    fk = big.as_strided((1, 250, 2, 128), (0, tok, 128, 1))
    fv = big.as_strided((1, 250, 2, 128), (0, tok, 128, 1), storage_offset=512)
    fk.copy_(full[:1, 20:270]), fv.copy_(other[:1, 20:270])
    check_evict(akvs, mass[:1], fk, fv, 90, 3, 20)


# ------------------------------------------------------------------------- all of them together

@pytest.mark.parametrize("dt", TYPES)
def test_answering_from_a_shared_context(akvs, dt):
    """Decoding steps of several sequences over one context: norm and rotation of the new tokens, their
    K/V appended, attention, the context's weights, then eviction and a step over what is left;
    each step against the plain forms on the same inputs."""
    g = gen(31)
    nq, nkv, hd, P, S, cap, base = 8, 2, 128, 777, 3, 8, 1e4
    ck, cv = rnd(g, P, nkv, hd, dt=dt), rnd(g, P, nkv, hd, dt=dt)
    sk, sv = (torch.full((S, cap, nkv, hd), math.nan, device="cuda", dtype=dt) for _ in range(2))
    gq, gk = rnd(g, hd) * 0.1 + 1, rnd(g, hd) * 0.1 + 1
    lens = torch.zeros(S, dtype=torch.int32, device="cuda")
    mass = torch.zeros((nkv, P), device="cuda")
    zero, last = torch.zeros(S, dtype=torch.int32, device="cuda"), torch.full((S,), P - 1, dtype=torch.int32, device="cuda")
    for step in range(6):
        qkv = rnd(g, S, nq + 2 * nkv, hd, dt=dt, scale=2.0)
        pos = (P + lens).int()
        q, k = akvs.op_qk_norm_rope(qkv[:, :nq], qkv[:, nq:nq + nkv], gq, gk, pos, 1e-6, base)
        check_norm(q, qkv[:, :nq], gq, pos, 1e-6, base)
        at = lens.long()
        sk[torch.arange(S), at], sv[torch.arange(S), at] = k, qkv[:, nq + nkv:]
        lens += 1
        out = akvs.op_attention_shared(q, ck, cv, sk, sv, lens)
        check_shared(out, q, ck, cv, sk, sv, lens.tolist(), list(range(S + 1)))
        n = ck.shape[0]
        old = mass.clone()
        akvs.op_attention_mass(q, ck, out[1], zero, last.clamp(max=n - 1), mass, mass)
        check_mass(mass, q, ck, out[1], zero, last.clamp(max=n - 1), old)
        if step == 3:
            check_evict(akvs, mass[None], ck[None], cv[None], 200, 4, 32)
            _, k2, v2, m2 = akvs.op_evict(mass[None], ck[None], cv[None], 200, 4, 32)
            ck, cv, mass = k2[0], v2[0], m2[0]
