"""The operators that decode from a 4-bit cache with 4-bit weights, against plain forms in 64 bits.

Tolerances count roundings.  eps / 2 of the output type is one rounding of a result.  Codes, records and 16-bit
inputs enter the products exactly; a float sum of n terms is off by at most n * 2^-23 of the sum of its terms'
magnitudes (an addition rounds by 2^-24 and the tensor cores may truncate, which doubles it).  |k| of a key counts
as 15 scale + |minimum|, which its parts are below.  A score that is off by d changes its weight by a factor of at
most 1 + 2d for small d; a weight enters as two bfloat16 (2^-17 of itself; float rows: three, 2^-25), exp2 and its
argument's rounding add under 2^-17 for scores below 64.
"""
import copy
import gc
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


# ------------------------------------------------------------------------------------- rotation

def rope_ref(x, pos, rope):
    """In 64 bits from the formulas; and |a| + |b| of every value's pair."""
    d = rope.desc
    rot, half_ = d.rot_dim, d.rot_dim // 2
    i = np.arange(half_, dtype=np.float64)
    base, factor, orig, low, high = d.base, d.factor, d.orig_ctx, d.low, d.high
    if d.scaling == 2:
        base = base * factor ** (rot / (rot - 2))
    f = base ** (-2 * i / rot)
    mag = d.magnitude or 1.0
    if d.scaling == 1:
        f = f / factor
    if d.scaling == 3:
        w = np.clip((orig * f / (2 * np.pi) - low) / (high - low), 0, 1)
        f = f * (w + (1 - w) / factor)
    if d.scaling == 4:
        at = [rot * np.log(orig / (2 * np.pi * r)) / (2 * np.log(base)) for r in (high, low)]
        a, b = max(np.floor(at[0]), 0), min(np.ceil(at[1]), rot - 1)
        w = 1 - np.clip((i - a) / max(b - a, 0.001), 0, 1)
        f = f * (w + (1 - w) / factor)
        mag = d.magnitude or (0.1 * np.log(factor) + 1 if factor > 1 else 1.0)
    ang = torch.from_numpy(pos.cpu().numpy().astype(np.float64)[:, None] * f).cuda()[:, None]
    y = x.double()
    out, both = y.clone(), y.abs()
    at = (slice(0, half_), slice(half_, rot)) if d.layout == 0 else (slice(0, rot, 2), slice(1, rot, 2))
    u, v = y[..., at[0]], y[..., at[1]]
    out[..., at[0]], out[..., at[1]] = mag * (u * ang.cos() - v * ang.sin()), mag * (v * ang.cos() + u * ang.sin())
    both[..., at[0]] = both[..., at[1]] = mag * (u.abs() + v.abs())
    return out, both


def check_rope(got, x, pos, rope):
    ref, both = rope_ref(x, pos, rope)
    # cosine and sine are right to 2^-22 (angles up to 2^31 are reduced in double), two products, a sum and the
    # magnitude: under 2^-20 of |a| + |b|
    tol = half(got.dtype) * ref.abs() + 2.0 ** -20 * both + TINY[got.dtype]
    assert ((got.double() - ref).abs() <= tol).all(), ((got.double() - ref).abs() - tol).max()
    rot = rope.desc.rot_dim
    assert torch.equal(got[..., rot:], x[..., rot:])


ROPES = [dict(scaling="plain"), dict(scaling="linear", factor=4.0), dict(scaling="ntk", factor=8.0),
         dict(scaling="bands", factor=8.0, orig_ctx=8192.0, low=1.0, high=4.0), dict(scaling="yarn", factor=16.0, orig_ctx=4096.0),
         dict(scaling="yarn", factor=4.0, orig_ctx=4096.0, low=1.0, high=32.0, magnitude=0.75)]


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("hd,rot", [(64, 64), (128, 128), (128, 64), (128, 32), (128, 20), (80, 32), (8, 6), (256, 256), (256, 16), (72, 70)])
def test_rope_scaled(akvs, dt, hd, rot):
    for n, nq, nkv in ((1, 32, 8), (37, 5, 1), (300, 6, 2), (3, 0, 2), (3, 2, 0)):
        g = gen(n + hd + rot)
        qkv = rnd(g, n, nq + 2 * nkv + 1, hd, dt=dt, scale=3.0)
        q, k = qkv[:, :nq], qkv[:, nq:nq + nkv]
        pos = torch.randint(0, 200000, (n,), generator=g, device="cuda", dtype=torch.int32)
        pos[0] = [0, 2 ** 31 - 1, -5, 1000003][(n + hd // 8) % 4]
        before = qkv.clone()
        for i, kind in enumerate(ROPES):
            rope = akvs.Rope(1e4 if i % 2 else 5e5, rot, layout="half" if (i + n) % 2 else "interleaved", **kind)
            oq, ok = akvs.op_rope_scaled(q, k, pos, rope)
            assert torch.equal(qkv, before)
            check_rope(oq, q, pos, rope)
            check_rope(ok, k, pos, rope)
        # in place, in the columns of one tensor: the same bits, and the others untouched
        akvs.op_rope_scaled(q, k, pos, rope, q, k)
        assert torch.equal(q, oq) and torch.equal(k, ok)
        assert torch.equal(qkv[:, nq + nkv:], before[:, nq + nkv:])


def test_rope_scaled_agrees_with_rope(akvs):
    g = gen(4)
    x, pos = rnd(g, 50, 4, 128), torch.arange(50, device="cuda", dtype=torch.int32) * 241
    q, _ = akvs.op_rope_scaled(x, x[:, :1], pos, akvs.Rope(5e5, 128))
    assert (q - akvs.op_rope(x.clone(), pos, 5e5)).abs().max() <= 2.0 ** -20 * 2 * x.abs().max()


def test_rope_copied(akvs):
    """A Rope's copy outlives it."""
    g = gen(6)
    x, pos, rope = rnd(g, 9, 2, 64), torch.arange(9, device="cuda", dtype=torch.int32), akvs.Rope(1e4, 64, scaling="linear", factor=2.0)
    want, _ = akvs.op_rope_scaled(x, x[:, :1], pos, rope)
    twin = copy.deepcopy(rope)
    del rope
    gc.collect()
    others = [akvs.Rope(3.0, 32) for _ in range(50)]
    got, _ = akvs.op_rope_scaled(x, x[:, :1], pos, twin)
    assert torch.equal(got, want) and len(others) == 50


def test_rope_scaled_far_rows(akvs):
    """Rows beyond 2^31 elements."""
    n, ld = 3, 1 << 30
    room = torch.empty(2 * ld + 256, dtype=F16, device="cuda")
    x = torch.as_strided(room, (n, 1, 128), (ld, 128, 1))
    x.copy_(rnd(gen(1), n, 1, 128, dt=F16))
    pos, rope = ints([1, 2, 3]), akvs.Rope(1e4, 128, layout="interleaved")
    q, _ = akvs.op_rope_scaled(x, x[:, :0], pos, rope)
    check_rope(q, x, pos, rope)


# ---------------------------------------------------------------------------------------- pages

class Cache:
    """Sequences of given lengths in random places of a pool whose other bytes are ones: codes of 15, records of NaN."""

    def __init__(self, akvs, g, lens, nkv, hd, dt, k=None, v=None, spare=2):
        self.akvs, self.lens, self.nkv, self.hd = akvs, list(lens), nkv, hd
        T = sum(lens)
        self.k = rnd(g, T, nkv, hd, dt=dt) if k is None else k
        self.v = rnd(g, T, nkv, hd, dt=dt) if v is None else v
        need = [-(-n // 64) for n in lens]
        self.width = max(need + [1])
        n_pages = sum(need) + spare
        self.pool = torch.full((n_pages, akvs.page_bytes(nkv, hd)), 255, dtype=torch.uint8, device="cuda")
        place = torch.randperm(n_pages, generator=g, device="cuda").tolist()
        rows, at = [], 0
        for n in need:
            rows.append(place[at:at + n] + [-1 if (at + n) % 2 else 10 ** 6] * (self.width - n))
            at += n
        self.table = ints(rows).reshape(len(lens), self.width)
        self.len = ints(self.lens)
        self.start = np.concatenate([[0], np.cumsum(lens)]).astype(int)
        if T:
            akvs.op_pages_append(self.k, self.v, self.pool, self.table, self.len, ints(self.start.tolist()))
        self.records = [self._records(x) for x in (self.k, self.v)]

    def _records(self, x):
        """(codes, scale, minimum) in 64 bits, by the framework's quantiser of flat caches."""
        n = x.shape[0]
        if n == 0:
            z = torch.zeros((0, self.nkv, self.hd), dtype=torch.float64, device="cuda")
            return z, z, z
        codes, meta = self.akvs.op_quantize(x.contiguous(), 4)
        c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).double()
        s, m = (meta[..., i].double().repeat_interleave(64, -1) for i in (0, 1))
        return c, s, m

    def values(self, which, at=slice(None)):
        c, s, m = (x[at] for x in self.records[which])
        return c * s + m

    def size(self, which, at=slice(None)):
        c, s, m = (x[at] for x in self.records[which])
        return 15 * s + m.abs()


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("nkv", [1, 2, 8])
def test_append_and_read(akvs, dt, hd, nkv):
    g = gen(hd + nkv)
    lens = [5, 0, 64, 65, 1, 700, 63]
    k = rnd(g, sum(lens), nkv, hd, dt=dt) * torch.arange(1, nkv + 1, device="cuda", dtype=dt)[:, None]
    v = rnd(g, sum(lens), nkv, hd, dt=dt)
    k[3] = 0                                           # a group without extent
    v[4] = 7.5
    v[6, 0, 5] = 3e4                                   # and one with an outlier
    c = Cache(akvs, g, lens, nkv, hd, dt, k, v)
    off = ints(c.start.tolist())
    ko, vo = torch.full_like(k, 9), torch.full_like(v, 9)
    akvs.op_pages_read(c.pool, c.table, c.len, ko, vo, off)
    for got, which in ((ko, 0), (vo, 1)):
        # the value is formed by one float fma, then rounded: within half a step of the type and one of float
        ref = c.values(which)
        assert ((got.double() - ref).abs() <= (half(dt) + (0 if dt == F32 else 2.0 ** -24)) * ref.abs() + TINY[dt]).all()
    # bytes of no token are as they were
    free = sorted(set(range(c.pool.shape[0])) - set(c.table.flatten().tolist()))
    assert (c.pool[free] == 255).all()
    # token by token, strided, the same bytes (the last token of every sequence that has one)
    again = Cache(akvs, gen(hd + nkv + 1), lens, nkv, hd, dt, k, v)
    again.pool.fill_(255)
    wide = torch.cat([k, v], 1)                        # k and v as column ranges
    for t in range(max(lens)):
        live = [s for s in range(len(lens)) if lens[s] > t]
        rows = torch.tensor([c.start[s] + t for s in live], device="cuda")
        w = wide[rows]
        akvs.op_pages_append(w[:, :nkv], w[:, nkv:], again.pool, again.table[live].contiguous(), ints([t + 1] * len(live)))
        if t > 70:
            break
    short = [min(n, 72) for n in lens]
    soff = np.concatenate([[0], np.cumsum(short)]).tolist()
    a = [torch.zeros((sum(short), nkv, hd), dtype=dt, device="cuda") for _ in range(4)]
    akvs.op_pages_read(c.pool, c.table, ints(short), a[0], a[1], ints(soff))
    akvs.op_pages_read(again.pool, again.table, ints(short), a[2], a[3], ints(soff))
    assert torch.equal(a[0], a[2]) and torch.equal(a[1], a[3])


def test_append_edges(akvs):
    """Rows of no sequence, rows before token 0, pages outside the pool and behind the table: nothing is written."""
    g, nkv, hd = gen(3), 2, 64
    k, v = rnd(g, 12, nkv, hd, dt=BF16), rnd(g, 12, nkv, hd, dt=BF16)
    pool = torch.full((4, akvs.page_bytes(nkv, hd)), 255, dtype=torch.uint8, device="cuda")
    table = ints([[0, -1], [1, 4], [2, 3]])
    # sequence 0: 3 rows, of which the first lies before token 0; sequence 1: 4 rows over a missing page; sequence 2: 3 rows
    akvs.op_pages_append(k, v, pool, table, ints([2, 66, 67]), ints([1, 4, 8, 11]))
    ko, vo = torch.full_like(k, 9), torch.full_like(v, 9)
    akvs.op_pages_read(pool, table, ints([2, 66, 67]), ko, vo, ints([1, 4, 8, 11]))
    got = [not (ko[r] == 9).all() for r in range(12)]
    assert got == [False, False, True, True, True, True, False, False, True, True, True, False]
    codes = Cache(akvs, g, [12], nkv, hd, BF16, k, v)
    assert ((ko[2:6].double() - codes.values(0)[2:6]).abs() <= 2.0 ** -8 * codes.values(0)[2:6].abs() + 1e-12).all()
    before = pool.clone()
    akvs.op_pages_append(k, v, pool, table, ints([10 ** 9, -7, 128]), ints([0, 2, 5, 5]))     # clamped: tokens 126, 127 of sequence 0
    assert torch.equal(pool, before)                                                       # on a page outside, and none at all


@pytest.mark.parametrize("S", [31, 32, 33, 64, 200])
def test_append_to_many_sequences(akvs, S):
    """0 to 3 rows of each of many sequences, rows before the first and behind the last: what one call per sequence does."""
    g = gen(S)
    n = torch.randint(0, 4, (S,), generator=g, device="cuda")
    n[S // 2:S // 2 + 5] = 0
    had = torch.randint(0, 190, (S,), generator=g, device="cuda")
    off, lens = ints([2] + (2 + n.cumsum(0)).tolist()), (had + n).int()
    R = int(off[-1]) + 3
    k, v = rnd(g, R, 2, 64, dt=F16), rnd(g, R, 2, 64, dt=F16)
    table = torch.randperm(3 * S, generator=g, device="cuda").int().view(S, 3)
    pools = [torch.full((3 * S, akvs.page_bytes(2, 64)), 255, dtype=torch.uint8, device="cuda") for _ in range(2)]
    akvs.op_pages_append(k, v, pools[0], table, lens, off)
    out = [torch.full_like(k, 9) for _ in range(4)]
    akvs.op_pages_read(pools[0], table, lens, out[0], out[1], off)
    for s, (a, b) in enumerate(zip(off.tolist(), off.tolist()[1:])):
        at = (table[s:s + 1], lens[s:s + 1])
        akvs.op_pages_append(k[a:b], v[a:b], pools[1], *at, ints([0, b - a]))
        akvs.op_pages_read(pools[1], *at, out[2][a:b], out[3][a:b], ints([0, b - a]))
    assert torch.equal(pools[0], pools[1])
    assert torch.equal(out[0], out[2]) and torch.equal(out[1], out[3]) and (out[0][:2] == 9).all() and (out[0][-3:] == 9).all()
    x = k[2:-3].float()
    lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    # half a step; 15 steps off by the scale's rounding, the minimum's, the value's own (of float16, each under 2^-10 of these)
    assert ((out[0][2:-3].float() - x).abs() <= (hi - lo) / 30 + 2.0 ** -10 * (2 * (hi - lo) + 2 * x.abs().amax(-1, keepdim=True))).all()


def test_copy(akvs):
    g = gen(9)
    pool = torch.randint(0, 256, (3, 11, 48), generator=g, device="cuda", dtype=torch.uint8)
    wide = torch.randint(0, 256, (3, 14, 64), generator=g, device="cuda", dtype=torch.uint8)
    for p in (pool, wide[:, 1:12, 16:], torch.randint(0, 256, (1, 11, 73728 * 3 + 16), generator=g, device="cuda", dtype=torch.uint8)):
        whole, want = (wide.clone() if p.shape[0] == 3 and not p.is_contiguous() else None), p.clone()
        src, dst = [3, 3, 0, 7, 20, -1, 5], [1, 2, 4, 9, 8, 8, 11]
        for a, b in list(zip(src, dst))[:4]:
            want[:, b] = p[:, a]
        akvs.op_pages_copy(p, ints(src), ints(dst))
        assert torch.equal(p, want)
        if whole is not None:
            whole[:, 1:12, 16:] = want
            assert torch.equal(wide, whole)
    assert akvs.op_pages_copy(pool, ints([]), ints([])) is pool


# ------------------------------------------------------------------------------------ attention

def attention_ref(c, q, off, table=None):
    """out, lse, sum of p |v|, and the largest error a score of the row may have."""
    R, nq, hd = q.shape
    gr, f64 = nq // c.nkv, torch.float64
    out, lse = torch.zeros((R, nq, hd), dtype=f64, device="cuda"), torch.full((R, nq), -math.inf, dtype=f64, device="cuda")
    mag, err = torch.zeros_like(out), torch.zeros_like(lse)
    for s, n in enumerate(c.lens):
        rows = off[s + 1] - off[s]
        if rows == 0 or n == 0:
            continue
        at = slice(c.start[s], c.start[s] + n)
        k, v, ka, va = c.values(0, at), c.values(1, at), c.size(0, at), c.size(1, at)
        x = q[off[s]:off[s + 1]].double().reshape(rows, c.nkv, gr, hd)
        y = torch.einsum("rhgd,thd->rhgt", x, k) / math.sqrt(hd)
        e = torch.einsum("rhgd,thd->rhgt", x.abs(), ka) / math.sqrt(hd) * hd * 2.0 ** -23
        seen = torch.arange(n, device="cuda")[None, :] < n - torch.arange(rows - 1, -1, -1, device="cuda")[:, None]
        y = y.masked_fill(~seen[:, None, None, :], -math.inf)
        z = torch.logsumexp(y, -1)
        p = (y - z[..., None]).exp().nan_to_num(0.0)
        sl = slice(off[s], off[s + 1])
        out[sl] = torch.einsum("rhgt,thd->rhgd", p, v).reshape(rows, nq, hd)
        mag[sl] = torch.einsum("rhgt,thd->rhgd", p, va).reshape(rows, nq, hd)
        lse[sl] = z.reshape(rows, nq)
        err[sl] = e.amax(-1).reshape(rows, nq)
    return out, lse, mag, err


def check_attention(got, c, q, off):
    (o, l), dt = got, q.dtype
    ref, lse, mag, err = attention_ref(c, q, off)
    used = slice(off[0], off[-1])
    o, l, ref, lse, mag, err = (x[used] for x in (o, l, ref, lse, mag, err))
    none = lse == -math.inf
    assert torch.equal(l == -math.inf, none) and (o[none] == 0).all()
    tol = half(dt) * ref.abs() + (2 * err[..., None] + 2.0 ** -15) * mag + TINY[dt]
    assert ((o.double() - ref).abs() <= tol).all(), ((o.double() - ref).abs() / tol).max()
    d = (l.double() - lse)[~none].abs()
    assert (d <= (err + 2.0 ** -18 + 2.0 ** -22 * lse.abs())[~none]).all()


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("nq,nkv", [(1, 1), (4, 2), (8, 2), (5, 1), (16, 2), (32, 8), (20, 1)])
def test_attention(akvs, dt, hd, nq, nkv):
    for case, lens in enumerate(([0], [1], [64], [17, 0, 65, 63, 500, 16, 1], [3000])):
        g = gen(case + nq + hd)
        c = Cache(akvs, g, lens, nkv, hd, dt)
        S = len(lens)
        q = rnd(g, S, nq, hd, dt=dt, scale=1.5)
        check_attention(akvs.op_attention_pages(q, c.pool, c.table, c.len, nkv), c, q, list(range(S + 1)))
        for most in (3, 40):
            rows = [(7 * s + 3) % (most + 1) for s in range(S)]
            off = np.concatenate([[0], np.cumsum(rows)]).tolist()
            q = rnd(g, off[-1], nq, hd, dt=dt, scale=1.5)
            if off[-1]:
                check_attention(akvs.op_attention_pages(q, c.pool, c.table, c.len, nkv, ints(off)), c, q, off)


@pytest.mark.parametrize("dt", TYPES)
def test_attention_is_as_exact_as_its_output(akvs, dt):
    """Root mean square errors: the output's own rounding (a uniform error of half a step at most, 0.289 steps) and
    little else; float rows against the size of their terms."""
    g = gen(5)
    for nq, nkv, lens in ((8, 2, [4000, 900]), (16, 2, [4000, 900]), (12, 1, [5000])):
        c = Cache(akvs, g, lens, nkv, 128, dt)
        q = rnd(g, len(lens), nq, 128, dt=dt)
        o, _ = akvs.op_attention_pages(q, c.pool, c.table, c.len, nkv)
        ref, _, mag, _ = attention_ref(c, q, list(range(len(lens) + 1)))
        rms = lambda x: x.double().square().mean().sqrt()  # noqa: E731
        if dt == F32:
            assert rms(o - ref) <= 2.0 ** -20 * rms(mag)
        else:
            assert rms(o - ref) <= 1.1 * rms(ref.to(dt).double() - ref)


def test_attention_many_sequences_and_long_ones(akvs):
    g = gen(11)
    lens = [(37 * s * s + 11 * s) % 700 for s in range(300)]
    c = Cache(akvs, g, lens, 2, 64, BF16)
    rows = [min(n, (s * 5) % 4) for s, n in enumerate(lens)]
    off = np.concatenate([[0], np.cumsum(rows)]).tolist()
    q = rnd(g, off[-1] + 3, 8, 64, dt=BF16)
    out, lse = torch.full_like(q, 5), torch.full((off[-1] + 3, 8), 5.0, device="cuda")
    akvs.op_attention_pages(q, c.pool, c.table, c.len, 2, ints(off), out, lse)
    check_attention((out, lse), c, q[:off[-1]], off)
    assert (out[off[-1]:] == 5).all() and (lse[off[-1]:] == 5).all()         # rows of no sequence
    c = Cache(akvs, g, [100003, 3], 1, 128, F16)
    q = rnd(g, 2, 5, 128, dt=F16)
    check_attention(akvs.op_attention_pages(q, c.pool, c.table, c.len, 1), c, q, [0, 1, 2])


def test_attention_far_scores_and_sizes(akvs):
    """One key that outweighs all, weights over many orders, q and K and V near the ends of the types."""
    g = gen(2)
    for dt in (F32, BF16, F16):
        for qs, ks, vs in ((300.0, 1.0, 1.0), (1e-3, 1.0, 1e-3), (2.0 ** -20, 2.0 ** 10, 2.0 ** 12), (1.0, 2.0 ** -9, 2.0 ** -9), (6e4, 2.0 ** -10, 4e3)):
            lens = [700, 90]
            k, v = rnd(g, 790, 2, 128, scale=ks).to(dt), rnd(g, 790, 2, 128, scale=vs).to(dt)
            c = Cache(akvs, g, lens, 2, 128, dt, k, v)
            q = rnd(g, 2, 8, 128, scale=qs).clamp(-6e4, 6e4).to(dt)
            o, l = akvs.op_attention_pages(q, c.pool, c.table, c.len, 2)
            ref, lse, mag, err = attention_ref(c, q, [0, 1, 2])
            # scores of thousands: float holds them to 2^-22 of themselves, exp's factor is 1 + 2 d, d below 1/4
            far = err + 2.0 ** -22 * lse.abs()
            tol = half(dt) * ref.abs() + (2 * far[..., None].expm1().clamp_max(1.0) + 2.0 ** -15) * mag + TINY[dt]
            assert ((o.double() - ref).abs() <= tol).all(), (dt, qs, ((o.double() - ref).abs() / tol).max())
            assert ((l.double() - lse).abs() <= far + 2.0 ** -18).all()


def test_attention_light_weights(akvs):
    """30000 keys of weight 2^-26 beside one of 1: their sum reaches the output."""
    n, hd = 30001, 64
    k, v = torch.zeros((n, 1, hd), dtype=F16, device="cuda"), torch.zeros((n, 1, hd), dtype=F16, device="cuda")
    k[0, 0] = 15.0
    k[:, 0, 1] = 0.0                                   # a group of zeros and one 15 has codes that stand for both exactly
    v[1:, 0] = 1024.0
    k[0, 0, 1] = 0.0
    q = torch.zeros((1, 1, hd), dtype=F16, device="cuda")
    q[0, 0, 0] = 26 * math.log(2) * 8 / 15
    c = Cache(akvs, gen(1), [n], 1, hd, F16, k, v)
    check_attention(akvs.op_attention_pages(q, c.pool, c.table, c.len, 1), c, q, [0, 1])


def test_attention_hidden_and_seen_infinities(akvs):
    """An infinity in K or V beyond a row's limit does not reach it; one that it sees does."""
    g = gen(6)
    for nq in (4, 8, 32):
        k, v = rnd(g, 130, 1, 128, dt=BF16), rnd(g, 130, 1, 128, dt=BF16)
        good = Cache(akvs, gen(7), [130], 1, 128, BF16, k, v)
        kb, vb = k.clone(), v.clone()
        kb[129, 0, 3], vb[129, 0, 70] = math.nan, math.inf
        kb[128, 0, 3] = math.inf
        bad = Cache(akvs, gen(7), [130], 1, 128, BF16, kb, vb)
        q = rnd(g, 4, nq, 128, dt=BF16)
        a = akvs.op_attention_pages(q, good.pool, good.table, good.len, 1, ints([0, 4]))
        b = akvs.op_attention_pages(q, bad.pool, bad.table, bad.len, 1, ints([0, 4]))
        assert torch.equal(a[0][:2], b[0][:2]) and torch.equal(a[1][:2], b[1][:2])       # rows that see 127 and 128 tokens
        assert not b[0][2:].float().isfinite().all(-1).any()
        q[1, 0, 5] = math.inf                           # a row of q with an infinity: itself only
        d = akvs.op_attention_pages(q, good.pool, good.table, good.len, 1, ints([0, 4]))
        assert d[0][1, 0].isnan().all() and torch.equal(d[0][0], a[0][0]) and torch.equal(d[0][2:], a[0][2:])


def test_attention_missing_pages(akvs):
    """A page number outside the pool: its tokens are not seen."""
    g, hd = gen(8), 128
    k, v = rnd(g, 300, 2, hd, dt=F16), rnd(g, 300, 2, hd, dt=F16)
    c = Cache(akvs, g, [300], 2, hd, F16, k, v)
    keep = torch.cat([torch.arange(64), torch.arange(192, 300)]).cuda()
    want = Cache(akvs, g, [172], 2, hd, F16, k[keep], v[keep])
    q = rnd(g, 1, 8, hd, dt=F16)
    table = c.table.clone()
    table[0, 1], table[0, 2] = -3, c.pool.shape[0]
    check_attention(akvs.op_attention_pages(q, c.pool, table, c.len, 2), want, q, [0, 1])
    table[:] = -1
    o, l = akvs.op_attention_pages(q, c.pool, table, c.len, 2)
    assert (o == 0).all() and (l == -math.inf).all()


def test_attention_offsets_out_of_order(akvs):
    """Offsets that run backwards, overlap or leave the rows: nothing outside the tensors is touched."""
    g = gen(12)
    c = Cache(akvs, g, [200] * 6, 2, 64, BF16)
    guard = torch.zeros(1 << 22, dtype=torch.uint8, device="cuda")
    need = akvs.lib.akvs_op_attention_pages_scratch_bytes(9, 6, 8, 2, 64)
    scratch = guard[1 << 20:][:need]
    q = rnd(g, 9, 8, 64, dt=BF16)
    for off in ([0, 9, 0, 9, 0, 9, 0], [9, 8, 7, 6, 5, 4, 3], [-5, 100, -5, 100, 3, 9, 9], [0, 9, 2, 9, 1, 9, 9]):
        akvs.op_attention_pages(q, c.pool, c.table, ints([10 ** 9, -1, 200, 200, 200, 200]), 2, ints(off), scratch=scratch)
    assert (guard[:1 << 20] == 0).all() and (guard[(1 << 20) + need:] == 0).all()


def test_attention_strides_and_layers(akvs):
    """q as columns of a projection, a layer of a pool of several, tables wider than needed, pages far apart."""
    g = gen(13)
    c = Cache(akvs, g, [100, 333], 2, 128, BF16)
    qkv = rnd(g, 2, 12, 128, dt=BF16)
    want = akvs.op_attention_pages(qkv[:, :8].contiguous(), c.pool, c.table, c.len, 2)
    layers = torch.full((3, *c.pool.shape), 255, dtype=torch.uint8, device="cuda")
    layers[1] = c.pool
    wide = torch.full((2, c.width + 5), 10 ** 8, dtype=torch.int32, device="cuda")
    wide[:, :c.width] = c.table
    got = akvs.op_attention_pages(qkv[:, :8], layers[1], wide, c.len, 2)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    far = torch.empty((c.pool.shape[0], (1 << 29)), dtype=torch.uint8, device="cuda")      # offsets beyond 2^32 bytes
    assert far.numel() > 1 << 32
    spread = far[:, 64:64 + c.pool.shape[1]]
    spread.copy_(c.pool)
    got = akvs.op_attention_pages(qkv[:, :8], spread, c.table, c.len, 2)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    k, v = (torch.zeros((433, 2, 128), dtype=BF16, device="cuda") for _ in range(2))
    akvs.op_pages_append(c.k, c.v, spread, c.table, c.len, ints([0, 100, 433]))
    akvs.op_pages_read(spread, c.table, c.len, k, v, ints([0, 100, 433]))
    k2, v2 = torch.empty_like(k), torch.empty_like(v)
    akvs.op_pages_read(c.pool, c.table, c.len, k2, v2, ints([0, 100, 433]))
    assert torch.equal(k, k2) and torch.equal(v, v2)


# --------------------------------------------------------------------------------------- linear

def linear_ref(akvs, x, w):
    """y, and the sum of its terms' magnitudes."""
    N, K = w.shape
    codes, meta = akvs.op_quantize(w.view(N, 1, K), 4)
    c = torch.stack([codes & 15, codes >> 4], -1).reshape(N, K).double()
    s, m = (meta[..., i].reshape(N, K // 64).double().repeat_interleave(64, 1) for i in (0, 1))
    return x.double() @ (c * s + m).T, x.double().abs() @ (15 * s + m.abs()).T


def linear_tol(K):
    """Sums of 64 products in the tensor cores, then one term and one minimum a group, joined over up to 8 ranges."""
    return (64 + 3 * (K // 64) + 8) * 2.0 ** -23


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("N,K", [(1, 64), (16, 128), (17, 512), (130, 576), (1000, 4160), (6000, 192), (300, 9024)])
def test_linear(akvs, dt, N, K):
    g = gen(N + K)
    w = rnd(g, N, K, dt=dt, scale=0.02)
    lw = akvs.LinearQ4(w)
    for M in (1, 2, 7, 8, 9, 16, 17, 33, 64, 65, 100, 130):
        wide = rnd(g, M, K + 64, dt=dt)
        x = wide[:, 32:32 + K] if M % 2 else wide[:, :K].contiguous()
        ref, mag = linear_ref(akvs, x, w)
        y = akvs.op_linear_q4(x, lw)
        tol = half(dt) * ref.abs() + linear_tol(K) * mag + TINY[dt]
        assert ((y.double() - ref).abs() <= tol).all(), (M, ((y.double() - ref).abs() / tol).max())
        assert torch.equal(y, akvs.op_linear_q4(x, lw))
        h = rnd(g, M, N)
        out = akvs.op_linear_q4_residual(x, lw, h, torch.empty_like(h))
        ref = ref + h.double()
        assert ((out.double() - ref).abs() <= half(F32) * ref.abs() + linear_tol(K) * mag).all()
        assert akvs.op_linear_q4_residual(x, lw, h) is h and torch.equal(h, out)


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("N,K", [(2368, 1088), (2369, 192), (4736, 1088), (4737, 2048), (4800, 64), (9472, 320), (9473, 1088), (19001, 1088)])
def test_linear_rounds(akvs, dt, N, K):
    """Up to 8 rows: one tile of features for an SM, two, a round, several; ends within a round, a tile and the columns."""
    g = gen(N + K)
    w = rnd(g, N, K, dt=dt, scale=0.02)
    lw = akvs.LinearQ4(w)
    for M in (1, 5, 8):
        x = rnd(g, M, K, dt=dt)
        ref, mag = linear_ref(akvs, x, w)
        y = akvs.op_linear_q4(x, lw)
        assert ((y.double() - ref).abs() <= half(dt) * ref.abs() + linear_tol(K) * mag + TINY[dt]).all(), M
        assert torch.equal(y, akvs.op_linear_q4(x, lw))


def test_linear_large(akvs):
    """Weights so large that other kernels take them; more features than one range of a CTA, rows of every block."""
    g = gen(23)
    N, K = 4300, 27648
    w = rnd(g, N, K, dt=BF16, scale=0.02)
    lw = akvs.LinearQ4(w)
    for M in (1, 3, 4, 9, 33, 70):
        x = rnd(g, M, K, dt=BF16)
        ref, mag = linear_ref(akvs, x, w)
        y = akvs.op_linear_q4(x, lw)
        assert ((y.double() - ref).abs() <= half(BF16) * ref.abs() + linear_tol(K) * mag).all(), M
        h = rnd(g, M, N)
        out = akvs.op_linear_q4_residual(x, lw, h, torch.empty_like(h))
        assert ((out.double() - ref - h.double()).abs() <= half(F32) * out.abs() + linear_tol(K) * mag).all(), M


@pytest.mark.parametrize("M", [2, 12, 40])
def test_linear_outputs_anywhere(akvs, M):
    """Outputs that start on any value: the same bits, and nothing beside them touched."""
    g = gen(29)
    lw, x = akvs.LinearQ4(rnd(g, 516, 640, dt=F16, scale=0.05)), rnd(g, M, 640, dt=F16)
    h = rnd(g, M, 516)
    want, sums = akvs.op_linear_q4(x, lw), akvs.op_linear_q4_residual(x, lw, h, torch.empty_like(h))
    for first in (1, 2, 3, 4):
        flat, fh, fo = torch.full((M * 516 + 8,), 7.0, dtype=F16, device="cuda"), *(torch.full((M * 516 + 8,), 7.0, device="cuda") for _ in range(2))
        y, hi, ho = (t[first:first + M * 516].view(M, 516) for t in (flat, fh, fo))
        hi.copy_(h)
        akvs.op_linear_q4(x, lw, y)
        akvs.op_linear_q4_residual(x, lw, hi, ho)
        assert torch.equal(y, want) and torch.equal(ho, sums)
        assert all((t[:first] == 7).all() and (t[first + M * 516:] == 7).all() for t in (flat, fo))
        assert torch.equal(akvs.op_linear_q4_residual(x, lw, hi), sums)


def test_linear_is_as_exact_as_its_output(akvs):
    g = gen(21)
    for dt in (BF16, F16):
        w = rnd(g, 512, 8192, dt=dt, scale=0.02)
        for M in (4, 40, 100):
            x = rnd(g, M, 8192, dt=dt)
            ref, _ = linear_ref(akvs, x, w)
            err = (akvs.op_linear_q4(x, akvs.LinearQ4(w)).double() - ref).square().mean().sqrt()
            assert err <= 1.1 * (ref.to(dt).double() - ref).square().mean().sqrt()


def test_linear_sizes_of_x(akvs):
    """Rows of very different size, one with a NaN, one with an infinity, one of zeros: each by itself."""
    g = gen(22)
    for dt, sizes in ((F32, [1e-30, 1e30, 1.0]), (BF16, [1e-30, 1e30, 1.0]), (F16, [2.0 ** -20, 2.0 ** 14, 1.0])):
        for extra in (0, 40):
            w = rnd(g, 200, 1024, dt=dt, scale=0.02)
            x = torch.cat([rnd(g, 1, 1024).clamp(-3.9, 3.9) * s for s in sizes] + [rnd(g, 3 + extra, 1024)]).to(dt)
            x[3] = 0
            y = akvs.op_linear_q4(x, akvs.LinearQ4(w))
            ref, mag = linear_ref(akvs, x, w)
            if dt == F16:
                ref = ref.clamp(-65504, 65504)            # float16 saturates
            assert ((y.double() - ref).abs() <= half(dt) * ref.abs() + linear_tol(1024) * mag + TINY[dt]).all()
            x[4, 100], x[5, 1000] = math.nan, math.inf
            z = akvs.op_linear_q4(x, akvs.LinearQ4(w))
            assert torch.equal(z[:4], y[:4]) and torch.equal(z[6:], y[6:])
            assert z[4].isnan().all() and not z[5].isfinite().any()


def test_linear_from_codes(akvs):
    w = rnd(gen(1), 70, 256, dt=F16)
    codes, meta = akvs.op_quantize(w.view(70, 1, 256), 4)
    a, b = akvs.LinearQ4(w), akvs.LinearQ4.from_codes(codes, meta)
    assert torch.equal(a.packed, b.packed) and (b.N, b.K) == (70, 256)


# ----------------------------------------------------------------------------- streams and graphs

def test_streams_and_graphs(akvs):
    """A whole step captured and replayed with other inputs, lengths and pages; two steps on two streams at once."""
    g = gen(31)
    nq, nkv, hd, S = 8, 2, 128, 3
    rope = akvs.Rope(1e4, 64, layout="interleaved", scaling="yarn", factor=4.0, orig_ctx=4096)
    wo = akvs.LinearQ4(rnd(g, 256, nq * hd, dt=BF16, scale=0.02))

    class Step:
        def __init__(self, seed):
            g = gen(seed)
            self.c = Cache(akvs, g, [70, 200, 5], nkv, hd, BF16, spare=6)
            self.qkv = rnd(g, S, nq + 2 * nkv, hd, dt=BF16)
            self.h = rnd(g, S, 256)
            self.len = self.c.len + 1
            self.table = torch.full((S, 6), -1, dtype=torch.int32, device="cuda")
            self.table[:, :self.c.width] = self.c.table
            self.pos = self.c.len.clone()

        def run(self):
            q, k = akvs.op_rope_scaled(self.qkv[:, :nq], self.qkv[:, nq:nq + nkv], self.pos, rope)
            akvs.op_pages_append(k, self.qkv[:, nq + nkv:], self.c.pool, self.table, self.len)
            o, l = akvs.op_attention_pages(q, self.c.pool, self.table, self.len, nkv)
            return o, l, akvs.op_linear_q4_residual(o.view(S, -1), wo, self.h, torch.empty_like(self.h))

    one, two = Step(1), Step(2)
    want = [[y.clone() for y in x.run()] for x in (one, two)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for _ in range(20):
        for st, x in zip(streams, (one, two)):
            with torch.cuda.stream(st):
                got.append(x.run())
    torch.cuda.synchronize()
    for i, y in enumerate(got):
        assert all(torch.equal(a, b) for a, b in zip(y, want[i % 2]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = one.run()
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(out, want[0]))
    for a, b in ((one.qkv, two.qkv), (one.c.pool, two.c.pool), (one.table, two.table), (one.pos, two.pos), (one.h, two.h)):
        a.copy_(b)
    one.len.copy_(two.len)
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(out, want[1]))
    del graph


@pytest.mark.parametrize("M", [3, 12, 40, 70])
def test_linear_streams_and_graphs(akvs, M):
    """Two layers on two streams at once, each with its own scratch, and captured; the kernels for few and for many rows."""
    g = gen(M)
    ws = [akvs.LinearQ4(rnd(g, N, 1024, dt=F16, scale=0.05)) for N in (272, 1000)]
    xs = [rnd(g, M, 1024, dt=F16) for _ in range(2)]
    room = [akvs.op_linear_q4_scratch(F16, M, w.N, w.K) for w in ws]
    want = [akvs.op_linear_q4(x, w) for x, w in zip(xs, ws)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for _ in range(20):
        for st, x, w, r in zip(streams, xs, ws, room):
            with torch.cuda.stream(st):
                got.append(akvs.op_linear_q4(x, w, scratch=r))
    torch.cuda.synchronize()
    assert all(torch.equal(y, want[i % 2]) for i, y in enumerate(got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):                     # the second layer's call follows the first on one scratch
        shared = max(room, key=lambda r: r.nbytes)
        out = [akvs.op_linear_q4(x, w, scratch=shared) for x, w in zip(xs, ws)]
    for _ in range(3):
        graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(out, want))
    xs[0].copy_(xs[1])
    want = akvs.op_linear_q4(xs[1], ws[0])
    graph.replay()
    assert torch.equal(out[0], want)
    del graph


@pytest.mark.parametrize("dt", TYPES)
def test_append_codes_at_their_edges(akvs, dt):
    """Values in the middle of two codes and the next ones on either side, over scales of all sizes, and groups with
    infinities and NaN: the codes and records of the flat quantiser, bit for bit."""
    g = gen(41)
    n = 4000
    scale = (2.0 ** torch.randint(-20, 9, (n, 1, 1), generator=g, device="cuda")) * (1 + torch.rand((n, 1, 1), generator=g, device="cuda"))
    least = torch.randn((n, 1, 1), generator=g, device="cuda") * scale * 5
    steps = torch.randint(0, 31, (n, 1, 64), generator=g, device="cuda") / 2
    x = (least + steps * scale).to(dt)
    x[:, :, 0], x[:, :, 1] = least[:, :, 0].to(dt), (least + 15 * scale)[:, :, 0].to(dt)
    c, m = akvs.op_quantize(x, 4)                      # then by the records that come out of it
    s16, m16 = m[..., 0].float(), m[..., 1].float()
    y = (m16 + (torch.randint(0, 30, (n, 1, 64), generator=g, device="cuda") + 0.5) * s16)
    y = torch.nextafter(y, y + torch.randint(-1, 2, (n, 1, 64), generator=g, device="cuda")).to(dt)
    y[:, :, 0], y[:, :, 1] = x[:, :, 0], x[:, :, 1]
    x = torch.cat([x, y.clamp(x.amin(-1, keepdim=True), x.amax(-1, keepdim=True))])
    x[5, 0, 7], x[6, 0, 8], x[7, 0, 9], x[8] = math.inf, -math.inf, math.nan, math.nan
    pool = torch.zeros((n * 2 // 64 + 1, akvs.page_bytes(1, 64)), dtype=torch.uint8, device="cuda")
    table = torch.arange(pool.shape[0], device="cuda", dtype=torch.int32)[None]
    akvs.op_pages_append(x, x, pool, table, ints([2 * n]), ints([0, 2 * n]))
    codes, meta = akvs.op_quantize(x, 4)
    tok = torch.arange(2 * n, device="cuda")
    blocks = pool.reshape(-1, 4608)
    rec = blocks[:, 4096:].reshape(-1, 2, 64, 4)[tok // 64, :, tok % 64].contiguous().view(torch.int16)
    want = meta.view(torch.int16).reshape(2 * n, 1, 2)
    assert torch.equal(rec, want.expand(-1, 2, -1))
    k = blocks[:, :2048].reshape(-1, 64, 32)[tok // 64, tok % 64]                       # one group: the words in their order
    assert torch.equal(k, codes.reshape(2 * n, 32))
    at = (2048 + tok % 64 // 16 * 512 + tok // 8 % 2 * 256 + tok % 8 // 2 * 8 + tok % 2 * 2)[:, None, None, None]
    at = at + torch.arange(8, device="cuda")[:, None, None] * 32 + torch.arange(2, device="cuda")[:, None] * 4 + torch.arange(2, device="cuda")
    v = blocks[(tok // 64)[:, None], at.reshape(2 * n, 32)]
    assert torch.equal(v, codes.reshape(2 * n, 32))


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("hd,rot", [(128, 128), (128, 64), (128, 20), (72, 70)])
def test_rope_scaled_infinities(akvs, dt, layout, hd, rot):
    """An infinity reaches both values of its pair and no other; a finite float16 beyond the type's end saturates."""
    g = gen(hd + rot)
    x, rope = rnd(g, 5, 3, hd, dt=dt), akvs.Rope(1e4, rot, layout=layout)
    pos = ints([3, 100, 2001, 7, 1])
    i, j = (5, 5 + rot // 2) if layout == "half" else (4, 5)
    x[0, 1, i], x[1, 2, j], x[2, 0, i] = math.inf, -math.inf, math.nan
    if dt == F16:
        x[3, 0, i] = x[3, 0, j] = 65504.0
        x[4, 1, i] = 65504.0
    got, _ = akvs.op_rope_scaled(x, x[:, :0], pos, rope)
    ref, both = rope_ref(x, pos, rope)
    assert int(ref.isinf().sum()) == 4 and int(ref.isnan().sum()) == 2       # (no cosine or sine here is near zero)
    if dt == F16:
        assert int((ref[3:].abs() > 65504).sum()) >= 1
        ref = torch.where(ref.isfinite(), ref.clamp(-65504, 65504), ref)
    assert torch.equal(got.isnan(), ref.isnan()) and torch.equal(got.isinf(), ref.isinf())
    assert torch.equal(got[got.isinf()].double(), ref[ref.isinf()])
    fine = ref.isfinite()
    tol = half(dt) * ref.abs() + 2.0 ** -20 * both + TINY[dt]
    assert ((got.double() - ref).abs()[fine] <= tol[fine]).all()


@pytest.mark.parametrize("hd", [64, 128])
def test_read_infinities(akvs, hd):
    """Groups whose minimum is beyond float16 stand for infinities or NaN in every type; finite values beyond it saturate."""
    x = rnd(gen(hd), 6, 2, hd)
    x[0, 0, 3], x[1, 1, 3], x[2, 0, :64] = -1e5, math.nan, 1e5
    x[3, 1, 5:64], x[3, 1, :5] = 65504.0, -65504.0     # scale 8736: code 15 stands for 65536 (and 1e5 of -x for itself)
    x[4, 0, 7], x[5, 0, :] = -math.inf, -7e4
    c = Cache(akvs, gen(1), [6], 2, hd, F32, x, -x)
    for dt in TYPES:
        ko, vo = (torch.full((6, 2, hd), 9, dtype=dt, device="cuda") for _ in range(2))
        akvs.op_pages_read(c.pool, c.table, c.len, ko, vo, ints([0, 6]))
        for got, which in ((ko, 0), (vo, 1)):
            code, scale, least = c.records[which]
            ref = code * scale + least                 # (0 * inf is NaN here as there)
            if dt == F16:
                assert int((ref[ref.isfinite()].abs() > 65504).sum()) == (59 if which == 0 else 6)
                ref = torch.where(ref.isfinite(), ref.clamp(-65504, 65504), ref)
            assert int(ref.isinf().sum()) > 64 and torch.equal(got.isnan(), ref.isnan()) and torch.equal(got.isinf(), ref.isinf())
            assert torch.equal(got[got.isinf()].double(), ref[ref.isinf()])
            fine = ref.isfinite()
            assert ((got.double() - ref).abs()[fine] <= ((half(dt) + 2.0 ** -24) * ref.abs() + TINY[dt])[fine]).all()


@pytest.mark.parametrize("dt,M,N", [(F32, 9, 65535 * 128 + 200), (F16, 17, 65535 * 256 + 200), (F32, 65535 * 8 + 9, 24), (BF16, 65535 * 64 + 33, 24)])
def test_linear_many_blocks(akvs, dt, M, N):
    """More than 65535 ranges of features, or blocks of rows: the first, the last and some others."""
    g, K = gen(M + N), 64
    codes = torch.randint(0, 256, (N, 1, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    meta = torch.rand((N, 1, K // 64, 2), generator=g, device="cuda").to(F16)
    x = rnd(g, M, K, dt=dt)
    lw = akvs.LinearQ4.from_codes(codes, meta)
    assert akvs.lib.akvs_op_linear_q4_scratch_bytes({F32: 0, BF16: 1, F16: 2}[dt], M, N, K) >= 0
    y = akvs.op_linear_q4(x, lw)

    def some(n):
        return torch.cat([torch.arange(min(n, 150), device="cuda"), torch.randint(0, n, (200,), generator=g, device="cuda"),
                          torch.arange(max(0, n - 500), n, device="cuda")])
    rows, feats = some(M), some(N)
    c = torch.stack([codes[feats, 0] & 15, codes[feats, 0] >> 4], -1).reshape(len(feats), K).double()
    s, m = (meta[feats, 0, :, i].double().repeat_interleave(64, 1) for i in (0, 1))
    ref, mag = x[rows].double() @ (c * s + m).T, x[rows].double().abs() @ (15 * s + m.abs()).T
    got = y[rows][:, feats]
    assert ((got.double() - ref).abs() <= half(dt) * ref.abs() + linear_tol(K) * mag + TINY[dt]).all()
    h = torch.full((M, N), 3.0, device="cuda")
    akvs.op_linear_q4_residual(x, lw, h)
    assert ((h[rows][:, feats].double() - ref - 3).abs() <= half(F32) * (ref + 3).abs() + linear_tol(K) * mag).all()


@pytest.mark.parametrize("M", [5, 9, 40])
def test_linear_float_sums_of_x(akvs, M):
    """The sums of x that minima are multiplied by keep all bits of a float: rows with one value of 24 bits, weights without
    extent.  (Every step is exact; half a last bit is left for the one sum.)"""
    g = gen(M)
    lw = akvs.LinearQ4(torch.ones((130, 64), device="cuda"))
    value = torch.randint(1 << 23, 1 << 24, (M,), generator=g, device="cuda").float() * 2.0 ** torch.randint(-30, 8, (M,), generator=g, device="cuda")
    x = torch.zeros((M, 64), device="cuda")
    x[torch.arange(M), torch.randint(0, 64, (M,), generator=g, device="cuda")] = value
    y = akvs.op_linear_q4(x, lw)
    assert ((y.double() - value[:, None].double()).abs() <= 2.0 ** -24 * value[:, None].double()).all()


@pytest.mark.parametrize("M", [5, 9, 40])
def test_linear_float_x_is_whole(akvs, M):
    """Float rows enter the products with all 24 bits: weights of exactly 1 (code 1, scale 1, minimum 0) and one value a row,
    so that every step is exact; half a last bit is left for the sum of the pieces."""
    g = gen(M + 1)
    codes = torch.full((130, 1, 64), 0x11, dtype=torch.uint8, device="cuda")
    meta = torch.tensor([1.0, 0.0], dtype=F16, device="cuda").expand(130, 1, 2, 2).contiguous()
    lw = akvs.LinearQ4.from_codes(codes, meta)
    value = torch.randint(1 << 23, 1 << 24, (M,), generator=g, device="cuda").float() * 2.0 ** torch.randint(-30, 8, (M,), generator=g, device="cuda")
    x = torch.zeros((M, 128), device="cuda")
    x[torch.arange(M), torch.randint(0, 128, (M,), generator=g, device="cuda")] = value
    y = akvs.op_linear_q4(x, lw)
    assert ((y.double() - value[:, None].double()).abs() <= 2.0 ** -24 * value[:, None].double()).all()


def test_linear_float_is_exact_enough(akvs):
    """Root mean square error of float rows.  A group's products are cut off 12 times (4 steps of 16 columns, 3 pieces) by up to
    2^-23 of a sum of codes times x, which is 65 here (codes of mean 7.5, deviation 3.3, 64 columns); uniform and independent, times
    the scale of 0.0061, over 128 groups that is 5.9e-7 of y's 1.81, and 400 float additions of a sum below that make 2e-7:
    together under 2^-20."""
    g = gen(24)
    w = rnd(g, 512, 8192, scale=0.02)
    lw = akvs.LinearQ4(w)
    for M in (1, 4, 8, 9, 40):
        x = rnd(g, M, 8192)
        ref, _ = linear_ref(akvs, x, w)
        err = (akvs.op_linear_q4(x, lw).double() - ref).square().mean().sqrt()
        assert err <= 2.0 ** -20 * ref.square().mean().sqrt(), M


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("nq,nkv", [(4, 2), (8, 2), (16, 1)])
def test_attention_float_is_exact_enough(akvs, hd, nq, nkv):
    """Root mean square errors of float rows, several a sequence: the bound of one row a sequence above."""
    g = gen(hd + nq)
    c = Cache(akvs, g, [2500, 700, 65], nkv, hd, F32)
    off = [0, 7, 8, 40]
    q = rnd(g, 40, nq, hd)
    o, l = akvs.op_attention_pages(q, c.pool, c.table, c.len, nkv, ints(off))
    ref, lse, mag, _ = attention_ref(c, q, off)
    rms = lambda x: x.double().square().mean().sqrt()  # noqa: E731
    assert rms(o - ref) <= 2.0 ** -20 * rms(mag)
    assert rms(l - lse) <= 2.0 ** -20 * 8                  # scores and log-sum-exps are below 16 here


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("nq,nkv,hd", [(32, 8, 128), (8, 8, 64), (20, 4, 128)])
def test_attention_questions(akvs, dt, nq, nkv, hd):
    """Questions of 64 and 128 rows over a context, beside an answer's one row and a sequence that is no longer than its rows."""
    g = gen(nq + hd)
    for rows, lens in (([128], [1500]), ([64, 1, 100], [900, 333, 100]), ([65, 128], [65, 130])):
        c = Cache(akvs, g, lens, nkv, hd, dt)
        off = np.concatenate([[0], np.cumsum(rows)]).tolist()
        q = rnd(g, off[-1], nq, hd, dt=dt, scale=1.5)
        check_attention(akvs.op_attention_pages(q, c.pool, c.table, c.len, nkv, ints(off)), c, q, off)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("nq,nkv", [(2, 2), (8, 1), (4, 2)])
def test_attention_float_against_its_output(akvs, hd, nq, nkv):
    """Root mean square error of float rows against the output, which is a mean of thousands of values and smaller than they
    are.  Terms and output both grow with the root of the number of tokens, so they are compared a token: a product's sum over 16
    tokens is cut off by up to 2^-23 of itself, whose codes (8.2 steps with the complements) stand beside values of 3.3 steps:
    3e-7; the additions of such sums, 20 a CTA, 1.5e-7; exp2, 2^-22 of a weight, 1.4e-7; scores, of 2^-22 at most, as much.
    Independent, these are under 5e-7, and together at worst under 2^-20."""
    g = gen(hd + nq)
    lens = [5556, 2000, 1200]
    c = Cache(akvs, g, lens, nkv, hd, F32)
    q = rnd(g, 3, nq, hd, scale=1.5)
    o, _ = akvs.op_attention_pages(q, c.pool, c.table, c.len, nkv)
    ref, _, _, _ = attention_ref(c, q, [0, 1, 2, 3])
    assert (o - ref).square().mean().sqrt() <= 2.0 ** -20 * ref.square().mean().sqrt()


@pytest.mark.parametrize("dt", [BF16, F16])
@pytest.mark.parametrize("M", [1, 2, 9, 17, 40])
def test_linear_residual_is_exact_enough(akvs, dt, M):
    """Root mean square error of float results of 16-bit rows.  A group's products are cut off 4 times by up to 2^-23 of a sum of
    codes times x, 65 here; uniform and independent, times the scale of 0.0061, over 64 groups that is 3.4e-7 of y's 1.28, and 200
    float additions make 2e-7: under 2^-20."""
    g = gen(M)
    for N in (40, 300):
        for _ in range(8):
            w, x = rnd(g, N, 4096, dt=dt, scale=0.02), rnd(g, M, 4096, dt=dt)
            ref, _ = linear_ref(akvs, x, w)
            out = akvs.op_linear_q4_residual(x, akvs.LinearQ4(w), torch.zeros((M, N), device="cuda"))
            assert (out - ref).square().mean().sqrt() <= 2.0 ** -20 * ref.square().mean().sqrt()


@pytest.mark.parametrize("dt", TYPES)
def test_attention_scores_of_short_sequences(akvs, dt):
    """A sequence of one token has its score for a log-sum-exp: the score's own error, 2^-22 of the terms it is a sum of, which are
    as large as their root mean square sum over head_dim here."""
    g = gen(51)
    for hd, nq, nkv in ((64, 4, 2), (128, 8, 1)):
        c = Cache(akvs, g, [1] * 40, nkv, hd, dt)
        q = rnd(g, 40, nq, hd, dt=dt, scale=1.5)
        _, lse = akvs.op_attention_pages(q, c.pool, c.table, c.len, nkv)
        _, ref, _, _ = attention_ref(c, q, list(range(41)))
        size = (q.double().reshape(40, nkv, nq // nkv, hd).square()[..., None, :] * c.size(0).reshape(40, nkv, 1, 1, hd).square()).sum(-1).sqrt() / math.sqrt(hd)
        assert (lse - ref).square().mean().sqrt() <= 2.0 ** -22 * size.square().mean().sqrt()
