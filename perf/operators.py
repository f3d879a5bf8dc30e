"""The operators that answer from a shared context cache, as measurable cases.

A corrected prefill leaves the K/V of a context.  What a program does next with it: normalise
and rotate the queries and keys of new tokens (`qk_norm_rope`), let many sequences attend to
the one context and to their own tokens (`attention_shared`), keep account of how much weight
each cached key received (`attention_mass`), and shrink the cache to its heaviest tokens
(`evict`).  With `own` false, `run` computes them from elementary torch operations in 32 bits;
with `own` true it calls the library.
"""
import math
import random

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
EPS, BASE = 1e-6, 1e4


# ------------------------------------------------------------------------------------- cases

def _norm(n, nq, nkv, hd, dtype, far=0):
    return {"op": "qk_norm_rope", "n": n, "nq": nq, "nkv": nkv, "hd": hd, "dtype": dtype, "far": far}


def _shared(S, rows, P, cap, nq, nkv, hd, dtype, room=0):
    return {"op": "attention_shared", "S": S, "rows": rows, "P": P, "cap": cap, "nq": nq, "nkv": nkv, "hd": hd,
            "dtype": dtype, "room": room}


def _mass(R, T, causal, nq, nkv, hd, dtype):
    return {"op": "attention_mass", "R": R, "T": T, "causal": causal, "nq": nq, "nkv": nkv, "hd": hd, "dtype": dtype}


def _evict(L, T, budget, sink, recent, nkv, hd, dtype):
    return {"op": "evict", "L": L, "T": T, "budget": budget, "sink": sink, "recent": recent, "nkv": nkv, "hd": hd,
            "dtype": dtype}


def listed():
    """Head counts, widths and context lengths are those of the benchmark configurations where
    they name them (16/2, 32/8 and 40/8 heads of 128, 4/2 heads of 64; contexts of 8192 to 12288
    tokens with 128 query tokens); the longer contexts are generic."""
    return [
        # one new token of one sequence: nothing but latency
        dict(_norm(1, 32, 8, 128, "bf16", far=8320), name="norm+rope, one token"),
        # the float configuration's whole prompt
        dict(_norm(288, 4, 2, 64, "f32"), name="norm+rope, float prompt"),
        # a whole prompt of the widest configuration: memory traffic
        dict(_norm(11648, 40, 8, 128, "f16"), name="norm+rope, wide prompt"),
        # a few float sequences over a short context
        dict(_shared(4, 1, 256, 32, 4, 2, 64, "f32"), name="shared, float"),
        # one answer being generated from one context
        dict(_shared(1, 1, 8320, 256, 32, 8, 128, "bf16"), name="shared, one answer"),
        # a batch of sampled answers to the same question
        dict(_shared(16, 1, 12416, 256, 32, 8, 128, "f16"), name="shared, 16 answers"),
        # a serving batch over one long context, answers of up to 1024 tokens
        dict(_shared(128, 1, 32768, 1024, 32, 8, 128, "bf16"), name="shared, 128 answers"),
        # many questions of 1 to 64 tokens put to the same units at once (their first pass)
        dict(_shared(24, 64, 16384, 96, 16, 2, 128, "f16", room=17), name="shared, 24 questions"),
        # accounting for one decoding step of 16 sequences
        dict(_mass(16, 12416, False, 32, 8, 128, "bf16"), name="mass, one step"),
        # accounting for the last 512 tokens of a long prompt
        dict(_mass(512, 32768, True, 40, 8, 128, "f16"), name="mass, window"),
        # one layer's cache cut to a quarter
        dict(_evict(1, 8320, 2048, 4, 128, 8, 128, "bf16"), name="evict, one layer"),
        # the whole cache of 32 layers cut to a third
        dict(_evict(32, 12416, 4096, 4, 256, 8, 128, "f16"), name="evict, all layers"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def draw(rng):
    op = rng.choice(("qk_norm_rope", "attention_shared", "attention_shared", "attention_mass", "evict"))
    dtype = rng.choice(("f32", "bf16", "bf16", "f16", "f16"))
    nkv, hd = rng.choice((1, 2, 2, 4, 8)), rng.choice((64, 128, 128))
    nq = nkv * rng.choice((1, 2, 4, 4, 5, 8))
    most = {}
    for c in listed():
        w = work(c)
        b = most.setdefault(c["op"], {"bytes": 0.0, "flops": 0.0})
        b["bytes"], b["flops"] = max(b["bytes"], w["bytes"]), max(b["flops"], w["flops"])
    # the 32-bit products run on the CUDA cores, at some hundredth of the 16-bit rate
    room = most[op]["flops"] / (64 if dtype == "f32" else 1)
    while True:
        if op == "qk_norm_rope":
            c = _norm(_log(rng, 1, 12000), nq, nkv, hd, dtype, far=rng.choice((0, 0, 100000)))
        elif op == "attention_shared":
            rows = rng.choice((1, 1, 1, 4, 48))
            c = _shared(_log(rng, 1, 160), rows, _log(rng, 1, 50000), _log(rng, rows, 1200), nq, nkv, hd, dtype,
                        room=rng.choice((0, 0, 5)))
        elif op == "attention_mass":
            T = _log(rng, 1, 50000)
            causal = rng.random() < 0.5
            c = _mass(min(_log(rng, 1, 600), T), T, causal, nq, nkv, hd, dtype)
        else:
            T = _log(rng, 16, 40000)
            B = rng.randint(1, T)
            sink = rng.randint(0, min(8, B))
            c = _evict(rng.choice((1, 1, 2, 7, 24)), T, B, sink, rng.randint(0, min(512, B - sink)), nkv, hd, dtype)
        w = work(c)
        if w["bytes"] <= most[op]["bytes"] and w["flops"] <= room:
            return c


def _rows_of(c):
    """Rows of every sequence: 1, or an odd mixture of 1 to `rows`."""
    r = random.Random(c["S"] * 1000 + c["rows"])
    return [1 if c["rows"] == 1 else r.randint(1, c["rows"]) for _ in range(c["S"])]


def _lens_of(c):
    """Tokens of its own that every sequence holds, its new rows included."""
    r = random.Random(c["S"] * 7 + c["cap"])
    return [r.randint(min(n, c["cap"]), c["cap"]) for n in _rows_of(c)]


def _span(c):
    """Keys that the rows of an attention_mass case see, all together."""
    return c["R"] * c["T"] - (c["R"] * (c["R"] - 1) // 2 if c["causal"] else 0)


def work(c):
    es, hd = BYTES[c["dtype"]], c["hd"]
    if c["op"] == "qk_norm_rope":
        el = c["n"] * (c["nq"] + c["nkv"]) * hd
        return {"bytes": 2.0 * el * es + c["n"] * 4 + 2 * hd * 4, "flops": 7.0 * el}
    if c["op"] == "attention_shared":
        rows, lens = _rows_of(c), _lens_of(c)
        R, row = sum(rows), c["nkv"] * hd * es
        seen = R * c["P"] + sum(n * l - n * (n - 1) // 2 for n, l in zip(rows, lens))
        return {"bytes": 2.0 * R * c["nq"] * hd * es + 2.0 * (c["P"] + sum(lens)) * row + R * c["nq"] * 4.0,
                "flops": 4.0 * hd * c["nq"] * seen}
    if c["op"] == "attention_mass":
        return {"bytes": float(c["R"] * c["nq"] * (hd * es + 4) + c["T"] * c["nkv"] * (hd * es + 8)),
                "flops": 2.0 * hd * c["nq"] * _span(c)}
    kept = c["L"] * c["budget"] * c["nkv"]
    return {"bytes": float(c["L"] * c["T"] * c["nkv"] * 4 + kept * (4 * hd * es + 8)), "flops": 0.0}


# ------------------------------------------------------------------------------------ inputs

def _visible(c, dev):
    lo = torch.zeros(c["R"], dtype=torch.int32, device=dev)
    hi = torch.full((c["R"],), c["T"] - 1, dtype=torch.int32, device=dev)
    if c["causal"]:
        hi -= torch.arange(c["R"] - 1, -1, -1, dtype=torch.int32, device=dev)
    return lo, hi


def prepare(c, seed):
    dev, dt = "cuda", DTYPES[c["dtype"]]
    g = torch.Generator(device=dev).manual_seed(int(seed))
    nkv, hd = c["nkv"], c["hd"]

    def rnd(*shape, scale=1.0, dtype=dt):
        return (torch.randn(shape, generator=g, device=dev) * scale).to(dtype)

    s = {"case": c}
    if c["op"] == "qk_norm_rope":
        n, nq = c["n"], c["nq"]
        # q and k are column ranges of one projection's output, as a fused product leaves them
        qkv = rnd(n, nq + 2 * nkv, hd, scale=1.5)
        s["q"], s["k"] = qkv[:, :nq], qkv[:, nq:nq + nkv]
        s["gq"], s["gk"] = (1 + rnd(hd, scale=0.3, dtype=torch.float32) for _ in range(2))
        s["pos"] = torch.arange(c["far"], c["far"] + n, dtype=torch.int32, device=dev)
    elif c["op"] == "attention_shared":
        rows, lens = _rows_of(c), _lens_of(c)
        R = sum(rows)
        # scores of standard deviation about 1.5: some keys matter, most do not
        s["q"] = rnd(R, c["nq"], hd, scale=1.5)
        s["pk"], s["pv"] = rnd(c["P"], nkv, hd), rnd(c["P"], nkv, hd)
        s["sk"], s["sv"] = rnd(c["S"], c["cap"], nkv, hd), rnd(c["S"], c["cap"], nkv, hd)
        s["lens"] = torch.tensor(lens, dtype=torch.int32, device=dev)
        off = np.concatenate([[0], np.cumsum(rows)])
        s["off"] = None if c["rows"] == 1 else torch.tensor(off, dtype=torch.int32, device=dev)
        # a padded batch: rows behind the last sequence's, which belong to nobody
        if c["room"] and c["rows"] > 1:
            s["q"] = torch.cat([s["q"], rnd(c["room"], c["nq"], hd)])
        s["used"] = R
        s["out"], s["lse"] = torch.zeros_like(s["q"]), torch.zeros(s["q"].shape[:2], device=dev)
        s["row_seq"] = torch.repeat_interleave(torch.arange(c["S"], device=dev), torch.tensor(rows, device=dev))
        after = torch.cat([torch.arange(n - 1, -1, -1) for n in rows]).to(dev)
        s["row_len"] = s["lens"].long()[s["row_seq"]] - after
    elif c["op"] == "attention_mass":
        s["q"], s["k"] = rnd(c["R"], c["nq"], hd, scale=1.5), rnd(c["T"], nkv, hd)
        s["lo"], s["hi"] = _visible(c, dev)
        s["mass"] = torch.rand((nkv, c["T"]), generator=g, device=dev)
        seen = torch.arange(c["T"], device=dev)[None, :] <= s["hi"][:, None]
        lse = torch.empty((c["R"], c["nq"]), device=dev)
        gr = c["nq"] // nkv
        for h in range(nkv):      # head by head: the scores of all of them need not exist at once
            x = torch.einsum("rgd,td->rgt", s["q"][:, h * gr:(h + 1) * gr].float(), s["k"][:, h].float()) / math.sqrt(hd)
            lse[:, h * gr:(h + 1) * gr] = torch.logsumexp(x.masked_fill(~seen[:, None, :], -math.inf), -1)
        s["lse"] = lse
    else:
        L, T = c["L"], c["T"]
        # weights fall off steeply and keys that were never looked at tie at zero
        m = torch.rand((L, nkv, T), generator=g, device=dev)
        s["mass"] = torch.where(m < 0.3, torch.zeros_like(m), (m * 9).exp())
        s["k"], s["v"] = rnd(L, T, nkv, hd), rnd(L, T, nkv, hd)
    return s


# --------------------------------------------------------------------------------- plain forms

def _norm_rope(x, gain, cos, sin):
    x = x.float()
    x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * gain
    a, b = x.chunk(2, -1)
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _plain_qk_norm_rope(s):
    hd = s["q"].shape[-1]
    # the angle of a far position needs more than 24 bits
    freq = BASE ** (-2.0 * torch.arange(hd // 2, device=s["q"].device, dtype=torch.float64) / hd)
    ang = s["pos"].double()[:, None, None] * freq
    cos, sin = ang.cos().float(), ang.sin().float()
    return [_norm_rope(x, g, cos, sin).to(x.dtype) for x, g in ((s["q"], s["gq"]), (s["k"], s["gk"]))]


def _plain_attention_shared(s):
    R, (_, nq, hd), nkv = s["used"], s["q"].shape, s["pk"].shape[1]
    q = s["q"][:R].float().reshape(R, nkv, nq // nkv, hd).permute(1, 0, 2, 3) / math.sqrt(hd)      # [h][r][g][d]
    pk, pv = (x.float().permute(1, 0, 2) for x in (s["pk"], s["pv"]))                              # [h][t][d]
    sk, sv = (x.float().permute(2, 0, 1, 3)[:, s["row_seq"]] for x in (s["sk"], s["sv"]))          # [h][r][t][d]
    seen = torch.arange(sk.shape[2], device=q.device)[None, :] < s["row_len"][:, None]             # [r][t]
    x = torch.matmul(q.flatten(1, 2), pk.transpose(1, 2)).reshape(*q.shape[:3], -1)
    y = torch.matmul(q, sk.transpose(2, 3)).masked_fill(~seen[None, :, None, :], -math.inf)
    top = torch.maximum(x.amax(-1), y.amax(-1))[..., None]
    x, y = (x - top).exp_(), (y - top).exp_()
    total = x.sum(-1, keepdim=True) + y.sum(-1, keepdim=True)
    o = torch.matmul(x.flatten(1, 2), pv).reshape(q.shape) + torch.matmul(y, sv.masked_fill(~seen[None, :, :, None], 0))
    s["out"][:R] = (o / total).permute(1, 0, 2, 3).reshape(R, nq, hd).to(s["q"].dtype)
    s["lse"][:R] = (top + total.log())[..., 0].permute(1, 0, 2).reshape(R, nq)
    return [s["out"], s["lse"]]


def _plain_attention_mass(s):
    (R, nq, hd), (T, nkv, _) = s["q"].shape, s["k"].shape
    q = s["q"].float().reshape(R, nkv, nq // nkv, hd).permute(1, 0, 2, 3)
    x = torch.matmul(q.flatten(1, 2), s["k"].float().permute(1, 2, 0)).reshape(*q.shape[:3], T) / math.sqrt(hd)
    x = (x - s["lse"].reshape(R, nkv, -1).permute(1, 0, 2)[..., None]).exp_()
    t = torch.arange(T, device=x.device)[None, :]
    seen = (s["lo"][:, None] <= t) & (t <= s["hi"][:, None])
    return s["mass"] + x.masked_fill_(~seen[None, :, None, :], 0).sum((1, 2))


def _plain_evict(s):
    c, mass = s["case"], s["mass"]
    L, nkv, T = mass.shape
    m = mass.clone()
    m[..., :c["sink"]] = math.inf
    m[..., T - c["recent"]:] = math.inf
    idx = torch.sort(m, dim=-1, descending=True, stable=True).indices[..., :c["budget"]].sort(-1).values
    at = idx.transpose(1, 2)[..., None].expand(L, c["budget"], nkv, c["hd"])
    return [idx.int(), torch.gather(s["k"], 1, at), torch.gather(s["v"], 1, at), torch.gather(mass, 2, idx)]


def run(s):
    op = s["case"]["op"]
    if own:
        import paper_2607_21604_b200 as akvs
        if op == "qk_norm_rope":
            return akvs.op_qk_norm_rope(s["q"], s["k"], s["gq"], s["gk"], s["pos"], EPS, BASE)
        if op == "attention_shared":
            return akvs.op_attention_shared(s["q"], s["pk"], s["pv"], s["sk"], s["sv"], s["lens"], s["off"], s["out"], s["lse"])
        if op == "attention_mass":
            return akvs.op_attention_mass(s["q"], s["k"], s["lse"], s["lo"], s["hi"], s["mass"])
        c = s["case"]
        return akvs.op_evict(s["mass"], s["k"], s["v"], c["budget"], c["sink"], c["recent"])
    return {"qk_norm_rope": _plain_qk_norm_rope, "attention_shared": _plain_attention_shared,
            "attention_mass": _plain_attention_mass, "evict": _plain_evict}[op](s)


# ------------------------------------------------------------------------- definition, 64 bits

def exact(c, seed):
    s = prepare(c, seed)
    if c["op"] == "qk_norm_rope":
        out = []
        i = np.arange(c["hd"] // 2)
        ang = s["pos"].cpu().numpy()[:, None].astype(np.float64) * np.power(BASE, -i / (c["hd"] / 2))
        turn = torch.from_numpy(np.exp(1j * ang)).cuda()[:, None]
        for x, gain in ((s["q"], s["gq"]), (s["k"], s["gk"])):
            x = x.double()
            x = x / (x.pow(2).sum(-1, keepdim=True) / c["hd"] + EPS).sqrt() * gain.double()
            z = torch.complex(x[..., :c["hd"] // 2], x[..., c["hd"] // 2:]) * turn
            out.append(torch.cat([z.real, z.imag], -1))
        return out
    if c["op"] == "attention_shared":
        o, lse = s["out"].double(), s["lse"].double()
        group = c["nq"] // c["nkv"]
        seq, n = s["row_seq"].tolist(), s["row_len"].tolist()
        # sequence by sequence, head by head, over its keys laid end to end
        for b in range(c["S"]):
            rows = [r for r in range(s["used"]) if seq[r] == b]
            own_keys = max(0, max(n[r] for r in rows))
            for h in range(c["nkv"]):
                k = torch.cat([s["pk"][:, h], s["sk"][b, :own_keys, h]]).double()
                v = torch.cat([s["pv"][:, h], s["sv"][b, :own_keys, h]]).double()
                q = s["q"][rows, h * group:(h + 1) * group].double()
                x = torch.einsum("rgd,td->rgt", q, k) * c["hd"] ** -0.5
                for i, r in enumerate(rows):
                    x[i, :, c["P"] + max(0, n[r]):] = -math.inf
                z = torch.logsumexp(x, -1)
                lse[rows[0]:rows[-1] + 1, h * group:(h + 1) * group] = z
                o[rows[0]:rows[-1] + 1, h * group:(h + 1) * group] = torch.einsum("rgt,td->rgd", (x - z[..., None]).exp(), v)
        return [o, lse]
    if c["op"] == "attention_mass":
        group = c["nq"] // c["nkv"]
        mass = s["mass"].double()
        t = torch.arange(c["T"], device="cuda")
        for h in range(c["nq"]):
            x = s["q"][:, h].double() @ s["k"][:, h // group].double().T * c["hd"] ** -0.5
            p = (x - s["lse"][:, h, None].double()).exp()
            mass[h // group] += (p * (t >= s["lo"][:, None]) * (t <= s["hi"][:, None])).sum(0)
        return mass
    m, T = s["mass"].cpu().numpy(), c["T"]
    idx = np.empty((c["L"], c["nkv"], c["budget"]), np.int64)
    always = np.concatenate([np.arange(c["sink"]), np.arange(T - c["recent"], T)])
    for l in range(c["L"]):
        for h in range(c["nkv"]):
            order = np.lexsort((np.arange(T), -m[l, h]))
            free = order[(order >= c["sink"]) & (order < T - c["recent"])][:c["budget"] - len(always)]
            idx[l, h] = np.sort(np.concatenate([always, free]))
    at = torch.from_numpy(idx).cuda()
    pick = lambda x: torch.stack([torch.stack([x[l][at[l, h], h] for h in range(c["nkv"])], 1) for l in range(c["L"])])  # noqa: E731
    return [at.int(), pick(s["k"]).double(), pick(s["v"]).double(), torch.gather(s["mass"], 2, at).double()]
