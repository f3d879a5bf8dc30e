"""Answers that go on from a prefill's cache in 4 bits: the context goes into pages, the answers branch off it, and every
step runs on 4-bit weights.  The same steps in 64 bits, from the values that weights and pages stand for."""
import math

import pytest
import torch

import testgen
from gpu_helpers import Case

pytestmark = pytest.mark.gpu


def rms(h, gain, eps):
    return h * torch.rsqrt(h.square().mean(-1, keepdim=True) + eps) * gain


class Weights:
    """A layer's matrices in 4 bits, q, k and v as one and gate and up as one; and the values they stand for."""

    def __init__(self, akvs, w):
        self.lin, self.val = {}, {}
        for name, parts in (("qkv", ("wq", "wk", "wv")), ("o", ("wo",)), ("up", ("w_gate", "w_up")), ("down", ("w_down",))):
            m = torch.cat([w[p] for p in parts]).contiguous()
            N, K = m.shape
            codes, meta = akvs.op_quantize(m.view(N, 1, K), 4)
            self.lin[name] = akvs.LinearQ4.from_codes(codes, meta)
            c = torch.stack([codes & 15, codes >> 4], -1).reshape(N, K // 64, 64).double()
            self.val[name] = (c * meta[:, 0, :, :1].double() + meta[:, 0, :, 1:].double()).reshape(N, K)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_answers_in_four_bits(dtype, layout):
    import paper_2607_21604_b200 as akvs
    hd, d, ff = (64, 128, 192) if dtype == "f32" else (128, 256, 768)
    case = Case(testgen.Workload("q4-" + dtype, testgen.ModelCfg("q4-" + dtype, 2, d, 4, 2, hd, ff, 512, dtype), 4, 30, 70, 9, (2500,)))
    cfg, model = case.cfg, case.gmodel
    nq, nkv, L = cfg.n_q_heads, cfg.n_kv_heads, cfg.n_layers
    hid, k, v = akvs.alloc_outputs(model, case.N, case.nq)
    case.encode()
    akvs.prefill_corrected(model, case.store, case.req, None, akvs.MODE_FULL, hid, k, v, None, case.workspace(2))
    layers = [Weights(akvs, w) for w in model.layers]
    # the context into pages; three answers branch off
    T, S, steps = k.shape[1], 3, 4
    pool = akvs.PagePool(L, 24, nkv, hd)
    context = pool.open()
    pool.grow([context], T)
    table, lens = pool.table([context])
    for l in range(L):
        akvs.op_pages_append(k[l], v[l], pool[l], table, lens, torch.tensor([0, T], dtype=torch.int32, device="cuda"))
    answers = pool.fork(context, S)
    pool.close(context)
    # the prefill turns halves by plain frequencies; another layout stands for a cache that its caller turned alike
    rope = akvs.Rope(cfg.rope_base, hd, layout=layout)
    ids = torch.randint(0, cfg.vocab, (steps, S), generator=torch.Generator().manual_seed(3)).cuda()
    values = {}                                        # (answer, layer): K and V that stand in its pages

    for step in range(steps):
        pool.grow(answers)
        if step == 2:
            pool.compact()
        table, lens = pool.table(answers)
        pos = lens - 1
        h = model.tok_emb[ids[step]].float()
        ref = h.double()
        for l, (w, q4) in enumerate(zip(model.layers, layers)):
            x = rms(h, w["attn_norm"], cfg.rms_eps).to(k.dtype)
            qkv = akvs.op_linear_q4(x, q4.lin["qkv"]).view(S, nq + 2 * nkv, hd)
            q, kn = akvs.op_rope_scaled(qkv[:, :nq], qkv[:, nq:nq + nkv], pos, rope)
            akvs.op_pages_append(kn, qkv[:, nq + nkv:], pool[l], table, lens)
            o, lse = akvs.op_attention_pages(q, pool[l], table, lens, nkv)
            akvs.op_linear_q4_residual(o.view(S, -1), q4.lin["o"], h)
            x = rms(h, w["mlp_norm"], cfg.rms_eps).to(k.dtype)
            g, u = akvs.op_linear_q4(x, q4.lin["up"]).float().chunk(2, -1)
            akvs.op_linear_q4_residual((torch.nn.functional.silu(g) * u).to(k.dtype), q4.lin["down"], h)

            # in 64 bits
            y = rms(ref, w["attn_norm"].double(), cfg.rms_eps) @ q4.val["qkv"].T
            y = y.view(S, nq + 2 * nkv, hd)
            f = cfg.rope_base ** (-2.0 * torch.arange(hd // 2, device="cuda", dtype=torch.float64) / hd)
            ang = pos.double()[:, None, None] * f
            a, b = (slice(0, hd // 2), slice(hd // 2, hd)) if layout == "half" else (slice(0, hd, 2), slice(1, hd, 2))
            z = y.clone()
            z[..., a], z[..., b] = y[..., a] * ang.cos() - y[..., b] * ang.sin(), y[..., b] * ang.cos() + y[..., a] * ang.sin()
            att = torch.empty((S, nq, hd), dtype=torch.float64, device="cuda")
            for s, seq in enumerate(answers):
                n = int(lens[s])
                kv = [torch.empty((n, nkv, hd), device="cuda") for _ in range(2)]
                akvs.op_pages_read(pool[l], table[s:s + 1], lens[s:s + 1], kv[0], kv[1], torch.tensor([0, n], dtype=torch.int32, device="cuda"))
                # the new token's values: half a step of its groups, which are off like the row itself; the older ones as before
                for got, want in ((kv[0][-1], z[s, nq:nq + nkv]), (kv[1][-1], y[s, nq + nkv:])):
                    group = want.view(nkv, hd // 64, 64)
                    width = (group.amax(-1) - group.amin(-1)).repeat_interleave(64, -1).view(nkv, hd)
                    assert ((got - want).abs() <= width / 30 * 1.05 + 0.03 * want.abs().amax()).all()
                if (seq, l) in values:
                    assert all(torch.equal(p, c[:-1]) for p, c in zip(values[seq, l], kv))
                values[seq, l] = kv
                kk, vv = (c.double().repeat_interleave(nq // nkv, 1) for c in kv)
                p = (torch.einsum("hd,thd->ht", z[s, :nq], kk) / math.sqrt(hd)).softmax(-1)
                att[s] = torch.einsum("ht,thd->hd", p, vv)
            ref = ref + att.view(S, -1) @ q4.val["o"].T
            y = rms(ref, w["mlp_norm"].double(), cfg.rms_eps) @ q4.val["up"].T
            g, u = y.chunk(2, -1)
            ref = ref + (g * g.sigmoid() * u) @ q4.val["down"].T
        # about six roundings of half a step a layer, added up like independent ones, under the 1e-2 (floats: 2e-3) of the
        # prefill's tests
        assert ((h - ref).norm(dim=-1) <= case.tol * ref.norm(dim=-1)).all(), ((h - ref).norm(dim=-1) / ref.norm(dim=-1))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_answers_over_moved_and_cut_pages(dtype):
    """Answers go on over pages that a compaction moved, and one of them from where it was cut within a page that another
    still holds: the same bits as before the move, and the values of the tokens that are left."""
    import paper_2607_21604_b200 as akvs
    L, nq, nkv, hd, T = 2, 8, 2, 128, 150
    g = torch.Generator(device="cuda").manual_seed(17)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda").to(dtype)  # noqa: E731
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    pool = akvs.PagePool(L, 30, nkv, hd)
    first, context = pool.open(), pool.open()
    pool.grow([first], 300)                            # the lowest pages; it leaves before the others do
    pool.grow([context], T)
    table, lens = pool.table([context])
    for l in range(L):
        akvs.op_pages_append(rnd(T, nkv, hd), rnd(T, nkv, hd), pool[l], table, lens, ints(0, T))

    def step(seqs):
        """A new token of each; its row of every layer."""
        pool.grow(seqs)
        table, lens = pool.table(seqs)
        for l in range(L):
            akvs.op_pages_append(rnd(len(seqs), nkv, hd), rnd(len(seqs), nkv, hd), pool[l], table, lens)

    def attend(seqs, q):
        table, lens = pool.table(seqs)
        return [akvs.op_attention_pages(q[l], pool[l], table, lens, nkv) for l in range(L)]

    def values(seq):
        table, lens = pool.table([seq])
        n, out = pool.length[seq], []
        for l in range(L):
            kv = [torch.empty((n, nkv, hd), device="cuda") for _ in range(2)]
            akvs.op_pages_read(pool[l], table, lens, *kv, ints(0, n))
            out.append(kv)
        return out

    answers = pool.fork(context, 3)
    pool.close(context)
    step(answers)
    q = rnd(L, 3, nq, hd)
    before, held = attend(answers, q), [values(s) for s in answers]
    pool.close(first)
    assert pool.compact() > 0
    assert all(torch.equal(a, b) for x, y in zip(attend(answers, q), before) for a, b in zip(x, y))
    step(answers)
    for s, old in zip(answers, held):                  # the new token came behind what there was
        assert all(torch.equal(a[:T + 1], b) for x, y in zip(values(s), old) for a, b in zip(x, y))
    # a branch goes back to within the page that it shares with where it comes from
    before, old = attend(answers, q), values(answers[0])
    (branch,) = pool.fork(answers[0])
    pool.cut(branch, T - 10)
    assert pool.users[pool.pages[branch][-1]] == 2
    step([branch])
    assert all(torch.equal(a, b) for x, y in zip(attend(answers, q), before) for a, b in zip(x, y))
    new = values(branch)
    assert all(len(a) == T - 9 and torch.equal(a[:T - 10], b[:T - 10]) for x, y in zip(new, old) for a, b in zip(x, y))
    got = attend([branch], q[:, :1])
    for (o, lse), (k, v), x in zip(got, new, q[:, 0]):
        k, v = (t.double().repeat_interleave(nq // nkv, 1) for t in (k, v))
        s = torch.einsum("hd,thd->ht", x.double(), k) / math.sqrt(hd)
        ref = torch.einsum("ht,thd->hd", s.softmax(-1), v)
        # the output's rounding, and 2^-15 of the values it is a mean of, whose parts are below 4 times as large
        tol = torch.finfo(dtype).eps / 2 * ref.abs() + 2.0 ** -15 * 4 * v.abs().amax() + 2.0 ** -25
        assert ((o[0].double() - ref).abs() <= tol).all()
        assert ((lse[0].double() - torch.logsumexp(s, -1)).abs() <= 2.0 ** -15).all()
