"""Answers that go on from the cache a prefill left: each token's hidden state against the oracle's prefill
of the same tokens, in all three modes of the prefill."""
import numpy as np
import pytest
import torch

import testgen
from gpu_helpers import Case, t2n
from oracle import akvs_oracle as orc

pytestmark = pytest.mark.gpu


def workload(dtype):
    hd, d, ff = (64, 128, 200) if dtype == "f32" else (128, 256, 768)
    return testgen.Workload("decode-" + dtype, testgen.ModelCfg("decode-" + dtype, 3, d, 4, 2, hd, ff, 512, dtype), 4, 30, 70, 9, (2500,))


def rms(h, gain, eps, dt):
    return (h * torch.rsqrt(h.square().mean(-1, keepdim=True) + eps) * gain).to(dt)


class Answers:
    """S answers over one context: a step takes one token of each and gives their final hidden states."""

    def __init__(self, akvs, model, k, v, S, cap):
        self.akvs, self.model, self.k, self.v = akvs, model, k, v
        c = model.cfg
        self.own_k, self.own_v = (torch.full((c.n_layers, S, cap, c.n_kv_heads, c.head_dim), float("nan"), dtype=k.dtype, device="cuda")
                                  for _ in range(2))
        self.own_len = torch.zeros(S, dtype=torch.int32, device="cuda")

    def step(self, ids):
        a, m, c, dt = self.akvs, self.model, self.model.cfg, self.k.dtype
        S, seq, at = len(ids), torch.arange(len(ids), device="cuda"), self.own_len.long()
        pos = self.own_len + self.k.shape[1]
        self.own_len = self.own_len + 1
        h = m.tok_emb[torch.as_tensor(ids, device="cuda").long()].float()
        for l, w in enumerate(m.layers):
            x = rms(h, w["attn_norm"], c.rms_eps, dt)
            q = a.op_rope(a.op_linear(x, w["wq"]).view(S, c.n_q_heads, c.head_dim), pos, c.rope_base)
            kn = a.op_rope(a.op_linear(x, w["wk"]).view(S, c.n_kv_heads, c.head_dim), pos, c.rope_base)
            self.own_k[l][seq, at], self.own_v[l][seq, at] = kn, a.op_linear(x, w["wv"]).view_as(kn)
            o, _ = a.op_attention_shared(q, self.k[l], self.v[l], self.own_k[l], self.own_v[l], self.own_len)
            a.op_linear_residual(o.view(S, -1), w["wo"], h)
            x = rms(h, w["mlp_norm"], c.rms_eps, dt)
            y = torch.nn.functional.silu(a.op_linear(x, w["w_gate"]).float()) * a.op_linear(x, w["w_up"]).float()
            a.op_linear_residual(y.to(dt), w["w_down"], h)
        return rms(h, m.final_norm, c.rms_eps, torch.float32)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("S", [3, 12])                        # rows of one tile, and of several
def test_answers_go_on_from_the_prefills_cache(dtype, S):
    import paper_2607_21604_b200 as akvs
    case = Case(workload(dtype))
    units = case.oracle_units()
    case.load_oracle_cache(units)
    steps, bp = 3, 2500
    ids = np.random.default_rng(7).integers(0, case.cfg.vocab, (S, steps)).astype(np.int32)

    def oracle(mode, qry):
        if mode == akvs.MODE_FULL:
            return orc.full_recompute(case.omodel, case.ctx, qry)[0]
        if mode == akvs.MODE_NAIVE:
            return orc.naive_reuse(case.omodel, units, case.order, qry)[0]
        return orc.corrected_reuse(case.omodel, units, case.order, case.ctx, qry, bp, 2)["hidden"]

    for mode in (akvs.MODE_FULL, akvs.MODE_NAIVE, akvs.MODE_CORRECTED):
        probes = ctx = None
        ws = case.workspace(2)
        if mode == akvs.MODE_CORRECTED:
            probes, ctx, ws = case.gpu_select(bp, 2)
            case.set_probes(probes, orc.corrected_reuse(case.omodel, units, case.order, case.ctx, case.qry, bp, 2)["probes"])
        hid, k, v = akvs.alloc_outputs(case.gmodel, case.N, case.nq)
        akvs.prefill_corrected(case.gmodel, case.store, case.req, probes, mode, hid, k, v, ctx, ws)
        assert akvs.check(ws) == 0
        answers = Answers(akvs, case.gmodel, k, v, S, steps + 2)
        got = torch.stack([answers.step(ids[:, t]) for t in range(steps)], 1)
        akvs.free(ctx)
        for s in range(S):
            want = oracle(mode, np.concatenate([case.qry, ids[s]]))[-steps:]
            for t in range(steps):
                assert orc.rel_l2(t2n(got[s, t]), want[t]) < case.tol, (mode, s, t)
