"""What the operators that answer from a context cache refuse, on the host: nothing is launched, so
the pointers are never followed and no GPU is needed."""

import importlib.util
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 0x10000000          # a 256-byte aligned address that is never read
STEP = 0x1000000        # far enough apart that the ranges of these small shapes do not meet


@pytest.fixture(scope="module")
def b():
    spec = importlib.util.spec_from_file_location("akvs_build", os.path.join(ROOT, "paper_2607_21604_b200", "build.py"))
    build = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(build)                  # by path: importing the package needs the library built
    build.build()
    import paper_2607_21604_b200.binding as binding
    return binding


def _at(i):
    return A + i * STEP


NORM = dict(dtype=1, q=_at(0), q_ld=512, k=_at(1), k_ld=256, q_gain=_at(2), k_gain=_at(3), pos=_at(4), n=3, nq=4, nkv=2,
            hd=128, eps=1e-6, base=1e4, q_out=_at(5), q_out_ld=512, k_out=_at(6), k_out_ld=256, stream=None)
SHARED = dict(dtype=1, q=_at(0), q_ld=512, R=3, ck=_at(1), cv=_at(2), c_ld=256, P=100, ok=_at(3), ov=_at(4), o_ld=256,
              o_seq=256 * 20, S=3, cap=20, lens=_at(5), off=None, nq=4, nkv=2, hd=128, out=_at(6), lse=_at(7),
              scratch=_at(8), scratch_bytes=1 << 23, stream=None)
MASS = dict(dtype=1, q=_at(0), q_ld=512, k=_at(1), k_ld=256, lse=_at(2), lo=_at(3), hi=_at(4), R=3, T=100, nq=4, nkv=2,
            hd=128, mass=_at(5), out=_at(6), stream=None)
EVICT = dict(dtype=1, mass=_at(0), k=_at(1), v=_at(2), layer_ld=256 * 100, tok_ld=256, L=2, T=100, nkv=2, hd=128, budget=40,
             sink=2, recent=5, idx=_at(3), k_out=_at(4), v_out=_at(5), mass_out=_at(6), stream=None)

INVALID, SHAPE, WORKSPACE, UNSUPPORTED, TOO_LARGE = -1, -2, -3, -4, -8


@pytest.mark.parametrize("change,code", [
    (dict(dtype=3), UNSUPPORTED), (dict(hd=96), UNSUPPORTED), (dict(n=-1), INVALID), (dict(nq=-1), INVALID),
    (dict(q=None), INVALID), (dict(k_gain=None), INVALID), (dict(pos=None), INVALID), (dict(k_out=None), INVALID),
    (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(base=0.0), INVALID), (dict(base=float("inf")), INVALID),
    (dict(q_ld=504), SHAPE), (dict(k_out_ld=128), SHAPE), (dict(q=_at(0) + 2), INVALID), (dict(k_ld=257), INVALID),
    (dict(k_out=_at(5) + 256), INVALID),                                   # outputs that meet
    (dict(q_out=_at(0), q_out_ld=768), INVALID),                           # in place with another stride
    (dict(q_out=_at(1)), INVALID),                                         # q's output over k
    (dict(k_out=_at(4)), INVALID), (dict(q_out=_at(3) - 1024), INVALID),   # over the positions, over a gain
])
def test_norm_rope_refuses(b, change, code):
    assert b.lib.akvs_op_qk_norm_rope(*{**NORM, **change}.values()) == code


def test_norm_rope_accepts_nothing_to_do(b):
    assert b.lib.akvs_op_qk_norm_rope(*{**NORM, "n": 0, "q": None}.values()) == 0
    assert b.lib.akvs_op_qk_norm_rope(*{**NORM, "nq": 0, "nkv": 0}.values()) == 0


@pytest.mark.parametrize("change,code", [
    (dict(dtype=9), UNSUPPORTED), (dict(hd=32), UNSUPPORTED), (dict(R=-1), INVALID), (dict(P=-1), INVALID),
    (dict(cap=-2), INVALID), (dict(S=-1), INVALID), (dict(nq=5), SHAPE), (dict(nkv=0), SHAPE), (dict(nq=258), SHAPE),
    (dict(R=2), SHAPE),                                                    # one row per sequence needs S rows
    (dict(q=None), INVALID), (dict(out=None), INVALID), (dict(lse=None), INVALID), (dict(ck=None), INVALID),
    (dict(ov=None), INVALID), (dict(lens=None), INVALID), (dict(q_ld=256), SHAPE), (dict(c_ld=128), SHAPE),
    (dict(o_ld=128), SHAPE), (dict(o_seq=-256), SHAPE), (dict(ck=_at(1) + 8), INVALID), (dict(c_ld=260), INVALID),
    (dict(o_seq=256 * 20 + 4), INVALID), (dict(scratch=None), WORKSPACE), (dict(scratch=_at(8) + 16), WORKSPACE),
    (dict(scratch_bytes=64), WORKSPACE), (dict(out=_at(0)), INVALID), (dict(lse=_at(5)), INVALID),
    (dict(scratch=_at(1)), INVALID), (dict(R=1 << 30, q_ld=512), TOO_LARGE),
])
def test_shared_attention_refuses(b, change, code):
    assert b.lib.akvs_op_attention_shared(*{**SHARED, **change}.values()) == code


def test_shared_attention_sizes(b):
    f = b.lib.akvs_op_attention_shared_scratch_bytes
    assert f(1, 3, 100, 3, 20, 4, 2, 128) >= 2 * 3 * 4 * (128 + 2) * 4
    for bad in ((3, 3, 100, 3, 20, 4, 2, 128), (1, -1, 100, 3, 20, 4, 2, 128), (1, 3, 100, 3, 20, 5, 2, 128), (1, 3, 100, 3, -1, 4, 2, 128),
                (1, 3, 100, 3, 20, 4, 2, 96)):
        assert f(*bad) == -1
    assert b.lib.akvs_op_attention_shared(*{**SHARED, "R": 0, "S": 0, "q": None}.values()) == 0


@pytest.mark.parametrize("change,code", [
    (dict(dtype=-1), UNSUPPORTED), (dict(hd=256), UNSUPPORTED), (dict(R=-1), INVALID), (dict(T=-1), INVALID),
    (dict(nq=3), SHAPE), (dict(k=None), INVALID), (dict(lse=None), INVALID), (dict(lo=None), INVALID), (dict(out=None), INVALID),
    (dict(k_ld=128), SHAPE), (dict(q_ld=128), SHAPE), (dict(k=_at(1) + 4), INVALID), (dict(q_ld=513), INVALID),
    (dict(out=_at(1)), INVALID), (dict(out=_at(5) + 4), INVALID), (dict(R=1 << 30), TOO_LARGE),
])
def test_mass_refuses(b, change, code):
    assert b.lib.akvs_op_attention_mass(*{**MASS, **change}.values()) == code


@pytest.mark.parametrize("change,code", [
    (dict(dtype=7), UNSUPPORTED), (dict(hd=32), UNSUPPORTED), (dict(budget=101), SHAPE), (dict(sink=36), SHAPE),
    (dict(sink=-1), INVALID), (dict(recent=-1), INVALID), (dict(L=-1), INVALID), (dict(nkv=0), INVALID),
    (dict(mass=None), INVALID), (dict(v=None), INVALID), (dict(idx=None), INVALID), (dict(mass_out=None), INVALID),
    (dict(tok_ld=128), SHAPE), (dict(layer_ld=256), SHAPE), (dict(k=_at(1) + 8), INVALID), (dict(tok_ld=260, layer_ld=26000), INVALID),
    (dict(k_out=_at(1)), INVALID), (dict(v_out=_at(4)), INVALID), (dict(idx=_at(0)), INVALID),
    (dict(L=40000, layer_ld=256 * 100), TOO_LARGE),
])
def test_evict_refuses(b, change, code):
    assert b.lib.akvs_op_evict(*{**EVICT, **change}.values()) == code


def test_evict_accepts_nothing_to_do(b):
    assert b.lib.akvs_op_evict(*{**EVICT, "budget": 0, "sink": 0, "recent": 0, "k": None}.values()) == 0
    assert b.lib.akvs_op_evict(*{**EVICT, "L": 0}.values()) == 0


def test_host_tensors_are_refused(b):
    import torch
    x = torch.zeros((2, 2, 64))
    g, i = torch.ones(64), torch.zeros(2, dtype=torch.int32)
    for call in (lambda: b.op_qk_norm_rope(x, x, g, g, i, 1e-6, 1e4),
                 lambda: b.op_attention_shared(x, x, x, x[None], x[None], i[:1]),
                 lambda: b.op_attention_mass(x, x, torch.zeros(2, 2), i, i),
                 lambda: b.op_evict(torch.zeros(1, 2, 2), x[None], x[None], 1)):
        with pytest.raises(b.AkvsError):
            call()
