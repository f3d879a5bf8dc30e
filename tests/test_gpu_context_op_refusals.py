"""What the Python calls of the operators that answer from a context cache refuse and accept of device
tensors.  A refused call launches nothing."""
import pytest
import torch

pytestmark = pytest.mark.gpu
SHAPE = -2


@pytest.fixture(scope="module")
def akvs():
    import paper_2607_21604_b200 as a
    return a


def test_tensors_of_another_rank_are_refused(akvs):
    z = torch.zeros((2, 2, 64), device="cuda")
    gain, i, f = torch.ones(64, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros((2, 2), device="cuda")
    calls = [lambda x: akvs.op_qk_norm_rope(x, z, gain, gain, i, 1e-6, 1e4), lambda x: akvs.op_qk_norm_rope(z, x, gain, gain, i, 1e-6, 1e4),
             lambda x: akvs.op_attention_shared(x, z, z, z[None], z[None], i[:1]),
             lambda x: akvs.op_attention_shared(z, x, x, z[None], z[None], i[:1]),
             lambda x: akvs.op_attention_shared(z, z, z, x, x, i[:1]),
             lambda x: akvs.op_attention_mass(x, z, f, i, i), lambda x: akvs.op_attention_mass(z, x, f, i, i),
             lambda x: akvs.op_evict(f[None], x, x, 1)]
    for call in calls:
        for x in (z[0], z[0, 0], z[None, None]):
            with pytest.raises(akvs.AkvsError) as e:
                call(x)
            assert e.value.code == SHAPE


def test_strides_of_single_elements_mean_nothing(akvs):
    """One kv head, one sequence, one layer: K and V lie alike although the strides of those dimensions
    differ."""
    g = torch.Generator(device="cuda").manual_seed(1)
    P, cap, hd = 50, 9, 64
    kv, own = (torch.randn((n, 2 * hd), generator=g, device="cuda") for n in (P, cap))
    q = torch.randn((1, 3, hd), generator=g, device="cuda")
    ctx = kv.as_strided((P, 1, hd), (2 * hd, 2 * hd, 1)), kv.as_strided((P, 1, hd), (2 * hd, hd, 1), hd)
    slot = own.as_strided((1, cap, 1, hd), (7, 2 * hd, 5, 1)), own.as_strided((1, cap, 1, hd), (1, 2 * hd, hd, 1), hd)
    length = torch.full((1,), cap, dtype=torch.int32, device="cuda")
    got = akvs.op_attention_shared(q, *ctx, *slot, length)
    want = akvs.op_attention_shared(q, *(x.contiguous() for x in ctx + slot), length)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    mass = torch.rand((1, 1, P), generator=g, device="cuda")
    layer = kv.as_strided((1, P, 1, hd), (3, 2 * hd, 1, 1)), kv.as_strided((1, P, 1, hd), (P * 2 * hd, 2 * hd, hd, 1), hd)
    for x, y in zip(akvs.op_evict(mass, *layer, 20), akvs.op_evict(mass, *(x.contiguous() for x in layer), 20)):
        assert torch.equal(x, y)
    # strides that do mean something still have to agree
    two = torch.randn((2, P, 1, hd), generator=g, device="cuda")
    far = torch.randn((2, 2 * P, 1, hd), generator=g, device="cuda")
    for call in (lambda: akvs.op_attention_shared(q, ctx[0], ctx[1].contiguous(), *slot, length),
                 lambda: akvs.op_attention_shared(q, *ctx, slot[0], slot[1].contiguous(), length),
                 lambda: akvs.op_attention_shared(q.expand(2, 3, hd).contiguous(), *ctx, two, far[:, :P], length.expand(2).contiguous()),
                 lambda: akvs.op_evict(mass.expand(2, 1, P).contiguous(), two, far[:, :P], 20)):
        with pytest.raises(akvs.AkvsError) as e:
            call()
        assert e.value.code == SHAPE
