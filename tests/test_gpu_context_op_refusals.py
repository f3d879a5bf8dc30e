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
