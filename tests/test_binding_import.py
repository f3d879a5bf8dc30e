"""The binding loads and works with a torch that lacks the private short cuts it prefers."""
import importlib.util
import os

import pytest
import torch

from test_context_op_refusals import b  # noqa: F401  (builds the library)

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_binding_without_private_names(b, monkeypatch):  # noqa: F811
    for name in ("_cuda_getDevice", "_cuda_getCurrentRawStream"):
        monkeypatch.delattr(torch._C, name, raising=False)
    spec = importlib.util.spec_from_file_location("binding_of_another_torch", os.path.join(ROOT, "paper_2607_21604_b200", "binding.py"))
    other = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(other)

    class Stream:
        cuda_stream = 77

    monkeypatch.setattr(torch.cuda, "current_stream", lambda dev: Stream())
    assert other._device is torch.cuda.current_device and other._raw_stream(0) == 77
    x = torch.zeros((2, 2, 64))
    with pytest.raises(other.AkvsError):
        other.op_attention_mass(x, x, torch.zeros(2, 2), torch.zeros(2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32))
