"""A stream of another device than the tensors': the call would run there, on memory of this one.  Refused before anything else is done (no GPU needed)."""
from types import SimpleNamespace

import pytest

import paper_2002_03629_b200 as pkg
from paper_2002_03629_b200 import adamw, binding, linear_attention, policy_loss


def test_a_stream_of_another_device_is_refused(monkeypatch):
    monkeypatch.setattr(binding.torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    assert not binding._elsewhere(0, None) and binding._elsewhere(1, None)
    assert binding._elsewhere(0, SimpleNamespace(device_index=0, cuda_stream=0)) and binding._elsewhere(1, SimpleNamespace(device_index=1, cuda_stream=0))
    for index in (0, 1):
        with pytest.raises(pkg.JsError):
            binding._elsewhere(index, SimpleNamespace(device_index=1 - index, cuda_stream=0))
    for module in (adamw, linear_attention, policy_loss):
        assert module._elsewhere is binding._elsewhere             # (all their calls ask this)
