"""Packed sequences of odd widths and odd numbers of heads that are cut into segments: what the device keeps of their order lies behind an odd number of
state values.  Tolerances: those of the operator's own tests."""
import numpy as np
import pytest
import torch

from tests import test_gpu_linear_attention as tla

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("lens,H,Dk,Dv", [([4096], 1, 33, 33), ([2048], 3, 47, 33), ([2600, 0, 1, 1399], 1, 7, 9), ([3000, 700], 1, 65, 127)], ids=str)
def test_cut(lens, H, Dk, Dv, dtype):
    x = tla.make(1, sum(lens), H, Dk, Dv, dtype, seed=Dk, state=False, decays=[-0.002, -0.4, -0.03][:H])
    g = torch.Generator().manual_seed(1)
    x["state"], x["dstate"] = (torch.randn(len(lens), H, Dk, Dv, generator=g) for _ in range(2))
    at = np.concatenate([[0], np.cumsum(lens)])
    cu = torch.tensor(at, dtype=torch.int32).cuda()
    seqs = [(0, int(a), n) for a, n in zip(at, lens)]
    o, S = tla.forward(x, 0.2, cu_seqlens=cu)
    tla.check_forward(x, o, S, 0.2, seqs)
    tla.check_backward(x, tla.backward(x, 0.2, cu_seqlens=cu), 0.2, seqs)
