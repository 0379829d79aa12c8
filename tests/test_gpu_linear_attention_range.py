"""Linear attention of very large and very small queries, and gradients of very large and very small losses: outputs and gradients are linear in them, so they
keep the accuracy that they have at 1 as long as no product of the formulas leaves fp32.  Tolerances: those of the 2-norm's tests."""
import pytest
import torch

from tests import test_gpu_linear_attention as tla
from tests import test_gpu_linear_attention_norms as norms

pytestmark = pytest.mark.gpu

REGIMES = norms.REGIMES | {"between": [-0.2, -0.5]}


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("decays", REGIMES.values(), ids=REGIMES.keys())
@pytest.mark.parametrize("power", [-90, -64, 64, 100])
def test_powers_of_two(power, decays, dtype):
    for B, T, Dk, Dv in ((1, 400, 64, 64), (2, 130, 128, 32)):
        x = tla.make(B, T, 2, Dk, Dv, dtype, seed=T, decays=decays)
        x["q"], x["do"], x["dstate"] = (x[a] * 2.0 ** power for a in ("q", "do", "dstate"))
        q = x | {"do": x["do"] * 0, "dstate": x["dstate"] * 0}               # outputs and states: linear in q
        o, S = tla.forward(q, 0.125)
        zero = tla.backward(q, 0.125)
        assert all((t == 0).all() for t in zero)
        g = x | {"q": x["q"] * 2.0 ** -power}                                # gradients: linear in do and dstate
        grads = tla.backward(g, 0.125)
        norms.check(g, *tla.forward(g, 0.125), grads, 0.125, [(b, 0, T) for b in range(B)])
        for h in range(2):
            for b in range(B):
                a = [x[n][b, :, h].double().numpy() for n in "qkv"]
                wo, wS = norms.so.linear_attention(*a, float(x["ld"][h]), 0.125, x["state"][b, h].double().numpy())
                norms.near(o[b, :, h], wo, norms.BOUND[dtype], f"o {b} {h}")
                norms.near(S[b, h], wS, 2e-6, f"state {b} {h}")
