"""Linear attention and its gradients against the oracle in the 2-norm, for each sequence and head as a whole and for each 128 steps of it: the elementwise
tolerances of the operator's own tests go by sums of magnitudes, which over long ranges are many times the outputs.

Tolerance.  bf16: a rounding is uniform within half a step, 2^-8 of a value at most, so 2^-8 / sqrt 3 = 2.3e-3 in the mean square at most.  On the tensor cores
an output is rounded once itself, and each of its terms, a score or a value of the state times a row, once before: with terms of independent signs (the
inputs are normal) the terms' errors add up as the terms do, to the same share of the output.  Together sqrt 2 * 2.3e-3 = 3.2e-3; 4e-3 leaves a quarter for
sums that come out small.  fp32: factors in two pieces are off by 3 * 2^-22 = 7.2e-7 a product at most, two products in a row by sqrt 2 of that in the mean
square, 1.0e-6; sums cut towards zero by a step of 2^-23 each, at 8 terms a cut and 128 terms a sum 16 steps at most, half of one each in the mean: 1e-6 more."""
import numpy as np
import pytest
import torch

from oracle import sequence_oracle as so
from tests import test_gpu_linear_attention as tla

pytestmark = pytest.mark.gpu

BOUND = {torch.float32: 2e-6, torch.bfloat16: 4e-3}
REGIMES = {"none": [0.0, -1e-5], "weak": [-0.003, -0.03], "border": [-0.68, -0.7], "strong": [-1.5, -6.0]}


def near(got, want, bound, what):
    """(The mean square is that of many rows: under strong decay a row is little more than one score times one vector, and a score, whose error goes by its
    products' norm, sqrt D on average, comes out at 1/30 of that in one row of forty.  A last part of fewer than 32 rows is taken together with the one before.)"""
    g = got.double().cpu().numpy()
    n = len(want)
    starts = [at for at in range(0, n, 128) if at == 0 or n - at >= 32]
    for at, end in zip(starts, starts[1:] + [n]):
        part = slice(at, end)
        off, size = np.linalg.norm(g[part] - want[part]), np.linalg.norm(want[part])
        assert off <= bound * size, (what, at, off / size)
    assert np.linalg.norm(g - want) <= bound * np.linalg.norm(want), what


def check(x, o, S, grads, scale, seqs):
    bound = BOUND[x["q"].dtype]
    for i, (b, at, n) in enumerate(seqs):
        if n == 0:
            continue
        for h in range(x["q"].shape[2]):
            q, k, v, do = (x[a][b, at:at + n, h].double().numpy() for a in ("q", "k", "v", "do"))
            S0, dS = (None if x[a] is None else x[a][i, h].double().numpy() for a in ("state", "dstate"))
            ld = float(x["ld"][h])
            wo, wS = so.linear_attention(q, k, v, ld, scale, S0)
            near(o[b, at:at + n, h], wo, bound, f"o {i} {h}")
            near(S[i, h], wS, 2e-6, f"state {i} {h}")
            dq, dk, dv, dS0 = so.linear_attention_backward(q, k, v, ld, do, scale, S0, dS)
            for name, g, w in (("dq", grads[0], dq), ("dk", grads[1], dk), ("dv", grads[2], dv)):
                near(g[b, at:at + n, h], w, bound, f"{name} {i} {h}")
            near(grads[3][i, h], dS0, 2e-6, f"dstate {i} {h}")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("decays", REGIMES.values(), ids=REGIMES.keys())
@pytest.mark.parametrize("size", [(2, 250, 64, 64), (1, 2100, 64, 64), (1, 1500, 128, 128), (1, 700, 32, 96), (12, 131, 128, 64)], ids=str)
def test_sequences(size, decays, dtype):
    B, T, Dk, Dv = size
    for state in (False, True):
        x = tla.make(B, T, 2, Dk, Dv, dtype, seed=T + 1, state=state, decays=decays)
        check(x, *tla.forward(x, Dk ** -0.5), tla.backward(x, Dk ** -0.5), Dk ** -0.5, [(b, 0, T) for b in range(B)])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("decays", REGIMES.values(), ids=REGIMES.keys())
def test_packed_sequences(decays, dtype):
    lens = [1900, 129, 0, 700, 128, 33, 512]
    at = np.concatenate([[0], np.cumsum(lens)])
    x = tla.make(1, sum(lens), 2, 64, 128, dtype, seed=3, state=False, decays=decays)
    g = torch.Generator().manual_seed(2)
    x["state"], x["dstate"] = (torch.randn(len(lens), 2, 64, 128, generator=g) for _ in range(2))
    cu = torch.tensor(at, dtype=torch.int32).cuda()
    check(x, *tla.forward(x, 0.125, cu_seqlens=cu), tla.backward(x, 0.125, cu_seqlens=cu), 0.125, [(0, int(a), n) for a, n in zip(at, lens)])
