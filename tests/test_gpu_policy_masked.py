"""Rows of the policy loss of which only a few classes are possible, the others -infinity: whole slices of the CTAs that share a row hold nothing.  What
is possible lies far below zero, as log-probabilities divided by a low temperature do.  Tolerances: those of the operator's own tests, over the
possible classes; the others have the gradient 0."""
import pytest
import torch

from tests import test_gpu_policy_loss as tpl

pytestmark = pytest.mark.gpu

# (rows, classes) of fp32, twice as many of bf16: one CTA, 2, 4, 8 CTAs a row (few rows), 2 CTAs a row (rows that leave no room in one)
SIZES = [(3, 6000), (3, 12000), (3, 24001), (3, 40003), (76, 30001)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("top", [0.0, -100.0, -1000.0, 1000.0])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_slices_without_a_class(size, top, dtype):
    from paper_2002_03629_b200 import policy_loss as pl
    N, V = size[0], size[1] * (1 if dtype == torch.float32 else 2)
    for first in (0, V // 2 + 5, V - 200):
        base, a, old, adv, w, ref = tpl.rows(N, 200, torch.float32, seed=first)
        base = (base + top).to(dtype)
        lp = torch.log_softmax(base.double(), 1).gather(1, a[:, None])[:, 0]
        old, w = (lp - torch.tensor([0.1, -0.1, 0.5], dtype=torch.float64)[torch.arange(N) % 3]).float(), w + 0.1
        z = torch.full((N, V), -float("inf"), dtype=dtype)
        z[:, first:first + 200] = base
        loss, logp, dz = (t.cpu() for t in pl.policy_loss(z.cuda(), (a + first).cuda(), old.cuda(), adv.cuda(), weights=w.cuda()))
        rows = slice(0, 3)
        tpl.check(base[rows], 200, a[rows], old[rows], adv[rows], w[rows], None, 0.0, loss[rows], logp[rows], dz[rows, first:first + 200])
        assert torch.isfinite(loss).all() and torch.isfinite(dz).all()
        dz[:, first:first + 200] = 0
        assert (dz == 0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_nan_in_a_slice_without_a_class(size, dtype):
    """A NaN between masked classes still makes its row NaN, and no other; so does a row without any class."""
    from paper_2002_03629_b200 import policy_loss as pl
    N, V = size[0], size[1] * (1 if dtype == torch.float32 else 2)
    z = torch.full((N, V), -float("inf"), dtype=dtype)
    z[:, :50] = -300.0
    z[0, V - 3] = float("nan")
    z[1, :50] = -float("inf")
    x = torch.ones(N, device="cuda")
    loss, logp, dz = (t.cpu() for t in pl.policy_loss(z.cuda(), torch.zeros(N, dtype=torch.long, device="cuda"), -4 * x, x, weights=x))
    for t in (loss, logp, dz):
        assert torch.isnan(t[:2]).all() and torch.isfinite(t[2:]).all()
