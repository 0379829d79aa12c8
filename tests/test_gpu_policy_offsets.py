"""The policy loss of rows whose logits share a large offset: the gradient is that of the same row without it.  Sizes for every kernel: a row in a
warp's and in a CTA's registers, in one CTA's ring, shared by 2 and by 4 CTAs.  Tolerances: those of the operator's own tests; in particular a gradient of
bf16 is rounded once."""
import pytest
import torch

from tests import test_gpu_policy_loss as tpl

pytestmark = pytest.mark.gpu


class Shifted:
    """Logits as differences from their row's largest, in 64 bits: all that the operator knows of them, and at offsets like 1e20 the oracle's logarithm of a
    sum would be lost in 64 bits as well.  (The tolerances go by the logits' own type.)"""

    def __init__(self, z):
        self.dtype, z = z.dtype, z.double()
        self.z = z - z.max(1, keepdim=True).values

    def __getitem__(self, i):
        return self.z[i]


SIZES = [(5, 100), (4, 3001), (76, 11003), (3, 20001), (2, 50001)]


def tied(N, V, dtype, offset, seed):
    """Logits of `offset` and of the three values of the type next below it: shares of many classes each, or next to nothing."""
    g = torch.Generator().manual_seed(seed)
    steps = [torch.tensor(offset).to(dtype)]
    for _ in range(3):
        steps.append(torch.nextafter(steps[-1], torch.tensor(-float("inf")).to(dtype)))
    z = torch.stack(steps)[torch.randint(0, 4, (N, V), generator=g)]
    z[:, 0] = steps[0]
    a = torch.where(torch.arange(N) % 2 == 0, 0, z.float().argmax(1))
    lp = torch.log_softmax(z.double(), 1).gather(1, a[:, None])[:, 0]
    old = (lp - torch.tensor([0.1, -0.1], dtype=torch.float64)[torch.arange(N) % 2]).float()
    adv = torch.randn(N, generator=g)
    return z, a, old, adv, torch.rand(N, generator=g) + 0.1


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("offset", [-1e3, 1e4, 2e5, -3e5, 1e6, -1e7, 1e8])
def test_gradient_does_not_depend_on_a_common_offset(offset, dtype):
    from paper_2002_03629_b200 import policy_loss as pl
    for N, V in SIZES:
        z, a, old, adv, w = tied(N, V, dtype, offset, V)
        loss, logp, dz = (t.cpu() for t in pl.policy_loss(z.cuda(), a.cuda(), old.cuda(), adv.cuda(), weights=w.cuda()))
        rows = slice(0, 3)                                   # (the oracle's rows; all of them for their signs and sums)
        tpl.check(Shifted(z[rows]), V, a[rows], old[rows], adv[rows], w[rows], None, 0.0, loss[rows], logp[rows], dz[rows])
        assert torch.isfinite(dz).all() and torch.isfinite(loss).all()
