"""The policy loss of rows of the types' largest and lowest values and of offsets beyond 1e9: finite rows have finite results.  Sizes for every
kernel: a row in a warp's and in a CTA's registers, in one CTA's ring, shared by 2, 4 and 8 CTAs.  Tolerances: those of the operator's own tests."""
import numpy as np
import pytest
import torch

from oracle import sequence_oracle as so
from tests import test_gpu_policy_loss as tpl
from tests import test_gpu_policy_offsets as tpo

pytestmark = pytest.mark.gpu

SIZES = tpo.SIZES + [(2, 90001)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("N,V", SIZES)
def test_rows_of_one_value(N, V, dtype):
    """Every class has the share 1 / V, whatever the value."""
    from paper_2002_03629_b200 import policy_loss as pl
    f = torch.finfo(dtype)
    values = [f.min, f.max, -2.0 ** 127, 2.0 ** 127, 1e10, -1e20, 3e9, -5e9, 32768.0, -32768.0, 32767.0, -33000.0]
    z = torch.tensor(values).to(dtype)[:, None].expand(len(values), V).contiguous()
    rows = len(values)
    a = torch.arange(rows) * (V - 1) // rows
    old, adv, w = torch.full((rows,), -float(np.log(V)) - 0.1), torch.randn(rows, generator=torch.Generator().manual_seed(1)), torch.ones(rows)
    loss, logp, dz = (t.cpu() for t in pl.policy_loss(z.cuda(), a.cuda(), old.cuda(), adv.cuda(), weights=w.cuda()))
    tpl.check(tpo.Shifted(z), V, a, old, adv, w, None, 0.0, loss, logp, dz)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("offset", [1e9, -3e9, 1e10, -1e15, 1e20, -1e30, 3e38, -3e38, 32768.0, -32768.0, 40000.0])
def test_ties_at_far_offsets(offset, dtype):
    from paper_2002_03629_b200 import policy_loss as pl
    for N, V in SIZES:
        z, a, old, adv, w = tpo.tied(N, V, dtype, offset, V)
        loss, logp, dz = (t.cpu() for t in pl.policy_loss(z.cuda(), a.cuda(), old.cuda(), adv.cuda(), weights=w.cuda()))
        rows = slice(0, 2)
        tpl.check(tpo.Shifted(z[rows]), V, a[rows], old[rows], adv[rows], w[rows], None, 0.0, loss[rows], logp[rows], dz[rows])
        assert torch.isfinite(dz).all() and torch.isfinite(loss).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("N,V", SIZES)
def test_masks_of_the_lowest_value_and_slices_of_different_size(N, V, dtype):
    """Rows whose parts lie at very different heights: one class counts, or those of one part do.  The action's class is the part's first."""
    from paper_2002_03629_b200 import policy_loss as pl
    f, g = torch.finfo(dtype), torch.Generator().manual_seed(V)
    half, parts = V // 2, [(0.0, f.min), (f.min, 0.0), (-100.0, f.min), (f.min, -1000.0), (-32768.0, -32640.0), (-32640.0, -32768.0), (-40000.0, 0.0), (1e9, 5.0),
                           (5.0, 1e9), (f.max, 0.0), (0.0, f.max), (1e30, -1e30), (-1e30, f.min), (f.min, -1e30), (32768.0, 32512.0), (32512.0, 32768.0)]
    n = len(parts)
    z = torch.randn(n, V, generator=g)
    far = torch.tensor([abs(p) < 1e4 for p in sum(map(list, parts), [])]).view(n, 2)
    for i, (x, y) in enumerate(parts):
        z[i, :half] = x + z[i, :half] * far[i, 0]
        z[i, half:] = y + z[i, half:] * far[i, 1]
    z = z.to(dtype)
    a = z.float().argmax(1)
    lp = torch.log_softmax(z.double(), 1).gather(1, a[:, None])[:, 0]
    old, adv, w = (lp - 0.1).float(), torch.randn(n, generator=g), torch.ones(n)
    loss, logp, dz = (t.cpu() for t in pl.policy_loss(z.cuda(), a.cuda(), old.cuda(), adv.cuda(), weights=w.cuda()))
    tpl.check(tpo.Shifted(z), V, a, old, adv, w, None, 0.0, loss, logp, dz)
    # an action that has next to no chance: its probability's logarithm to the type's precision, ratio and gradients 0 (the loss, with a negative
    # advantage, is the clip bound's)
    a = z.float().argmin(1)
    keep = [i for i in range(n) if float(z[i].double().max() - z[i].double().min()) < 3e38 and float(z[i].double().max() - z[i].double().min()) > 200]
    loss, logp, dz = (t.cpu() for t in pl.policy_loss(z[keep].cuda(), a[keep].cuda(), torch.full((len(keep),), -5.0).cuda(), adv[keep].cuda(), weights=w[keep].cuda()))
    for j, i in enumerate(keep):
        bound, want, _ = so.policy_loss(z[i].double().numpy(), int(a[i]), -5.0, float(adv[i]), 1.0)
        assert abs(float(logp[j]) - want) <= 100 * tpl.U + 8 * tpl.U * abs(want)
        assert abs(float(loss[j]) - bound) <= 4 * tpl.U * abs(bound) + 2.0 ** -126       # (below fp32's range: zero)
    assert (dz == 0).all()
