"""The training operators on what the library's own paths leave behind: the loss over the logits of a sampled categorical model, and AdamW steps with the
recurrent network's parameter gradients.  Every operator is held against its oracle on the inputs that it really had, with its own tests' tolerances."""
import numpy as np
import pytest
import torch

import synth_inputs as si
from oracle import sequence_oracle as so
from tests import test_gpu_policy_loss as tpl
from tests import test_gpu_rnn as trnn

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def test_the_loss_of_sampled_symbols():
    """Samples of a 256-way model by Jacobi iterations, the model's logits for them, and the loss of every sampled symbol with its gradient."""
    import paper_2002_03629_b200 as p
    from paper_2002_03629_b200 import policy_loss as pl
    cfg = si.scaled(si.CONFIGS["made_cat"], D=24, H=(128, 96), batch=9)
    model = p.Model.from_config(cfg, *si.made_weights(cfg), si.made_lut(cfg))
    x = torch.empty((cfg.batch, cfg.D), dtype=torch.uint8, device="cuda")
    assert p.jacobi_sample(model, torch.from_numpy(si.draw_noise(cfg)).cuda(), cfg.noise_kind, None, p.JS_JACOBI, 0, 0, x) == 0
    logits = torch.empty((cfg.batch, cfg.D, cfg.C), dtype=torch.float32, device="cuda")
    assert p.js_forward_logits(model, x, logits) == 0
    model.close()
    z, a = logits.view(-1, cfg.C), x.view(-1).long()
    N, g = z.shape[0], torch.Generator().manual_seed(1)
    lp = torch.log_softmax(z.double(), 1).gather(1, a[:, None])[:, 0].cpu()
    old = (lp - torch.tensor([0.1, -0.1, 0.5, -0.5], dtype=torch.float64)[torch.arange(N) % 4]).float()
    adv, w = torch.randn(N, generator=g), torch.rand(N, generator=g) * (torch.rand(N, generator=g) < 0.9)
    ref = (lp + 0.3 * torch.randn(N, generator=g).double()).float()
    loss, logp, dz = pl.policy_loss(z, a, old.cuda(), adv.cuda(), weights=w.cuda(), ref_logp=ref.cuda(), kl_coef=0.1)
    tpl.check(z.cpu(), cfg.C, a.cpu(), old, adv, w, ref, 0.1, loss.cpu(), logp.cpu(), dz.cpu())


@pytest.mark.parametrize("name", ["rnn_small", "rnn_100"])
def test_steps_of_the_recurrent_network(name):
    """Forward pass, state gradients by Jacobi iterations, parameter gradients (one of each sequence, summed over the batch here) and the step, three times
    over: the parameters follow the step's formula, and the next forward pass is that of the new ones."""
    import paper_2002_03629_b200.rnn as rnn
    from paper_2002_03629_b200 import adamw as aw
    cfg, params, x, r = trnn.case(name)
    dW, (dx, dr) = trnn.dev(*params), trnn.dev(x, r)
    trained, opt = dW[:3], dict(betas=(0.9, 0.99), eps=1e-6, weight_decay=0.1)
    state = aw.adamw_state(trained)
    for number in (1, 2, 3):
        h, d, l, loss = rnn.rnn_forward(*dW, dx, dr)
        want = trnn.oracle_all([t.cpu().numpy() for t in dW], x, r)
        trnn.close(h, want["h"], "h")
        trnn.close(loss, want["loss"], "loss")
        s = rnn.rnn_bptt_jacobi(dW[0], l, d, cfg.T)
        grads = [t.sum(0) for t in rnn.rnn_param_grads(s, d, h, dx)]
        assert [t.numel() for t in grads] == [t.numel() for t in trained]
        before = [t.cpu().numpy().copy().reshape(-1) for t in trained]
        m, v = (t.cpu().numpy().copy() for t in state[:2])
        aw.adamw_step(trained, grads, state, number, 0.01, **opt)
        at = 0
        for old, new, grad in zip(before, trained, grads):
            n = len(old)
            p64, *_ = so.adamw(old, grad.cpu().numpy().reshape(-1), m[at:at + n], v[at:at + n], number, 0.01, **opt)
            moved = np.abs(p64 - old)
            # (p within 12 u of the update and 3 u of itself; a moment whose terms cancel is off by u of the larger one)
            assert (np.abs(new.cpu().numpy().reshape(-1) - p64) <= 12 * U * (moved + 0.1) + 3 * U * (np.abs(p64) + moved)).all()
            assert (moved > 0).any()
            at += (n + 255) // 256 * 256
