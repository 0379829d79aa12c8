"""AdamW on gradients that are not finite, and on finite ones whose square is not: what the header says of each, and nothing beside it."""
import numpy as np
import pytest
import torch

from oracle import sequence_oracle as so

pytestmark = pytest.mark.gpu

OPT = dict(betas=(0.9, 0.99), eps=1e-6, weight_decay=0.1)
BAD = [float("nan"), float("inf"), -float("inf"), 2e19, -3e38]


def program(bits, bad):
    from paper_2002_03629_b200 import adamw as aw
    g = torch.Generator().manual_seed(1)
    params = [torch.randn(900, generator=g).cuda()]
    grads = [torch.randn(900, generator=g).cuda()]
    state = aw.adamw_state(params, bits)
    aw.adamw_step(params, grads, state, 1, 0.01, **OPT)
    if bad is not None:
        grads[0][300] = bad
    return aw, params, grads, state


@pytest.mark.parametrize("bad", BAD, ids=str)
def test_32_bits(bad):
    """The formulas' own infinities and NaN, bit for bit where they are numbers, for that value alone."""
    aw, params, grads, state = program(32, bad)
    p, m, v = (t.cpu().numpy().copy() for t in (params[0], state.m[:900], state.v[:900]))
    aw.adamw_step(params, grads, state, 2, 0.01, **OPT)
    with np.errstate(all="ignore"):
        want = so.adamw_f32(p, grads[0].cpu().numpy(), m, v, 2, 0.01, **OPT)[:3]
    for got, w in zip((params[0], state.m[:900], state.v[:900]), want):
        np.testing.assert_array_equal(got.cpu().numpy(), w)
        assert np.isfinite(np.delete(w, 300)).all()
    assert not np.isfinite(want[2][300])


@pytest.mark.parametrize("bad", BAD, ids=str)
def test_8_bits(bad):
    """The state of the value's block of 256 is NaN; the other blocks, and this step's other parameters, are those of the step without it."""
    aw, params, grads, state = program(8, bad)
    _, clean, other, right = program(8, None)
    aw.adamw_step(params, grads, state, 2, 0.01, **OPT)
    aw.adamw_step(clean, other, right, 2, 0.01, **OPT)
    for codes, want in ((state.m, right.m), (state.v, right.v)):
        codes, want = codes.float().cpu(), want.float().cpu()
        assert torch.isnan(codes[256:512]).all()
        for part in (slice(0, 256), slice(512, 900)):
            assert torch.equal(codes[part], want[part])
    keep = torch.arange(900) != 300
    assert torch.equal(params[0].cpu()[keep], clean[0].cpu()[keep])
