"""Pins of the oracle of the sequence operators: closed forms, central differences, automatic differentiation."""
import numpy as np
import pytest
import torch

from oracle import sequence_oracle as so


def closed_form(q, k, v, ld, scale, S0):
    n = len(q)
    i = np.arange(n)
    D = np.where(i[:, None] >= i[None], np.exp(ld * (i[:, None] - i[None])), 0.0)
    o = ((q @ k.T) * D) @ v + np.exp(ld * (i + 1))[:, None] * (q @ S0)
    S = (k * np.exp(ld * (n - 1 - i))[:, None]).T @ v + np.exp(ld * n) * S0
    return scale * o, S


def case(n=7, Dk=3, Dv=4, seed=0):
    r = np.random.default_rng(seed)
    return r.normal(size=(n, Dk)), r.normal(size=(n, Dk)), r.normal(size=(n, Dv)), r.normal(size=(Dk, Dv)), r.normal(size=(n, Dv)), r.normal(size=(Dk, Dv))


@pytest.mark.parametrize("ld", [0.0, -0.01, -0.7, -5.0])
def test_recurrence_is_the_masked_product(ld):
    q, k, v, S0, _, _ = case()
    for a, b in zip(so.linear_attention(q, k, v, ld, 0.3, S0), closed_form(q, k, v, ld, 0.3, S0)):
        np.testing.assert_allclose(a, b, rtol=1e-12, atol=1e-13)


def test_one_step_and_none():
    q, k, v, S0, _, _ = case(n=1)
    o, S = so.linear_attention(q, k, v, -0.5, 1.0, S0)
    np.testing.assert_allclose(S, np.exp(-0.5) * S0 + np.outer(k[0], v[0]))
    np.testing.assert_allclose(o[0], S.T @ q[0])
    o, S = so.linear_attention(q[:0], k[:0], v[:0], -0.5, 1.0, S0)
    assert o.shape == (0, 4) and np.array_equal(S, S0)


def test_gradients_against_differences():
    q, k, v, S0, do, dS = case(n=5)
    ld, scale, h = -0.3, 0.7, 1e-6

    def loss(q, k, v, S0):
        o, S = so.linear_attention(q, k, v, ld, scale, S0)
        return (o * do).sum() + (S * dS).sum()
    got = so.linear_attention_backward(q, k, v, ld, do, scale, S0, dS)
    args = [q, k, v, S0]
    for a, g in enumerate(got):
        for at in np.ndindex(args[a].shape):
            up, down = [x.copy() for x in args], [x.copy() for x in args]
            up[a][at] += h
            down[a][at] -= h
            assert abs((loss(*up) - loss(*down)) / (2 * h) - g[at]) < 1e-7 * max(1, abs(g[at]))


@pytest.mark.parametrize("adv,old,ref", [(1.0, -1.0, None), (-1.0, -1.5, -1.2), (2.0, -4.0, -1.0), (-0.5, 3.0, -2.0)])
def test_policy_gradient_against_differences(adv, old, ref):
    z = np.random.default_rng(3).normal(size=6)
    loss, logp, dz = so.policy_loss(z, 2, old, adv, 0.4, ref, kl=0.1)
    h = 1e-6
    for c in range(6):
        up, down = z.copy(), z.copy()
        up[c] += h
        down[c] -= h
        d = (so.policy_loss(up, 2, old, adv, 0.4, ref, kl=0.1)[0] - so.policy_loss(down, 2, old, adv, 0.4, ref, kl=0.1)[0]) / (2 * h)
        assert abs(d - dz[c]) < 1e-7 * max(1, abs(d))
    assert abs(logp - (z[2] - np.log(np.exp(z).sum()))) < 1e-12


def test_policy_loss_closed_forms():
    z = np.log(np.array([0.5, 0.25, 0.25]))
    # ratio 2, advantage 1: clipped at 1.2, no gradient; advantage -1: not clipped
    loss, logp, dz = so.policy_loss(z, 0, np.log(0.25), 1.0, 1.0)
    assert abs(loss + 1.2) < 1e-12 and np.all(dz == 0)
    loss, logp, dz = so.policy_loss(z, 0, np.log(0.25), -1.0, 1.0)
    assert abs(loss - 2) < 1e-12
    np.testing.assert_allclose(dz, 2 * np.array([0.5, -0.25, -0.25]))
    assert so.policy_loss(z, 7, 0.0, 1.0, 0.0)[0] == 0


def test_adamw_is_torchs():
    r = np.random.default_rng(5)
    p0 = torch.tensor(r.normal(size=37), dtype=torch.float64, requires_grad=True)
    opt = torch.optim.AdamW([p0], lr=1e-2, betas=(0.8, 0.95), eps=1e-6, weight_decay=0.1)
    p, m, v = p0.detach().numpy().copy(), np.zeros(37), np.zeros(37)
    for t in range(1, 6):
        g = r.normal(size=37)
        p0.grad = torch.from_numpy(g.copy())
        opt.step()
        p, m, v = so.adamw(p, g, m, v, t, 1e-2, (0.8, 0.95), 1e-6, 0.1)
        np.testing.assert_allclose(p, p0.detach().numpy(), rtol=1e-12, atol=1e-14)


def test_float8_codes():
    t = torch.arange(256, dtype=torch.int16).to(torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(so.float8_value(np.arange(256)), t)
    # a value that is a code keeps it whatever the bits; between two codes the mean over all bits is the value
    x = np.array([so.float8_value(c) for c in (0, 1, 7, 8, 100, 119, 0x83, 0x90)], np.float32)
    x = np.append(x, np.float32(200.0))
    for r in (0, 1, 40000, 65535):
        codes, scale = so.float8_cut(x, [r] * len(x))
        assert scale == 1.0
        np.testing.assert_array_equal(so.float8_value(codes[:-1]), x[:-1])
    for a in (0.0123, 0.0021, 3.3, 130.0):
        y = np.array([a, 200.0], np.float32)
        got = [float(so.float8_value(so.float8_cut(y, [r, 0])[0][0])) for r in range(0, 65536, 64)]
        assert len(set(got)) <= 2 and abs(np.mean(got) - y[0]) < 2e-3 * (max(got) - min(got)) + 1e-9


def test_random_bits_are_spread():
    b = so.random_bits(np.arange(4096), 17)
    assert len(set(b.tolist())) == 4096                           # the mixing can be undone: no two places alike
    for half in (b & 0xFFFF, b >> 16):
        u = half.astype(np.float64) / 65536
        # mean of 4096 uniform numbers: standard error 0.0045; six of them
        assert abs(u.mean() - 0.5) < 0.027
        assert abs(np.corrcoef(u[:-1], u[1:])[0, 1]) < 6 / 64
