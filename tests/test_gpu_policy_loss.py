"""The clipped policy loss and its gradient against the oracle in 64 bits.

Tolerance, with u = 2^-24.  logp: z_a - m and log(sum) are rounded to u of their size, the sum of V exponentials of 2 ulp each, added in parts
of at most 64 in a row, is off by (3 + 64 + 16) u relative at most (bf16 logits: 2^x by the special function, 2^-22 more, of arguments (z - m) log2 e
rounded to u |z - m| each, whose weights are e^-|z - m|: below 2 u).  So |d logp| <= 96 u + 4 u (|z_a - m| + |log sum| + |logp|) =: e.  Everything after
it is a factor e^{logp - ..}: the ratio is off by (e + 4 u + u |logp - old|) relative, loss and g follow with |A| r and kl e^d; near a clip bound either
side is right, so the cases keep away from it.  p_c = exp(z_c - lse): e + 4 u (1 + |z_c - m|) relative.  dlogits are rounded once more, by eps / 2."""
import numpy as np
import pytest
import torch

from oracle import sequence_oracle as so

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def rows(N, V, dtype, seed=0, std=2.0, pad=0):
    g = torch.Generator().manual_seed(seed)
    base = (torch.randn(N, V + pad, generator=g) * std).to(dtype)
    z = base[:, :V]
    a = torch.randint(0, V, (N,), generator=g)
    lp = torch.log_softmax(z.double(), 1).gather(1, a[:, None])[:, 0]
    # ratios away from the clip bounds 0.8 and 1.2: exp(+-0.1), exp(+-0.5)
    old = (lp - torch.tensor([0.1, -0.1, 0.5, -0.5], dtype=torch.float64)[torch.arange(N) % 4]).float()
    adv = torch.randn(N, generator=g)
    w = torch.rand(N, generator=g) * (torch.rand(N, generator=g) < 0.8)
    ref = (lp + 0.3 * torch.randn(N, generator=g).double()).float()
    return base, a, old, adv, w, ref


def check(base, V, a, old, adv, w, ref, kl, loss, logp, dz):
    z, eps = base[:, :V].double().numpy(), torch.finfo(base.dtype).eps / 2
    for i in range(z.shape[0]):
        L, lp, d = so.policy_loss(z[i], int(a[i]), float(old[i]), float(adv[i]), float(w[i]), None if ref is None else float(ref[i]), kl=kl)
        m = z[i].max()
        lse = z[i][int(a[i])] - lp
        e = 96 * U + 4 * U * (abs(z[i][int(a[i])] - m) + abs(lse - m) + abs(lp))
        assert abs(float(logp[i]) - lp) <= e, (i, float(logp[i]), lp)
        r, A, wi = np.exp(lp - float(old[i])), abs(float(adv[i])), float(w[i])
        er = e + 4 * U + U * abs(lp - float(old[i]))
        eg = wi * A * max(r, 1.2) * (er + 6 * U)
        if ref is not None:
            x = np.exp(float(ref[i]) - lp)
            eg += wi * kl * (x + 1 + abs(float(ref[i]) - lp)) * (e + 8 * U)
        assert abs(float(loss[i]) - L) <= eg + 4 * U * abs(L) + 1e-30, (i, float(loss[i]), L)
        if dz is None:
            continue
        g = 0.0 if wi == 0 else abs(d[int(a[i])]) / max(1e-300, 1 - np.exp(lp))
        p = np.exp(z[i] - lse)
        one = np.arange(V) == int(a[i])
        tol = (p + one) * (eg + 4 * U * g) + g * p * (e + 4 * U * (1 + np.abs(z[i] - m)) + 4 * U) + eps * np.abs(d) * (1 + 1e-3) + 1e-37
        bad = np.abs(dz[i].double().numpy() - d) > tol
        assert not bad.any(), (i, np.flatnonzero(bad)[:4], dz[i][bad][:4], d[bad][:4])


SIZES = [(1, 1), (3, 2), (7, 31), (9, 256), (5, 257), (4, 1000), (3, 1281), (2, 4099), (3, 10241), (5, 20483), (2, 50001)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N,V", SIZES)
def test_against_the_oracle(N, V, dtype):
    from paper_2002_03629_b200 import policy_loss as pl
    base, a, old, adv, w, ref = rows(N, V, dtype, seed=V)
    dev = [t.cuda() for t in (base, a, old, adv, w, ref)]
    loss, logp, dz = pl.policy_loss(*dev[:4], weights=dev[4], ref_logp=dev[5], kl_coef=0.3)
    assert dz.dtype == dtype and dz.shape == (N, V)
    check(base, V, a, old, adv, w, ref, 0.3, loss.cpu(), logp.cpu(), dz.cpu())
    # no KL term, no gradient; default weights
    one = torch.full((N,), 1.0 / N)
    loss, logp, none = pl.policy_loss(*dev[:4], need_grad=False)
    assert none is None
    check(base, V, a, old, adv, one, None, 0.0, loss.cpu(), logp.cpu(), None)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,pad", [(256, 5), (255, 8), (20481, 3), (33, 0)])
def test_strides_and_in_place(V, pad, dtype):
    """Rows further apart than they are long, gradients somewhere else or over the logits: same bits, and nothing beside the rows changes."""
    from paper_2002_03629_b200 import policy_loss as pl
    base, a, old, adv, w, ref = rows(6, V, dtype, seed=3, pad=pad)
    dev = [t.cuda() for t in (a, old, adv)]
    plain = pl.policy_loss(base[:, :V].contiguous().cuda(), *dev, weights=w.cuda())
    z = base.cuda()
    got = pl.policy_loss(z[:, :V], *dev, weights=w.cuda())
    check(base, V, a, old, adv, w, None, 0.0, got[0].cpu(), got[1].cpu(), got[2].cpu())
    out = torch.full((6, V + 7), 5.0, dtype=dtype, device="cuda")
    other = pl.policy_loss(z[:, :V], *dev, weights=w.cuda(), dlogits=out[:, 1:V + 1])
    assert (out[:, 0] == 5).all() and (out[:, V + 1:] == 5).all()
    for x, y in zip(got, other):
        assert torch.equal(x, y)
    tail = z[:, V:].clone()
    same = pl.policy_loss(z[:, :V], *dev, weights=w.cuda(), dlogits=z[:, :V])
    assert torch.equal(z[:, V:], tail) and same[2].data_ptr() == z.data_ptr()
    for x, y in zip(got, same):
        assert torch.equal(x, y)
    check(base, V, a, old, adv, w, None, 0.0, plain[0].cpu(), plain[1].cpu(), plain[2].cpu())


@pytest.mark.parametrize("V", [5, 300, 2000, 30001])
def test_rows_that_need_care(V):
    from paper_2002_03629_b200 import policy_loss as pl
    nan, inf = float("nan"), float("inf")
    base, a, old, adv, w, ref = rows(8, V, torch.float32, seed=1)
    w[:] = 0.5
    z = base.clone()
    a[:] = 0
    z[0, 1:] = -inf                     # only the action is possible: logp 0
    z[1, 2] = -inf
    z[2, :] = -inf                      # nothing is
    z[3, 3] = nan
    z[4, 1] = inf
    a[5] = V                            # no such symbol
    w[6], a[6], z[6, :] = 0.0, -100, nan          # padding
    w[7], z[7, V // 2] = 0.0, inf
    loss, logp, dz = (t.cpu() for t in pl.policy_loss(z.cuda(), a.cuda(), old.cuda(), adv.cuda(), weights=w.cuda(), ref_logp=ref.cuda(), kl_coef=0.1))
    assert logp[0] == 0 and torch.isfinite(loss[0]) and (dz[0] == 0).all()
    for i in (0, 1):
        lw, lp, d = so.policy_loss(z[i].double().numpy(), 0, float(old[i]), float(adv[i]), 0.5, float(ref[i]), kl=0.1)
        assert abs(float(loss[i]) - lw) < 1e-4 * (1 + abs(lw)) and np.abs(dz[i].double().numpy() - d).max() < 1e-4 * (1 + np.abs(d).max())
    assert dz[1, 2] == 0
    for i in (2, 3, 4, 5):
        assert torch.isnan(loss[i]) and torch.isnan(logp[i]) and torch.isnan(dz[i]).all(), i
    for i in (6, 7):
        assert loss[i] == 0 and (dz[i] == 0).all(), i
    assert torch.isnan(logp[6])


def test_all_rows_are_padding_and_no_rows():
    from paper_2002_03629_b200 import policy_loss as pl
    z = torch.full((4, 9), float("nan"), device="cuda")
    none = torch.full((4,), -1, device="cuda")
    x = torch.zeros(4, device="cuda")
    loss, logp, dz = pl.policy_loss(z, none, x, x, weights=x)
    assert (loss == 0).all() and (dz == 0).all()
    out = pl.policy_loss(z[:0], none[:0], x[:0], x[:0])
    assert [t.shape[0] for t in out] == [0, 0, 0]


def test_gradient_against_differences():
    """Central differences of the oracle's summed loss."""
    from paper_2002_03629_b200 import policy_loss as pl
    base, a, old, adv, w, ref = rows(4, 11, torch.float32, seed=8)
    dz = pl.policy_loss(base.cuda(), a.cuda(), old.cuda(), adv.cuda(), weights=w.cuda(), ref_logp=ref.cuda(), kl_coef=0.2)[2].cpu().double()
    h = 1e-5
    for i in range(4):
        for c in range(11):
            z = base[i].double().numpy()
            up, down = z.copy(), z.copy()
            up[c] += h
            down[c] -= h
            d = [so.policy_loss(x, int(a[i]), float(old[i]), float(adv[i]), float(w[i]), float(ref[i]), kl=0.2)[0] for x in (up, down)]
            assert abs((d[0] - d[1]) / (2 * h) - dz[i, c]) < 1e-5


def test_captured_twice_and_another_stream():
    from paper_2002_03629_b200 import policy_loss as pl
    base, a, old, adv, w, ref = (t.cuda() for t in rows(33, 5000, torch.bfloat16, seed=2))
    want = pl.policy_loss(base, a, old, adv, weights=w)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = pl.policy_loss(base, a, old, adv, weights=w)
    for _ in range(2):
        g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(want, got))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = pl.policy_loss(base, a, old, adv, weights=w, stream=s)
    s.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(want, got))


def test_refusals_of_the_binding():
    import paper_2002_03629_b200 as pkg
    from paper_2002_03629_b200 import policy_loss as pl
    base, a, old, adv, w, ref = (t.cuda() for t in rows(4, 8, torch.float32))
    for args, kw in (((base.half(), a, old, adv), {}), ((base.t(), a[:4].repeat(2), old.repeat(2), adv.repeat(2)), {}), ((base, a.int(), old, adv), {}),
                     ((base, a[:3], old, adv), {}), ((base, a, old.double(), adv), {}), ((base, a, old, adv), dict(weights=w[:2])),
                     ((base, a, old, adv), dict(kl_coef=0.1)), ((base, a, old, adv), dict(dlogits=base.bfloat16())), ((base, a, old, adv), dict(dlogits=base[:3])),
                     ((base, a, old, adv), dict(clip_low=-1.0)), ((base[:1].expand(4, 8), a, old, adv), {}), ((base, a, None, adv), {})):
        with pytest.raises(pkg.JsError):
            pl.policy_loss(*args, **kw)
