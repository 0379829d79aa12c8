"""What the sequence operators refuse, without a device: the C entry points with bad sizes and pointers, the binding with host tensors."""
import ctypes as C

import pytest
import torch


@pytest.fixture(scope="module")
def pkg():
    import __graft_entry__ as ge
    ge.build()
    import paper_2002_03629_b200 as p
    return p


FAKE = 1 << 20          # an address that is never read: every one of these calls is refused before a launch


def la_args(**changes):
    from paper_2002_03629_b200 import linear_attention as la
    s = la._Shape(type=0, B=2, N=0, T=5, H=3, Dk=8, Dv=8, cu_seqlens=None, log_decay=FAKE, scale=1.0)
    for k, v in changes.items():
        setattr(s, k, v)
    return s


@pytest.mark.parametrize("changes", [dict(type=2), dict(H=0), dict(Dk=0), dict(Dk=129), dict(Dv=0), dict(Dv=200), dict(B=-1), dict(T=-1), dict(T=1 << 31),
                                     dict(log_decay=None), dict(cu_seqlens=FAKE, B=2), dict(cu_seqlens=FAKE, B=1, N=-1), dict(B=1 << 24, H=2),
                                     dict(scale=float("nan")), dict(scale=float("inf"))], ids=str)
def test_linear_attention_shapes(pkg, changes):
    from paper_2002_03629_b200 import linear_attention as la
    lib, s, t = la._lib(), la_args(**changes), la._Tensor(FAKE, 120, 24, 8)
    p, r = C.byref(s), C.byref(t)
    assert lib.la_workspace(p, 0) == 0 and lib.la_workspace(p, 1) == 0
    assert lib.la_forward(p, r, r, r, None, r, None, FAKE, 1 << 30, None) == la.LA_ERR_INVALID
    assert lib.la_backward(p, r, r, r, None, r, None, r, r, r, None, FAKE, 1 << 30, None) == la.LA_ERR_INVALID
    s.T = 1 if s.T == 5 else s.T
    assert lib.la_step(p, r, r, r, FAKE, r, None) == la.LA_ERR_INVALID


def test_linear_attention_pointers(pkg):
    from paper_2002_03629_b200 import linear_attention as la
    lib, s, t, bad, odd = la._lib(), la_args(), la._Tensor(FAKE, 120, 24, 8), la._Tensor(None, 120, 24, 8), la._Tensor(FAKE + 2, 120, 24, 8)
    p, r = C.byref(s), C.byref(t)
    for x in (None, C.byref(bad), C.byref(odd)):
        for i in range(4):
            a = [r] * 4
            a[i] = x
            assert lib.la_forward(p, a[0], a[1], a[2], None, a[3], None, FAKE, 1 << 30, None) == la.LA_ERR_INVALID
        for i in range(7):
            a = [r] * 7
            a[i] = x
            assert lib.la_backward(p, a[0], a[1], a[2], None, a[3], None, a[4], a[5], a[6], None, FAKE, 1 << 30, None) == la.LA_ERR_INVALID
    need = lib.la_workspace(p, 0)
    assert lib.la_forward(p, r, r, r, None, r, None, FAKE, need - 1, None) == la.LA_ERR_INVALID
    assert lib.la_forward(p, r, r, r, None, r, None, None, need, None) == la.LA_ERR_INVALID
    assert lib.la_step(p, r, r, r, FAKE, r, None) == la.LA_ERR_INVALID              # T = 5
    s.T = 1
    assert lib.la_step(p, r, r, r, None, r, None) == la.LA_ERR_INVALID
    assert lib.la_step(p, r, r, r, FAKE + 2, r, None) == la.LA_ERR_INVALID
    s.B = 0
    assert lib.la_step(p, r, r, r, None, r, None) == la.LA_OK                       # nothing to do


def test_policy_loss_arguments(pkg):
    from paper_2002_03629_b200 import policy_loss as pl
    lib = pl._lib()

    def call(z=FAKE, type=0, N=4, V=7, stride=7, a=FAKE, old=FAKE, adv=FAKE, lo=0.2, hi=0.2, kl=0.0, loss=FAKE, logp=FAKE, dz=FAKE, ds=7):
        return lib.policy_loss(z, type, N, V, stride, a, old, adv, None, None, lo, hi, kl, loss, logp, dz, ds, None)
    nan, inf = float("nan"), float("inf")
    for bad in (dict(z=None), dict(type=2), dict(N=-1), dict(V=0), dict(V=200001, stride=1 << 25, ds=1 << 25), dict(stride=6), dict(ds=6), dict(a=None),
                dict(old=None), dict(adv=None), dict(loss=None), dict(logp=None), dict(z=FAKE + 2), dict(dz=FAKE + 1), dict(lo=-0.1), dict(hi=-0.1), dict(lo=nan),
                dict(hi=inf), dict(kl=nan), dict(ds=9), dict(N=1 << 29)):
        assert call(**bad) == pl.PL_ERR_INVALID, bad
    assert call(N=0, z=None) == pl.PL_OK


def test_adamw_arguments(pkg):
    from paper_2002_03629_b200 import adamw as aw
    import numpy as np
    lib = aw._lib()

    def call(p=FAKE, g=FAKE, copy=0, n=9, count=1, gt=0, bits=32, m=FAKE, v=FAKE, ms=None, vs=None, **opt):
        t = np.array([[p or 0, g or 0, copy, n]], np.int64)
        o = aw._Options(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, step=1, seed=-1)
        for k, x in opt.items():
            setattr(o, k, x)
        return lib.adamw_step(t.ctypes.data, count, gt, bits, m, v, ms, vs, C.byref(o), None)
    nan, inf = float("nan"), float("inf")
    for bad in (dict(p=None), dict(g=None), dict(p=FAKE + 2), dict(g=FAKE + 2), dict(copy=FAKE + 1), dict(n=-1), dict(n=(1 << 33) + 1), dict(count=-1), dict(gt=2),
                dict(bits=16), dict(m=None), dict(v=None), dict(m=FAKE + 4), dict(bits=8), dict(bits=8, ms=FAKE), dict(beta1=1.0), dict(beta2=1.0), dict(beta1=-0.1),
                dict(beta2=nan), dict(eps=0.0), dict(eps=-1.0), dict(eps=1e-60), dict(eps=inf), dict(lr=inf), dict(weight_decay=nan), dict(step=0), dict(step=-3)):
        assert call(**bad) == aw.ADAMW_ERR_INVALID, bad
    assert call(n=0, p=None, g=None, m=None) == aw.ADAMW_OK                         # nothing to do
    assert lib.adamw_step(None, 0, 0, 32, None, None, None, None, C.byref(aw._Options(lr=0, beta1=0, beta2=0, eps=1, step=1)), None) == aw.ADAMW_OK


def test_binding_refuses_host_tensors(pkg):
    from paper_2002_03629_b200 import adamw as aw, linear_attention as la, policy_loss as pl
    x, ld = torch.zeros(2, 5, 3, 8), torch.zeros(3)
    for call in (lambda: la.linear_attention(x, x, x, ld), lambda: la.linear_attention_backward(x, x, x, ld, x),
                 lambda: la.linear_attention_step(x[:, 0], x[:, 0], x[:, 0], ld, torch.zeros(2, 3, 8, 8)),
                 lambda: pl.policy_loss(torch.zeros(4, 7), torch.zeros(4, dtype=torch.long), torch.zeros(4), torch.zeros(4)),
                 lambda: aw.adamw_step([torch.zeros(3)], [torch.zeros(3)], aw.adamw_state([torch.zeros(3)]), 1, 1e-3)):
        with pytest.raises(pkg.JsError):
            call()
    with pytest.raises(pkg.JsError):
        aw.adamw_state([torch.zeros(3)], bits=4)
    with pytest.raises(pkg.JsError):
        aw.adamw_state([])
    with pytest.raises(pkg.JsError):
        aw.adamw_step([torch.zeros(3)], [], aw.adamw_state([torch.zeros(3)]), 1, 1e-3)


def test_overlapping_results_are_seen(pkg):
    from paper_2002_03629_b200 import linear_attention as la
    t = torch.zeros(2, 5, 3, 8)
    assert la._apart(t.shape, t.stride())
    assert la._apart((2, 5, 3, 8), t.transpose(1, 2).contiguous().transpose(1, 2).stride())
    assert not la._apart((2, 5, 3, 8), t[:1].expand(2, 5, 3, 8).stride())
    assert not la._apart((2, 5, 3, 8), (120, 24, 4, 1))
    assert la._apart((1, 5, 1, 8), (0, 8, 0, 1))
