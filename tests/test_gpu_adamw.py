"""The AdamW step against the oracle: in fp32 with the documented roundings bit for bit (8-bit codes included), and in 64 bits.

Tolerance against 64 bits.  With u = 2^-24, a new moment is three roundings of terms of its own size, v the same with g'^2 rounded once more;
the update then takes the root (half of v's relative error + u), its factor, eps, the quotient and two factors rounded: below 12 u of the update;
p is rounded twice more, below 3 u of |p| + |update|, factor 1 - lr wd included.  A moment whose terms cancel is off by u of its larger term."""
import numpy as np
import pytest
import torch

from oracle import sequence_oracle as so

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
SIZES = [1, 3, 255, 256, 257, 1000, 4096, 4097, 0, 70001]
OPT = dict(betas=(0.9, 0.99), eps=1e-6, weight_decay=0.1)


def make(sizes, grad, bits, seed=0, offset=0, copies=True):
    from paper_2002_03629_b200 import adamw as aw
    g = torch.Generator().manual_seed(seed)
    total = sum(sizes)

    def views(dtype, std):
        flat = torch.empty(total + offset, dtype=dtype)
        flat.copy_(torch.randn(total + offset, generator=g) * std)
        return list(flat.cuda()[offset:].split(sizes))
    params, grads = views(torch.float32, 0.05), views(grad, 0.01)
    cps = [torch.full_like(p, 7.0, dtype=torch.bfloat16) for p in params] if copies else None
    return params, grads, aw.adamw_state(params, bits), cps


def pieces(sizes):
    at = 0
    for n in sizes:
        yield at, n
        at += (n + 255) // 256 * 256


def state32(state, sizes):
    """m and v as fp32 values per tensor."""
    out = []
    for at, n in pieces(sizes):
        m, v = (t[at:at + n].float().cpu().numpy() if t.dtype == torch.float32 else t[at:at + n].view(torch.uint8).cpu().numpy() for t in state[:2])
        if state.m_scale is not None:
            blocks = np.arange(at, at + n) // 256
            m = (so.float8_value(m) * state.m_scale.cpu().numpy()[blocks]).astype(np.float32)
            v = (so.float8_value(v) * state.v_scale.cpu().numpy()[blocks]).astype(np.float32)
            v = v * v
        out.append((m, v))
    return out


@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("grad", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("bits", [32, 8])
def test_steps_bit_for_bit(bits, grad, offset):
    from paper_2002_03629_b200 import adamw as aw
    params, grads, state, copies = make(SIZES, grad, bits, offset=offset)
    gs = torch.full((1,), 0.75, device="cuda")
    want = [p.cpu().numpy().copy() for p in params]
    for step in (1, 2, 3):
        before = state32(state, SIZES)
        aw.adamw_step(params, grads, state, step, 0.01, copies=copies, grad_scale=gs, seed=step + 100, **OPT)
        m8, v8 = (t.view(torch.uint8).cpu().numpy() if bits == 8 else t.cpu().numpy() for t in state[:2])
        for i, (at, n) in enumerate(pieces(SIZES)):
            if n == 0:
                continue
            g = grads[i].float().cpu().numpy()
            p, m, v, root = so.adamw_f32(want[i], g, *before[i], step, 0.01, grad_scale=0.75, **OPT)
            np.testing.assert_array_equal(params[i].cpu().numpy(), p, err_msg=f"p {n}")
            np.testing.assert_array_equal(copies[i].float().cpu().numpy(), torch.from_numpy(p).to(torch.bfloat16).float().numpy())
            p64 = so.adamw(want[i], g, *before[i], step, 0.01, grad_scale=0.75, **OPT)[0]
            upd = np.abs(p64 - want[i])
            assert np.all(np.abs(p - p64) <= 12 * U * upd + 3 * U * (np.abs(want[i]) + upd) + 1e-30)
            want[i] = p
            if bits == 32:
                np.testing.assert_array_equal(m8[at:at + n], m)
                np.testing.assert_array_equal(v8[at:at + n], v)
            else:
                for b in range(0, n, 256):
                    if n > 5000 and b not in (0, 256 * 100, n // 256 * 256):       # the oracle takes its time
                        continue
                    e = min(n, b + 256)
                    r = so.random_bits(np.arange(at + b, at + e), step + 100)
                    mc, ms = so.float8_cut(m[b:e], r & 0xFFFF)
                    vc, vs = so.float8_cut(root[b:e], r >> 16)
                    vc = np.where((root[b:e] > 0) & (vc == 0), 1, vc)
                    assert float(state.m_scale[(at + b) // 256]) == ms and float(state.v_scale[(at + b) // 256]) == vs
                    np.testing.assert_array_equal(m8[at + b:at + e], mc)
                    np.testing.assert_array_equal(v8[at + b:at + e], vc)
            # places behind the tensor's end stay as they were
            end = (n + 255) // 256 * 256
            assert not m8[at + n:at + end].any() and not v8[at + n:at + end].any()


def test_same_call_same_bits_and_no_seed_is_the_step():
    from paper_2002_03629_b200 import adamw as aw
    out = []
    for seed in (5, None):
        params, grads, state, _ = make([5000, 33], torch.float32, 8, copies=False)
        aw.adamw_step(params, grads, state, 5, 0.01, seed=seed, **OPT)
        out.append([t.view(torch.uint8).clone() for t in state[:2]] + [p.clone() for p in params])
    assert all(torch.equal(a, b) for a, b in zip(*out))


def test_more_tensors_than_one_launch_takes():
    from paper_2002_03629_b200 import adamw as aw
    sizes = [(7 * i) % 300 for i in range(1500)]
    params, grads, state, _ = make(sizes, torch.float32, 32, copies=False)
    want = [so.adamw_f32(p.cpu().numpy(), g.cpu().numpy(), np.zeros(n, np.float32), np.zeros(n, np.float32), 1, 0.01, **OPT)[0]
            for p, g, n in zip(params, grads, sizes)]
    aw.adamw_step(params, grads, state, 1, 0.01, **OPT)
    for p, w in zip(params, want):
        np.testing.assert_array_equal(p.cpu().numpy(), w)


def test_numbers_on_the_device_and_a_captured_step():
    """step, lr, grad_scale and skip as device values: a replay reads them anew; the same results as with plain numbers."""
    from paper_2002_03629_b200 import adamw as aw
    sizes = [300, 5000]
    a, b = make(sizes, torch.float32, 8, copies=False), make(sizes, torch.float32, 8, copies=False)
    step, lr = torch.ones(1, dtype=torch.int64, device="cuda"), torch.full((1,), 0.01, device="cuda")
    skip, gs = torch.ones(1, dtype=torch.int32, device="cuda"), torch.ones(1, device="cuda")
    aw.adamw_step(a[0], a[1], a[2], step, lr, grad_scale=gs, skip=skip, **OPT)         # skipped: also a warm-up
    assert all(torch.equal(p, q) for p, q in zip(a[0], b[0])) and not a[2].m.view(torch.uint8).any()
    skip.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        aw.adamw_step(a[0], a[1], a[2], step, lr, grad_scale=gs, skip=skip, **OPT)
    for t in range(1, 5):
        step.fill_(t)
        lr.fill_(0.01 / t)
        gs.fill_(0.5 * t)
        skip.fill_(int(t == 3))
        graph.replay()
        if t != 3:
            aw.adamw_step(b[0], b[1], b[2], t, float(lr), grad_scale=gs, **OPT)
        torch.cuda.synchronize()
        for p, q in zip(a[0], b[0]):
            # the factors' powers in 64 bits may differ in their last bit between host and device: then one factor's last fp32 bit
            assert (p - q).abs().max().item() <= 4 * U * (1 + q.abs().max().item())


def test_zero_and_non_finite_gradients():
    from paper_2002_03629_b200 import adamw as aw
    for bits in (32, 8):
        params, grads, state, _ = make([600], torch.float32, bits, copies=False)
        grads[0].zero_()
        before = params[0].clone()
        aw.adamw_step(params, grads, state, 1, 0.01, **OPT)
        assert torch.equal(params[0], before * np.float32(1 - 0.01 * 0.1))
        assert not state.m.view(torch.uint8).any() and not state.v.view(torch.uint8).any()
        grads[0][300] = float("inf")
        aw.adamw_step(params, grads, state, 2, 0.01, **OPT)
        ok = torch.isfinite(params[0])
        assert ok.sum() == 599 and not ok[300]
        aw.adamw_step(params, grads, state, 3, 0.01, **OPT)              # the state keeps it: its value, or its block
        bad = ~torch.isfinite(params[0])
        assert bad[300] and not bad[:256].any() and not bad[512:].any() and (bits == 8 or bad.sum() == 1)


def test_refusals_of_the_binding():
    import paper_2002_03629_b200 as pkg
    from paper_2002_03629_b200 import adamw as aw
    params, grads, state, copies = make([300, 20], torch.float32, 32)
    half = [g.to(torch.float16) for g in grads]
    for kw in (dict(grads=half), dict(grads=[grads[0], grads[1].bfloat16()]), dict(grads=[grads[1], grads[0]]), dict(params=[params[0], params[1].double()]),
               dict(params=[params[0], params[0][:20]]), dict(copies=[copies[0]]), dict(copies=[copies[0], copies[1].float()]),
               dict(state=aw.adamw_state([params[0]])), dict(state=state._replace(v=state.v.double())), dict(step=0), dict(step=torch.ones(1, device="cuda")),
               dict(lr=torch.ones(2, device="cuda")), dict(grad_scale=torch.ones(1)), dict(skip=torch.ones(1, device="cuda")), dict(betas=(1.0, 0.9)),
               dict(eps=0.0), dict(params=[params[0], torch.zeros(40, device="cuda")[::2]])):
        a = dict(params=params, grads=grads, state=state, step=1, lr=0.1, copies=copies) | kw
        with pytest.raises(pkg.JsError):
            aw.adamw_step(**a)
    assert not state.m.any()


def test_another_stream():
    from paper_2002_03629_b200 import adamw as aw
    params, grads, state, _ = make([100000], torch.float32, 32, copies=False)
    want = so.adamw_f32(params[0].cpu().numpy(), 3 * grads[0].cpu().numpy(), np.zeros(100000, np.float32), np.zeros(100000, np.float32), 1, 0.01, **OPT)[0]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        torch.cuda._sleep(1_000_000)
        grads[0].mul_(3)
    aw.adamw_step(params, grads, state, 1, 0.01, stream=s, **OPT)
    s.synchronize()
    np.testing.assert_array_equal(params[0].cpu().numpy(), want)
