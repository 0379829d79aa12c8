"""The sequence operators where offsets pass 32 bits (values, and bytes): the last rows against the oracle, the tolerances those of the operators' own tests."""
import numpy as np
import pytest
import torch

from oracle import sequence_oracle as so
from tests import test_gpu_linear_attention as tla
from tests import test_gpu_policy_loss as tpl

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def room():
    if torch.cuda.mem_get_info()[0] < 80 << 30:
        pytest.skip("80 GB of device memory")
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("packed", [False, True], ids=["one sequence", "packed"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_linear_attention(dtype, packed):
    """2^31 values a tensor and more.  At decays of e^-1 the outputs of the last steps know nothing of steps 300 before them (e^-300)."""
    from paper_2002_03629_b200 import linear_attention as la
    T, H, D, tail = (1 << 20) + 77, 16, 128, 400
    g = torch.Generator(device="cuda").manual_seed(0)
    q, k, v = (torch.empty(1, T, H, D, dtype=dtype, device="cuda").normal_(generator=g) for _ in range(3))
    ld = torch.full((H,), -1.0, device="cuda")
    cu = torch.tensor([0, 5, 1 << 19, T], dtype=torch.int32, device="cuda") if packed else None
    o, S = la.linear_attention(q, k, v, ld, scale=0.1, cu_seqlens=cu)
    host = {"ld": ld.cpu()[:2], "state": None} | {a: t[:, T - tail:, [0, H - 1]].cpu() for a, t in (("q", q), ("k", k), ("v", v))}
    # (the oracle starts from zero at step T - 400; the first 300 of its outputs are left out)
    want = [so.linear_attention(*(host[a][0, :, h].double().numpy() for a in "qkv"), -1.0, 0.1) for h in range(2)]
    mag = [so.linear_attention(*(abs(host[a][0, :, h].double().numpy()) for a in "qkv"), -1.0, 0.1) for h in range(2)]
    for i, h in enumerate((0, H - 1)):
        tla.close(o[0, T - 100:, h], want[i][0][300:], mag[i][0][300:], tla.slack(tail, D), "o", dtype)
        tla.close(S[-1, h], want[i][1], mag[i][1], tla.slack(tail, D), "state")
    del o
    grads = la.linear_attention_backward(q, k, v, ld, v, scale=0.1, cu_seqlens=cu)
    for i, h in enumerate((0, H - 1)):
        a = [host[x][0, :, i].double().numpy() for x in "qkv"]
        w, m = so.linear_attention_backward(*a, -1.0, a[2], 0.1), so.linear_attention_backward(*map(abs, a), -1.0, abs(a[2]), 0.1)
        for n, name in enumerate(("dq", "dk", "dv")):
            tla.close(grads[n][0, T - 100:, h], w[n][300:], m[n][300:], tla.slack(tail, D), name, dtype)


def test_single_steps():
    from paper_2002_03629_b200 import linear_attention as la
    B, H, D = 8300, 16, 128
    g = torch.Generator(device="cuda").manual_seed(1)
    S = torch.zeros(B, H, D, D, device="cuda")
    assert S.numel() > 1 << 31
    S[-1].normal_(generator=g)
    q, k, v = (torch.empty(B, H, D, device="cuda").normal_(generator=g) for _ in range(3))
    ld = torch.linspace(-0.1, 0, H).cuda()
    x = {"q": q[-1:, None].cpu(), "k": k[-1:, None].cpu(), "v": v[-1:, None].cpu(), "ld": ld.cpu(), "state": S[-1:].cpu()}
    o = la.linear_attention_step(q, k, v, ld, S, scale=0.1)
    tla.check_forward(x, o[-1:, None], S[-1:], 0.1)


@pytest.mark.parametrize("N,V", [(50001, 50001), (2, 200000), ((1 << 23) + 5, 300)], ids=str)
def test_policy_loss(N, V):
    """Rows behind 2^31 values; the longest rows; many short ones."""
    from paper_2002_03629_b200 import policy_loss as pl
    base, a, old, adv, w, ref = tpl.rows(4, V, torch.bfloat16, seed=N)
    z = torch.zeros(N, V, dtype=torch.bfloat16, device="cuda")
    n = min(4, N)
    z[N - n:] = base[:n].cuda()

    def rows(t, fill):
        full = torch.full((N,), fill, dtype=t.dtype, device="cuda")
        full[N - n:] = t[:n].cuda()
        return full
    loss, logp, dz = pl.policy_loss(z, rows(a, 0), rows(old, -1.0), rows(adv, 0.5), weights=rows(w, 1.0), ref_logp=rows(ref, -1.0), kl_coef=0.3)
    tpl.check(base[:n], V, a[:n], old[:n], adv[:n], w[:n], ref[:n], 0.3, loss[N - n:].cpu(), logp[N - n:].cpu(), dz[N - n:].cpu())


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw(bits):
    """One tensor of 2^32 values and more (32-bit states: 2^31), another behind it: the last values bit for bit, 8-bit codes and the random bits of
    their places included."""
    from paper_2002_03629_b200 import adamw as aw
    n, tail = ((1 << 32) if bits == 8 else (1 << 31)) + 700, 512 + 188             # (two whole blocks and a part of one)
    g = torch.Generator().manual_seed(3)
    sizes = [n, 300]
    params = [torch.zeros(k, device="cuda") for k in sizes]
    grads = [torch.zeros(k, dtype=torch.bfloat16, device="cuda") for k in sizes]
    for p, gr in zip(params, grads):
        k = min(tail, p.numel())
        p[-k:] = torch.randn(k, generator=g).cuda()
        gr[-k:] = torch.randn(k, generator=g).cuda().to(torch.bfloat16)
    before = [p[-min(tail, p.numel()):].cpu().numpy().copy() for p in params]
    state = aw.adamw_state(params, bits)
    aw.adamw_step(params, grads, state, 1, 0.01, seed=7)
    first = (n + 255) // 256 * 256
    for i, (at, k) in enumerate(((n - tail, tail), (first, 300))):
        zero = np.zeros(k, np.float32)
        p, m, v, root = so.adamw_f32(before[i], grads[i][-k:].float().cpu().numpy(), zero, zero, 1, 0.01)
        assert np.array_equal(params[i][-k:].cpu().numpy(), p)
        if bits == 32:
            assert np.array_equal(state.m[at:at + k].cpu().numpy(), m) and np.array_equal(state.v[at:at + k].cpu().numpy(), v)
            continue
        for b in range(0, k, 256):
            e = min(b + 256, k)
            r = so.random_bits(list(range(at + b, at + e)), 7)
            for got, scale, x, bits16 in ((state.m, state.m_scale, m, r & 0xFFFF), (state.v, state.v_scale, root, r >> 16)):
                codes, s = so.float8_cut(x[b:e], bits16)
                if got is state.v:
                    codes = np.maximum(codes, (x[b:e] > 0).astype(codes.dtype))
                assert np.array_equal(got[at + b:at + e].view(torch.uint8).cpu().numpy(), codes) and float(scale[(at + b) // 256]) == s
