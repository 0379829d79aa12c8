"""Linear attention with a decay for each head against the oracle in 64 bits.

Tolerance.  With M the same recurrence of the magnitudes |q|, |k|, |v|, |S0| (every term of an output is a product of them, with weights
lambda^n > 0), an fp32 computation whose longest chain of additions has c terms is off by at most (c + 16) u M, u = 2^-24: a product, a
weight (an exponential of 2 ulp of an argument rounded once, n |log lambda| <= 90 where it counts: below 8 u for the weights that matter) and c additions.  Chains: Dk
terms of a score, at most 128 steps of a chunk, then one addition for every chunk and two roundings of the state: c = Dk + 128 + 3 n / 32.
Products of fp32 factors in two TF32 pieces are off by 3 * 2^-22 = 12 u each, two of them in a row by 24 u, and sums that are cut towards zero by 2 u an
addition, of eight terms at a time: with chunks of 32 steps Dk / 4 + 8 of them, in all 24 + Dk / 4 + 8 < Dk + 128.
bf16 outputs are rounded by eps / 2 of themselves; on the tensor cores the scores and the state at the chunk's start are rounded to
bf16 before their product, each by eps / 2 of its magnitude, below eps / 2 M together."""
import numpy as np
import pytest
import torch

from oracle import sequence_oracle as so

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def make(B, T, H, Dk, Dv, dtype, seed=0, state=True, decays=None):
    g = torch.Generator().manual_seed(seed)

    def normal(*s):
        return torch.randn(*s, generator=g)
    x = {"q": normal(B, T, H, Dk).to(dtype), "k": normal(B, T, H, Dk).to(dtype), "v": normal(B, T, H, Dv).to(dtype), "do": normal(B, T, H, Dv).to(dtype)}
    if decays is None:
        decays = [-0.5 * 0.25 ** i for i in range(H)]                # 0.61, 0.88, 0.97, ...
    x["ld"] = torch.tensor(decays, dtype=torch.float32)
    x["state"], x["dstate"] = (normal(B, H, Dk, Dv), normal(B, H, Dk, Dv)) if state else (None, None)
    return x


def dev(x):
    return {k: (v.cuda() if v is not None else None) for k, v in x.items()}


def slack(n, D):
    return (D + 128 + 3 * (n // 32 + 1) + 16) * U


def close(got, want, mag, tol, what, dtype=None):
    r = 0.0 if dtype in (None, torch.float32) else torch.finfo(dtype).eps / 2
    g = got.double().cpu().numpy()
    bad = ~(np.abs(g - want) <= r * np.abs(want) * 1.01 + (tol + r) * mag + 1e-30)
    assert not bad.any(), (what, np.argwhere(bad)[:3], g[bad][:3], want[bad][:3], mag[bad][:3], int(bad.sum()))


def check_forward(x, o, S, scale, seqs=None):
    """seqs: (row, first step, steps) of each sequence"""
    B, T, H, Dk = x["q"].shape
    dtype = x["q"].dtype
    for i, (b, at, n) in enumerate(seqs or [(b, 0, T) for b in range(B)]):
        for h in range(H):
            q, k, v = (x[a][b, at:at + n, h].double().numpy() for a in "qkv")
            S0 = None if x["state"] is None else x["state"][i, h].double().numpy()
            ld = float(x["ld"][h])
            want = so.linear_attention(q, k, v, ld, scale, S0)
            mag = so.linear_attention(abs(q), abs(k), abs(v), ld, abs(scale), None if S0 is None else abs(S0))
            close(o[b, at:at + n, h], want[0], mag[0], slack(n, Dk), f"o {i} {h}", dtype)
            if S is not None:
                close(S[i, h], want[1], mag[1], slack(n, Dk), f"state {i} {h}")


def check_backward(x, grads, scale, seqs=None):
    B, T, H, Dk = x["q"].shape
    dtype = x["q"].dtype
    for i, (b, at, n) in enumerate(seqs or [(b, 0, T) for b in range(B)]):
        for h in range(H):
            q, k, v, do = (x[a][b, at:at + n, h].double().numpy() for a in ("q", "k", "v", "do"))
            S0, dS = (None if x[a] is None else x[a][i, h].double().numpy() for a in ("state", "dstate"))
            ld = float(x["ld"][h])
            want = so.linear_attention_backward(q, k, v, ld, do, scale, S0, dS)
            mag = so.linear_attention_backward(abs(q), abs(k), abs(v), ld, abs(do), abs(scale), None if S0 is None else abs(S0), None if dS is None else abs(dS))
            for name, g, w, m in zip(("dq", "dk", "dv"), grads, want, mag):
                close(g[b, at:at + n, h], w, m, slack(n, max(Dk, v.shape[1])), f"{name} {i} {h}", dtype)
            close(grads[3][i, h], want[3], mag[3], slack(n, Dk), f"dstate {i} {h}")


def forward(x, scale, **kw):
    from paper_2002_03629_b200 import linear_attention as la
    d = dev(x)
    return la.linear_attention(d["q"], d["k"], d["v"], d["ld"], scale=scale, state=d["state"], **kw)


def backward(x, scale, **kw):
    from paper_2002_03629_b200 import linear_attention as la
    d = dev(x)
    return la.linear_attention_backward(d["q"], d["k"], d["v"], d["ld"], d["do"], scale=scale, state=d["state"], dstate=d["dstate"], **kw)


SIZES = [(1, 1, 1, 1, 1), (2, 7, 3, 5, 3), (1, 33, 2, 16, 16), (2, 100, 2, 64, 64), (1, 127, 1, 128, 128), (1, 128, 2, 64, 128), (1, 129, 2, 128, 64),
         (2, 257, 1, 96, 32), (1, 300, 2, 20, 128), (1, 640, 1, 128, 128), (3, 1, 2, 128, 128), (1, 391, 2, 32, 48), (1, 16, 1, 112, 80)]
IDS = ["x".join(map(str, s)) for s in SIZES]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=IDS)
def test_forward(size, dtype):
    B, T, H, Dk, Dv = size
    for state in (False, True):
        x = make(*size, dtype, seed=T, state=state)
        o, S = forward(x, Dk ** -0.5)
        assert o.dtype == dtype and S.dtype == torch.float32
        check_forward(x, o, S, Dk ** -0.5)
    assert forward(x, 1.0, need_state=False)[1] is None


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=IDS)
def test_backward(size, dtype):
    for state in (False, True):
        x = make(*size, dtype, seed=size[1] + 1, state=state)
        check_backward(x, backward(x, size[3] ** -0.5), size[3] ** -0.5)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("size", [(45, 37, 2, 64, 64), (40, 33, 2, 47, 50), (160, 3, 1, 30, 32), (80, 40, 1, 128, 65)], ids=str)
def test_many_sequences(size, dtype):
    """Enough of them that no head's columns are split to fill the GPU."""
    x = make(*size, dtype, seed=2)
    o, S = forward(x, 0.2)
    check_forward(x, o, S, 0.2)
    check_backward(x, backward(x, 0.2), 0.2)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("size", [(1, 2100, 2, 64, 64), (2, 1500, 1, 128, 96), (1, 1300, 3, 20, 30), (1, 2048, 1, 32, 128), (1, 1999, 1, 40, 7)], ids=str)
def test_few_long_sequences(size, dtype):
    """Cut into segments, on either path (widths that are no multiples of 16 take the one of fp32)."""
    for state in (False, True):
        x = make(*size, dtype, seed=3, state=state, decays=[-0.003, -0.7, -0.05][:size[2]])
        o, S = forward(x, 0.2)
        check_forward(x, o, S, 0.2)
        check_backward(x, backward(x, 0.2), 0.2)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("decays", [[0.0, -30.0], [-1e-6, -100.0], [float("-inf"), -2e-4]], ids=str)
def test_decays_from_none_to_everything(decays, dtype):
    x = make(1, 270, 2, 64, 64, dtype, decays=decays)
    o, S = forward(x, 0.125)
    check_forward(x, o, S, 0.125)
    check_backward(x, backward(x, 0.125), 0.125)


def test_whole_numbers_are_exact_on_the_tensor_cores():
    """Without decay, entries -1, 0, 1: every score, state and sum is a whole number below 256, which bf16 holds: outputs equal, each rounded once."""
    g = torch.Generator().manual_seed(4)
    x = {a: torch.randint(-1, 2, (2, 250, 2, 64), generator=g).to(torch.bfloat16) for a in ("q", "k", "v", "do")}
    x |= {"ld": torch.zeros(2), "state": None, "dstate": None}
    o, S = forward(x, 1.0)
    grads = backward(x, 1.0)
    for b in range(2):
        for h in range(2):
            q, k, v, do = (x[a][b, :, h].double().numpy() for a in ("q", "k", "v", "do"))
            wo, wS = so.linear_attention(q, k, v, 0.0)
            assert np.abs(np.tril(q @ k.T)).max() < 256 and np.abs(wS).max() < 256
            assert torch.equal(o[b, :, h].cpu(), torch.from_numpy(wo).to(torch.bfloat16)) and np.array_equal(S[b, h].cpu().numpy(), wS)
            for got, want in zip(grads, so.linear_attention_backward(q, k, v, 0.0, do)):
                got = got[b, :, h] if got.dim() == 4 and got.shape[1] == 250 else got[b, h]
                assert torch.equal(got.cpu(), torch.from_numpy(want).to(got.dtype))


LENS = [[1, 130, 0, 64, 257, 5], [0, 0, 3], [128, 128], [1] * 40, [500], [2600, 1, 1024, 1025, 0, 130, 2048], [17] * 100 + [700]]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("lens", LENS, ids=lambda v: "-".join(map(str, v))[:30])
def test_packed_sequences(lens, dtype):
    """Sequences of different lengths, empty ones among them, between rows of no sequence, which hold NaN and stay as they are."""
    N, first, behind = len(lens), 3, 70
    T = first + sum(lens) + behind
    x = make(1, T, 2, 64, 64, dtype, seed=9, state=False)
    g = torch.Generator().manual_seed(1)
    x["state"], x["dstate"] = (torch.randn(N, 2, 64, 64, generator=g) for _ in range(2))
    starts = first + np.concatenate([[0], np.cumsum(lens)])
    cu = torch.tensor(starts, dtype=torch.int32).cuda()
    seqs = [(0, int(a), n) for a, n in zip(starts, lens)]
    for a in ("q", "k", "v", "do"):
        x[a][:, :first] = float("nan")
        x[a][:, first + sum(lens):] = float("nan")
    out = torch.full((1, T, 2, 64), 3.0, dtype=dtype, device="cuda")
    o, S = forward(x, 0.2, cu_seqlens=cu, out=out)
    assert o is out
    check_forward(x, o, S, 0.2, seqs)
    for rows in (slice(0, first), slice(first + sum(lens), T)):
        assert (o[:, rows] == 3).all()
    grads = backward(x, 0.2, cu_seqlens=cu)
    check_backward(x, grads, 0.2, seqs)
    for gr in grads[:3]:
        assert (gr[:, :first] == 0).all() and (gr[:, first + sum(lens):] == 0).all()


def test_offsets_outside_the_rows_touch_nothing_else():
    """cu_seqlens is the device's: what lies outside the rows or descends is cut to them."""
    x = make(1, 40, 1, 32, 32, torch.bfloat16, state=False)
    whole = torch.full((3, 40, 1, 32), 9.0, dtype=torch.bfloat16, device="cuda")
    cu = torch.tensor([-5, 10, 4, 30, 1000], dtype=torch.int32).cuda()       # 0..10, 10..10, 4..30, 30..40
    from paper_2002_03629_b200 import linear_attention as la
    d = dev(x)
    o, S = la.linear_attention(d["q"], d["k"], d["v"], d["ld"], cu_seqlens=cu, out=whole[1:2])
    torch.cuda.synchronize()
    assert (whole[0] == 9).all() and (whole[2] == 9).all() and torch.isfinite(S).all() and (S[1] == 0).all()
    # rows that many sequences claim, more of them than there is room for segments of
    x = make(1, 3000, 1, 32, 32, torch.bfloat16, state=False)
    d, whole = dev(x), torch.full((3, 3000, 1, 32), 9.0, dtype=torch.bfloat16, device="cuda")
    cu = torch.tensor([0, 3000] * 60, dtype=torch.int32).cuda()
    la.linear_attention(d["q"], d["k"], d["v"], d["ld"], cu_seqlens=cu, out=whole[1:2])
    la.linear_attention_backward(d["q"], d["k"], d["v"], d["ld"], d["do"], cu_seqlens=cu)
    torch.cuda.synchronize()
    assert (whole[0] == 9).all() and (whole[2] == 9).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("layout", ["heads first", "one projection", "odd start", "shared keys"])
def test_strides(layout, dtype):
    from paper_2002_03629_b200 import linear_attention as la
    B, T, H, D = 2, 150, 2, 64
    x = make(B, T, H, D, D, dtype, seed=6)
    d = dev(x)
    if layout == "heads first":
        d |= {a: d[a].transpose(1, 2).contiguous().transpose(1, 2) for a in ("q", "k", "v", "do")}
    elif layout == "one projection":
        qkv = torch.cat([d["q"], d["k"], d["v"], d["do"]], -1)                   # [B, T, H, 4 D]
        d |= {a: qkv[..., i * D:(i + 1) * D] for i, a in enumerate(("q", "k", "v", "do"))}
    elif layout == "odd start":
        for a in ("q", "k", "v", "do"):
            room = torch.empty(B * T * H * (D + 1) + 1, dtype=dtype, device="cuda")[1:].view(B, T, H, D + 1)[..., :D]
            room.copy_(d[a])
            d[a] = room
    else:
        d["k"] = d["k"][:, :, :1].expand(B, T, H, D)
        x["k"] = d["k"].cpu()
    out = torch.empty(B, H, T, D, dtype=dtype, device="cuda").transpose(1, 2)
    o, S = la.linear_attention(d["q"], d["k"], d["v"], d["ld"], scale=0.1, state=d["state"], out=out)
    check_forward(x, o, S, 0.1)
    check_backward(x, la.linear_attention_backward(d["q"], d["k"], d["v"], d["ld"], d["do"], scale=0.1, state=d["state"], dstate=d["dstate"]), 0.1)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_sequences_in_parts_and_step_by_step(dtype):
    """A sequence in two calls, the second from the first one's state, then token by token."""
    from paper_2002_03629_b200 import linear_attention as la
    x = make(2, 200, 2, 64, 32, dtype, seed=12)
    d = dev(x)
    S, outs = d["state"], []
    for a, b in ((0, 130), (130, 131), (131, 190)):
        o, S = la.linear_attention(d["q"][:, a:b], d["k"][:, a:b], d["v"][:, a:b], d["ld"], scale=0.3, state=S)
        outs.append(o)
    for t in range(190, 200):
        outs.append(la.linear_attention_step(d["q"][:, t], d["k"][:, t], d["v"][:, t], d["ld"], S, scale=0.3)[:, None])
    check_forward(x, torch.cat(outs, 1), S, 0.3)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("size", [(1, 1, 1, 1), (3, 2, 64, 64), (2, 3, 128, 128), (5, 1, 7, 33), (2, 2, 128, 20), (300, 2, 16, 128), (1, 2, 100, 97)], ids=str)
def test_single_steps(size, dtype):
    from paper_2002_03629_b200 import linear_attention as la
    B, H, Dk, Dv = size
    x = make(B, 1, H, Dk, Dv, dtype, seed=B)
    d = dev(x)
    S = d["state"].clone()
    o = la.linear_attention_step(d["q"][:, 0], d["k"][:, 0], d["v"][:, 0], d["ld"], S, scale=0.3)
    check_forward(x, o[:, None], S, 0.3)
    # a state that does not lie on 16 bytes, rows that do not lie together
    room = torch.empty(S.numel() + 1, device="cuda")[1:].view_as(S)
    room.copy_(d["state"])
    q2 = torch.stack([d["q"][:, 0], d["q"][:, 0]], 2)[:, :, 1]
    out = torch.empty(B, 2, H, Dv, dtype=dtype, device="cuda")[:, 1]
    o2 = la.linear_attention_step(q2, d["k"][:, 0], d["v"][:, 0], d["ld"], room, scale=0.3, out=out)
    assert torch.equal(o2, o) and torch.equal(room, S)


def test_long_sequences_over_few_and_many_heads():
    """Long enough to be shared between thread blocks, against the masked product in 64 bits on the device."""
    for T, H, Dk, Dv, dtype in ((5000, 1, 128, 128, torch.bfloat16), (4111, 3, 64, 64, torch.bfloat16), (2500, 2, 64, 64, torch.float32)):
        x = make(1, T, H, Dk, Dv, dtype, seed=T, decays=[-0.3, -0.004, -0.0002][:H])
        o, S = forward(x, Dk ** -0.5)
        grads = backward(x, Dk ** -0.5)
        d = {a: (v.double().cuda() if v is not None else None) for a, v in x.items()}
        i = torch.arange(T, device="cuda", dtype=torch.float64)
        for h in range(H):
            ld = d["ld"][h]
            q, k, v, do = (d[a][0, :, h] for a in ("q", "k", "v", "do"))
            S0, dS, sc = d["state"][0, h], d["dstate"][0, h], Dk ** -0.5
            D = torch.tril(torch.exp(ld * (i[:, None] - i[None]).clamp(min=0)))
            up, down = torch.exp(ld * (i + 1))[:, None], torch.exp(ld * (T - 1 - i))[:, None]

            def both(f):
                return f(q, k, v, do, S0, dS).cpu().numpy(), f(*(t.abs() for t in (q, k, v, do, S0, dS))).cpu().numpy()
            for got, f, dt in ((o[0, :, h], lambda q, k, v, do, S0, dS: sc * (((q @ k.T) * D) @ v + up * (q @ S0)), dtype),
                               (S[0, h], lambda q, k, v, do, S0, dS: (k * down).T @ v + torch.exp(ld * T) * S0, None),
                               (grads[0][0, :, h], lambda q, k, v, do, S0, dS: sc * (((do @ v.T) * D) @ k + up * (do @ S0.T)), dtype),
                               (grads[1][0, :, h], lambda q, k, v, do, S0, dS: sc * (((do @ v.T) * D).T @ q) + down * (v @ dS.T), dtype),
                               (grads[2][0, :, h], lambda q, k, v, do, S0, dS: sc * (((q @ k.T) * D).T @ do) + down * (k @ dS), dtype),
                               (grads[3][0, h], lambda q, k, v, do, S0, dS: sc * ((q * up).T @ do) + torch.exp(ld * T) * dS, None)):
                want, mag = both(f)
                close(got, want, mag, slack(T, Dk), f"{T} {h}", dt)


def test_nothing_to_do():
    from paper_2002_03629_b200 import linear_attention as la
    z = torch.zeros(2, 0, 1, 16, device="cuda")
    ld, S0 = torch.zeros(1, device="cuda"), torch.randn(2, 1, 16, 16, device="cuda")
    o, S = la.linear_attention(z, z, z, ld, state=S0)
    assert o.shape == (2, 0, 1, 16) and torch.equal(S, S0)
    assert torch.equal(la.linear_attention_backward(z, z, z, ld, z, state=S0, dstate=S0)[3], S0)
    e = torch.zeros(0, 5, 1, 16, device="cuda")
    assert la.linear_attention(e, e, e, ld)[1].shape == (0, 1, 16, 16)
    y = torch.zeros(1, 5, 1, 16, device="cuda")
    assert la.linear_attention(y, y, y, ld, cu_seqlens=torch.zeros(1, dtype=torch.int32, device="cuda"))[1].shape == (0, 1, 16, 16)
    assert la.linear_attention_step(z.view(0, 1, 16), z.view(0, 1, 16), z.view(0, 1, 16), ld, S0[:0]).shape == (0, 1, 16)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_captured_replayed_and_on_two_streams(dtype):
    """Two graphs of the same call replayed side by side with an eager call: every one its own workspace, all the same bits."""
    from paper_2002_03629_b200 import linear_attention as la
    d = dev(make(1, 3000, 2, 64, 64, dtype, seed=5))

    def call():
        return (*la.linear_attention(d["q"], d["k"], d["v"], d["ld"], state=d["state"]),
                *la.linear_attention_backward(d["q"], d["k"], d["v"], d["ld"], d["do"], state=d["state"], dstate=d["dstate"]))
    want = call()
    graphs, outs = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(call())
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in range(3)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        with torch.cuda.stream(streams[2]):
            eager = call()
    torch.cuda.synchronize()
    for o in (*outs, eager):
        assert all(torch.equal(a, b) for a, b in zip(o, want))
    s = streams[0]
    other = la.linear_attention(d["q"], d["k"], d["v"], d["ld"], state=d["state"], stream=s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(other, want))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("decays", [[-0.01, -0.3], [-2.0, -0.9]], ids=["weak", "strong"])
def test_what_is_not_finite_stays_in_its_sequence_and_head(decays, dtype):
    """NaN, infinities and the types' largest values in one sequence, then in one head: all the others keep their bits."""
    from paper_2002_03629_b200 import linear_attention as la
    lens = [130, 45, 300, 7]
    at = np.concatenate([[0], np.cumsum(lens)])
    x = make(1, sum(lens), 2, 64, 64, dtype, seed=8, decays=decays, state=False)
    g = torch.Generator().manual_seed(5)
    x["state"], x["dstate"] = (torch.randn(4, 2, 64, 64, generator=g) for _ in range(2))
    cu = torch.tensor(at, dtype=torch.int32).cuda()
    bad = torch.tensor([float("nan"), float("inf"), -float("inf"), torch.finfo(dtype).max, torch.finfo(dtype).min, 1.0]).to(dtype)

    def run(y):
        d = dev(y)
        return (*la.linear_attention(d["q"], d["k"], d["v"], d["ld"], scale=0.1, state=d["state"], cu_seqlens=cu),
                *la.linear_attention_backward(d["q"], d["k"], d["v"], d["ld"], d["do"], scale=0.1, state=d["state"], dstate=d["dstate"], cu_seqlens=cu))
    want = run(x)
    for part in (1, 2):
        y = {a: t.clone() for a, t in x.items()}
        for a in ("q", "k", "v", "do"):
            y[a][:, at[part]:at[part + 1]] = bad[torch.randint(0, 6, y[a][:, at[part]:at[part + 1]].shape, generator=g)]
        for a, b in zip(run(y), want):
            rows = [i for i in range(4) if i != part]
            if a.shape[0] == 4:
                assert torch.equal(a[rows], b[rows])
            else:
                for i in rows:
                    assert torch.equal(a[:, at[i]:at[i + 1]], b[:, at[i]:at[i + 1]])
    y = {a: t.clone() for a, t in x.items()}
    for a in ("q", "k", "v", "do"):
        y[a][:, :, 0] = bad[torch.randint(0, 6, y[a][:, :, 0].shape, generator=g)]
    for a, b in zip(run(y), want):
        assert torch.equal(a[:, 1], b[:, 1]) if a.shape[0] == 4 else torch.equal(a[:, :, 1], b[:, :, 1])


@pytest.mark.parametrize("heads", [2, 40])
def test_packed_sequences_replayed_on_two_streams(heads):
    """The counter that the units are taken by, and the order of the segments, belong to the call: graphs and an eager call side by side, the same bits."""
    from paper_2002_03629_b200 import linear_attention as la
    lens = [1500, 3, 0, 700, 129, 1024, 64]
    cu = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32).cuda()
    d = dev(make(1, sum(lens), heads, 64, 64, torch.bfloat16, seed=6, state=False, decays=[-0.02] * heads))

    def call():
        return (*la.linear_attention(d["q"], d["k"], d["v"], d["ld"], cu_seqlens=cu),
                *la.linear_attention_backward(d["q"], d["k"], d["v"], d["ld"], d["do"], cu_seqlens=cu))
    want = call()
    graphs, outs = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(call())
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in range(3)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(4):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        with torch.cuda.stream(streams[2]):
            eager = call()
    torch.cuda.synchronize()
    for o in (*outs, eager):
        assert all(torch.equal(a, b) for a, b in zip(o, want))


def test_gradient_against_differences():
    """Directional differences of the fp32 kernel's own forward pass.  The loss is linear in v, S0 and (q, k apart) in q and in k: the
    difference over a step of 1 has no error but rounding, about 2^-24 of the summed magnitudes (100 steps of 64 products, 1e4 terms of size 1)."""
    from paper_2002_03629_b200 import linear_attention as la
    x = make(1, 100, 1, 32, 32, torch.float32, seed=21)
    d = dev(x)

    def loss(a):
        o, S = la.linear_attention(a["q"], a["k"], a["v"], a["ld"], scale=0.2, state=a["state"])
        return ((o.double() * d["do"].double()).sum() + (S.double() * d["dstate"].double()).sum()).item()
    grads = la.linear_attention_backward(d["q"], d["k"], d["v"], d["ld"], d["do"], scale=0.2, state=d["state"], dstate=d["dstate"])
    g = torch.Generator().manual_seed(2)
    for name, gr in zip(("q", "k", "v", "state"), grads):
        step = torch.randn(d[name].shape, generator=g).cuda()
        got = loss(d | {name: d[name] + step}) - loss(d)
        want = (gr.double() * step.double()).sum().item()
        assert abs(got - want) <= 1e-3 * max(1.0, abs(want)), name


def test_refusals_of_the_binding():
    import paper_2002_03629_b200 as pkg
    from paper_2002_03629_b200 import linear_attention as la
    d = dev(make(2, 9, 2, 16, 8, torch.float32))
    cu = torch.tensor([0, 9], dtype=torch.int32, device="cuda")
    ok = dict(q=d["q"], k=d["k"], v=d["v"], log_decay=d["ld"], state=d["state"])
    for kw in (dict(q=d["q"].half()), dict(q=d["q"].bfloat16()), dict(k=d["k"][:, :8]), dict(k=d["k"][..., :8]), dict(v=d["v"][:1]), dict(v=d["v"][0]),
               dict(log_decay=d["ld"][:1]), dict(log_decay=d["ld"].double()), dict(state=d["state"][:1]), dict(state=d["state"].transpose(2, 3)),
               dict(state=d["state"].cpu()), dict(q=d["q"].transpose(2, 3).contiguous().transpose(2, 3)), dict(cu_seqlens=cu), dict(scale=float("nan")),
               dict(out=torch.empty_like(d["q"])), dict(out=torch.empty(2, 1, 2, 8, device="cuda").expand(2, 9, 2, 8)), dict(k=d["k"].cpu())):
        with pytest.raises(pkg.JsError):
            la.linear_attention(**(ok | kw))
    wide = torch.zeros(1, 3, 1, 144, device="cuda")
    with pytest.raises(pkg.JsError):
        la.linear_attention(wide, wide, wide, torch.zeros(1, device="cuda"))
    one = dict(q=d["q"][:1], k=d["k"][:1], v=d["v"][:1], log_decay=d["ld"])
    for bad in (cu.long(), cu.cpu(), cu[:0], cu[None]):
        with pytest.raises(pkg.JsError):
            la.linear_attention(**one, cu_seqlens=bad)
    with pytest.raises(pkg.JsError):
        la.linear_attention_backward(d["q"], d["k"], d["v"], d["ld"], d["q"])
    step = dict(q=d["q"][:, 0], k=d["k"][:, 0], v=d["v"][:, 0], log_decay=d["ld"], state=d["state"])
    for kw in (dict(state=None), dict(state=d["state"][:1]), dict(q=d["q"]), dict(v=d["v"])):
        with pytest.raises(pkg.JsError):
            la.linear_attention_step(**(step | kw))
