"""The sequence operators as a training program uses them together: tokens -> linear attention over packed sequences -> logits -> clipped policy loss ->
gradients -> AdamW, and the decoding that such training starts from.  The matrix products around them are torch's, in 64 bits, their results rounded to the
operators' type; so every operator's result can be held against the oracle on the inputs that it really had, with its own tests' tolerances."""
import numpy as np
import pytest
import torch

from oracle import sequence_oracle as so
from tests import test_gpu_linear_attention as tla
from tests import test_gpu_policy_loss as tpl

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
V, DM, H, D, SCALE = 50, 40, 2, 32, 32 ** -0.5
LENS, BEHIND = [40, 1, 0, 133], 6                          # steps of the sequences, rows behind the last one
T = sum(LENS) + BEHIND
OPT = dict(betas=(0.9, 0.99), eps=1e-6, weight_decay=0.1)


class Program:
    """Weights, a batch of rollouts, and one training step."""

    def __init__(self, dtype, bits, seed=0):
        from paper_2002_03629_b200 import adamw as aw
        g = torch.Generator().manual_seed(seed)
        self.dtype = dtype

        def normal(*s, std=1.0):
            return (torch.randn(*s, generator=g) * std).cuda()
        self.params = [normal(V, DM), normal(DM, H * D, std=DM ** -0.5), normal(DM, H * D, std=DM ** -0.5), normal(DM, H * D, std=DM ** -0.5),
                       normal(H * D, V, std=0.2)]
        self.copies = [p.to(torch.bfloat16) for p in self.params] if dtype == torch.bfloat16 else None
        self.state = aw.adamw_state(self.params, bits)
        self.ld = torch.tensor([-0.02, -0.3]).cuda()
        self.cu = torch.tensor(np.concatenate([[0], np.cumsum(LENS)]), dtype=torch.int32).cuda()
        self.tokens, self.actions = (torch.randint(0, V, (T,), generator=g).cuda() for _ in range(2))
        self.adv = torch.randn(T, generator=g).cuda()
        self.weights = torch.full((T,), 1.0 / (T - BEHIND)).cuda()
        self.weights[T - BEHIND:] = 0
        self.out = torch.zeros(1, T, H, D, dtype=dtype).cuda()                     # (rows behind the last sequence: zeros that nobody writes)
        # ratios away from the clip bounds
        logp = torch.log_softmax(self.forward()[-1].double(), 1).gather(1, self.actions[:, None])[:, 0]
        self.old = (logp - torch.tensor([0.1, -0.1, 0.5, -0.5], dtype=torch.float64).cuda()[torch.arange(T) % 4]).float()

    def used(self):
        return [w.double() for w in (self.params if self.copies is None else self.copies)]

    def forward(self):
        from paper_2002_03629_b200 import linear_attention as la
        E, Wq, Wk, Wv, Wo = self.used()
        x = E[self.tokens]
        q, k, v = ((x @ W).to(self.dtype).view(1, T, H, D) for W in (Wq, Wk, Wv))
        o, _ = la.linear_attention(q, k, v, self.ld, scale=SCALE, cu_seqlens=self.cu, need_state=False, out=self.out)
        return x, q, k, v, o, (o.view(T, H * D).double() @ Wo).to(self.dtype)

    def gradients(self):
        """Everything that the step computes, the parameters' gradients last."""
        from paper_2002_03629_b200 import linear_attention as la, policy_loss as pl
        E, Wq, Wk, Wv, Wo = self.used()
        x, q, k, v, o, z = self.forward()
        loss, logp, dz = pl.policy_loss(z, self.actions, self.old, self.adv, weights=self.weights)
        do = (dz.double() @ Wo.T).to(self.dtype).view(1, T, H, D)
        dq, dk, dv, dS = la.linear_attention_backward(q, k, v, self.ld, do, scale=SCALE, cu_seqlens=self.cu)
        heads = [t.view(T, H * D).double() for t in (dq, dk, dv)]
        dx = sum(t @ W.T for t, W in zip(heads, (Wq, Wk, Wv)))
        one = torch.zeros(V, T, dtype=torch.float64, device="cuda").scatter_(0, self.tokens[None], 1.0)
        grads = [one @ dx, *(x.T @ t for t in heads), o.view(T, H * D).double().T @ dz.double()]
        return dict(q=q, k=k, v=v, o=o, z=z, loss=loss, logp=logp, dz=dz, do=do, d=(dq, dk, dv, dS)), [t.float() for t in grads]

    def step(self, number, grads=None):
        from paper_2002_03629_b200 import adamw as aw
        aw.adamw_step(self.params, self.gradients()[1] if grads is None else grads, self.state, number, 0.01, copies=self.copies, **OPT)


def rows():
    at = np.concatenate([[0], np.cumsum(LENS)])
    return [(0, int(a), n) for a, n in zip(at, LENS)]


@pytest.mark.parametrize("dtype,bits", [(torch.float32, 32), (torch.bfloat16, 8)], ids=["f32", "bf16, 8-bit states"])
def test_every_operator_of_a_step_on_what_it_got(dtype, bits):
    p = Program(dtype, bits)
    for number in (1, 2):
        x, grads = p.gradients()
        # linear attention and its gradients
        host = {a: x[a].cpu() for a in ("q", "k", "v", "do")} | {"ld": p.ld.cpu(), "state": None, "dstate": None}
        tla.check_forward(host, x["o"], None, SCALE, rows())
        tla.check_backward(host, x["d"], SCALE, rows())
        assert (x["o"][:, T - BEHIND:] == 0).all() and all((t[:, T - BEHIND:] == 0).all() for t in x["d"][:3])
        # the loss: padding rows give nothing
        tpl.check(x["z"].cpu(), V, p.actions.cpu(), p.old.cpu(), p.adv.cpu(), p.weights.cpu(), None, 0.0, x["loss"].cpu(), x["logp"].cpu(), x["dz"].cpu())
        assert (x["loss"][T - BEHIND:] == 0).all() and (x["dz"][T - BEHIND:] == 0).all()
        # the step; 32-bit states: p within 12 u of the update and 3 u of itself of the 64-bit step (the operator's own tolerance)
        before = [t.cpu().numpy().copy() for t in p.params]
        m, v = (t.float().cpu().numpy().copy() for t in p.state[:2])
        p.step(number, grads)
        at = 0
        for i, (w, g) in enumerate(zip(p.params, grads)):
            n, g = w.numel(), g.cpu().numpy().reshape(-1)
            if bits == 32:
                want, *_ = so.adamw(before[i].reshape(-1), g, m[at:at + n], v[at:at + n], number, 0.01, **OPT)
                moved = np.abs(want - before[i].reshape(-1))
                # (a moment whose terms cancel is off by u of the larger one: its share of the update is below lr / (1 - beta1) in all)
                assert (np.abs(w.cpu().numpy().reshape(-1) - want) <= 12 * U * (moved + 0.1) + 3 * U * (np.abs(want) + moved)).all()
            at += (n + 255) // 256 * 256
            assert not np.array_equal(w.cpu().numpy(), before[i])
            if p.copies is not None:
                assert torch.equal(p.copies[i], w.to(torch.bfloat16))


def loss64(params, p):
    """The whole batch's loss from the weights, in 64 bits, and the gradients in all of them."""
    E, Wq, Wk, Wv, Wo = params
    tok, act = p.tokens.cpu().numpy(), p.actions.cpu().numpy()
    old, adv, w, ld = (t.cpu().double().numpy() for t in (p.old, p.adv, p.weights, p.ld))
    x = E[tok]
    q, k, v = ((x @ W).reshape(T, H, D) for W in (Wq, Wk, Wv))
    o = np.zeros((T, H, D))
    for _, a, n in rows():
        for h in range(H):
            o[a:a + n, h] = so.linear_attention(q[a:a + n, h], k[a:a + n, h], v[a:a + n, h], ld[h], SCALE)[0]
    z = o.reshape(T, H * D) @ Wo
    per = [so.policy_loss(z[i], int(act[i]), old[i], adv[i], w[i]) for i in range(T)]
    dz = np.stack([r[2] for r in per])
    do = (dz @ Wo.T).reshape(T, H, D)
    d = [np.zeros((T, H, D)) for _ in range(3)]
    for _, a, n in rows():
        for h in range(H):
            for t, y in zip(d, so.linear_attention_backward(q[a:a + n, h], k[a:a + n, h], v[a:a + n, h], ld[h], do[a:a + n, h], SCALE)):
                t[a:a + n, h] = y
    d = [t.reshape(T, H * D) for t in d]
    dE = np.zeros_like(E)
    np.add.at(dE, tok, sum(t @ W.T for t, W in zip(d, (Wq, Wk, Wv))))
    return sum(r[0] for r in per), [dE, *(x.T @ t for t in d), o.reshape(T, H * D).T @ dz]


def test_gradients_of_the_whole_program_against_differences():
    """64 bits against central differences of step 1e-5: off by h^2 times a third derivative, and 2^-52 / h of the loss.  The fp32 program against
    64 bits: a chain of four stages, each within (D + 128 + 3 * 5 + 16) u = 191 u = 1.2e-5 of its terms' magnitudes, which exceed a gradient's norm by the
    root of the number of terms of an entry at most where their signs are random: sqrt(64 ... 180) < 14.  4 * 14 * 1.2e-5 = 6.4e-4 of the norm."""
    p = Program(torch.float32, 32, seed=3)
    w = [t.cpu().double().numpy() for t in p.params]
    _, want = loss64(w, p)
    rng, h = np.random.default_rng(0), 1e-5
    for i in range(len(w)):
        step = rng.standard_normal(w[i].shape)
        up, down = ([*w[:i], w[i] + s * h * step, *w[i + 1:]] for s in (1, -1))
        num = (loss64(up, p)[0] - loss64(down, p)[0]) / (2 * h)
        assert abs(num - (want[i] * step).sum()) <= 1e-6 * np.abs(want[i] * step).sum()
    _, got = p.gradients()
    for g, t in zip(got, want):
        assert np.linalg.norm(g.cpu().double().numpy() - t) <= 6.4e-4 * np.linalg.norm(t)


@pytest.mark.parametrize("dtype,bits", [(torch.float32, 32), (torch.bfloat16, 8)], ids=["f32", "bf16, 8-bit states"])
def test_a_captured_step_is_the_eager_one(dtype, bits):
    """The whole step as a CUDA graph, the step's number on the device, replayed: the same bits as eager steps, while the eager program lives on."""
    eager, graphed = Program(dtype, bits, seed=1), Program(dtype, bits, seed=1)
    number = torch.ones(1, dtype=torch.int64, device="cuda")
    keep = [t.clone() for t in (*graphed.params, *(graphed.copies or []), *(s for s in graphed.state if s is not None))]
    graphed.step(number)                                                           # (libraries set up outside the capture)
    for t, c in zip((*graphed.params, *(graphed.copies or []), *(s for s in graphed.state if s is not None)), keep):
        t.view(torch.uint8).copy_(c.view(torch.uint8))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        graphed.step(number)
        number.add_(1)
    number.fill_(1)
    for i in (1, 2, 3):
        eager.step(i)
        graph.replay()
    torch.cuda.synchronize()
    assert int(number) == 4
    for a, b in zip((*eager.params, *(eager.copies or []), *(s for s in eager.state if s is not None)),
                    (*graphed.params, *(graphed.copies or []), *(s for s in graphed.state if s is not None))):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_decoding_from_a_prompt(dtype):
    """Prompts in one call, then token after token: the rollouts' logarithms of probabilities are those of one pass over prompt and tokens."""
    from paper_2002_03629_b200 import linear_attention as la, policy_loss as pl
    p = Program(dtype, 32, seed=2)
    _, q, k, v, o, z = p.forward()
    lens, cut = [n for n in LENS if n > 1], 20                 # the last `cut` steps of each sequence are decoded
    starts = [int(a) for (_, a, n) in rows() if n > 1]
    prompt = torch.cat([torch.arange(a, a + n - cut) for a, n in zip(starts, lens)]).cuda()
    cu = torch.tensor(np.concatenate([[0], np.cumsum([n - cut for n in lens])]), dtype=torch.int32).cuda()
    _, S = la.linear_attention(q[:, prompt], k[:, prompt], v[:, prompt], p.ld, scale=SCALE, cu_seqlens=cu)
    decoded = torch.zeros_like(o)
    for t in range(cut):
        at = torch.tensor([a + n - cut + t for a, n in zip(starts, lens)]).cuda()
        decoded[0, at] = la.linear_attention_step(q[0, at], k[0, at], v[0, at], p.ld, S, scale=SCALE)
    host = {a: x.cpu() for a, x in (("q", q), ("k", k), ("v", v))} | {"ld": p.ld.cpu(), "state": None}
    tail = torch.cat([torch.arange(a + n - cut, a + n) for a, n in zip(starts, lens)])
    mixed = o.clone()
    mixed[0, tail] = decoded[0, tail]
    tla.check_forward(host, mixed, None, SCALE, rows())
    z = (mixed.view(T, H * D).double() @ p.used()[-1]).to(dtype)
    loss, logp, none = pl.policy_loss(z, p.actions, p.old, p.adv, need_grad=False)
    tpl.check(z.cpu(), V, p.actions.cpu(), p.old.cpu(), p.adv.cpu(), torch.full((T,), 1.0 / T), None, 0.0, loss.cpu(), logp.cpu(), None)
