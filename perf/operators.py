"""Performance cases of the operators for training recurrent sequence models: linear attention with a decay for each
head (prompts, gradients, single tokens), the clipped policy loss with its gradient, the AdamW step over many tensors.

A case is one call as a user's program makes it.  ``own`` says which side ``run`` takes: the plain form in elementary
torch operations, or the package's own calls.  ``exact`` computes the same outputs in 64 bits from the definitions.
"""
import math

import numpy as np
import torch

own = False

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
BLOCK = 256            # values of an 8-bit state that share a scale; every tensor's state starts at a multiple of it


def listed():
    return [
        # one sequence of 100 steps in fp32, the recurrent network's setting, through a layer of 8 heads: latency counts
        {"name": "prompt_100", "op": "forward", "dtype": "f32", "lens": "100", "H": 8, "Dk": 64, "Dv": 64, "state": False},
        # a server's batch of prompts of very different lengths that continue from states it holds
        {"name": "prompts_packed", "op": "forward", "dtype": "bf16", "state": True, "H": 16, "Dk": 128, "Dv": 128, "packed": True,
         "lens": "1,2047,333,64,1500,17,900,129,2500,640,41,1100,777,256,1999,5,1300,450,88,2237"},
        # one very long prompt
        {"name": "prompt_long", "op": "forward", "dtype": "bf16", "lens": "65536", "H": 16, "Dk": 128, "Dv": 128, "state": False},
        # gradients of the recurrent network's batch: 592 sequences of 100 steps, 128 units as four heads, fp32
        {"name": "train_100", "op": "backward", "dtype": "f32", "lens": "592x100", "H": 4, "Dk": 32, "Dv": 32, "state": False},
        # gradients of a training batch of long sequences
        {"name": "train_2048", "op": "backward", "dtype": "bf16", "lens": "8x2048", "H": 16, "Dk": 128, "Dv": 128, "state": True},
        # one token of one sequence: nothing but latency
        {"name": "token_1", "op": "step", "dtype": "f32", "B": 1, "H": 8, "Dk": 64, "Dv": 64},
        # one token for each of 256 sequences
        {"name": "tokens_256", "op": "step", "dtype": "bf16", "B": 256, "H": 16, "Dk": 128, "Dv": 128},
        # the 256-way sub-pixels of one sampled 32 x 32 image
        {"name": "policy_image", "op": "policy", "dtype": "f32", "N": 1024, "V": 256, "kl": 0.05},
        # a large batch over an odd number of classes
        {"name": "policy_wide", "op": "policy", "dtype": "bf16", "N": 8192, "V": 50001, "kl": 0.05},
        # the recurrent network's five parameters
        {"name": "adamw_rnn", "op": "adamw", "bits": 32, "tensors": 5, "total": 16769, "copies": False, "grad": "f32"},
        # many tensors of all sizes, gradients in bf16, states in 8 bits, a bf16 copy for the next forward pass
        {"name": "adamw_8bit", "op": "adamw", "bits": 8, "tensors": 300, "total": 50_000_000, "copies": True, "grad": "bf16"},
        # a large model's masters and states in fp32
        {"name": "adamw_32bit", "op": "adamw", "bits": 32, "tensors": 40, "total": 128_000_000, "copies": False, "grad": "f32"},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("forward", "forward", "forward", "backward", "backward", "step", "policy", "policy", "adamw", "adamw"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    if op in ("forward", "backward"):
        Dk = rng.choice((32, 64, 64, 96, 128, 128))
        Dv = rng.choice((Dk, Dk, 32, 64, 128))
        H = rng.choice((1, 2, 4, 8, 16, 32))
        most = (1 << 25 if op == "forward" else 1 << 24) // (H * max(Dk, Dv))
        if dtype == "f32":
            most //= 4
        T = min(most, _log_int(rng, 1, 16384))
        B = min(max(1, most // T), _log_int(rng, 1, 600))
        c = {"op": op, "dtype": dtype, "H": H, "Dk": Dk, "Dv": Dv, "state": rng.random() < 0.5}
        if rng.random() < 0.4:
            c |= {"packed": True, "lens": ",".join(str(_log_int(rng, 1, T)) for _ in range(min(B, 48)))}
        else:
            c["lens"] = "%dx%d" % (B, T)
        return c
    if op == "step":
        return {"op": op, "dtype": dtype, "B": _log_int(rng, 1, 256), "H": rng.choice((1, 4, 8, 16)), "Dk": rng.choice((32, 64, 96, 128)),
                "Dv": rng.choice((32, 64, 96, 128))}
    if op == "policy":
        V = _log_int(rng, 2, 65536)
        return {"op": op, "dtype": dtype, "N": _log_int(rng, 1, max(2, min(65536, (1 << 27) // V))), "V": V, "kl": rng.choice((0.0, 0.05))}
    n = _log_int(rng, 1, 400)
    return {"op": op, "bits": rng.choice((8, 32)), "tensors": n, "total": _log_int(rng, 64 * n, 40_000_000), "copies": rng.random() < 0.5,
            "grad": rng.choice(("f32", "bf16"))}


# ---------------------------------------------------------------- inputs
def _lens(c):
    if "x" in c["lens"]:
        b, t = c["lens"].split("x")
        return [int(t)] * int(b)
    return [int(n) for n in c["lens"].split(",")]


def _sizes(c):
    """Elements of the tensors: the recurrent network's parameters, or sizes spread over three decades."""
    if c["tensors"] == 5 and c["total"] == 16769:
        return [128 * 128, 128, 128, 128, 1]
    r = np.random.RandomState(c["tensors"])
    w = np.exp(r.uniform(0.0, math.log(1000.0), c["tensors"]))
    return [max(1, int(n)) for n in w / w.sum() * c["total"]]


def _decays(H):
    """Logarithms of the decays, from fast heads to slow ones: -2^(-8 (h + 1) / H)."""
    return (-torch.exp2(-8.0 * torch.arange(1, H + 1, dtype=torch.float64) / H)).to(torch.float32).cuda()


def prepare(case, seed):
    c = case
    g = torch.Generator("cuda").manual_seed(seed)

    def normal(*shape, dtype=torch.float32, std=1.0):
        return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)
    if c["op"] in ("forward", "backward"):
        lens, H, Dk, Dv, dt = _lens(c), c["H"], c["Dk"], c["Dv"], DT[c["dtype"]]
        N, packed = len(lens), bool(c.get("packed"))
        B, T = (1, sum(lens)) if packed else (N, lens[0])
        s = {"case": c, "scale": Dk ** -0.5, "ld": _decays(H), "q": normal(B, T, H, Dk, dtype=dt), "k": normal(B, T, H, Dk, dtype=dt),
             "v": normal(B, T, H, Dv, dtype=dt), "state": normal(N, H, Dk, Dv) if c["state"] else None, "cu": None}
        if packed:
            s["cu"] = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32).cuda()
        if c["op"] == "backward":
            s["do"] = normal(B, T, H, Dv, dtype=dt)
            s["dstate"] = normal(N, H, Dk, Dv) if c["state"] else None
        return s
    if c["op"] == "step":
        B, H, Dk, Dv, dt = c["B"], c["H"], c["Dk"], c["Dv"], DT[c["dtype"]]
        return {"case": c, "scale": Dk ** -0.5, "ld": _decays(H), "q": normal(B, H, Dk, dtype=dt), "k": normal(B, H, Dk, dtype=dt),
                "v": normal(B, H, Dv, dtype=dt), "state": normal(B, H, Dk, Dv)}
    if c["op"] == "policy":
        N, V = c["N"], c["V"]
        logits = normal(N, V, dtype=DT[c["dtype"]], std=2.0)
        actions = torch.randint(0, V, (N,), generator=g, device="cuda")
        logp = _logp(logits, actions)
        w = (torch.rand((N,), generator=g, device="cuda") < 0.9).to(torch.float32) / N         # a tenth is padding
        return {"case": c, "logits": logits, "actions": actions, "old": logp + normal(N, std=0.2), "adv": normal(N), "w": w,
                "ref": logp + normal(N, std=0.3) if c["kl"] else None}
    sizes, gd = _sizes(c), DT[c["grad"]]
    total = sum(sizes)
    flat, grads = normal(total, std=0.05), normal(total, dtype=gd, std=0.01)
    padded = sum(_up(n) for n in sizes)
    m, v = normal(padded, std=0.003), (normal(padded, std=0.01) ** 2 + 1e-8)
    live = _live(sizes)
    m, v = m * live, v * live
    s = {"case": c, "flat": flat, "params": list(flat.split(sizes)), "grads": list(grads.split(sizes)), "step": 1000, "lr": 1e-3,
         "betas": (0.9, 0.999), "eps": 1e-8, "wd": 0.01, "scale": torch.full((1,), 0.75, device="cuda"), "copy": None, "copies": None}
    if c["copies"]:
        s["copy"] = torch.empty(total, dtype=torch.bfloat16, device="cuda")
        s["copies"] = list(s["copy"].split(sizes))
    if c["bits"] == 8:
        (mc, ms), (vc, vs) = _cut8(m, seed, 0), _cut8(v.sqrt(), seed, 16)
        s["adam"] = (mc, vc, ms, vs)
    else:
        s["adam"] = (m, v, None, None)
    return s


# ---------------------------------------------------------------- plain forms: linear attention
def _rows(s, back):
    """[N][L] row numbers of each sequence's tokens, in their order or from the last to the first, and which of them exist."""
    lens = _lens(s["case"])
    L = max(lens)
    n = torch.tensor(lens, device="cuda")[:, None]
    t = torch.arange(L, device="cuda")[None, :]
    start = torch.tensor(np.concatenate([[0], np.cumsum(lens)[:-1]]), device="cuda")[:, None]
    return start + torch.where(t < n, n - 1 - t if back else t, 0), t < n


def _recur(q, k, v, ld, S0, late, lens, C=128):
    """o_i = sum_{j<=i} lambda^(i-j) (q_i.k_j) v_j + lambda^(i+late) S0^T q_i for [N][L][H][D] in fp32, in chunks of C tokens;
    and sum_j lambda^(n-1-j) k_j v_j^T + lambda^(n-1+late) S0 for every sequence's length n."""
    N, L, H, Dk = q.shape
    Dv, nc = v.shape[3], (L + C - 1) // C
    e = ld.double()

    def power(n):                                      # lambda^n, [H][...]
        return torch.exp(n.double()[None] * e.view(H, *([1] * n.dim()))).float()

    def chunks(x):
        x = torch.nn.functional.pad(x, (0, 0, 0, 0, 0, nc * C - L))
        return x.view(N, nc, C, H, -1).permute(0, 3, 1, 2, 4)
    i = torch.arange(C, device="cuda")
    far = i[:, None] - i[None, :]
    D = power(far.clamp(min=0)) * (far >= 0)
    qc, kc, vc = chunks(q), chunks(k), chunks(v)
    o = ((qc @ kc.transpose(-1, -2)) * D[:, None]) @ vc
    if nc > 1 or S0 is not None:
        U = (kc * power(C - 1 - i)[None, :, None, :, None]).transpose(-1, -2) @ vc            # every chunk's own sum
        c = torch.arange(nc, device="cuda")
        gap = c[:, None] - c[None, :] - 1
        W = power(C * gap.clamp(min=0)) * (gap >= 0)
        S = (W[None] @ U.reshape(N, H, nc, Dk * Dv)).view(N, H, nc, Dk, Dv)
        del U
        if S0 is not None:                             # lambda^(C c + late - 1) S0 before chunk c, times lambda^(i + 1)
            first = power((C * c[:, None] + i[None, :] + late))                               # [H][nc][C]
            o = o + first[None, :, :, :, None] * (qc @ S0[:, :, None])
        o = o + power(i + 1)[None, :, None, :, None] * (qc @ S)
    o = o.permute(0, 2, 3, 1, 4).reshape(N, nc * C, H, Dv)[:, :L]
    n = torch.tensor(lens, device="cuda")
    left = n[:, None] - 1 - torch.arange(L, device="cuda")[None]                              # [N][L]
    kw = k * (power(left.clamp(min=0)) * (left >= 0)).permute(1, 2, 0)[..., None]
    S = kw.permute(0, 2, 3, 1) @ v.permute(0, 2, 1, 3)
    if S0 is not None:
        S = S + power(n - 1 + late).t()[:, :, None, None] * S0
    return o, S


def _gather(x, rows, live):
    x = x.reshape(-1, *x.shape[2:])
    return x[rows].float() * live[:, :, None, None]


def _scatter(y, rows, live, like):
    out = torch.empty((like.shape[0] * like.shape[1],) + y.shape[2:], dtype=like.dtype, device="cuda")
    out[rows[live]] = y[live].to(like.dtype)
    return out.view(*like.shape[:2], *y.shape[2:])


def _plain_forward(s):
    rows, live = _rows(s, False)
    q, k, v = (_gather(s[n], rows, live) for n in "qkv")
    o, S = _recur(q, k, v, s["ld"], s["state"], 1, _lens(s["case"]))
    return _scatter(o * s["scale"], rows, live, s["v"]), S


def _plain_backward(s):
    lens = _lens(s["case"])
    rows, live = _rows(s, False)
    q, k, v, do = (_gather(s[n], rows, live) for n in ("q", "k", "v", "do"))
    S0 = s["state"].transpose(-1, -2).contiguous() if s["state"] is not None else None
    dq = _scatter(_recur(do, v, k, s["ld"], S0, 1, lens)[0] * s["scale"], rows, live, s["q"])
    rows, live = _rows(s, True)
    q, k, v, do = (_gather(s[n], rows, live) for n in ("q", "k", "v", "do"))
    do = do * s["scale"]
    dS = s["dstate"]
    dv, dS0 = _recur(k, q, do, s["ld"], dS, 0, lens)
    dk, _ = _recur(v, do, q, s["ld"], dS.transpose(-1, -2).contiguous() if dS is not None else None, 0, lens)
    dS0 = dS0 * torch.exp(s["ld"].double()).float()[None, :, None, None]
    return dq, _scatter(dk, rows, live, s["k"]), _scatter(dv, rows, live, s["v"]), dS0


def _plain_step(s):
    S = s["state"]
    S.mul_(torch.exp(s["ld"].double()).float()[None, :, None, None]).add_(s["k"].float()[..., None] * s["v"].float()[:, :, None, :])
    return ((s["q"].float()[..., None] * S).sum(2) * s["scale"]).to(s["v"].dtype), S


# ---------------------------------------------------------------- plain forms: policy loss
CLIP = 0.2


def _logp(logits, actions):
    z = logits.float()
    return z.gather(1, actions[:, None])[:, 0] - torch.logsumexp(z, 1)


def _plain_policy(s):
    z = s["logits"].float()
    top = z.max(1, keepdim=True).values
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    logp = z.gather(1, s["actions"][:, None])[:, 0] - top[:, 0] - torch.log(total[:, 0])
    r = torch.exp(logp - s["old"])
    a, b = r * s["adv"], r.clamp(1 - CLIP, 1 + CLIP) * s["adv"]
    loss = -torch.minimum(a, b)
    g = torch.where(a <= b, -a, 0.0)
    if s["ref"] is not None:
        d = s["ref"] - logp
        loss = loss + s["case"]["kl"] * (torch.expm1(d) - d)
        g = g - s["case"]["kl"] * torch.expm1(d)
    g = g * s["w"]
    dz = e.mul_(-(g / total[:, 0])[:, None])
    dz.scatter_add_(1, s["actions"][:, None], g[:, None])
    return loss * s["w"], logp, dz.to(s["logits"].dtype)


# ---------------------------------------------------------------- plain forms: AdamW
def _up(n):
    return (n + BLOCK - 1) // BLOCK * BLOCK


def _live(sizes):
    """1 where the state belongs to a value, 0 behind a tensor's end."""
    n = torch.tensor([x for k in sizes for x in (k, _up(k) - k)], device="cuda")
    return torch.tensor([1.0, 0.0], device="cuda").repeat(len(sizes)).repeat_interleave(n)


def _bits(n, seed):
    """32 random bits for each place of a state: a mixing of the place's number and the seed."""
    w = 0xFFFFFFFF
    x = (torch.arange(n, dtype=torch.int64, device="cuda") + seed * 0x6A09E667) & w
    x = (x ^ (x >> 16)) * 0x6A09E667 & w
    x = (x ^ (x >> 15)) * 0xBB67AE85 & w
    x = (x ^ (x >> 16)) * 0x3C6EF373 & w
    return x ^ (x >> 15)


def _cut8(x, seed, shift):
    """fp32 values as 8-bit floats (4 exponent bits, 3 of mantissa) in blocks with a power of two as their scale: the largest
    magnitude's power of two lies at 2^7.  A value between two codes takes the upper one with its distance's probability, by 16 random bits."""
    r = (_bits(x.numel(), seed) >> shift) & 0xFFFF
    big = x.view(-1, BLOCK).abs().amax(1)
    scale = (big.view(torch.int32) & 0x7F800000).view(torch.float32) * 2.0 ** -7
    scale = scale.clamp(min=2.0 ** -120)
    y = (x.view(-1, BLOCK) * (1.0 / scale)[:, None]).view(-1)
    a = y.abs()
    high = ((a.view(torch.int32).long() + (r << 4)) >> 20) - (120 << 3)
    low = torch.floor(a * 512.0 + r.float() * 2.0 ** -16).long()
    code = torch.where(a >= 2.0 ** -6, high, low) | torch.where(torch.signbit(y), 128, 0)
    return code.to(torch.uint8).view(torch.float8_e4m3fn), scale


def _value8(code, scale):
    return (code.to(torch.float32).view(-1, BLOCK) * scale[:, None]).view(-1)


def _plain_adamw(s):
    sizes = _sizes(s["case"])
    ends = torch.zeros(BLOCK, device="cuda")

    def spread(ts):
        return torch.cat([x for t, n in zip(ts, sizes) for x in (t.float(), ends[: _up(n) - n])])
    b1, b2 = s["betas"]
    m, v, ms, vs = s["adam"]
    g = spread(s["grads"]) * s["scale"]
    p = spread(s["params"])
    if ms is None:
        m1 = m
        v1 = v
    else:
        m1 = _value8(m, ms)
        v1 = _value8(v, vs)
        v1 = v1 * v1
    m1 = m1 * b1 + g * (1 - b1)
    v1 = v1 * b2 + g * g * (1 - b2)
    p = p * (1 - s["lr"] * s["wd"]) - (m1 * (s["lr"] / (1 - b1 ** s["step"]))) / (v1.sqrt() * (1 / math.sqrt(1 - b2 ** s["step"])) + s["eps"])
    parts = list(p.split([x for n in sizes for x in (n, _up(n) - n)]))[::2]
    torch._foreach_copy_(s["params"], parts)
    if s["copies"] is not None:
        torch._foreach_copy_(s["copies"], parts)
    if ms is None:
        m.copy_(m1)
        v.copy_(v1)
    else:
        root = v1.sqrt()
        mc, mz = _cut8(m1, s["step"], 0)
        vc, vz = _cut8(root, s["step"], 16)
        vc = torch.where((root > 0) & (vc.view(torch.uint8) == 0), 1, vc.view(torch.uint8)).view(torch.float8_e4m3fn)
        m.view(torch.uint8).copy_(mc.view(torch.uint8))
        v.view(torch.uint8).copy_(vc.view(torch.uint8))
        ms.copy_(mz)
        vs.copy_(vz)


# ---------------------------------------------------------------- a pass
def run(state):
    s = state
    op = s["case"]["op"]
    if own:
        from paper_2002_03629_b200 import adamw, linear_attention as la, policy_loss as pl
        if op == "forward":
            o, S = la.linear_attention(s["q"], s["k"], s["v"], s["ld"], scale=s["scale"], state=s["state"], cu_seqlens=s["cu"])
            return {"o": o, "state": S}
        if op == "backward":
            dq, dk, dv, dS0 = la.linear_attention_backward(s["q"], s["k"], s["v"], s["ld"], s["do"], scale=s["scale"], state=s["state"],
                                                           dstate=s["dstate"], cu_seqlens=s["cu"])
            return {"dq": dq, "dk": dk, "dv": dv, "dstate": dS0}
        if op == "step":
            o = la.linear_attention_step(s["q"], s["k"], s["v"], s["ld"], s["state"], scale=s["scale"])
            return {"o": o, "state": s["state"]}
        if op == "policy":
            loss, logp, dz = pl.policy_loss(s["logits"], s["actions"], s["old"], s["adv"], weights=s["w"], ref_logp=s["ref"], clip_low=CLIP,
                                            clip_high=CLIP, kl_coef=s["case"]["kl"])
            return {"loss": loss, "logp": logp, "dlogits": dz}
        adamw.adamw_step(s["params"], s["grads"], s["adam"], s["step"], s["lr"], betas=s["betas"], eps=s["eps"], weight_decay=s["wd"],
                         copies=s["copies"], grad_scale=s["scale"], seed=s["step"])
        return _adamw_out(s)
    if op == "forward":
        o, S = _plain_forward(s)
        return {"o": o, "state": S}
    if op == "backward":
        dq, dk, dv, dS0 = _plain_backward(s)
        return {"dq": dq, "dk": dk, "dv": dv, "dstate": dS0}
    if op == "step":
        o, S = _plain_step(s)
        return {"o": o, "state": S}
    if op == "policy":
        loss, logp, dz = _plain_policy(s)
        return {"loss": loss, "logp": logp, "dlogits": dz}
    _plain_adamw(s)
    return _adamw_out(s)


def _adamw_out(s):
    """Parameters, their bf16 copies and the states (8-bit ones as floats of that type, with their scales)."""
    out = dict(zip(("m", "v", "m_scale", "v_scale"), s["adam"]))
    out["params"], out["copies"] = s["flat"], s["copy"]
    return out


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    c = case
    if c["op"] in ("forward", "backward"):
        lens, size = _lens(c), 2 if c["dtype"] == "bf16" else 4
        rows, Dk, Dv = sum(lens) * c["H"], c["Dk"], c["Dv"]
        state = 4.0 * len(lens) * c["H"] * Dk * Dv
        if c["op"] == "forward":
            return {"bytes": size * rows * (2.0 * Dk + 2 * Dv) + state * (2 if c["state"] else 1), "flops": 4.0 * rows * Dk * Dv}
        return {"bytes": size * rows * (4.0 * Dk + 3 * Dv) + state * (3 if c["state"] else 1), "flops": 10.0 * rows * Dk * Dv}
    if c["op"] == "step":
        rows, Dk, Dv = c["B"] * c["H"], c["Dk"], c["Dv"]
        return {"bytes": rows * (8.0 * Dk * Dv + (2 if c["dtype"] == "bf16" else 4) * (2 * Dk + 2 * Dv)), "flops": 5.0 * rows * Dk * Dv}
    if c["op"] == "policy":
        size = 2 if c["dtype"] == "bf16" else 4
        return {"bytes": c["N"] * (2.0 * size * c["V"] + 8 + 4 * (5 + bool(c["kl"]))), "flops": 6.0 * c["N"] * c["V"]}
    n = sum(_sizes(c))
    one = 8 + (2 if c["grad"] == "bf16" else 4) + (2 if c["copies"] else 0) + (16 if c["bits"] == 32 else 4 + 16 / BLOCK)
    return {"bytes": float(n * one), "flops": 15.0 * n}


# ---------------------------------------------------------------- the definitions in 64 bits
def _exact_rows(lens):
    at = 0
    for i, n in enumerate(lens):
        yield i, at, n
        at += n


def _sum_before(q, k, v, e, step=1024):
    """sum_{j<=i} exp(e (i - j)) (q_i.k_j) v_j for one sequence and head, row by row."""
    n = q.shape[0]
    out = torch.empty((n, v.shape[1]), dtype=torch.float64, device="cuda")
    j = torch.arange(n, device="cuda", dtype=torch.float64)
    for a in range(0, n, step):
        b = min(n, a + step)
        w = torch.exp((j[a:b, None] - j[None, :b]).clamp(min=0) * e)
        out[a:b] = torch.tril((q[a:b] @ k[:b].T) * w, diagonal=a) @ v[:b]
    return out


def _sum_after(q, k, v, e, step=1024):
    """sum_{i>=j} exp(e (i - j)) (q_j.k_i) v_i: row j looks at what comes after it."""
    n = q.shape[0]
    out = torch.empty((n, v.shape[1]), dtype=torch.float64, device="cuda")
    j = torch.arange(n, device="cuda", dtype=torch.float64)
    for a in range(0, n, step):
        b = min(n, a + step)
        w = torch.exp((j[None, a:] - j[a:b, None]).clamp(min=0) * e)
        out[a:b] = torch.triu((q[a:b] @ k[a:].T) * w) @ v[a:]
    return out


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    if c["op"] in ("forward", "backward"):
        lens, H = _lens(c), c["H"]
        pairs = H * sum(float(n) * max(n, 1024) for n in lens)
        if pairs > 1e11 or H * len(lens) > 6000:
            return None
        x = {n: s[n].reshape(-1, H, s[n].shape[3]).double() for n in ("q", "k", "v", "do") if n in s}
        S0, dS = (s[n].double() if s.get(n) is not None else None for n in ("state", "dstate"))
        ld, scale = s["ld"].double().tolist(), s["scale"]
        like = {n: torch.empty_like(x[n]) for n in x}
        S = torch.empty((len(lens), H, c["Dk"], c["Dv"]), dtype=torch.float64, device="cuda")
        for i, at, n in _exact_rows(lens):
            t = torch.arange(n, device="cuda", dtype=torch.float64)[:, None]
            for h in range(H):
                e = ld[h]
                q, k, v = (x[a][at:at + n, h] for a in "qkv")
                if c["op"] == "forward":
                    o = _sum_before(q, k, v, e)
                    S[i, h] = (k * torch.exp(e * (n - 1 - t))).T @ v
                    if S0 is not None:
                        o += torch.exp(e * (t + 1)) * (q @ S0[i, h])
                        S[i, h] += math.exp(e * n) * S0[i, h]
                    like["v"][at:at + n, h] = o * scale
                else:
                    do = x["do"][at:at + n, h] * scale
                    dq, dk, dv = _sum_before(do, v, k, e), _sum_after(v, do, q, e), _sum_after(k, q, do, e)
                    S[i, h] = (q * torch.exp(e * (t + 1))).T @ do
                    if S0 is not None:
                        dq += torch.exp(e * (t + 1)) * (do @ S0[i, h].T)
                    if dS is not None:
                        dk += torch.exp(e * (n - 1 - t)) * (v @ dS[i, h].T)
                        dv += torch.exp(e * (n - 1 - t)) * (k @ dS[i, h])
                        S[i, h] += math.exp(e * n) * dS[i, h]
                    for name, y in (("q", dq), ("k", dk), ("v", dv)):
                        like[name][at:at + n, h] = y
        shaped = {n: like[n].view(*s[n].shape[:2], H, -1) for n in like}
        if c["op"] == "forward":
            return {"o": shaped["v"], "state": S}
        return {"dq": shaped["q"], "dk": shaped["k"], "dv": shaped["v"], "dstate": S}
    if c["op"] == "step":
        S = torch.exp(s["ld"].double()).view(1, -1, 1, 1) * s["state"].double() + torch.einsum("bhi,bhj->bhij", s["k"].double(), s["v"].double())
        return {"o": torch.einsum("bhi,bhij->bhj", s["q"].double(), S) * s["scale"], "state": S}
    if c["op"] == "policy":
        loss, logp, dz = [], [], torch.empty(s["logits"].shape, dtype=torch.float64, device="cuda")
        for a in range(0, c["N"], 1024):
            cut = slice(a, a + 1024)
            lp = torch.log_softmax(s["logits"][cut].double(), 1)
            act = s["actions"][cut, None]
            mine, A, w = lp.gather(1, act)[:, 0], s["adv"][cut].double(), s["w"][cut].double()
            ratio = torch.exp(mine - s["old"][cut].double())
            free = ratio * A
            held = torch.minimum(torch.maximum(ratio, torch.tensor(1 - CLIP, dtype=torch.float64, device="cuda")),
                                 torch.tensor(1 + CLIP, dtype=torch.float64, device="cuda")) * A
            value, slope = -torch.where(free <= held, free, held), torch.where(free <= held, -free, torch.zeros_like(free))
            if s["ref"] is not None:
                d = s["ref"][cut].double() - mine
                value, slope = value + c["kl"] * (torch.exp(d) - d - 1), slope + c["kl"] * (1 - torch.exp(d))
            one = torch.zeros_like(lp).scatter_(1, act, 1.0)
            dz[cut] = (w * slope)[:, None] * (one - torch.exp(lp))
            loss.append(w * value)
            logp.append(mine)
        return {"loss": torch.cat(loss), "logp": torch.cat(logp), "dlogits": dz}
    b1, b2 = s["betas"]
    t, lr = s["step"], s["lr"]
    m, v, ms, vs = s["adam"]
    params = torch.empty(s["flat"].numel(), dtype=torch.float64, device="cuda")
    m2, v2 = (torch.zeros(m.numel(), dtype=torch.float64, device="cuda") for _ in range(2))
    at = to = 0
    for p, g in zip(s["params"], s["grads"]):
        n = p.numel()
        mi, vi = m[to:to + n].double(), v[to:to + n].double()
        if ms is not None:
            cut = slice(to // BLOCK, (to + _up(n)) // BLOCK)
            mi = mi * ms[cut].double().repeat_interleave(BLOCK)[:n]
            vi = (vi * vs[cut].double().repeat_interleave(BLOCK)[:n]) ** 2
        gi = g.double() * 0.75
        mi, vi = b1 * mi + (1 - b1) * gi, b2 * vi + (1 - b2) * gi * gi
        params[at:at + n] = (1 - lr * s["wd"]) * p.double() - lr * (mi / (1 - b1 ** t)) / (torch.sqrt(vi / (1 - b2 ** t)) + s["eps"])
        m2[to:to + n], v2[to:to + n] = mi, vi
        at, to = at + n, to + _up(n)
    eight = ms is not None                  # what the 8-bit states hold goes by random roundings: no value of its own
    return {"m": None if eight else m2, "v": None if eight else v2, "m_scale": None, "v_scale": None, "params": params,
            "copies": None if s["copy"] is None else params}
