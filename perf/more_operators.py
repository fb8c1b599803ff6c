"""Workloads of the operators around the gated block: the matrix product with bias, activation and residual in its
epilogue, the layer norm with its weight gradients, and the cross entropy over a vocabulary, each for K local workers
with weights of their own.

`own` selects between the plain form (elementary torch operations in 32 bits, rounded once) and the package's kernels.
Sizes: width 768 and 256 (inner 1024), vocabularies 50257 and 8192 are those of the GPT-Neo-125M and GPT-Neo-8M shaped
tensor lists of `workloads`; the others are generic.
"""
import math
import random

import torch

own = False

GROUP = 32                                   # values per exponent of an 8-bit checkpoint
EPS = 1e-5
ACTS = ("none", "silu", "gelu", "gelu_tanh", "relu")


def listed():
    return [
        # one token of one replica being sampled from: the weights are read once, launch latency counts
        dict(name="linear_fwd_one", op="linear_fwd", dtype="bf16", K=1, M=1, D=2048, N=5632, act="gelu_tanh", save="none",
             bias=True, residual=False),
        # a short last batch in fp32: ragged token count, odd output size, everything in the epilogue
        dict(name="linear_fwd_small", op="linear_fwd", dtype="fp32", K=4, M=17, D=256, N=683, act="gelu", save="full",
             bias=True, residual=True),
        # first product of the plain feed-forward block, eight workers, its pre-activation kept in 8 bits
        dict(name="linear_fwd_mid_8bit", op="linear_fwd", dtype="bf16", K=8, M=1024, D=768, N=2048, act="gelu_tanh",
             save="8bit", bias=True, residual=False),
        # second product of a wide model's block, added to the residual stream: the largest forward
        dict(name="linear_fwd_large", op="linear_fwd", dtype="bf16", K=2, M=8192, D=5632, N=2048, act="none", save="none",
             bias=True, residual=True),
        # the backward pass of the 125M-shaped model's second product: no activation, gradient of the bias
        dict(name="linear_bwd_mid", op="linear_bwd", dtype="bf16", K=8, M=1024, D=2048, N=768, act="none", save="none",
             bias=True, residual=False),
        # the 8M-shaped model's first product in fp32
        dict(name="linear_bwd_fp32", op="linear_bwd", dtype="fp32", K=8, M=500, D=256, N=1024, act="gelu", save="full",
             bias=True, residual=False),
        # a wide model's first product: the largest backward
        dict(name="linear_bwd_large", op="linear_bwd", dtype="bf16", K=2, M=8192, D=2048, N=5632, act="gelu_tanh",
             save="full", bias=True, residual=False),
        # a short ragged batch in fp32, rows that start anywhere
        dict(name="norm_fwd_small", op="norm_fwd", dtype="fp32", K=3, M=77, D=257, residual=False),
        # a block's entry in the 125M-shaped model: residual stream and branch added, then normed
        dict(name="norm_fwd_mid", op="norm_fwd", dtype="bf16", K=8, M=2048, D=768, residual=True),
        # its backward pass in a wide model with long batches, the residual stream's gradient added in
        dict(name="norm_bwd_large", op="norm_bwd", dtype="bf16", K=2, M=32768, D=2048, residual=True),
        # the loss of a small model's batch in fp32
        dict(name="loss_fwd_small", op="loss_fwd", dtype="fp32", K=4, M=64, V=8192),
        # gradient of the logits over the 125M-shaped model's vocabulary (odd: rows start anywhere)
        dict(name="loss_bwd_large", op="loss_bwd", dtype="bf16", K=8, M=512, V=50257),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    op = rng.choice(["linear_fwd", "linear_bwd", "linear_fwd", "linear_bwd", "norm_fwd", "norm_bwd", "loss_fwd", "loss_bwd"])
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    half = 1 if dtype == "bf16" else 2
    while True:
        if op.startswith("linear"):
            even = rng.random() < 0.6                        # most models' sizes are multiples of 8, some are not
            D, N, M = _log(rng, 64, 5632), _log(rng, 64, 5632), _log(rng, 1, 8192)
            if even:
                D, N = (D + 7) // 8 * 8, (N + 7) // 8 * 8
            act = rng.choice(ACTS)
            save = "none" if act == "none" else rng.choice(["full", "8bit"])
            if op == "linear_fwd" and rng.random() < 0.3:
                save = "none"                                # evaluation: nothing is kept
            c = dict(op=op, dtype=dtype, K=rng.randint(1, 8), M=M, D=D, N=N, act=act, save=save, bias=rng.random() < 0.8,
                     residual=op == "linear_fwd" and rng.random() < 0.4)
            if c["K"] * M * D * N <= 2 * 8192 * 2048 * 5632 // (1 if dtype == "bf16" else 8):
                return c
        elif op.startswith("norm"):
            even = rng.random() < 0.7
            D = _log(rng, 16, 8192)
            if even:
                D = (D + 7) // 8 * 8
            c = dict(op=op, dtype=dtype, K=rng.randint(1, 8), M=_log(rng, 1, 32768), D=D, residual=rng.random() < 0.5)
            if c["K"] * c["M"] * D <= 2 * 32768 * 2048 // half:
                return c
        else:
            V = rng.choice([50257, 8192, _log(rng, 2, 65536), _log(rng, 2, 65536)])
            c = dict(op=op, dtype=dtype, K=rng.randint(1, 8), M=_log(rng, 1, 8192), V=V)
            if c["K"] * c["M"] * V <= 8 * 512 * 50257 // half:
                return c


# ------------------------------------------------------------------------------------------------ inputs

def _dtype(case):
    return torch.float32 if case["dtype"] == "fp32" else torch.bfloat16


def _randn(gen, *shape, std=1.0):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32).mul_(std)


def _groups(x):
    """x (..., C) as (..., groups, 32), zeros behind the end."""
    C = x.shape[-1]
    G = (C + GROUP - 1) // GROUP
    pad = torch.zeros(*x.shape[:-1], G * GROUP, dtype=x.dtype, device=x.device)
    pad[..., :C] = x
    return pad.view(*x.shape[:-1], G, GROUP)


def _pack(x):
    """The 8-bit form of x: (q int8 (..., C), exponent uint8 (..., groups)), elementary operations in 32 bits."""
    g = _groups(x.float())
    amax = g.abs().amax(-1)
    E = (((amax.view(torch.int32) + 0x10000) >> 23) - 6).clamp_min(1)
    q = torch.round(g * ((254 - E) << 23).view(torch.float32)[..., None])
    return q.to(torch.int8).flatten(-2)[..., :x.shape[-1]].contiguous(), E.to(torch.uint8)


def _value(q, E):
    """The 32-bit values that an 8-bit checkpoint stands for."""
    s = (E.to(torch.int32) << 23).view(torch.float32)
    return (_groups(q.float()) * s[..., None]).flatten(-2)[..., :q.shape[-1]]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 17)
    op, dt, s = case["op"], _dtype(case), dict(case=dict(case))
    K, M = case["K"], case["M"]
    if op.startswith("linear"):
        D, N = case["D"], case["N"]
        x = _randn(gen, K, M, D)
        x *= 1 + 7 * (_randn(gen, D) > 2.3)                  # a few loud channels, as behind a trained norm
        s["x"], s["w"] = x.to(dt), _randn(gen, K, N, D, std=D ** -0.5).to(dt)
        if op == "linear_fwd":
            s["bias"] = _randn(gen, K, N, std=0.2).to(dt) if case["bias"] else None
            s["residual"] = _randn(gen, K, M, N, std=2.0).to(dt) if case["residual"] else None
        else:
            s["dy"] = _randn(gen, K, M, N, std=1e-2).to(dt)
            if case["save"] != "none":
                z = _randn(gen, K, M, N, std=1.5).to(dt)
                s["z"] = z if case["save"] == "full" else _pack(z)
                if case["save"] == "8bit":
                    s["x"] = _pack(s["x"])
    elif op.startswith("norm"):
        D = case["D"]
        x = _randn(gen, K, M, D, std=1.5) + _randn(gen, D, std=0.5)      # channels with a mean of their own
        x *= 1 + 9 * (_randn(gen, D) > 2.5)
        s["w"] = (1 + _randn(gen, K, D, std=0.1)).to(dt)
        if op == "norm_fwd":
            s["x"], s["b"] = x.to(dt), _randn(gen, K, D, std=0.1).to(dt)
            s["residual"] = _randn(gen, K, M, D).to(dt) if case["residual"] else None
        else:
            s["x"], s["dy"] = x.to(dt), _randn(gen, K, M, D, std=1e-2).to(dt)
            s["dtotal"] = _randn(gen, K, M, D, std=1e-2).to(dt) if case["residual"] else None
            h = s["x"].float()
            s["mean"] = h.mean(-1)
            s["rstd"] = torch.rsqrt((h - s["mean"][..., None]).square().mean(-1) + EPS)
    else:
        V = case["V"]
        logits = _randn(gen, K, M, V, std=2.0)
        t = torch.randint(0, V, (K, M), generator=gen, device="cuda")
        logits.scatter_add_(2, t[..., None], 4 * torch.rand(K, M, 1, generator=gen, device="cuda"))   # some are learnt
        pad = torch.rand(K, M, generator=gen, device="cuda") < 0.1       # the ends of padded sequences count for nothing
        s["logits"], s["targets"] = logits.to(dt), torch.where(pad, -1, t).to(torch.int32)
        if op == "loss_bwd":
            count = (~pad).sum(-1, keepdim=True).clamp_min(1)
            s["dloss"] = (torch.ones(K, M, device="cuda") / count).contiguous()
            z = s["logits"].float()
            top = z.amax(-1)
            s["lse"] = torch.log(torch.exp(z - top[..., None]).sum(-1)) + top
    return s


# ------------------------------------------------------------------------------------------------ plain form

def _act(name, g):
    """(act(g), act'(g)) in g's precision."""
    if name == "none":
        return g, torch.ones_like(g)
    if name == "silu":
        sg = 1 / (1 + torch.exp(-g))
        return g * sg, sg * (1 + g * (1 - sg))
    if name == "gelu":
        cdf = 0.5 * (1 + torch.erf(g * 0.5 ** 0.5))
        return g * cdf, cdf + g * torch.exp(-0.5 * g * g) * (2 * math.pi) ** -0.5
    if name == "gelu_tanh":
        c = (2 / math.pi) ** 0.5
        t = torch.tanh(c * (g + 0.044715 * g * g * g))
        return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * c * (1 + 3 * 0.044715 * g * g)
    return torch.where(g > 0, g, torch.zeros_like(g)), (g > 0).to(g.dtype)


def _plain(s):
    case = s["case"]
    op, dt = case["op"], _dtype(case)
    if op == "linear_fwd":
        z = s["x"].float() @ s["w"].float().mT
        if s["bias"] is not None:
            z = z + s["bias"].float()[:, None]
        y = _act(case["act"], z)[0]
        if s["residual"] is not None:
            y = y + s["residual"].float()
        out = {"y": y.to(dt)}
        if case["save"] == "full":
            out["z"] = z.to(dt)
        elif case["save"] == "8bit":                         # eight significant bits: exact in bf16
            out["z"] = _value(*_pack(z)).to(torch.bfloat16)
        return out
    if op == "linear_bwd":
        x, w, dz = _value(*s["x"]) if case["save"] == "8bit" else s["x"].float(), s["w"].float(), s["dy"].float()
        if case["save"] != "none":
            dz = dz * _act(case["act"], s["z"].float() if case["save"] == "full" else _value(*s["z"]))[1]
        out = {"dx": (dz @ w).to(dt), "dw": (dz.mT @ x).to(dt)}
        if case["bias"]:
            out["dbias"] = dz.sum(1).to(dt)
        return out
    if op == "norm_fwd":
        h = s["x"].float()
        if s["residual"] is not None:
            h = h + s["residual"].float()
        mean = h.mean(-1)
        c = h - mean[..., None]
        rstd = torch.rsqrt((c * c).mean(-1) + EPS)
        y = c * rstd[..., None] * s["w"].float()[:, None] + s["b"].float()[:, None]
        out = {"y": y.to(dt), "mean": mean, "rstd": rstd}
        if s["residual"] is not None:
            out["total"] = h.to(dt)
        return out
    if op == "norm_bwd":
        r, dy = s["rstd"][..., None], s["dy"].float()
        xh = (s["x"].float() - s["mean"][..., None]) * r
        g = dy * s["w"].float()[:, None]
        dx = r * (g - g.mean(-1, keepdim=True) - xh * (g * xh).mean(-1, keepdim=True))
        if s["dtotal"] is not None:
            dx = dx + s["dtotal"].float()
        return {"dx": dx.to(dt), "dw": (dy * xh).sum(1).to(dt), "db": dy.sum(1).to(dt)}
    z, t = s["logits"].float(), s["targets"].long()
    counts = t >= 0
    if op == "loss_fwd":
        top = z.amax(-1)
        lse = torch.log(torch.exp(z - top[..., None]).sum(-1)) + top
        at = z.gather(-1, t.clamp_min(0)[..., None])[..., 0]
        return {"loss": torch.where(counts, lse - at, torch.zeros_like(lse)), "lse": lse}
    p = torch.exp(z - s["lse"][..., None])
    p.scatter_add_(-1, t.clamp_min(0)[..., None], torch.full_like(p[..., :1], -1.0))
    return {"dlogits": (p * torch.where(counts, s["dloss"], torch.zeros_like(s["dloss"]))[..., None]).to(dt)}


# ------------------------------------------------------------------------------------------------ the package's kernels

def _own(s):
    import paper_2504_18454_b200 as P
    case = s["case"]
    op, dt = case["op"], _dtype(case)
    if op.startswith("linear"):
        act = dict(none=P.ACT_NONE, silu=P.ACT_SILU, gelu=P.ACT_GELU, gelu_tanh=P.ACT_GELU_TANH, relu=P.ACT_RELU)[case["act"]]
        if op == "linear_fwd":
            save = dict(none=P.SAVE_NONE, full=P.SAVE_FULL)[case["save"]] if case["save"] != "8bit" else P.SAVE_8BIT
            y, z = P.linear_forward(s["x"], s["w"], s["bias"], s["residual"], activation=act, save=save)
            if case["save"] == "none":
                return {"y": y}
            return {"y": y, "z": z if case["save"] == "full" else P.act8_unpack(z, dtype=torch.bfloat16)}
        z, x = s.get("z"), s["x"]
        if case["save"] == "8bit":
            z, x = P.Act8(*z, dt), P.Act8(*x, dt)
        dx, dw, dbias = P.linear_backward(s["dy"], x, s["w"], z, activation=act, need_dbias=case["bias"])
        return {"dx": dx, "dw": dw, "dbias": dbias} if case["bias"] else {"dx": dx, "dw": dw}
    if op == "norm_fwd":
        y, total, mean, rstd = P.layer_norm_forward(s["x"], s["w"], s["b"], s["residual"], eps=EPS)
        out = {"y": y, "mean": mean, "rstd": rstd}
        if case["residual"]:
            out["total"] = total
        return out
    if op == "norm_bwd":
        dx, dw, db = P.layer_norm_backward(s["dy"], s["x"], s["w"], s["mean"], s["rstd"], s["dtotal"])
        return {"dx": dx, "dw": dw, "db": db}
    if op == "loss_fwd":
        loss, lse = P.cross_entropy_forward(s["logits"], s["targets"])
        return {"loss": loss, "lse": lse}
    return {"dlogits": P.cross_entropy_backward(s["dloss"], s["logits"], s["targets"], s["lse"])}


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------------------------------------ what a pass needs

def work(case):
    b = 4 if case["dtype"] == "fp32" else 2
    K, M = case["K"], case["M"]
    if case["op"].startswith("linear"):
        D, N = case["D"], case["N"]
        eight = lambda c: c + (c + GROUP - 1) // GROUP       # bytes of a row of c values in 8 bits
        vec = K * N * b if case["bias"] else 0
        z = {"none": 0, "full": K * M * N * b, "8bit": K * M * eight(N)}[case["save"]]
        if case["op"] == "linear_fwd":
            back = K * M * (eight(N) + 2 * N) if case["save"] == "8bit" else 0       # and the values read back
            return {"bytes": K * (M * D + N * D + M * N * (2 if case["residual"] else 1)) * b + vec + z + back,
                    "flops": 2 * K * M * D * N}
        x = K * M * (eight(D) if case["save"] == "8bit" else D * b)
        return {"bytes": K * (M * N + 2 * N * D + M * D) * b + x + vec + z, "flops": 4 * K * M * D * N}
    if case["op"].startswith("norm"):
        D = case["D"]
        n = K * M * D
        if case["op"] == "norm_fwd":
            return {"bytes": n * b * (4 if case["residual"] else 2) + 8 * K * M + 2 * K * D * b, "flops": 8 * n}
        return {"bytes": n * b * (4 if case["residual"] else 3) + 8 * K * M + 3 * K * D * b, "flops": 14 * n}
    n = K * M * case["V"]
    if case["op"] == "loss_fwd":
        return {"bytes": n * b + 12 * K * M, "flops": 4 * n}
    return {"bytes": 2 * n * b + 12 * K * M, "flops": 4 * n}


# ------------------------------------------------------------------------------------------------ 64 bits

def _exact8(x):
    """The values of the 8-bit form of x by its definition: the smallest power of two with rint(|x| / step) <= 127."""
    C = x.shape[-1]
    t = torch.nn.functional.pad(x, (0, -C % GROUP)).unflatten(-1, (-1, GROUP))
    top = t.abs().amax(-1, keepdim=True)
    e = torch.frexp(top)[1].double() - 7                     # top = m 2^(e + 7), 1/2 <= m < 1: top / 2^e in 64 .. 128
    e = e + (torch.round(top * torch.exp2(-e)) > 127)
    step = torch.exp2(e.clamp_min(-126.0))
    return (torch.round(t / step) * step).flatten(-2)[..., :C]


def exact(case, seed):
    s = prepare(case, seed)
    op, d, K = case["op"], torch.float64, case["K"]
    name = case.get("act")

    def act(g):
        if name == "none":
            return g
        if name == "silu":
            return g * torch.sigmoid(g)
        if name == "relu":
            return g.clamp_min(0)
        if name == "gelu":
            return g * torch.special.ndtr(g)
        return g * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3))

    def slope(g):
        g = g.detach().requires_grad_()
        return torch.autograd.grad(act(g).sum(), g)[0]

    def read(t, k):                                          # a tensor's values, or those of an 8-bit checkpoint
        if torch.is_tensor(t):
            return t[k].to(d)
        q, E = t
        return q[k].to(d) * torch.exp2(E[k].to(d) - 127).repeat_interleave(GROUP, -1)[..., :q.shape[-1]]

    outs = []
    for k in range(K):                                       # one worker at a time: 64-bit copies of one replica only
        if op == "linear_fwd":
            z = torch.einsum("md,nd->mn", s["x"][k].to(d), s["w"][k].to(d))
            z = z + (s["bias"][k].to(d) if case["bias"] else 0.0)
            o = {"y": act(z) + (s["residual"][k].to(d) if case["residual"] else 0.0)}
            if case["save"] != "none":
                o["z"] = z if case["save"] == "full" else _exact8(z)
        elif op == "linear_bwd":
            dz = s["dy"][k].to(d) * (slope(read(s["z"], k)) if case["save"] != "none" else 1.0)
            o = {"dx": torch.einsum("mn,nd->md", dz, s["w"][k].to(d)), "dw": torch.einsum("mn,md->nd", dz, read(s["x"], k))}
            if case["bias"]:
                o["dbias"] = torch.einsum("mn->n", dz)
        elif op == "norm_fwd":
            h = s["x"][k].to(d) + (s["residual"][k].to(d) if case["residual"] else 0.0)
            var, mean = torch.var_mean(h, -1, correction=0, keepdim=True)
            r = 1 / torch.sqrt(var + EPS)
            o = {"y": torch.addcmul(s["b"][k].to(d), (h - mean) * r, s["w"][k].to(d)), "mean": mean[:, 0], "rstd": r[:, 0]}
            if case["residual"]:
                o["total"] = h
        elif op == "norm_bwd":
            r, dy = s["rstd"][k].to(d)[:, None], s["dy"][k].to(d)
            xh = (s["x"][k].to(d) - s["mean"][k].to(d)[:, None]) * r
            D = xh.shape[-1]
            g = dy * s["w"][k].to(d)
            along = torch.einsum("md,md->m", g, xh)[:, None]
            o = {"dx": r / D * (D * g - g.sum(-1, keepdim=True) - xh * along), "dw": torch.einsum("md,md->d", dy, xh),
                 "db": torch.einsum("md->d", dy)}
            if case["residual"]:
                o["dx"] = o["dx"] + s["dtotal"][k].to(d)
        else:
            z, t = s["logits"][k].to(d), s["targets"][k].long()
            on = (t >= 0).to(d)
            hot = torch.zeros_like(z)
            hot[torch.arange(len(t), device=t.device), t.clamp_min(0)] = 1.0
            if op == "loss_fwd":
                lse = torch.logsumexp(z, -1)
                o = {"loss": on * (lse - (z * hot).sum(-1)), "lse": lse}
            else:
                p = torch.exp(z - s["lse"][k].to(d)[:, None])
                o = {"dlogits": (p - hot) * (on * s["dloss"][k].to(d))[:, None]}
        outs.append(o)
    return {n: torch.stack([o[n] for o in outs]) for n in outs[0]}
