"""Workloads of the block operators: the gated feed-forward block, 8-bit activation checkpoints and the
query/key norm with position rotation, each for K local workers with weights of their own.

`own` selects between the plain form (elementary torch operations in 32 bits, rounded once) and the package's
kernels.  Sizes: d_model 768 and 256 (d_ff 1024) are those of the GPT-Neo-125M and GPT-Neo-8M shaped tensor lists of
`workloads`; the others are generic.
"""
import math
import random

import torch

own = False

GROUP = 32                                   # values per exponent of an 8-bit checkpoint
ACTS = ("silu", "gelu", "gelu_tanh", "relu")


def listed():
    return [
        # a short last batch of a small model: a ragged token count, an odd hidden size, launch latency counts
        dict(name="ffn_fwd_small", op="ffn_fwd", dtype="bf16", K=4, M=17, D=256, F=683, act="silu", save="full"),
        # one micro-batch of the 125M-shaped model, eight workers, activations kept in 8 bits
        dict(name="ffn_fwd_mid_8bit", op="ffn_fwd", dtype="bf16", K=8, M=1024, D=768, F=2048, act="silu", save="8bit"),
        # its backward pass with gate and up kept in full
        dict(name="ffn_bwd_mid", op="ffn_bwd", dtype="bf16", K=8, M=1024, D=768, F=2048, act="silu", save="full"),
        # the 8M-shaped model in fp32, with the other activation
        dict(name="ffn_bwd_fp32", op="ffn_bwd", dtype="fp32", K=8, M=500, D=256, F=1024, act="gelu", save="full"),
        # a wide model with few workers: the largest forward
        dict(name="ffn_fwd_large", op="ffn_fwd", dtype="bf16", K=2, M=8192, D=2048, F=5632, act="gelu_tanh", save="full"),
        # its backward pass from 8-bit checkpoints of the input, gate and up
        dict(name="ffn_bwd_large_8bit", op="ffn_bwd", dtype="bf16", K=2, M=8192, D=2048, F=5632, act="silu", save="8bit"),
        # a small activation with rows that end inside a group: write the checkpoint, read it back
        dict(name="act8_small", op="act8", dtype="fp32", rows=37, cols=257),
        # a block's hidden activations of one step: write the checkpoint, read it back
        dict(name="act8_large", op="act8", dtype="bf16", rows=32768, cols=5632),
        # a short ragged batch in fp32 with grouped key heads
        dict(name="qk_fwd_small", op="qk_fwd", dtype="fp32", K=3, M=77, HQ=6, HK=2, DH=40, R=40, interleaved=True),
        # the 125M-shaped model's heads, eight workers, out of one fused projection
        dict(name="qk_fwd_mid", op="qk_fwd", dtype="bf16", K=8, M=2048, HQ=12, HK=12, DH=64, R=64, interleaved=False),
        dict(name="qk_bwd_mid", op="qk_bwd", dtype="bf16", K=8, M=2048, HQ=12, HK=12, DH=64, R=64, interleaved=False),
        # long sequences, wide heads, grouped key heads, half of the head rotated
        dict(name="qk_bwd_large", op="qk_bwd", dtype="bf16", K=2, M=32768, HQ=16, HK=4, DH=128, R=64, interleaved=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    op = rng.choice(["ffn_fwd", "ffn_bwd", "ffn_fwd", "ffn_bwd", "act8", "qk_fwd", "qk_bwd"])
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    if op.startswith("ffn"):
        while True:
            even = rng.random() < 0.6                        # most models' sizes are multiples of 8, some are not
            D, F, M = _log(rng, 64, 2048), _log(rng, 64, 5632), _log(rng, 1, 8192)
            if even:
                D, F = (D + 7) // 8 * 8, (F + 7) // 8 * 8
            c = dict(op=op, dtype=dtype, K=rng.randint(1, 8), M=M, D=D, F=F, act=rng.choice(ACTS),
                     save=rng.choice(["full", "8bit"]))
            most = 2 * 8192 * 2048 * 5632 // (1 if dtype == "bf16" else 8)
            if c["K"] * M * D * F <= most:
                return c
    if op == "act8":
        while True:
            c = dict(op=op, dtype=dtype, rows=_log(rng, 1, 65536), cols=_log(rng, 1, 16384))
            if c["rows"] * c["cols"] <= 32768 * 5632 // (1 if dtype == "bf16" else 2):
                return c
    while True:
        DH = rng.choice([8, 16, 24, 32, 40, 64, 80, 96, 128, 128, 160, 192, 256])
        HK = rng.randint(1, 8)
        c = dict(op=op, dtype=dtype, K=rng.randint(1, 8), M=_log(rng, 1, 32768), HQ=HK * rng.choice([1, 2, 3, 4]), HK=HK,
                 DH=DH, R=DH if rng.random() < 0.6 else 2 * rng.randint(1, DH // 2), interleaved=rng.random() < 0.4)
        if c["K"] * c["M"] * (c["HQ"] + HK) * DH <= 2 * 32768 * 20 * 128 // (1 if dtype == "bf16" else 2):
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
    bits = amax.view(torch.int32)
    E = (((bits + 0x10000) >> 23) - 6).clamp_min(1)
    E = torch.where(torch.isfinite(amax), E, torch.full_like(E, 255))
    inv = ((254 - E.clamp_max(254)) << 23).view(torch.float32)
    q = torch.where((E == 255)[..., None], torch.zeros_like(g), torch.round(g * inv[..., None]))
    return q.to(torch.int8).flatten(-2)[..., :x.shape[-1]].contiguous(), E.to(torch.uint8)


def _value(q, E):
    """The 32-bit values that an 8-bit checkpoint stands for."""
    s = torch.where(E == 255, torch.full_like(E, 0, dtype=torch.float32).fill_(float("nan")),
                    (E.to(torch.int32) << 23).view(torch.float32))
    return (_groups(q.float()) * s[..., None]).flatten(-2)[..., :q.shape[-1]]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 13)
    op, dt, s = case["op"], _dtype(case), dict(case=dict(case))
    if op.startswith("ffn"):
        K, M, D, F = (case[n] for n in ("K", "M", "D", "F"))
        x = _randn(gen, K, M, D)
        x *= 1 + 7 * (_randn(gen, D) > 2.3)                  # a few loud channels, as behind a trained norm
        s["wg"] = _randn(gen, K, F, D, std=D ** -0.5).to(dt)
        s["wu"] = _randn(gen, K, F, D, std=D ** -0.5).to(dt)
        s["wd"] = _randn(gen, K, D, F, std=F ** -0.5).to(dt)
        s["x"] = x.to(dt)
        if op == "ffn_bwd":
            s["dy"] = _randn(gen, K, M, D, std=1e-2).to(dt)
            g, u = _randn(gen, K, M, F, std=1.5).to(dt), _randn(gen, K, M, F, std=1.5).to(dt)
            if case["save"] == "full":
                s["g"], s["u"] = g, u
            else:
                s["g"], s["u"], s["x"] = _pack(g), _pack(u), _pack(s["x"])
    elif op == "act8":
        x = _randn(gen, case["rows"], case["cols"])
        x *= torch.exp(_randn(gen, case["rows"], 1))         # rows of different loudness
        s["x"] = x.to(dt)
    else:
        K, M, HQ, HK, DH, R = (case[n] for n in ("K", "M", "HQ", "HK", "DH", "R"))
        qkv = _randn(gen, K, M, HQ + 2 * HK, DH).to(dt)      # one fused projection; q and k are views of it
        s["q"], s["k"] = qkv[:, :, :HQ], qkv[:, :, HQ:HQ + HK]
        s["wq"], s["wk"] = (1 + _randn(gen, K, DH, std=0.1)).to(dt), (1 + _randn(gen, K, DH, std=0.1)).to(dt)
        doc = max(1, M // 3)                                 # documents packed into the batch: positions start anew
        s["pos"] = (torch.arange(M, device="cuda", dtype=torch.int32) % doc)[None].expand(K, M).contiguous()
        inv = 10000.0 ** (-torch.arange(0, R, 2, device="cuda", dtype=torch.float64) / R)
        ang = torch.arange(doc, device="cuda", dtype=torch.float64)[:, None] * inv[None]
        s["cos"], s["sin"] = ang.cos().float(), ang.sin().float()
        if op == "qk_bwd":
            s["dq"], s["dk"] = _randn(gen, K, M, HQ, DH, std=1e-2).to(dt), _randn(gen, K, M, HK, DH, std=1e-2).to(dt)
    return s


EPS = 1e-6


# ------------------------------------------------------------------------------------------------ plain form

def _act(name, g):
    """(act(g), act'(g)) in g's precision."""
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


def _rotate(x, c, s, R, interleaved, back):
    """The first R of the last axis rotated by pairs; `back`: by the opposite angle."""
    s = -s if back else s
    if interleaved:
        a, b = x[..., 0:R:2], x[..., 1:R:2]
    else:
        a, b = x[..., :R // 2], x[..., R // 2:R]
    ra, rb = a * c - b * s, b * c + a * s
    out = x.clone()
    if interleaved:
        out[..., 0:R:2], out[..., 1:R:2] = ra, rb
    else:
        out[..., :R // 2], out[..., R // 2:R] = ra, rb
    return out


def _plain(s):
    case = s["case"]
    op, dt = case["op"], _dtype(case)
    if op.startswith("ffn"):
        wg, wu, wd = s["wg"].float(), s["wu"].float(), s["wd"].float()
        if op == "ffn_fwd":
            x = s["x"].float()
            g, u = x @ wg.mT, x @ wu.mT
            y = (_act(case["act"], g)[0] * u) @ wd.mT
            if case["save"] == "8bit":                       # eight significant bits: exact in bf16
                g, u, dt = _value(*_pack(g)), _value(*_pack(u)), torch.bfloat16
            return {"y": y.to(_dtype(case)), "gate": g.to(dt), "up": u.to(dt)}
        full = case["save"] == "full"
        x, g, u = (s[n].float() if full else _value(*s[n]) for n in ("x", "g", "u"))
        dy = s["dy"].float()
        dh = dy @ wd
        a, da = _act(case["act"], g)
        du, dg, h = dh * a, dh * u * da, a * u
        return {"dx": (dg @ wg + du @ wu).to(dt), "dwg": (dg.mT @ x).to(dt), "dwu": (du.mT @ x).to(dt),
                "dwd": (dy.mT @ h).to(dt)}
    if op == "act8":
        return _value(*_pack(s["x"])).to(dt)
    R, il = case["R"], case["interleaved"]
    c, sn = s["cos"][s["pos"].long()][:, :, None], s["sin"][s["pos"].long()][:, :, None]
    out = {}
    for n in "qk":
        x, w = s[n].float(), s["w" + n].float()[:, None, None]
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        if op == "qk_fwd":
            out[n] = _rotate(x * r * w, c, sn, R, il, False).to(dt)
        else:
            dn, xh = _rotate(s["d" + n].float(), c, sn, R, il, True), x * r
            wdn = w * dn
            out["d" + n] = (r * (wdn - xh * (wdn * xh).mean(-1, keepdim=True))).to(dt)
            out["dw" + n] = (dn * xh).sum((1, 2)).to(dt)
    return out


# ------------------------------------------------------------------------------------------------ the package's kernels

def _own(s):
    import paper_2504_18454_b200 as P
    case = s["case"]
    op, dt = case["op"], _dtype(case)
    if op.startswith("ffn"):
        act = dict(silu=P.ACT_SILU, gelu=P.ACT_GELU, gelu_tanh=P.ACT_GELU_TANH, relu=P.ACT_RELU)[case["act"]]
        full = case["save"] == "full"
        if op == "ffn_fwd":
            y, saved = P.ffn_forward(s["x"], s["wg"], s["wu"], s["wd"], activation=act,
                                     save=P.SAVE_FULL if full else P.SAVE_8BIT)
            g, u = saved if full else (P.act8_unpack(a, dtype=torch.bfloat16) for a in saved)
            return {"y": y, "gate": g, "up": u}
        x, g, u = (s[n] if full else P.Act8(*s[n], dt) for n in ("x", "g", "u"))
        dx, dwg, dwu, dwd = P.ffn_backward(s["dy"], x, s["wg"], s["wu"], s["wd"], (g, u), activation=act)
        return {"dx": dx, "dwg": dwg, "dwu": dwu, "dwd": dwd}
    if op == "act8":
        return P.act8_unpack(P.act8_pack(s["x"]))
    args = (s["wq"], s["wk"], s["cos"], s["sin"], s["pos"])
    if op == "qk_fwd":
        q, k = P.qk_norm_rope(s["q"], s["k"], *args, eps=EPS, interleaved=case["interleaved"])
        return {"q": q, "k": k}
    dq, dk, dwq, dwk = P.qk_norm_rope_backward(s["dq"], s["dk"], s["q"], s["k"], *args, eps=EPS,
                                               interleaved=case["interleaved"])
    return {"dq": dq, "dk": dk, "dwq": dwq, "dwk": dwk}


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------------------------------------ what a pass needs

def work(case):
    b = 4 if case["dtype"] == "fp32" else 2
    if case["op"].startswith("ffn"):
        K, M, D, F = (case[n] for n in ("K", "M", "D", "F"))
        eight = lambda c: c + (c + GROUP - 1) // GROUP       # bytes of a row of c values in 8 bits
        gu = 2 * K * M * (F * b if case["save"] == "full" else eight(F))
        if case["op"] == "ffn_fwd":
            back = 0 if case["save"] == "full" else 2 * K * M * (eight(F) + F * 2)   # and the values read back
            return {"bytes": 3 * K * D * F * b + 2 * K * M * D * b + gu + back, "flops": 6 * K * M * D * F}
        x = K * M * (D * b if case["save"] == "full" else eight(D))
        return {"bytes": 6 * K * D * F * b + 2 * K * M * D * b + x + gu, "flops": 12 * K * M * D * F}
    if case["op"] == "act8":
        R, C = case["rows"], case["cols"]
        return {"bytes": 2 * R * C * b + 2 * R * (C + (C + GROUP - 1) // GROUP), "flops": 4 * R * C}
    K, M, H, DH, R = case["K"], case["M"], case["HQ"] + case["HK"], case["DH"], case["R"]
    side = 4 * K * M + 4 * max(1, M // 3) * R + 2 * K * DH * b
    n = K * M * H * DH
    if case["op"] == "qk_fwd":
        return {"bytes": 2 * n * b + side, "flops": 8 * n}
    return {"bytes": 3 * n * b + side + 2 * K * DH * b, "flops": 16 * n}


# ------------------------------------------------------------------------------------------------ 64 bits

def _exact8(x):
    """The values of the 8-bit form of x by its definition: the smallest power of two with rint(|x| / step) <= 127."""
    C = x.shape[-1]
    G = (C + GROUP - 1) // GROUP
    t = torch.nn.functional.pad(x, (0, G * GROUP - C)).unflatten(-1, (G, GROUP))
    top = t.abs().amax(-1, keepdim=True)
    e = torch.frexp(top)[1].double() - 7                     # top = m 2^(e + 7), 1/2 <= m < 1: top / 2^e in 64 .. 128
    e = e + (torch.round(top * torch.exp2(-e)) > 127)
    step = torch.exp2(e.clamp_min(-126.0))
    return (torch.round(t / step) * step).flatten(-2)[..., :C]


def exact(case, seed):
    s = prepare(case, seed)
    op, d = case["op"], torch.float64
    if op.startswith("ffn"):
        K = case["K"]
        name, outs = case["act"], []

        def act(g):
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

        for k in range(K):                                   # one worker at a time: 64-bit copies of one replica only
            wg, wu, wd = (s[n][k].to(d) for n in ("wg", "wu", "wd"))
            if op == "ffn_fwd":
                x = s["x"][k].to(d)
                g, u = torch.einsum("md,fd->mf", x, wg), torch.einsum("md,fd->mf", x, wu)
                y = torch.einsum("mf,df->md", act(g) * u, wd)
                # a checkpoint in 8 bits stands for g and u themselves: its rounding counts as error on both sides
                outs.append({"y": y, "gate": g, "up": u})
            else:
                read = lambda n: (s[n][k].to(d) if case["save"] == "full" else
                                  s[n][0][k].to(d) * torch.exp2(s[n][1][k].to(d) - 127).repeat_interleave(GROUP, -1)[..., :s[n][0].shape[-1]])
                x, g, u, dy = read("x"), read("g"), read("u"), s["dy"][k].to(d)
                dh = torch.einsum("md,df->mf", dy, wd)
                du, dg = dh * act(g), dh * u * slope(g)
                outs.append({"dx": torch.einsum("mf,fd->md", dg, wg) + torch.einsum("mf,fd->md", du, wu),
                             "dwg": torch.einsum("mf,md->fd", dg, x), "dwu": torch.einsum("mf,md->fd", du, x),
                             "dwd": torch.einsum("md,mf->df", dy, act(g) * u)})
        return {n: torch.stack([o[n] for o in outs]) for n in outs[0]}
    if op == "act8":
        return _exact8(s["x"].to(d))
    R, out = case["R"], {}
    c, sn = s["cos"].to(d)[s["pos"].long()], s["sin"].to(d)[s["pos"].long()]
    turn = torch.complex(c, sn)[:, :, None]                  # a rotation by pairs is a complex product
    for n in "qk":
        x, w = s[n].to(d), s["w" + n].to(d)[:, None, None]
        r = 1 / torch.sqrt(x.square().mean(-1, keepdim=True) + EPS)

        def spin(t, by):
            p = t[..., :R].unflatten(-1, (R // 2, 2)) if case["interleaved"] else t[..., :R].unflatten(-1, (2, R // 2)).mT
            z = torch.view_as_real(torch.view_as_complex(p.contiguous()) * by)
            z = z.flatten(-2) if case["interleaved"] else z.mT.flatten(-2)
            return torch.cat([z, t[..., R:]], -1)

        if op == "qk_fwd":
            out[n] = spin(x * r * w, turn)
        else:
            dn = spin(s["d" + n].to(d), turn.conj())
            out["dw" + n] = torch.einsum("kmhd,kmhd->kd", dn, x * r)
            t = dn * w
            out["d" + n] = r * t - x * r ** 3 * (t * x).mean(-1, keepdim=True)
    return out
