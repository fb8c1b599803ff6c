"""K local workers train a small language model end to end on one GPU: the block operators make the gradients, PALSGD
takes the steps.

    python -m paper_2504_18454_b200.train [--workers 4] [--steps 120] [--layers 2] [--width 256] [--block gated|neo] [--fp32] [--full]

All K workers run in one batch: their replicas are the rows of a ReplicaArena, and every tensor of the model is a
(K, ...) view of it.  A layer is: norm, fused q/k/v projection, the norm of queries and keys with the position rotation
(`autograd.qk_norm_rope`), causal attention, output projection; norm, gated feed-forward (`autograd.gated_ffn`, whose
activations are kept in 8 bits unless --full).  Norms, projections and attention are plain torch.  With --block neo a layer is
that of the GPT-Neo shaped tensor lists, its operators the package's but for the attention's inner part: layer norm
(`autograd.layer_norm`, which also adds the attention's branch to the residual stream), projections and plain feed-forward block
with their biases, activation and residual (`autograd.linear`), and the loss (`autograd.cross_entropy`).  The data are
synthetic: sequences x[t+1] = (a x[t] + b) mod vocabulary with a rule (a, b) per sequence out of a few, so a model has to
find the rule in the prefix.
"""
from __future__ import annotations

import argparse
import math
from typing import Dict, List, Tuple

import torch

from . import INNER_ADAMW, PREC_BF16_MASTER, PREC_FP32
from .arena import ReplicaArena
from .autograd import cross_entropy, gated_ffn, layer_norm, linear, qk_norm_rope
from .block import ACT_GELU_TANH, block_status

HEAD = 64


def shapes(vocab: int, width: int, hidden: int, layers: int) -> List[Tuple[str, Tuple[int, ...]]]:
    out = [("embed", (vocab, width))]
    for i in range(layers):
        out += [(f"{i}.norm1", (width,)), (f"{i}.qkv", (3 * width, width)), (f"{i}.wq", (HEAD,)), (f"{i}.wk", (HEAD,)),
                (f"{i}.proj", (width, width)), (f"{i}.norm2", (width,)), (f"{i}.gate", (hidden, width)),
                (f"{i}.up", (hidden, width)), (f"{i}.down", (width, hidden))]
    return out + [("norm", (width,)), ("head", (vocab, width))]


def neo_shapes(vocab: int, width: int, hidden: int, layers: int, seq: int) -> List[Tuple[str, Tuple[int, ...]]]:
    """As the GPT-Neo shaped lists of `workloads`, matrices with a row for each output; the head is a tensor of its own."""
    out = [("embed", (vocab, width)), ("wpe", (seq, width))]
    for i in range(layers):
        for name, rows, cols in (("ln1", width, 0), ("qkv", 3 * width, width), ("proj", width, width), ("ln2", width, 0),
                                 ("fc", hidden, width), ("fc2", width, hidden)):
            out += [(f"{i}.{name}.w", (rows, cols) if cols else (rows,)), (f"{i}.{name}.b", (rows,))]
    return out + [("ln_f.w", (width,)), ("ln_f.b", (width,)), ("head", (vocab, width))]


def rms(x: torch.Tensor, w: torch.Tensor) -> torch.Tensor:
    return (x.float() * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + 1e-6)).to(x.dtype) * w[:, None]


class Workers:
    """K replicas of the model in an arena, and their gradients."""

    def __init__(self, K: int, vocab: int, width: int, hidden: int, layers: int, seq: int, *, precision: int,
                 checkpoint8: bool, seed: int = 0, neo: bool = False):
        self.K, self.width, self.layers, self.vocab, self.checkpoint8, self.neo = K, width, layers, vocab, checkpoint8, neo
        self.shapes = neo_shapes(vocab, width, hidden, layers, seq) if neo else shapes(vocab, width, hidden, layers)
        self.arena = ReplicaArena([math.prod(s) for _, s in self.shapes], K, precision=precision, inner=INNER_ADAMW)
        gen = torch.Generator(device="cuda").manual_seed(seed)
        flat = []
        for name, s in self.shapes:
            one = len(s) == 1
            flat.append(torch.full(s, 0.0 if name.endswith(".b") else 1.0, device="cuda") if one else
                        torch.randn(s, generator=gen, device="cuda") * (0.02 if name in ("embed", "wpe") else s[1] ** -0.5))
        self.arena.model.copy_(torch.cat([t.reshape(-1) for t in flat])[None].expand(K, -1))
        inv = 10000.0 ** (-torch.arange(0, HEAD, 2, device="cuda", dtype=torch.float64) / HEAD)
        ang = torch.arange(seq, device="cuda", dtype=torch.float64)[:, None] * inv
        self.cos, self.sin = ang.cos().float(), ang.sin().float()
        self.mask = torch.full((seq, seq), float("-inf"), device="cuda").triu(1)

    def weights(self) -> Dict[str, torch.Tensor]:
        return {name: self.arena.worker_tensor("param", j, *s).detach().requires_grad_()
                for j, (name, s) in enumerate(self.shapes)}

    def loss(self, p: Dict[str, torch.Tensor], tokens: torch.Tensor) -> torch.Tensor:
        """tokens (K, batch, seq + 1) -> the K mean losses."""
        if self.neo:
            return self.neo_loss(p, tokens)
        K, B, S = tokens.shape[0], tokens.shape[1], tokens.shape[2] - 1
        D, H = self.width, self.width // HEAD
        ids = tokens[:, :, :-1].reshape(K, B * S)
        x = torch.stack([p["embed"][k][ids[k]] for k in range(K)])
        pos = torch.arange(S, device="cuda", dtype=torch.int32).repeat(B)[None].expand(K, -1)
        for i in range(self.layers):
            qkv = (rms(x, p[f"{i}.norm1"]) @ p[f"{i}.qkv"].mT).unflatten(2, (3 * H, HEAD))
            q, k = qk_norm_rope(qkv[:, :, :H], qkv[:, :, H:2 * H], p[f"{i}.wq"], p[f"{i}.wk"], self.cos, self.sin, pos)
            q, k, v = (t.unflatten(1, (B, S)).transpose(2, 3) for t in (q, k, qkv[:, :, 2 * H:]))
            a = torch.softmax((q @ k.mT).float() * HEAD ** -0.5 + self.mask, -1).to(x.dtype) @ v
            x = x + a.transpose(2, 3).reshape(K, B * S, D) @ p[f"{i}.proj"].mT
            x = x + gated_ffn(rms(x, p[f"{i}.norm2"]), p[f"{i}.gate"], p[f"{i}.up"], p[f"{i}.down"],
                              checkpoint8=self.checkpoint8)
        logits = (rms(x, p["norm"]) @ p["head"].mT).float()
        nll = torch.logsumexp(logits, -1) - logits.gather(-1, tokens[:, :, 1:].reshape(K, B * S, 1))[..., 0]
        return nll.mean(-1)

    def neo_loss(self, p: Dict[str, torch.Tensor], tokens: torch.Tensor) -> torch.Tensor:
        K, B, S = tokens.shape[0], tokens.shape[1], tokens.shape[2] - 1
        H = self.width // HEAD
        ids = tokens[:, :, :-1].reshape(K, B * S)
        x = torch.stack([p["embed"][k][ids[k]] for k in range(K)]) + p["wpe"][:, :S].repeat(1, B, 1)
        wb = lambda name: (p[name + ".w"], p[name + ".b"])
        for i in range(self.layers):
            qkv = linear(layer_norm(x, *wb(f"{i}.ln1")), *wb(f"{i}.qkv"), checkpoint8=self.checkpoint8)
            q, k, v = (t.unflatten(1, (B, S)).unflatten(3, (H, HEAD)).transpose(2, 3) for t in qkv.split(self.width, 2))
            a = torch.softmax((q @ k.mT).float() * HEAD ** -0.5 + self.mask[:S, :S], -1).to(x.dtype) @ v
            branch = linear(a.transpose(2, 3).reshape(K, B * S, self.width), *wb(f"{i}.proj"), checkpoint8=self.checkpoint8)
            y, x = layer_norm(branch, *wb(f"{i}.ln2"), x)
            h = linear(y, *wb(f"{i}.fc"), activation=ACT_GELU_TANH, checkpoint8=self.checkpoint8)
            x = linear(h, *wb(f"{i}.fc2"), x, checkpoint8=self.checkpoint8)
        logits = linear(layer_norm(x, *wb("ln_f")), p["head"], checkpoint8=self.checkpoint8)
        return cross_entropy(logits, tokens[:, :, 1:].reshape(K, B * S).int(), in_place=True).mean(-1)

    def gradients(self, tokens: torch.Tensor) -> torch.Tensor:
        """Every worker's gradient of its own batch, into the arena; the K losses."""
        p = self.weights()
        losses = self.loss(p, tokens)
        losses.sum().backward()
        for j, (name, s) in enumerate(self.shapes):
            self.arena.worker_tensor("grad", j, *s).copy_(p[name].grad)
        return losses.detach()


def batch(K: int, B: int, S: int, vocab: int, gen: torch.Generator) -> torch.Tensor:
    rules = torch.tensor([[1, 1], [1, 3], [1, 5], [1, 7]], device="cuda")
    r = rules[torch.randint(0, len(rules), (K, B), generator=gen, device="cuda")]
    x = torch.randint(0, vocab, (K, B), generator=gen, device="cuda")
    out = [x]
    for _ in range(S):
        x = (r[..., 0] * x + r[..., 1]) % vocab
        out.append(x)
    return torch.stack(out, -1)


def run(K: int = 4, steps: int = 120, layers: int = 2, width: int = 256, hidden: int = 512, vocab: int = 64, seq: int = 64,
        per_worker: int = 8, precision: int = PREC_BF16_MASTER, checkpoint8: bool = True, lr: float = 2e-3, H: int = 16,
        p: float = 0.1, seed: int = 0, report=None, neo: bool = False) -> List[float]:
    """The mean loss of the workers at every step."""
    w = Workers(K, vocab, width, hidden, layers, seq, precision=precision, checkpoint8=checkpoint8, seed=seed, neo=neo)
    stream = torch.cuda.current_stream().cuda_stream
    ctx = w.arena.make_context(stream=stream, H=H, p=p, seed=seed + 2025, weight_decay=0.01)
    ctx.set_grad_clip(1.0)
    gen = torch.Generator(device="cuda").manual_seed(seed + 1)
    history = []
    for t in range(steps):
        losses = w.gradients(batch(K, per_worker, seq, vocab, gen))
        ctx.step(lr * min(1.0, (t + 1) / 10), 0.25 * p / lr, stream)      # a pull moves a quarter of the way
        history.append(losses)
        if t % 10 == 0 or t + 1 == steps:
            block_status(stream)                         # raises if a matrix kernel gave up: its results are not to be trained on
            if report:
                report(t, float(losses.mean()))
    return torch.stack(history).mean(1).tolist()


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--workers", type=int, default=4)
    ap.add_argument("--steps", type=int, default=120)
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--width", type=int, default=256, help=f"a multiple of {HEAD}")
    ap.add_argument("--block", choices=("gated", "neo"), default="gated", help="RMS norms and a gated feed-forward block, or GPT-Neo's")
    ap.add_argument("--fp32", action="store_true", help="fp32 parameters (default: bf16 with fp32 masters)")
    ap.add_argument("--full", action="store_true", help="keep the feed-forward activations in full, not in 8 bits")
    a = ap.parse_args()
    run(a.workers, a.steps, a.layers, a.width, 2 * a.width, neo=a.block == "neo", precision=PREC_FP32 if a.fp32 else PREC_BF16_MASTER,
        checkpoint8=not a.full, report=lambda t, v: print(f"step {t:4d}  loss {v:.4f}", flush=True))


if __name__ == "__main__":
    main()
