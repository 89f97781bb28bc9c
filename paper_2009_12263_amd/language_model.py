"""A small language model on the library's operators, forward, backward and update: token embedding, layer norm, one
hidden layer (fg_gemm with bias and ReLU, or with --hidden a gated feed-forward block), layer norm, and the cross entropy of an output layer that shares the
embedding's matrix.

    python -m paper_2009_12263_amd.language_model [--steps 200] [--tokens 2048] [--vocab 8192] [--dim 512] [--hidden 0] [--adamw 0]

trains it on synthetic text, a chain in which a word is followed by one of its own most of the time, and prints the loss.  The update is gradient descent, or
with --adamw 32 or 8 a step of AdamW with clipped gradients and moments of so many bits.
Every product, normalisation, lookup, loss and AdamW step runs in the library; torch holds the memory and does the
element-wise rest (rounding activations to bfloat16, the mask of the ReLU's gradient, the update of gradient descent)."""
from __future__ import annotations

import argparse
import math

import torch

from . import binding as fg


def rows(t: torch.Tensor) -> fg.Matrix:
    return fg.Matrix(t, fg.FG_ROW, t.stride(0))


def transposed(t: torch.Tensor) -> fg.Matrix:
    """The transpose of a matrix with contiguous rows, for fg_gemm."""
    return fg.Matrix(t, fg.FG_COL, t.stride(0))


class LanguageModel:
    """Parameters in bfloat16, layer norm's in FP32; buffers for `tokens` tokens.  With ids i and targets j,

        h = sqrt(dim) table[i],  a = layernorm(h),  u = relu(a W^T + b),  n = layernorm(u),  loss = cross entropy(scale n table^T, j)

    and with hidden > 0   u = (silu(a G^T) * (a U^T)) W_out^T,  W_in = [G; U] of 2 hidden rows, in place of relu(a W^T + b).
    """
    EPS = 1e-5

    def __init__(self, tokens: int, vocab: int, dim: int, seed: int = 0, device: str = "cuda", hidden: int = 0):
        g = torch.Generator(device=device).manual_seed(seed)
        new = lambda *shape, dtype=torch.bfloat16: torch.empty(*shape, dtype=dtype, device=device)
        normal = lambda *shape, std: torch.randn(*shape, generator=g, device=device).mul_(std).bfloat16()
        f32 = torch.float32
        self.embed_scale, self.logit_scale = math.sqrt(dim), 1.0
        self.params = dict(table=normal(vocab, dim, std=dim ** -0.5), W=normal(dim, dim, std=dim ** -0.5), b=torch.zeros(dim, device=device),
                           gamma1=torch.ones(dim, device=device), beta1=torch.zeros(dim, device=device),
                           gamma2=torch.ones(dim, device=device), beta2=torch.zeros(dim, device=device))
        self.hidden = hidden
        if hidden:
            del self.params["W"], self.params["b"]
            self.params.update(W_in=normal(2 * hidden, dim, std=dim ** -0.5), W_out=normal(dim, hidden, std=hidden ** -0.5))
        self.grads = {k: torch.empty_like(v) for k, v in self.params.items()}
        if not hidden:
            self.grads["W"] = new(dim, dim, dtype=f32)
        self.h, self.a, self.u, self.n = (new(tokens, dim) for _ in range(4))
        self.dn, self.du, self.da, self.dh = (new(tokens, dim) for _ in range(4))
        self.mean1, self.rstd1, self.mean2, self.rstd2, self.loss, self.lse = (new(tokens, dtype=f32) for _ in range(6))
        space = lambda n: torch.empty(n, dtype=torch.uint8, device=device)
        self.spaces = dict(norm=space(fg.fg_layernorm_grad_workspace(tokens, dim, torch.bfloat16)), embed=space(fg.fg_embedding_grad_workspace(tokens, vocab, dim)),
                           xent=space(fg.fg_linear_xent_workspace(tokens, vocab, dim)), xent_grad=space(fg.fg_linear_xent_grad_workspace(tokens, vocab, dim)))
        if hidden:
            self.gu = new(tokens, 2 * hidden, dtype=f32)
            self.spaces.update(ffn=space(fg.fg_gated_ffn_workspace(tokens, dim, hidden)), ffn_grad=space(fg.fg_gated_ffn_grad_workspace(tokens, dim, hidden)))
        else:
            self.u32, self.da32 = new(tokens, dim, dtype=f32), new(tokens, dim, dtype=f32)

    def forward(self, ids: torch.Tensor, targets: torch.Tensor) -> torch.Tensor:
        """The losses of the tokens (0 where there is no target)."""
        p, T, K = self.params, self.h.shape[0], self.h.shape[1]
        fg.fg_embedding(p["table"], ids, self.embed_scale, self.h)
        fg.fg_layernorm(self.h, p["gamma1"], p["beta1"], self.EPS, self.a, self.mean1, self.rstd1)
        if self.hidden:
            fg.fg_gated_ffn(self.a, p["W_in"], p["W_out"], fg.FG_ACT_SILU, self.u, self.gu, workspace=self.spaces["ffn"])
        else:
            fg.fg_gemm(T, K, K, 1.0, rows(self.a), transposed(p["W"]), 0.0, None, rows(self.u32), bias=p["b"], bias_dim=1, act=fg.FG_ACT_RELU)
            self.u.copy_(self.u32)
        fg.fg_layernorm(self.u, p["gamma2"], p["beta2"], self.EPS, self.n, self.mean2, self.rstd2)
        fg.fg_linear_xent(self.n, p["table"], targets, self.logit_scale, self.loss, self.lse, workspace=self.spaces["xent"])
        return self.loss

    def backward(self, ids: torch.Tensor, targets: torch.Tensor, dloss: torch.Tensor) -> dict:
        """The gradients of sum(dloss * loss); the table's is that of both its uses."""
        p, d, T, K = self.params, self.grads, self.h.shape[0], self.h.shape[1]
        fg.fg_linear_xent_grad(self.n, p["table"], targets, self.logit_scale, self.lse, dloss, self.dn, d["table"], workspace=self.spaces["xent_grad"])
        fg.fg_layernorm_grad(self.dn, self.u, p["gamma2"], self.mean2, self.rstd2, self.du, d["gamma2"], d["beta2"], workspace=self.spaces["norm"])
        if self.hidden:
            fg.fg_gated_ffn_grad(self.du, self.a, p["W_in"], p["W_out"], fg.FG_ACT_SILU, self.gu, self.da, d["W_in"], d["W_out"], workspace=self.spaces["ffn_grad"])
        else:
            self.du.mul_(self.u > 0)
            torch.sum(self.du, 0, dtype=torch.float32, out=d["b"])
            fg.fg_gemm(K, K, T, 1.0, transposed(self.du), rows(self.a), 0.0, None, rows(d["W"]))
            fg.fg_gemm(T, K, K, 1.0, rows(self.du), rows(p["W"]), 0.0, None, rows(self.da32))
            self.da.copy_(self.da32)
        fg.fg_layernorm_grad(self.da, self.h, p["gamma1"], self.mean1, self.rstd1, self.dh, d["gamma1"], d["beta1"], workspace=self.spaces["norm"])
        fg.fg_embedding_grad(self.dh, ids, self.embed_scale, d["table"], d["table"], workspace=self.spaces["embed"])
        return d

    def mean_grads(self, ids: torch.Tensor, targets: torch.Tensor):
        """The losses, and the gradients of their mean over the tokens with a target."""
        loss = self.forward(ids, targets).clone()
        count = ((targets >= 0) & (targets < self.params["table"].shape[0])).sum().clamp_(min=1)
        return loss, self.backward(ids, targets, (1.0 / count.float()).expand(len(targets)))

    def step(self, ids: torch.Tensor, targets: torch.Tensor, rate: float) -> torch.Tensor:
        """One step of gradient descent on the mean loss; returns the losses before it."""
        loss, grads = self.mean_grads(ids, targets)
        for name, g in grads.items():
            self.params[name].sub_((rate * g.float()).to(self.params[name].dtype))
        return loss


class AdamW:
    """The state of AdamW for a model's parameters: FP32 copies of the 16-bit ones, moments in FP32 or (bits=8) in eight bits."""
    BETA1, BETA2, EPS, DECAY, MAX_NORM = 0.9, 0.95, 1e-8, 0.01, 1.0

    def __init__(self, model: LanguageModel, bits: int = 32):
        if bits not in (8, 32):
            raise ValueError("bits: the moments have 8 or 32")
        self.model, self.names = model, list(model.params)
        params = list(model.params.values())
        zeros = lambda p, dtype: torch.zeros(p.shape, dtype=dtype, device=p.device)
        moments = lambda: [zeros(p, torch.float32 if bits == 32 else torch.float8_e4m3fn) for p in params]
        scales = lambda: None if bits == 32 else [torch.zeros((p.numel() + 255) // 256, device=p.device) for p in params]
        self.masters = [None if p.dtype == torch.float32 else p.float() for p in params]
        self.avg, self.sq, self.avg_scales, self.sq_scales = moments(), moments(), scales(), scales()
        self.count = torch.zeros(1, dtype=torch.int64, device=params[0].device)
        self.norm, self.factor = (torch.zeros(1, device=params[0].device) for _ in range(2))
        self.space = torch.empty(fg.fg_grad_norm_workspace(len(params)), dtype=torch.uint8, device=params[0].device)

    def step(self, ids: torch.Tensor, targets: torch.Tensor, rate: float) -> torch.Tensor:
        """One step on the mean loss, its gradients scaled to a norm of MAX_NORM at most; returns the losses before it."""
        loss, grads = self.model.mean_grads(ids, targets)
        grads = [grads[name] for name in self.names]
        fg.fg_grad_norm(grads, 1.0, self.MAX_NORM, self.norm, self.factor, workspace=self.space)
        self.count.add_(torch.isfinite(self.factor))            # (gradients that overflowed change nothing: no step of the moments' either)
        fg.fg_adamw([self.model.params[name] for name in self.names], grads, self.avg, self.sq, self.count, rate, self.BETA1, self.BETA2, self.EPS, self.DECAY,
                    masters=self.masters, avg_scales=self.avg_scales, sq_scales=self.sq_scales, grad_factor=self.factor)
        return loss


def chain(tokens: int, vocab: int, seed: int, device: str = "cuda"):
    """ids and targets: word w is followed by (5 w + 7) mod vocab three times of four, else by any word; the last has no target."""
    g = torch.Generator(device=device).manual_seed(seed)
    ids = torch.randint(0, vocab, (tokens,), generator=g, device=device)
    follows = torch.rand(tokens, generator=g, device=device) < 0.75
    targets = torch.where(follows, (5 * ids + 7) % vocab, torch.randint(0, vocab, (tokens,), generator=g, device=device))
    targets[-1] = -1
    return ids, targets


def main(argv=None) -> float:
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--tokens", type=int, default=2048)
    ap.add_argument("--vocab", type=int, default=8192)
    ap.add_argument("--dim", type=int, default=512)
    ap.add_argument("--rate", type=float, default=None, help="1, or 0.003 with --adamw")
    ap.add_argument("--hidden", type=int, default=0, help="width of a gated feed-forward block; 0: a plain hidden layer")
    ap.add_argument("--adamw", type=int, default=0, choices=(0, 8, 32), help="bits of AdamW's moments; 0: gradient descent")
    a = ap.parse_args(argv)
    model, mean = LanguageModel(a.tokens, a.vocab, a.dim, hidden=a.hidden), 0.0
    update = AdamW(model, a.adamw) if a.adamw else model
    rate = a.rate if a.rate is not None else 0.003 if a.adamw else 1.0
    for i in range(a.steps):
        loss = update.step(*chain(a.tokens, a.vocab, i), rate)
        if i % 20 == 0 or i + 1 == a.steps:
            mean = float(loss.sum() / max(a.tokens - 1, 1))
            print("step %4d  loss %.4f" % (i, mean), flush=True)
    return mean


if __name__ == "__main__":
    main()
