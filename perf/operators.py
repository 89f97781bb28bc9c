"""The operators at the two ends of a language model, as cases that can be timed and checked: layer norm, the
embedding of tokens, and the softmax cross entropy of a linear layer over the vocabulary.

A case is one call of an operator, or the forward and the backward call of a training step, on operands that
are on the GPU already, with the result buffers that a program keeps.  Keys: ``op``; ``dtype`` of activations, weights and their gradients;
``train``: the gradients are computed as well.  ``layernorm``: ``rows``, ``cols``, ``pdtype`` of gamma and beta.
``embedding``: ``tokens``, ``vocab``, ``dim``, ``skew`` (0: all ids equally likely; larger: text-like, a few ids make up most
of the tokens), ``add``: the gradient is added to one that is there.  ``xent``: ``tokens``, ``vocab``, ``dim``, ``left_out``: the share of
tokens without a target (padding, prompts), ``sharp``: the standard deviation of the logits, ``mean``: one gradient for
all tokens (the mean of the losses) instead of one for each.
"""
import math

import torch

own = False

_TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
_EPS = 1e-5


def _layernorm(rows, cols, dtype, pdtype, train):
    return dict(op="layernorm", rows=rows, cols=cols, dtype=dtype, pdtype=pdtype, train=train)


def _embedding(tokens, vocab, dim, dtype, train, skew=1.0, add=False):
    return dict(op="embedding", tokens=tokens, vocab=vocab, dim=dim, dtype=dtype, train=train, skew=skew, add=add)


def _xent(tokens, vocab, dim, dtype, train, left_out=0.05, sharp=2.0, mean=False):
    return dict(op="xent", tokens=tokens, vocab=vocab, dim=dim, dtype=dtype, train=train, left_out=left_out, sharp=sharp, mean=mean)


def listed():
    return [
        # one step of generation for a handful of sequences: bound by the call
        dict(_layernorm(8, 1024, "bf16", "bf16", False), name="layernorm_few_rows"),
        # a prompt or an evaluation batch
        dict(_layernorm(16384, 4096, "bf16", "bf16", False), name="layernorm_forward"),
        # a training step's layer norm, full precision, nothing a multiple of anything
        dict(_layernorm(4099, 2049, "f32", "f32", True), name="layernorm_train_odd"),
        # a large model's training step, 16-bit activations with FP32 parameters
        dict(_layernorm(16384, 8192, "f16", "f32", True), name="layernorm_train"),
        # the tokens of one generation step
        dict(_embedding(16, 32768, 2048, "bf16", False), name="embedding_few_tokens"),
        # a training step: lookup, and the dense gradient of the table
        dict(_embedding(16384, 65536, 4096, "bf16", True), name="embedding_train"),
        # tied weights: the gradient is added to the head's; an odd vocabulary and width, a few ids hold most tokens
        dict(_embedding(9999, 50001, 1001, "f32", True, skew=2.0, add=True), name="embedding_train_tied_odd"),
        # scoring a few tokens: bound by reading the vocabulary matrix
        dict(_xent(16, 65536, 2048, "bf16", False), name="xent_score_few"),
        # a perplexity evaluation, loss alone
        dict(_xent(4096, 32768, 2048, "f16", False), name="xent_evaluate"),
        # a small training step, binary16 with a scaled loss, sharp predictions, a gradient per token
        dict(_xent(2048, 32768, 1024, "f16", True, sharp=6.0), name="xent_train_small"),
        # odd numbers of tokens and words, most of the tokens left out (prompts)
        dict(_xent(1999, 50001, 1536, "bf16", True, left_out=0.6, mean=True), name="xent_train_odd"),
        # a large model's training step
        dict(_xent(8192, 131072, 4096, "bf16", True, mean=True), name="xent_train_large"),
    ]


def _log_uniform(rng, lo, hi):
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return max(lo, min(hi, n))


def _size(rng, lo, hi, step):
    """Over the logarithm of the range; half of them multiples of `step`."""
    n = _log_uniform(rng, lo, hi)
    return n if rng.random() < 0.5 else max(lo, n // step * step)


def draw(rng):
    op = rng.choice(["layernorm", "embedding", "xent"])
    train = rng.random() < 0.6
    if op == "layernorm":
        dtype = rng.choice(["bf16", "f16", "f32"])
        return _layernorm(_size(rng, 1, 16384, 8), _size(rng, 64, 8192, 64), dtype, rng.choice([dtype, "f32"]), train)
    if op == "embedding":
        dtype = rng.choice(["bf16", "f16", "f32"])
        return _embedding(_size(rng, 1, 32768, 8), _size(rng, 1000, 131072, 64), _size(rng, 64, 4096, 64), dtype, train,
                          skew=rng.choice([0.0, 1.0, 2.0]), add=train and rng.random() < 0.4)
    dim = _log_uniform(rng, 64, 4096)
    if rng.random() < 0.75:
        dim = max(64, dim // 8 * 8)             # a model's width; any other is rare
    return _xent(_size(rng, 1, 8192, 8), _size(rng, 1000, 131072, 64), dim, rng.choice(["bf16", "f16"]), train,
                 left_out=rng.choice([0.0, 0.05, 0.6]), sharp=rng.choice([1.0, 3.0, 8.0]), mean=rng.random() < 0.5)


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    dt = _TYPES[case["dtype"]]

    def normal(*shape, dtype=dt, std=1.0, mean=0.0):
        return torch.randn(*shape, generator=g, device=dev, dtype=torch.float32).mul_(std).add_(mean).to(dtype)

    s = dict(case=case)
    if case["op"] == "layernorm":
        R, n, pt = case["rows"], case["cols"], _TYPES[case["pdtype"]]
        # hidden states: a few columns much larger than the rest, each row with an offset
        s["x"] = (torch.randn(R, n, generator=g, device=dev) * (1 + 4 * (torch.rand(n, generator=g, device=dev) < 0.01).float())
                  + 0.5 * torch.randn(R, 1, generator=g, device=dev) + 0.25).to(dt)
        s["gamma"], s["beta"] = normal(n, dtype=pt, std=0.1, mean=1.0), normal(n, dtype=pt, std=0.1)
        s["y"] = torch.empty(R, n, device=dev, dtype=dt)
        s["mean"], s["rstd"] = torch.empty(R, device=dev), torch.empty(R, device=dev)
        if case["train"]:
            s["dy"] = normal(R, n)
            s["dx"], s["dgamma"], s["dbeta"] = torch.empty_like(s["x"]), torch.empty_like(s["gamma"]), torch.empty_like(s["beta"])
    elif case["op"] == "embedding":
        T, V, K = case["tokens"], case["vocab"], case["dim"]
        s["table"] = normal(V, K, std=0.02)
        u = torch.rand(T, generator=g, device=dev, dtype=torch.float64)
        # text-like: the id V^u has a frequency that falls with its inverse; a larger power of u prefers the first ids more
        ids = (u * V if case["skew"] == 0 else torch.exp(math.log(V) * u ** (0.5 + 0.5 * case["skew"])) - 1).long().clamp_(0, V - 1)
        perm = torch.randperm(V, generator=g, device=dev)
        s["ids"] = perm[ids]
        s["ids"][torch.rand(T, generator=g, device=dev) < 0.01] = -1            # padding
        s["scale"] = math.sqrt(K)
        s["y"] = torch.empty(T, K, device=dev, dtype=dt)
        if case["train"]:
            s["dy"] = normal(T, K)
            s["there"] = normal(V, K) if case["add"] else None
            s["dtable"] = torch.empty(V, K, device=dev, dtype=dt)
    else:
        T, V, K = case["tokens"], case["vocab"], case["dim"]
        s["x"], s["w"] = normal(T, K), normal(V, K, std=1.0 / math.sqrt(K))
        s["scale"] = case["sharp"]
        s["targets"] = torch.randint(0, V, (T,), generator=g, device=dev)
        out = torch.rand(T, generator=g, device=dev) < case["left_out"]
        s["targets"][out] = -100
        s["loss"], s["lse"] = torch.empty(T, device=dev), torch.empty(T, device=dev)
        if case["train"]:
            # binary16 gradients are kept in range by a scaled loss, as its users do
            one = torch.full((1,), (16384.0 if case["dtype"] == "f16" else 1.0) / max(1.0, T * (1 - case["left_out"])), device=dev)
            s["dloss"] = one.expand(T) if case["mean"] else one * (0.5 + torch.rand(T, generator=g, device=dev))
            s["dx"], s["dw"] = torch.empty_like(s["x"]), torch.empty_like(s["w"])
    return s


def _run_own(s):
    from paper_2009_12263_amd import binding as fg
    case = s["case"]
    if case["op"] == "layernorm":
        fg.fg_layernorm(s["x"], s["gamma"], s["beta"], _EPS, s["y"], s["mean"], s["rstd"])
        out = dict(y=s["y"], mean=s["mean"], rstd=s["rstd"])
        if case["train"]:
            fg.fg_layernorm_grad(s["dy"], s["x"], s["gamma"], s["mean"], s["rstd"], s["dx"], s["dgamma"], s["dbeta"])
            out.update(dx=s["dx"], dgamma=s["dgamma"], dbeta=s["dbeta"])
        return out
    if case["op"] == "embedding":
        fg.fg_embedding(s["table"], s["ids"], s["scale"], s["y"])
        out = dict(y=s["y"])
        if case["train"]:
            fg.fg_embedding_grad(s["dy"], s["ids"], s["scale"], s["there"], s["dtable"])
            out["dtable"] = s["dtable"]
        return out
    fg.fg_linear_xent(s["x"], s["w"], s["targets"], s["scale"], s["loss"], s["lse"])
    out = dict(loss=s["loss"], lse=s["lse"])
    if case["train"]:
        fg.fg_linear_xent_grad(s["x"], s["w"], s["targets"], s["scale"], s["lse"], s["dloss"], s["dx"], s["dw"])
        out.update(dx=s["dx"], dw=s["dw"])
    return out


def _run_plain(s):
    case = s["case"]
    dt = _TYPES[case["dtype"]]
    if case["op"] == "layernorm":
        x, gamma, beta = s["x"].float(), s["gamma"].float(), s["beta"].float()
        n = x.shape[1]
        mean = x.sum(1, keepdim=True) / n
        xh = x - mean
        rstd = 1 / torch.sqrt((xh * xh).sum(1, keepdim=True) / n + _EPS)
        xh *= rstd
        out = dict(y=(xh * gamma + beta).to(dt), mean=mean[:, 0], rstd=rstd[:, 0])
        if case["train"]:
            dy = s["dy"].float()
            h = dy * gamma
            dx = (h - h.sum(1, keepdim=True) / n - xh * ((h * xh).sum(1, keepdim=True) / n)) * rstd
            out.update(dx=dx.to(dt), dgamma=(dy * xh).sum(0).to(s["gamma"].dtype), dbeta=dy.sum(0).to(s["beta"].dtype))
        return out
    if case["op"] == "embedding":
        ids = s["ids"]
        there = ((ids >= 0) & (ids < case["vocab"])).float()[:, None]
        at = ids.clamp(0, case["vocab"] - 1)
        out = dict(y=(s["table"][at].float() * (there * s["scale"])).to(dt))
        if case["train"]:
            total = s["there"].to(torch.float32, copy=True) if case["add"] else torch.zeros(case["vocab"], case["dim"], device=ids.device)
            out["dtable"] = total.index_add_(0, at, s["dy"].float() * (there * s["scale"])).to(dt)
        return out
    x, w, targets = s["x"].float(), s["w"].float(), s["targets"]
    z = torch.matmul(x, w.t()) * s["scale"]
    has = (targets >= 0) & (targets < case["vocab"])
    at = targets.clamp(0, case["vocab"] - 1)[:, None]
    top = z.amax(1, keepdim=True)
    z_target = z.gather(1, at)
    e = z.sub_(top).exp_()
    total = e.sum(1, keepdim=True)
    lse = top + torch.log(total)
    out = dict(loss=torch.where(has, (lse - z_target)[:, 0], 0.0), lse=lse[:, 0])
    if case["train"]:
        dz = e.div_(total)
        dz.scatter_add_(1, at, torch.full_like(total, -1.0))
        dz *= torch.where(has, s["dloss"] * s["scale"], 0.0)[:, None]
        out.update(dx=torch.matmul(dz, w).to(dt), dw=torch.matmul(dz.t(), x).to(dt))
    return out


def run(state):
    return _run_own(state) if own else _run_plain(state)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "layernorm":
        x, gamma, beta = s["x"].double(), s["gamma"].double(), s["beta"].double()
        mean = torch.mean(x, 1, keepdim=True)
        rstd = (torch.var(x, 1, keepdim=True, unbiased=False) + _EPS).rsqrt()
        out = dict(y=(x - mean) * rstd * gamma + beta, mean=mean.squeeze(1), rstd=rstd.squeeze(1))
        if case["train"]:
            dy = s["dy"].double()
            # from y = gamma xh + beta and the projection of dxh off the directions 1 and xh
            xh = (x - mean) * rstd
            dxh = dy * gamma
            dxh = dxh - torch.mean(dxh, 1, keepdim=True) - xh * torch.mean(dxh * xh, 1, keepdim=True)
            out.update(dx=dxh * rstd, dgamma=torch.sum(dy * xh, 0), dbeta=torch.sum(dy, 0))
        return out
    if case["op"] == "embedding":
        V, ids = case["vocab"], s["ids"]
        rows = torch.cat([s["table"].double(), torch.zeros(1, case["dim"], device=ids.device, dtype=torch.float64)])
        at = torch.where((ids < 0) | (ids >= V), V, ids)
        out = dict(y=rows.index_select(0, at) * s["scale"])
        if case["train"]:
            d = torch.zeros_like(rows).index_put_((at,), s["dy"].double(), accumulate=True)[:V] * s["scale"]
            out["dtable"] = d + s["there"].double() if case["add"] else d
        return out
    V, scale = case["vocab"], s["scale"]
    w = s["w"].double()
    loss, lse, dx, dw = [], [], [], torch.zeros_like(w) if case["train"] else None
    for t in range(0, case["tokens"], 1024):            # 1024 tokens x 131072 words: 1 GB
        x, target = s["x"][t:t + 1024].double(), s["targets"][t:t + 1024]
        z = scale * (x @ w.T)
        has = torch.logical_and(target >= 0, target < V)
        total = torch.logsumexp(z, 1)
        lse.append(total)
        loss.append((total - z[torch.arange(len(x), device=z.device), target.where(has, 0)]) * has)
        if case["train"]:
            dz = torch.exp(z - total[:, None])
            dz[torch.arange(len(x), device=z.device), target.where(has, 0)] -= 1
            dz *= (scale * s["dloss"][t:t + 1024].double() * has)[:, None]
            dx.append(dz @ w)
            dw += dz.T @ x
    out = dict(loss=torch.cat(loss), lse=torch.cat(lse))
    if case["train"]:
        out.update(dx=torch.cat(dx), dw=dw)
    return out


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "layernorm":
        e, p = case["rows"] * case["cols"], case["cols"] * (4 if case["pdtype"] == "f32" else 2)
        if not case["train"]:
            return {"bytes": 2 * e * size + 2 * p + 8 * case["rows"], "flops": 8 * e}
        return {"bytes": 4 * e * size + 4 * p + 8 * case["rows"], "flops": 22 * e}      # x, dy, y, dx
    if case["op"] == "embedding":
        e, t = case["tokens"] * case["dim"], case["vocab"] * case["dim"]
        if not case["train"]:
            return {"bytes": 2 * e * size + 8 * case["tokens"], "flops": e}
        return {"bytes": 3 * e * size + (2 if case["add"] else 1) * t * size + 8 * case["tokens"], "flops": 3 * e}
    T, V, K = case["tokens"], case["vocab"], case["dim"]
    if not case["train"]:
        return {"bytes": (T + V) * K * size + 16 * T, "flops": 2 * T * V * K}
    return {"bytes": 2 * (T + V) * K * size + 20 * T, "flops": 6 * T * V * K}
