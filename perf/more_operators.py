"""What stands between the two ends of a language model, and what comes after its backward pass, as cases that can be timed and
checked: the gated feed-forward block, the AdamW step over all parameters, and the norm of all gradients.

A case is one call of an operator, or the forward and the backward call of a training step, on operands that
are on the GPU already, with the buffers that a program keeps.  Keys: ``op``; ``dtype`` of activations, weights, gradients and parameters.
``ffn``: ``tokens``, ``dim``, ``hidden``, ``act`` (relu, silu, gelu_tanh), ``train``: the gradients are computed as well.
``adamw``: the tensors of a model of ``layers`` such blocks and norms with an embedding of ``vocab`` rows; ``gdtype`` of the gradients; ``master``:
FP32 parameters are kept beside the 16-bit ones; ``bits`` of the moments (32, or 8 with a scale for each 256 values); ``clip``: gradients
are multiplied by a factor that is on the GPU.  ``norm``: the same tensors' gradients.
"""
import math

import torch

own = False

_TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
_BETA1, _BETA2, _EPS, _RATE, _DECAY = 0.9, 0.95, 1e-8, 3e-4, 0.1
_BLOCK, _TOP = 256, 448.0               # values that share a scale, and the largest value of eight bits
_LEAST, _SMALLEST = 2.0 ** -9, 1e-30    # its smallest one; what is taken for nothing in a whole block
_CONST = math.sqrt(2 / math.pi)


def _ffn(tokens, dim, hidden, dtype, act, train):
    return dict(op="ffn", tokens=tokens, dim=dim, hidden=hidden, dtype=dtype, act=act, train=train)


def _adamw(layers, dim, hidden, vocab, dtype, gdtype, master, bits, clip):
    return dict(op="adamw", layers=layers, dim=dim, hidden=hidden, vocab=vocab, dtype=dtype, gdtype=gdtype, master=master, bits=bits, clip=clip)


def _norm(layers, dim, hidden, vocab, dtype, scale, limit):
    return dict(op="norm", layers=layers, dim=dim, hidden=hidden, vocab=vocab, dtype=dtype, scale=scale, limit=limit)


def listed():
    return [
        # generation for one sequence: bound by reading a small block's weights, and by the call
        dict(_ffn(1, 1024, 2560, "bf16", "silu", False), name="ffn_one_token"),
        # one step of generation for a handful of sequences: bound by reading the weights
        dict(_ffn(16, 4096, 10240, "bf16", "silu", False), name="ffn_few_tokens"),
        # a prompt
        dict(_ffn(2048, 2048, 5120, "f16", "gelu_tanh", False), name="ffn_prompt"),
        # a training step in which nothing is a multiple of anything
        dict(_ffn(1003, 1001, 2729, "bf16", "silu", True), name="ffn_train_odd"),
        # a small model's training step, binary16 with a scaled loss
        dict(_ffn(8192, 1024, 2560, "f16", "silu", True), name="ffn_train_small"),
        # a large model's training step
        dict(_ffn(8192, 4096, 10240, "bf16", "silu", True), name="ffn_train_large"),
        # a small model of many layers: 193 tensors, most of them short
        dict(_adamw(48, 64, 170, 1000, "bf16", "bf16", True, 32, True), name="adamw_many_tensors"),
        # full precision, nothing a multiple of anything
        dict(_adamw(3, 1001, 2729, 50001, "f32", "f32", False, 32, False), name="adamw_f32_odd"),
        # mixed precision: 16-bit parameters with FP32 ones beside them, clipped gradients
        dict(_adamw(2, 4096, 10240, 32768, "bf16", "bf16", True, 32, True), name="adamw_train"),
        # the same with moments in eight bits and no second copy of the parameters
        dict(_adamw(2, 4096, 10240, 32768, "bf16", "bf16", False, 8, True), name="adamw_train_8_bits"),
        # the gradients of a small model
        dict(_norm(4, 256, 680, 4001, "bf16", 1.0, 1.0), name="norm_small"),
        # the gradients of a large one in binary16, of a scaled loss
        dict(_norm(2, 4096, 10240, 32768, "f16", 2.0 ** -10, 1.0), name="norm_large"),
    ]


def _log_uniform(rng, lo, hi):
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return max(lo, min(hi, n))


def _size(rng, lo, hi, step):
    """Over the logarithm of the range; half of them multiples of `step`."""
    n = _log_uniform(rng, lo, hi)
    return n if rng.random() < 0.5 else max(lo, n // step * step)


def draw(rng):
    op = rng.choice(["ffn", "adamw", "norm"]) if rng.random() < 0.6 else "ffn"
    if op == "ffn":
        dim, hidden = _log_uniform(rng, 64, 4096), _log_uniform(rng, 64, 10240)
        if rng.random() < 0.75:         # a model's widths; any others are rare
            dim, hidden = max(64, dim // 8 * 8), max(64, hidden // 8 * 8)
        return _ffn(_size(rng, 1, 8192, 8), dim, hidden, rng.choice(["bf16", "f16"]), rng.choice(["relu", "silu", "silu", "gelu_tanh"]), rng.random() < 0.5)
    dim = _size(rng, 32, 2048, 64)
    sizes = (rng.randint(1, 24), dim, _size(rng, dim, 2 * dim, 64), _size(rng, 100, 32768, 64))
    if op == "norm":
        return _norm(*sizes, rng.choice(["bf16", "f16", "f32"]), rng.choice([1.0, 2.0 ** -10]), rng.choice([1.0, 1e6]))
    dtype = rng.choice(["bf16", "f16", "f32"])
    return _adamw(*sizes, dtype, rng.choice([dtype, "f32"]), dtype != "f32" and rng.random() < 0.5, rng.choice([32, 8]), rng.random() < 0.5)


def _shapes(case):
    d, h = case["dim"], case["hidden"]
    return [(case["vocab"], d)] + [s for _ in range(case["layers"]) for s in ((2 * h, d), (d, h), (d,), (d,))]


def _places(case):
    """Where each tensor begins in memory that holds all of them, at multiples of 256 values, and how much that is."""
    at, end = [], 0
    for s in _shapes(case):
        at.append(end)
        end += -(-math.prod(s) // _BLOCK) * _BLOCK
    return at, end


def _views(flat, case, at):
    return [flat[o:o + math.prod(s)].view(s) for o, s in zip(at, _shapes(case))]


def _in_8_bits(x):
    """Values relative to their block's scale, not yet rounded, and the scales."""
    blocks = x.view(-1, _BLOCK)
    top = blocks.abs().amax(1, keepdim=True)
    some = top >= _SMALLEST
    return (blocks * torch.where(some, _TOP / top, 0.0)).view(-1), torch.where(some, top / _TOP, 0.0).view(-1)


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    dt = _TYPES[case["dtype"]]

    def normal(*shape, dtype=dt, std=1.0):
        return torch.randn(*shape, generator=g, device=dev, dtype=torch.float32).mul_(std).to(dtype)

    s = dict(case=case)
    if case["op"] == "ffn":
        T, D, H = case["tokens"], case["dim"], case["hidden"]
        s["x"] = normal(T, D)
        s["w_in"], s["w_out"] = normal(2 * H, D, std=1.5 / math.sqrt(D)), normal(D, H, std=1 / math.sqrt(H))
        s["y"] = torch.empty_like(s["x"])
        if case["train"]:
            # binary16 gradients are kept in range by a scaled loss, as its users do
            s["dy"] = normal(T, D, std=0.05 if case["dtype"] == "f16" else 1.0 / T)
            s["gu"] = torch.empty(T, 2 * H, device=dev)
            s["dx"], s["dw_in"], s["dw_out"] = torch.empty_like(s["x"]), torch.empty_like(s["w_in"]), torch.empty_like(s["w_out"])
        return s
    at, n = _places(case)
    tail = torch.ones(n, device=dev)            # zeros between the tensors
    for o, shape, end in zip(at, _shapes(case), at[1:] + [n]):
        tail[o + math.prod(shape):end] = 0
    if case["op"] == "norm":
        s["grad"] = (normal(n, dtype=torch.float32, std=0.02) * tail).to(dt)
        s["grads"] = _views(s["grad"], case, at)
        s["norm"], s["factor"] = torch.empty(1, device=dev), torch.empty(1, device=dev)
        return s
    gt = _TYPES[case["gdtype"]]
    params = normal(n, dtype=torch.float32, std=0.02).mul_(tail)
    # gradients and their moments: of very different sizes from row to row, as in a table of words
    size = torch.exp(2 * torch.randn(n // _BLOCK, 1, generator=g, device=dev) - 6).expand(-1, _BLOCK).reshape(-1).mul_(tail)
    s["grad"] = (normal(n, dtype=torch.float32) * size).to(gt)
    avg = normal(n, dtype=torch.float32, std=0.3).mul_(size)
    sq = normal(n, dtype=torch.float32, std=0.3).add_(1).mul_(size).square_()
    del size, tail
    s["param"] = params.to(dt)
    s["params"], s["grads"] = _views(s["param"], case, at), _views(s["grad"], case, at)
    s["masters"] = s["avg_scales"] = s["sq_scales"] = None
    if case["master"]:
        s["master"] = params
        s["masters"] = _views(params, case, at)
    if case["bits"] == 8:
        (a, s["avg_scale"]), (r, s["sq_scale"]) = _in_8_bits(avg), _in_8_bits(sq.sqrt_())
        avg, sq = a.to(torch.float8_e4m3fn), torch.where(r > 0, r.clamp(min=_LEAST), 0.0).to(torch.float8_e4m3fn)
        parts = [(o // _BLOCK, -(-math.prod(shape) // _BLOCK)) for o, shape in zip(at, _shapes(case))]
        s["avg_scales"] = [s["avg_scale"][o:o + k] for o, k in parts]
        s["sq_scales"] = [s["sq_scale"][o:o + k] for o, k in parts]
    s["avg"], s["sq"] = avg, sq
    s["avgs"], s["sqs"] = _views(avg, case, at), _views(sq, case, at)
    s["step"] = torch.full((1,), 7 + seed % 1000, dtype=torch.int64, device=dev)
    s["steps"] = 7 + seed % 1000
    s["factor"] = torch.full((1,), 0.37, device=dev) if case["clip"] else None
    return s


def _state(s):
    """The parameters and the state that a step has updated."""
    return {k: s[k] for k in ("param", "master", "avg", "sq", "avg_scale", "sq_scale") if k in s}


def _run_own(s):
    from paper_2009_12263_amd import binding as fg
    case = s["case"]
    if case["op"] == "ffn":
        act = dict(relu=fg.FG_ACT_RELU, silu=fg.FG_ACT_SILU, gelu_tanh=fg.FG_ACT_GELU_TANH)[case["act"]]
        if not case["train"]:
            fg.fg_gated_ffn(s["x"], s["w_in"], s["w_out"], act, s["y"])
            return dict(y=s["y"])
        fg.fg_gated_ffn(s["x"], s["w_in"], s["w_out"], act, s["y"], s["gu"])
        fg.fg_gated_ffn_grad(s["dy"], s["x"], s["w_in"], s["w_out"], act, s["gu"], s["dx"], s["dw_in"], s["dw_out"])
        return dict(y=s["y"], dx=s["dx"], dw_in=s["dw_in"], dw_out=s["dw_out"])
    if case["op"] == "norm":
        fg.fg_grad_norm(s["grads"], case["scale"], case["limit"], s["norm"], s["factor"])
        return dict(norm=s["norm"], factor=s["factor"])
    fg.fg_adamw(s["params"], s["grads"], s["avgs"], s["sqs"], s["step"], _RATE, _BETA1, _BETA2, _EPS, _DECAY, masters=s["masters"],
                avg_scales=s["avg_scales"], sq_scales=s["sq_scales"], grad_factor=s["factor"])
    return _state(s)


def _act_plain(g, act):
    """The activation, and its derivative."""
    if act == "relu":
        on = (g > 0).float()
        return g * on, on
    if act == "silu":
        q = 1 / (1 + torch.exp(-g))
        return g * q, q * (1 + g * (1 - q))
    q = 1 / (1 + torch.exp(-2 * _CONST * (g + 0.044715 * g * g * g)))           # (1 + tanh u) / 2 = 1 / (1 + exp(-2 u))
    return g * q, q + 2 * _CONST * g * q * (1 - q) * (1 + 3 * 0.044715 * g * g)


def _run_plain(s):
    case = s["case"]
    dt = _TYPES[case["dtype"]]
    if case["op"] == "ffn":
        x, w_in, w_out, H = s["x"].float(), s["w_in"].float(), s["w_out"].float(), case["hidden"]
        gu = torch.matmul(x, w_in.t())
        gate, up = gu[:, :H], gu[:, H:]
        a, da = _act_plain(gate, case["act"])
        h = a * up
        out = dict(y=torch.matmul(h, w_out.t()).to(dt))
        if case["train"]:
            dy = s["dy"].float()
            dh = torch.matmul(dy, w_out)
            dgu = torch.cat([dh * up * da, dh * a], 1)
            out.update(dx=torch.matmul(dgu, w_in).to(dt), dw_in=torch.matmul(dgu.t(), x).to(dt), dw_out=torch.matmul(dy.t(), h).to(dt))
        return out
    if case["op"] == "norm":
        norm = torch.sqrt(s["grad"].double().square().sum()) * case["scale"]
        factor = torch.where(norm > case["limit"], case["limit"] / norm, 1.0) * case["scale"]
        s["norm"].copy_(norm)
        s["factor"].copy_(factor)
        return dict(norm=s["norm"], factor=s["factor"])
    t, small = s["steps"], case["bits"] == 8
    param = s["master"] if case["master"] else s["param"].float()
    grad = s["grad"].float()
    if case["clip"]:
        grad = grad * s["factor"]
    avg, sq = s["avg"], s["sq"]
    if small:
        avg = (avg.float().view(-1, _BLOCK) * s["avg_scale"][:, None]).view(-1)
        sq = (sq.float().view(-1, _BLOCK) * s["sq_scale"][:, None]).view(-1)
        sq = sq * sq
    avg = avg * _BETA1 + grad * (1 - _BETA1)
    sq = sq * _BETA2 + grad * grad * (1 - _BETA2)
    root = torch.sqrt(sq)
    new = param * (1 - _RATE * _DECAY) - _RATE / (1 - _BETA1 ** t) * (avg / (root * (1 / math.sqrt(1 - _BETA2 ** t)) + _EPS))
    s["param"].copy_(new)
    if case["master"]:
        s["master"].copy_(new)
    if small:
        (avg, scale), (root, of_root) = _in_8_bits(avg), _in_8_bits(root)
        sq = torch.where(root > 0, torch.where(root < _LEAST, _LEAST, root), 0.0)
        s["avg_scale"].copy_(scale)
        s["sq_scale"].copy_(of_root)
    s["avg"].copy_(avg)
    s["sq"].copy_(sq)
    return _state(s)


def run(state):
    return _run_own(state) if own else _run_plain(state)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "ffn":
        x, w_in, w_out = (s[k].double().requires_grad_(case["train"]) for k in ("x", "w_in", "w_out"))
        gate, up = torch.split(x @ w_in.T, case["hidden"], 1)
        F = torch.nn.functional
        y = ({"relu": F.relu, "silu": F.silu, "gelu_tanh": lambda v: F.gelu(v, approximate="tanh")}[case["act"]](gate) * up) @ w_out.T
        if not case["train"]:
            return dict(y=y)
        dx, dw_in, dw_out = torch.autograd.grad(y, (x, w_in, w_out), s["dy"].double())
        return dict(y=y.detach(), dx=dx, dw_in=dw_in, dw_out=dw_out)
    if case["op"] == "norm":
        norm = torch.linalg.vector_norm(s["grad"].double()).reshape(1) * case["scale"]
        return dict(norm=norm, factor=case["scale"] * (case["limit"] / norm).clamp(max=1))
    small, t = case["bits"] == 8, s["steps"]
    avg, sq, grad = s["avg"].double(), s["sq"].double(), s["grad"].double()
    if small:
        avg = avg * s["avg_scale"].double().repeat_interleave(_BLOCK)
        sq = (sq * s["sq_scale"].double().repeat_interleave(_BLOCK)) ** 2
    if case["clip"]:
        grad *= s["factor"].double()
    avg = torch.lerp(grad, avg, _BETA1)
    sq = torch.lerp(grad * grad, sq, _BETA2)
    w = (s["master"] if case["master"] else s["param"]).double()
    w = w - _RATE * (_DECAY * w + avg / (1 - _BETA1 ** t) / (torch.sqrt(sq / (1 - _BETA2 ** t)) + _EPS))
    out = dict(param=w, avg=avg, sq=sq)
    if case["master"]:
        out["master"] = w
    if small:           # what eight bits round, beside the scales
        tops = [v.view(-1, _BLOCK).abs().amax(1) for v in (avg, sq.sqrt())]
        out.update(avg_scale=tops[0] / _TOP, sq_scale=tops[1] / _TOP)
        out.update({k: v * (_TOP / top.clamp(min=_SMALLEST)).repeat_interleave(_BLOCK) for k, v, top in (("avg", avg, tops[0]), ("sq", sq.sqrt(), tops[1]))})
    return out


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "ffn":
        T, D, H = case["tokens"], case["dim"], case["hidden"]
        if not case["train"]:
            return {"bytes": (2 * T * D + 3 * D * H) * size, "flops": 6 * T * D * H}
        return {"bytes": (4 * T * D + 6 * D * H) * size, "flops": 18 * T * D * H}
    n = sum(math.prod(s) for s in _shapes(case))
    if case["op"] == "norm":
        return {"bytes": n * size, "flops": 2 * n}
    # the parameters are written, and read where there is no FP32 copy; the copy and both moments are read and written
    each = (1 if case["master"] else 2) * size + (8 if case["master"] else 0) + (4 if case["gdtype"] == "f32" else 2) + (16 if case["bits"] == 32 else 4)
    return {"bytes": n * each, "flops": 18 * n}
