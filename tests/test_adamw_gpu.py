"""GPU tests of the AdamW step over many tensors and of the norm of many gradients, against the formulas in 64 bits.

Tolerances.  e = 2^-24 is half a step of FP32.  beta and 1 - beta are rounded (e each), products and sums once each: exp_avg is off by at most 6 e
(|beta1 m| + |(1 - beta1) g|), the factor's product in g being one of them; exp_avg_sq by 8 e of itself.  The step's denominator is off by 10 e of itself
(half of the root's argument, the root, the correction, the product, eps and the sum) and the rate, quotient and product by 4 e; the new parameter by those of the update and 3 e of
the parameter.  16-bit parameters are rounded once more: half a step, or half of the smallest number.  Eight bits: 2^-4 of the value, 2^-10 of the scale below the
normal numbers, 2^-9 for roots held at the smallest number; the scale itself 4 e."""
import math

import pytest
import torch

from paper_2009_12263_amd import binding as fg

pytestmark = pytest.mark.gpu
E, BLOCK = 2.0 ** -24, 256
HYPER = dict(lr=3e-3, beta1=0.9, beta2=0.97, eps=1e-8, weight_decay=0.1)


def of(n, dtype, g, std=1.0, offset=0):
    return torch.empty(n + offset, dtype=dtype, device="cuda")[offset:].copy_(torch.randn(n, generator=g, device="cuda") * std)


def blocks_of(x):
    n = x.numel()
    return torch.nn.functional.pad(x, (0, -n % BLOCK)).view(-1, BLOCK)


class Model:
    def __init__(self, sizes, dtype=torch.bfloat16, gdtype=None, master=False, bits=32, seed=0, offset=0, step=3):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.bits, self.steps = bits, step
        self.step = torch.full((1,), step, dtype=torch.int64, device="cuda")
        self.params, self.grads, self.avg, self.sq = [], [], [], []
        self.masters, self.avg_scales, self.sq_scales = [] if master else None, [] if bits == 8 else None, [] if bits == 8 else None
        for n in sizes:
            w = of(n, torch.float32, g)
            self.params.append(torch.empty(n + offset, dtype=dtype, device="cuda")[offset:].copy_(w))
            self.grads.append(of(n, gdtype or dtype, g, 0.01, offset))
            if master:
                self.masters.append(w)
            m, v = of(n, torch.float32, g, 0.01), of(n, torch.float32, g, 0.01).square_()
            if bits == 8:
                ms, m = self.in_8_bits(m)
                vs, v = self.in_8_bits(v.sqrt())
                self.avg_scales.append(ms)
                self.sq_scales.append(vs)
            self.avg.append(m)
            self.sq.append(v)

    @staticmethod
    def in_8_bits(x):
        b = blocks_of(x)
        scale = b.abs().amax(1) / 448 if b.numel() else torch.empty(0, device="cuda")
        return scale, (b / scale.clamp(min=1e-30)[:, None]).view(-1)[:x.numel()].to(torch.float8_e4m3fn)

    def moments(self, i):
        """exp_avg and exp_avg_sq of tensor i in 64 bits, and the scales of each value."""
        m, v = self.avg[i].double(), self.sq[i].double()
        if self.bits == 32:
            return m, v, None, None
        sm, sv = (s[i].double().repeat_interleave(BLOCK)[:m.numel()] for s in (self.avg_scales, self.sq_scales))
        return m * sm, (v * sv) ** 2, sm, sv

    def want(self, factor=1.0, lr_factor=1.0):
        out = []
        h = HYPER
        t, lr = self.steps, h["lr"] * lr_factor
        for i, p in enumerate(self.params):
            w = (self.masters[i] if self.masters else p).double()
            m, v, _, _ = self.moments(i)
            g = self.grads[i].double() * factor
            em = 6 * E * ((h["beta1"] * m).abs() + ((1 - h["beta1"]) * g).abs())
            m = h["beta1"] * m + (1 - h["beta1"]) * g
            v = h["beta2"] * v + (1 - h["beta2"]) * g * g
            below = torch.sqrt(v / (1 - h["beta2"] ** t)) + h["eps"]
            rate = lr / (1 - h["beta1"] ** t)
            update = rate * m / below
            new = (1 - lr * h["weight_decay"]) * w - update
            off = rate * em / below + 14 * E * update.abs() + 3 * E * w.abs() + 1e-38
            out.append(dict(w=new, off=off, m=m, em=em + 1e-38, v=v, ev=8 * E * v + 1e-38))
        return out

    def call(self, **kw):
        fg.fg_adamw(self.params, self.grads, self.avg, self.sq, self.step, *HYPER.values(), masters=self.masters, avg_scales=self.avg_scales, sq_scales=self.sq_scales, **kw)

    def check(self, want):
        for i, (p, x) in enumerate(zip(self.params, want)):
            n, half = p.numel(), torch.finfo(p.dtype).eps / 2 if p.dtype != torch.float32 else 0.0
            off = x["off"] + half * (x["w"].abs() + x["off"]) + (2 ** -25 if p.dtype == torch.float16 else 0)
            assert bool(((p.double() - x["w"]).abs() <= off).all()), ("param", i, n)
            if self.masters:
                assert bool(((self.masters[i].double() - x["w"]).abs() <= x["off"]).all()), ("master", i, n)
                assert torch.equal(p, self.masters[i].to(p.dtype))
            m, v, sm, sv = self.moments(i)
            if self.bits == 32:
                assert bool(((m - x["m"]).abs() <= x["em"]).all()) and bool(((v - x["v"]).abs() <= x["ev"]).all()), ("moments", i, n)
                continue
            assert bool(((m - x["m"]).abs() <= x["em"] + (2 ** -4 + 8 * E) * (x["m"].abs() + x["em"]) + 2 ** -10 * sm).all()), ("exp_avg", i, n)
            r, want_r = v.sqrt(), x["v"].sqrt()
            assert bool(((r - want_r).abs() <= (2 ** -4 + 16 * E) * want_r + 2 ** -9 * sv).all()), ("root", i, n)
            assert bool((r[want_r > 1e-25] > 0).all())
            for s, exact in ((self.avg_scales[i], x["m"]), (self.sq_scales[i], want_r)):
                top = blocks_of(exact).abs().amax(1) if n else exact
                assert bool(((s.double() * 448 - top).abs() <= 16 * E * top + blocks_of(x["em"]).amax(1) if n else True).all()) if n else True


SIZES = [1, 7, 8, 9, 255, 256, 257, 1000, 4095, 4097, 8191, 8192, 8193, 0, 30000, 100003]
KINDS = [(torch.bfloat16, torch.bfloat16, False), (torch.bfloat16, torch.bfloat16, True), (torch.bfloat16, torch.float32, False), (torch.bfloat16, torch.float32, True),
         (torch.float16, torch.float16, False), (torch.float16, torch.float16, True), (torch.float16, torch.float32, False), (torch.float16, torch.float32, True),
         (torch.float32, torch.float32, False)]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype,gdtype,master", KINDS)
def test_step(dtype, gdtype, master, bits):
    for offset in (0, 1):
        m = Model(SIZES, dtype, gdtype, master, bits, seed=offset, offset=offset)
        for _ in range(2):              # the second on what the first has left
            want = m.want()
            m.call()
            m.check(want)
            m.steps += 1
            m.step += 1


@pytest.mark.parametrize("bits", [32, 8])
def test_many_tensors_of_all_kinds(bits):
    """More tensors than a launch takes, with and without values, of all types in one call."""
    models = [Model([(37 * i + k) % 700 for i in range(14)] + [0, 9000], *kind, bits, seed=k) for k, kind in enumerate(KINDS)]
    wants = [m.want(0.5, 2.0) for m in models]
    one = Model([])
    for name in ("params", "grads", "avg", "sq"):
        setattr(one, name, [t for m in models for t in getattr(m, name)])
    one.masters = [t for m in models for t in (m.masters or [None] * len(m.params))]
    if bits == 8:
        one.avg_scales, one.sq_scales = ([t for m in models for t in getattr(m, name)] for name in ("avg_scales", "sq_scales"))
    one.call(grad_factor=torch.full((1,), 0.5, device="cuda"), lr_factor=torch.full((1,), 2.0, device="cuda"))
    for m, want in zip(models, wants):
        m.check(want)


@pytest.mark.parametrize("bits", [32, 8])
def test_what_lies_beside_a_tensor_stays(bits):
    """Tensors packed into one memory with values between them that are nobody's."""
    m = Model([1001, 17, 8193], torch.bfloat16, master=True, bits=bits, seed=2)

    def packed(items, dtype, gap):
        memory = torch.full((sum(len(t) + gap for t in items),), 7.0, device="cuda").to(dtype)
        inside, views, at = torch.zeros(len(memory), dtype=torch.bool, device="cuda"), [], 0
        for t in items:
            views.append(memory[at:at + len(t)])
            views[-1].copy_(t)
            inside[at:at + len(t)] = True
            at += len(t) + gap - (0 if dtype != torch.float8_e4m3fn else (len(t) + gap) % 16)        # (moments in eight bits are aligned)
        return memory, inside, views
    memories = []
    for name, gap in (("params", 3), ("masters", 5), ("avg", 16), ("sq", 16), ("avg_scales", 1), ("sq_scales", 2)):
        items = getattr(m, name)
        if items is not None:
            memory, inside, views = packed(items, items[0].dtype, gap)
            memories.append((name, memory, inside))
            setattr(m, name, views)
    want = m.want()
    m.call()
    m.check(want)
    for name, memory, inside in memories:
        assert bool((memory[~inside].float() == 7.0).all()), name


def test_one_tensor_and_none():
    m = Model([12345])
    want = m.want()
    m.call()
    m.check(want)
    Model([]).call()
    Model([0, 0]).call()


@pytest.mark.parametrize("step", [1, 2, 1000, 10 ** 6, 2 ** 40])
def test_corrections(step):
    m = Model([600], torch.float32, step=step)
    want = m.want()
    m.call()
    m.check(want)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("factor,step", [(float("inf"), 3), (float("nan"), 3), (1.0, 0), (1.0, -5)])
def test_steps_that_change_nothing(factor, step, bits):
    m = Model([500, 9000], torch.float16, master=True, bits=bits, step=step)
    before = [t.clone() for t in m.params + m.masters + m.avg + m.sq]
    m.call(grad_factor=torch.full((1,), factor, device="cuda"))
    bits_of = lambda t: t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t
    assert all(torch.equal(bits_of(a), bits_of(b)) for a, b in zip(before, m.params + m.masters + m.avg + m.sq))


def test_gradients_of_zero():
    """Blocks of nothing: moments stay zero, parameters decay."""
    for bits in (32, 8):
        m = Model([1000], torch.float32, bits=bits)
        for t in m.grads + m.avg + m.sq + (m.avg_scales or []) + (m.sq_scales or []):
            t.zero_()
        p = m.params[0].clone()
        m.call()
        assert not m.avg[0].float().any() and not m.sq[0].float().any()
        assert bool(((m.params[0].double() - p.double() * (1 - HYPER["lr"] * HYPER["weight_decay"])).abs() <= 3 * E * p.double().abs()).all())


def test_a_root_never_becomes_zero():
    """A value whose gradients were far smaller than its neighbours' keeps a second moment, and its step stays of the learning rate's size."""
    m = Model([512], torch.float32, bits=8)
    m.grads[0].fill_(1.0)
    m.grads[0][5] = 1e-4
    for t in m.avg + m.sq:
        t.zero_()
    for k in range(1, 40):
        m.step.fill_(k)
        before = m.params[0].clone()
        m.call()
        m.grads[0][5] = 0.0
        assert float(m.sq[0][5].float()) > 0
        assert abs(float(m.params[0][5] - before[5])) < 4 * HYPER["lr"]


def test_replayed_steps():
    """A captured step reads the step's number and the factors when it is replayed."""
    fg.fg_init()
    kinds = [Model(SIZES, torch.bfloat16, master=True, bits=b, seed=4, step=1) for b in (32, 8)]
    for m in kinds:
        twin = Model(SIZES, torch.bfloat16, master=True, bits=m.bits, seed=4, step=1)
        lr, factor = torch.ones(1, device="cuda"), torch.ones(1, device="cuda")
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            m.call(grad_factor=factor, lr_factor=lr)
        for k in range(4):
            for one in (m, twin):
                one.step.fill_(1 + k)
            lr.fill_(1 - 0.2 * k)
            factor.fill_(1 + 0.5 * k)
            twin.call(grad_factor=factor, lr_factor=lr)
            graph.replay()
            torch.cuda.synchronize()
            for a, b in zip(m.params + m.masters + m.avg + m.sq, twin.params + twin.masters + twin.avg + twin.sq):
                assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_refused_tensors():
    m = Model([64, 64])
    args = dict(params=m.params, grads=m.grads, exp_avg=m.avg, exp_avg_sq=m.sq, step=m.step, **HYPER)
    for change, word in ((dict(grads=m.grads[:1]), "grads"), (dict(params=[m.params[0].cpu(), m.params[1]]), "current GPU"), (dict(step=m.step.int()), "step"),
                         (dict(exp_avg=[m.avg[0].bfloat16(), m.avg[1]]), "exp_avg"), (dict(avg_scales=[m.avg[0]] * 2), "eight bits"),
                         (dict(params=[m.params[0].view(8, 8).t(), m.params[1]]), "contiguous"), (dict(masters=[m.params[0], None]), "masters")):
        with pytest.raises(ValueError, match=word):
            fg.fg_adamw(**(args | change))
    with pytest.raises(fg.FlexGemmError, match="in common"):
        fg.fg_adamw(**(args | dict(params=[m.params[0], m.params[0]])))
    with pytest.raises(fg.FlexGemmError, match="beta1"):
        fg.fg_adamw(**(args | dict(beta1=1.0)))


# ---- the norm ----------------------------------------------------------------------------------------
# The sum is formed in 64 bits: the norm and the factor are rounded once (and the factor's scale before), 2 steps of FP32 at most.

def norm_of(grads, scale=1.0, limit=1.0, **kw):
    norm, factor = (torch.full((1,), 5.0, device="cuda") for _ in range(2))
    fg.fg_grad_norm(grads, scale, limit, norm, factor, **kw)
    return float(norm), float(factor)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("scale,limit", [(1.0, 1.0), (2.0 ** -10, 0.01), (0.3, 1e6)])
def test_norm(dtype, scale, limit):
    g = torch.Generator(device="cuda").manual_seed(1)
    for sizes in (SIZES, [1], [5], [257] * 300, [3000001]):
        grads = [of(n, dtype, g, 0.02, offset=i % 2) for i, n in enumerate(sizes)]
        exact = scale * math.sqrt(sum(float(t.double().square().sum()) for t in grads))
        norm, factor = norm_of(grads, scale, limit)
        assert abs(norm - exact) <= 4 * E * exact
        want = scale * min(1.0, limit / exact)
        assert abs(factor - want) <= 8 * E * want
        assert norm_of(grads, scale, limit) == (norm, factor)


def test_norm_at_the_ends():
    big = torch.full((1000,), 3e38, device="cuda")
    assert norm_of([big])[0] == math.inf and math.isnan(norm_of([big])[1])          # (the norm itself is no FP32 number)
    norm, factor = norm_of([big[:1]], 1.0, 1.0)
    assert abs(norm - 3e38) <= 4 * E * 3e38 and 0 < factor < 1e-37
    tiny = torch.full((4,), 1e-38, device="cuda")
    assert abs(norm_of([tiny])[0] - 2e-38) <= 2e-38 * 2 ** -20 and norm_of([tiny])[1] == 1.0
    for bad in (math.inf, -math.inf, math.nan):
        x = torch.ones(5000, device="cuda", dtype=torch.float16)
        x[4321] = bad
        norm, factor = norm_of([torch.ones(3, device="cuda"), x])
        assert not math.isfinite(norm) and math.isnan(factor)
    zero = torch.zeros(100, device="cuda")
    assert norm_of([zero], 0.5) == (0.0, 0.5) and norm_of([], 0.5) == (0.0, 0.5) and norm_of([zero[:0]]) == (0.0, 1.0)


def test_clipped_step_in_a_graph():
    """Norm and step together, as a training program captures them; an overflowed gradient leaves everything as it was."""
    fg.fg_init()
    m = Model([3000, 17, 9001], torch.float16, master=True)
    norm, factor = torch.empty(1, device="cuda"), torch.empty(1, device="cuda")
    space = torch.empty(fg.fg_grad_norm_workspace(3), dtype=torch.uint8, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        fg.fg_grad_norm(m.grads, 0.5, 0.1, norm, factor, workspace=space)
        m.call(grad_factor=factor)
    for k in range(3):
        exact = 0.5 * math.sqrt(sum(float(t.double().square().sum()) for t in m.grads))
        f32 = torch.tensor(0.5 * min(1.0, 0.1 / exact)).item()
        want = m.want(f32)
        for x in want:                                      # (the factor is off by 4 steps)
            x["off"] = x["off"] + 8 * E * HYPER["lr"] * 40
            x["em"] = x["em"] + 8 * E * x["m"].abs() + 8 * E * 0.02
            x["ev"] = x["ev"] * 3
        graph.replay()
        torch.cuda.synchronize()
        m.check(want)
        m.steps += 1
        m.step += 1
        for t in m.grads:
            t.mul_(1.5)
    m.grads[1][3] = float("inf")
    before = [t.clone() for t in m.params + m.masters + m.avg + m.sq]
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(before, m.params + m.masters + m.avg + m.sq))
