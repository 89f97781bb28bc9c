"""GPU tests of the gated feed-forward block and its gradient against the formulas in 64 bits.

Tolerances are bounds, element by element.  h is half a step of the 16-bit type (2^-8 or 2^-11 of a value; binary16 has no steps below 2^-25).
A product of K terms in FP32 is off by at most 2 K 2^-24 times the product of the absolute values.  The activations are Lipschitz
with L = 1.13 and their derivatives with 0.9 (silu: 1.10 and 0.5; gelu: 1.13 and 0.81), but relu's derivative, which may be the other one where |g| is
smaller than its error; exponential, division and products of an activation are off by fewer than 2^-18 (1 + |g|) of it.  The errors of G, U, H, dH, dG and dU are
carried through the products that follow."""
import pytest
import torch

from paper_2009_12263_amd import binding as fg

pytestmark = pytest.mark.gpu
ACTS = {"none": fg.FG_ACT_NONE, "relu": fg.FG_ACT_RELU, "silu": fg.FG_ACT_SILU, "gelu": fg.FG_ACT_GELU_TANH}
LIP, LIP2 = 1.13, 0.9


def act64(g, act):
    """The activation and its derivative."""
    if act == "none":
        return g, torch.ones_like(g)
    if act == "relu":
        return g.clamp(min=0), (g > 0).double()
    if act == "silu":
        q = torch.sigmoid(g)
        return g * q, q + g * q * (1 - q)
    c = (2 / torch.pi) ** 0.5
    t = torch.tanh(c * (g + 0.044715 * g ** 3))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * c * (1 + 3 * 0.044715 * g * g)


def product(a, ea, b, eb=0.0):
    """a b^T of operands with these errors, and its error in FP32."""
    aa, ab = a.abs(), b.abs()
    e = 2 * a.shape[1] * 2 ** -24 * (aa @ ab.T)
    if torch.is_tensor(ea):
        e = e + ea @ (ab if not torch.is_tensor(eb) else ab + eb).T
    if torch.is_tensor(eb):
        e = e + aa @ eb.T
    return a @ b.T, e


def rounded(x, e, dtype):
    return e + (x.abs() + e) * torch.finfo(dtype).eps / 2 + (2 ** -25 if dtype == torch.float16 else 0)


def reference(x, w_in, w_out, act, dtype, dy=None):
    """{name: (value, bound)}"""
    x, w_in, w_out = x.double(), w_in.double(), w_out.double()
    hidden = w_out.shape[1]
    gu, egu = product(x, 0.0, w_in)
    g, u, eg, eu = gu[:, :hidden], gu[:, hidden:], egu[:, :hidden], egu[:, hidden:]
    a, d = act64(g, act)
    ea = LIP * eg + 2 ** -18 * (1 + g.abs()) * a.abs() + 2 ** -30
    h = a * u
    eh = rounded(h, ea * (u.abs() + eu) + a.abs() * eu + 2 ** -23 * h.abs(), dtype)
    y, ey = product(h, eh, w_out)
    out = dict(y=(y, rounded(y, ey, dtype)), gu=(gu, egu))
    if dy is not None:
        dy = dy.double()
        dh, edh = product(dy, 0.0, w_out.T)
        ed = LIP2 * eg + 2 ** -18 * (1 + g.abs()) + (g.abs() <= eg).double() * (act == "relu")
        dg = dh * u * d
        edg = rounded(dg, edh * (u.abs() + eu) * (d.abs() + ed) + dh.abs() * eu * (d.abs() + ed) + (dh * u).abs() * ed + 2 ** -22 * dg.abs(), dtype)
        du = dh * a
        edu = rounded(du, edh * (a.abs() + ea) + dh.abs() * ea + 2 ** -23 * du.abs(), dtype)
        dgu, edgu = torch.cat([dg, du], 1), torch.cat([edg, edu], 1)
        for name, (v, e) in dict(dx=product(dgu, edgu, w_in.T), dw_in=product(dgu.T, edgu.T, x.T), dw_out=product(dy.T, 0.0, h.T, eh.T)).items():
            out[name] = (v, rounded(v, e, dtype))
    return out


def check(name, got, want):
    value, bound = want
    off = (got.double() - value).abs() - bound
    assert torch.isfinite(got).all() and float(off.max()) <= 0, (name, float(off.max()), float((off > 0).double().mean()))


def matrix(rows, cols, dtype, g, std=1.0, ld=0, offset=0, fill=None):
    """A matrix of rows x cols inside other memory, and that memory."""
    ld = max(ld, cols)
    memory = torch.full((offset + max(rows, 1) * ld + 16,), float("nan") if fill is None else fill, device="cuda", dtype=dtype)
    m = memory[offset:offset + rows * ld].view(rows, ld)[:, :cols]
    if fill is None:
        m.copy_(torch.randn(rows, cols, generator=g, device="cuda") * std)
    return m, memory


class Case:
    """Operands and results, results in memory whose other values must stay."""
    SENTINEL = 7.0

    def __init__(self, tokens, dim, hidden, dtype, seed=0, pad=0, offset=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.dtype = dtype
        new = lambda rows, cols, std: matrix(rows, cols, dtype, g, std, cols + pad if pad else 0, offset)[0]
        self.x, self.dy = new(tokens, dim, 1.0), new(tokens, dim, 0.25)
        self.w_in, self.w_out = new(2 * hidden, dim, 1.5 * max(dim, 1) ** -0.5), new(dim, hidden, max(hidden, 1) ** -0.5)
        self.results = {}
        for name, rows, cols, t in (("y", tokens, dim, dtype), ("gu", tokens, 2 * hidden, torch.float32), ("dx", tokens, dim, dtype),
                                    ("dw_in", 2 * hidden, dim, dtype), ("dw_out", dim, hidden, dtype)):
            self.results[name] = matrix(rows, cols, t, None, ld=cols + pad if pad else 0, offset=offset, fill=self.SENTINEL)
        self.r = {k: v[0] for k, v in self.results.items()}

    def forward(self, act, keep=True, **kw):
        fg.fg_gated_ffn(self.x, self.w_in, self.w_out, ACTS[act], self.r["y"], self.r["gu"] if keep else None, **kw)

    def backward(self, act, which=("dx", "dw_in", "dw_out"), **kw):
        fg.fg_gated_ffn_grad(self.dy, self.x, self.w_in, self.w_out, ACTS[act], self.r["gu"], **{{"dx": "dX", "dw_in": "dW_in", "dw_out": "dW_out"}[k]: self.r[k] for k in which}, **kw)

    def check(self, act, names):
        want = reference(self.x, self.w_in, self.w_out, act, self.dtype, self.dy)
        for name in names:
            check(name, self.r[name], want[name])

    def untouched(self, names):
        """Every value outside these results is as it was."""
        for name in names:
            m, memory = self.results[name]
            inside = torch.zeros_like(memory, dtype=torch.bool)
            torch.as_strided(inside, m.shape, m.stride(), m.storage_offset()).fill_(True)
            assert bool((memory[~inside] == self.SENTINEL).all()), name


ALL = ("y", "gu", "dx", "dw_in", "dw_out")
SIZES = [(1, 8, 8), (1, 1, 1), (1, 64, 128), (2, 1024, 2560), (5, 33, 17), (15, 129, 40), (16, 256, 512), (17, 72, 264), (33, 500, 31), (48, 264, 1000), (64, 512, 136),
         (65, 100, 36), (65, 520, 264), (96, 1000, 500), (129, 128, 1032), (200, 256, 40), (300, 257, 131), (513, 264, 520), (777, 1024, 768),
         (2100, 200, 1104), (2101, 203, 1103), (1290, 1024, 1664)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("size", SIZES)
def test_block_and_gradient(size, dtype):
    act = ("silu", "gelu", "relu", "none")[(size[0] + size[2]) % 4]
    c = Case(*size, dtype, seed=size[0])
    c.forward(act)
    c.backward(act)
    c.check(act, ALL)
    y = c.r["y"].clone()
    c.forward(act, keep=False)
    assert torch.equal(c.r["y"], y)
    c.untouched(ALL)


@pytest.mark.parametrize("act", list(ACTS))
def test_activations(act):
    c = Case(70, 136, 200, torch.bfloat16, seed=3)
    c.x *= 3
    c.forward(act)
    c.backward(act)
    c.check(act, ALL)
    few = Case(3, 136, 200, torch.float16, seed=4)
    few.forward(act)
    few.check(act, ("y", "gu"))


@pytest.mark.parametrize("act", ["relu", "silu", "gelu"])
def test_large_preactivations(act):
    """Sigmoids and tanh at their ends: no NaN from infinities inside."""
    for tokens in (4, 80):
        c = Case(tokens, 64, 72, torch.bfloat16, seed=5)
        c.x *= 200
        c.forward(act)
        c.backward(act)
        g = c.r["gu"]
        assert float(g.max()) > 300 and float(g.min()) < -300
        c.check(act, ALL)


@pytest.mark.parametrize("tokens", [1, 7, 64, 70, 260])
@pytest.mark.parametrize("pad,offset", [(8, 8), (3, 1), (5, 0), (0, 3)])
def test_strides_and_alignment(tokens, pad, offset):
    c = Case(tokens, 136, 72, torch.bfloat16, seed=tokens, pad=pad, offset=offset)
    c.forward("silu")
    c.backward("silu")
    c.check("silu", ALL)
    c.untouched(ALL)


@pytest.mark.parametrize("tokens", [12, 150])
def test_some_gradients(tokens):
    c = Case(tokens, 96, 80, torch.float16)
    c.forward("silu")
    for which in (("dx",), ("dw_in",), ("dw_out",), ("dx", "dw_out"), ()):
        for k in ("dx", "dw_in", "dw_out"):
            c.r[k].fill_(c.SENTINEL)
        c.backward("silu", which)
        c.check("silu", which)
        assert all(bool((c.r[k] == c.SENTINEL).all()) for k in ("dx", "dw_in", "dw_out") if k not in which)


def test_gradient_against_differences():
    """<grad, v> against the central difference of <dY, Y> in 64 bits along v, within the sum of the bounds.  v has the gradient's signs, so that its slope is the
    sum of all absolute values and the bounds say something."""
    c = Case(90, 64, 48, torch.bfloat16, seed=9)
    c.forward("gelu")
    c.backward("gelu")
    want = reference(c.x, c.w_in, c.w_out, "gelu", c.dtype, c.dy)
    args = {"dx": c.x, "dw_in": c.w_in, "dw_out": c.w_out}

    def value(**moved):
        x, w_in, w_out = (moved.get(k, args[k].double()) for k in ("dx", "dw_in", "dw_out"))
        gu = x @ w_in.T
        return float(((act64(gu[:, :48], "gelu")[0] * gu[:, 48:]) @ w_out.T * c.dy.double()).sum())
    for k, at in args.items():
        v = want[k][0].sign()
        e = 1e-5
        slope = (value(**{k: at.double() + e * v}) - value(**{k: at.double() - e * v})) / (2 * e)
        got, bound = float((c.r[k].double() * v).sum()), float((want[k][1] * v.abs()).sum())
        assert abs(got - slope) <= bound + 1e-6 * abs(slope) and slope > 10 * bound, (k, got, slope, bound)


@pytest.mark.parametrize("tokens", [1, 20, 130])
def test_rows_do_not_mix(tokens):
    """What a row holds reaches its own results and the weights' gradients only."""
    c = Case(tokens + 1, 72, 56, torch.bfloat16, seed=1)
    c.forward("silu")
    c.backward("silu", ("dx",))
    y, dx = c.r["y"].clone(), c.r["dx"].clone()
    c.x[tokens // 2] = float("nan")
    c.forward("silu")
    c.backward("silu", ("dx",))
    keep = torch.arange(tokens + 1, device="cuda") != tokens // 2
    assert torch.equal(c.r["y"][keep], y[keep]) and torch.equal(c.r["dx"][keep], dx[keep])
    assert bool(c.r["y"][~keep].isnan().all()) and bool(c.r["dx"][~keep].isnan().all())


def test_sizes_of_zero():
    for size in ((0, 16, 24), (5, 16, 0), (5, 0, 24), (0, 0, 0)):
        c = Case(*size, torch.bfloat16)
        c.forward("silu")
        c.backward("silu")
        assert all(not c.r[k].numel() or bool((c.r[k] == 0).all()) for k in ("y", "dx", "dw_in", "dw_out")), size


def test_the_same_bits_every_time():
    for size in ((3, 640, 1000), (150, 264, 520), (40, 2048, 96)):
        c = Case(*size, torch.bfloat16)
        c.forward("silu")
        c.backward("silu")
        first = {k: v.clone() for k, v in c.r.items()}
        torch.empty(1 << 24, device="cuda").fill_(float("nan"))          # workspaces hold something else
        c.forward("silu")
        c.backward("silu")
        assert all(torch.equal(first[k], c.r[k]) for k in ALL)


@pytest.mark.parametrize("tokens", [2, 96])
def test_other_streams_and_captured_calls(tokens):
    """Two captured steps with workspaces of their own, replayed side by side between eager calls."""
    fg.fg_init()
    cases = [Case(tokens, 200, 104, torch.bfloat16, seed=s) for s in (1, 2)]
    space = lambda n: torch.empty(n, dtype=torch.uint8, device="cuda")
    graphs, streams = [], [torch.cuda.Stream() for _ in cases]
    for c, s in zip(cases, streams):
        c.spaces = space(fg.fg_gated_ffn_workspace(tokens, 200, 104)), space(fg.fg_gated_ffn_grad_workspace(tokens, 200, 104))
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            c.forward("silu", stream=s)                 # (workspaces of the binding)
            c.backward("silu", stream=s)
        s.synchronize()
        c.check("silu", ALL)
        c.want = {k: v.clone() for k, v in c.r.items()}
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            c.forward("silu", workspace=c.spaces[0])
            c.backward("silu", workspace=c.spaces[1])
        graphs.append(graph)
    for _ in range(3):
        for c in cases:
            for v in c.r.values():
                v.fill_(float("nan"))
        torch.cuda.synchronize()
        for graph, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        for c in cases:
            assert all(torch.equal(c.r[k], c.want[k]) for k in ALL)
        cases[0].forward("silu")
        torch.cuda.synchronize()


def test_weights_whose_halves_lie_far_apart():
    """U's rows of W_in begin more than 2^31 bytes behind G's: such weights are copied."""
    T, D, H, ld = 70, 64, 600, 1 << 21
    g = torch.Generator(device="cuda").manual_seed(0)
    memory = torch.empty(2 * H * ld, dtype=torch.bfloat16, device="cuda")
    c = Case(T, D, H, torch.bfloat16, seed=1)
    w_in = memory.view(2 * H, ld)[:, :D]
    w_in.copy_(torch.randn(2 * H, D, generator=g, device="cuda") * D ** -0.5)
    c.w_in = w_in
    c.forward("silu")
    c.backward("silu")
    c.check("silu", ALL)
    few = Case(3, D, H, torch.bfloat16, seed=2)
    few.w_in = w_in
    few.forward("silu")
    few.check("silu", ("y", "gu"))


def test_offsets_beyond_32_bits():
    """Results and kept values of more than 2^32 bytes: tokens at the end are those of a call on them alone."""
    T, D, H = 140000, 64, 4100
    c = Case(T, D, H, torch.bfloat16, seed=3)
    assert c.r["gu"].numel() * 4 > 1 << 32
    c.forward("silu")
    c.backward("silu", ("dx",))
    last = slice(T - 200, T)
    want = reference(c.x[last], c.w_in, c.w_out, "silu", c.dtype, c.dy[last])
    for name in ("y", "gu", "dx"):
        check(name, c.r[name][last], want[name])


def test_long_sums_of_a_weight_gradient():
    """dW over many tokens, against 64 bits in blocks of tokens."""
    T, D, H = 40000, 72, 136
    c = Case(T, D, H, torch.float16, seed=4)
    c.dy *= 2 ** -6
    c.forward("gelu")
    c.backward("gelu", ("dw_in", "dw_out"))
    want = {}
    for t in range(0, T, 8000):
        part = reference(c.x[t:t + 8000], c.w_in, c.w_out, "gelu", c.dtype, c.dy[t:t + 8000])
        for name in ("dw_in", "dw_out"):
            v, e = want.get(name, (0.0, 0.0))
            want[name] = v + part[name][0], e + part[name][1]
    # (a block's bound holds for its 8000 terms of the FP32 sum; 40000 have five times that, and each block's bound already holds one rounding of its result)
    for name in want:
        check(name, c.r[name], (want[name][0], 5 * want[name][1]))


def test_refused_tensors():
    c = Case(4, 16, 24, torch.bfloat16)
    for change, word in ((dict(X=c.x.cpu()), "current GPU"), (dict(W_in=c.w_in[:47]), "W_in"), (dict(W_out=c.w_out[:, :23]), "W_out"),
                         (dict(Y=c.r["y"][:3]), "Y"), (dict(GU=c.r["gu"][:, :47]), "GU"), (dict(X=c.x.t().contiguous().t()), "contiguous")):
        args = dict(X=c.x, W_in=c.w_in, W_out=c.w_out, act=fg.FG_ACT_SILU, Y=c.r["y"], GU=c.r["gu"]) | change
        with pytest.raises(ValueError, match=word):
            fg.fg_gated_ffn(**args)
    for change, word in ((dict(act=9), "activation"), (dict(Y=c.r["y"].float()), "Y"), (dict(GU=c.r["gu"].bfloat16()), "GU"), (dict(W_in=c.w_in.half()), "W_in")):
        args = dict(X=c.x, W_in=c.w_in, W_out=c.w_out, act=fg.FG_ACT_SILU, Y=c.r["y"], GU=c.r["gu"]) | change
        with pytest.raises(fg.FlexGemmError, match=word):
            fg.fg_gated_ffn(**args)
