"""GPU tests of fg_layernorm and fg_layernorm_grad against the formulas in 64 bits on the CPU.

Tolerances, derived from the arithmetic (u = 2^-24, n values a row, R rows, e = half a unit in the last place of the result's type):
  * sums are formed by lanes of at most 32 values, then by trees: at most 32 + 11 roundings follow one another, in 16 waves 26 more,
    so a sum is within 72 u of the sum of its terms' magnitudes, and mean and variance with it; wider rows add one lane's
    n / 1024 values;
  * y: |error| <= e |y| + (|xh| (s + 8) u + |d mean| rstd) |gamma| + 2 u (|xh gamma| + |beta|);
  * dgamma, dbeta: R / groups <= 64 rows in turn, then at most 64 sums of those in turn and 32 more: 200 u of the terms' magnitudes.
"""
import pytest
import torch

from paper_2009_12263_amd import binding as fg

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF_ULP = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}


def make(rows, cols, dtype, ptype, seed, ld=None, offset=0, mean=0.5, device="cuda"):
    g = torch.Generator().manual_seed(seed)
    ld = ld or cols
    def rowsof(scale, shift):
        buf = torch.full((rows * ld + offset + 8,), float("nan"), dtype=dtype)
        v = buf[offset:offset + rows * ld].view(rows, ld)[:, :cols]
        v.copy_((torch.randn(rows, cols, generator=g) * scale + shift).to(dtype))
        return buf.to(device)[offset:offset + rows * ld].view(rows, ld)[:, :cols]
    x, dy = rowsof(1.5, mean), rowsof(1.0, 0.0)
    gamma, beta = (torch.randn(cols, generator=g) * 0.3 + 1).to(ptype).to(device), (torch.randn(cols, generator=g) * 0.3).to(ptype).to(device)
    return x, dy, gamma, beta


def reference(x, dy, gamma, beta, eps):
    x, dy = x.double().cpu(), dy.double().cpu()
    gamma = torch.ones(x.shape[1], dtype=torch.float64) if gamma is None else gamma.double().cpu()
    beta = torch.zeros(x.shape[1], dtype=torch.float64) if beta is None else beta.double().cpu()
    n = x.shape[1]
    mean = x.sum(1, keepdim=True) / n
    rstd = 1 / (((x - mean) ** 2).sum(1, keepdim=True) / n + eps).sqrt()
    xh = (x - mean) * rstd
    g = dy * gamma
    c1, c2 = g.sum(1, keepdim=True) / n, (g * xh).sum(1, keepdim=True) / n
    mag = rstd * (g.abs() + g.abs().sum(1, keepdim=True) / n + xh.abs() * (g * xh).abs().sum(1, keepdim=True) / n)
    return dict(mean=mean, rstd=rstd, xh=xh, y=xh * gamma + beta, dx=rstd * (g - c1 - xh * c2), dx_mag=mag, dgamma=(dy * xh).sum(0), dbeta=dy.sum(0),
                dgamma_mag=(dy * xh).abs().sum(0), dbeta_mag=dy.abs().sum(0), gamma=gamma, beta=beta, x=x, dy=dy)


def check(rows, cols, dtype, ptype, seed=1, eps=1e-5, ld=None, offset=0, mean=0.5, in_place=False, no_params=False, broadcast=False, workspace=None):
    print("[case] layernorm", rows, cols, dtype, ptype, ld, offset, flush=True)
    x, dy, gamma, beta = make(rows, cols, dtype, ptype, seed, ld, offset, mean)
    if broadcast:
        dy = dy[:1].expand(rows, cols)
    if no_params:
        gamma = beta = None
    r = reference(x, dy, gamma, beta, eps)
    x_then = x.clone()
    m, s = torch.full((rows,), float("nan"), device="cuda"), torch.full((rows,), float("nan"), device="cuda")
    y = x.clone() if in_place else torch.full_like(x, float("nan"))
    fg.fg_layernorm(y if in_place else x, gamma, beta, eps, y, m, s)
    dx = torch.full_like(x_then, float("nan"))
    dgamma, dbeta = torch.full((cols,), float("nan"), dtype=ptype, device="cuda"), torch.full((cols,), float("nan"), dtype=ptype, device="cuda")
    if in_place:
        dx = dy.clone()
    fg.fg_layernorm_grad(dx if in_place else dy, x, gamma, m, s, dx, dgamma, dbeta, workspace=workspace)
    torch.cuda.synchronize()
    steps = 72 + cols // 1024
    half, tiny, phalf, ptiny = HALF_ULP[dtype], TINY[dtype], HALF_ULP[ptype], TINY[ptype]
    d_mean = steps * U * r["x"].abs().mean(1, keepdim=True)
    # relative error of rstd: half of the variance's, which the error of the mean enters squared, and its own roundings
    d_rstd = (steps + 8) * U + (d_mean * r["rstd"]) ** 2
    d_xh = r["xh"].abs() * (d_rstd + 4 * U) + d_mean * r["rstd"] + 2 * U * r["x"].abs() * r["rstd"]
    assert ((m.cpu().double()[:, None] - r["mean"]).abs() <= d_mean + 2 * U * r["mean"].abs()).all()
    assert ((s.cpu().double()[:, None] - r["rstd"]).abs() <= r["rstd"] * (d_rstd + 4 * U)).all()
    err = (y.cpu().double() - r["y"]).abs()
    assert (err <= half * r["y"].abs() + tiny + 1.01 * d_xh * r["gamma"].abs() + 4 * U * ((r["xh"] * r["gamma"]).abs() + r["beta"].abs())).all(), err.max()
    err = (dx.cpu().double() - r["dx"]).abs()
    g_all = (r["dy"] * r["gamma"]).abs()
    d_dx = r["rstd"] * ((d_xh * g_all).mean(1, keepdim=True) * r["xh"].abs() + d_xh * (g_all * r["xh"].abs()).mean(1, keepdim=True))
    assert (err <= half * r["dx"].abs() + tiny + r["dx_mag"] * (d_rstd + (steps + 8) * U) + 1.01 * d_dx).all(), err.max()
    err = (dgamma.cpu().double() - r["dgamma"]).abs()
    assert (err <= phalf * r["dgamma"].abs() + ptiny + 200 * U * r["dgamma_mag"] + 1.01 * (r["dy"].abs() * d_xh).sum(0)).all(), err.max()
    err = (dbeta.cpu().double() - r["dbeta"]).abs()
    assert (err <= phalf * r["dbeta"].abs() + ptiny + 200 * U * r["dbeta_mag"]).all(), err.max()
    assert torch.equal(x, x_then)


T16 = [torch.bfloat16, torch.float16]


@pytest.mark.parametrize("dtype,ptype", [(torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float16, torch.float16),
                                         (torch.float16, torch.float32), (torch.float32, torch.float32)])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (5, 8), (4, 64), (33, 511), (7, 2048), (2, 2049), (9, 4104), (5, 8191), (3, 16384), (2, 32768), (2, 40001)])
def test_sizes_and_types(rows, cols, dtype, ptype):
    check(rows, cols, dtype, ptype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_more_rows_than_the_gpu_holds_at_once(dtype):
    check(5000, 100, dtype, torch.float32)
    check(2500, 1000, dtype, torch.float32)


@pytest.mark.parametrize("dtype,cols,ld,offset", [(torch.bfloat16, 1000, 1003, 1), (torch.float16, 257, 300, 3), (torch.float32, 2049, 2051, 1), (torch.bfloat16, 64, 4096, 0)])
def test_strides_and_pointers_of_any_alignment(dtype, cols, ld, offset):
    check(37, cols, dtype, torch.float32, ld=ld, offset=offset)


def test_in_place_without_parameters_and_with_a_broadcast_gradient():
    check(65, 777, torch.bfloat16, torch.float32, in_place=True)
    check(3, 40001, torch.float16, torch.float32, in_place=True)
    check(65, 777, torch.float16, torch.float16, no_params=True)
    check(65, 777, torch.float32, torch.float32, broadcast=True)
    check(1, 777, torch.float32, torch.float32, mean=100.0)


def test_workspace_of_the_caller():
    need = fg.fg_layernorm_grad_workspace(300, 1024, torch.bfloat16)
    check(300, 1024, torch.bfloat16, torch.float32, workspace=torch.empty(need, dtype=torch.uint8, device="cuda"))
    x, dy, gamma, beta = make(300, 1024, torch.bfloat16, torch.float32, 1)
    v = torch.zeros(300, device="cuda")
    g = torch.empty(1024, device="cuda")
    assert fg.fg_layernorm_grad(dy, x, gamma, v, v, torch.empty_like(x), g, g, workspace=torch.empty(need - 1, dtype=torch.uint8, device="cuda"),
                                raise_on_error=False) == fg.FG_ERR_SHAPE
    assert "workspace" in fg.fg_last_error()


def test_no_rows_and_no_columns():
    for rows, cols in ((0, 64), (5, 0), (0, 0)):
        e = torch.empty(rows, cols, device="cuda")
        g = torch.full((cols,), 7.0, device="cuda")
        dgamma, dbeta = g.clone(), g.clone()
        v = torch.empty(rows, device="cuda")
        fg.fg_layernorm(e, g, g, 1e-5, torch.empty_like(e), v, v)
        fg.fg_layernorm_grad(e, e, g, v, v, torch.empty_like(e), dgamma, dbeta)
        assert (dgamma == 0).all() and (dbeta == 0).all()


def test_non_finite_values_stay_in_their_row_and_constant_rows_are_defined():
    x = torch.randn(6, 300, device="cuda")
    x[1, 5] = float("nan"); x[3, 299] = float("inf"); x[4] = 3.0
    y = torch.empty_like(x)
    fg.fg_layernorm(x, None, None, 1e-5, y)
    assert torch.isnan(y[1]).all() and torch.isnan(y[3]).any()
    assert torch.isfinite(y[[0, 2, 4, 5]]).all() and (y[4] == 0).all()


def test_difference_quotient():
    """The gradient against central differences of the forward formula in 64 bits."""
    x, dy, gamma, beta = make(2, 33, torch.float32, torch.float32, 5)
    m, s = torch.empty(2, device="cuda"), torch.empty(2, device="cuda")
    fg.fg_layernorm(x, gamma, beta, 1e-5, torch.empty_like(x), m, s)
    dx, dg, db = torch.empty_like(x), torch.empty_like(gamma), torch.empty_like(beta)
    fg.fg_layernorm_grad(dy, x, gamma, m, s, dx, dg, db)
    h = 1e-5
    value = lambda x, gamma, beta: (reference(x, dy, gamma, beta, 1e-5)["y"] * dy.double().cpu()).sum()
    x64, g64, b64 = x.double().cpu(), gamma.double().cpu(), beta.double().cpu()
    for at in ((0, 0), (1, 17), (0, 32)):
        step = torch.zeros_like(x64); step[at] = h
        assert abs(float((value(x64 + step, g64, b64) - value(x64 - step, g64, b64)) / (2 * h)) - float(dx[at])) < 1e-5
    step = torch.zeros_like(g64); step[7] = h
    assert abs(float((value(x64, g64 + step, b64) - value(x64, g64 - step, b64)) / (2 * h)) - float(dg[7])) < 1e-5
    assert abs(float((value(x64, g64, b64 + step) - value(x64, g64, b64 - step)) / (2 * h)) - float(db[7])) < 1e-5


def test_streams_repeats_and_graph():
    x, dy, gamma, beta = make(700, 1001, torch.bfloat16, torch.float32, 9)
    outs = lambda: [torch.zeros_like(x), torch.zeros(700, device="cuda"), torch.zeros(700, device="cuda"), torch.zeros_like(x), torch.zeros_like(gamma), torch.zeros_like(beta)]
    ws = torch.empty(fg.fg_layernorm_grad_workspace(700, 1001, x.dtype), dtype=torch.uint8, device="cuda")
    def step(o, **kw):
        fg.fg_layernorm(x, gamma, beta, 1e-5, o[0], o[1], o[2], **kw)
        fg.fg_layernorm_grad(dy, x, gamma, o[1], o[2], o[3], o[4], o[5], **kw)
    first = outs(); step(first)
    side = torch.cuda.Stream(); side.wait_stream(torch.cuda.current_stream())
    other = outs(); torch.cuda.synchronize()
    step(other, stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, other))
    captured = outs(); torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fg.fg_layernorm(x, gamma, beta, 1e-5, captured[0], captured[1], captured[2])
        fg.fg_layernorm_grad(dy, x, gamma, captured[1], captured[2], captured[3], captured[4], captured[5], workspace=ws)
    for _ in range(3):
        for t in captured:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, captured))


def test_offsets_beyond_32_bits():
    """Rows of which the last begin past 2^32 bytes; first and last against the same rows by themselves (which the other tests check)."""
    rows, cols = 270000, 8192
    x = torch.empty(rows, cols, dtype=torch.float16, device="cuda")
    part, dy, gamma, beta = make(64, cols, torch.float16, torch.float32, 3)
    pick = torch.cat([torch.arange(32), torch.arange(rows - 32, rows)]).cuda()
    x.zero_(); x[pick] = part
    y, m, s = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    fg.fg_layernorm(x, gamma, beta, 1e-5, y, m, s)
    y2, m2, s2 = torch.empty_like(part), torch.empty(64, device="cuda"), torch.empty(64, device="cuda")
    fg.fg_layernorm(part, gamma, beta, 1e-5, y2, m2, s2)
    assert torch.equal(y[pick], y2) and torch.equal(m[pick], m2) and torch.equal(s[pick], s2)
    dx2 = torch.empty_like(part)
    fg.fg_layernorm_grad(dy, part, gamma, m2, s2, dx2)
    y.zero_(); y[pick] = dy
    fg.fg_layernorm_grad(y, x, gamma, m, s, x)
    assert torch.equal(x[pick], dx2)
