"""GPU tests of fg_linear_xent and fg_linear_xent_grad against the formulas in 64 bits on the CPU.

Tolerances, derived from the arithmetic (u = 2^-24, e = half a unit in the last place of the 16-bit type):
  * a logit is a sum of K exact products in FP32: |error| <= 4 sqrt(K) u sum |scale x w| + 4 u |z| =: dz (the bar of the matrix products);
  * lse: log-sum-exp moves by at most the largest logit's error; the exponential's argument is rounded (4 u of |z - max|, weighted by the
    exponentials, at most 4 u (max |z| + |lse|)), the sum has V / 256 + 400 roundings of positive terms at most in a row;
  * dz: exp(z - lse) moves by exp of what z and lse do; the difference to the one of the target and the product with dloss are rounded, then
    the value to 16 bits: e |dz|; binary16 keeps dz relative to the largest |dloss|, to 2^-38 of it;
  * dX, dW: dz's errors times the magnitudes of W, X, the sum's 4 sqrt(n) u of its terms' magnitudes, and one rounding to 16 bits."""
import math

import pytest
import torch

from paper_2009_12263_amd import binding as fg

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF_ULP = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}


def rows(n, cols, dtype, g, std, ld=None, offset=0):
    ld = ld or cols
    buf = torch.full((n * ld + offset + 8,), float("nan"), dtype=dtype)
    v = buf[offset:offset + n * ld].view(n, ld)[:, :cols]
    v.copy_((torch.randn(n, cols, generator=g) * std).to(dtype))
    return buf.cuda()[offset:offset + n * ld].view(n, ld)[:, :cols]


def reference(x, w, targets, scale, dloss):
    x, w = x.double().cpu(), w.double().cpu()
    T, K = x.shape
    V = w.shape[0]
    z = scale * (x @ w.T)
    mag = abs(scale) * (x.abs() @ w.abs().T)
    lse = torch.logsumexp(z, 1)
    has = (targets >= 0) & (targets < V)
    at = torch.where(has, targets, 0)
    one = torch.zeros_like(z).scatter_(1, at[:, None], 1.0)
    g = torch.where(has, dloss.double(), 0.0)[:, None]
    p = torch.exp(z - lse[:, None])
    dz = (p - one) * g
    return dict(x=x, w=w, z=z, mag=mag, lse=lse, has=has, at=at, g=g, p=p, dz=dz, loss=torch.where(has, lse - z.gather(1, at[:, None])[:, 0], 0.0),
                dx=scale * dz @ w, dw=scale * dz.T @ x)


def check(T, V, K, dtype, kind="some", std=2.0, scale=1.0, ld=None, offset=0, index=torch.int64, one_dloss=False, top=1.0, seed=11, workspace=None, grad_workspace=None):
    print("[case] xent", T, V, K, dtype, kind, scale, ld, flush=True)
    gen = torch.Generator().manual_seed(seed)
    x, w = rows(T, K, dtype, gen, 1.0, ld, offset), rows(V, K, dtype, gen, std / math.sqrt(K), ld, offset)
    targets = torch.randint(0, V, (T,), generator=gen)
    if kind == "some":
        targets[::5] = -100
        targets[1::7] = V
        if index == torch.int64:
            targets[2::11] = 2 ** 33 + 1
    elif kind == "none":
        targets[:] = -1
    dloss = torch.full((1,), 0.3 * top).expand(T) if one_dloss else top * (torch.rand(T, generator=gen) - 0.3)
    r = reference(x, w, targets, scale, dloss)
    dev_targets, dev_dloss = targets.to(index).cuda(), dloss[:1].cuda().expand(T) if one_dloss else dloss.cuda()
    loss, lse = torch.full((T,), float("nan"), device="cuda"), torch.full((T,), float("nan"), device="cuda")
    fg.fg_linear_xent(x, w, dev_targets, scale, loss, lse, workspace=workspace)
    dx, dw = torch.full((T, ld or K), float("nan"), dtype=dtype, device="cuda")[:, :K], torch.full((V, ld or K), float("nan"), dtype=dtype, device="cuda")[:, :K]
    fg.fg_linear_xent_grad(x, w, dev_targets, scale, lse, dev_dloss, dx, dw, workspace=grad_workspace)
    torch.cuda.synchronize()
    d_z = 4 * math.sqrt(K) * U * r["mag"] + 4 * U * r["z"].abs()
    zmax = r["z"].abs().max(1, keepdim=True)[0]
    d_lse = d_z.max(1, keepdim=True)[0] + 4 * U * (zmax + r["lse"].abs()[:, None] + 1) + (V / 256 + 400) * U
    err = (lse.double().cpu() - r["lse"]).abs()
    assert (err <= d_lse[:, 0]).all(), float((err / d_lse[:, 0]).max())
    err = (loss.double().cpu() - r["loss"]).abs()
    assert (err <= d_lse[:, 0] + d_z.gather(1, r["at"][:, None])[:, 0] + 2 * U * r["loss"].abs()).all(), float(err.max())
    assert (loss.cpu()[~r["has"]] == 0).all()
    half = HALF_ULP[dtype]
    d_p = r["p"] * torch.expm1(d_z + d_lse + 4 * U * (r["z"].abs() + r["lse"].abs()[:, None] + 1))
    gmax = float(r["g"].abs().max())
    d_dz = (d_p + 2 * U) * r["g"].abs() + half * r["dz"].abs() * 1.01 + (2.0 ** -38 * gmax if dtype == torch.float16 else 2.0 ** -133) * r["has"][:, None]
    for name, got, want, other, dd, terms in (("dx", dx, r["dx"], r["w"].abs(), d_dz, r["dz"].abs()), ("dw", dw, r["dw"], r["x"].abs(), d_dz.T, r["dz"].abs().T)):
        n = terms.shape[1]
        tol = abs(scale) * (dd @ other + (4 * math.sqrt(n) + 40) * U * (terms @ other)) * 1.01 + half * want.abs() * 1.01 + TINY[dtype]
        got, most = got.double().cpu(), torch.finfo(dtype).max
        beyond = torch.isinf(got)               # rounded to 16 bits: out of the type's range, or within the tolerance of its end
        assert ((want.abs() + tol >= most) & (want.sign() == got.sign()))[beyond].all() and beyond[want.abs() - tol > most * (1 + half)].all(), name
        err = (got - want).abs().masked_fill(beyond, 0.0)
        assert (err <= tol).all(), (name, float((err / tol).max()))
    assert (dx[(~r["has"]).cuda()] == 0).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,V,K", [(1, 1, 8), (1, 1000, 64), (2, 7, 1), (5, 300, 33), (16, 4097, 72), (33, 2049, 64), (64, 130, 256), (130, 9001, 40),
                                   (257, 515, 128), (300, 1000, 100), (1000, 260, 24)])
def test_sizes_and_types(T, V, K, dtype):
    check(T, V, K, dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_more_words_than_a_piece(dtype):
    check(260, 70001, 64, dtype)
    check(9000, 8500, 16, dtype)                # (pieces of fewer words)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T", [7, 8, 9, 31, 32, 33, 63, 64, 65])
@pytest.mark.parametrize("V,K,ld,offset", [(127, 129, 131, 1), (129, 128, 128, 0), (1030, 7, 7, 0), (264, 264, 272, 8)])
def test_few_tokens(T, V, K, ld, offset, dtype):
    check(T, V, K, dtype, ld=ld, offset=offset)


def test_few_tokens_in_small_pieces():
    """A workspace of four pieces of 256 words, full of NaNs: the last piece ends inside a run of 128 words."""
    check(40, 1001, 72, torch.bfloat16, grad_workspace=torch.full((fg.fg_linear_xent_grad_workspace(40, 256, 72),), 255, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("kind", ["all", "some", "none"])
@pytest.mark.parametrize("K", [64, 63])
def test_targets_and_gradients_of_the_loss(kind, K):
    check(100, 777, K, torch.bfloat16, kind, one_dloss=True)
    check(100, 777, K, torch.float16, kind, index=torch.int32, top=1e-6)
    check(100, 777, K, torch.float16, kind, top=60000.0)
    check(100, 777, K, torch.bfloat16, kind, top=1e-20)


@pytest.mark.parametrize("K,ld,offset", [(64, 72, 0), (64, 65, 1), (50, 56, 0), (8, 8, 3)])
def test_strides_and_pointers_of_any_alignment(K, ld, offset):
    for dtype in (torch.bfloat16, torch.float16):
        check(77, 1001, K, dtype, ld=ld, offset=offset)


def test_scales_and_sharp_logits():
    check(65, 3000, 128, torch.bfloat16, std=30.0)
    check(65, 3000, 128, torch.float16, scale=-0.25)
    check(65, 3000, 127, torch.float16, scale=3.5)


def test_difference_quotient():
    gen = torch.Generator().manual_seed(2)
    x, w = rows(9, 24, torch.float16, gen, 1.0), rows(50, 24, torch.float16, gen, 0.5)
    targets = torch.randint(0, 50, (9,), generator=gen); targets[4] = -1
    dloss = torch.rand(9, generator=gen)
    loss, lse, dx, dw = torch.empty(9, device="cuda"), torch.empty(9, device="cuda"), torch.empty_like(x), torch.empty_like(w)
    fg.fg_linear_xent(x, w, targets.cuda(), 1.5, loss, lse)
    fg.fg_linear_xent_grad(x, w, targets.cuda(), 1.5, lse, dloss.cuda(), dx, dw)
    value = lambda x, w: float((reference(x, w, targets, 1.5, dloss)["loss"] * dloss).sum())
    x64, w64, h = x.double().cpu(), w.double().cpu(), 1e-4
    for t, k in ((0, 0), (4, 3), (8, 23)):
        step = torch.zeros_like(x64); step[t, k] = h
        assert abs((value(x64 + step, w64) - value(x64 - step, w64)) / (2 * h) - float(dx[t, k])) < 4e-3      # 2^-11 of dz, times |w| <= 2, and of dx
    for v, k in ((0, 0), (int(targets[0]), 5), (49, 23)):
        step = torch.zeros_like(w64); step[v, k] = h
        assert abs((value(x64, w64 + step) - value(x64, w64 - step)) / (2 * h) - float(dw[v, k])) < 1e-2      # nine tokens, |x| <= 3


def test_non_finite_rows_do_not_reach_other_tokens():
    gen = torch.Generator().manual_seed(2)
    x, w = rows(70, 64, torch.bfloat16, gen, 1.0), rows(600, 64, torch.bfloat16, gen, 0.5)
    targets = torch.randint(0, 600, (70,), generator=gen).cuda()
    loss, lse = torch.empty(70, device="cuda"), torch.empty(70, device="cuda")
    fg.fg_linear_xent(x, w, targets, 1.0, loss, lse)
    x[13] = float("nan")
    loss2, lse2 = torch.empty(70, device="cuda"), torch.empty(70, device="cuda")
    fg.fg_linear_xent(x, w, targets, 1.0, loss2, lse2)
    keep = torch.arange(70) != 13
    assert torch.isnan(loss2[13]) and torch.equal(loss[keep.cuda()], loss2[keep.cuda()])


def test_no_tokens():
    e = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")
    w = torch.randn(30, 64, device="cuda").bfloat16()
    v, targets = torch.empty(0, device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda")
    dw = torch.full_like(w, float("nan"))
    fg.fg_linear_xent(e, w, targets, 1.0, v, v)
    fg.fg_linear_xent_grad(e, w, targets, 1.0, v, v, torch.empty_like(e), dw)
    assert (dw == 0).all()


@pytest.mark.parametrize("K", [64, 65])
def test_repeats_streams_and_graph(K):
    fg.fg_init()
    gen = torch.Generator().manual_seed(4)
    T, V = 300, 5000
    x, w = rows(T, K, torch.bfloat16, gen, 1.0), rows(V, K, torch.bfloat16, gen, 0.3)
    targets, dloss = torch.randint(0, V, (T,), generator=gen).cuda(), torch.rand(T, generator=gen).cuda()
    outs = lambda: [torch.zeros(T, device="cuda"), torch.zeros(T, device="cuda"), torch.zeros_like(x), torch.zeros_like(w)]
    ws = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in (fg.fg_linear_xent_workspace(T, V, K), fg.fg_linear_xent_grad_workspace(T, V, K))]
    def step(o, ws=(None, None), **kw):
        fg.fg_linear_xent(x, w, targets, 0.5, o[0], o[1], workspace=ws[0], **kw)
        fg.fg_linear_xent_grad(x, w, targets, 0.5, o[1], dloss, o[2], o[3], workspace=ws[1], **kw)
    first, other, captured = outs(), outs(), outs()
    step(first)
    torch.cuda.synchronize()
    step(other, stream=torch.cuda.Stream())
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, other))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(captured, ws)
    for _ in range(3):
        for t in captured + ws:
            t.fill_(255 if t.dtype == torch.uint8 else float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, captured))


@pytest.mark.parametrize("K,ld", [(4096, 4096), (4095, 4096)])
def test_offsets_beyond_32_bits(K, ld):
    """A vocabulary matrix of which the last rows begin past 2^32 bytes, with and without copies.  All rows but a few are zero, so that the
    logits of the others are exactly zero and the formulas can be evaluated on the few."""
    T, V = 24, 600000
    gen = torch.Generator().manual_seed(6)
    few = torch.cat([torch.arange(20), torch.arange(V - 20, V)])
    w = torch.zeros(V, ld, dtype=torch.bfloat16, device="cuda")[:, :K]
    some = rows(40, K, torch.bfloat16, gen, 4.0 / math.sqrt(K))
    w[few.cuda()] = some
    x = rows(T, K, torch.bfloat16, gen, 1.0)
    targets = few[torch.randint(0, 40, (T,), generator=gen)]
    loss, lse = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    fg.fg_linear_xent(x, w, targets.cuda(), 1.0, loss, lse)
    z = x.double().cpu() @ some.double().cpu().T
    want = torch.log(torch.exp(z).sum(1) + (V - 40))
    at = (targets[:, None] == few[None]).long().argmax(1)
    tol = 4 * math.sqrt(K) * U * (x.double().cpu().abs() @ some.double().cpu().abs().T).max() + (V / 256 + 400) * U + 16 * U * (want.abs() + z.abs().max())
    assert ((lse.double().cpu() - want).abs() <= tol).all()
    assert ((loss.double().cpu() - (want - z.gather(1, at[:, None])[:, 0])).abs() <= 2 * tol).all()
    dloss = torch.full((1,), 0.5).expand(T)
    dx, dw = torch.empty_like(x), torch.empty(V, ld, dtype=torch.bfloat16, device="cuda")[:, :K]
    fg.fg_linear_xent_grad(x, w, targets.cuda(), 1.0, lse, dloss.cuda(), dx, dw)
    dz = (torch.exp(z - want[:, None]) - torch.zeros_like(z).scatter_(1, at[:, None], 1.0)) * 0.5
    got, exact = dw[few.cuda()].double().cpu(), dz.T @ x.double().cpu()
    bar = 2.0 ** -8 * 1.02 * (dz.abs().T @ x.double().cpu().abs() + exact.abs()) + 2 * tol.max() * (dz.abs().T @ x.double().cpu().abs())
    assert ((got - exact).abs() <= bar).all()
    bar = 2.0 ** -8 * 1.02 * (dz.abs() @ some.double().cpu().abs() + (dz @ some.double().cpu()).abs()) + 2 * tol.max() * (dz.abs() @ some.double().cpu().abs())
    assert ((dx.double().cpu() - dz @ some.double().cpu()).abs() <= bar + 1e-30).all()
    # a row of zero logits, in the middle: p is the same for all of them
    p0 = (torch.exp(-want) * 0.5)[None] @ x.double().cpu()
    mags = (torch.exp(-want) * 0.5)[None] @ x.double().cpu().abs()
    assert ((dw[V // 2].double().cpu() - p0[0]).abs() <= 2.0 ** -8 * 1.02 * (p0[0].abs() + mags[0]) + 2 * tol.max() * mags[0]).all()
