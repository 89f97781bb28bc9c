"""GPU tests of fg_linear_xent and fg_linear_xent_grad in further forms, against the formulas in 64 bits on the CPU.

Tolerances: those of test_linear_xent_gpu.py for each value (derived there), and one for the norm of each gradient's error, which a lost bit
of dz would pass.  Rounding to nearest errs by a uniform part of half a unit in the last place e: its root mean square is at most e / sqrt(3) of the
value (1 / sqrt(3) where the significand is 1, less above).  The errors of the entries of dz are independent, so the norm of what they make of
dX is e / sqrt(3) times the root of sum (scale dz[t][v])^2 |w[v]|^2, and rounding dX itself adds e / sqrt(3) |dX|; FP32's errors, each entry's at most
what the bound per value allows with e = 0, are added, and a tenth for the spread of sums of thousands of entries."""
import math

import pytest
import torch

from paper_2009_12263_amd import binding as fg
from tests.test_linear_xent_gpu import HALF_ULP, TINY, U, reference, rows

pytestmark = pytest.mark.gpu


def run(x, w, targets, scale, dloss, dx=None, dw=None, workspace=None, grad_workspace=None, stream=None):
    T, V = x.shape[0], w.shape[0]
    loss, lse = torch.full((T,), float("nan"), device="cuda"), torch.full((T,), float("nan"), device="cuda")
    dx = torch.full(x.shape, float("nan"), dtype=x.dtype, device="cuda") if dx is None else dx
    dw = torch.full(w.shape, float("nan"), dtype=w.dtype, device="cuda") if dw is None else dw
    fg.fg_linear_xent(x, w, targets, scale, loss, lse, workspace=workspace, stream=stream)
    fg.fg_linear_xent_grad(x, w, targets, scale, lse, dloss, dx, dw, workspace=grad_workspace, stream=stream)
    return loss, lse, dx, dw


def compare(x, w, targets, scale, dloss, got, norms=True):
    """x, w on the GPU, targets and dloss on the CPU; got: what run() returns."""
    loss, lse, dx, dw = (t.double().cpu() for t in got)
    T, K = x.shape
    V, dtype = w.shape[0], x.dtype
    r = reference(x, w, targets, scale, dloss)
    d_z = 4 * math.sqrt(K) * U * r["mag"] + 4 * U * r["z"].abs()
    zmax = r["z"].abs().max(1, keepdim=True)[0]
    d_lse = d_z.max(1, keepdim=True)[0] + 4 * U * (zmax + r["lse"].abs()[:, None] + 1) + (V / 256 + 400) * U
    assert ((lse - r["lse"]).abs() <= d_lse[:, 0]).all()
    assert ((loss - r["loss"]).abs() <= d_lse[:, 0] + d_z.gather(1, r["at"][:, None])[:, 0] + 2 * U * r["loss"].abs()).all()
    half = HALF_ULP[dtype]
    d_p = r["p"] * torch.expm1(d_z + d_lse + 4 * U * (r["z"].abs() + r["lse"].abs()[:, None] + 1))
    gmax = float(r["g"].abs().max())
    d_32 = (d_p + 2 * U) * r["g"].abs() + (2.0 ** -38 * gmax if dtype == torch.float16 else 2.0 ** -133) * r["has"][:, None]
    for name, out, want, other, dd, terms in (("dx", dx, r["dx"], r["w"], d_32, r["dz"].abs()), ("dw", dw, r["dw"], r["x"], d_32.T, r["dz"].abs().T)):
        n = terms.shape[1]
        tol_32 = abs(scale) * (dd @ other.abs() + (4 * math.sqrt(n) + 40) * U * (terms @ other.abs())) * 1.01 + TINY[dtype]
        tol = tol_32 + abs(scale) * 1.01 * half * 1.01 * (terms @ other.abs()) + half * want.abs() * 1.01
        err = (out - want).abs()
        assert (err <= tol).all(), (name, float((err / tol).max()))
        if norms:
            of_dz = abs(scale) * (terms.square() @ other.square().sum(1)).sum().sqrt()
            bound = 1.1 * half / math.sqrt(3) * (of_dz ** 2 + want.norm() ** 2).sqrt() + tol_32.norm()
            assert err.norm() <= bound, (name, float(err.norm() / bound))
    assert (dx[~r["has"]] == 0).all()


def inputs(T, V, K, dtype, seed, x_ld=None, x_offset=0, w_ld=None, w_offset=0, std=2.0):
    gen = torch.Generator().manual_seed(seed)
    x, w = rows(T, K, dtype, gen, 1.0, x_ld, x_offset), rows(V, K, dtype, gen, std / math.sqrt(K), w_ld, w_offset)
    targets = torch.randint(0, V, (T,), generator=gen)
    targets[::5] = -100
    return x, w, targets, torch.rand(T, generator=gen) - 0.3


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,V,K", [(20, 1500, 64), (300, 1000, 128), (1044, 5000, 40)])
@pytest.mark.parametrize("which", ["x", "w", "neither"])
def test_one_operand_is_copied(T, V, K, dtype, which):
    print("[case] one copied", T, V, K, dtype, which, flush=True)
    x, w, targets, dloss = inputs(T, V, K, dtype, 3, x_ld=K + 1 if which == "x" else K, x_offset=which == "x", w_ld=K + 1 if which == "w" else K, w_offset=which == "w")
    compare(x, w, targets, 0.75, dloss, run(x, w, targets.cuda(), 0.75, dloss.cuda()))


def test_statistics_of_a_copied_operand_fit_the_queried_workspace():
    """X one element off: the tile follows the whole vocabulary and has narrower waves than that of 256 words."""
    print("[case] copied x, 15348 x 1044 x 8", flush=True)
    x, w, targets, _ = inputs(15348, 1044, 8, torch.bfloat16, 4, x_offset=1)
    loss, lse = torch.empty(15348, device="cuda"), torch.empty(15348, device="cuda")
    fg.fg_linear_xent(x, w, targets.cuda(), 1.0, loss, lse)
    plain, plain_lse = torch.empty_like(loss), torch.empty_like(lse)
    fg.fg_linear_xent(x.contiguous().clone(), w, targets.cuda(), 1.0, plain, plain_lse)
    assert torch.equal(loss, plain) and torch.equal(lse, plain_lse)


@pytest.mark.parametrize("T,V", [(3, 2 ** 22 + 5000), (31, 2 ** 22 + 3)])
def test_more_words_than_a_row_of_dz_holds(T, V):
    """Few tokens whose dz would be one piece by its size, but of rows longer than a product takes."""
    print("[case] many words", T, V, flush=True)
    x, w, targets, dloss = inputs(T, V, 8, torch.bfloat16, 6)
    targets[1] = V - 1
    compare(x, w, targets, 1.0, dloss, run(x, w, targets.cuda(), 1.0, dloss.cuda()), norms=False)


def test_captured_calls_with_workspaces_of_their_own_run_side_by_side():
    """Two graphs, each with the gradient of its own loss (a product with dX that is split over K), replayed on two streams at a time."""
    fg.fg_init()
    T, V, K = 300, 20000, 256
    graphs, outs, firsts, keep = [], [], [], []
    for seed in (1, 2):
        x, w, targets, dloss = inputs(T, V, K, torch.bfloat16, seed)
        targets, dloss = targets.cuda(), dloss.cuda()
        loss, lse, dx, dw = run(x, w, targets, 0.5, dloss)
        firsts.append((dx, dw))
        mine, ws = (torch.empty_like(dx), torch.empty_like(dw)), torch.empty(fg.fg_linear_xent_grad_workspace(T, V, K), dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            fg.fg_linear_xent_grad(x, w, targets, 0.5, lse, dloss, *mine, workspace=ws)
        graphs.append(graph); outs.append(mine); keep.append((x, w, targets, dloss, lse, ws))
    streams = [torch.cuda.Stream() for _ in graphs]
    for _ in range(10):
        for o in outs:
            for t in o:
                t.fill_(float("nan"))
        torch.cuda.synchronize()
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for got, want in zip(outs, firsts):
            assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("T,V,K,shift", [(20, 700, 64, 0), (50, 700, 63, 0), (64, 300, 128, 1), (65, 700, 64, 0), (300, 2000, 128, 0), (300, 1001, 99, 1)])
def test_what_a_left_out_token_holds_has_no_part_in_a_gradient(T, V, K, shift, value, dtype):
    """Rows of X, and values of dloss, of tokens without a target: dX is zero there, and dW that of a call where they hold nothing unusual, bit by bit."""
    print("[case] left out", T, V, K, shift, value, dtype, flush=True)
    x, w, targets, dloss = inputs(T, V, K, dtype, 9, x_ld=K + shift)
    out = targets < 0
    targets[out & (torch.arange(T) % 2 == 0)] = V
    targets, dloss = targets.cuda(), dloss.cuda()
    loss, lse, dx, dw = run(x, w, targets, 0.5, dloss)
    x[out.cuda()] = value
    dloss[out.cuda()] = value
    loss2, lse2, dx2, dw2 = run(x, w, targets, 0.5, dloss)
    assert torch.isfinite(dw).all() and torch.equal(dw, dw2) and torch.equal(dx, dx2) and torch.equal(loss, loss2)
    assert (dx2[out.cuda()] == 0).all() and torch.equal(lse[~out.cuda()], lse2[~out.cuda()])


@pytest.mark.parametrize("T", [20, 300])
def test_left_out_tokens_have_no_gradient_where_the_vocabulary_matrix_is_not_finite(T):
    """A word whose logits are all minus infinity (its probability is zero): dX of left-out tokens stays zero."""
    x, w, targets, dloss = inputs(T, 700, 64, torch.bfloat16, 10)
    x.abs_()
    w[13] = float("-inf")
    targets[targets == 13] = 14
    loss, lse, dx, dw = run(x, w, targets.cuda(), 1.0, dloss.cuda())
    assert torch.isfinite(lse).all() and (dx[(targets < 0).cuda()] == 0).all()
    keep = torch.arange(700) != 13
    assert torch.isfinite(dw[keep.cuda()]).all() and (dw[13] == 0).all()


@pytest.mark.parametrize("K", [16, 15])
def test_more_tokens_than_a_block(K):
    """The statistics of 16384 tokens are kept at a time; the last block is shorter.  With 15 values a row both operands are copied, block by block."""
    T, V = 16384 + 77, 300
    print("[case] blocks", T, V, K, flush=True)
    x, w, targets, dloss = inputs(T, V, K, torch.bfloat16, 12)
    compare(x, w, targets, 1.0, dloss, run(x, w, targets.cuda(), 1.0, dloss.cuda()))


def test_rows_without_values():
    """All logits are zero."""
    for T, V in ((5, 7), (300, 3000)):
        x, w = torch.empty(T, 0, dtype=torch.float16, device="cuda"), torch.empty(V, 0, dtype=torch.float16, device="cuda")
        targets = torch.arange(T, device="cuda") % V
        targets[2] = -1
        loss, lse, dx, dw = run(x, w, targets, 1.0, torch.ones(T, device="cuda"))
        want = torch.full((T,), math.log(V), dtype=torch.float64)
        assert ((lse.double().cpu() - want).abs() <= (V / 256 + 400) * U).all()
        want[2] = 0
        assert ((loss.double().cpu() - want).abs() <= (V / 256 + 400) * U).all() and loss[2] == 0
