"""GPU test of where a NaN of one column of G or U goes: into every result that the formulas put it in, and into no other, whichever kernels a size takes."""
import pytest
import torch

from paper_2009_12263_amd import binding as fg
from tests.test_gated_ffn_gpu import ACTS

pytestmark = pytest.mark.gpu

# few tokens, two parts by passes, split products with passes over their sums, tiled products with epilogues, copies
SIZES = [(3, 136, 72), (100, 64, 72), (130, 1024, 72), (64, 2048, 520), (700, 256, 512), (2101, 203, 331), (1290, 1024, 264)]


@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("of_gate", [True, False])
def test_a_column_without_a_number(size, act, of_gate):
    T, D, H = size
    g = torch.Generator(device="cuda").manual_seed(T)
    new = lambda rows, cols, std=1.0: (torch.randn(rows, cols, generator=g, device="cuda") * std).bfloat16()
    x, dy, w_in, w_out = new(T, D), new(T, D), new(2 * H, D, D ** -0.5), new(D, H, H ** -0.5)
    at = H - 5
    w_in[at if of_gate else H + at] = float("nan")
    y, dx, dw_in, dw_out = (torch.zeros_like(m) for m in (x, x, w_in, w_out))
    gu = torch.zeros(T, 2 * H, device="cuda")
    fg.fg_gated_ffn(x, w_in, w_out, ACTS[act], y, gu)
    fg.fg_gated_ffn_grad(dy, x, w_in, w_out, ACTS[act], gu, dx, dw_in, dw_out)
    assert bool(y.isnan().all()) and bool(dx.isnan().all())
    columns = torch.zeros(2 * H, dtype=torch.bool, device="cuda")
    columns[at if of_gate else H + at] = True
    assert torch.equal(gu.isnan(), columns.expand(T, -1))
    # dG = dH U act'(G): of a NaN in U, and of one in G but where the activation is none; dU = dH act(G): of one in G
    rows = torch.zeros_like(columns)
    rows[at] = not of_gate or act != "none"
    rows[H + at] = of_gate
    assert torch.equal(dw_in.isnan(), rows[:, None].expand(-1, D))
    only = torch.zeros(H, dtype=torch.bool, device="cuda")
    only[at] = True
    assert torch.equal(dw_out.isnan(), only.expand(D, -1))


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_an_infinite_gate_has_the_same_derivative_at_every_size(act):
    seen = set()
    for T, D, H in SIZES:
        x, dy = (torch.ones(T, D, device="cuda", dtype=torch.bfloat16) for _ in range(2))
        w_in, w_out = torch.full((2 * H, D), 0.01, device="cuda", dtype=torch.bfloat16), torch.full((D, H), 0.01, device="cuda", dtype=torch.bfloat16)
        gu = torch.ones(T, 2 * H, device="cuda")
        gu[:, 1] = float("inf")
        dw_in = torch.zeros_like(w_in)
        fg.fg_gated_ffn_grad(dy, x, w_in, w_out, ACTS[act], gu, dW_in=dw_in)
        assert torch.isfinite(dw_in[0]).all() and torch.isfinite(dw_in[2:H]).all()
        seen.add((bool(dw_in[1].isnan().all()), bool(dw_in[1].isfinite().all())))
    assert len(seen) == 1 and any(*seen), seen
