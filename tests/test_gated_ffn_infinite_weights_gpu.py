"""GPU test of an infinite weight of the gated block: its column of a result is infinite, with the sign that the formulas give it, at every size; where results are few and H, dG and dU have a
second part (which may be zero, or of the other sign), too."""
import pytest
import torch

from paper_2009_12263_amd import binding as fg
from tests.test_gated_ffn_gpu import act64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("size", [(1, 160, 128), (3, 65, 600), (8, 300, 264), (16, 129, 77), (30, 80, 96), (70, 100, 100), (100, 64, 72), (130, 1024, 72), (700, 256, 512)])
def test_signs(size, dtype):
    T, D, H = size
    g = torch.Generator(device="cuda").manual_seed(T)
    new = lambda rows, cols, std=1.0: (torch.randn(rows, cols, generator=g, device="cuda") * std).to(dtype)
    x, dy, w_in, w_out = new(T, D), new(T, D), new(2 * H, D, D ** -0.5), new(D, H, H ** -0.5)
    y, dx, gu = torch.zeros_like(x), torch.zeros_like(x), torch.zeros(T, 2 * H, device="cuda")
    inf, at, other = float("inf"), D // 3, H - 3
    fg.fg_gated_ffn(x, w_in, w_out, fg.FG_ACT_SILU, y, gu)
    plain = y.clone()
    a = act64(gu[:, :H].double(), "silu")[0]
    h, du = a * gu[:, H:].double(), dy.double() @ w_out.double() * a
    far = w_out.clone()
    far[at, other] = inf
    fg.fg_gated_ffn(x, w_in, far, fg.FG_ACT_SILU, y, gu)
    assert torch.equal(y[:, at].double(), h[:, other].sign() * inf)
    keep = torch.arange(D, device="cuda") != at
    assert torch.equal(y[:, keep], plain[:, keep])
    fg.fg_gated_ffn_grad(dy, x, w_in, w_out, fg.FG_ACT_SILU, gu, dx)
    plain = dx.clone()
    far = w_in.clone()
    far[H + other, at] = -inf
    fg.fg_gated_ffn_grad(dy, x, far, w_out, fg.FG_ACT_SILU, gu, dx)
    assert torch.equal(dx[:, at].double(), du[:, other].sign() * -inf)
    assert torch.equal(dx[:, keep], plain[:, keep])
