"""Tests of how exact the gated feed-forward block is where results are few (tokens times the smaller of dim and hidden below 16384): H, dG and dU are then two 16-bit numbers
each, a value and what its rounding left, and results are as exact as their own rounding.

Tolerance.  A result is round(z) with z = exact + d.  How far a number is from the nearest 16-bit one changes by |d| at most where the number moves by d, so
|round(z) - exact| <= |round(exact) - exact| + 2 |d|, and the same holds for norms.  d has three parts, relative to the norm of a result: two parts of bfloat16 leave
2^-16 of a value, of binary16 2^-22; an activation is off by fewer than 2^-20; sums of up to 600 terms in FP32 round 600 times by 2^-24 of a partial sum, with signs of their own,
together less than 2^-19.  That is 2^-15 or less in bfloat16 and 2^-18 in binary16, where rounding is off by 0.42 of half a step's 2^-8 and 2^-11 (over the mantissas):
2 |d| is below 0.04 of it, and 0.1 is allowed.  Without the second parts the rounding of H comes on top of that of the result, 1.4 times as much in all: the first
test shows on the CPU that this, and the second part of another token, are seen at every size."""
import pytest
import torch

from paper_2009_12263_amd import binding as fg
from tests.test_gated_ffn_gpu import ACTS, act64

# rows of both parts: 2 to 16, 18 to 32, 60 to 64 (the kernel for few tokens), 80 to 300 (products and passes); up to 64 also for the weights' gradients
SIZES = [(1, 160, 128), (2, 224, 224), (3, 65, 600), (8, 300, 264), (9, 500, 120), (16, 129, 77), (30, 80, 96), (32, 75, 203), (40, 120, 88), (70, 100, 100), (71, 101, 99), (150, 96, 104)]
TYPES = [torch.bfloat16, torch.float16]
NAMES = ("y", "dx", "dw_in", "dw_out")
ALLOWED = 1.1


class Operands:
    def __init__(self, tokens, dim, hidden, dtype):
        g = torch.Generator().manual_seed(tokens + dim)
        new = lambda rows, cols, std: (torch.randn(rows, cols, generator=g) * std).to(dtype)
        self.x, self.dy, self.w_in, self.w_out = new(tokens, dim, 1.0), new(tokens, dim, 0.25), new(2 * hidden, dim, 1.5 * dim ** -0.5), new(dim, hidden, hidden ** -0.5)
        self.hidden, self.act = hidden, ("silu", "gelu", "relu", "none")[(tokens + hidden) % 4]

    def results(self, held=lambda v: v):
        """The formulas in 64 bits with H, dG and dU as they are held."""
        x, dy, w_in, w_out = (m.double() for m in (self.x, self.dy, self.w_in, self.w_out))
        g, u = (x @ w_in.T).split(self.hidden, 1)
        a, d = act64(g, self.act)
        h, dh = held(a * u), dy @ w_out
        dgu = torch.cat([held(dh * u * d), held(dh * a)], 1)
        return dict(y=h @ w_out.T, dx=dgu @ w_in, dw_in=dgu.T @ x, dw_out=dy.T @ h)


def ratio(got, exact, dtype):
    """The error, as a multiple of that of rounding alone."""
    return float((got.to(dtype).double() - exact).norm() / (exact.to(dtype).double() - exact).norm())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", SIZES)
def test_what_the_second_parts_are_worth(size, dtype):
    c = Operands(*size, dtype)
    exact = c.results()
    first = lambda v: v.to(dtype).double()
    second = lambda v: (v - first(v)).to(dtype).double()
    both, alone = c.results(lambda v: first(v) + second(v)), c.results(first)
    other = c.results(lambda v: first(v) + second(v).roll(1, 0)) if size[0] > 1 else alone
    for name in NAMES:
        assert ratio(both[name], exact[name], dtype) <= 1.02, name
        for wrong in (alone, other):
            assert ratio(wrong[name], exact[name], dtype) > 1.05 * ALLOWED, (name, ratio(wrong[name], exact[name], dtype))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", SIZES)
def test_few_results_are_as_exact_as_their_rounding(size, dtype):
    c = Operands(*size, dtype)
    exact = c.results()
    x, dy, w_in, w_out = (m.cuda() for m in (c.x, c.dy, c.w_in, c.w_out))
    y, dx, dw_in, dw_out = (torch.full_like(m, 7.0) for m in (x, x, w_in, w_out))
    gu = torch.empty(size[0], 2 * size[2], device="cuda")
    fg.fg_gated_ffn(x, w_in, w_out, ACTS[c.act], y, gu)
    fg.fg_gated_ffn_grad(dy, x, w_in, w_out, ACTS[c.act], gu, dx, dw_in, dw_out)
    for name, got in zip(NAMES, (y, dx, dw_in, dw_out)):
        assert ratio(got.cpu(), exact[name], dtype) <= ALLOWED, (name, ratio(got.cpu(), exact[name], dtype))
