"""Tests of a norm of gradients whose results would share memory with each other or with a gradient: refused."""
import pytest
import torch

from paper_2009_12263_amd import binding as fg
from tests.test_middle_operators_abi import PTR, norm

GRADS = ((1 << 20, 100, fg.FG_BF16), (1 << 21, 0, fg.FG_F32), (1 << 22, 64, fg.FG_F32))


@pytest.mark.parametrize("out,factor,word", [
    (PTR, PTR, "norm and factor"),
    ((1 << 20) + 196, PTR, "norm is in gradient 0"),
    ((1 << 22), PTR, "norm is in gradient 2"),
    (PTR, (1 << 22) + 252, "factor is in gradient 2"),
])
def test_refused(out, factor, word):
    assert norm(GRADS, out=out, factor=factor) == fg.FG_ERR_LAYOUT and word in fg.fg_last_error(), fg.fg_last_error()


@pytest.mark.gpu
def test_beside_them_is_not():
    """A gradient, and the results in the values before and behind it."""
    memory = torch.full((1002,), 3.0, device="cuda")
    for out, factor in ((0, 1001), (1001, 0)):
        fg.fg_grad_norm([memory[1:1001]], 1.0, 1.0, memory[out:out + 1], memory[factor:factor + 1])
        assert abs(float(memory[out]) - 9000 ** 0.5) <= 2 ** -23 * 100 and abs(float(memory[factor]) - 9000 ** -0.5) <= 2 ** -23 * 0.02
    assert bool((memory[1:1001] == 3.0).all())
