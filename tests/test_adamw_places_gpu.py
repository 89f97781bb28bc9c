"""GPU tests of AdamW on lists whose tensors lie where a program's do: allocated one by one, in any order, one kind of array between those of another.  Results are those of calls with one
tensor each, to the bit."""
import random

import pytest
import torch

from paper_2009_12263_amd import binding as fg
from tests.test_adamw_lists_gpu import NAMES, Lists, one_by_one, same

pytestmark = pytest.mark.gpu


class Own(Lists):
    """Every array in memory of its own."""

    def put(self, values, align=4):
        return values.cuda()


def reordered(lists, order):
    for name in NAMES:
        items = getattr(lists, name)
        if items:
            setattr(lists, name, [items[i] for i in order])


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("kind,count", [("own", 5), ("own", 193), ("own", 700), ("packed", 193), ("packed", 5)])
def test_order_does_not_matter(kind, count, bits):
    """Packed: each tensor's arrays beside each other (the kinds lie between each other's)."""
    want = one_by_one(count, bits)
    for shuffled in (False, True):
        memory = torch.zeros(count * 16384, dtype=torch.uint8, device="cuda")
        lists = Own(count, bits, None) if kind == "own" else Lists(count, bits, memory)
        order = list(range(count))
        if shuffled:
            random.Random(count).shuffle(order)
        reordered(lists, order)
        lists.step()
        reordered(lists, [order.index(i) for i in range(count)])
        assert same(lists.bytes(), want)


def test_gradients_may_be_shared():
    """Two parameters with the same gradient, which is only read."""
    grad = torch.randn(5000, device="cuda")
    params = [torch.ones(5000, device="cuda") for _ in range(2)]
    avg, sq = ([torch.zeros(5000, device="cuda") for _ in range(2)] for _ in range(2))
    step = torch.ones(1, dtype=torch.int64, device="cuda")
    fg.fg_adamw(params, [grad, grad], avg, sq, step, 1e-2, 0.9, 0.99, 1e-8, 0.1)
    assert torch.equal(params[0], params[1]) and not torch.equal(params[0], torch.ones_like(params[0]))
    with pytest.raises(fg.FlexGemmError, match="in common"):
        fg.fg_adamw(params, [grad, params[0]], avg, sq, step, 1e-2, 0.9, 0.99, 1e-8, 0.1)
    with pytest.raises(fg.FlexGemmError, match="in common"):
        fg.fg_adamw(params, [grad, grad], [avg[0], sq[0]], sq, step, 1e-2, 0.9, 0.99, 1e-8, 0.1)
    with pytest.raises(fg.FlexGemmError, match="in common"):
        fg.fg_adamw([params[0], params[0]], [grad, grad], avg, sq, step, 1e-2, 0.9, 0.99, 1e-8, 0.1)
