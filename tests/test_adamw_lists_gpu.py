"""GPU tests of long lists of tensors: the step's and the norm's results are those of calls with one tensor each, to the bit, wherever the tensors lie."""
import math

import pytest
import torch

from paper_2009_12263_amd import binding as fg

pytestmark = pytest.mark.gpu
NAMES = ["params", "grads", "masters", "avg", "sq", "avg_scales", "sq_scales"]


class Lists:
    """`count` tensors, all of them in `memory`: one behind the other from its start, the last one from `last` on where that is given."""

    def __init__(self, count, bits, memory, last=None, largest=0):
        g = torch.Generator().manual_seed(count)
        self.at, self.memory, self.bits = 0, memory, bits
        for name in NAMES:
            setattr(self, name, [])
        for i in range(count):
            if last is not None and i == count - 1:
                self.at = last
            n = 0 if i % 17 == 5 else 1 + (61 * i) % 900
            n = largest if largest and i == 3 else n
            blocks = (n + 255) // 256
            w = torch.randn(n, generator=g)
            self.params.append(self.put(w.to(torch.bfloat16)))
            self.grads.append(self.put((torch.randn(n, generator=g) * 0.01).to(torch.bfloat16 if i % 3 else torch.float32)))
            self.masters.append(self.put(w) if i % 2 else None)
            if bits == 8:
                self.avg.append(self.put((torch.randn(n, generator=g) * 100).to(torch.float8_e4m3fn), 16))
                self.sq.append(self.put((torch.rand(n, generator=g) * 400).to(torch.float8_e4m3fn), 16))
                self.avg_scales.append(self.put(torch.rand(blocks, generator=g) * 1e-3))
                self.sq_scales.append(self.put(torch.rand(blocks, generator=g) * 1e-4))
            else:
                self.avg.append(self.put(torch.randn(n, generator=g) * 0.01))
                self.sq.append(self.put(torch.rand(n, generator=g) * 1e-4))

    def put(self, values, align=4):
        self.at += -self.at % align
        size = values.numel() * values.element_size()
        there = self.memory[self.at:self.at + size].view(values.dtype)
        self.at += size
        return there.copy_(values)

    def step(self, begin=0, end=None):
        part = {name: getattr(self, name)[begin:end] for name in NAMES}
        fg.fg_adamw(part["params"], part["grads"], part["avg"], part["sq"], torch.full((1,), 4, dtype=torch.int64, device="cuda"), 3e-3, 0.9, 0.97, 1e-8, 0.1,
                    masters=part["masters"], avg_scales=part["avg_scales"] if self.bits == 8 else None, sq_scales=part["sq_scales"] if self.bits == 8 else None,
                    grad_factor=torch.full((1,), 0.5, device="cuda"))

    def bytes(self):
        return [t.reshape(-1).view(torch.uint8).cpu() if t is not None else None for name in NAMES for t in getattr(self, name)]


def same(a, b):
    return all((x is None) == (y is None) and (x is None or torch.equal(x, y)) for x, y in zip(a, b))


def one_by_one(count, bits, largest=0):
    lists = Lists(count, bits, torch.zeros(count * 16384 + largest * 22, dtype=torch.uint8, device="cuda"), None, largest)
    for i in range(count):
        lists.step(i, i + 1)
    return lists.bytes()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("count", [47, 49, 63, 64, 65, 95, 96, 97, 119, 120, 121, 127, 128, 129, 185, 241, 500])
def test_lengths_of_lists(count, bits):
    memory = torch.zeros(count * 16384, dtype=torch.uint8, device="cuda")
    lists = Lists(count, bits, memory)
    lists.step()
    assert same(lists.bytes(), one_by_one(count, bits))
    assert not bool(memory[lists.at:].any())


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("last", [2 ** 31 - 64, 2 ** 32, 2 ** 33 - 16384, 2 ** 33 - 64, 2 ** 33, 2 ** 34 + 2 ** 20, 2 ** 36 + 2 ** 30])
def test_tensors_far_from_each_other(last, bits):
    """Offsets from the first tensor to the last one of 31 to 37 bits."""
    memory = torch.empty(last + 2 ** 16, dtype=torch.uint8, device="cuda")
    for count in (100, 130):
        lists = Lists(count, bits, memory, last)
        lists.step()
        assert same(lists.bytes(), one_by_one(count, bits))


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("largest", [2 ** 23 - 70000, 2 ** 23 - 1, 2 ** 23, 2 ** 23 + 1])
def test_long_lists_with_a_large_tensor(largest, bits):
    count = 130
    lists = Lists(count, bits, torch.zeros(count * 16384 + largest * 22, dtype=torch.uint8, device="cuda"), None, largest)
    lists.step()
    assert same(lists.bytes(), one_by_one(count, bits, largest))


@pytest.mark.parametrize("count", [16, 17, 64, 65, 127, 128, 129, 300])
def test_norms_of_long_lists(count):
    lists = Lists(count, 32, torch.zeros(count * 16384, dtype=torch.uint8, device="cuda"))
    exact = math.sqrt(sum(float(g.double().square().sum()) for g in lists.grads))
    norm, factor = (torch.zeros(1, device="cuda") for _ in range(2))
    fg.fg_grad_norm(lists.grads, 1.0, 1e-3, norm, factor)
    assert abs(float(norm) - exact) <= 2 ** -22 * exact and abs(float(factor) - 1e-3 / exact) <= 2 ** -21 * 1e-3 / exact
