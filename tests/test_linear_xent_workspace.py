"""CPU test: the workspace that the queries of the linear cross entropy give is enough for rows of any alignment.  Without a GPU a call that
passes its checks ends at its first launch (FG_ERR_LAUNCH); the addresses are made up, so this does not run where there is one."""
import ctypes as C
import random
import re

import pytest
import torch

from paper_2009_12263_amd import binding as fg

pytestmark = pytest.mark.skipif(torch.cuda.device_count() > 0, reason="made-up addresses: not where a GPU would follow them")

PTR = 0x100000


def rows(ld, shift=0):
    return C.byref(fg.fg_matrix(PTR + 2 * shift, None, fg.FG_BF16, fg.FG_ROW, ld))


def forward(T, V, K, x_shift, w_shift):
    lib = fg.load_library()
    return lib.fg_linear_xent(T, V, K, rows(K, x_shift), rows(K, w_shift), PTR, fg.FG_I64, 1.0, PTR, PTR, PTR, lib.fg_linear_xent_workspace(T, V, K), None)


def gradient(T, V, K, x_shift, w_shift):
    lib = fg.load_library()
    return lib.fg_linear_xent_grad(T, V, K, rows(K, x_shift), rows(K, w_shift), PTR, fg.FG_I64, 1.0, PTR, PTR, 1, rows(K), rows(K), PTR,
                                   lib.fg_linear_xent_grad_workspace(T, V, K), None)


@pytest.mark.parametrize("call", [forward, gradient])
@pytest.mark.parametrize("x_shift,w_shift", [(0, 0), (1, 0), (0, 1), (1, 1)])
def test_the_queried_workspace_serves_any_alignment(call, x_shift, w_shift):
    rng = random.Random(5)
    sizes = [(16384, 320, 256), (15348, 1044, 8), (32277, 548, 304), (13148, 636, 24), (4784, 3338, 728), (1, 1, 1), (1, 1, 8), (64, 100000, 72)]
    sizes += [(rng.randrange(1, 1 << rng.randrange(1, 17)), rng.randrange(1, 1 << rng.randrange(1, 18)), rng.randrange(1, 600) * rng.choice([1, 8])) for _ in range(2000)]
    refused = [s for s in sizes if call(*s, x_shift, w_shift) != fg.FG_ERR_LAUNCH]
    assert not refused, (len(refused), refused[:5], fg.fg_last_error())


@pytest.mark.parametrize("T,V,K", [(300, 20000, 256), (2048, 32768, 1024), (1999, 50001, 1536), (16, 4096, 64), (9000, 8500, 16), (8192, 131072, 4096)])
def test_partial_products_are_part_of_the_workspace(T, V, K):
    """A product with dX that is split over K: 4 bytes for each of its tiles' values and ranges, behind dz (2) and the sums of dX (4)."""
    words = min(max(2048, 2 ** 28 // (2 * T) // 256 * 256), (V + 7) // 8 * 8)
    need = 2 * T * words + 4 * T * K
    plan = fg.fg_gemm_plan(T, K, words, fg.FG_ROW, fg.FG_ROW, fg.FG_ROW, fg.FG_PLAN_REAL_BF16)
    bm, bn, splits = (int(v or 1) for v in re.search(r"_(\d+)x(\d+)x64(?:_[a-z0-9]+)*(?:\+splitk(\d+))?", plan).groups())
    assert (splits > 1) == (V < 100000), plan
    if splits > 1:          # (the planner's rows are D's columns)
        need += 4 * splits * (-(-K // bm) * bm) * (-(-T // bn) * bn)
    assert fg.load_library().fg_linear_xent_grad_workspace(T, V, K) >= need
