"""CPU test: what fg_linear_xent_grad cannot compute it refuses before anything is launched.  Without a GPU a launch ends a call with FG_ERR_LAUNCH; the
addresses are made up, so this does not run where there is one."""
import ctypes as C

import pytest
import torch

from paper_2009_12263_amd import binding as fg

pytestmark = pytest.mark.skipif(torch.cuda.device_count() > 0, reason="made-up addresses: not where a GPU would follow them")

PTR = 0x100000


def gradient(tokens, vocab, dim):
    rows = C.byref(fg.fg_matrix(PTR, None, fg.FG_BF16, fg.FG_ROW, dim))
    return fg.load_library().fg_linear_xent_grad(tokens, vocab, dim, rows, rows, PTR, fg.FG_I64, 1.0, PTR, PTR, 1, rows, rows, PTR, 1 << 45, None)


@pytest.mark.parametrize("dim,status", [(2 ** 21 - 4, fg.FG_ERR_LAUNCH), (2 ** 21 - 3, fg.FG_ERR_UNSUPPORTED), (2 ** 21 - 1, fg.FG_ERR_UNSUPPORTED), (2 ** 21, fg.FG_ERR_UNSUPPORTED)])
def test_rows_that_the_sums_of_dx_cannot_have(dim, status):
    assert gradient(4, 100, dim) == status


@pytest.mark.parametrize("tokens", [1, 16, 31, 32])
def test_pieces_of_few_tokens_are_rows_that_a_product_takes(tokens):
    """A row of dz in the workspace stays below 2^22 words however large the vocabulary."""
    lib = fg.load_library()
    most = lib.fg_linear_xent_grad_workspace(tokens, 2 ** 30, 8)
    assert most == lib.fg_linear_xent_grad_workspace(tokens, 2 ** 22, 8)
    assert gradient(tokens, 2 ** 30, 8) == fg.FG_ERR_LAUNCH         # (accepted)
