"""CPU test: a layer norm in place whose rows would lie elsewhere than the operand's is refused (workgroups would write what others read)."""
import ctypes as C

import pytest

from paper_2009_12263_amd import binding as fg

PTR, OTHER = 0x100000, 0x900000


def row(re=PTR, ld=64):
    return C.byref(fg.fg_matrix(re, None, fg.FG_BF16, fg.FG_ROW, ld))


def layernorm(X, Y):
    return fg.load_library().fg_layernorm(4, 64, X, None, None, fg.FG_F32, 1e-5, Y, None, None, None)


def gradient(dY, X, dX):
    return fg.load_library().fg_layernorm_grad(4, 64, dY, X, None, fg.FG_F32, PTR, PTR, dX, None, None, None, 0, None)


@pytest.mark.parametrize("call,args,word", [
    (layernorm, (row(), row(ld=72)), "Y in the place of X"),
    (gradient, (row(OTHER), row(), row(ld=72)), "dX in the place of X"),
    (gradient, (row(OTHER, 64), row(), row(OTHER, 65)), "dX in the place of dY"),
    (gradient, (row(OTHER, 0), row(), row(OTHER, 64)), "dX in the place of dY"),
])
def test_rows_elsewhere_are_refused(call, args, word):
    assert call(*args) == fg.FG_ERR_LAYOUT and word in fg.fg_last_error()
