"""CPU test of sizes of the gated feed-forward block at the ends of 64 bits: refused, and without a workspace."""
import pytest

from paper_2009_12263_amd import binding as fg
from tests.test_middle_operators_abi import ffn, ffn_grad, row

MOST = (1 << 63) - 1


@pytest.mark.parametrize("call", [ffn, ffn_grad])
@pytest.mark.parametrize("size", [dict(hidden=1 << 62), dict(hidden=MOST), dict(hidden=(1 << 62) + (1 << 20)), dict(tokens=MOST), dict(dim=MOST), dict(tokens=MOST, dim=MOST, hidden=MOST),
                                  dict(tokens=1 << 30, hidden=1 << 19), dict(dim=(1 << 21) - 8), dict(hidden=(1 << 20) - 4)])
def test_refused(call, size):
    wide = {k: row(ld=MOST, re=0x100000000 * (i + 1)) for i, k in enumerate(("X", "W_in", "W_out"))}
    assert call(**size, **wide, size=0) == fg.FG_ERR_UNSUPPORTED, fg.fg_last_error()


@pytest.mark.parametrize("tokens,dim,hidden", [(1, 8, 1 << 62), (1, 8, MOST), (MOST, 8, 8), (1, MOST, 8), (MOST, MOST, MOST), (1 << 30, 8, 1 << 19), (1, (1 << 21) - 8, 8), (1, 8, (1 << 20) - 4)])
def test_no_workspace(tokens, dim, hidden):
    assert fg.fg_gated_ffn_workspace(tokens, dim, hidden) == 0 and fg.fg_gated_ffn_grad_workspace(tokens, dim, hidden) == 0


def test_largest_sizes_have_one():
    for size in ((1 << 18, 4096, 10240), (1, (1 << 21) - 9, 8), (1, 8, (1 << 20) - 5), (1 << 24, 8, 8)):
        assert fg.fg_gated_ffn_workspace(*size) > 0 and fg.fg_gated_ffn_grad_workspace(*size) > 0, size
