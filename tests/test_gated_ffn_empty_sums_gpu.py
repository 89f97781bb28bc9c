"""GPU test of the gated block of rows without values: G and U are empty sums, zero, and are written."""
import pytest
import torch

from paper_2009_12263_amd import binding as fg

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("tokens,hidden,ld", [(5, 24, 48), (3, 13, 40), (700, 100, 200)])
def test_kept_values_of_empty_rows(tokens, hidden, ld, dtype):
    memory = torch.full((tokens * ld + 8,), 7.0, device="cuda")
    gu = memory[1:1 + tokens * ld].view(tokens, ld)[:, :2 * hidden]
    empty = lambda rows, cols: torch.empty(rows, cols, device="cuda", dtype=dtype)
    fg.fg_gated_ffn(empty(tokens, 0), empty(2 * hidden, 0), empty(0, hidden), fg.FG_ACT_SILU, empty(tokens, 0), gu)
    assert not bool(gu.any())
    gu.fill_(7.0)
    assert bool((memory == 7.0).all())
