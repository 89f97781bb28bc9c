"""GPU test of fg_embedding_grad where more ids reach over the edges of tiles than there are workgroups to join them: small integers, exact."""
import pytest
import torch

from paper_2009_12263_amd import binding as fg
from tests.test_embedding_gpu import rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim", [40, 600])
@pytest.mark.parametrize("add", [False, True])
def test_a_workgroup_joins_several_ids(dim, add):
    tokens, vocab = 20000, 1500
    print("[case] embedding joins", dim, add, flush=True)
    g = torch.Generator().manual_seed(4)
    ids = torch.randint(-1, vocab, (tokens,), generator=g)
    ordered = torch.sort(torch.where(ids < 0, vocab, ids))[0]
    edge = torch.arange(16, tokens, 16)
    assert len(torch.unique(ordered[edge][(ordered[edge] == ordered[edge - 1]) & (ordered[edge] < vocab)])) > 2 * 512
    dy, there = rows(tokens, dim, torch.bfloat16, g, ints=True), rows(vocab, dim, torch.float32, g, ints=True)
    got = torch.full((vocab, dim), float("nan"), device="cuda")
    fg.fg_embedding_grad(dy, ids.cuda(), 2.0, there if add else None, got)
    want = torch.zeros(vocab, dim, dtype=torch.float64).index_add_(0, ids[ids >= 0], 2 * dy.double().cpu()[ids >= 0])
    assert torch.equal(got.double().cpu(), want + there.double().cpu() if add else want)
