"""GPU tests of the operators on rows at sizes whose launches have 2^32 threads and more, which are made in parts."""
import pytest
import torch

from paper_2009_12263_amd import binding as fg

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _leaves_the_memory_to_others():
    yield
    torch.cuda.empty_cache()


def _needs(gigabytes):
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gigabytes * 10 ** 9:
        pytest.skip("%d GB of GPU memory are needed" % gigabytes)


def test_more_wide_rows_than_a_launch_holds():
    """2^22 + 3 rows of 8193 FP32 values in place, a workgroup of 1024 threads each: some of them against the same rows by themselves (which other tests
    check), all others are zero before and after."""
    _needs(160)
    rows, cols = (1 << 22) + 3, 8193
    print("[case] layernorm", rows, cols, flush=True)
    pick = torch.tensor([0, 1, (1 << 21) - 1, 1 << 21, (1 << 21) + 1, (1 << 22) - 1, 1 << 22, rows - 1], device="cuda")
    g = torch.Generator().manual_seed(1)
    part, dy = torch.randn(len(pick), cols, generator=g).cuda(), torch.randn(1, cols, generator=g).cuda()
    gamma = (torch.randn(cols, generator=g) * 0.3 + 1).cuda()
    x = torch.zeros(rows, cols, device="cuda")
    x[pick] = part
    m, s = torch.full((rows,), float("nan"), device="cuda"), torch.full((rows,), float("nan"), device="cuda")
    fg.fg_layernorm(x, gamma, None, 1e-5, x, m, s)
    y, m2, s2 = torch.empty_like(part), torch.empty(len(pick), device="cuda"), torch.empty(len(pick), device="cuda")
    fg.fg_layernorm(part, gamma, None, 1e-5, y, m2, s2)
    assert torch.equal(x[pick], y) and torch.equal(m[pick], m2) and torch.equal(s[pick], s2)
    x[pick] = 0
    assert not any(x[i:i + (1 << 19)].any() for i in range(0, rows, 1 << 19)) and torch.isfinite(s).all()
    x[pick] = part
    fg.fg_layernorm_grad(dy.expand(rows, cols), x, gamma, m, s, x)
    dx = torch.empty_like(part)
    fg.fg_layernorm_grad(dy.expand(len(pick), cols), part, gamma, m2, s2, dx)
    assert torch.equal(x[pick], dx)
    dx0 = torch.empty_like(dy)
    fg.fg_layernorm_grad(dy, torch.zeros_like(dy), gamma, torch.zeros(1, device="cuda"), s[2:3].clone(), dx0)
    x[pick] = dx0
    assert all((x[i:i + (1 << 19)] == dx0).all() for i in range(0, rows, 1 << 19))


def test_sums_of_more_columns_than_a_launch_holds():
    """2^26 + 5 columns, 2^27 + 10 sums: with one row dbeta is dY itself and dgamma is dY (X - mean) rstd, three roundings either way."""
    cols = (1 << 26) + 5
    print("[case] layernorm gradient", 1, cols, flush=True)
    x, dy = torch.randn(1, cols, device="cuda").half(), torch.randn(1, cols, device="cuda").half()
    m, s = torch.full((1,), 0.25, device="cuda"), torch.full((1,), 1.5, device="cuda")
    dgamma, dbeta = (torch.full((cols,), float("nan"), device="cuda") for _ in range(2))
    dx = torch.empty_like(x)
    fg.fg_layernorm_grad(dy, x, None, m, s, dx, dgamma, dbeta)
    assert torch.equal(dbeta, dy[0].float())
    want = dy[0].double() * ((x[0].double() - 0.25) * 1.5)
    assert ((dgamma.double() - want).abs() <= 4 * 2.0 ** -24 * want.abs()).all()


def test_more_tokens_than_a_launch_holds():
    """2^30 tokens of rows of 66 values, 16 to a wave: 2^32 lanes."""
    _needs(200)
    tokens, dim, vocab = 1 << 30, 66, 5
    print("[case] embedding", tokens, dim, flush=True)
    table = torch.randint(-9, 10, (vocab, dim), device="cuda").half()
    ids = torch.empty(tokens, dtype=torch.int32, device="cuda").random_(-1, vocab)
    y = torch.full((tokens, dim), float("nan"), dtype=torch.float16, device="cuda")
    fg.fg_embedding(table, ids, 2.0, y)
    twice = torch.cat([table * 2, torch.zeros(1, dim, dtype=torch.float16, device="cuda")])
    for i in range(0, tokens, 1 << 25):
        assert torch.equal(y[i:i + (1 << 25)], twice[ids[i:i + (1 << 25)].long() % (vocab + 1)]), i
