"""GPU tests of fg_embedding and fg_embedding_grad against the formulas in 64 bits on the CPU.

Tolerances (u = 2^-24, e = half a unit in the last place of the result's type): a looked-up value is one FP32 product, rounded once:
(e + u) |y|.  A sum of m values of FP32 is within (m + 2) u of the sum of the magnitudes whatever the order, and rounded once.
With values that are small integers and a scale that is a power of two every sum is exact, and so is the result if it fits the type."""
import pytest
import torch

from paper_2009_12263_amd import binding as fg

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF_ULP = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}


def rows(n, cols, dtype, g, ld=None, offset=0, ints=False, scale=1.0):
    ld = ld or cols
    buf = torch.full((n * ld + offset + 8,), float("nan"), dtype=dtype)
    v = buf[offset:offset + n * ld].view(n, ld)[:, :cols]
    v.copy_((torch.randint(-3, 4, (n, cols), generator=g).float() if ints else torch.randn(n, cols, generator=g) * scale).to(dtype))
    return buf.cuda()[offset:offset + n * ld].view(n, ld)[:, :cols]


def ids_of(kind, tokens, vocab, g):
    if kind == "uniform":
        return torch.randint(0, vocab, (tokens,), generator=g)
    if kind == "one":
        return torch.full((tokens,), vocab - 1)
    if kind == "none":
        return torch.randint(-5, 0, (tokens,), generator=g)
    if kind == "skewed":
        return (torch.rand(tokens, generator=g) ** 6 * vocab).long().clamp(max=vocab - 1)
    if kind == "sorted":
        return torch.sort(torch.randint(0, vocab, (tokens,), generator=g))[0]
    ids = torch.randint(0, vocab, (tokens,), generator=g)           # "some": with ids that name no row, far outside too
    ids[::3] = -1
    ids[1::7] = vocab
    ids[2::11] = 2 ** 40 + 3
    return ids


def check(tokens, vocab, dim, dtype, out=None, kind="uniform", scale=0.75, add="", ints=False, ld=None, offset=0, index=torch.int64, seed=3, broadcast=False):
    print("[case] embedding", tokens, vocab, dim, dtype, out, kind, add, flush=True)
    out = out or dtype
    g = torch.Generator().manual_seed(seed)
    ids = ids_of(kind, tokens, vocab, g)
    if index == torch.int32:
        ids = torch.where(ids > 2 ** 31 - 1, torch.tensor(-1), ids)
    table, dy = rows(vocab, dim, dtype, g, ld, offset, ints), rows(tokens, dim, dtype, g, ld, offset, ints)
    if broadcast:
        dy = dy[:1].expand(tokens, dim)
    dev_ids = ids.to(index).cuda()
    has = (ids >= 0) & (ids < vocab)
    at = ids[has]
    y = torch.full((tokens, ld or dim), float("nan"), dtype=dtype, device="cuda")[:, :dim]
    fg.fg_embedding(table, dev_ids, scale, y)
    want = torch.zeros(tokens, dim, dtype=torch.float64)
    want[has] = table.double().cpu()[at] * scale
    assert ((y.double().cpu() - want).abs() <= (HALF_ULP[dtype] + U) * want.abs() + TINY[dtype]).all()
    assert (y[(~has).cuda()] == 0).all()

    there = rows(vocab, dim, out, g, ld, offset, ints) if add else None
    d = there.clone() if add == "in place" else torch.full((vocab, ld or dim), float("nan"), dtype=out, device="cuda")[:, :dim]
    fg.fg_embedding_grad(dy, dev_ids, scale, d if add == "in place" else there, d)
    sums, mags = torch.zeros(vocab, dim, dtype=torch.float64), torch.zeros(vocab, dim, dtype=torch.float64)
    sums.index_add_(0, at, dy.double().cpu()[has] * scale)
    mags.index_add_(0, at, (dy.double().cpu()[has] * scale).abs())
    n = torch.bincount(at, minlength=vocab).double()[:, None]
    want = sums + there.double().cpu() if add else sums
    if add:
        mags += there.double().cpu().abs()
    err = (d.double().cpu() - want).abs()
    if ints and scale in (0.5, 1.0, 2.0):
        assert torch.equal(d.cpu(), want.to(out))
    else:
        assert (err <= HALF_ULP[out] * want.abs() + TINY[out] + (n + 2) * U * mags).all(), float(err.max())
    untouched = (n[:, 0] == 0).cuda()
    assert torch.equal(d[untouched], there[untouched] if add else torch.zeros_like(d[untouched]))


TYPES = [(torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float16, torch.float16), (torch.float16, torch.float32), (torch.float32, torch.float32)]


@pytest.mark.parametrize("dtype,out", TYPES)
@pytest.mark.parametrize("tokens,vocab,dim", [(1, 1, 1), (1, 50, 8), (17, 33, 65), (100, 7, 300), (1000, 4097, 129), (4096, 500, 64), (4097, 1000, 40), (13000, 70000, 24)])
def test_sizes_and_types(tokens, vocab, dim, dtype, out):
    check(tokens, vocab, dim, dtype, out)


@pytest.mark.parametrize("kind", ["uniform", "one", "none", "skewed", "sorted", "some"])
@pytest.mark.parametrize("tokens", [15, 16, 33, 5000])
@pytest.mark.parametrize("add", ["", "beside", "in place"])
def test_ids(kind, tokens, add):
    check(tokens, 300, 72, torch.bfloat16, torch.float32, kind, add=add)
    check(tokens, 300, 72, torch.float32, torch.float32, kind, add=add, ints=True, scale=0.5)


def test_wide_rows_more_tokens_than_a_run_and_other_index_types():
    check(300, 50, 4096 + 8, torch.bfloat16, kind="skewed")
    check(70000, 60, 16, torch.float32, kind="some", ints=True, scale=2.0)
    check(70000, 3, 9, torch.float16, torch.float32, kind="uniform", ints=True, scale=1.0)
    check(500, 300, 72, torch.bfloat16, kind="some", index=torch.int32)
    check(500, (1 << 18) + 1, 8, torch.bfloat16, kind="uniform")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_strides_pointers_and_broadcast_gradients(dtype):
    check(129, 77, 1001, dtype, ld=1003, offset=1, kind="skewed", add="beside")
    check(129, 77, 1001, dtype, ld=1003, offset=1, kind="skewed", add="in place")
    check(129, 77, 64, dtype, broadcast=True, kind="some")


def test_no_tokens():
    ids = torch.empty(0, dtype=torch.int64, device="cuda")
    there = torch.randn(10, 5, device="cuda")
    d = torch.full((10, 5), float("nan"), device="cuda")
    fg.fg_embedding(there, ids, 1.0, torch.empty(0, 5, device="cuda"))
    fg.fg_embedding_grad(torch.empty(0, 5, device="cuda"), ids, 1.0, None, d)
    assert (d == 0).all()
    fg.fg_embedding_grad(torch.empty(0, 5, device="cuda"), ids, 1.0, there, d)
    assert torch.equal(d, there)


def test_non_finite_values_stay_in_their_row_and_in_that_of_their_id():
    table = torch.randn(20, 40, device="cuda"); table[3] = float("inf"); table[4] = float("nan")
    ids = torch.tensor([3, 5, -1, 4], device="cuda")
    y = torch.empty(4, 40, device="cuda")
    fg.fg_embedding(table, ids, 2.0, y)
    assert torch.isinf(y[0]).all() and torch.isfinite(y[1]).all() and (y[2] == 0).all() and torch.isnan(y[3]).all()
    dy = torch.ones(4, 40, device="cuda"); dy[2] = float("nan"); dy[3] = float("inf")
    d = torch.empty(20, 40, device="cuda")
    fg.fg_embedding_grad(dy, ids, 2.0, None, d)
    assert torch.isinf(d[4]).all() and torch.isfinite(torch.cat([d[:4], d[5:]])).all() and (d[3] == 2).all()


def test_repeats_streams_and_graph():
    g = torch.Generator().manual_seed(1)
    tokens, vocab, dim = 9000, 800, 200
    ids, dy = ids_of("skewed", tokens, vocab, g).cuda(), rows(tokens, dim, torch.bfloat16, g)
    first = torch.empty(vocab, dim, device="cuda")
    fg.fg_embedding_grad(dy, ids, 1.5, None, first)
    other = torch.empty_like(first)
    torch.cuda.synchronize()
    fg.fg_embedding_grad(dy, ids, 1.5, None, other, stream=torch.cuda.Stream())
    torch.cuda.synchronize()
    assert torch.equal(first, other)
    ws = torch.empty(fg.fg_embedding_grad_workspace(tokens, vocab, dim), dtype=torch.uint8, device="cuda")
    captured = torch.empty_like(first)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fg.fg_embedding_grad(dy, ids, 1.5, None, captured, workspace=ws)
    for _ in range(3):
        captured.fill_(float("nan")); ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(first, captured)


def test_offsets_beyond_32_bits():
    """A table of which the last rows begin past 2^32 bytes: small integers, exact."""
    vocab, dim, tokens = 600000, 4096, 200
    g = torch.Generator().manual_seed(7)
    ids = torch.cat([torch.randint(vocab - 50, vocab, (tokens // 2,), generator=g), torch.randint(0, vocab, (tokens // 2,), generator=g)]).cuda()
    table = torch.zeros(vocab, dim, dtype=torch.float16, device="cuda")
    table[ids] = rows(tokens, dim, torch.float16, g, ints=True)
    y = torch.empty(tokens, dim, dtype=torch.float16, device="cuda")
    fg.fg_embedding(table, ids, 2.0, y)
    assert torch.equal(y, table[ids] * 2)
    dy = rows(tokens, dim, torch.float16, g, ints=True)
    fg.fg_embedding_grad(dy, ids, 1.0, None, table)
    want = torch.zeros(tokens, dim, device="cuda")
    rows_of, at = torch.unique(ids, return_inverse=True)
    want.index_add_(0, at, dy.float())
    assert torch.equal(table[rows_of].float(), want[:len(rows_of)])
    table[rows_of] = 0
    assert not table.any()
