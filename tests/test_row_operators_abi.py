"""CPU tests: what the operators on rows refuse, and with which status, before anything is launched."""
import ctypes as C

import pytest
import torch

from paper_2009_12263_amd import binding as fg

PTR = 0x10000


def row(dtype=fg.FG_BF16, ld=64, re=PTR, layout=fg.FG_ROW, im=None):
    return C.byref(fg.fg_matrix(re, im, dtype, layout, ld))


def layernorm(rows=4, cols=64, X=None, gamma=PTR, beta=PTR, pt=fg.FG_F32, eps=1e-5, Y=None, mean=PTR, rstd=PTR):
    X = row() if X is None else X
    Y = row() if Y is None else Y
    return fg.load_library().fg_layernorm(rows, cols, X, gamma, beta, pt, eps, Y, mean, rstd, None)


def layernorm_grad(rows=4, cols=64, dY=None, X=None, gamma=PTR, pt=fg.FG_F32, mean=PTR, rstd=PTR, dX=None, dgamma=PTR, dbeta=PTR, ws=PTR, size=1 << 30):
    dY, X, dX = (row() if m is None else m for m in (dY, X, dX))
    return fg.load_library().fg_layernorm_grad(rows, cols, dY, X, gamma, pt, mean, rstd, dX, dgamma, dbeta, ws, size, None)


def embedding(tokens=4, vocab=100, dim=64, table=None, ids=PTR, kind=fg.FG_I64, Y=None):
    table, Y = (row() if m is None else m for m in (table, Y))
    return fg.load_library().fg_embedding(tokens, vocab, dim, table, ids, kind, 1.0, Y, None)


def embedding_grad(tokens=4, vocab=100, dim=64, dY=None, ids=PTR, kind=fg.FG_I64, Cin=None, dtable=None, ws=PTR, size=1 << 30):
    dY, dtable = (row() if m is None else m for m in (dY, dtable))
    return fg.load_library().fg_embedding_grad(tokens, vocab, dim, dY, ids, kind, 1.0, Cin, dtable, ws, size, None)


def xent(tokens=4, vocab=100, dim=64, X=None, W=None, targets=PTR, kind=fg.FG_I64, loss=PTR, lse=PTR, ws=PTR, size=1 << 40):
    X, W = (row() if m is None else m for m in (X, W))
    return fg.load_library().fg_linear_xent(tokens, vocab, dim, X, W, targets, kind, 1.0, loss, lse, ws, size, None)


def xent_grad(tokens=4, vocab=100, dim=64, X=None, W=None, targets=PTR, kind=fg.FG_I64, lse=PTR, dloss=PTR, inc=1, dX=None, dW=None, ws=PTR, size=1 << 40):
    X, W, dX, dW = (row() if m is None else m for m in (X, W, dX, dW))
    return fg.load_library().fg_linear_xent_grad(tokens, vocab, dim, X, W, targets, kind, 1.0, lse, dloss, inc, dX, dW, ws, size, None)


NULL = C.POINTER(fg.fg_matrix)()


@pytest.mark.parametrize("call,args,status,word", [
    (layernorm, dict(rows=-1), fg.FG_ERR_SHAPE, "negative"),
    (layernorm, dict(X=NULL), fg.FG_ERR_NULL, "X is NULL"),
    (layernorm, dict(Y=NULL), fg.FG_ERR_NULL, "Y is NULL"),
    (layernorm, dict(X=row(re=None)), fg.FG_ERR_NULL, "X->re"),
    (layernorm, dict(X=row(layout=fg.FG_COL)), fg.FG_ERR_LAYOUT, "row-major"),
    (layernorm, dict(X=row(dtype=fg.FG_CF16)), fg.FG_ERR_LAYOUT, "FG_F16, FG_BF16 or FG_F32"),
    (layernorm, dict(X=row(im=PTR)), fg.FG_ERR_LAYOUT, "real"),
    (layernorm, dict(X=row(ld=63)), fg.FG_ERR_SHAPE, "ld=63"),
    (layernorm, dict(X=row(ld=0)), fg.FG_ERR_SHAPE, "ld=0"),
    (layernorm, dict(X=row(re=PTR + 1)), fg.FG_ERR_ALIGN, "aligned"),
    (layernorm, dict(Y=row(dtype=fg.FG_F16)), fg.FG_ERR_UNSUPPORTED, "same element type"),
    (layernorm, dict(pt=fg.FG_F16), fg.FG_ERR_LAYOUT, "gamma"),
    (layernorm, dict(gamma=PTR + 2), fg.FG_ERR_ALIGN, "gamma"),
    (layernorm, dict(mean=PTR + 2), fg.FG_ERR_ALIGN, "mean"),
    (layernorm, dict(eps=-1.0), fg.FG_ERR_SHAPE, "eps"),
    (layernorm, dict(eps=float("nan")), fg.FG_ERR_SHAPE, "eps"),
    (layernorm, dict(rows=2 << 30), fg.FG_ERR_UNSUPPORTED, "2^30"),
    (layernorm_grad, dict(dY=NULL), fg.FG_ERR_NULL, "dY is NULL"),
    (layernorm_grad, dict(dX=row(ld=3)), fg.FG_ERR_SHAPE, "dX"),
    (layernorm_grad, dict(dY=row(dtype=fg.FG_F32)), fg.FG_ERR_UNSUPPORTED, "dY"),
    (layernorm_grad, dict(mean=None), fg.FG_ERR_NULL, "mean"),
    (layernorm_grad, dict(ws=None), fg.FG_ERR_NULL, "workspace"),
    (layernorm_grad, dict(size=100), fg.FG_ERR_SHAPE, "workspace"),
    (layernorm_grad, dict(dgamma=PTR + 1), fg.FG_ERR_ALIGN, "dgamma"),
    (layernorm_grad, dict(ws=PTR + 4), fg.FG_ERR_ALIGN, "workspace"),
    (embedding, dict(tokens=-1), fg.FG_ERR_SHAPE, "negative"),
    (embedding, dict(vocab=2 << 30), fg.FG_ERR_UNSUPPORTED, "2^30"),
    (embedding, dict(ids=None), fg.FG_ERR_NULL, "ids"),
    (embedding, dict(ids=PTR + 4), fg.FG_ERR_ALIGN, "ids"),
    (embedding, dict(kind=fg.FG_F32), fg.FG_ERR_LAYOUT, "FG_I32"),
    (embedding, dict(table=row(ld=63)), fg.FG_ERR_SHAPE, "table"),
    (embedding, dict(Y=row(dtype=fg.FG_F32)), fg.FG_ERR_UNSUPPORTED, "same element type"),
    (embedding_grad, dict(dY=NULL), fg.FG_ERR_NULL, "dY"),
    (embedding_grad, dict(dtable=row(dtype=fg.FG_F16)), fg.FG_ERR_UNSUPPORTED, "dtable"),
    (embedding_grad, dict(Cin=row(dtype=fg.FG_F32, re=2 * PTR)), fg.FG_ERR_UNSUPPORTED, "Cin"),
    (embedding_grad, dict(Cin=row(ld=128)), fg.FG_ERR_LAYOUT, "Cin"),
    (embedding_grad, dict(ws=None), fg.FG_ERR_NULL, "workspace"),
    (embedding_grad, dict(size=64), fg.FG_ERR_SHAPE, "workspace"),
    (xent, dict(dim=-8), fg.FG_ERR_SHAPE, "negative"),
    (xent, dict(vocab=0), fg.FG_ERR_SHAPE, "empty"),
    (xent, dict(vocab=2 << 30), fg.FG_ERR_UNSUPPORTED, "2^30"),
    (xent, dict(X=row(dtype=fg.FG_F32), W=row(dtype=fg.FG_F32)), fg.FG_ERR_UNSUPPORTED, "FG_F16"),
    (xent, dict(X=row(dtype=fg.FG_F16)), fg.FG_ERR_UNSUPPORTED, "both"),
    (xent, dict(W=row(layout=fg.FG_COL)), fg.FG_ERR_LAYOUT, "row-major"),
    (xent, dict(targets=None), fg.FG_ERR_NULL, "targets"),
    (xent, dict(loss=None), fg.FG_ERR_NULL, "loss"),
    (xent, dict(lse=PTR + 2), fg.FG_ERR_ALIGN, "lse"),
    (xent, dict(ws=None), fg.FG_ERR_NULL, "workspace"),
    (xent, dict(size=16), fg.FG_ERR_SHAPE, "workspace"),
    (xent_grad, dict(dX=row(dtype=fg.FG_F32)), fg.FG_ERR_UNSUPPORTED, "dX"),
    (xent_grad, dict(dW=row(ld=8)), fg.FG_ERR_SHAPE, "dW"),
    (xent_grad, dict(inc=2), fg.FG_ERR_SHAPE, "dloss_inc"),
    (xent_grad, dict(lse=None), fg.FG_ERR_NULL, "lse"),
    (xent_grad, dict(dloss=None), fg.FG_ERR_NULL, "dloss"),
    (xent_grad, dict(size=16), fg.FG_ERR_SHAPE, "workspace"),
])
def test_refusals(call, args, status, word):
    assert call(**args) == status
    assert word in fg.fg_last_error()


def test_sizes_of_zero_launch_nothing():
    assert layernorm(rows=0) == fg.FG_OK and layernorm(cols=0) == fg.FG_OK and layernorm_grad(cols=0) == fg.FG_OK
    assert embedding(tokens=0, ids=None) == fg.FG_OK and embedding(dim=0) == fg.FG_OK
    assert xent(tokens=0) == fg.FG_OK and xent_grad(dim=0) == fg.FG_OK
    assert embedding_grad(vocab=0) == fg.FG_OK and embedding_grad(dim=0) == fg.FG_OK


def test_workspace_queries():
    lib = fg.load_library()
    assert lib.fg_layernorm_grad_workspace(0, 64, fg.FG_F32) == 0 and lib.fg_layernorm_grad_workspace(4, 64, 77) == 0
    assert lib.fg_layernorm_grad_workspace(4, 64, fg.FG_F32) >= 2 * 64 * 4


def test_binding_wants_tensors_on_the_gpu():
    x = torch.zeros(4, 64)
    with pytest.raises((ValueError, RuntimeError)):
        fg.fg_layernorm(x, None, None, 1e-5, x)
