"""CPU tests: what the gated feed-forward block, the AdamW step and the norm of gradients refuse, and with which status, before anything is launched."""
import ctypes as C
import math

import pytest

from paper_2009_12263_amd import binding as fg

PTR = 0x10000
NULL = C.POINTER(fg.fg_matrix)()


def row(dtype=fg.FG_BF16, ld=128, re=PTR, layout=fg.FG_ROW, im=None):
    return C.byref(fg.fg_matrix(re, im, dtype, layout, ld))


def ffn(tokens=4, dim=64, hidden=48, X=None, W_in=None, W_out=None, act=fg.FG_ACT_SILU, Y=None, GU=NULL, ws=PTR, size=1 << 40):
    X, W_in, W_out, Y = (row(re=PTR * (k + 1)) if m is None else m for k, m in enumerate((X, W_in, W_out, Y)))
    return fg.load_library().fg_gated_ffn(tokens, dim, hidden, X, W_in, W_out, act, Y, GU, ws, size, None)


def ffn_grad(tokens=4, dim=64, hidden=48, dY=None, X=None, W_in=None, W_out=None, act=fg.FG_ACT_SILU, GU=None, dX=None, dW_in=None, dW_out=None, ws=PTR, size=1 << 40):
    dY, X, W_in, W_out, dX, dW_in, dW_out = (row(re=PTR * (k + 1)) if m is None else m for k, m in enumerate((dY, X, W_in, W_out, dX, dW_in, dW_out)))
    GU = row(fg.FG_F32) if GU is None else GU
    return fg.load_library().fg_gated_ffn_grad(tokens, dim, hidden, dY, X, W_in, W_out, act, GU, dX, dW_in, dW_out, ws, size, None)


def tensor(**change):
    t = dict(param=PTR, grad=PTR, master=None, exp_avg=PTR, exp_avg_sq=PTR, avg_scale=None, sq_scale=None, n=100, param_dtype=fg.FG_BF16, grad_dtype=fg.FG_BF16) | change
    return fg.fg_adamw_tensor(*t.values())


def apart(i, **change):
    """Tensors whose arrays have memory of their own."""
    at = (1 << 30) + (i << 16)
    return tensor(**(dict(param=at, grad=at + 4096, exp_avg=at + 8192, exp_avg_sq=at + 16384) | change))


def adamw(tensors=None, count=None, step=PTR, lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, decay=0.1, factor=None, lr_factor=None):
    tensors = [tensor()] if tensors is None else tensors
    items = (fg.fg_adamw_tensor * len(tensors))(*tensors) if tensors != "NULL" else None
    return fg.load_library().fg_adamw(len(tensors) if count is None else count, items, step, lr, beta1, beta2, eps, decay, factor, lr_factor, None)


def norm(grads=((PTR, 100, fg.FG_BF16),), count=None, scale=1.0, limit=1.0, out=PTR, factor=PTR, ws=PTR, size=1 << 30):
    items = (fg.fg_values * len(grads))(*(fg.fg_values(*g) for g in grads)) if grads != "NULL" else None
    return fg.load_library().fg_grad_norm(len(grads) if count is None else count, items, scale, limit, out, factor, ws, size, None)


@pytest.mark.parametrize("call,args,status,word", [
    (ffn, dict(tokens=-1), fg.FG_ERR_SHAPE, "negative"),
    (ffn, dict(hidden=-1), fg.FG_ERR_SHAPE, "negative"),
    (ffn, dict(X=NULL), fg.FG_ERR_NULL, "X is NULL"),
    (ffn, dict(W_in=NULL), fg.FG_ERR_NULL, "W_in is NULL"),
    (ffn, dict(W_out=row(re=None)), fg.FG_ERR_NULL, "W_out->re"),
    (ffn, dict(Y=NULL), fg.FG_ERR_NULL, "Y is NULL"),
    (ffn, dict(W_in=row(ld=63)), fg.FG_ERR_SHAPE, "ld=63"),
    (ffn, dict(W_out=row(ld=47)), fg.FG_ERR_SHAPE, "ld=47"),
    (ffn, dict(X=row(ld=0)), fg.FG_ERR_SHAPE, "ld=0"),
    (ffn, dict(X=row(layout=fg.FG_COL)), fg.FG_ERR_LAYOUT, "row-major"),
    (ffn, dict(X=row(im=PTR)), fg.FG_ERR_LAYOUT, "real"),
    (ffn, dict(X=row(re=PTR + 1)), fg.FG_ERR_ALIGN, "aligned"),
    (ffn, dict(X=row(fg.FG_F32), W_in=row(fg.FG_F32), W_out=row(fg.FG_F32), Y=row(fg.FG_F32)), fg.FG_ERR_UNSUPPORTED, "FG_F16 or all FG_BF16"),
    (ffn, dict(W_in=row(fg.FG_F16)), fg.FG_ERR_UNSUPPORTED, "FG_F16 or all FG_BF16"),
    (ffn, dict(Y=row(fg.FG_F32)), fg.FG_ERR_UNSUPPORTED, "Y"),
    (ffn, dict(GU=row(fg.FG_BF16)), fg.FG_ERR_UNSUPPORTED, "GU"),
    (ffn, dict(GU=row(fg.FG_F32, ld=95)), fg.FG_ERR_SHAPE, "GU"),
    (ffn, dict(act=4), fg.FG_ERR_LAYOUT, "activation"),
    (ffn, dict(act=-1), fg.FG_ERR_LAYOUT, "activation"),
    (ffn, dict(tokens=2 << 30), fg.FG_ERR_UNSUPPORTED, "2^30"),
    (ffn, dict(dim=1 << 21, X=row(ld=1 << 21), W_in=row(ld=1 << 21), Y=row(ld=1 << 21)), fg.FG_ERR_UNSUPPORTED, "2^21"),
    (ffn, dict(hidden=1 << 20, W_out=row(ld=1 << 20)), fg.FG_ERR_UNSUPPORTED, "2^21"),
    (ffn, dict(tokens=1 << 30, hidden=1 << 10, W_out=row(ld=1 << 10)), fg.FG_ERR_UNSUPPORTED, "tiles"),
    (ffn, dict(Y=row()), fg.FG_ERR_LAYOUT, "Y must be in other memory than X"),
    (ffn, dict(Y=row(re=3 * PTR)), fg.FG_ERR_LAYOUT, "Y must be in other memory than W_out"),
    (ffn, dict(GU=row(fg.FG_F32)), fg.FG_ERR_LAYOUT, "GU must be in other memory than X"),
    (ffn, dict(GU=row(fg.FG_F32, re=4 * PTR)), fg.FG_ERR_LAYOUT, "GU must be in other memory than Y"),
    (ffn_grad, dict(GU=row(fg.FG_F32, re=6 * PTR)), fg.FG_ERR_LAYOUT, "dW_in must be in other memory than GU"),
    (ffn_grad, dict(dX=row(re=6 * PTR)), fg.FG_ERR_LAYOUT, "dX must be in other memory than dW_in"),
    (ffn_grad, dict(dX=row(re=7 * PTR)), fg.FG_ERR_LAYOUT, "dX must be in other memory than dW_out"),
    (ffn_grad, dict(dW_out=row(re=6 * PTR)), fg.FG_ERR_LAYOUT, "dW_in must be in other memory than dW_out"),
    (ffn_grad, dict(dX=row()), fg.FG_ERR_LAYOUT, "dX must be in other memory than dY"),
    (ffn_grad, dict(dX=row(re=2 * PTR)), fg.FG_ERR_LAYOUT, "dX must be in other memory than X"),
    (ffn_grad, dict(dW_in=row(re=3 * PTR)), fg.FG_ERR_LAYOUT, "dW_in must be in other memory than W_in"),
    (ffn_grad, dict(dW_out=row(re=4 * PTR)), fg.FG_ERR_LAYOUT, "dW_out must be in other memory than W_out"),
    (ffn, dict(ws=None), fg.FG_ERR_NULL, "workspace"),
    (ffn, dict(size=16), fg.FG_ERR_SHAPE, "workspace"),
    (ffn, dict(ws=PTR + 8), fg.FG_ERR_ALIGN, "workspace"),
    (ffn_grad, dict(dY=NULL), fg.FG_ERR_NULL, "dY is NULL"),
    (ffn_grad, dict(GU=NULL), fg.FG_ERR_NULL, "GU is NULL"),
    (ffn_grad, dict(GU=row()), fg.FG_ERR_UNSUPPORTED, "GU"),
    (ffn_grad, dict(dY=row(fg.FG_F32)), fg.FG_ERR_UNSUPPORTED, "dY"),
    (ffn_grad, dict(dX=row(ld=63)), fg.FG_ERR_SHAPE, "dX"),
    (ffn_grad, dict(dW_in=row(fg.FG_F32)), fg.FG_ERR_UNSUPPORTED, "dW_in"),
    (ffn_grad, dict(dW_out=row(re=None)), fg.FG_ERR_NULL, "dW_out"),
    (ffn_grad, dict(act=9), fg.FG_ERR_LAYOUT, "activation"),
    (ffn_grad, dict(ws=None), fg.FG_ERR_NULL, "workspace"),
    (ffn_grad, dict(size=64), fg.FG_ERR_SHAPE, "workspace"),
    (adamw, dict(count=-1), fg.FG_ERR_SHAPE, "negative"),
    (adamw, dict(tensors="NULL", count=2), fg.FG_ERR_NULL, "list"),
    (adamw, dict(step=None), fg.FG_ERR_NULL, "step"),
    (adamw, dict(step=PTR + 4), fg.FG_ERR_ALIGN, "step"),
    (adamw, dict(factor=PTR + 2), fg.FG_ERR_ALIGN, "grad_factor"),
    (adamw, dict(beta1=1.0), fg.FG_ERR_SHAPE, "beta1"),
    (adamw, dict(beta2=-0.1), fg.FG_ERR_SHAPE, "beta2"),
    (adamw, dict(beta2=math.nan), fg.FG_ERR_SHAPE, "beta2"),
    (adamw, dict(eps=-1.0), fg.FG_ERR_SHAPE, "eps"),
    (adamw, dict(eps=math.nan), fg.FG_ERR_SHAPE, "eps"),
    (adamw, dict(lr=math.inf), fg.FG_ERR_SHAPE, "lr"),
    (adamw, dict(decay=math.nan), fg.FG_ERR_SHAPE, "weight_decay"),
    (adamw, dict(tensors=[tensor(n=-1)]), fg.FG_ERR_SHAPE, "negative"),
    (adamw, dict(tensors=[tensor(n=1 << 40)]), fg.FG_ERR_UNSUPPORTED, "2^36"),
    (adamw, dict(tensors=[tensor(param=None)]), fg.FG_ERR_NULL, "param"),
    (adamw, dict(tensors=[tensor(), tensor(grad=None)]), fg.FG_ERR_NULL, "tensor 1: grad"),
    (adamw, dict(tensors=[tensor(exp_avg=None)]), fg.FG_ERR_NULL, "exp_avg"),
    (adamw, dict(tensors=[tensor(param_dtype=fg.FG_I32)]), fg.FG_ERR_LAYOUT, "param"),
    (adamw, dict(tensors=[tensor(grad_dtype=fg.FG_F16)]), fg.FG_ERR_LAYOUT, "grad"),
    (adamw, dict(tensors=[tensor(param_dtype=fg.FG_F32, grad_dtype=fg.FG_BF16)]), fg.FG_ERR_LAYOUT, "grad"),
    (adamw, dict(tensors=[tensor(param_dtype=fg.FG_F32, grad_dtype=fg.FG_F32, master=PTR)]), fg.FG_ERR_LAYOUT, "copy"),
    (adamw, dict(tensors=[tensor(avg_scale=PTR)]), fg.FG_ERR_NULL, "scales"),
    (adamw, dict(tensors=[tensor(param=PTR + 1)]), fg.FG_ERR_ALIGN, "param"),
    (adamw, dict(tensors=[tensor(exp_avg=PTR + 2)]), fg.FG_ERR_ALIGN, "4 bytes"),
    (adamw, dict(tensors=[tensor(exp_avg=PTR + 4, avg_scale=PTR, sq_scale=PTR)]), fg.FG_ERR_ALIGN, "16 bytes"),
    (adamw, dict(tensors=[tensor(master=PTR + 2)]), fg.FG_ERR_ALIGN, "master"),
    (adamw, dict(tensors=[tensor(), tensor(param=1 << 20, avg_scale=PTR, sq_scale=PTR)]), fg.FG_ERR_UNSUPPORTED, "eight bits"),
    (adamw, dict(tensors=[tensor(), tensor()]), fg.FG_ERR_LAYOUT, "in common"),
    (adamw, dict(tensors=[tensor(param=PTR + 198), tensor(param=1 << 20), tensor(n=100)]), fg.FG_ERR_LAYOUT, "tensors 2 and 0"),
    (adamw, dict(tensors=[apart(0), apart(1, master=1 << 20), apart(2, master=(1 << 20) + 396)]), fg.FG_ERR_LAYOUT, "tensors 1 and 2 have values of master"),
    (adamw, dict(tensors=[apart(1), apart(0, exp_avg=apart(1).exp_avg)]), fg.FG_ERR_LAYOUT, "values of exp_avg in"),
    (adamw, dict(tensors=[apart(0), apart(2), apart(1, exp_avg_sq=apart(0).exp_avg_sq + 4)]), fg.FG_ERR_LAYOUT, "tensors 0 and 2 have values of exp_avg_sq"),
    (adamw, dict(tensors=[apart(0, avg_scale=1 << 20, sq_scale=1 << 21), apart(1, avg_scale=1 << 20, sq_scale=1 << 22)]), fg.FG_ERR_LAYOUT, "avg_scale in"),
    (adamw, dict(tensors=[apart(0, avg_scale=1 << 20, sq_scale=1 << 21), apart(1, avg_scale=1 << 22, sq_scale=1 << 21)]), fg.FG_ERR_LAYOUT, "sq_scale in"),
    (adamw, dict(tensors=[apart(0), tensor(param=1 << 20)]), fg.FG_ERR_LAYOUT, "tensor 1: both moments"),
    (adamw, dict(tensors=[apart(0, avg_scale=1 << 20, sq_scale=1 << 20)]), fg.FG_ERR_LAYOUT, "tensor 0: both moments"),
    (norm, dict(count=-1), fg.FG_ERR_SHAPE, "negative"),
    (norm, dict(grads="NULL", count=1), fg.FG_ERR_NULL, "list"),
    (norm, dict(out=None), fg.FG_ERR_NULL, "norm"),
    (norm, dict(factor=PTR + 1), fg.FG_ERR_ALIGN, "factor"),
    (norm, dict(scale=0.0), fg.FG_ERR_SHAPE, "scale"),
    (norm, dict(scale=math.inf), fg.FG_ERR_SHAPE, "scale"),
    (norm, dict(limit=0.0), fg.FG_ERR_SHAPE, "max_norm"),
    (norm, dict(limit=math.nan), fg.FG_ERR_SHAPE, "max_norm"),
    (norm, dict(grads=((None, 4, fg.FG_F32),)), fg.FG_ERR_NULL, "grad"),
    (norm, dict(grads=((PTR, 4, fg.FG_I64),)), fg.FG_ERR_LAYOUT, "grad"),
    (norm, dict(grads=((PTR + 2, 4, fg.FG_F32),)), fg.FG_ERR_ALIGN, "grad"),
    (norm, dict(grads=((PTR, -4, fg.FG_F32),)), fg.FG_ERR_SHAPE, "negative"),
    (norm, dict(ws=None), fg.FG_ERR_NULL, "workspace"),
    (norm, dict(size=0), fg.FG_ERR_SHAPE, "workspace"),
])
def test_refusals(call, args, status, word):
    assert call(**args) == status
    assert word in fg.fg_last_error(), fg.fg_last_error()


def test_calls_without_work():
    """Sizes of zero need neither memory nor a GPU."""
    none = dict(re=None)
    assert ffn(tokens=0, X=row(**none), Y=row(**none), ws=None, size=0) == fg.FG_OK
    assert ffn(dim=0, X=row(**none), W_in=row(**none), W_out=row(**none), Y=row(**none), ws=None, size=0) == fg.FG_OK
    assert ffn_grad(dX=NULL, dW_in=NULL, dW_out=NULL, ws=None, size=0) == fg.FG_OK
    assert adamw([]) == fg.FG_OK and adamw([tensor(n=0, param=None, grad=None, exp_avg=None, exp_avg_sq=None)]) == fg.FG_OK


def test_workspace_queries():
    lib = fg.load_library()
    for sizes in ((0, 64, 64), (4, 0, 64), (4, 64, 0), (-1, 64, 64)):
        assert lib.fg_gated_ffn_workspace(*sizes) == 0 and lib.fg_gated_ffn_grad_workspace(*sizes) == 0
    for tokens in (1, 64, 65, 1000, 8192):
        for dim, hidden in ((64, 48), (1001, 2729), (4096, 10240)):
            assert 0 < lib.fg_gated_ffn_workspace(tokens, dim, hidden) < 1 << 34
            assert 0 < lib.fg_gated_ffn_grad_workspace(tokens, dim, hidden) < 1 << 34
    assert lib.fg_grad_norm_workspace(0) == 0 and lib.fg_grad_norm_workspace(1) > 0


def test_products_keep_their_activations():
    """The activations of the gated block are no epilogue of a product."""
    lib = fg.load_library()
    ep = fg.fg_epilogue()
    ep.act = fg.FG_ACT_SILU
    a = fg.fg_matrix(PTR, None, fg.FG_F16, fg.FG_COL, 8)
    d = fg.fg_matrix(PTR, None, fg.FG_F32, fg.FG_COL, 8)
    assert lib.fg_gemm(8, 8, 8, 1.0, C.byref(a), C.byref(a), 0.0, None, C.byref(d), C.byref(ep), None) == fg.FG_ERR_LAYOUT
