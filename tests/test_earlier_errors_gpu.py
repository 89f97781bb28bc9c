"""GPU test: an error that an earlier call of the program left behind in the HIP runtime is not taken for one of the library's launches, and stays the
program's to read."""
import ctypes as C

import pytest
import torch

from paper_2009_12263_amd import binding as fg

pytestmark = pytest.mark.gpu


def _calls():
    T, V, K = 300, 5000, 64
    g = torch.Generator().manual_seed(3)
    x, w = (torch.randn(n, K, generator=g).bfloat16().cuda() for n in (T, V))
    ids = torch.randint(0, V, (T,), generator=g).cuda()
    new = lambda *shape, dtype=torch.float32: torch.empty(*shape, dtype=dtype, device="cuda")
    mean, rstd, loss, lse, dloss, gamma = new(T), new(T), new(T), new(T), torch.ones(T, device="cuda"), torch.ones(K, device="cuda")
    y, dw, dgamma = torch.empty_like(x), torch.empty_like(w), new(K)
    wide = torch.randn(3, 20000, device="cuda")
    a, b, d = torch.randn(304, 4096, device="cuda").half(), torch.randn(304, 4096, device="cuda").half(), new(304, 304)
    odd = new(301, 303)
    R = lambda t: fg.Matrix(t, fg.FG_ROW, t.stride(0))
    return [
        lambda: fg.fg_layernorm(x, gamma, None, 1e-5, y, mean, rstd),
        lambda: fg.fg_layernorm_grad(x, x, gamma, mean, rstd, y, dgamma, None),
        lambda: fg.fg_layernorm(wide, None, None, 1e-5, torch.empty_like(wide)),
        lambda: fg.fg_embedding(w, ids, 1.0, y),
        lambda: fg.fg_embedding_grad(x, ids, 1.0, None, dw),
        lambda: fg.fg_linear_xent(x, w, ids, 1.0, loss, lse),
        lambda: fg.fg_linear_xent_grad(x, w, ids, 1.0, lse, dloss, y, dw),
        lambda: fg.fg_linear_xent_grad(x[:20], w, ids[:20], 1.0, lse[:20], dloss[:20], y[:20], dw),
        lambda: fg.fg_gemm(304, 304, 4096, 1.0, R(a), fg.Matrix(b, fg.FG_COL, 4096), 0.0, None, R(d)),             # (split over K)
        lambda: fg.fg_gemm(301, 303, 4001, 1.0, R(a), fg.Matrix(b, fg.FG_COL, 4096), 0.0, None, R(odd)),           # (the general kernel)
    ]


def test_an_earlier_error_is_not_the_librarys():
    calls = _calls()
    for call in calls:
        call()
    torch.cuda.synchronize()
    hip = C.CDLL("libamdhip64.so")
    failed = []
    for i, call in enumerate(calls):
        assert hip.hipSetDevice(4096) != 0
        left = hip.hipPeekAtLastError()
        try:
            call()
            if hip.hipPeekAtLastError() != left:
                failed.append((i, "the error is gone"))
        except fg.FlexGemmError as e:
            failed.append((i, str(e)))
        finally:
            hip.hipGetLastError()
    torch.cuda.synchronize()
    assert left != 0 and not failed, failed
