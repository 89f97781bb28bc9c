"""Thin binding of libflexgemm.so: argument marshalling only, natively for plain device tensors
(csrc/fastcall.cpp, where it is built), with ctypes for everything else.

The functions have the names and arguments of the C ABI (include/flexgemm.h).  Torch is used
for device memory and streams; every step of the computation runs in the library's kernels.
There is no fallback: if the shared library is missing, importing the entry points raises.
"""
from __future__ import annotations

import ctypes as C
import importlib.util
import os
import sysconfig
from dataclasses import dataclass
from typing import Optional, Sequence

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libflexgemm.so")
# The native marshalling uses Python's and torch's C++ interfaces: it is built for one version of each, which its name holds.
FASTCALL_PATH = os.path.join(_PKG, "_fastcall.%s.torch-%s.so" % (sysconfig.get_config_var("SOABI"), torch.__version__))

FG_OK = 0
FG_ERR_NULL, FG_ERR_SHAPE, FG_ERR_LAYOUT, FG_ERR_ALIGN, FG_ERR_UNSUPPORTED, FG_ERR_MODES, FG_ERR_LAUNCH = range(1, 8)
FG_F16, FG_BF16, FG_F32, FG_CF16, FG_CF32, FG_I32, FG_I64 = 0, 1, 2, 3, 4, 5, 6
FG_COL, FG_ROW, FG_DIAG, FG_ZERO = 0, 1, 2, 3
FG_ACT_NONE, FG_ACT_RELU = 0, 1

EXPORTS = ("fg_init", "fg_gemm", "fg_gemm_ex", "fg_gemm_noalloc", "fg_gemm_dual", "fg_contract", "fg_contract_plan", "fg_last_error", "fg_version",
           "fg_reload_tuning", "fg_gemm_plan", "fg_probe_mfma", "fg_probe_mfma_k32", "fg_probe_kloop_mix",
           "fg_layernorm", "fg_layernorm_grad", "fg_layernorm_grad_workspace", "fg_embedding", "fg_embedding_grad", "fg_embedding_grad_workspace",
           "fg_linear_xent", "fg_linear_xent_workspace", "fg_linear_xent_grad", "fg_linear_xent_grad_workspace")
FG_PLAN_REAL, FG_PLAN_COMPLEX, FG_PLAN_DUAL, FG_PLAN_REAL_BF16, FG_PLAN_COMPLEX_INTERLEAVED, FG_PLAN_REAL_F16_CD = 0, 1, 2, 3, 4, 5
FG_PLAN_REAL_AB_ADD = 6


class fg_matrix(C.Structure):
    _fields_ = [("re", C.c_void_p), ("im", C.c_void_p), ("dtype", C.c_int32), ("layout", C.c_int32), ("ld", C.c_int64)]


class fg_epilogue(C.Structure):
    _fields_ = [("bias", C.c_void_p), ("bias_dim", C.c_int32), ("act", C.c_int32)]


class fg_load_transforms(C.Structure):
    _fields_ = [("a_add", C.c_float), ("b_add", C.c_float), ("c_act", C.c_int32)]


class FlexGemmError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__("flexgemm status %d: %s" % (status, message))
        self.status = status


_current_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda dev: torch.cuda.current_stream(dev).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
_lib = None
_fast = None


def load_library() -> C.CDLL:
    """Load libflexgemm.so (built in-tree by ``paper_2009_12263_amd.build``).  Fails loudly."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError("libflexgemm.so is not built: run `python -m paper_2009_12263_amd.build` "
                              "(there is no CPU or PyTorch fallback)")
        lib = C.CDLL(LIB_PATH)
        i32, i64, f32, vp = C.c_int32, C.c_int64, C.c_float, C.c_void_p
        lib.fg_gemm.restype = C.c_int
        lib.fg_gemm.argtypes = [i64, i64, i64, f32, C.POINTER(fg_matrix), C.POINTER(fg_matrix), f32,
                                C.POINTER(fg_matrix), C.POINTER(fg_matrix), C.POINTER(fg_epilogue), vp]
        lib.fg_gemm_ex.restype = C.c_int
        lib.fg_gemm_ex.argtypes = [i64, i64, i64, f32, C.POINTER(fg_matrix), C.POINTER(fg_matrix), f32,
                                   C.POINTER(fg_matrix), C.POINTER(fg_matrix), C.POINTER(fg_epilogue),
                                   C.POINTER(fg_load_transforms), vp]
        lib.fg_gemm_noalloc.restype = C.c_int
        lib.fg_gemm_noalloc.argtypes = lib.fg_gemm_ex.argtypes
        lib.fg_reload_tuning.restype = None
        lib.fg_reload_tuning.argtypes = []
        lib.fg_gemm_dual.restype = C.c_int
        lib.fg_gemm_dual.argtypes = [i64, i64, i64, f32, C.POINTER(fg_matrix), C.POINTER(fg_matrix), f32,
                                     C.POINTER(fg_matrix), C.POINTER(fg_matrix), vp]
        lib.fg_contract.restype = C.c_int
        lib.fg_contract.argtypes = [i32, vp, vp, vp, i32, vp, vp, vp, i32, vp, vp, vp, vp, i32, vp, vp, f32, f32, vp]
        lib.fg_contract_plan.restype = C.c_int
        lib.fg_contract_plan.argtypes = [i32, vp, vp, vp, i32, vp, vp, vp, i32, vp, vp, vp, vp, i32, vp, vp, C.c_char_p, i32]
        lib.fg_last_error.restype = C.c_char_p
        lib.fg_last_error.argtypes = []
        lib.fg_version.restype = i32
        lib.fg_version.argtypes = []
        lib.fg_init.restype = C.c_int
        lib.fg_init.argtypes = []
        lib.fg_gemm_plan.restype = C.c_int
        lib.fg_gemm_plan.argtypes = [i64, i64, i64, i32, i32, i32, i32, C.c_char_p, i32]
        lib.fg_probe_mfma.restype = C.c_int
        lib.fg_probe_mfma.argtypes = [vp, i64, i32, C.POINTER(C.c_int64), vp]
        lib.fg_probe_mfma_k32.restype = C.c_int
        lib.fg_probe_mfma_k32.argtypes = [vp, i64, i32, C.POINTER(C.c_int64), vp]
        lib.fg_probe_kloop_mix.restype = C.c_int
        lib.fg_probe_kloop_mix.argtypes = [vp, i64, i32, C.POINTER(C.c_int64), vp]
        mp = C.POINTER(fg_matrix)
        lib.fg_layernorm.restype = C.c_int
        lib.fg_layernorm.argtypes = [i64, i64, mp, vp, vp, i32, f32, mp, vp, vp, vp]
        lib.fg_layernorm_grad.restype = C.c_int
        lib.fg_layernorm_grad.argtypes = [i64, i64, mp, mp, vp, i32, vp, vp, mp, vp, vp, vp, i64, vp]
        lib.fg_layernorm_grad_workspace.restype = i64
        lib.fg_layernorm_grad_workspace.argtypes = [i64, i64, i32]
        lib.fg_embedding.restype = C.c_int
        lib.fg_embedding.argtypes = [i64, i64, i64, mp, vp, i32, f32, mp, vp]
        lib.fg_embedding_grad.restype = C.c_int
        lib.fg_embedding_grad.argtypes = [i64, i64, i64, mp, vp, i32, f32, mp, mp, vp, i64, vp]
        lib.fg_embedding_grad_workspace.restype = i64
        lib.fg_embedding_grad_workspace.argtypes = [i64, i64, i64]
        lib.fg_linear_xent.restype = C.c_int
        lib.fg_linear_xent.argtypes = [i64, i64, i64, mp, mp, vp, i32, f32, vp, vp, vp, i64, vp]
        lib.fg_linear_xent_grad.restype = C.c_int
        lib.fg_linear_xent_grad.argtypes = [i64, i64, i64, mp, mp, vp, i32, f32, vp, vp, i64, mp, mp, vp, i64, vp]
        lib.fg_linear_xent_workspace.restype = lib.fg_linear_xent_grad_workspace.restype = i64
        lib.fg_linear_xent_workspace.argtypes = lib.fg_linear_xent_grad_workspace.argtypes = [i64, i64, i64]
        _load_fastcall(lib)
        _lib = lib
    return _lib


_in_bad_fork = getattr(torch._C, "_cuda_isInBadFork", lambda: False)


class _CtypesOnly:
    """In place of the native marshalling where it is not built: leaves every call to the binding (4 to 8 us more each)."""
    gemm = dual = contract = layernorm = layernorm_grad = embedding = embedding_grad = xent = xent_grad = staticmethod(lambda *args: -1)


def _load_fastcall(lib: C.CDLL) -> None:
    global _fast
    # A child of fork() cannot use its parent's GPU tensors.  torch says so when the binding asks for the stream; the native
    # marshalling, which does not ask that way, sees a fork that comes after it is loaded, but not one before.
    if not os.path.exists(FASTCALL_PATH) or _in_bad_fork():
        _fast = _CtypesOnly
        return
    spec = importlib.util.spec_from_file_location(__package__ + "._fastcall", FASTCALL_PATH)
    fast = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(fast)
    fast.setup(Matrix, _current_raw_stream, _current_device,
               *(C.cast(fn, C.c_void_p).value for fn in (lib.fg_gemm, lib.fg_gemm_ex, lib.fg_gemm_noalloc, lib.fg_gemm_dual, lib.fg_contract)))
    fast.setup_rows(*(C.cast(fn, C.c_void_p).value for fn in (
        lib.fg_layernorm, lib.fg_layernorm_grad, lib.fg_layernorm_grad_workspace, lib.fg_embedding, lib.fg_embedding_grad, lib.fg_embedding_grad_workspace,
        lib.fg_linear_xent, lib.fg_linear_xent_workspace, lib.fg_linear_xent_grad, lib.fg_linear_xent_grad_workspace)))
    _fast = fast


_DTYPES = {torch.float16: FG_F16, torch.bfloat16: FG_BF16, torch.float32: FG_F32, torch.complex32: FG_CF16, torch.complex64: FG_CF32,
           torch.int32: FG_I32, torch.int64: FG_I64}


@dataclass
class Matrix:
    """Host-side description of a device matrix: the tensors only provide the pointers."""
    re: Optional[torch.Tensor]
    layout: int = FG_COL
    ld: int = 0
    im: Optional[torch.Tensor] = None
    dtype: Optional[int] = None

    def _struct(self) -> fg_matrix:
        re, im, dtype = self.re, self.im, self.dtype
        if dtype is None:
            t = re if re is not None else im
            dtype = _DTYPES.get(t.dtype if t is not None else torch.float32, -1)
        return fg_matrix(re.data_ptr() if re is not None else None, im.data_ptr() if im is not None else None, dtype, self.layout, self.ld)


def _check_extent(m: Optional["Matrix"], rows: int, cols: int, name: str) -> None:
    """The library sees pointers only and cannot know how much memory is behind them: before a call
    that will launch kernels, check here that every device tensor holds the matrix it is said to
    hold (a matrix larger than its tensor would be read or written out of bounds on the GPU).
    Descriptions the library rejects by itself (a leading dimension that is too small, ...) are
    left to it."""
    if m is None or rows <= 0 or cols <= 0:
        return
    layout, ld = m.layout, m.ld
    if layout == FG_COL:
        need = (cols - 1) * ld + rows if ld >= rows else 0
    elif layout == FG_ROW:
        need = (rows - 1) * ld + cols if ld >= cols else 0
    elif layout == FG_DIAG:
        need = min(rows, cols)
    else:
        need = 0
    for t in (m.re, m.im):
        if t is None or not getattr(t, "is_cuda", False):     # only real device tensors are checked
            continue
        per_entry = 2 if (m.dtype in (FG_CF16, FG_CF32) and not t.is_complex()) else 1
        if need * per_entry > t.numel():
            raise ValueError("%s: a %d x %d matrix with leading dimension %d needs %d elements, the tensor has %d"
                             % (name, rows, cols, ld, need * per_entry, t.numel()))


def _stream_handle(stream) -> Optional[int]:
    if stream is None:
        if torch.cuda.is_initialized():
            # the current device's current stream as torch.cuda.current_stream() gives it, without the
            # Stream object around the handle (0.2 us per call instead of 2.9)
            return _current_raw_stream(_current_device())
        return torch.cuda.current_stream().cuda_stream if torch.cuda.is_available() else None
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def fg_last_error() -> str:
    return load_library().fg_last_error().decode()


def fg_version() -> int:
    return int(load_library().fg_version())


def fg_init(raise_on_error: bool = True) -> int:
    """Prepare every kernel variant on the current device; see fg_init in include/flexgemm.h."""
    return _check(load_library().fg_init(), raise_on_error)


def fg_reload_tuning() -> None:
    """Re-read the FG_FORCE_* tuning overrides from the environment (read once at load otherwise)."""
    load_library().fg_reload_tuning()


def _ref(s):
    return C.byref(s) if s is not None else None


def _check(status: int, raise_on_error: bool) -> int:
    if status != FG_OK and raise_on_error:
        raise FlexGemmError(status, fg_last_error())
    return status


def fg_gemm(M: int, N: int, K: int, alpha: float, A: Optional[Matrix], B: Optional[Matrix], beta: float,
            C_: Optional[Matrix], D: Optional[Matrix], bias: Optional[torch.Tensor] = None, bias_dim: int = 0,
            act: int = FG_ACT_NONE, stream=None, raise_on_error: bool = True,
            a_add: float = 0.0, b_add: float = 0.0, c_act: int = FG_ACT_NONE, noalloc: bool = False) -> int:
    """D = act(alpha * op(A) * op(B) + beta * C + bias); see fg_gemm in include/flexgemm.h.
    With ``a_add``, ``b_add`` or ``c_act`` the call goes to fg_gemm_ex (transforms on loaded elements);
    with ``noalloc`` to fg_gemm_noalloc (same arguments as fg_gemm_ex)."""
    lib = _lib or load_library()
    st = _fast.gemm(M, N, K, alpha, A, B, beta, C_, D, bias, bias_dim, act, stream, a_add, b_add, c_act, noalloc)
    if st >= 0:
        return st if st == FG_OK else _check(st, raise_on_error)
    if M > 0 and N > 0:          # an empty result launches nothing
        _check_extent(A, M, K, "A"); _check_extent(B, K, N, "B"); _check_extent(C_, M, N, "C"); _check_extent(D, M, N, "D")
    sa = A._struct() if A is not None else None
    sb = B._struct() if B is not None else None
    sc = C_._struct() if C_ is not None else None
    sd = D._struct() if D is not None else None
    ep = None
    if bias is not None or act != FG_ACT_NONE:
        ep = fg_epilogue(bias.data_ptr() if bias is not None else None, bias_dim, act)
    ref = _ref
    if noalloc:
        lt = fg_load_transforms(a_add, b_add, c_act)
        st = lib.fg_gemm_noalloc(M, N, K, alpha, ref(sa), ref(sb), beta, ref(sc), ref(sd), ref(ep), C.byref(lt), _stream_handle(stream))
    elif a_add != 0.0 or b_add != 0.0 or c_act != FG_ACT_NONE:
        lt = fg_load_transforms(a_add, b_add, c_act)
        st = lib.fg_gemm_ex(M, N, K, alpha, ref(sa), ref(sb), beta, ref(sc), ref(sd), ref(ep), C.byref(lt), _stream_handle(stream))
    else:
        st = lib.fg_gemm(M, N, K, alpha, ref(sa), ref(sb), beta, ref(sc), ref(sd), ref(ep), _stream_handle(stream))
    return _check(st, raise_on_error)


def fg_gemm_dual(M: int, N: int, K: int, alpha: float, A: Optional[Matrix], B: Optional[Matrix], beta: float,
                 C_: Optional[Matrix], D: Optional[Matrix], stream=None, raise_on_error: bool = True) -> int:
    """Dual-number product on planar (value, dual part) matrices; see fg_gemm_dual in include/flexgemm.h."""
    lib = _lib or load_library()
    st = _fast.dual(M, N, K, alpha, A, B, beta, C_, D, stream)
    if st >= 0:
        return st if st == FG_OK else _check(st, raise_on_error)
    if M > 0 and N > 0:          # an empty result launches nothing
        _check_extent(A, M, K, "A"); _check_extent(B, K, N, "B"); _check_extent(C_, M, N, "C"); _check_extent(D, M, N, "D")
    sa = A._struct() if A is not None else None
    sb = B._struct() if B is not None else None
    sc = C_._struct() if C_ is not None else None
    sd = D._struct() if D is not None else None
    ref = _ref
    st = lib.fg_gemm_dual(M, N, K, alpha, ref(sa), ref(sb), beta, ref(sc), ref(sd), _stream_handle(stream))
    return _check(st, raise_on_error)


def fg_gemm_plan(M: int, N: int, K: int, layoutA: int = FG_COL, layoutB: int = FG_COL, layoutD: int = FG_COL,
                 variant: int = FG_PLAN_REAL) -> str:
    buf = C.create_string_buffer(128)
    st = load_library().fg_gemm_plan(M, N, K, layoutA, layoutB, layoutD, int(variant), buf, 128)
    _check(st, True)
    return buf.value.decode()


def _i32(xs):
    return (C.c_int32 * len(xs))(*map(int, xs))


def _i64(xs):
    return (C.c_int64 * len(xs))(*map(int, xs))


def fg_contract(modesA: Sequence[int], stridesA: Sequence[int], A: torch.Tensor,
                modesB: Sequence[int], stridesB: Sequence[int], B: torch.Tensor,
                modesC: Sequence[int], stridesC: Sequence[int], Cin: Optional[torch.Tensor], Cout: torch.Tensor,
                extents: dict, alpha: float = 1.0, beta: float = 0.0, stream=None, raise_on_error: bool = True) -> int:
    """Cout = alpha * contraction(A, B) + beta * Cin; see fg_contract in include/flexgemm.h.
    ``extents`` maps each integer mode label to its extent."""
    lib = _lib or load_library()
    st = _fast.contract(modesA, stridesA, A, modesB, stridesB, B, modesC, stridesC, Cin, Cout, extents, alpha, beta, stream)
    if st >= 0:
        return st if st == FG_OK else _check(st, raise_on_error)
    positive = all(int(v) > 0 for v in extents.values())
    for name, t, modes, strides in (("A", A, modesA, stridesA), ("B", B, modesB, stridesB), ("Cin", Cin, modesC, stridesC),
                                    ("Cout", Cout, modesC, stridesC)):
        # the same protection as _check_extent: the last element the description reaches must exist
        if t is not None and positive and getattr(t, "is_cuda", False) and len(modes) == len(strides):
            need = 1
            for m, x in zip(modes, strides):
                if m not in extents or x < 0:
                    break
                need += (int(extents[m]) - 1) * int(x)
            else:
                if need > t.numel():
                    raise ValueError("%s: the modes and strides reach element %d, the tensor has %d" % (name, need - 1, t.numel()))
    mA, sA, mB, sB, mC, sC = _i32(modesA), _i64(stridesA), _i32(modesB), _i64(stridesB), _i32(modesC), _i64(stridesC)
    labels, exts = _i32(extents.keys()), _i64(extents.values())
    ptr = lambda t: t.data_ptr() if t is not None else None
    st = lib.fg_contract(len(mA), mA, sA, ptr(A), len(mB), mB, sB, ptr(B), len(mC), mC, sC, ptr(Cin), ptr(Cout),
                         len(labels), labels, exts, alpha, beta, _stream_handle(stream))
    return _check(st, raise_on_error)


def fg_contract_plan(modesA: Sequence[int], stridesA: Sequence[int], A, modesB: Sequence[int], stridesB: Sequence[int], B,
                     modesC: Sequence[int], stridesC: Sequence[int], Cin, Cout, extents: dict) -> str:
    """Name of the kernel fg_contract would use; see fg_contract_plan in include/flexgemm.h."""
    lib = load_library()
    mA, sA, mB, sB, mC, sC = _i32(modesA), _i64(stridesA), _i32(modesB), _i64(stridesB), _i32(modesC), _i64(stridesC)
    labels, exts = _i32(extents.keys()), _i64(extents.values())
    ptr = lambda t: t.data_ptr() if t is not None else None
    buf = C.create_string_buffer(256)
    st = lib.fg_contract_plan(len(mA), mA, sA, ptr(A), len(mB), mB, sB, ptr(B), len(mC), mC, sC, ptr(Cin), ptr(Cout),
                              len(labels), labels, exts, buf, 256)
    _check(st, True)
    return buf.value.decode()


def fg_probe_mfma(fp16_operands: torch.Tensor, iters: int, stream=None, k32: bool = False, kloop_mix: bool = False) -> int:
    """Launch the MFMA-only measurement kernel on operands from ``fp16_operands``; returns the
    number of floating-point operations of the launch (see fg_probe_mfma, fg_probe_mfma_k32 and
    fg_probe_kloop_mix in include/flexgemm.h; ``k32`` selects the 16x16x32 instruction,
    ``kloop_mix`` that instruction together with the K loop's LDS reads and direct loads)."""
    flops = C.c_int64(0)
    lib = load_library()
    fn = lib.fg_probe_kloop_mix if kloop_mix else lib.fg_probe_mfma_k32 if k32 else lib.fg_probe_mfma
    st = fn(fp16_operands.data_ptr(), fp16_operands.numel() * fp16_operands.element_size(), iters, C.byref(flops), _stream_handle(stream))
    _check(st, True)
    return int(flops.value)


# ---- operators on the rows of a matrix ------------------------------------------------------------
# These take device tensors and read sizes, strides and types off them; see include/flexgemm.h for what they compute.  The library sees
# pointers only, so what it cannot know is checked here: device, extents, and that a row is contiguous.

def _rows(t: torch.Tensor, name: str, shape=None, dev: Optional[int] = None) -> fg_matrix:
    if t.dim() != 2 or (shape is not None and t.shape != shape):
        raise ValueError("%s: expected a matrix%s, got shape %s" % (name, "" if shape is None else " of shape %s" % (tuple(shape),), tuple(t.shape)))
    if not t.is_cuda or (dev is not None and t.get_device() != dev):
        raise ValueError("%s: a tensor on the current GPU is needed, got one on %s" % (name, t.device))
    rows, cols = t.shape
    ld, inner = t.stride()
    if inner != 1 and cols > 1:
        raise ValueError("%s: rows must be contiguous, the stride along a row is %d" % (name, inner))
    return fg_matrix(t.data_ptr(), None, _DTYPES.get(t.dtype, -1), FG_ROW, ld if rows > 1 else max(ld, cols))


def _vector(t: Optional[torch.Tensor], n: int, name: str, dtype, dev: int) -> Optional[int]:
    """The address of n contiguous values of type dtype."""
    if t is None:
        return None
    if t.dim() != 1 or t.shape[0] != n or (n > 1 and t.stride(0) != 1):
        raise ValueError("%s: expected %d contiguous values, got shape %s, strides %s" % (name, n, tuple(t.shape), t.stride()))
    if t.dtype != dtype:
        raise ValueError("%s: expected %s, got %s" % (name, dtype, t.dtype))
    if t.get_device() != dev:
        raise ValueError("%s: a tensor on the current GPU is needed, got one on %s" % (name, t.device))
    return t.data_ptr()


def _torch_stream(stream):
    """A stream argument as torch's allocator knows streams."""
    if isinstance(stream, torch.cuda.Stream):
        return stream
    handle = _stream_handle(stream)
    if handle == 2:                 # hipStreamPerThread: one handle for the streams of all threads, which the allocator would take for one
        raise ValueError("workspace: a call on hipStreamPerThread needs one from the caller")
    return torch.cuda.ExternalStream(0 if handle == 1 else handle)        # (1: the default stream by its other name)


def _workspace(given: Optional[torch.Tensor], need: int, stream, dev: int):
    """(address, bytes, what keeps it alive) of the caller's workspace, or of one from torch's allocator for the stream of the call."""
    if given is not None:
        if not given.is_cuda or given.get_device() != dev or not given.is_contiguous():
            raise ValueError("workspace: a contiguous tensor on the current GPU is needed")
        return given.data_ptr(), given.numel() * given.element_size(), given
    if need <= 0:
        return None, 0, None
    make = lambda: torch.empty(need, dtype=torch.uint8, device=torch.device("cuda", dev))
    if stream is None:
        t = make()
    else:
        # Memory of the call's own stream: what the current stream has freed may still be written by kernels waiting there, and nothing
        # orders the call behind them.
        with torch.cuda.stream(_torch_stream(stream)):
            t = make()
    return t.data_ptr(), need, t


def fg_layernorm(X: torch.Tensor, gamma: Optional[torch.Tensor], beta: Optional[torch.Tensor], eps: float, Y: torch.Tensor,
                 mean: Optional[torch.Tensor] = None, rstd: Optional[torch.Tensor] = None, stream=None, raise_on_error: bool = True) -> int:
    """Y = layer norm of the rows of X; mean and rstd of the rows are kept for fg_layernorm_grad."""
    lib = _lib or load_library()
    st = _fast.layernorm(X, gamma, beta, eps, Y, mean, rstd, stream)
    if st >= 0:
        return st if st == FG_OK else _check(st, raise_on_error)
    dev = _current_device()
    x = _rows(X, "X", None, dev)
    y = _rows(Y, "Y", X.shape, dev)
    rows, cols = X.shape
    ptype = gamma.dtype if gamma is not None else beta.dtype if beta is not None else X.dtype
    st = lib.fg_layernorm(rows, cols, C.byref(x), _vector(gamma, cols, "gamma", ptype, dev), _vector(beta, cols, "beta", ptype, dev),
                          _DTYPES.get(ptype, -1), eps, C.byref(y), _vector(mean, rows, "mean", torch.float32, dev),
                          _vector(rstd, rows, "rstd", torch.float32, dev), _stream_handle(stream))
    return _check(st, raise_on_error)


def fg_layernorm_grad_workspace(rows: int, cols: int, dtype: torch.dtype) -> int:
    return int(load_library().fg_layernorm_grad_workspace(rows, cols, _DTYPES.get(dtype, -1)))


def fg_layernorm_grad(dY: torch.Tensor, X: torch.Tensor, gamma: Optional[torch.Tensor], mean: torch.Tensor, rstd: torch.Tensor, dX: torch.Tensor,
                      dgamma: Optional[torch.Tensor] = None, dbeta: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                      stream=None, raise_on_error: bool = True) -> int:
    """Gradients of fg_layernorm with respect to X, gamma and beta."""
    lib = _lib or load_library()
    st = _fast.layernorm_grad(dY, X, gamma, mean, rstd, dX, dgamma, dbeta, workspace, stream)
    if st >= 0:
        return st if st == FG_OK else _check(st, raise_on_error)
    dev = _current_device()
    x = _rows(X, "X", None, dev)
    dy = _rows(dY, "dY", X.shape, dev)
    dx = _rows(dX, "dX", X.shape, dev)
    rows, cols = X.shape
    ptype = next((t.dtype for t in (gamma, dgamma, dbeta) if t is not None), X.dtype)
    need = lib.fg_layernorm_grad_workspace(rows, cols, x.dtype) if dgamma is not None or dbeta is not None else 0
    ws, ws_bytes, _keep = _workspace(workspace, need, stream, dev)
    st = lib.fg_layernorm_grad(rows, cols, C.byref(dy), C.byref(x), _vector(gamma, cols, "gamma", ptype, dev), _DTYPES.get(ptype, -1),
                               _vector(mean, rows, "mean", torch.float32, dev), _vector(rstd, rows, "rstd", torch.float32, dev), C.byref(dx),
                               _vector(dgamma, cols, "dgamma", ptype, dev), _vector(dbeta, cols, "dbeta", ptype, dev), ws, ws_bytes, _stream_handle(stream))
    return _check(st, raise_on_error)


def _indices(t: torch.Tensor, n: int, name: str, dev: int):
    if t.dtype not in (torch.int32, torch.int64):
        raise ValueError("%s: expected int32 or int64, got %s" % (name, t.dtype))
    return _vector(t, n, name, t.dtype, dev), _DTYPES[t.dtype]


def fg_embedding(table: torch.Tensor, ids: torch.Tensor, scale: float, Y: torch.Tensor, stream=None, raise_on_error: bool = True) -> int:
    """Y[t] = scale * table[ids[t]]; zeros where ids[t] names no row."""
    lib = _lib or load_library()
    st = _fast.embedding(table, ids, scale, Y, stream)
    if st >= 0:
        return st if st == FG_OK else _check(st, raise_on_error)
    dev = _current_device()
    m = _rows(table, "table", None, dev)
    vocab, dim = table.shape
    tokens = ids.shape[0]
    y = _rows(Y, "Y", (tokens, dim), dev)
    at, kind = _indices(ids, tokens, "ids", dev)
    return _check(lib.fg_embedding(tokens, vocab, dim, C.byref(m), at, kind, scale, C.byref(y), _stream_handle(stream)), raise_on_error)


def fg_embedding_grad_workspace(tokens: int, vocab: int, dim: int) -> int:
    return int(load_library().fg_embedding_grad_workspace(tokens, vocab, dim))


def fg_embedding_grad(dY: torch.Tensor, ids: torch.Tensor, scale: float, Cin: Optional[torch.Tensor], dtable: torch.Tensor,
                      workspace: Optional[torch.Tensor] = None, stream=None, raise_on_error: bool = True) -> int:
    """dtable[v] = scale * sum of dY[t] over the t with ids[t] == v, + Cin[v] (None: nothing; dtable itself: only rows with tokens are touched)."""
    lib = _lib or load_library()
    st = _fast.embedding_grad(dY, ids, scale, Cin, dtable, workspace, stream)
    if st >= 0:
        return st if st == FG_OK else _check(st, raise_on_error)
    dev = _current_device()
    d = _rows(dtable, "dtable", None, dev)
    vocab, dim = dtable.shape
    tokens = ids.shape[0]
    dy = _rows(dY, "dY", (tokens, dim), dev)
    c = _rows(Cin, "Cin", (vocab, dim), dev) if Cin is not None else None
    at, kind = _indices(ids, tokens, "ids", dev)
    ws, ws_bytes, _keep = _workspace(workspace, lib.fg_embedding_grad_workspace(tokens, vocab, dim), stream, dev)
    st = lib.fg_embedding_grad(tokens, vocab, dim, C.byref(dy), at, kind, scale, _ref(c), C.byref(d), ws, ws_bytes, _stream_handle(stream))
    return _check(st, raise_on_error)


def fg_linear_xent_workspace(tokens: int, vocab: int, dim: int) -> int:
    return int(load_library().fg_linear_xent_workspace(tokens, vocab, dim))


def fg_linear_xent(X: torch.Tensor, W: torch.Tensor, targets: torch.Tensor, scale: float, loss: torch.Tensor, lse: torch.Tensor,
                   workspace: Optional[torch.Tensor] = None, stream=None, raise_on_error: bool = True) -> int:
    """loss[t] = lse[t] - z[t][targets[t]] with z = scale * X W^T, lse its log-sum-exp over the words; 0 where the target names no word."""
    lib = _lib or load_library()
    st = _fast.xent(X, W, targets, scale, loss, lse, workspace, stream)
    if st >= 0:
        return st if st == FG_OK else _check(st, raise_on_error)
    dev = _current_device()
    x, w = _rows(X, "X", None, dev), _rows(W, "W", None, dev)
    (tokens, dim), vocab = X.shape, W.shape[0]
    if W.shape[1] != dim:
        raise ValueError("X and W: rows of %d and %d values" % (dim, W.shape[1]))
    at, kind = _indices(targets, tokens, "targets", dev)
    ws, ws_bytes, _keep = _workspace(workspace, lib.fg_linear_xent_workspace(tokens, vocab, dim), stream, dev)
    st = lib.fg_linear_xent(tokens, vocab, dim, C.byref(x), C.byref(w), at, kind, scale, _vector(loss, tokens, "loss", torch.float32, dev),
                            _vector(lse, tokens, "lse", torch.float32, dev), ws, ws_bytes, _stream_handle(stream))
    return _check(st, raise_on_error)


def fg_linear_xent_grad_workspace(tokens: int, vocab: int, dim: int) -> int:
    return int(load_library().fg_linear_xent_grad_workspace(tokens, vocab, dim))


def fg_linear_xent_grad(X: torch.Tensor, W: torch.Tensor, targets: torch.Tensor, scale: float, lse: torch.Tensor, dloss: torch.Tensor,
                        dX: torch.Tensor, dW: torch.Tensor, workspace: Optional[torch.Tensor] = None, stream=None, raise_on_error: bool = True) -> int:
    """Gradients of the losses of fg_linear_xent, weighted with dloss (one value per token, which may be a single one expanded)."""
    lib = _lib or load_library()
    st = _fast.xent_grad(X, W, targets, scale, lse, dloss, dX, dW, workspace, stream)
    if st >= 0:
        return st if st == FG_OK else _check(st, raise_on_error)
    dev = _current_device()
    x, w = _rows(X, "X", None, dev), _rows(W, "W", None, dev)
    (tokens, dim), vocab = X.shape, W.shape[0]
    if W.shape[1] != dim:
        raise ValueError("X and W: rows of %d and %d values" % (dim, W.shape[1]))
    dx, dw = _rows(dX, "dX", X.shape, dev), _rows(dW, "dW", W.shape, dev)
    at, kind = _indices(targets, tokens, "targets", dev)
    inc = 1
    if dloss.dim() == 1 and dloss.shape[0] == tokens and tokens > 1 and dloss.stride(0) == 0:
        dloss, inc = dloss[:1], 0
    g = _vector(dloss, tokens if inc else 1, "dloss", torch.float32, dev)
    ws, ws_bytes, _keep = _workspace(workspace, lib.fg_linear_xent_grad_workspace(tokens, vocab, dim), stream, dev)
    st = lib.fg_linear_xent_grad(tokens, vocab, dim, C.byref(x), C.byref(w), at, kind, scale, _vector(lse, tokens, "lse", torch.float32, dev), g, inc,
                                 C.byref(dx), C.byref(dw), ws, ws_bytes, _stream_handle(stream))
    return _check(st, raise_on_error)
