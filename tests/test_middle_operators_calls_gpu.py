"""GPU tests of how the gated feed-forward block, the norm of gradients and the AdamW step are called: on a stream of the caller's with a workspace of the binding's,
after an error that the program left in the runtime, by the binding's own marshalling and the native one, from several threads."""
import ctypes as C
import threading

import pytest
import torch

from paper_2009_12263_amd import binding as fg

pytestmark = pytest.mark.gpu

# tokens, dim, hidden: few rows, tiled products, split products, copies
SIZES = [(5, 256, 512), (700, 256, 512), (130, 1024, 72), (333, 201, 111)]


class Calls:
    def __init__(self, seed=8):
        g = torch.Generator().manual_seed(seed)
        half = lambda *shape: torch.randn(*shape, generator=g).bfloat16().cuda()
        f32 = lambda *shape: torch.zeros(*shape, device="cuda")
        self.blocks = [(half(T, D), half(T, D), half(2 * H, D) * 0.1, half(D, H) * 0.1) for T, D, H in SIZES]
        self.step = torch.ones(1, dtype=torch.int64, device="cuda")
        self.grads = [half(n) for n in (5, 3000, 70000)]
        self.f32, self.half = f32, half

    def outputs(self, name):
        if name == "norm":
            return [self.f32(1), self.f32(1)]
        if name == "adamw":
            return [t for n in (5, 3000, 70000) for t in (torch.ones(n, device="cuda").bfloat16(), self.f32(n), self.f32(n))]
        x, _, w_in, w_out = self.blocks[int(name[-1])]
        out = [torch.zeros_like(x), self.f32(x.shape[0], w_in.shape[0])]
        return out if name.startswith("ffn") else out + [torch.zeros_like(x), torch.zeros_like(w_in), torch.zeros_like(w_out)]

    def size(self, name):
        if name == "norm":
            return fg.fg_grad_norm_workspace(3)
        if name == "adamw":
            return 4096
        T, D, H = SIZES[int(name[-1])]
        return (fg.fg_gated_ffn_workspace if name.startswith("ffn") else fg.fg_gated_ffn_grad_workspace)(T, D, H)

    def call(self, name, o, stream=None):
        if name == "norm":
            return fg.fg_grad_norm(self.grads, 0.5, 1.0, o[0], o[1], stream=stream)
        if name == "adamw":
            return fg.fg_adamw(o[0::3], self.grads, o[1::3], o[2::3], self.step, 1e-2, 0.9, 0.99, 1e-8, 0.1, stream=stream)
        x, dy, w_in, w_out = self.blocks[int(name[-1])]
        fg.fg_gated_ffn(x, w_in, w_out, fg.FG_ACT_SILU, o[0], o[1], stream=stream)
        if name.startswith("grad"):
            fg.fg_gated_ffn_grad(dy, x, w_in, w_out, fg.FG_ACT_SILU, o[1], o[2], o[3], o[4], stream=stream)


NAMES = ["norm", "adamw"] + ["%s%d" % (k, i) for k in ("ffn", "grad") for i in range(len(SIZES))]


@pytest.mark.parametrize("name", NAMES)
def test_memory_that_the_current_stream_still_writes_is_not_used(name):
    fg.fg_init()
    calls = Calls()
    first, second = calls.outputs(name), calls.outputs(name)
    calls.call(name, first)
    side = torch.cuda.Stream()
    junk = torch.empty(calls.size(name), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    torch.cuda._sleep(50_000_000)
    for _ in range(50):
        junk.fill_(255)
    del junk                                    # its memory is the current stream's to give away, its kernels are still to run
    calls.call(name, second, side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, second))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, second))


def test_an_earlier_error_is_not_the_librarys():
    calls = Calls()
    outputs = {name: calls.outputs(name) for name in NAMES}
    for name in NAMES:
        calls.call(name, outputs[name])
    torch.cuda.synchronize()
    hip = C.CDLL("libamdhip64.so")
    failed = []
    for name in NAMES:
        assert hip.hipSetDevice(4096) != 0
        left = hip.hipPeekAtLastError()
        try:
            calls.call(name, outputs[name])
            if hip.hipPeekAtLastError() != left:
                failed.append((name, "the error is gone"))
        except fg.FlexGemmError as e:
            failed.append((name, str(e)))
        finally:
            hip.hipGetLastError()
    torch.cuda.synchronize()
    assert left != 0 and not failed, failed


@pytest.mark.parametrize("name", NAMES)
def test_both_ways_of_marshalling(name, monkeypatch):
    calls = Calls()
    native, plain = calls.outputs(name), calls.outputs(name)
    calls.call(name, native)
    assert fg._fast is not fg._CtypesOnly, "the native marshalling is not built"
    monkeypatch.setattr(fg, "_fast", fg._CtypesOnly)
    calls.call(name, plain)
    assert all(torch.equal(a, b) for a, b in zip(native, plain))


def test_calls_from_several_threads():
    """Each thread with a stream, operands and results of its own."""
    fg.fg_init()
    want = {}
    alone = Calls()
    for name in NAMES:
        want[name] = alone.outputs(name)
        alone.call(name, want[name])
    torch.cuda.synchronize()
    wrong = []

    def work():
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            calls = Calls()
            for _ in range(3):
                for name in NAMES:
                    got = calls.outputs(name)
                    calls.call(name, got)
                    stream.synchronize()
                    if not all(torch.equal(a, b) for a, b in zip(got, want[name])):
                        wrong.append(name)
    threads = [threading.Thread(target=work) for _ in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong, wrong


def test_lists_and_other_sequences():
    """Tuples, whole numbers for rates, single values: what the native marshalling leaves to the binding's."""
    calls = Calls()
    a, b = calls.outputs("adamw"), calls.outputs("adamw")
    fg.fg_adamw(a[0::3], calls.grads, a[1::3], a[2::3], calls.step, 1.0, 0.0, 0.0, 1.0, 0.0)
    fg.fg_adamw(tuple(b[0::3]), tuple(calls.grads), tuple(b[1::3]), tuple(b[2::3]), calls.step, 1, 0, 0, 1, 0)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    norm = calls.f32(1)
    fg.fg_grad_norm(tuple(calls.grads), 1, 1, norm)
    assert abs(float(norm) - float(torch.cat(calls.grads).double().norm())) <= 2 ** -22 * float(norm)
