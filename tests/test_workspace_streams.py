"""The workspace that the binding takes for a call on a stream of the caller's: it is memory of that stream.  Memory of the current stream may have
been freed by a tensor whose kernels are still to run there, and nothing orders them before the call's."""
import pytest
import torch

from paper_2009_12263_amd import binding as fg


def test_memory_is_taken_from_the_stream_of_the_call(monkeypatch):
    entered, at_empty, empty = [], [], torch.empty

    class Inside:
        def __init__(self, stream):
            self.stream = stream

        def __enter__(self):
            entered.append(self.stream)

        def __exit__(self, *_):
            entered.pop()

    def recorded(*size, device=None, **kw):
        at_empty.append(list(entered))
        return empty(*size, **kw)

    monkeypatch.setattr(torch.cuda, "stream", Inside)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle: ("external", handle))
    monkeypatch.setattr(torch, "empty", recorded)
    for stream, want in ((None, []), (0x5000, [("external", 0x5000)]), (0, [("external", 0)]), (1, [("external", 0)])):
        address, size, keep = fg._workspace(None, 1000, stream, 0)
        assert at_empty.pop() == want and not entered and size == 1000 and address == keep.data_ptr()
    with pytest.raises(ValueError, match="hipStreamPerThread"):
        fg._workspace(None, 1000, 2, 0)
    assert fg._workspace(None, 0, 0x5000, 0) == (None, 0, None)


def _calls(T=700, V=3000, K=256):
    """Calls that take a workspace: (bytes, call(outputs, stream), outputs)."""
    g = torch.Generator().manual_seed(8)
    half = lambda *shape: torch.randn(*shape, generator=g).bfloat16().cuda()
    x, dy, w = half(T, K), half(T, K), half(V, K)
    gamma, ids = torch.ones(K, device="cuda"), torch.randint(0, V, (T,), generator=g).cuda()
    mean, rstd, loss, lse = (torch.empty(T, device="cuda") for _ in range(4))
    dloss = torch.rand(T, generator=g).cuda()
    fg.fg_layernorm(x, gamma, None, 1e-5, torch.empty_like(x), mean, rstd)
    fg.fg_linear_xent(x, w, ids, 0.5, loss, lse)
    f32 = lambda *shape: torch.zeros(*shape, device="cuda")
    return {
        "layernorm": (fg.fg_layernorm_grad_workspace(T, K, x.dtype), lambda o, s: fg.fg_layernorm_grad(dy, x, gamma, mean, rstd, o[0], o[1], o[2], stream=s), lambda: [torch.zeros_like(x), f32(K), f32(K)]),
        "embedding": (fg.fg_embedding_grad_workspace(T, V, K), lambda o, s: fg.fg_embedding_grad(dy, ids, 2.0, None, o[0], stream=s), lambda: [torch.zeros_like(w)]),
        "xent": (fg.fg_linear_xent_workspace(T, V, K), lambda o, s: fg.fg_linear_xent(x, w, ids, 0.5, o[0], o[1], stream=s), lambda: [f32(T), f32(T)]),
        "xent_grad": (fg.fg_linear_xent_grad_workspace(T, V, K), lambda o, s: fg.fg_linear_xent_grad(x, w, ids, 0.5, lse, dloss, o[0], o[1], stream=s), lambda: [torch.zeros_like(x), torch.zeros_like(w)]),
    }


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["layernorm", "embedding", "xent", "xent_grad"])
def test_memory_that_the_current_stream_still_writes_is_not_used(name):
    size, call, outputs = _calls()[name]
    fg.fg_init()
    first, second = outputs(), outputs()
    call(first, None)
    side = torch.cuda.Stream()
    junk = torch.empty(size, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    torch.cuda._sleep(50_000_000)
    for _ in range(50):
        junk.fill_(255)
    del junk                                    # its memory is the current stream's to give away, its kernels are still to run
    for stream in (side, side.cuda_stream):
        call(second, stream)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, second)), stream
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, second))
