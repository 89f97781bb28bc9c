"""GPU tests of the gated feed-forward block on rows that begin between two 32-bit words, of few and of more tokens, against the formulas in 64 bits within the bounds of
tests/test_gated_ffn_gpu.py.  What lies beside the operands is NaN."""
import pytest
import torch

from tests.test_gated_ffn_gpu import Case, check, reference

pytestmark = pytest.mark.gpu


# pad, offset: odd and even leading dimensions, first values on a word and between two
@pytest.mark.parametrize("pad,offset", [(0, 0), (0, 1), (1, 0), (1, 1), (2, 1), (7, 3)])
@pytest.mark.parametrize("size", [(1, 63, 65), (1, 255, 1027), (2, 513, 129), (4, 127, 2049), (7, 1000, 333), (8, 335, 1024), (9, 1025, 77), (16, 131, 515), (17, 133, 511),
                                  (31, 777, 129), (32, 65, 1023), (33, 195, 257), (64, 259, 131)])
def test_odd_rows(size, pad, offset):
    c = Case(*size, torch.bfloat16 if (size[0] + pad) % 2 else torch.float16, seed=size[1], pad=pad, offset=offset)
    c.forward("silu")
    c.backward("silu")
    want = reference(c.x, c.w_in, c.w_out, "silu", c.dtype, c.dy)
    for name, got in c.r.items():
        check(name, got, want[name])


@pytest.mark.parametrize("tokens", [1, 3, 16])
def test_single_operands_between_words(tokens):
    """X or one of the weights alone begins between two words."""
    plain, odd = (Case(tokens, 320, 448, torch.bfloat16, seed=tokens, pad=pad, offset=offset) for pad, offset in ((8, 8), (2, 1)))
    want = reference(plain.x, plain.w_in, plain.w_out, "gelu", plain.dtype)
    for name in ("x", "w_in", "w_out"):
        getattr(odd, name).copy_(getattr(plain, name))
    for names in (["x"], ["w_in"], ["w_out"], ["x", "w_out"], ["x", "w_in", "w_out"]):
        c = Case(tokens, 320, 448, torch.bfloat16, seed=tokens, pad=8, offset=8)
        for name in names:
            setattr(c, name, getattr(odd, name))
        c.forward("gelu")
        check("y", c.r["y"], want["y"])
        check("gu", c.r["gu"], want["gu"])


@pytest.mark.parametrize("pad,offset", [(0, 0), (8, 8), (3, 1), (2, 1)])
@pytest.mark.parametrize("size", [(17, 1000, 2000), (20, 40, 24), (29, 70, 3000), (32, 511, 2000), (33, 600, 1200), (40, 1001, 2729), (47, 400, 3500), (48, 360, 3501), (50, 2048, 1500),
                                  (63, 2049, 264), (64, 512, 1536), (64, 300, 333), (65, 512, 1536)])
def test_up_to_64_rows(size, pad, offset):
    c = Case(*size, torch.bfloat16 if (size[0] + pad) % 2 else torch.float16, seed=size[2], pad=pad, offset=offset)
    want = reference(c.x, c.w_in, c.w_out, "silu", c.dtype)
    for keep in (True, False):
        c.r["y"].fill_(3.0)
        c.forward("silu", keep)
        check("y", c.r["y"], want["y"])
    check("gu", c.r["gu"], want["gu"])
    for name in ("y", "gu"):                # what lies beside the results stays
        values, memory = c.results[name]
        values.fill_(c.SENTINEL)
        assert bool((memory == c.SENTINEL).all())
