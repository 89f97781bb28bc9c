"""GPU test of lists of the wrong length in a step of AdamW, empty ones among them: refused by the native marshalling as by the binding's."""
import pytest
import torch

from paper_2009_12263_amd import binding as fg

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("kind", [list, tuple])
def test_lists_of_the_wrong_length(native, kind, monkeypatch):
    if not native:
        monkeypatch.setattr(fg, "_fast", fg._CtypesOnly)
    new = lambda n, dtype=torch.float32: torch.zeros(n, device="cuda", dtype=dtype)
    params, avg, sq = kind([new(300, torch.bfloat16)]), kind([new(300)]), kind([new(300)])
    small = lambda: kind([new(300, torch.float8_e4m3fn)])
    step = torch.ones(1, dtype=torch.int64, device="cuda")
    call = lambda *lists, **kw: fg.fg_adamw(*lists, step, 1e-2, 0.9, 0.99, 1e-8, 0.1, **kw)
    for extra in (dict(masters=kind()), dict(avg_scales=kind(), sq_scales=kind()), dict(avg_scales=kind(), sq_scales=kind([new(2)])),
                  dict(avg_scales=kind([new(2)]), sq_scales=kind()), dict(masters=kind([new(300)] * 2)), dict(avg_scales=kind([new(2)]))):
        m, v = (small(), small()) if extra.get("avg_scales") else (avg, sq)
        with pytest.raises(ValueError, match="masters|scales"):
            call(params, params, m, v, **extra)
    for short in range(1, 4):
        with pytest.raises(ValueError, match="grads|exp_avg"):
            call(*(kind() if k == short else v for k, v in enumerate((params, kind([new(300, torch.bfloat16)]), avg, sq))))
    with pytest.raises(TypeError):
        call(None, None, None, None)
    for name in ("avg_scales", "sq_scales"):
        with pytest.raises(ValueError, match="both"):
            call(kind(), kind(), kind(), kind(), **{name: kind()})
    assert call(kind(), kind(), kind(), kind(), masters=kind(), avg_scales=kind(), sq_scales=kind()) == fg.FG_OK
