"""GPU test of the small language model's memory: it has the buffers that its steps use."""
import pytest
import torch

from paper_2009_12263_amd.language_model import LanguageModel, chain

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hidden", [0, 72])
def test_every_buffer_is_used(hidden):
    model = LanguageModel(96, 300, 64, hidden=hidden)
    text = chain(96, 300, 0)
    model.step(*text, 0.1)
    for buffer in vars(model).values():
        if torch.is_tensor(buffer):
            buffer.fill_(float("nan"))
    model.step(*text, 0.1)
    unused = [name for name, buffer in vars(model).items() if torch.is_tensor(buffer) and bool(buffer.isnan().all())]
    assert not unused, unused
