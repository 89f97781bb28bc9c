"""GPU test of AdamW in the small language model where gradients overflow: such a step changes nothing, and those behind it are what they would have been without it."""
import pytest
import torch

from paper_2009_12263_amd.language_model import AdamW, LanguageModel, chain

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("bad", [0, 1, 2])
def test_a_step_that_overflows_leaves_no_trace(bad, bits):
    models = [LanguageModel(96, 300, 64, seed=4, hidden=72) for _ in range(2)]
    updates = [AdamW(m, bits) for m in models]
    for k in range(3):
        text = chain(96, 300, k)
        if k == bad:
            plain = models[0].mean_grads

            def overflowed(*args):
                loss, grads = plain(*args)
                grads["W_in"][3, 5] = float("inf")
                return loss, grads
            models[0].mean_grads = overflowed
            before = {n: p.clone() for n, p in models[0].params.items()}
            updates[0].step(*text, 0.01)
            models[0].mean_grads = plain
            assert not bool(torch.isfinite(updates[0].factor))
            assert all(torch.equal(p, before[n]) for n, p in models[0].params.items())
        for u in updates:
            u.step(*text, 0.01)
        assert int(updates[0].count) == int(updates[1].count) == k + 1
        for name in models[0].params:
            assert torch.equal(models[0].params[name], models[1].params[name]), (k, name)
