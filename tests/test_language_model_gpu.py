"""GPU test of the operators at work together: the gradients of the small language model against torch's in 64 bits, and its training.

Tolerance of a gradient: every activation and gradient of an activation is rounded to bfloat16 (2^-9 of itself, half a unit in the
last place relative to the norm), nine of them on the longest way from the loss to the table; errors of that size in a chain of
as many maps of condition near 1 stay within 9 * 2^-8 of the gradient's norm, and are allowed 2 ** -4."""
import torch

import pytest

from paper_2009_12263_amd.language_model import LanguageModel, chain, main

pytestmark = pytest.mark.gpu


def test_gradients():
    T, V, K = 320, 1001, 128
    model = LanguageModel(T, V, K, seed=3)
    ids, targets = chain(T, V, 5)
    ids[7] = -1
    loss = model.forward(ids, targets)
    dloss = torch.rand(T, device="cuda") / T
    got = {k: v.clone() for k, v in model.backward(ids, targets, dloss).items()}
    p = {k: v.double().cpu().requires_grad_() for k, v in model.params.items()}
    i, t = ids.cpu(), targets.cpu()
    norm = torch.nn.functional.layer_norm
    h = model.embed_scale * p["table"][i.clamp(min=0)] * (i >= 0)[:, None]
    a = norm(h, (K,), p["gamma1"], p["beta1"], model.EPS)
    n = norm(torch.relu(a @ p["W"].T + p["b"]), (K,), p["gamma2"], p["beta2"], model.EPS)
    z = model.logit_scale * n @ p["table"].T
    want = torch.where(t >= 0, torch.logsumexp(z, 1) - z.gather(1, t.clamp(min=0)[:, None])[:, 0], 0.0)
    (want * dloss.double().cpu()).sum().backward()
    assert (loss.double().cpu() - want.detach()).norm() <= 2 ** -6 * want.detach().norm()
    for k, v in got.items():
        g = p[k].grad
        assert (v.double().cpu() - g).norm() <= 2 ** -4 * g.norm(), (k, float((v.double().cpu() - g).norm() / g.norm()))


def test_training_learns_the_chain():
    # the best loss of the chain, 0.75 and 0.25 / V mixed, is 0.56 + 0.25 log V = 2.3 for V = 1024; log V = 6.9 knows nothing
    assert main(["--steps", "150", "--tokens", "2048", "--vocab", "1024", "--dim", "256"]) < 4.0
