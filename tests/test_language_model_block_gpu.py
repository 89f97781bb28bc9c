"""GPU test of the gated feed-forward block, the norm of the gradients and the AdamW step at work in the small language model: its gradients
against torch's in 64 bits, a step against the formulas, and its commands.

Tolerance of a gradient: rounded activations and gradients of activations as in the model with a plain hidden layer, nine on the longest way, and two more inside
the block (H, and dG or dU): eleven errors of 2^-9 of a norm each, in a chain of maps of condition near 1, stay within 11 * 2^-8 and are allowed 2 ** -4."""
import torch

import pytest

from paper_2009_12263_amd.language_model import AdamW, LanguageModel, chain, main

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens", [24, 320])
def test_gradients(tokens):
    T, V, K, H = tokens, 1001, 128, 200
    model = LanguageModel(T, V, K, seed=3, hidden=H)
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
    g, u = (a @ p["W_in"].T).split(H, 1)
    n = norm((torch.nn.functional.silu(g) * u) @ p["W_out"].T, (K,), p["gamma2"], p["beta2"], model.EPS)
    z = model.logit_scale * n @ p["table"].T
    want = torch.where(t >= 0, torch.logsumexp(z, 1) - z.gather(1, t.clamp(min=0)[:, None])[:, 0], 0.0)
    (want * dloss.double().cpu()).sum().backward()
    assert (loss.double().cpu() - want.detach()).norm() <= 2 ** -6 * want.detach().norm()
    assert set(got) == set(p)
    for k, v in got.items():
        g = p[k].grad
        assert (v.double().cpu() - g).norm() <= 2 ** -4 * g.norm(), (k, float((v.double().cpu() - g).norm() / g.norm()))


@pytest.mark.parametrize("hidden", [0, 96])
@pytest.mark.parametrize("bits", [32, 8])
def test_first_step(bits, hidden):
    """The first step from moments of zero moves each value by rate * g / (|g| + eps') and its decay, whatever the bits: within the rounding of the parameters and of the moments."""
    model = LanguageModel(128, 500, 64, seed=1, hidden=hidden)
    update = AdamW(model, bits)
    before = {k: v.double().clone() for k, v in model.params.items()}
    rate = 0.01
    update.step(*chain(128, 500, 2), rate)
    total = sum(float(g.double().square().sum()) for g in model.grads.values()) ** 0.5
    assert abs(float(update.norm) - total) <= 2 ** -22 * total
    factor = min(1.0, update.MAX_NORM / total)
    for i, (name, p) in enumerate(model.params.items()):
        g = model.grads[name].double() * factor
        want = before[name] * (1 - rate * update.DECAY) - rate * g / (g.abs() + update.EPS)
        at = update.masters[i] if update.masters[i] is not None else p
        # 1 - beta^1 rounded once, 14 further roundings of the update, 3 of the parameter
        bound = 40 * 2 ** -24 * rate + 3 * 2 ** -24 * before[name].abs()
        assert bool(((at.double() - want).abs() <= bound).all()), name
        if at is not p:
            assert torch.equal(p, at.to(p.dtype))
    assert int(update.count) == 1


@pytest.mark.parametrize("args", [["--hidden", "160"], ["--adamw", "32"], ["--hidden", "160", "--adamw", "32"], ["--hidden", "160", "--adamw", "8"]])
def test_commands(args):
    assert main(["--steps", "3", "--tokens", "200", "--vocab", "300", "--dim", "64"] + args) > 0.0


def test_captured_training_step():
    """Forward, backward, norm and AdamW as one graph, replayed on other text: the same bits as eager steps."""
    from paper_2009_12263_amd import binding as fg
    fg.fg_init()
    models = [LanguageModel(96, 300, 64, seed=2, hidden=72) for _ in range(2)]
    updates = [AdamW(m, 8) for m in models]
    ids, targets = chain(96, 300, 0)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):                   # (torch's own kernels of a step, once before they are captured)
        AdamW(LanguageModel(96, 300, 64, seed=9, hidden=72), 8).step(ids, targets, 0.01)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        loss = updates[0].step(ids, targets, 0.01)
    for k in range(3):
        new = chain(96, 300, k)
        ids.copy_(new[0])
        targets.copy_(new[1])
        graph.replay()
        want = updates[1].step(*new, 0.01)
        torch.cuda.synchronize()
        assert torch.equal(loss, want)
        for name in models[0].params:
            assert torch.equal(models[0].params[name], models[1].params[name]), (k, name)
