"""Norms, experts and distillation together, as a training step uses them: the demonstration's gradients against automatic differentiation in 64
bits, and that it runs."""
import math

import pytest
import torch

from paper_2509_11254_amd import demo_experts

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("temperature", [1.0, 2.0])
def test_gradients_against_autograd(temperature):
    model = demo_experts.Model(tokens=200, d=72, hidden=144, experts=3, slots=2, vocab=333, top=9, temperature=temperature, seed=3)
    for i, v in enumerate(model.vectors):
        v += 0.2 * torch.randn(v.shape, generator=torch.Generator().manual_seed(i)).cuda()
    tokens, index, teacher = model.batch()
    got = [torch.empty(s, dtype=torch.bfloat16, device="cuda") for s in model.shapes]
    got_vectors = [torch.empty_like(v) for v in model.vectors]
    loss = model.gradients(tokens, index, teacher, got, got_vectors)

    w = [x.bfloat16().double().cpu().requires_grad_() for x in model.weights]
    v = [x.double().cpu().requires_grad_() for x in model.vectors]
    x = model.table[tokens].double().cpu()
    norm = torch.nn.functional.layer_norm
    a = norm(x, (72,), v[0], v[1])
    # which experts were chosen is no function of the weights: the library's own, wherever two are all but alike
    place, offsets = model.order.place.cpu(), model.order.offsets.cpu()
    choice = torch.searchsorted(offsets[1:].contiguous(), place.reshape(-1).contiguous(), right=True).view(place.shape)
    weight = torch.softmax((a @ w[-2].T).gather(1, choice), 1)
    mixed = 0.0
    for s in range(2):
        each = [torch.nn.functional.silu(a @ w[3 * e].T) * (a @ w[3 * e + 1].T) @ w[3 * e + 2].T for e in range(3)]
        picked = torch.stack(each, 1)[torch.arange(200), choice[:, s]]
        mixed = mixed + weight[:, s:s + 1] * picked
    y = norm(x + mixed, (72,), v[2], v[3])
    log_p = torch.log_softmax(y @ w[-1].T / temperature, 1)
    index, teacher = index.cpu(), teacher.double().cpu()
    counted = (index >= 0).any(1)
    q = torch.softmax(teacher / temperature, 1)
    want = torch.where(counted, (q * (q.log() - log_p.gather(1, index.clamp(min=0)))).sum(1), 0.0)
    # as for the gated unit alone: activations in bf16 and some of them in 8 bits with a common scale, 2^-9 and 2^-8 of an element's size each, a dozen of them
    # one after the other, and none adds up
    assert (loss.double().cpu() - want).abs().max() < 0.15
    (want.sum() / counted.sum()).backward()
    for name, g, b in zip(["gate", "up", "down"] * 3 + ["router", "head"] + ["weight", "bias"] * 2, got + got_vectors, w + v):
        error = (g.double().cpu() - b.grad).norm() / b.grad.norm()
        assert error < 0.05, (name, float(error))


def test_it_runs():
    losses = demo_experts.run(steps=25)
    print("loss %.3f -> %.3f" % (losses[0], losses[-1]))
    assert len(losses) == 25 and all(math.isfinite(x) and x >= 0 for x in losses)
