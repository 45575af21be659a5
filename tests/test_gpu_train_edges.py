"""The training operators at the ends of what their arguments may be."""
import math

import pytest
import torch

from paper_2509_11254_amd import psgd
from test_gpu_act import CODE, DT, padded
from test_gpu_head import inputs

pytestmark = pytest.mark.gpu


def test_losses_of_more_tokens_than_one_launch_takes():
    """More than 2^24 tokens and a small vocabulary: pieces that a launch of 256 threads for each token still takes."""
    tokens, d, vocab = (1 << 24) + 77, 8, 64
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    w = torch.randn((vocab, d), generator=gen, device="cuda").bfloat16()
    x = torch.randn((tokens, d), generator=gen, device="cuda").bfloat16()
    labels = torch.randint(-8, vocab, (tokens,), generator=gen, device="cuda")
    loss = torch.full((tokens,), float("nan"), device="cuda")
    psgd.HeadLoss(tokens, d, vocab, grad=False).loss(x, w, labels, loss)
    for first in range(0, tokens, 1 << 22):
        part = slice(first, min(tokens, first + (1 << 22)))
        logits = x[part].float() @ w.float().t()
        want = torch.logsumexp(logits, 1) - logits.gather(1, labels[part].clamp(min=0)[:, None])[:, 0]
        # eight products summed in fp32, here and there: 8 x 2^-24 of |x| |w|, up to 30, twice in a loss
        assert (loss[part] - torch.where(labels[part] >= 0, want, 0.0)).abs().max() < 1e-4


# up to 512 tokens whose rows need no padding X is multiplied where it is: few launches, two products in one or in two; else a copy of it
@pytest.mark.parametrize("tokens,d,vocab,dtype", [(200, 136, 1000, "bf16"), (16, 512, 4400, "bf16"), (500, 1024, 10008, "bf16"), (200, 131, 1000, "bf16"),
                                                 (700, 136, 1000, "bf16"), (90, 67, 300, "f32")])
def test_gradient_in_the_place_of_the_tokens(tokens, d, vocab, dtype):
    x, w, labels = inputs(tokens, d, vocab, DT[dtype], 4)
    plan = psgd.HeadLoss(tokens, d, vocab, CODE[dtype], psgd.PSGD_F32)
    results = []
    for in_place in (False, True):
        here = padded(x, DT[dtype], 8)[0]
        loss, dw = torch.empty(tokens, device="cuda"), torch.empty((vocab, (d + 7) // 8 * 8), device="cuda")[:, :d]
        dx = here if in_place else padded(torch.zeros((tokens, d)), DT[dtype], 8)[0]
        plan.workspace.fill_(0xFF)
        plan.loss_grad(here, w, labels, loss, dx, dw)
        results.append((loss, dx, dw))
    assert all(torch.equal(a, b) for a, b in zip(*results))
    assert torch.isfinite(results[1][2]).all() and (results[1][1] != 0).any()


def test_gradient_beside_the_tokens():
    """X and dX as columns of one buffer."""
    tokens, d, vocab = 100, 64, 300
    x, w, labels = inputs(tokens, d, vocab, torch.bfloat16, 5)
    plan = psgd.HeadLoss(tokens, d, vocab)
    results = []
    for right in (True, False, None):
        buf = torch.zeros((tokens, 2 * d), dtype=torch.bfloat16, device="cuda")
        here, dx = (buf[:, :d], buf[:, d:]) if right else (buf[:, d:], buf[:, :d])
        dx = torch.zeros((tokens, d), dtype=torch.bfloat16, device="cuda") if right is None else dx
        here.copy_(x)
        loss, dw = torch.empty(tokens, device="cuda"), torch.empty((vocab, d), dtype=torch.bfloat16, device="cuda")
        plan.loss_grad(here, w, labels, loss, dx, dw)
        results.append((loss, dx.clone(), dw))
    assert all(torch.equal(a, b) for r in results[:2] for a, b in zip(r, results[2]))


@pytest.mark.parametrize("gated", [False, True])
def test_gelu_far_below_zero(gated):
    """fp32, to -12, where the distribution function is 1e-33: its relative error, not that of one minus nearly one."""
    x = torch.linspace(-12, 0, 4096, dtype=torch.float64).reshape(16, 256)
    gate, _ = padded(x, torch.float32)
    up = padded(torch.full_like(x, 0.75), torch.float32)[0] if gated else None
    dh, _ = padded(torch.full_like(x, 0.5), torch.float32)
    h, dgate = (padded(torch.zeros_like(x), torch.float32)[0] for _ in range(2))
    dup = padded(torch.zeros_like(x), torch.float32)[0] if gated else None
    kg, ku = psgd.act_empty(16, 256), psgd.act_empty(16, 256) if gated else None
    psgd.act_glu(gate, up, h, kg, ku, act=psgd.PSGD_GELU)
    psgd.act_glu_backward(kg, ku, dh, dgate, dup, act=psgd.PSGD_GELU)
    kept, _ = padded(torch.zeros_like(x), torch.float32)
    psgd.act_restore(kg, kept)
    factor = 0.75 if gated else 1.0          # (0.75 is 96 times a power of two: exact in 8 bits)

    def parts(t):
        # the function and its density; an error of 2^-23 of x or of x^2 / 2 is x^2 times as much of either, the functions' own is a few 2^-24
        t = t.double().cpu()
        return t, 0.5 * torch.erfc(-t / math.sqrt(2)), torch.exp(-t * t / 2) / math.sqrt(2 * math.pi), 2.0 ** -20 + t * t * 2.0 ** -22

    g, cdf, _, unit = parts(gate)
    assert ((h.double().cpu() - g * cdf * factor).abs() <= unit * (g * cdf * factor).abs() + 1e-37).all()
    g, cdf, density, unit = parts(kept)
    want = 0.5 * factor * (cdf + g * density)
    assert ((dgate.double().cpu() - want).abs() <= unit * 0.5 * factor * (cdf + (g * density).abs()) + 1e-37).all()
    if gated:
        assert ((dup.double().cpu() - 0.5 * g * cdf).abs() <= unit * (0.5 * g * cdf).abs() + 1e-37).all()


@pytest.mark.parametrize("tokens", [20, 600])
def test_errors_of_others_before_the_call(tokens):
    """An error that an earlier HIP call of the program left behind (here: a device that does not exist) is not the library's: its calls do their work and
    say so."""
    d, vocab = 64, 300
    lib = psgd.load_library()
    x, w, labels = inputs(tokens, d, vocab, torch.bfloat16, 6)
    head, wgrad = psgd.HeadLoss(tokens, d, vocab), psgd.WeightGrad(tokens, d, d)
    gate = padded(torch.randn((tokens, d)), torch.bfloat16)[0]

    def step(before):
        loss, dx, dw = torch.zeros(tokens, device="cuda"), torch.zeros_like(gate), torch.zeros((vocab, d), dtype=torch.bfloat16, device="cuda")
        h, y, dg, du = (torch.zeros_like(gate) for _ in range(4))
        g = torch.zeros((d, d), dtype=torch.bfloat16, device="cuda")
        alone = torch.zeros_like(loss)
        kg, ku, kh = (psgd.act_empty(tokens, d) for _ in range(3))
        for call in (lambda: head.loss(x, w, labels, alone), lambda: head.loss_grad(x, w, labels, loss, dx, dw), lambda: psgd.act_glu(gate, gate, h, kg, ku),
                     lambda: psgd.act_store(h, kh), lambda: psgd.act_restore(kh, y), lambda: wgrad.run(gate, kh, g),
                     lambda: psgd.act_glu_backward(kg, ku, gate, dg, du)):
            before()
            call()
        return alone, loss, dx, dw, h, y, g, dg, du

    want = step(lambda: None)
    got = step(lambda: lib["hipSetDevice"](1 << 20))
    assert lib["hipGetLastError"]() in (0, 101)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
