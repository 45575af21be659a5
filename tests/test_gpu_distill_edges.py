"""Distillation's gradients along themselves, where they are largest, against differences of the loss that the library itself computes."""
import math

import pytest
import torch

from paper_2509_11254_amd import psgd
from test_gpu_act import padded
from test_gpu_distill import inputs
from test_gpu_head import logit_error

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("temperature", [1.0, 1.5])
@pytest.mark.parametrize("which", ["dx", "dw"])
def test_gradients_against_differences(which, temperature):
    """A difference's error is a small part of the derivative here, and so is the loss' own."""
    tokens, d, vocab, top, h = 48, 40, 300, 12, 0.125
    x, w, index, teacher = inputs(tokens, d, vocab, top, torch.float32, 11, masked=0.0, ragged=0.1)
    plan = psgd.HeadDistill(tokens, d, vocab, top, psgd.PSGD_F32)
    loss, dx, dw = torch.empty(tokens, device="cuda"), torch.empty_like(x), torch.empty((vocab, d), device="cuda")
    plan.loss_grad(x, w, index, teacher, loss, dx, dw, temperature=temperature, weight=torch.ones(tokens, device="cuda"))
    gen = torch.Generator().manual_seed(12)

    def total(x, w):
        out = torch.empty(tokens, device="cuda")
        plan.loss(padded(x, torch.float32, 8)[0], padded(w, torch.float32, 8)[0], index, teacher, out, temperature=temperature)
        return float(out.double().sum())

    for _ in range(3):
        got = dx if which == "dx" else dw
        along = got.double() * (0.5 + torch.rand(got.shape, generator=gen, dtype=torch.float64).cuda())
        # how far the logits of a token move apart along it: at most by 1, for one of them
        move = (along @ w.double().t() if which == "dx" else x.double() @ along.t()) / temperature
        reach = move.amax(1) - move.amin(1)
        along, reach = along / reach.max(), reach / reach.max()
        step = (h * along).float()
        by_x, by_w = (step, 0.0) if which == "dx" else (0.0, step)
        difference = (total(x + by_x, w + by_w) - total(x - by_x, w - by_w)) / (2 * h)
        want = float((got.double() * step.double()).sum()) / h
        # The third derivative is the third central moment of what lies within `reach`, below a tenth of its third power; a loss is
        # off by two logits' errors and roundings of numbers of the size of their spread, 60 at most.
        noise = 2 * (2 * float(logit_error(x.double().cpu(), w)) / temperature + 2.0 ** -22 * 60) + 2.0 ** -20 * 32
        bound = float((h * h / 6 * reach ** 3 / 10).sum()) + tokens * noise / h
        assert abs(difference - want) <= bound, (difference, want, bound)
        assert bound < 0.1 * abs(want), (bound, want)
