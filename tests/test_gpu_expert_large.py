"""Experts' rows in calls that are large enough for the non-temporal hint, and in sums that are exact, against plain implementations."""
import pytest
import torch

from paper_2509_11254_amd import psgd
from test_gpu_act import DT, UNIT, padded
from test_gpu_expert import sort

pytestmark = pytest.mark.gpu


def random_rows(rows, cols, dtype, seed, extra=8):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return padded(torch.randn((rows, cols), generator=gen, device="cuda"), DT[dtype], extra)


# 16 and 32 lanes to a row, one piece to a lane, several rounds of pieces; a row's end inside a piece
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pieces", [13, 25, 63, 501])
def test_large_calls(pieces, dtype):
    """Rows, combine with weights and its gradients, to other rows and in their place, 100 MiB and more; some choices do not count."""
    per = 4 if dtype == "f32" else 8
    cols, size, slots, experts = per * pieces - 3, 16 // per, 4, 30
    tokens = (100 << 20) // (slots * cols * size) + 77
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    order = sort(torch.randint(-2, experts, (tokens, slots), generator=gen, device="cuda"), experts)
    n, place = int(order.offsets[-1]), order.place.long()
    there, rows = place >= 0, order.order[:n].long()
    assert 0 < n < tokens * slots

    x, _ = random_rows(tokens, cols, dtype, 2)
    xs, xs_buf = random_rows(tokens * slots, cols, dtype, 3, 16)
    before = xs_buf.clone()
    psgd.expert_rows(x, order, xs)
    assert torch.equal(xs[:n], x[rows // slots])
    assert torch.equal(xs_buf.view(torch.uint8)[n:], before.view(torch.uint8)[n:]) and xs_buf[:, cols:].isnan().all()

    ys, ys_buf = random_rows(tokens * slots, cols, dtype, 4)
    weight = torch.randn((tokens, slots), generator=gen, device="cuda")
    w = torch.where(there, weight.double(), 0.0)
    y, y_buf = padded(torch.full((tokens, cols), float("nan")), DT[dtype], 16)
    psgd.expert_combine(ys, order, y, weight=weight)
    want, terms = torch.zeros((tokens, cols), dtype=torch.float64, device="cuda"), torch.zeros((tokens, cols), dtype=torch.float64, device="cuda")
    for s in range(slots):
        one = ys[place[:, s].clamp(min=0)].double() * w[:, s:s + 1]
        want += one
        terms += one.abs()
    assert ((y.double() - want).abs() <= slots * 2.0 ** -24 * terms + UNIT[dtype] * 1.01 * want.abs()).all() and y_buf[:, cols:].isnan().all()

    dy, _ = random_rows(tokens, cols, dtype, 5)
    want_dots, terms_dots = torch.zeros((tokens, slots), dtype=torch.float64, device="cuda"), torch.zeros((tokens, slots), dtype=torch.float64, device="cuda")
    for s in range(slots):
        one = torch.where(there[:, s:s + 1], ys[place[:, s].clamp(min=0)].double() * dy.double(), 0.0)
        want_dots[:, s], terms_dots[:, s] = one.sum(1), one.abs().sum(1)
    for in_place in (False, True):
        out, out_buf = (ys, ys_buf) if in_place else random_rows(tokens * slots, cols, dtype, 6, 24)
        before = out_buf.clone()
        dots = torch.full((tokens, slots), float("nan"), device="cuda")
        psgd.expert_combine_backward(dy, ys, order, out, weight=weight, dweight=dots)
        want = dy[rows // slots].double() * w.view(-1)[rows][:, None]
        assert ((out[:n].double() - want).abs() <= (UNIT[dtype] + 2.0 ** -24) * 1.01 * want.abs()).all()
        assert torch.equal(out_buf.view(torch.uint8)[n:], before.view(torch.uint8)[n:]) and out_buf[:, cols:].isnan().all()
        # a lane adds up a 16th of the columns at most, then up to 6 steps over the lanes
        assert ((dots.double() - want_dots).abs() <= (cols / 16 + 32) * 2.0 ** -24 * terms_dots).all() and (dots[~there] == 0).all()


def test_sums_of_very_many_tokens_are_exact():
    """24 million choices of whole numbers below a thousand: eight of them add up exactly, and no token's are its neighbour's."""
    tokens, slots, experts = 3000001, 8, 60
    choice = torch.randint(-2, experts + 2, (tokens, slots), generator=torch.Generator(device="cuda"), device="cuda")
    order = sort(choice, experts)
    x = (torch.arange(tokens, device="cuda") % 997 + 1).float()[:, None] * torch.tensor([1.0, 2, 3, 1, 2, 3, 1, 2], device="cuda")
    xs, y = torch.full((tokens * slots, 8), float("nan"), device="cuda"), torch.empty_like(x)
    psgd.expert_rows(x, order, xs)
    psgd.expert_combine(xs, order, y)
    there = ((choice >= 0) & (choice < experts)).sum(1)
    assert torch.equal(y, x * there[:, None].float())
