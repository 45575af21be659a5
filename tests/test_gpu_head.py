"""The output head's loss and gradients against the definition in 64 bits."""
import math

import pytest
import torch

from paper_2509_11254_amd import psgd
from test_gpu_act import CODE, DT, UNIT, padded

pytestmark = pytest.mark.gpu

# (tokens, d, vocab): single tokens, one column, less than a tile, odd sizes, tile borders, several tiles and splits
SIZES = [(1, 8, 1), (1, 1, 2), (3, 64, 255), (2, 515, 256), (64, 72, 257), (65, 64, 1000), (130, 40, 512), (257, 200, 1031), (300, 520, 33),
         (513, 264, 300), (40, 1032, 5003)]


def inputs(tokens, d, vocab, dtype, seed, masked=0.2, extra=8):
    gen = torch.Generator().manual_seed(seed)
    w = torch.randn((vocab, d), generator=gen, dtype=torch.float64) / math.sqrt(d)
    labels = torch.randint(0, vocab, (tokens,), generator=gen)
    x = torch.randn((tokens, d), generator=gen, dtype=torch.float64) + 12 * torch.rand((tokens, 1), generator=gen) * w[labels]
    out = torch.rand(tokens, generator=gen) < masked
    labels = torch.where(out, torch.where(torch.rand(tokens, generator=gen) < 0.5, -100, vocab), labels)
    # what a token that does not count holds is looked at nowhere
    x[out] = float("nan")
    return padded(x, dtype, extra)[0], padded(w, dtype, extra)[0], labels.cuda()


def plain(x, w, labels, weight=None):
    """loss, D, dX, dW in 64 bits, by the formulas."""
    x, w, labels = x.double().cpu(), w.double().cpu(), labels.cpu()
    counted = (labels >= 0) & (labels < w.shape[0])
    x = torch.where(counted[:, None], x, 0.0)
    at = torch.where(counted, labels, 0)[:, None]
    logits = x @ w.T
    lse = torch.logsumexp(logits, 1, keepdim=True)
    loss = torch.where(counted, (lse - logits.gather(1, at))[:, 0], 0.0)
    c = weight.double().cpu() if weight is not None else torch.full((len(labels),), 1.0 / max(1, int(counted.sum())), dtype=torch.float64)
    D = torch.exp(logits - lse)
    D.scatter_add_(1, at, -torch.ones_like(lse))
    D *= torch.where(counted, c, 0.0)[:, None]
    return loss, D, D @ w, D.T @ x, x


def logit_error(x, w):
    """Bound of a logit's error: d products (exact for bf16, 24 bits for fp32) summed in fp32, sixteen at a time."""
    d = x.shape[1]
    return (d / 16 + 32) * 2.0 ** -24 * x.norm(dim=1).max() * w.double().cpu().norm(dim=1).max()


def check(x, w, labels, loss, dx, dw, weight, before=None):
    dtype, g_dtype = x.dtype, dw.dtype
    l64, D, dx64, dw64, x0 = plain(x, w, labels, weight)
    w64, err = w.double().cpu(), logit_error(x0, w)
    assert ((loss.double().cpu() - l64).abs() <= 2 * err + 2.0 ** -21 * (1 + l64.abs())).all()
    # D relative to its elements: the logits' error and a few fp32 roundings, and where it is one or two bf16 planes their rounding
    base = 2 * (2 * err + 2.0 ** -20)
    p = D.abs() + 0.0
    for got, want, other, planes, length, out in (
            (dx, dx64, w64, 1 if dtype == torch.bfloat16 else 3, w.shape[0], dtype),
            (dw, dw64, x0, 3 if dtype == torch.float32 and g_dtype == torch.float32 else 2 if torch.float32 in (dtype, g_dtype) else 1,
             x.shape[0], g_dtype)):
        terms = (p @ other.abs()) if got is dx else (p.T @ other.abs())
        # e^(l - max) has absolute errors as well: fp16's 2^-25 / 2^15 of c where it is below the normal numbers
        most_c = D.abs().max() * 2 + 1e-30
        tiny = 2.0 ** -38 * most_c * (other.abs().sum(0, keepdim=True) if got is dx else other.abs().sum(0, keepdim=True))
        rel = base + 2.0 ** (-8 * planes) * 1.01 + (length / 16 + 32) * 2.0 ** -24
        unit = 2.0 ** -8 if out == torch.bfloat16 else 2.0 ** -24
        if got is dw and before is not None:
            want = want + before
            terms = terms + before.abs() * 2.0 ** -8
        bound = rel * terms + unit * want.abs() * 1.01 + tiny
        assert ((got.double().cpu() - want).abs() <= bound).all(), ("dx" if got is dx else "dw")


def run(tokens, d, vocab, dtype, g_dtype, *, seed=1, masked=0.2, weighted=False, accumulate=False, piece=0, plan=None):
    x, w, labels = inputs(tokens, d, vocab, DT[dtype], seed, masked)
    weight = torch.rand(tokens, generator=torch.Generator().manual_seed(seed)).cuda() if weighted else None
    loss = torch.full((tokens,), float("nan"), device="cuda")
    dx, dx_buf = padded(torch.full((tokens, d), float("nan")), DT[dtype], 8)
    before = torch.randn((vocab, d), generator=torch.Generator().manual_seed(3), dtype=torch.float64) if accumulate else None
    dw, dw_buf = padded(before if accumulate else torch.full((vocab, d), float("nan")), DT[g_dtype], 16)
    before = dw.double().cpu().clone() if accumulate else None
    plan = plan or psgd.HeadLoss(tokens, d, vocab, CODE[dtype], CODE[g_dtype], piece_tokens=piece)
    plan.workspace.fill_(0xFF)                # NaN in every type: nothing is expected of a workspace
    plan.loss_grad(x, w, labels, loss, dx, dw, weight=weight, accumulate=accumulate)
    check(x, w, labels, loss, dx, dw, weight, before)
    out = ~((labels >= 0) & (labels < vocab))
    assert (loss[out] == 0).all() and (dx[out] == 0).all()
    assert dx_buf[:, d:].isnan().all() and dw_buf[:, d:].isnan().all()
    alone = torch.full((tokens,), float("nan"), device="cuda")
    plan.workspace.fill_(0xFF)
    plan.loss(x, w, labels, alone)
    assert torch.equal(alone, loss)
    return loss, dx, dw


@pytest.mark.parametrize("dtype,g_dtype", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("tokens,d,vocab", SIZES)
def test_loss_and_gradients(tokens, d, vocab, dtype, g_dtype):
    run(tokens, d, vocab, dtype, g_dtype)


@pytest.mark.parametrize("dtype,g_dtype", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("weighted,accumulate,piece", [(True, False, 0), (False, True, 0), (True, True, 100), (False, False, 64), (False, True, 7)])
def test_weights_sums_and_pieces(dtype, g_dtype, weighted, accumulate, piece):
    run(333, 136, 700, dtype, g_dtype, weighted=weighted, accumulate=accumulate, piece=piece)


@pytest.mark.parametrize("tokens,d,vocab", [(1, 41, 9001), (65, 95, 33000), (130, 1028, 5000), (900, 33, 6001), (1500, 260, 3001)])
def test_fp32_over_tiles(tokens, d, vocab):
    """Wide and narrow tiles, contractions in parts that end inside four elements, one token to many."""
    run(tokens, d, vocab, "f32", "f32", masked=0.1)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("piece", [0, 32])
@pytest.mark.parametrize("dtype,g_dtype", [("bf16", "bf16"), ("f32", "f32")])
def test_no_token_counts(dtype, g_dtype, piece, accumulate):
    """All labels outside the vocabulary, in one piece and in several of which none has tokens: zeros, no NaN."""
    loss, dx, dw = run(100, 72, 300, dtype, g_dtype, masked=2.0, piece=piece, accumulate=accumulate)
    assert (loss == 0).all() and (dx == 0).all() and torch.isfinite(dw).all()


@pytest.mark.parametrize("masked", [0.0, 0.9])
def test_later_pieces_without_tokens(masked):
    """Tokens that count are taken together, so that most of the pieces find none."""
    run(1000, 64, 400, "bf16", "f32", masked=masked, piece=128)


def test_no_tokens():
    plan = psgd.HeadLoss(0, 64, 100, psgd.PSGD_BF16, psgd.PSGD_F32)
    x, w = torch.empty((0, 64), dtype=torch.bfloat16, device="cuda"), torch.ones((100, 64), dtype=torch.bfloat16, device="cuda")
    labels, loss = torch.empty(0, dtype=torch.int64, device="cuda"), torch.empty(0, device="cuda")
    dw = torch.ones((100, 64), device="cuda")
    plan.loss_grad(x, w, labels, loss, torch.empty_like(x), dw, accumulate=True)
    assert (dw == 1).all()
    plan.loss_grad(x, w, labels, loss, torch.empty_like(x), dw)
    assert (dw == 0).all()


@pytest.mark.parametrize("shift", [1e4, -1e4])
def test_large_logits(shift):
    """All logits of a token far from zero: the softmax does not change, and nothing overflows."""
    d, vocab = 64, 600
    gen = torch.Generator().manual_seed(5)
    w = torch.randn((vocab, d), generator=gen) / 8
    w[:, 0] = 1.0
    x = torch.randn((20, d), generator=gen)
    x[:, 0] = shift
    x, w = padded(x, torch.bfloat16)[0], padded(w, torch.bfloat16)[0]
    labels = torch.randint(0, vocab, (20,), generator=gen).cuda()
    loss, dx, dw = torch.empty(20, device="cuda"), torch.empty_like(x), torch.empty((vocab, d), dtype=torch.bfloat16, device="cuda")
    psgd.HeadLoss(20, d, vocab).loss_grad(x, w, labels, loss, dx, dw)
    check(x, w, labels, loss, dx, dw, None)


def test_a_certain_token():
    """A label whose probability is all but one: its D is the difference of nearly equal numbers."""
    d, vocab = 128, 1000
    gen = torch.Generator().manual_seed(6)
    w = torch.randn((vocab, d), generator=gen)
    labels = torch.randint(0, vocab, (64,), generator=gen)
    x = w[labels] * torch.linspace(0.05, 0.3, 64)[:, None]
    x, w = padded(x, torch.float32)[0], padded(w, torch.float32)[0]
    loss, dx, dw = torch.empty(64, device="cuda"), torch.empty_like(x), torch.empty_like(w)
    psgd.HeadLoss(64, d, vocab, psgd.PSGD_F32).loss_grad(x, w, labels.cuda(), loss, dx, dw)
    l64, D, dx64, dw64, x0 = plain(x, w, labels)
    assert l64.min() < 1e-6
    # the loss is lse - logit: its error is that of fp32 numbers of the logits' size
    err = logit_error(x0, w) + 2.0 ** -22 * 64
    assert ((loss.double().cpu() - l64).abs() <= 2 * err).all()
    assert ((dx.double().cpu() - dx64).abs() <= (4 * err / 64) * w.double().cpu().abs().sum(0).max()).all()


def test_gradients_against_differences():
    """<dX, U> and <dW, V> against central differences of the loss that the library itself computes (fp32)."""
    tokens, d, vocab = 48, 40, 300
    x, w, labels = inputs(tokens, d, vocab, torch.float32, 9, masked=0.0)
    plan = psgd.HeadLoss(tokens, d, vocab, psgd.PSGD_F32)
    loss, dx, dw = torch.empty(tokens, device="cuda"), torch.empty_like(x), torch.empty((vocab, d), device="cuda")
    weight = torch.ones(tokens, device="cuda")
    plan.loss_grad(x, w, labels, loss, dx, dw, weight=weight)
    gen = torch.Generator().manual_seed(10)
    step = 2.0 ** -6

    def total(xx, ww):
        out = torch.empty(tokens, device="cuda")
        plan.loss(padded(xx, torch.float32, 8)[0], padded(ww, torch.float32, 8)[0], labels, out)
        return float(out.double().sum())

    for _ in range(4):
        u = torch.randn((tokens, d), generator=gen).cuda()
        v = (torch.randn((vocab, d), generator=gen) / math.sqrt(d)).cuda()
        # logits move by at most a = step max|u| max|w| (resp. max|x| max|v|): the third derivative of lse along a line is below a^3, over
        # the tokens, and a loss is good to 2^-19 of its size
        for along, got, reach in (((u, None), float((dx.double() * u.double()).sum()), u.norm(dim=1).max() * w.norm(dim=1).max()),
                                  ((None, v), float((dw.double() * v.double()).sum()), x.norm(dim=1).max() * v.norm(dim=1).max())):
            a, b = along
            plus = total(x + step * a if a is not None else x, w + step * b if b is not None else w)
            minus = total(x - step * a if a is not None else x, w - step * b if b is not None else w)
            bound = tokens * (step ** 2 * min(float(reach), 30.0) ** 3 / 6 + 2.0 ** -19 * 20 / step)
            assert abs((plus - minus) / (2 * step) - got) <= bound
            # and it is no trivial bound
            assert bound < 40 * tokens


def test_the_same_every_time_and_on_another_stream():
    x, w, labels = inputs(700, 264, 3000, torch.bfloat16, 11)
    plan = psgd.HeadLoss(700, 264, 3000, psgd.PSGD_BF16, psgd.PSGD_F32)
    got = []
    for stream in (torch.cuda.current_stream(), torch.cuda.current_stream(), torch.cuda.Stream()):
        loss, dx, dw = torch.empty(700, device="cuda"), torch.empty_like(x), torch.empty((3000, 264), device="cuda")
        stream.wait_stream(torch.cuda.current_stream())
        plan.loss_grad(x, w, labels, loss, dx, dw, stream=stream)
        torch.cuda.synchronize()
        got.append((loss, dx, dw))
    for other in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(got[0], other))


def test_in_a_graph():
    """Replayed with other labels, of which another number counts."""
    tokens, d, vocab = 300, 136, 900
    x, w, labels = inputs(tokens, d, vocab, torch.bfloat16, 12, masked=0.0)
    plan = psgd.HeadLoss(tokens, d, vocab, piece_tokens=128)
    loss, dx, dw = torch.empty(tokens, device="cuda"), torch.empty_like(x), torch.empty((vocab, d), dtype=torch.bfloat16, device="cuda")
    plan.loss_grad(x, w, labels, loss, dx, dw)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.loss_grad(x, w, labels, loss, dx, dw)
    for part in (0.0, 0.5, 1.0, 0.2):
        labels.copy_(torch.where(torch.rand(tokens, device="cuda") < part, -100, torch.randint(0, vocab, (tokens,), device="cuda")))
        graph.replay()
        got = [t.clone() for t in (loss, dx, dw)]
        plan.loss_grad(x, w, labels, loss, dx, dw)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (loss, dx, dw)))
