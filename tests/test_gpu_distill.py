"""Distillation from a teacher's top logits at the output head: loss and gradients against the definition in 64 bits."""
import math

import pytest
import torch

from paper_2509_11254_amd import psgd
from test_gpu_act import CODE, DT, padded
from test_gpu_head import logit_error

pytestmark = pytest.mark.gpu

# (tokens, d, vocab, top): one word, all words, more entries than words, odd sizes, tile borders, several tiles and splits, the most entries
SIZES = [(1, 8, 1, 1), (1, 1, 2, 2), (3, 64, 255, 9), (2, 515, 256, 64), (64, 72, 257, 20), (65, 64, 1000, 65), (130, 40, 512, 300), (257, 200, 1031, 7),
         (300, 520, 33, 40), (513, 264, 300, 3), (40, 1032, 5003, 1024), (700, 136, 900, 33), (45, 64, 3000, 256),
         (33, 72, 2000, 257), (50, 64, 1500, 512), (1100, 64, 700, 513)]


def inputs(tokens, d, vocab, top, dtype, seed, masked=0.2, ragged=0.2, extra=8, t_dtype=torch.float32, distinct=True):
    gen = torch.Generator().manual_seed(seed)
    w = torch.randn((vocab, d), generator=gen, dtype=torch.float64) / math.sqrt(d)
    if distinct and top <= vocab:
        # low words more often, as frequent ones are
        key = torch.rand((tokens, vocab), generator=gen) * torch.linspace(0.2, 1.0, vocab)
        index = key.topk(top, 1, largest=False).indices
        index = index.gather(1, torch.rand((tokens, top), generator=gen).argsort(1))
    else:
        index = (vocab * torch.rand((tokens, top), generator=gen) ** 2).long()
    teacher = 3 * torch.randn((tokens, top), generator=gen) + 10
    x = torch.randn((tokens, d), generator=gen, dtype=torch.float64) + 12 * torch.rand((tokens, 1), generator=gen) * w[index[:, 0]]
    gone = torch.rand((tokens, top), generator=gen) < ragged
    index = torch.where(gone, torch.where(torch.rand((tokens, top), generator=gen) < 0.5, -100, vocab), index)
    # an entry that does not count may hold anything, one of no probability names a word all the same
    teacher = torch.where(gone, float("nan"), torch.where(torch.rand((tokens, top), generator=gen) < 0.05, -math.inf, teacher))
    out = torch.rand(tokens, generator=gen) < masked
    index[out] = -1
    counts = ((index >= 0) & (index < vocab) & (teacher != -math.inf)).any(1)
    # what a token that does not count holds is looked at nowhere
    x[~counts] = float("nan")
    return padded(x, dtype, extra)[0], padded(w, dtype, extra)[0], index.cuda(), teacher.to(t_dtype).cuda()


def plain(x, w, index, teacher, temperature, weight=None):
    """loss, p, q, c / T, dX, dW in 64 bits, by the formulas."""
    x, w, index, teacher = x.double().cpu(), w.double().cpu(), index.cpu(), teacher.double().cpu()
    there = (index >= 0) & (index < w.shape[0]) & (teacher != -math.inf)
    counted = there.any(1)
    x = torch.where(counted[:, None], x, 0.0)
    z = torch.where(there, teacher / temperature, -math.inf)
    z[~counted] = 0.0
    q_entries = torch.where(there, torch.softmax(z, 1), 0.0)
    q = torch.zeros((x.shape[0], w.shape[0]), dtype=torch.float64)
    q.scatter_add_(1, torch.where(there, index, 0), q_entries)
    logits = x @ w.T / temperature
    log_p = logits - torch.logsumexp(logits, 1, keepdim=True)
    loss = torch.where(counted, (torch.special.xlogy(q, q) - q * log_p).sum(1), 0.0)
    c = weight.double().cpu() if weight is not None else torch.full((len(counted),), 1.0 / max(1, int(counted.sum())), dtype=torch.float64)
    c = (torch.where(counted, c, 0.0) / temperature)[:, None]
    D = c * (log_p.exp() - q)
    # how far apart logits are, the head's and the teacher's: what fp32 differences and logarithms of them are relative to
    zt = torch.where(there, z, z.amax(1, keepdim=True).clamp(min=-1e30))
    spread = (logits.amax(1) - logits.amin(1)).max() + (zt.amax(1) - zt.amin(1)).max() + math.log(w.shape[0]) + math.log(index.shape[1]) + 1
    return loss, log_p.exp(), q, log_p, c, D, D @ w, D.T @ x, x, counted, float(spread)


def check(x, w, index, teacher, temperature, loss, dx, dw, weight, before=None):
    dtype = x.dtype
    l64, p, q, log_p, c, D, dx64, dw64, x0, counted, spread = plain(x, w, index, teacher, temperature, weight)
    w64, err = w.double().cpu(), logit_error(x0, w) / temperature
    # u = log p - log q of a word: two logits' errors, and roundings of numbers of the size of their spread.  The loss moves by p - q times that,
    # and by the roundings of its terms
    du = 2 * err + 2.0 ** -22 * spread
    size = torch.where(q > 0, q * (torch.log(torch.where(q > 0, q, 1.0)) - log_p).abs(), 0.0).sum(1)
    assert ((loss.double().cpu() - l64).abs() <= 2 * du + 2.0 ** -20 * (2 + size)).all()
    assert (loss.cpu()[~counted] == 0).all()
    if dx is None:
        return
    g_dtype = dw.dtype
    for got, want, other, planes, length, out in (
            (dx, dx64, w64, 1 if dtype == torch.bfloat16 else 3, w.shape[0], dtype),
            (dw, dw64, x0, 3 if dtype == torch.float32 and g_dtype == torch.float32 else 2 if torch.float32 in (dtype, g_dtype) else 1,
             x.shape[0], g_dtype)):
        turn = (lambda m: m) if got is dx else (lambda m: m.T)
        # D's elements: p and q with u's error and a few roundings, then D in planes
        terms = turn(c.abs() * (p + q)) @ other.abs() * 2 * (du + 2.0 ** -20) + turn(D.abs()) @ other.abs() * (2.0 ** (-8 * planes) * 1.01 + (length / 16 + 32) * 2.0 ** -24)
        # e^(l - max) has absolute errors as well: fp16's 2^-25 / 2^15 of c where it is below the normal numbers
        tiny = 2.0 ** -38 * (c.abs().max() * 2 + 1e-30) * other.abs().sum(0, keepdim=True)
        unit = 2.0 ** -8 if out == torch.bfloat16 else 2.0 ** -24
        if got is dw and before is not None:
            want = want + before
            terms = terms + before.abs() * 2.0 ** -16
        assert ((got.double().cpu() - want).abs() <= terms + unit * want.abs() * 1.01 + tiny).all(), ("dx" if got is dx else "dw")
    assert (dx.cpu()[~counted] == 0).all()


def run(tokens, d, vocab, top, dtype, g_dtype, *, seed=1, masked=0.2, ragged=0.2, temperature=1.0, weighted=False, accumulate=False, piece=0, t_dtype="f32",
        distinct=True):
    x, w, index, teacher = inputs(tokens, d, vocab, top, DT[dtype], seed, masked, ragged, t_dtype=DT[t_dtype], distinct=distinct)
    weight = torch.rand(tokens, generator=torch.Generator().manual_seed(seed)).cuda() if weighted else None
    loss = torch.full((tokens,), float("nan"), device="cuda")
    dx, dx_buf = padded(torch.full((tokens, d), float("nan")), DT[dtype], 8)
    before = torch.randn((vocab, d), generator=torch.Generator().manual_seed(3), dtype=torch.float64) if accumulate else None
    dw, dw_buf = padded(before if accumulate else torch.full((vocab, d), float("nan")), DT[g_dtype], 16)
    before = dw.double().cpu().clone() if accumulate else None
    plan = psgd.HeadDistill(tokens, d, vocab, top, CODE[dtype], CODE[g_dtype], piece_tokens=piece)
    plan.workspace.fill_(0xFF)                # NaN in every type: nothing is expected of a workspace
    plan.loss_grad(x, w, index, teacher, loss, dx, dw, temperature=temperature, weight=weight, accumulate=accumulate)
    check(x, w, index, teacher, temperature, loss, dx, dw, weight, before)
    assert dx_buf[:, d:].isnan().all() and dw_buf[:, d:].isnan().all()
    alone = torch.full((tokens,), float("nan"), device="cuda")
    plan.workspace.fill_(0xFF)
    plan.loss(x, w, index, teacher, alone, temperature=temperature)
    assert torch.equal(alone, loss)
    return loss, dx, dw


@pytest.mark.parametrize("dtype,g_dtype", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("tokens,d,vocab,top", SIZES)
def test_loss_and_gradients(tokens, d, vocab, top, dtype, g_dtype):
    run(tokens, d, vocab, top, dtype, g_dtype)


@pytest.mark.parametrize("dtype,g_dtype", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("change", [dict(weighted=True), dict(accumulate=True), dict(weighted=True, accumulate=True, piece=100), dict(piece=64), dict(piece=7, accumulate=True),
                                    dict(temperature=3.0), dict(temperature=0.25, weighted=True, piece=50), dict(t_dtype="bf16", temperature=2.0), dict(ragged=0.0, masked=0.0)])
def test_variants(dtype, g_dtype, change):
    run(333, 136, 700, 24, dtype, g_dtype, **change)


@pytest.mark.parametrize("tokens", [30, 600])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_words_that_several_entries_name(dtype, tokens):
    """Their probabilities are added up."""
    run(tokens, 72, 50, 100, dtype, "f32", distinct=False)


@pytest.mark.parametrize("tokens,dtype,vocab", [(5, "bf16", 700001), (3, "f32", 300001), (300, "bf16", 560000)])
def test_more_tiles_than_ranges_of_words(tokens, dtype, vocab):
    """Vocabularies of more tiles than the lists have ranges for: several tiles look through the same entries."""
    d, top = 8, 40
    x, w, index, teacher = inputs(tokens, d, vocab, top, DT[dtype], 21, distinct=False, masked=0.0)
    index[0, :6], teacher[0, :6] = torch.tensor([0, vocab - 1, 127, 128, 255, 256]), torch.arange(6.0)
    loss, dx, dw = torch.empty(tokens, device="cuda"), torch.empty_like(x), torch.empty((vocab, d), dtype=DT[dtype], device="cuda")
    psgd.HeadDistill(tokens, d, vocab, top, CODE[dtype]).loss_grad(x, w, index, teacher, loss, dx, dw)
    rows = list(range(0, tokens, 97)) if tokens > 100 else list(range(tokens))
    check(x[rows], w, index[rows], teacher[rows], 1.0, loss[rows], None, None, None)
    if tokens < 100:
        check(x, w, index, teacher, 1.0, loss, dx, dw, None)


def test_extreme_temperatures():
    """At 1e-30 the largest logit has all probability, on both sides; at 1e30 all words have the same, and the entries the same among them."""
    tokens, d, vocab, top = 20, 64, 500, 6
    x, w, index, teacher = inputs(tokens, d, vocab, top, torch.float32, 22, masked=0.0, ragged=0.0)
    teacher = torch.randn((tokens, top), device="cuda")
    best = index.gather(1, teacher.argmax(1, keepdim=True))[:, 0]
    x = torch.nan_to_num(x)
    x[:10] = 30 * w[best[:10]]                # these know the teacher's word
    plan, loss = psgd.HeadDistill(tokens, d, vocab, top, psgd.PSGD_F32, grad=False), torch.empty(tokens, device="cuda")
    plan.loss(padded(x, torch.float32, 8)[0], w, index, teacher, loss, temperature=1e-30)
    knows = (x.double() @ w.double().t()).argmax(1) == best
    assert (loss[knows] == 0).all() and (loss[~knows] > 1).all() and knows[:10].all() and not knows.all()
    plan.loss(padded(x, torch.float32, 8)[0], w, index, teacher, loss, temperature=1e30)
    assert (loss - math.log(vocab / top)).abs().max() < 2.0 ** -20 * 10


def test_entries_in_another_order():
    """The same bits, whatever the order of a token's entries."""
    tokens, d, vocab, top = 90, 72, 800, 50
    x, w, index, teacher = inputs(tokens, d, vocab, top, torch.bfloat16, 7)
    turn = torch.rand((tokens, top), device="cuda").argsort(1)
    plan = psgd.HeadDistill(tokens, d, vocab, top)
    got = []
    for i, t in ((index, teacher), (index.gather(1, turn), teacher.gather(1, turn))):
        loss, dx, dw = torch.empty(tokens, device="cuda"), torch.empty_like(x), torch.empty((vocab, d), dtype=torch.bfloat16, device="cuda")
        plan.loss_grad(x, w, i, t, loss, dx, dw)
        got.append((loss, dx, dw))
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_entries_as_columns_of_larger_ones():
    """The first 16 of 40 entries, a stride of 40."""
    tokens, d, vocab = 60, 72, 800
    x, w, index, teacher = inputs(tokens, d, vocab, 40, torch.float32, 8, masked=0.0)
    plan = psgd.HeadDistill(tokens, d, vocab, 16, psgd.PSGD_F32, grad=False)
    a, b = torch.empty(tokens, device="cuda"), torch.empty(tokens, device="cuda")
    plan.loss(x, w, index[:, :16], teacher[:, :16], a)
    plan.loss(x, w, index[:, :16].contiguous(), teacher[:, :16].contiguous(), b)
    assert torch.equal(a, b) and (a > 0).any()


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("piece", [0, 32])
@pytest.mark.parametrize("tokens", [100, 600])
@pytest.mark.parametrize("dtype,g_dtype", [("bf16", "bf16"), ("f32", "f32")])
def test_no_token_counts(dtype, g_dtype, tokens, piece, accumulate):
    loss, dx, dw = run(tokens, 72, 300, 10, dtype, g_dtype, masked=2.0, piece=piece, accumulate=accumulate)
    assert (loss == 0).all() and (dx == 0).all() and torch.isfinite(dw).all()


@pytest.mark.parametrize("masked", [0.0, 0.9])
def test_later_pieces_without_tokens(masked):
    run(1000, 64, 400, 12, "bf16", "f32", masked=masked, piece=128)


def test_no_tokens():
    plan = psgd.HeadDistill(0, 64, 100, 5, psgd.PSGD_BF16, psgd.PSGD_F32)
    x, w = torch.empty((0, 64), dtype=torch.bfloat16, device="cuda"), torch.ones((100, 64), dtype=torch.bfloat16, device="cuda")
    index, teacher, loss = torch.empty((0, 5), dtype=torch.int64, device="cuda"), torch.empty((0, 5), device="cuda"), torch.empty(0, device="cuda")
    dw = torch.ones((100, 64), device="cuda")
    plan.loss_grad(x, w, index, teacher, loss, torch.empty_like(x), dw, accumulate=True)
    assert (dw == 1).all()
    plan.loss_grad(x, w, index, teacher, loss, torch.empty_like(x), dw)
    assert (dw == 0).all()


@pytest.mark.parametrize("tokens", [100, 700])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_entry_is_a_label(dtype, tokens):
    """A teacher of one entry is the cross entropy against that word."""
    d, vocab = 136, 900
    x, w, index, _ = inputs(tokens, d, vocab, 1, DT[dtype], 9, ragged=0.0)
    index[x.isnan().any(1)] = -1            # (tokens whose only entry had no probability; here it has)
    teacher = torch.randn((tokens, 1), device="cuda")
    results = []
    for kind in range(2):
        loss, dx, dw = torch.empty(tokens, device="cuda"), torch.empty_like(x), torch.empty((vocab, d), device="cuda")
        if kind:
            psgd.HeadDistill(tokens, d, vocab, 1, CODE[dtype], psgd.PSGD_F32).loss_grad(x, w, index, teacher, loss, dx, dw)
        else:
            psgd.HeadLoss(tokens, d, vocab, CODE[dtype], psgd.PSGD_F32).loss_grad(x, w, index[:, 0].contiguous(), loss, dx, dw)
        results.append((loss.double(), dx.double(), dw.double()))
    # both have fp32 statistics of the same logits: a few roundings of the loss' parts (logarithms up to 20), and of a gradient's
    assert (results[0][0] - results[1][0]).abs().max() < 2.0 ** -20 * 20
    for a, b in zip(results[0][1:], results[1][1:]):
        assert (a - b).norm() < 2.0 ** -9 * a.norm()


def test_a_student_that_knows_its_teacher():
    """The teacher's entries are the head's own logits of all words: the loss is 0 and so are the gradients, to the logits' error."""
    tokens, d, vocab = 50, 64, 200
    x, w, _, _ = inputs(tokens, d, vocab, 1, torch.float32, 10, masked=0.0, ragged=0.0)
    x = torch.nan_to_num(x)
    logits = x.double() @ w.double().t()
    index = torch.arange(vocab, device="cuda").expand(tokens, vocab).contiguous()
    loss, dx, dw = torch.empty(tokens, device="cuda"), torch.empty_like(x), torch.empty((vocab, d), device="cuda")
    psgd.HeadDistill(tokens, d, vocab, vocab, psgd.PSGD_F32).loss_grad(x, w, index, logits.float(), loss, dx, dw)
    # a loss of sum q u^2 / 2 with |u| below the error of two logits and of fp32 numbers of their spread
    u = 2 * float(logit_error(x.double().cpu(), w)) + 2.0 ** -22 * (float(logits.max() - logits.min()) * 2 + 20)
    assert (loss >= 0).all() and (loss <= u * u).all()
    assert dx.abs().max() <= 2 * u * w.abs().max() / tokens and dw.abs().max() <= 2 * u * x.abs().max()


def test_gradients_against_differences():
    """<dX, U> and <dW, V> against central differences of the loss that the library itself computes (fp32)."""
    tokens, d, vocab, top, temperature = 48, 40, 300, 12, 1.5
    x, w, index, teacher = inputs(tokens, d, vocab, top, torch.float32, 11, masked=0.0, ragged=0.1)
    plan = psgd.HeadDistill(tokens, d, vocab, top, psgd.PSGD_F32)
    loss, dx, dw = torch.empty(tokens, device="cuda"), torch.empty_like(x), torch.empty((vocab, d), device="cuda")
    plan.loss_grad(x, w, index, teacher, loss, dx, dw, temperature=temperature, weight=torch.ones(tokens, device="cuda"))
    gen = torch.Generator().manual_seed(12)
    step = 2.0 ** -6

    def total(xx, ww):
        out = torch.empty(tokens, device="cuda")
        plan.loss(padded(xx, torch.float32, 8)[0], padded(ww, torch.float32, 8)[0], index, teacher, out, temperature=temperature)
        return float(out.double().sum())

    for _ in range(4):
        u = torch.randn((tokens, d), generator=gen).cuda()
        v = (torch.randn((vocab, d), generator=gen) / math.sqrt(d)).cuda()
        # as for the cross entropy: the third derivative of lse along a line that moves logits by a is below a^3, a loss is good to 2^-19 of its parts
        for along, got, reach in (((u, None), float((dx.double() * u.double()).sum()), u.norm(dim=1).max() * w.norm(dim=1).max()),
                                  ((None, v), float((dw.double() * v.double()).sum()), x.norm(dim=1).max() * v.norm(dim=1).max())):
            a, b = along
            plus = total(x + step * a if a is not None else x, w + step * b if b is not None else w)
            minus = total(x - step * a if a is not None else x, w - step * b if b is not None else w)
            bound = tokens * (step ** 2 * min(float(reach) / temperature, 30.0) ** 3 / 6 + 2.0 ** -19 * 20 / step)
            assert abs((plus - minus) / (2 * step) - got) <= bound
            assert bound < 40 * tokens


@pytest.mark.parametrize("tokens", [200, 700])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_what_is_not_finite_stays_in_its_token(bad, tokens):
    """A teacher's logit that is NaN or infinite makes NaN of its own token's results."""
    d, vocab, top = 72, 300, 8
    x, w, index, teacher = inputs(tokens, d, vocab, top, torch.bfloat16, 13, masked=0.0, ragged=0.0)
    teacher = torch.where(teacher == -math.inf, 0.0, teacher)
    plan = psgd.HeadDistill(tokens, d, vocab, top)
    weight = torch.full((tokens,), 1.0 / tokens, device="cuda")
    got = []
    for i in range(2):
        loss, dx, dw = torch.empty(tokens, device="cuda"), torch.empty_like(x), torch.empty((vocab, d), dtype=torch.bfloat16, device="cuda")
        plan.loss_grad(x, w, index, teacher, loss, dx, dw, weight=weight)
        got.append((loss, dx))
        teacher[5, 3] = bad
    keep = [i for i in range(tokens) if i != 5]
    assert torch.equal(got[0][0][keep], got[1][0][keep]) and torch.equal(got[0][1][keep], got[1][1][keep])
    assert got[1][0][5].isnan() and got[1][1][5].isnan().all()


@pytest.mark.parametrize("tokens,d,dtype", [(200, 136, "bf16"), (200, 131, "bf16"), (700, 136, "bf16"), (90, 67, "f32")])
def test_gradient_in_the_place_of_the_tokens(tokens, d, dtype):
    vocab, top = 1000, 20
    x, w, index, teacher = inputs(tokens, d, vocab, top, DT[dtype], 14)
    plan = psgd.HeadDistill(tokens, d, vocab, top, CODE[dtype], psgd.PSGD_F32)
    results = []
    for in_place in (False, True):
        here = padded(x, DT[dtype], 8)[0]
        loss, dw = torch.empty(tokens, device="cuda"), torch.empty((vocab, (d + 7) // 8 * 8), device="cuda")[:, :d]
        dx = here if in_place else padded(torch.zeros((tokens, d)), DT[dtype], 8)[0]
        plan.workspace.fill_(0xFF)
        plan.loss_grad(here, w, index, teacher, loss, dx, dw)
        results.append((loss, dx, dw))
    assert all(torch.equal(a, b) for a, b in zip(*results))


@pytest.mark.parametrize("tokens", [300, 1300])
def test_in_a_graph_and_on_another_stream(tokens):
    """Replayed with other entries, of which another number counts."""
    d, vocab, top = 136, 900, 30
    x, w, index, teacher = inputs(tokens, d, vocab, top, torch.bfloat16, 15, masked=0.0)
    x = torch.nan_to_num(x)
    plan = psgd.HeadDistill(tokens, d, vocab, top, piece_tokens=512)
    loss, dx, dw = torch.empty(tokens, device="cuda"), torch.empty_like(x), torch.empty((vocab, d), dtype=torch.bfloat16, device="cuda")

    def step(stream=None):
        plan.loss_grad(x, w, index, teacher, loss, dx, dw, stream=stream)

    def results(run):
        for t in (loss, dx, dw):
            t.fill_(0)
        torch.cuda.synchronize()
        run()
        torch.cuda.synchronize()
        return [t.clone() for t in (loss, dx, dw)]

    results(step)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph):
        step()
    for seed, part in ((16, 0.0), (17, 0.5), (18, 2.0), (19, 0.2)):
        _, _, i, t = inputs(tokens, d, vocab, top, torch.bfloat16, seed, masked=part)
        index.copy_(i)
        teacher.copy_(t)
        got = [results(graph.replay), results(step), results(lambda: step(side))]
        assert all(torch.equal(a, b) for other in got[1:] for a, b in zip(got[0], other))


def test_a_large_matrix():
    """W of more than 4 GiB, words at its ends."""
    tokens, d, vocab, top = 6, 16000, 140000, 5
    gen = torch.Generator(device="cuda")
    gen.manual_seed(2)
    w = torch.randn((vocab, d), generator=gen, device="cuda", dtype=torch.bfloat16).mul_(d ** -0.5)
    x = torch.randn((tokens, d), generator=gen, device="cuda").bfloat16()
    index = torch.tensor([[0, vocab - 1, 131072, 70000, 5], [vocab - 1, -1, -1, vocab, -1], [-1] * 5, [139999, 139998, 0, 1, 2], [255, 256, 257, 511, 512], [vocab] * 5], device="cuda")
    teacher = torch.randn((tokens, top), generator=gen, device="cuda")
    loss, dx, dw = torch.empty(tokens, device="cuda"), torch.empty_like(x), torch.empty_like(w)
    psgd.HeadDistill(tokens, d, vocab, top).loss_grad(x, w, index, teacher, loss, dx, dw)
    there = (index >= 0) & (index < vocab)
    logits = torch.cat([x.double() @ part.double().t() for part in w.split(20000)], 1)
    q = torch.softmax(torch.where(there, teacher.double(), -math.inf), 1)
    log_p = logits.gather(1, torch.where(there, index, 0)) - torch.logsumexp(logits, 1, keepdim=True)
    want = torch.where(there, q * (torch.log(q) - log_p), 0.0).sum(1)
    on = [0, 1, 3, 4]
    # fp32 sums of 16000 products of unit variance / sqrt(d): 2^-24 * 1000 steps of a logit's size
    assert (loss[on].double() - want[on]).abs().max() < 1e-4 and float(loss[2]) == 0 and float(loss[5]) == 0
    D = torch.softmax(logits[on], 1)
    D.scatter_add_(1, torch.where(there[on], index[on], 0), torch.where(there[on], -q[on], 0.0))
    D /= 4
    for v in (0, 5, 131072, vocab - 1):
        want = D[:, v] @ x[on].double()
        # D in bf16 (2^-8), four tokens, and the result's rounding
        assert ((dw[v].double() - want).abs() <= 2.0 ** -7 * 1.1 * (D[:, v].abs() @ x[on].double().abs())).all()
