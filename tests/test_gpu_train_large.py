"""Operands of more than 4 GiB: offsets beyond 32 bits in rows, tiles and pieces."""
import pytest
import torch

from paper_2509_11254_amd import psgd
from test_gpu_act import plain_kept

pytestmark = pytest.mark.gpu


def test_checkpoint_of_a_large_activation():
    rows, cols = 70000, 32800
    x = torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda")
    gen = torch.Generator().manual_seed(1)
    some = [0, 1, 32767, 65535, 65536, rows - 1]
    for r in some:
        x[r] = torch.randn(cols, generator=gen).bfloat16()
    kept = psgd.act_empty(rows, cols)
    psgd.act_store(x, kept)
    y = torch.full_like(x, 7.0)
    psgd.act_restore(kept, y)
    codes, scales, values = plain_kept(x[some])
    assert torch.equal(kept.codes[some][:, :cols].cpu().double(), codes) and torch.equal(kept.scales[some].cpu().long(), scales)
    assert torch.equal(y[some].double().cpu(), values)
    y[some] = 0
    assert int((y != 0).sum()) == 0


def test_weight_gradient_of_many_tokens():
    """All but a few of dY's rows are zero: the weight gradient is theirs alone."""
    tokens, out, inp = 300000, 8192, 40
    dy = torch.zeros((tokens, out), dtype=torch.bfloat16, device="cuda")
    x = torch.randn((tokens, inp), device="cuda").bfloat16()
    kept = psgd.act_empty(tokens, inp)
    psgd.act_store(x, kept)
    some = [0, 63, 131071, 262144, 262145, tokens - 2, tokens - 1]
    dy[some] = torch.randn((len(some), out), device="cuda").bfloat16()
    g = torch.empty((out, inp), device="cuda")
    psgd.WeightGrad(tokens, out, inp, psgd.PSGD_BF16, psgd.PSGD_F32).run(dy, kept, g)
    values = plain_kept(x[some])[2]
    d = dy[some].double().cpu()
    assert ((g.double().cpu() - d.T @ values).abs() <= 2.0 ** -22 * (d.abs().T @ values.abs()) + 1e-30).all()


def test_head_with_a_large_matrix():
    tokens, d, vocab = 6, 16000, 140000
    gen = torch.Generator(device="cuda")
    gen.manual_seed(2)
    w = torch.randn((vocab, d), generator=gen, device="cuda", dtype=torch.bfloat16).mul_(d ** -0.5)
    x = torch.randn((tokens, d), generator=gen, device="cuda").bfloat16()
    labels = torch.tensor([0, vocab - 1, -100, 131072, 70000, vocab], device="cuda")
    loss, dx, dw = torch.empty(tokens, device="cuda"), torch.empty_like(x), torch.empty_like(w)
    psgd.HeadLoss(tokens, d, vocab).loss_grad(x, w, labels, loss, dx, dw)
    on = [0, 1, 3, 4]
    x64 = x[on].double()
    logits = torch.cat([x64 @ part.double().t() for part in w.split(20000)], 1)
    lse = torch.logsumexp(logits, 1)
    want = lse - logits[torch.arange(4), labels[on]]
    # fp32 sums of 16000 products of unit variance / sqrt(d): 2^-24 * 1000 steps of a logit's size
    assert (loss[on].double() - want).abs().max() < 1e-4 and float(loss[2]) == 0 and float(loss[5]) == 0
    p = torch.exp(logits - lse[:, None])
    p[torch.arange(4), labels[on]] -= 1
    p /= 4
    rows = [0, 1, 70000, 131071, 131072, vocab - 2, vocab - 1]
    dw64 = p[:, rows].t() @ x64
    # D and dW rounded to bf16 once each
    assert ((dw[rows].double() - dw64).abs() <= 2.0 ** -7 * (p[:, rows].abs().t() @ x64.abs()) + 1e-12).all()
    dx64 = sum(p[:, 20000 * i:20000 * i + part.shape[0]] @ part.double() for i, part in enumerate(w.split(20000)))
    size = sum(p[:, 20000 * i:20000 * i + part.shape[0]].abs() @ part.double().abs() for i, part in enumerate(w.split(20000)))
    assert ((dx[on].double() - dx64).abs() <= 2.0 ** -7 * size).all() and (dx[[2, 5]] == 0).all()


def test_a_piece_of_many_tokens():
    """Exponentials of one piece of more than 2 GiB; most tokens are alike."""
    tokens, d, vocab = 18000, 64, 64000
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    w = torch.randn((vocab, d), generator=gen, device="cuda").mul_(0.125).bfloat16()
    x = torch.randn((tokens, d), generator=gen, device="cuda").bfloat16()
    labels = torch.randint(0, vocab, (tokens,), generator=gen, device="cuda")
    one, two = (psgd.HeadLoss(tokens, d, vocab, psgd.PSGD_BF16, psgd.PSGD_F32, piece_tokens=p) for p in (tokens, 4000))
    got = []
    for plan in (one, two):
        loss, dx, dw = torch.empty(tokens, device="cuda"), torch.empty_like(x), torch.empty((vocab, d), device="cuda")
        plan.loss_grad(x, w, labels, loss, dx, dw)
        got.append((loss, dx, dw))
    logits = x[-50:].double() @ w.double().t()
    want = torch.logsumexp(logits, 1) - logits[torch.arange(50), labels[-50:]]
    assert (got[0][0][-50:].double() - want).abs().max() < 1e-4
    assert torch.equal(got[0][0], got[1][0])        # a token's loss does not depend on the piece it is in
    assert (got[0][1].float() - got[1][1].float()).norm() <= 2.0 ** -8 * got[0][1].float().norm()
    assert (got[0][2] - got[1][2]).norm() <= 2.0 ** -16 * got[0][2].norm()


def test_head_with_a_large_fp32_matrix():
    tokens, d, vocab = 5, 8200, 140000
    gen = torch.Generator(device="cuda")
    gen.manual_seed(4)
    w = torch.randn((vocab, d), generator=gen, device="cuda").mul_(d ** -0.5)
    x = torch.randn((tokens, d), generator=gen, device="cuda")
    labels = torch.tensor([vocab - 1, -1, 131000, 0, 70000], device="cuda")
    loss, dx, dw = torch.empty(tokens, device="cuda"), torch.empty_like(x), torch.empty_like(w)
    psgd.HeadLoss(tokens, d, vocab, psgd.PSGD_F32, psgd.PSGD_F32).loss_grad(x, w, labels, loss, dx, dw)
    on = [0, 2, 3, 4]
    x64 = x[on].double()
    logits = torch.cat([x64 @ part.double().t() for part in w.split(20000)], 1)
    lse = torch.logsumexp(logits, 1)
    want = lse - logits[torch.arange(4), labels[on]]
    # fp32 sums of 8200 products, sixteen at a time
    assert (loss[on].double() - want).abs().max() < 1e-4 and float(loss[1]) == 0
    p = torch.exp(logits - lse[:, None])
    p[torch.arange(4), labels[on]] -= 1
    p /= 4
    rows = [0, 1, 70000, 130899, 131000, vocab - 2, vocab - 1]
    dw64 = p[:, rows].t() @ x64
    # the exponentials' error is the logits': 8200 / 16 steps of 2^-24 of a sum of unit variance
    assert ((dw[rows].double() - dw64).abs() <= 2.0 ** -12 * (p[:, rows].abs().t() @ x64.abs()) + 1e-12).all()
    dx64 = sum(p[:, 20000 * i:20000 * i + part.shape[0]] @ part.double() for i, part in enumerate(w.split(20000)))
    size = sum(p[:, 20000 * i:20000 * i + part.shape[0]].abs() @ part.double().abs() for i, part in enumerate(w.split(20000)))
    assert ((dx[on].double() - dx64).abs() <= 2.0 ** -12 * size).all() and (dx[1] == 0).all()
