"""Distillation on every tile that the head's logits are made by, and with as many entries as each of the lists' kernels takes, against the definition in
64 bits.  Each test looks up that the library takes the tile that it is about."""
import ctypes as C
import math

import pytest
import torch

from paper_2509_11254_amd import psgd
from test_gpu_act import CODE, DT, UNIT, padded
from test_gpu_tiles import MANY, T128, T256, THIN, TilePlan, chunks, tile_plan

pytestmark = pytest.mark.gpu
SPLIT, SPLIT_THIN = 4, 5


def logits_tile(tokens, d, vocab, dtype):
    if dtype == "bf16":
        return tile_plan(vocab, tokens, chunks(-(-d // 8) * 8), False)[0]
    fn = psgd.load_library()["_ZN4psgd10split_planElllb"]
    fn.restype, fn.argtypes = TilePlan, [C.c_int64, C.c_int64, C.c_int64, C.c_bool]
    return fn(vocab, tokens, -(-d // 32), False).shape


def inputs(tokens, d, vocab, top, dtype, seed, masked=0.2, ragged=0.2, twice=False):
    """Frequent words are low, so that a tile has many of them; each token knows one of its words well.  What does not count holds NaN."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def rand(*shape):
        return torch.rand(shape, generator=gen, device="cuda")

    def randn(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    w = randn(vocab, d) / math.sqrt(d)
    if twice:
        index = (vocab * rand(tokens, top) ** 3).long().clamp(max=vocab - 1)
    else:
        index = (rand(tokens, vocab) * torch.linspace(0.1, 1.0, vocab, device="cuda")).topk(top, 1, largest=False).indices
        index = index.gather(1, rand(tokens, top).argsort(1))
    teacher = 3 * randn(tokens, top) + 10
    x = randn(tokens, d) + 12 * rand(tokens, 1) * w[index[:, 0]]
    gone = rand(tokens, top) < ragged
    index = torch.where(gone, torch.where(rand(tokens, top) < 0.5, -100, vocab), index)
    teacher = torch.where(gone, float("nan"), torch.where(rand(tokens, top) < 0.05, -math.inf, teacher))
    index[rand(tokens) < masked] = -1
    counts = ((index >= 0) & (index < vocab) & (teacher != -math.inf)).any(1)
    x[~counts] = float("nan")
    return padded(x, DT[dtype], 8)[0], padded(w, DT[dtype], 16)[0], index, teacher


def check(x, w, index, teacher, temperature, weight, loss, dx, dw):
    dtype, g_dtype = ("bf16" if t.dtype == torch.bfloat16 else "f32" for t in (x, dw))
    vocab, d, tokens, top = w.shape[0], x.shape[1], x.shape[0], index.shape[1]
    there = (index >= 0) & (index < vocab) & (teacher != -math.inf)
    counted = there.any(1)
    x64, w64 = torch.where(counted[:, None], x.double(), 0.0), w.double()
    z = torch.where(there, teacher.double() / temperature, -math.inf)
    z[~counted] = 0.0
    q = torch.zeros((tokens, vocab), dtype=torch.float64, device="cuda")
    q.scatter_add_(1, torch.where(there, index, 0), torch.where(there, torch.softmax(z, 1), 0.0))
    logits = x64 @ w64.t() / temperature
    log_p = logits - torch.logsumexp(logits, 1, keepdim=True)
    # a logit: products (exact in bf16, 24 bits in fp32) summed in fp32, sixteen at a time
    err = (d / 16 + 32) * 2.0 ** -24 * x64.norm(dim=1).max() * w64.norm(dim=1).max() / temperature
    low = torch.where(there, z, z.amax(1, keepdim=True).clamp(min=-1e30))
    spread = (logits.amax(1) - logits.amin(1)).max() + (low.amax(1) - low.amin(1)).max() + math.log(vocab) + math.log(top) + 1
    # u = log p - log q: two logits' errors, and roundings of numbers of the size of their spread
    du = 2 * err + 2.0 ** -22 * spread
    want = torch.where(counted, (torch.special.xlogy(q, q) - q * log_p).sum(1), 0.0)
    size = torch.where(q > 0, q * (torch.log(torch.where(q > 0, q, 1.0)) - log_p).abs(), 0.0).sum(1)
    # (the loss moves by p - q times u's errors, and by its terms' roundings)
    assert ((loss.double() - want).abs() <= 2 * du + 2.0 ** -20 * (2 + size)).all(), "loss"
    assert (loss[~counted] == 0).all() and (dx[~counted] == 0).all()
    c = weight.double() if weight is not None else torch.full((tokens,), 1.0 / max(1, int(counted.sum())), dtype=torch.float64, device="cuda")
    c = (torch.where(counted, c, 0.0) / temperature)[:, None]
    p = log_p.exp()
    D = c * (p - q)
    # An element of D: u's error in p and q, a few roundings; where the results are bf16 the others' p in 11 bits, and absolute 2^-25 of
    # 2^15, in which fp16 is below its normal numbers, with a factor of two for what c is relative to.  D in one, two or three planes of 8 bits.
    half = dtype == "bf16" and g_dtype == "bf16"
    off = c * (p + q) * 2 * (du + 2.0 ** -20) + (c * p * 2.0 ** -11 if half else 0.0)
    tiny = 2.0 ** -38 * (2 * c.max() + 1e-30) if half else 0.0
    for name, got, other, planes, length, out in (
            ("dx", dx, w64, 1 if dtype == "bf16" else 3, vocab, dtype),
            ("dw", dw, x64, 3 if g_dtype == "f32" else 1 if dtype == "bf16" else 2, tokens, g_dtype)):
        side = (lambda m: m) if name == "dx" else (lambda m: m.t())
        want = side(D) @ other
        bound = (side(off) + side(D.abs()) * (1.01 * 2.0 ** (-8 * planes) + (length / 16 + 32) * 2.0 ** -24)) @ other.abs()
        bound += tiny * other.abs().sum(0, keepdim=True) + 1.01 * UNIT[out] * want.abs()
        assert ((got.double() - want).abs() <= bound).all(), name


def run(tokens, d, vocab, top, dtype, g_dtype, *, seed=1, temperature=1.0, weighted=False, piece=0, **how):
    x, w, index, teacher = inputs(tokens, d, vocab, top, dtype, seed, **how)
    weight = torch.rand(tokens, generator=torch.Generator().manual_seed(seed)).cuda() if weighted else None
    plan = psgd.HeadDistill(tokens, d, vocab, top, CODE[dtype], CODE[g_dtype], piece_tokens=piece)
    results = []
    for _ in range(2):
        loss, dx, dw = torch.full((tokens,), float("nan"), device="cuda"), padded(torch.full((tokens, d), float("nan")), DT[dtype], 8)[0], \
            padded(torch.full((vocab, d), float("nan")), DT[g_dtype], 16)[0]
        plan.workspace.fill_(0xFF)
        plan.loss_grad(x, w, index, teacher, loss, dx, dw, temperature=temperature, weight=weight)
        results.append((loss, dx, dw))
    check(x, w, index, teacher, temperature, weight, *results[0])
    assert all(torch.equal(a, b) for a, b in zip(*results)), "not the same again"
    alone = torch.full((tokens,), float("nan"), device="cuda")
    plan.workspace.fill_(0xFF)
    plan.loss(x, w, index, teacher, alone, temperature=temperature)
    assert torch.equal(alone, results[0][0])


# tile, tokens, d, vocab
TILES = {"256": (T256, 1100, 1032, 12011, "bf16"), "128": (T128, 777, 520, 4099, "bf16"), "many": (MANY, 1100, 264, 9001, "bf16"), "thin": (THIN, 150, 264, 2003, "bf16"),
         "split": (SPLIT, 700, 131, 12011, "f32"), "split_thin": (SPLIT_THIN, 333, 131, 5003, "f32")}


@pytest.mark.parametrize("top", [1, 20, 64, 65, 128, 200, 400, 1024])
@pytest.mark.parametrize("tile", TILES)
def test_each_number_of_entries(tile, top):
    shape, tokens, d, vocab, dtype = TILES[tile]
    assert logits_tile(tokens, d, vocab, dtype) == shape
    run(tokens, d, vocab, top, dtype, dtype)


@pytest.mark.parametrize("how", [dict(weighted=True, temperature=2.0), dict(twice=True), dict(masked=0.0, ragged=0.0), dict(masked=0.95), dict(ragged=0.97)])
@pytest.mark.parametrize("top", [30, 300])
@pytest.mark.parametrize("g_dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tile", TILES)
def test_variants(tile, g_dtype, top, how):
    shape, tokens, d, vocab, dtype = TILES[tile]
    run(tokens, d, vocab, top, dtype, g_dtype, seed=2, **how)


@pytest.mark.parametrize("tokens,d,vocab,shape", [(700, 1032, 20000, T256), (1601, 1032, 9001, T256), (200, 1024, 10007, T128)])
@pytest.mark.parametrize("g_dtype", ["bf16", "f32"])
def test_other_sizes(tokens, d, vocab, shape, g_dtype):
    assert logits_tile(tokens, d, vocab, "bf16") == shape
    run(tokens, d, vocab, 100, "bf16", g_dtype, seed=3, masked=0.3, weighted=True)


def test_pieces_on_the_largest_tile():
    """Two pieces, each with tokens that do not count."""
    assert logits_tile(1100, 1032, 12011, "bf16") == T256
    run(2200, 1032, 12011, 50, "bf16", "f32", seed=4, piece=1100)
