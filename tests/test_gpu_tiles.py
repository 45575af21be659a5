"""The large tiles of the matrix products -- 256 x 256 and the ringed 128 x 128 -- at borders that are no multiple of them, in parts of the contraction,
with several planes: logits, both gradients of the head and weight gradients against 64 bits.  The sizes are the smallest that the
library takes these tiles for, and each test looks up that it does."""
import ctypes as C
import math

import pytest
import torch

from paper_2509_11254_amd import psgd
from test_gpu_act import CODE, DT, UNIT, padded

pytestmark = pytest.mark.gpu
T256, T128, THIN, MANY = range(4)


class TilePlan(C.Structure):
    _fields_ = [("shape", C.c_int), ("n_split", C.c_int), ("from_codes", C.c_bool), ("us", C.c_double)]


def tile_plan(extent_p, extent_l, chunks, may_split, restore=0.0):
    """psgd::tile_plan: the tile and the parts of the contraction of a product of bf16 operands."""
    fn = psgd.load_library()["_ZN4psgd9tile_planElllbdb"]
    fn.restype, fn.argtypes = TilePlan, [C.c_int64, C.c_int64, C.c_int64, C.c_bool, C.c_double, C.c_bool]
    p = fn(extent_p, extent_l, chunks, may_split, restore, False)
    return p.shape, p.n_split


def chunks(steps):
    return -(-steps // 64)


# tokens, d, vocab, type of dW; tile and parts of the logits, dX and dW.  dW in fp32 has three planes of D one after the other.
HEADS = [(1100, 1032, 12011, "f32", (T256, 1), (MANY, 6), (T256, 1)), (1100, 1032, 12011, "bf16", (T256, 1), (MANY, 6), (T256, 1)),
         (1100, 2051, 12011, "bf16", (T256, 1), (T256, 5), (MANY, 1)), (1537, 2056, 9001, "bf16", (T256, 1), (T256, 4), (MANY, 1)),
         (1100, 1032, 4099, "f32", (MANY, 1), (T128, 3), (T256, 3)), (2050, 515, 4099, "f32", (MANY, 1), (T128, 3), (T256, 5)),
         (777, 520, 4099, "bf16", (T128, 1), (T128, 7), (T128, 1)), (777, 520, 4099, "f32", (T128, 1), (T128, 7), (T128, 1)),
         (777, 1032, 1000, "f32", (THIN, 1), (THIN, 1), (T128, 3))]


def peaked(tokens, d, vocab, seed):
    """Tokens that give each of eight words about a tenth of the probability: D has large elements everywhere, so that no part of a
    contraction can be missing unseen.  A fifth of the tokens does not count and holds NaN."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    w = torch.randn((vocab, d), generator=gen, device="cuda").div_(math.sqrt(d))
    near = torch.randint(0, vocab, (tokens, 8), generator=gen, device="cuda")
    x = 11.0 * sum(w[near[:, i]] for i in range(8))
    labels = torch.randint(0, vocab, (tokens,), generator=gen, device="cuda")
    out = torch.rand(tokens, generator=gen, device="cuda") < 0.2
    x[out] = float("nan")
    labels[out] = -100
    weight = torch.rand(tokens, generator=gen, device="cuda")
    return padded(x, torch.bfloat16, 8)[0], padded(w, torch.bfloat16, 16)[0], labels, weight


@pytest.mark.parametrize("tokens,d,vocab,g_dtype,logits,dx_tile,dw_tile", HEADS)
def test_head(tokens, d, vocab, g_dtype, logits, dx_tile, dw_tile):
    planes = 3 if g_dtype == "f32" else 1
    assert tile_plan(vocab, tokens, chunks(-(-d // 8) * 8), False) == logits
    assert tile_plan(d, tokens, chunks(vocab), True) == dx_tile
    assert tile_plan(d, vocab, chunks(tokens) * planes, True) == dw_tile
    x, w, labels, weight = peaked(tokens, d, vocab, 1)
    loss = torch.full((tokens,), float("nan"), device="cuda")
    dx, dx_buf = padded(torch.full((tokens, d), float("nan")), torch.bfloat16, 8)
    dw, dw_buf = padded(torch.full((vocab, d), float("nan")), DT[g_dtype], 16)
    plan = psgd.HeadLoss(tokens, d, vocab, psgd.PSGD_BF16, CODE[g_dtype])
    plan.workspace.fill_(0xFF)
    plan.loss_grad(x, w, labels, loss, dx, dw, weight=weight)
    alone = torch.full((tokens,), float("nan"), device="cuda")
    plan.workspace.fill_(0xFF)
    plan.loss(x, w, labels, alone)
    assert torch.equal(alone, loss)

    counted = labels >= 0
    x64 = torch.where(counted[:, None], x.double(), 0.0)
    w64, at = w.double(), labels.clamp(min=0)[:, None]
    l64 = x64 @ w64.t()
    lse = torch.logsumexp(l64, 1, keepdim=True)
    # a logit: exact products, summed in fp32, sixteen at a time
    err = (d / 16 + 32) * 2.0 ** -24 * x64.norm(dim=1) * w64.norm(dim=1).max()
    want = torch.where(counted, (lse - l64.gather(1, at))[:, 0], 0.0)
    assert ((loss.double() - want).abs() <= 2 * err + 2.0 ** -21 * (1 + want.abs())).all() and (loss[~counted] == 0).all()
    c = torch.where(counted, weight.double(), 0.0)[:, None]
    D = torch.exp_(l64 - lse).scatter_add_(1, at, -torch.ones_like(lse)).mul_(c)
    size = D.abs()
    # an element of D: the errors of its logit and of the others in the sum, exponentials, the few factors; kept in 11 bits for results in bf16
    exact = 2 * (2 * err[:, None] + 2.0 ** -20) + (2.0 ** -11 if planes == 1 else 0.0)
    below = 2.0 ** -39 * c if planes == 1 else 0.0 * c          # fp16 below its normal numbers
    for got, wanted, terms, wide, n_planes, length, out in (
            (dx, D @ w64, (size * (exact + 2.0 ** -8)) @ w64.abs(), size @ w64.abs(), 1, vocab, "bf16"),
            (dw, D.t() @ x64, (size * (exact + 2.0 ** (-8 * planes))).t() @ x64.abs(), size.t() @ x64.abs(), planes, tokens, g_dtype)):
        few = below * w64.abs().sum(0) if got is dx else (below * x64.abs()).sum(0, keepdim=True)
        bound = terms + (length / 16 + 32) * 2.0 ** -24 * wide + few + 1.01 * UNIT[out] * wanted.abs()
        assert ((got.double() - wanted).abs() <= bound).all(), "dx" if got is dx else "dw"
    assert (dx[~counted] == 0).all() and dx_buf[:, d:].isnan().all() and dw_buf[:, d:].isnan().all()


# tokens, out, in, type of dY (fp32: three planes one after the other); tile and parts
GRADIENTS = [(1001, 4093, 4001, "bf16", (T256, 1)), (700, 4093, 4001, "f32", (T256, 1)), (4001, 1999, 2041, "f32", (T256, 4)),
             (3001, 999, 2051, "f32", (T256, 7)), (4001, 1999, 2041, "bf16", (T128, 1)), (3001, 1999, 2041, "f32", (T128, 1)),
             (1500, 515, 1031, "f32", (T128, 5))]


@pytest.mark.parametrize("g_dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,out,inp,dtype,tile", GRADIENTS)
def test_weight_gradient(tokens, out, inp, dtype, tile, g_dtype):
    assert tile_plan(inp, out, chunks(tokens) * (3 if dtype == "f32" else 1), True, 3 + tokens * inp * 3e-6 / 5) == tile
    gen = torch.Generator(device="cuda")
    gen.manual_seed(2)
    dy, _ = padded(torch.randn((tokens, out), generator=gen, device="cuda"), DT[dtype], 8)
    x, _ = padded(torch.randn((tokens, inp), generator=gen, device="cuda"), torch.bfloat16)
    kept = psgd.act_empty(tokens, inp)
    psgd.act_store(x, kept)
    values, _ = padded(torch.zeros((tokens, inp)), torch.float32)
    psgd.act_restore(kept, values)
    g, g_buf = padded(torch.full((out, inp), float("nan")), DT[g_dtype], 8)
    plan = psgd.WeightGrad(tokens, out, inp, CODE[dtype], CODE[g_dtype])
    plan.workspace.fill_(0xFF)
    plan.run(dy, kept, g)
    d64, v64 = dy.double(), values.double()
    want = d64.t() @ v64
    # products are exact (fp32 dY: 24 bits kept); sums in fp32, sixteen terms at a time
    bound = UNIT[g_dtype] * want.abs() + 2.0 ** -24 * (tokens / 16 + 24) * (d64.abs().t() @ v64.abs())
    assert ((g.double() - want).abs() <= bound).all()
    assert g_buf[:, inp:].isnan().all()


@pytest.mark.parametrize("tokens,counted", [(1, [0]), (700, [3]), (700, [0, 650])])
def test_planes_of_gradients_in_fp32(tokens, counted):
    """dW in fp32 from bf16 activations, of few tokens that count: each element is one or two products, so that what is left out of D shows.  Three
    planes leave out 2^-24; with two it would be 2^-16."""
    d, vocab = 16, 3001
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    w = (0.005 * torch.randn((vocab, d), generator=gen, device="cuda")).bfloat16()
    x = torch.randn((tokens, d), generator=gen, device="cuda").bfloat16()
    labels = torch.full((tokens,), -1, device="cuda")
    labels[counted] = torch.randint(0, vocab, (len(counted),), generator=gen, device="cuda")
    loss, dx, dw = torch.empty(tokens, device="cuda"), torch.empty_like(x), torch.empty((vocab, d), device="cuda")
    psgd.HeadLoss(tokens, d, vocab, psgd.PSGD_BF16, psgd.PSGD_F32).loss_grad(x, w, labels, loss, dx, dw)
    x64, w64 = x[counted].double(), w.double()
    l64 = x64 @ w64.t()
    D = torch.softmax(l64, 1)
    D[torch.arange(len(counted)), labels[counted]] -= 1
    D /= len(counted)
    err = 33 * 2.0 ** -24 * x64.norm(dim=1, keepdim=True) * w64.norm(dim=1).max()
    bound = (D.abs() * (2 * (2 * err + 2.0 ** -20) + 2.0 ** -22)).t() @ x64.abs()
    assert float((2 * (2 * err + 2.0 ** -20) + 2.0 ** -22).max()) < 2.0 ** -17
    assert ((dw.double() - D.t() @ x64).abs() <= bound).all()
