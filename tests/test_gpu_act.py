"""8-bit checkpoints of activations, the gated units around them and the weight gradients formed from them, against plain
implementations in 64 bits."""
import math

import pytest
import torch

from paper_2509_11254_amd import psgd

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
CODE = {"f32": psgd.PSGD_F32, "bf16": psgd.PSGD_BF16}
# largest relative error of one rounding
UNIT = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
SHAPES = [(1, 1), (1, 31), (3, 32), (2, 33), (5, 515), (37, 47), (4, 4096), (129, 1000), (1000, 16)]


def padded(x, dtype, extra=0):
    """x in a buffer with rows a multiple of 8 elements apart and NaN behind the columns."""
    rows, cols = x.shape
    buf = torch.full((rows, (cols + 7) // 8 * 8 + extra), float("nan"), dtype=dtype, device="cuda")
    buf[:, :cols] = x
    return buf[:, :cols], buf


def activations(rows, cols, seed):
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, cols), generator=gen, dtype=torch.float64)
    return x * torch.where(torch.rand(cols, generator=gen) < 0.1, 20.0, 1.0)


def plain_kept(x):
    """Codes and values of a checkpoint by its definition: the scale is searched for, element by element in 64 bits."""
    x = x.double().cpu()
    rows, cols = x.shape
    codes = torch.zeros((rows, cols), dtype=torch.float64)
    scales = torch.zeros((rows, -(-cols // 32)), dtype=torch.int64)
    for g in range(scales.shape[1]):
        part = x[:, 32 * g:32 * g + 32]
        finite = torch.isfinite(part)
        most = torch.where(finite, part.abs(), 0.0).amax(1)
        e = torch.full((rows,), 121.0, dtype=torch.float64)
        for _ in range(247):            # the smallest exponent that holds the largest element
            e = torch.where((e > -126) & (127.0 * 2.0 ** (e - 1) >= most), e - 1, e)
        q = torch.round(torch.where(finite, part, 0.0) / 2.0 ** e[:, None]).clamp(-127, 127)
        codes[:, 32 * g:32 * g + 32] = torch.where(finite, q, -128.0)
        scales[:, g] = torch.where(most > 0, e + 127, 0.0).long()
    value = torch.where(codes == -128, float("nan"), codes * 2.0 ** (scales.double() - 127).repeat_interleave(32, 1)[:, :cols])
    return codes, scales, torch.where(scales.repeat_interleave(32, 1)[:, :cols] == 0, value * 0.0, value)


def check_kept(kept, x):
    codes, scales, values = plain_kept(x)
    assert torch.equal(kept.codes[:, :kept.cols].cpu().double(), codes)
    assert torch.equal(kept.scales.cpu().long(), scales)
    return values


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("extra", [0, 40])
def test_round_trip(rows, cols, dtype, extra):
    x, _ = padded(activations(rows, cols, 1), DT[dtype], extra)
    kept = psgd.act_empty(rows, cols)
    psgd.act_store(x, kept)
    values = check_kept(kept, x)
    for out in ("f32", "bf16"):                       # the values are numbers of both types
        y, buf = padded(torch.zeros((rows, cols)), DT[out], 8)
        psgd.act_restore(kept, y)
        assert torch.equal(y.double().cpu(), values)
        assert buf[:, cols:].isnan().all()            # the padding is not written


def test_round_trip_of_unusual_values():
    """Zeros, -0, the smallest and largest numbers of fp32, a maximum at the border between two scales, NaN and infinities."""
    top = 3.4028234663852886e38
    rows = [[0.0] * 32, [-0.0] * 31 + [1e-45], [1e-45, -1e-40, 1.2e-38] + [0.0] * 29, [top, -top, 1.0] + [0.5] * 29,
            [127.0] + [0.5, 1.5, 2.5, -0.5, -1.5] + [3.0] * 26, [127.00001] + [1.0] * 31, [float("nan")] * 32,
            [float("inf"), 1.0, -float("inf"), float("nan")] + [2.0] * 28, [float("inf")] + [0.0] * 31, [2.0 ** -126] * 32]
    x, _ = padded(torch.tensor(rows, dtype=torch.float64).float(), torch.float32)
    kept = psgd.act_empty(len(rows), 32)
    psgd.act_store(x, kept)
    values = check_kept(kept, x)
    y, _ = padded(torch.zeros((len(rows), 32)), torch.float32)
    psgd.act_restore(kept, y)
    assert torch.equal(torch.nan_to_num(y.double().cpu(), nan=77.0), torch.nan_to_num(values, nan=77.0))
    assert torch.equal(y.isnan().cpu(), ~torch.isfinite(x.cpu()))


def value(x, act):
    return x * torch.special.ndtr(x) if act == psgd.PSGD_GELU else x * torch.sigmoid(x)


def slope(x, act):
    if act == psgd.PSGD_GELU:
        return torch.special.ndtr(x) + x * torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)
    return torch.sigmoid(x) * (1 + x * torch.sigmoid(-x))


@pytest.mark.parametrize("act", [psgd.PSGD_SILU, psgd.PSGD_GELU])
def test_slopes_of_the_plain_form(act):
    x = torch.linspace(-9, 9, 181, dtype=torch.float64)
    step = 1e-5
    difference = (value(x + step, act) - value(x - step, act)) / (2 * step)
    # the third derivatives are below 2: step^2 / 6 * 2, and 64-bit rounding of values up to 9 over the step
    assert (difference - slope(x, act)).abs().max() < step ** 2 + 9 * 2.0 ** -52 / step


@pytest.mark.parametrize("act", [psgd.PSGD_SILU, psgd.PSGD_GELU])
@pytest.mark.parametrize("gated", [True, False])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_glu(rows, cols, dtype, gated, act):
    gate, _ = padded(activations(rows, cols, 2), DT[dtype], 16)
    up = padded(activations(rows, cols, 3), DT[dtype], 16)[0] if gated else None
    dh, _ = padded(activations(rows, cols, 4), DT[dtype])
    h, h_buf = padded(torch.zeros((rows, cols)), DT[dtype])
    kg, ku = psgd.act_empty(rows, cols), psgd.act_empty(rows, cols) if gated else None
    psgd.act_glu(gate, up, h, kg, ku, act=act)
    g8 = check_kept(kg, gate)
    u8 = check_kept(ku, up) if gated else torch.ones_like(g8)
    # the 32-bit steps before the one rounding: exponentials and error function are good to 2^-21 of 1, products of four factors
    unit, slack = UNIT[dtype], 2.0 ** -19
    g, u, d = gate.double().cpu(), up.double().cpu() if gated else torch.ones((), dtype=torch.float64), dh.double().cpu()
    want = value(g, act) * u
    assert ((h.double().cpu() - want).abs() <= unit * want.abs() + slack * (g * u).abs() + 1e-37).all()
    assert h_buf[:, cols:].isnan().all()
    dgate, dg_buf = padded(torch.zeros((rows, cols)), DT[dtype], 8)
    dup = padded(torch.zeros((rows, cols)), DT[dtype], 8)[0] if gated else None
    psgd.act_glu_backward(kg, ku, dh, dgate, dup, act=act)
    want = d * u8 * slope(g8, act)
    assert ((dgate.double().cpu() - want).abs() <= unit * want.abs() + slack * (d * u8).abs() * (1 + g8.abs()) + 1e-37).all()
    assert dg_buf[:, cols:].isnan().all()
    if gated:
        want = d * value(g8, act)
        assert ((dup.double().cpu() - want).abs() <= unit * want.abs() + slack * (d * g8).abs() + 1e-37).all()


@pytest.mark.parametrize("act", [psgd.PSGD_SILU, psgd.PSGD_GELU])
def test_glu_of_large_values(act):
    """Far from zero the exponential over- and underflows: act is x or 0, its slope 1 or 0, and nothing is NaN."""
    x = torch.tensor([[1e4, -1e4, 300.0, -300.0, 88.8, -88.8, 104.0, -104.0, 0.0, -0.0] + [1e30, -1e30] * 3]).cuda()
    gate, _ = padded(x, torch.float32)
    dh, _ = padded(torch.ones_like(x), torch.float32)
    h, _ = padded(torch.zeros_like(x), torch.float32)
    dgate, _ = padded(torch.zeros_like(x), torch.float32)
    kept = psgd.act_empty(1, 16)
    psgd.act_glu(gate, None, h, kept, None, act=act)
    psgd.act_glu_backward(kept, None, dh, dgate, None, act=act)
    assert torch.allclose(h.cpu(), torch.clamp(x.cpu(), min=0.0), rtol=1e-6, atol=1e-30)
    kept_values, _ = padded(torch.zeros_like(x), torch.float32)
    psgd.act_restore(kept, kept_values)
    assert torch.equal(dgate.cpu(), torch.where(kept_values.cpu() > 0, 1.0, torch.where(kept_values.cpu() < 0, 0.0, 0.5)))


# (tokens, out, in): single tokens, less than a tile, odd sizes, several tiles, contractions that are split
WGRAD = [(1, 1, 1), (1, 300, 70), (7, 33, 515), (63, 256, 256), (64, 257, 255), (65, 8, 1000), (200, 515, 300), (1000, 100, 40), (5000, 130, 270),
         (3000, 64, 1032)]


@pytest.mark.parametrize("dtype,g_dtype", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("tokens,out,inp", WGRAD)
@pytest.mark.parametrize("accumulate", [False, True])
def test_wgrad(tokens, out, inp, dtype, g_dtype, accumulate):
    dy, _ = padded(activations(tokens, out, 5), DT[dtype], 8)
    x, _ = padded(activations(tokens, inp, 6), torch.bfloat16)
    kept = psgd.act_empty(tokens, inp)
    psgd.act_store(x, kept)
    values = plain_kept(x)[2]
    g, g_buf = padded(activations(out, inp, 7) if accumulate else torch.full((out, inp), float("nan")), DT[g_dtype], 8)
    before = g.double().cpu().clone() if accumulate else 0.0
    psgd.WeightGrad(tokens, out, inp, CODE[dtype], CODE[g_dtype]).run(dy, kept, g, accumulate=accumulate)
    d = dy.double().cpu()
    want = before + d.T @ values
    # products are exact (fp32 dY: 24 bits kept); sums in fp32, sixteen terms at a time
    terms = d.abs().T @ values.abs()
    bound = UNIT[g_dtype] * want.abs() + 2.0 ** -24 * (tokens / 16 + 24) * (terms + (before.abs() if accumulate else 0.0))
    assert ((g.double().cpu() - want).abs() <= bound).all()
    assert g_buf[:, inp:].isnan().all()


@pytest.mark.parametrize("accumulate", [False, True])
def test_wgrad_of_no_tokens(accumulate):
    dy, x = torch.empty((0, 24), dtype=torch.bfloat16, device="cuda"), torch.empty((0, 40), dtype=torch.bfloat16, device="cuda")
    kept = psgd.act_empty(0, 40)
    psgd.act_store(x, kept)
    g = torch.ones((24, 40), device="cuda")
    psgd.WeightGrad(0, 24, 40, psgd.PSGD_BF16, psgd.PSGD_F32).run(dy, kept, g, accumulate=accumulate)
    assert torch.equal(g, torch.ones_like(g) if accumulate else torch.zeros_like(g))


def test_wgrad_is_the_same_every_time():
    dy, _ = padded(activations(4000, 300, 8), torch.bfloat16)
    x, _ = padded(activations(4000, 200, 9), torch.bfloat16)
    kept, plan = psgd.act_empty(4000, 200), psgd.WeightGrad(4000, 300, 200, psgd.PSGD_BF16, psgd.PSGD_F32)
    psgd.act_store(x, kept)
    out = []
    for _ in range(3):
        plan.workspace.fill_(0xFF)
        g = torch.empty((300, 200), device="cuda")
        plan.run(dy, kept, g)
        out.append(g)
    assert torch.equal(out[0], out[1]) and torch.equal(out[0], out[2])


def test_calls_on_another_stream():
    x, _ = padded(activations(300, 520, 10), torch.bfloat16)
    dy, _ = padded(activations(300, 128, 11), torch.bfloat16)
    kept, plan = psgd.act_empty(300, 520), psgd.WeightGrad(300, 128, 520)
    g0, g1 = (torch.empty((128, 520), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    psgd.act_store(x, kept)
    plan.run(dy, kept, g0)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    kept.codes.zero_()
    side.wait_stream(torch.cuda.current_stream())
    psgd.act_store(x, kept, stream=side)
    plan.run(dy, kept, g1, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(g0, g1)


def test_calls_in_a_graph():
    rows, cols, out = 200, 264, 96
    gate, _ = padded(activations(rows, cols, 12), torch.bfloat16)
    up, _ = padded(activations(rows, cols, 13), torch.bfloat16)
    dh, _ = padded(activations(rows, cols, 14), torch.bfloat16)
    dy, _ = padded(activations(rows, out, 15), torch.bfloat16)
    h, dgate, dup = (torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda") for _ in range(3))
    kg, ku, kh = (psgd.act_empty(rows, cols) for _ in range(3))
    g = torch.empty((out, cols), device="cuda")
    plan = psgd.WeightGrad(rows, out, cols, psgd.PSGD_BF16, psgd.PSGD_F32)

    def step():
        psgd.act_glu(gate, up, h, kg, ku)
        psgd.act_store(h, kh)
        plan.run(dy, kh, g)
        psgd.act_glu_backward(kg, ku, dh, dgate, dup)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in range(3):
        gate.copy_(activations(rows, cols, 20 + seed))
        graph.replay()
        got = [t.clone() for t in (h, dgate, dup, g)]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (h, dgate, dup, g)))
