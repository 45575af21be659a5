"""Layer norms and their gradients against the definition in 64 bits."""
import math

import pytest
import torch

from paper_2509_11254_amd import psgd
from test_gpu_act import CODE, DT, UNIT, padded

pytestmark = pytest.mark.gpu

# one column, less than a piece, odd sizes; the borders of one, four and sixteen wavefronts to a row in either type; many rows
SIZES = [(1, 1), (1, 8), (3, 31), (2, 33), (5, 515), (37, 64), (9, 1024), (7, 1025), (6, 2049), (4, 4096), (5, 4097), (3, 8200), (2, 16384), (1030, 40),
         (5000, 136), (4099, 1032), (1100, 64), (1501, 250), (1201, 120)]
# A row's sums are 32 terms on a lane after each other, then 6 + 16 steps over lanes and wavefronts: an error below 64 roundings of the terms' magnitudes
STEPS = 64 * 2.0 ** -24


def values(rows, cols, seed, shift=0.0):
    gen = torch.Generator().manual_seed(seed)
    scale = torch.where(torch.rand(cols, generator=gen) < 0.1, 20.0, 1.0)
    return torch.randn((rows, cols), generator=gen, dtype=torch.float64) * scale + shift


def plain(s, w, b, eps):
    """y, u, r in 64 bits, and a bound of u's error from the sums: the mean's, the variance's, the roundings of s - mean."""
    mean = s.mean(1, keepdim=True)
    var = ((s - mean) ** 2).mean(1, keepdim=True)
    r = 1 / torch.sqrt(var + eps)
    u = (s - mean) * r
    error = STEPS * ((var.sqrt() + 2.0 ** -18 * s.abs().amax(1, keepdim=True)) * r + u.abs())
    return u * w + b, u, mean, r, error


def vector(n, dtype, seed, scale, shift):
    x = torch.randn(n, generator=torch.Generator().manual_seed(seed)) * scale + shift
    return x.to(DT[dtype]).cuda()


def forward(rows, cols, dtype, wtype, *, add, affine="wb", shift=0.0, eps=1e-5, extra=8):
    x = padded(values(rows, cols, 1, shift), DT[dtype], extra)[0]
    o = padded(values(rows, cols, 2), DT[dtype], 2 * extra)[0] if add else None
    w = vector(cols, wtype, 3, 0.3, 1.0) if "w" in affine else None
    b = vector(cols, wtype, 4, 0.3, 0.0) if "b" in affine else None
    nan = torch.full((rows, cols), float("nan"))
    y, y_buf = padded(nan, DT[dtype], 16)
    total, total_buf = padded(nan, DT[dtype], 40) if add else (None, None)
    stats = torch.full((rows, 2), float("nan"), device="cuda")
    psgd.norm(x, w, b, y, stats, eps=eps, add=o, total=total)
    s = x
    if add:
        assert torch.equal(total, (x.float() + o.float()).to(DT[dtype])) and total_buf[:, cols:].isnan().all()
        s = total
    w64, b64 = w.double().cpu() if w is not None else 1.0, b.double().cpu() if b is not None else torch.zeros(cols, dtype=torch.float64)
    want, u, mean, r, error = plain(s.double().cpu(), w64, b64, eps)
    bound = error * torch.as_tensor(w64).abs() + 2.0 ** -23 * ((u * w64).abs() + b64.abs()) + UNIT[dtype] * 1.01 * want.abs()
    assert ((y.double().cpu() - want).abs() <= bound).all()
    assert y_buf[:, cols:].isnan().all()
    assert ((stats[:, 1].double().cpu() - r[:, 0]).abs() <= STEPS * r[:, 0]).all()
    spread = 1 / r[:, 0] + 2.0 ** -18 * s.double().cpu().abs().amax(1)
    assert ((stats[:, 0].double().cpu() - mean[:, 0]).abs() <= STEPS * spread + 2.0 ** -23 * mean[:, 0].abs()).all()
    return s, w, stats


@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("dtype,wtype", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_forward(rows, cols, dtype, wtype, add):
    forward(rows, cols, dtype, wtype, add=add)


@pytest.mark.parametrize("affine", ["", "w", "b"])
def test_without_weight_or_bias(affine):
    forward(20, 200, "f32", "f32", add=False, affine=affine)


@pytest.mark.parametrize("shift", [1e4, -3e5])
def test_rows_far_from_zero(shift):
    """The variance of what is small beside the mean, in fp32."""
    forward(20, 3000, "f32", "f32", add=False, shift=shift)


@pytest.mark.parametrize("cols", [1, 40, 5000])
def test_rows_without_variance(cols):
    """All elements of a row alike: y is the bias."""
    x = torch.linspace(-300, 300, 8)[:, None].expand(8, cols)
    x, _ = padded(x, torch.float32)
    b = vector(cols, "f32", 5, 1.0, 0.0)
    y, _ = padded(torch.zeros(8, cols), torch.float32)
    psgd.norm(x, None, b, y)
    assert ((y - b).abs() <= STEPS * STEPS * 300 * 320 + 2.0 ** -24 * b.abs()).all()


def backward(rows, cols, dtype, wtype, gtype, *, past=False, accumulate=False, affine="wb", which="wb", shift=0.0, place=None):
    s, w, stats = forward(rows, cols, dtype, wtype, add=False, affine=affine, shift=shift)
    dy, _ = padded(values(rows, cols, 6) * 1e-2, DT[dtype], 24)
    beyond, _ = padded(values(rows, cols, 7) * 1e-2, DT[dtype], 32) if past else (None, None)
    dx, dx_buf = padded(torch.full((rows, cols), float("nan")), DT[dtype], 16)
    first = {k: vector(cols, gtype, 8 + i, 1.0, 0.0) if accumulate else torch.full((cols,), float("nan"), dtype=DT[gtype], device="cuda")
             for i, k in enumerate("wb") if k in which}
    before = {k: t.double().cpu() if accumulate else 0.0 for k, t in first.items()}
    s64, dy64 = s.double().cpu(), dy.double().cpu()
    plan = psgd.NormGrad(rows, cols, CODE[dtype], CODE[wtype], CODE[gtype])
    plan.workspace.fill_(0xFF)
    past64 = beyond.double().cpu() if past else 0.0
    if place:
        dx = {"dy": dy, "x": s, "past": beyond}[place]
    plan.run(dy, s, w, stats, dx, first.get("w"), first.get("b"), dtotal=beyond, accumulate=accumulate)
    w64 = w.double().cpu() if w is not None else torch.ones(cols, dtype=torch.float64)
    _, u, mean, r, error = plain(s64, w64, 0.0, 1e-5)
    error = error + r * 2.0 ** -23 * mean.abs()          # (the mean as it is kept)
    g = dy64 * w64
    c1, c2 = g.mean(1, keepdim=True), (g * u).mean(1, keepdim=True)
    want = r * (g - c1 - u * c2) + past64
    bound = r * (STEPS * (g.abs() + g.abs().mean(1, keepdim=True) + 2 * u.abs() * (g * u).abs().mean(1, keepdim=True))
                 + error * c2.abs() + u.abs() * (g.abs() * error).mean(1, keepdim=True)) + 2.0 ** -23 * torch.as_tensor(past64).abs()
    assert ((dx.double().cpu() - want).abs() <= bound + UNIT[dtype] * 1.01 * want.abs()).all()
    if not place:
        assert dx_buf[:, cols:].isnan().all()
    # a column: rows / 1024 after each other, four rows' sums, 64 workgroups' sums after each other, 16 of these
    deep = (rows / 1024 + 90) * 2.0 ** -24
    for k, terms, more in (("w", dy64 * u, dy64.abs() * error), ("b", dy64, torch.zeros_like(dy64))):
        if k in first:
            want = terms.sum(0) + before[k]
            bound = deep * (terms.abs().sum(0) + torch.as_tensor(before[k]).abs()) + more.sum(0) + UNIT[gtype] * 1.01 * want.abs()
            assert ((first[k].double().cpu() - want).abs() <= bound).all(), k


@pytest.mark.parametrize("dtype,wtype,gtype", [("bf16", "bf16", "bf16"), ("bf16", "f32", "f32"), ("f32", "f32", "f32")])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_backward(rows, cols, dtype, wtype, gtype):
    backward(rows, cols, dtype, wtype, gtype, past=cols % 3 == 1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cols", [264, 3001])
@pytest.mark.parametrize("change", [dict(accumulate=True), dict(past=True), dict(affine=""), dict(which="w"), dict(which="b", accumulate=True), dict(which=""),
                                    dict(place="dy"), dict(place="x"), dict(past=True, place="past")])
def test_backward_variants(dtype, cols, change):
    change = dict(change)
    if change.get("place") == "past":
        change["past"] = True
    backward(301, cols, dtype, dtype, "f32", **change)


def test_backward_far_from_zero():
    backward(20, 3000, "f32", "f32", "f32", shift=1e3)


def test_gradients_against_differences():
    """<dx, v>, <dw, v> and <db, v> against central differences of <dy, y> that the library itself computes, in fp32."""
    rows, cols, eps, h = 12, 72, 1e-5, 2.0 ** -7
    gen = torch.Generator().manual_seed(11)
    x, w, b = torch.randn((rows, cols), generator=gen).cuda(), (torch.randn(cols, generator=gen) * 0.3 + 1).cuda(), torch.randn(cols, generator=gen).cuda()
    dy = torch.randn((rows, cols), generator=gen).cuda()
    stats, y, dx = torch.empty((rows, 2), device="cuda"), torch.empty_like(x), torch.empty_like(x)
    dw, db = torch.empty_like(w), torch.empty_like(b)
    psgd.norm(x, w, b, y, stats, eps=eps)
    psgd.NormGrad(rows, cols, psgd.PSGD_F32).run(dy, x, w, stats, dx, dw, db)

    def total(x, w, b):
        out = torch.empty_like(x)
        psgd.norm(x, w, b, out, eps=eps)
        return float((out.double() * dy.double()).sum())

    size = float((dy.abs().double() * 8).sum())
    for i, got in enumerate((dx, dw, db)):
        v = torch.randn(got.shape, generator=gen).cuda()
        plus, minus = [x, w, b], [x, w, b]
        plus[i], minus[i] = plus[i] + h * v, minus[i] - h * v
        # y is linear in w and b; along x its third derivative is below 30 |v| ^ 3 / sd^3 with sd = 1 here, elements up to 4
        curve = 0 if i else h * h * 30 / 6 * float((dy.abs().double() * 4).sum())
        assert abs((total(*plus) - total(*minus)) / (2 * h) - float((got.double() * v.double()).sum())) <= curve + 2.0 ** -20 * size / h


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_what_is_not_finite_stays_in_its_row(bad):
    rows, cols = 9, 300
    x, _ = padded(values(rows, cols, 12), torch.bfloat16)
    y0, y1 = torch.empty((rows, 304), dtype=torch.bfloat16, device="cuda")[:, :cols], torch.empty((rows, 304), dtype=torch.bfloat16, device="cuda")[:, :cols]
    w = vector(cols, "bf16", 3, 0.3, 1.0)
    psgd.norm(x, w, None, y0)
    x[4, 299] = bad
    psgd.norm(x, w, None, y1)
    keep = [i for i in range(rows) if i != 4]
    assert torch.equal(y0[keep], y1[keep]) and y1[4].isnan().all()


def test_in_place():
    """total in the place of x, y in that of add: the residual stream updated where it is."""
    rows, cols = 50, 1000
    x, o = padded(values(rows, cols, 1), torch.bfloat16)[0], padded(values(rows, cols, 2), torch.bfloat16)[0]
    w = vector(cols, "f32", 3, 0.3, 1.0)
    total, y = torch.empty_like(x), torch.empty_like(x)
    psgd.norm(x, w, None, y, add=o, total=total)
    x2, o2 = x.clone(), o.clone()
    psgd.norm(x2, w, None, o2, add=o2, total=x2)
    assert torch.equal(x2, total) and torch.equal(o2, y)


def test_y_in_the_place_of_x():
    for rows, cols, dtype in ((50, 1000, torch.bfloat16), (7, 16384, torch.float32), (999, 64, torch.bfloat16)):
        x = padded(values(rows, cols, 1), dtype)[0]
        y, here = torch.empty_like(x), x.clone()
        psgd.norm(x, None, None, y)
        psgd.norm(here, None, None, here)
        assert torch.equal(here, y)


def test_no_rows():
    e = torch.empty((0, 40), device="cuda")
    w, stats = torch.ones(40, device="cuda"), torch.empty((0, 2), device="cuda")
    psgd.norm(e, w, w, e.clone(), stats)
    dw, db = torch.ones(40, device="cuda"), torch.ones(40, device="cuda")
    plan = psgd.NormGrad(0, 40, psgd.PSGD_F32)
    plan.run(e.clone(), e, w, stats, e.clone(), dw, db, accumulate=True)
    assert (dw == 1).all() and (db == 1).all()
    plan.run(e.clone(), e, w, stats, e.clone(), dw, db)
    assert (dw == 0).all() and (db == 0).all()


def _step(rows, cols, seed):
    x, o = padded(values(rows, cols, seed), torch.bfloat16)[0], padded(values(rows, cols, seed + 1), torch.bfloat16)[0]
    w, b = vector(cols, "f32", 3, 0.3, 1.0), vector(cols, "f32", 4, 0.3, 0.0)
    dy = padded(values(rows, cols, seed + 2) * 1e-2, torch.bfloat16)[0]
    out = [torch.zeros_like(x) for _ in range(3)] + [torch.zeros((rows, 2), device="cuda"), torch.zeros(cols, device="cuda"), torch.zeros(cols, device="cuda")]
    plan = psgd.NormGrad(rows, cols, psgd.PSGD_BF16, psgd.PSGD_F32)

    def step(stream=None):
        psgd.norm(x, w, b, out[0], out[3], add=o, total=out[1], stream=stream)
        plan.run(dy, out[1], w, out[3], out[2], out[4], out[5], dtotal=dy, stream=stream)

    return x, out, step


def test_the_same_every_time_and_on_another_stream():
    _, out, step = _step(3000, 520, 20)
    got = []
    for stream in (None, None, torch.cuda.Stream()):
        for t in out:
            t.fill_(0)
        torch.cuda.synchronize()
        step(stream)
        torch.cuda.synchronize()
        got.append([t.clone() for t in out])
    for other in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(got[0], other))


def test_in_a_graph():
    x, out, step = _step(700, 1032, 30)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (31, 32, 33):
        x.copy_(values(700, 1032, seed))
        graph.replay()
        got = [t.clone() for t in out]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, out))


def test_more_than_4_gib():
    rows, cols = 300000, 8192
    x = torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda")
    some = [0, 131071, 262143, 262144, rows - 1]
    x[some] = torch.randn((len(some), cols), generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    y, stats = torch.full_like(x, 7.0), torch.empty((rows, 2), device="cuda")
    psgd.norm(x, None, None, y, stats)
    want, u, _, r, error = plain(x[some].double().cpu(), 1.0, 0.0, 1e-5)
    assert ((y[some].double().cpu() - want).abs() <= error + UNIT["bf16"] * 1.01 * want.abs()).all()
    assert int((y.view(torch.int16) << 1 != 0).any(1).sum()) == len(some)
    # dy = y where it is in place of it: g = u, c1 = 0, c2 = 1 - eps r^2
    plan, dw = psgd.NormGrad(rows, cols), torch.empty(cols, device="cuda")
    plan.grad_dtype = psgd.PSGD_F32
    dy64 = y[some].double().cpu()
    plan.run(y, x, None, stats, y, dw)
    c1, c2 = dy64.mean(1, keepdim=True), (dy64 * u).mean(1, keepdim=True)
    want = r * (dy64 - c1 - u * c2)
    bound = r * (STEPS * 4 * (dy64.abs() + u.abs() + 1) + error * c2.abs() + u.abs() * (dy64.abs() * error).mean(1, keepdim=True))
    assert ((y[some].double().cpu() - want).abs() <= bound + UNIT["bf16"] * 1.01 * want.abs()).all()
    terms = dy64 * u
    assert ((dw.double().cpu() - terms.sum(0)).abs() <= 400 * 2.0 ** -24 * terms.abs().sum(0) + (dy64.abs() * error).sum(0)).all()
