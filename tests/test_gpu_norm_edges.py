"""Layer norms and their gradients at the edges of what a row may hold, against the definition in 64 bits."""
import pytest
import torch

from paper_2509_11254_amd import psgd
from test_gpu_act import CODE, DT, UNIT, padded

pytestmark = pytest.mark.gpu

# A row's sums are 32 terms on a lane after each other, then 6 + 16 steps over lanes and wavefronts: an error below 64 roundings of the terms' magnitudes
STEPS = 64 * 2.0 ** -24


def random(rows, cols, seed, shift=0.0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    scale = torch.where(torch.rand(cols, generator=gen, device="cuda") < 0.1, 20.0, 1.0)
    return torch.randn((rows, cols), generator=gen, device="cuda") * scale + shift


def backward(rows, cols, dtype, *, shift=0.0, past=False, accumulate=False, place=None, affine=True, add=False, seed=1, eps=1e-5):
    """One forward and backward pass with sums in fp32; everything that comes out against 64 bits."""
    x, x_buf = padded(random(rows, cols, seed, shift), DT[dtype], 8)
    o = padded(random(rows, cols, seed + 1), DT[dtype], 16)[0] if add else None
    w = (random(1, cols, seed + 2)[0] * 0.1 + 1).to(DT[dtype]) if affine else None
    b = random(1, cols, seed + 3)[0].to(DT[dtype]) if affine else None
    y, y_buf = padded(torch.full((rows, cols), float("nan")), DT[dtype], 16)
    total, total_buf = padded(torch.full((rows, cols), float("nan")), DT[dtype], 24) if add else (None, None)
    stats = torch.full((rows, 2), float("nan"), device="cuda")
    psgd.norm(x, w, b, y, stats, eps=eps, add=o, total=total)
    s = x
    if add:
        assert torch.equal(total, (x.float() + o.float()).to(DT[dtype])) and total_buf[:, cols:].isnan().all()
        s = total
    dy, _ = padded(random(rows, cols, seed + 4) * 1e-2, DT[dtype], 24)
    beyond = padded(random(rows, cols, seed + 5) * 1e-2, DT[dtype], 32)[0] if past else None
    dx, dx_buf = padded(torch.full((rows, cols), float("nan")), DT[dtype], 16)
    sums = [random(1, cols, seed + 6 + i)[0] if accumulate else torch.full((cols,), float("nan"), device="cuda") for i in range(2)]
    before = [t.double() if accumulate else torch.zeros_like(t, dtype=torch.float64) for t in sums]

    s64, dy64, past64 = s.double(), dy.double(), beyond.double() if past else torch.zeros((), dtype=torch.float64, device="cuda")
    w64 = w.double() if affine else torch.ones(cols, dtype=torch.float64, device="cuda")
    b64 = b.double() if affine else torch.zeros(cols, dtype=torch.float64, device="cuda")
    mean = s64.mean(1, keepdim=True)
    var = ((s64 - mean) ** 2).mean(1, keepdim=True)
    r = 1 / torch.sqrt(var + eps)
    u = (s64 - mean) * r
    # u: what the sums of (s - first mean) lose, whose first mean is a rounding of the row's size away; r; a few roundings of u itself
    error = STEPS * ((var.sqrt() + 2.0 ** -18 * s64.abs().amax(1, keepdim=True)) * r + u.abs())
    want = u * w64 + b64
    assert ((y.double() - want).abs() <= error * w64.abs() + 2.0 ** -23 * ((u * w64).abs() + b64.abs()) + UNIT[dtype] * 1.01 * want.abs()).all()
    assert y_buf[:, cols:].isnan().all()
    del want

    if place:
        dx = {"dy": dy, "x": s, "past": beyond}[place]
    plan = psgd.NormGrad(rows, cols, CODE[dtype], grad_dtype=psgd.PSGD_F32)
    plan.workspace.fill_(0xFF)
    plan.run(dy, s, w, stats, dx, sums[0], sums[1], dtotal=beyond, accumulate=accumulate)
    g = dy64 * w64
    c1, c2 = g.mean(1, keepdim=True), (g * u).mean(1, keepdim=True)
    want = r * (g - c1 - u * c2) + past64
    bound = r * (STEPS * (g.abs() + g.abs().mean(1, keepdim=True) + 2 * u.abs() * (g * u).abs().mean(1, keepdim=True))
                 + error * c2.abs() + u.abs() * (g.abs() * error).mean(1, keepdim=True)) + 2.0 ** -23 * past64.abs()
    assert ((dx.double() - want).abs() <= bound + UNIT[dtype] * 1.01 * want.abs()).all(), "dx"
    if not place:
        assert dx_buf[:, cols:].isnan().all()
    del want, bound, g
    # A column of many rows: those of a workgroup after each other (256 workgroups at least), 3 steps over lanes and 4 over wavefronts, up to 32 workgroups'
    # sums after each other and 16 of these.  Of few: 16 after each other, 4 steps and 16.
    deep = (rows / 256 + 60) * 2.0 ** -24
    for got, terms, more, first in ((sums[0], dy64 * u, dy64.abs() * error, before[0]), (sums[1], dy64, None, before[1])):
        want = terms.sum(0) + first
        bound = deep * (terms.abs().sum(0) + first.abs()) + (more.sum(0) if more is not None else 0.0) + 2.0 ** -24 * 1.01 * want.abs()
        assert ((got.double() - want).abs() <= bound).all(), "dweight" if more is not None else "dbias"


# (rows, cols): sums of columns beside the rows; after them, of eight, sixteen and 32 lanes to a row, one, eight and sixteen wavefronts
FAR = [(1, 3000), (20, 3000), (700, 129), (1500, 20), (1200, 60), (1300, 100), (1100, 300), (1100, 1000), (1100, 2500), (1030, 8200), (300, 16000)]


@pytest.mark.parametrize("shift", [1e4, -3e5])
@pytest.mark.parametrize("rows,cols", FAR)
def test_far_from_zero(rows, cols, shift):
    """A mean that is kept in 32 bits is off by more than what lies around it is exact to."""
    backward(rows, cols, "f32", shift=shift, past=cols % 3 == 1)


@pytest.mark.parametrize("rows,cols", [(50, 3000), (1100, 60), (1100, 5000), (1030, 16000)])
def test_far_from_zero_in_bf16(rows, cols):
    backward(rows, cols, "bf16", shift=1e4)


@pytest.mark.parametrize("rows,cols", [(500, 120), (1500, 20), (1100, 100), (1100, 2500)])
def test_some_rows_far_from_zero(rows, cols):
    shift = torch.zeros((rows, 1), device="cuda")
    shift[torch.arange(rows) * 7 % 3 == 0] = 2e5
    backward(rows, cols, "f32", shift=shift, past=True, accumulate=True)


@pytest.mark.parametrize("rows,cols", [(40, 515), (1500, 20), (1030, 8200)])
@pytest.mark.parametrize("place", ["dy", "x", "past"])
def test_far_from_zero_in_place(rows, cols, place):
    backward(rows, cols, "f32", shift=1e5, past=place == "past", place=place)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(5, 20), (1500, 20), (30, 300), (1100, 2050), (30, 5000), (1030, 9000)])
def test_rows_without_variance_far_from_zero(rows, cols, dtype):
    """What a wavefront has behind the columns is no part of a row, whose mean times r is beyond 32 bits there."""
    x, _ = padded(torch.full((rows, cols), 2.0 ** 113), DT[dtype])         # (whose sum and mean are exact)
    dy, _ = padded(random(rows, cols, 1) * 1e-2, DT[dtype])
    y, _ = padded(torch.full((rows, cols), float("nan")), DT[dtype])
    dx, _ = padded(torch.full((rows, cols), float("nan")), DT[dtype])
    stats, dw, db = torch.empty((rows, 2), device="cuda"), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    psgd.norm(x, None, None, y, stats, eps=1e-12)
    assert (y == 0).all() and (stats[:, 0] == 2.0 ** 113).all()
    psgd.NormGrad(rows, cols, CODE[dtype], grad_dtype=psgd.PSGD_F32).run(dy, x, None, stats, dx, dw, db)
    g = dy.double()
    want = 1e6 * (g - g.mean(1, keepdim=True))
    assert ((dx.double() - want).abs() <= 1e6 * STEPS * (g.abs() + g.abs().mean(1, keepdim=True)) + UNIT[dtype] * 1.01 * want.abs()).all()
    assert (dw == 0).all() and ((db.double() - g.sum(0)).abs() <= (rows / 256 + 60) * 2.0 ** -24 * g.abs().sum(0)).all()


# several rows to a workgroup, the next on its way while one is added up: of every number of wavefronts and pieces that a row takes
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(9000, 60), (9000, 100), (9000, 250), (6000, 500), (6000, 1000), (6000, 1500), (4000, 2040), (1500, 2500), (1500, 4096), (1500, 8000),
                                       (1500, 10001), (1500, 12296), (1500, 16384)])
def test_many_rows(rows, cols, dtype):
    backward(rows, cols, dtype, past=True, accumulate=True)


# just beyond the 96 MiB from which on loads and stores have the non-temporal hint
@pytest.mark.parametrize("add,past", [(True, True), (False, False)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols", [60, 500, 1001, 3001, 6001, 9001, 12297, 16384])
def test_large(cols, dtype, add, past):
    size = 4 if dtype == "f32" else 2
    rows = (96 << 20) // (cols * size * (4 if add else 2)) + 1001
    backward(rows, cols, dtype, add=add, past=past)
