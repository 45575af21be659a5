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
