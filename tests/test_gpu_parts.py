"""A split contraction runs in as many parts as it was planned for."""
import ctypes as C

import pytest
import torch

from paper_2509_11254_amd import psgd
from test_gpu_tiles import TilePlan

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens,d,vocab", [(640, 64, 32), (999, 61, 30)])
def test_parts_of_fp32_gradients(tokens, d, vocab):
    """dW of fp32 tokens over a vocabulary of one chunk, for which only dW is in parts: their sums are the last thing in the workspace, and each has
    been written (what was there before is no number that a sum comes to)."""
    plan_of = psgd.load_library()["_ZN4psgd10split_planElllb"]
    plan_of.restype, plan_of.argtypes = TilePlan, [C.c_int64, C.c_int64, C.c_int64, C.c_bool]
    assert plan_of(d, tokens, 1, True).n_split == 1
    tile = plan_of(d, vocab, -(-tokens // 32), True)
    narrow, rows, ld = 64, 64 if tile.shape == 5 else 128, -(-d // 8) * 8
    assert tile.n_split > -(-tokens // 64) and d <= narrow and vocab <= narrow
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    x, w = torch.zeros((tokens, ld), device="cuda")[:, :d], torch.zeros((vocab, ld), device="cuda")[:, :d]
    x.copy_(torch.randn((tokens, d), generator=gen, device="cuda"))
    w.copy_(torch.randn((vocab, d), generator=gen, device="cuda"))
    labels = torch.randint(0, vocab, (tokens,), generator=gen, device="cuda")
    loss, dx, dw = torch.empty(tokens, device="cuda"), torch.zeros((tokens, ld), device="cuda")[:, :d], torch.zeros((vocab, ld), device="cuda")[:, :d]
    plan = psgd.HeadLoss(tokens, d, vocab, psgd.PSGD_F32)
    plan.workspace.fill_(0xFF)
    plan.loss_grad(x, w, labels, loss, dx, dw)
    n_bytes = int(plan.lib.psgd_head_workspace_bytes(C.byref(plan.desc), 1))
    start = plan._ws_ptr - plan.workspace.data_ptr() + n_bytes - (tile.n_split * rows * ld * 4 + 255) // 256 * 256
    parts = plan.workspace[start:start + tile.n_split * vocab * ld * 4].view(torch.int32).view(tile.n_split, vocab, ld)[:, :, :d]
    assert [bool((part != -1).all()) for part in parts] == [True] * tile.n_split
    # and they are the sums: in their order, they add up to dW
    total = parts.view(torch.float32).double().sum(0) / tokens
    assert ((total - dw.double()).abs() <= 2.0 ** -21 * parts.view(torch.float32).double().abs().sum(0) / tokens).all()
