"""Host-side checks of the head's, the checkpoints' and the weight gradient's entry points that need no GPU: refusals (nothing
is enqueued), workspace sizes, the descriptor's layout."""
import ctypes as C
import os
import subprocess

import pytest

from paper_2509_11254_amd import psgd

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 4096        # an aligned address that no refused call looks at
BIG = (1 << 22) + 8


@pytest.fixture(scope="module")
def lib():
    return psgd.load_library()


def head(**change):
    d = dict(tokens=100, d=64, vocab=1000, ldx=0, ldw=0, lddx=0, lddw=0, dtype=psgd.PSGD_BF16, grad_dtype=psgd.PSGD_F32, piece_tokens=0)
    d.update(change)
    return psgd.HeadDesc(*[d[f[0]] for f in psgd.HeadDesc._fields_])


def test_head_desc_layout(tmp_path):
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "psgd.h"', 'int main(void) {',
             'printf("%zu\\n", sizeof(psgd_head_desc));']
    lines += ['printf("%%zu\\n", offsetof(psgd_head_desc, %s));' % f[0] for f in psgd.HeadDesc._fields_]
    lines += ['printf("%d\\n%d\\n", PSGD_SILU, PSGD_GELU);', 'return 0; }']
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines))
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    assert got == [C.sizeof(psgd.HeadDesc)] + [getattr(psgd.HeadDesc, f[0]).offset for f in psgd.HeadDesc._fields_] + [psgd.PSGD_SILU, psgd.PSGD_GELU]


@pytest.mark.parametrize("change,want", [
    (dict(dtype=2), psgd.PSGD_E_INVALID_ARG), (dict(grad_dtype=-1), psgd.PSGD_E_INVALID_ARG), (dict(piece_tokens=-1), psgd.PSGD_E_INVALID_ARG),
    (dict(d=0), psgd.PSGD_E_SHAPE), (dict(vocab=0), psgd.PSGD_E_SHAPE), (dict(tokens=-1), psgd.PSGD_E_SHAPE), (dict(tokens=1 << 31), psgd.PSGD_E_SHAPE),
    (dict(d=BIG, ldx=BIG), psgd.PSGD_E_SHAPE), (dict(vocab=BIG), psgd.PSGD_E_SHAPE), (dict(ldx=BIG), psgd.PSGD_E_SHAPE),
    (dict(lddw=BIG), psgd.PSGD_E_SHAPE), (dict(ldx=60), psgd.PSGD_E_ALIGN), (dict(ldw=56), psgd.PSGD_E_ALIGN), (dict(lddx=68), psgd.PSGD_E_ALIGN),
    (dict(lddw=-64), psgd.PSGD_E_ALIGN), (dict(d=63), psgd.PSGD_E_ALIGN)])
def test_head_refuses(lib, change, want):
    d = head(**change)
    assert lib.psgd_head_loss_grad(C.byref(d), P, None, P, P, P, None, P, P, P, 0) == want
    if not {"grad_dtype", "lddx", "lddw"} & set(change):
        assert lib.psgd_head_loss(C.byref(d), P, None, P, P, P, P) == want
    if want != psgd.PSGD_E_ALIGN and not {"ldx", "lddw"} & (set(change) - {"d"}):
        assert lib.psgd_head_workspace_bytes(C.byref(d), 1) == 0


def test_head_refuses_pointers(lib):
    d = head()
    args = [C.byref(d), P, None, P, P, P, None, P, P, P, 0]
    for i in (0, 1, 3, 4, 5, 7, 8, 9):
        bad = list(args)
        bad[i] = None
        assert lib.psgd_head_loss_grad(*bad) == psgd.PSGD_E_INVALID_ARG, i
    for i, step in ((1, 16), (3, 8), (4, 8), (8, 4), (9, 2)):
        bad = list(args)
        bad[i] = P + step
        assert lib.psgd_head_loss_grad(*bad) == psgd.PSGD_E_ALIGN, i
    assert lib.psgd_head_workspace_bytes(None, 0) == 0


def test_head_workspace_is_bounded(lib):
    """Pieces of the tokens: the workspace does not grow with tokens * vocab."""
    small = lib.psgd_head_workspace_bytes(C.byref(head(tokens=1 << 14, vocab=64000, grad_dtype=psgd.PSGD_BF16)), 1)
    large = lib.psgd_head_workspace_bytes(C.byref(head(tokens=1 << 18, vocab=64000, grad_dtype=psgd.PSGD_BF16)), 1)
    assert 0 < small < 1.2 * 2 ** 30 and large < 1.4 * 2 ** 30
    piece = lib.psgd_head_workspace_bytes(C.byref(head(tokens=1 << 14, vocab=64000, grad_dtype=psgd.PSGD_BF16, piece_tokens=256)), 1)
    assert piece < 2 ** 27
    assert lib.psgd_head_workspace_bytes(C.byref(head(tokens=1 << 14)), 0) < lib.psgd_head_workspace_bytes(C.byref(head(tokens=1 << 14)), 1)
    assert lib.psgd_head_workspace_bytes(C.byref(head(tokens=0)), 1) > 0


F32, BF16 = psgd.PSGD_F32, psgd.PSGD_BF16
INVALID, SHAPE, ALIGN = psgd.PSGD_E_INVALID_ARG, psgd.PSGD_E_SHAPE, psgd.PSGD_E_ALIGN


@pytest.mark.parametrize("rows,cols,dtype,ld,ldc,want", [
    (4, 40, 9, 40, 48, INVALID), (-1, 40, F32, 40, 48, SHAPE), (4, 0, F32, 8, 16, SHAPE), (4, 40, F32, 32, 48, ALIGN), (4, 40, F32, 44, 48, ALIGN),
    (4, 40, F32, 40, 40, ALIGN), (4, 40, F32, 40, 32, ALIGN), (1 << 31, 40, F32, 40, 48, SHAPE), (1 << 30, 1 << 30, F32, 1 << 30, 1 << 30, SHAPE)])
def test_checkpoints_refuse(lib, rows, cols, dtype, ld, ldc, want):
    assert lib.psgd_act_store(None, rows, cols, P, dtype, ld, P, ldc, P) == want
    assert lib.psgd_act_restore(None, rows, cols, P, ldc, P, P, dtype, ld) == want
    assert lib.psgd_act_glu(None, rows, cols, 0, dtype, P, P, ld, P, ld, P, P, P, P, ldc) == want
    assert lib.psgd_act_glu_backward(None, rows, cols, 1, dtype, P, P, P, P, ldc, P, ld, P, P, ld) == want


def test_checkpoints_refuse_pointers(lib):
    assert lib.psgd_act_store(None, 4, 40, None, F32, 40, P, 48, P) == INVALID
    assert lib.psgd_act_store(None, 4, 40, P, F32, 40, None, 48, P) == INVALID
    assert lib.psgd_act_restore(None, 4, 40, P, 48, None, P, F32, 40) == INVALID
    assert lib.psgd_act_store(None, 4, 40, P + 8, F32, 40, P, 48, P) == ALIGN
    assert lib.psgd_act_restore(None, 4, 40, P + 8, 48, P, P, F32, 40) == ALIGN
    # act, a checkpoint of what is not there, and one that is missing
    assert lib.psgd_act_glu(None, 4, 40, 2, F32, P, P, 40, P, 40, P, P, P, P, 48) == INVALID
    assert lib.psgd_act_glu(None, 4, 40, 0, F32, P, None, 40, P, 40, P, P, P, P, 48) == INVALID
    assert lib.psgd_act_glu(None, 4, 40, 0, F32, P, P, 40, P, 40, P, P, None, P, 48) == INVALID
    assert lib.psgd_act_glu_backward(None, 4, 40, 0, F32, P, P, P, P, 48, P, 40, P, None, 40) == INVALID
    assert lib.psgd_act_glu_backward(None, 4, 40, 0, F32, P, P, None, None, 48, P, 40, P, P, 40) == INVALID
    assert lib.psgd_act_glu_backward(None, 4, 40, -1, F32, P, P, P, P, 48, P, 40, P, P, 40) == INVALID
    # no rows: nothing to do, and no pointers needed
    assert lib.psgd_act_store(None, 0, 40, None, F32, 40, None, 48, None) == psgd.PSGD_OK
    assert lib.psgd_act_glu(None, 0, 40, 0, F32, None, None, 40, None, 40, None, None, None, None, 48) == psgd.PSGD_OK


def test_weight_gradient_refuses(lib):
    def call(ws=P, tokens=8, out=24, inp=40, dy=P, dt=BF16, ldy=24, codes=P, ldc=48, scales=P, g=P, gt=F32, ldg=40):
        return lib.psgd_act_wgrad(ws, None, tokens, out, inp, dy, dt, ldy, codes, ldc, scales, g, gt, ldg, 0)

    for bad in (dict(ws=None), dict(dy=None), dict(codes=None), dict(scales=None), dict(g=None), dict(dt=5), dict(gt=-3)):
        assert call(**bad) == INVALID, bad
    for bad in (dict(tokens=-1), dict(out=0), dict(inp=0), dict(out=BIG, ldy=BIG), dict(inp=BIG, ldg=BIG), dict(ldy=BIG)):
        assert call(**bad) == SHAPE, bad
    for bad in (dict(ldy=16), dict(ldy=28), dict(ldg=32), dict(ldc=40), dict(ws=P + 128), dict(dy=P + 8), dict(g=P + 4), dict(codes=P + 1)):
        assert call(**bad) == ALIGN, bad
    assert lib.psgd_act_wgrad_workspace_bytes(8, 24, 40, 3) == 0 and lib.psgd_act_wgrad_workspace_bytes(8, 0, 40, F32) == 0
    assert lib.psgd_act_wgrad_workspace_bytes(0, 24, 40, F32) > 0


def test_binding_refuses_sizes():
    with pytest.raises(psgd.PsgdError):
        psgd.HeadLoss(10, 0, 100)
    with pytest.raises(psgd.PsgdError):
        psgd.WeightGrad(10, 10, 0)
    with pytest.raises(psgd.PsgdError):
        psgd.WeightGrad(10, 10, 10, psgd.PSGD_BF16, 7)
