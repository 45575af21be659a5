"""Host-side checks of the norms', the experts' and the distillation's entry points that need no GPU: refusals (nothing is enqueued), workspace sizes, the binding."""
import ctypes as C

import pytest
import torch

from paper_2509_11254_amd import psgd
from test_train_host import head
from test_train_binding import OnGpu, OnStream, matrix

F32, BF16 = psgd.PSGD_F32, psgd.PSGD_BF16
OK, INVALID, SHAPE, ALIGN = psgd.PSGD_OK, psgd.PSGD_E_INVALID_ARG, psgd.PSGD_E_SHAPE, psgd.PSGD_E_ALIGN
BIG = (1 << 22) + 8
M = 1 << 20         # apart, so that nothing overlaps


@pytest.fixture(scope="module")
def lib():
    return psgd.load_library()


def norm(lib, **change):
    a = dict(rows=6, cols=40, dtype=F32, x=M, ld_x=40, add=2 * M, ld_add=48, weight=3 * M, bias=4 * M, w_dtype=F32, eps=1e-5, total=5 * M, ld_total=56, y=6 * M, ld_y=40, stats=7 * M)
    assert not set(change) - set(a)
    a.update(change)
    return lib.psgd_norm(None, *a.values())


def norm_backward(lib, **change):
    a = dict(workspace=M, stream=None, rows=6, cols=40, dtype=F32, dy=2 * M, ld_dy=40, x=3 * M, ld_x=40, weight=4 * M, w_dtype=F32, stats=5 * M, dtotal=6 * M, ld_dtotal=48,
             dx=7 * M, ld_dx=40, dweight=8 * M, dbias=9 * M, g_dtype=F32, accumulate=0)
    assert not set(change) - set(a)
    a.update(change)
    return lib.psgd_norm_backward(*a.values())


@pytest.mark.parametrize("change,want", [
    (dict(dtype=2), INVALID), (dict(w_dtype=-1), INVALID), (dict(eps=-1e-9), INVALID), (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID),
    (dict(x=None), INVALID), (dict(y=None), INVALID), (dict(add=None), INVALID), (dict(total=None), INVALID),
    (dict(rows=-1), SHAPE), (dict(cols=0), SHAPE), (dict(cols=16385), SHAPE), (dict(rows=(1 << 30) + 1), SHAPE), (dict(ld_x=BIG), SHAPE),
    (dict(ld_add=BIG), SHAPE), (dict(ld_total=BIG), SHAPE), (dict(ld_y=BIG), SHAPE), (dict(ld_x=32), ALIGN), (dict(ld_add=36), ALIGN), (dict(ld_total=32), ALIGN), (dict(ld_y=44), ALIGN), (dict(x=M + 8), ALIGN), (dict(add=M // 2 + 4), ALIGN), (dict(weight=M + 4), ALIGN),
    (dict(bias=M + 8), ALIGN), (dict(total=M + 2), ALIGN), (dict(y=5 * M + 8), ALIGN), (dict(stats=M + 8), ALIGN),
    # 6 rows of 160 bytes: y begins in x's last row; over its rows by half; over the other output, over parameters and statistics
    (dict(y=M + 5 * 160), INVALID), (dict(y=M + 80), INVALID), (dict(y=M, ld_y=48), INVALID), (dict(total=2 * M), INVALID), (dict(y=5 * M), INVALID), (dict(total=3 * M), INVALID),
    (dict(y=4 * M + 144), INVALID), (dict(stats=M + 800), INVALID), (dict(stats=6 * M + 944), INVALID), (dict(stats=3 * M), INVALID)])
def test_norm_refuses(lib, change, want):
    assert norm(lib, **change) == want


@pytest.mark.parametrize("change,want", [
    (dict(dtype=2), INVALID), (dict(w_dtype=3), INVALID), (dict(g_dtype=-1), INVALID), (dict(workspace=None), INVALID), (dict(dy=None), INVALID), (dict(x=None), INVALID),
    (dict(stats=None), INVALID), (dict(dx=None), INVALID), (dict(rows=-1), SHAPE), (dict(cols=0), SHAPE), (dict(cols=16385), SHAPE), (dict(ld_dy=BIG), SHAPE),
    (dict(ld_x=BIG), SHAPE), (dict(ld_dx=BIG), SHAPE), (dict(ld_dtotal=BIG), SHAPE), (dict(ld_dtotal=32), ALIGN), (dict(dx=6 * M), INVALID), (dict(ld_dy=36), ALIGN), (dict(ld_x=32), ALIGN), (dict(ld_dx=44), ALIGN), (dict(workspace=M + 128), ALIGN),
    (dict(dy=M + 8), ALIGN), (dict(x=M + 8), ALIGN), (dict(weight=M + 8), ALIGN), (dict(stats=M + 8), ALIGN), (dict(dtotal=M + 8), ALIGN), (dict(dx=M + 8), ALIGN),
    (dict(dweight=M + 8), ALIGN), (dict(dbias=M + 8), ALIGN),
    (dict(dx=2 * M + 160), INVALID), (dict(dx=3 * M, ld_dx=48), INVALID), (dict(dx=4 * M), INVALID), (dict(dx=5 * M), INVALID), (dict(dweight=2 * M + 800), INVALID),
    (dict(dbias=8 * M), INVALID), (dict(dweight=4 * M), INVALID), (dict(dbias=7 * M + 944), INVALID)])
def test_norm_backward_refuses(lib, change, want):
    assert norm_backward(lib, **change) == want


def test_norm_without_rows(lib):
    assert norm(lib, rows=0, x=None, add=None, total=None, y=None, stats=None) == OK
    assert norm_backward(lib, rows=0, dy=None, x=None, stats=None, dx=None, accumulate=1) == OK
    assert norm_backward(lib, rows=0, dy=None, x=None, stats=None, dx=None, dweight=None, dbias=None, workspace=None) == OK


def test_norm_workspace(lib):
    size = lib.psgd_norm_backward_workspace_bytes
    assert size(0, 40, F32) > 0 and size(1 << 30, 16384, BF16) < 1 << 28
    for bad in ((-1, 40, F32), (4, 0, F32), (4, 16385, F32), (4, 40, 2)):
        assert size(*bad) == 0


def sort(lib, **change):
    a = dict(workspace=M, stream=None, tokens=6, slots=2, experts=5, choice=2 * M, place=3 * M, order=4 * M, offsets=5 * M)
    assert not set(change) - set(a)
    a.update(change)
    return lib.psgd_expert_sort(*a.values())


@pytest.mark.parametrize("change,want", [
    (dict(workspace=None), INVALID), (dict(choice=None), INVALID), (dict(place=None), INVALID), (dict(order=None), INVALID), (dict(offsets=None), INVALID),
    (dict(tokens=-1), SHAPE), (dict(slots=0), SHAPE), (dict(experts=0), SHAPE), (dict(experts=1025), SHAPE), (dict(tokens=1 << 29, slots=3), SHAPE),
    (dict(tokens=1 << 62, slots=4), SHAPE), (dict(slots=1 << 40), SHAPE), (dict(workspace=M + 64), ALIGN), (dict(choice=M + 8), ALIGN), (dict(place=M + 4), ALIGN),
    (dict(order=M + 8), ALIGN), (dict(offsets=M + 4), ALIGN), (dict(place=2 * M + 80), INVALID), (dict(order=3 * M + 32), INVALID), (dict(offsets=4 * M), INVALID)])
def test_sort_refuses(lib, change, want):
    assert sort(lib, **change) == want
    if want == SHAPE:
        a = dict(dict(tokens=6, slots=2, experts=5), **change)
        assert lib.psgd_expert_sort_workspace_bytes(a["tokens"], a["slots"], a["experts"]) == 0


def rows(lib, **change):
    a = dict(tokens=6, slots=2, cols=40, dtype=F32, x=M, ld_x=40, place=2 * M, xs=3 * M, ld_xs=40)
    a.update(change)
    return lib.psgd_expert_rows(None, *a.values())


def combine(lib, **change):
    a = dict(tokens=6, slots=2, cols=40, dtype=F32, ys=M, ld_ys=40, place=2 * M, weight=3 * M, y=4 * M, ld_y=40)
    a.update(change)
    return lib.psgd_expert_combine(None, *a.values())


def combine_backward(lib, **change):
    a = dict(tokens=6, slots=2, cols=40, dtype=F32, dy=M, ld_dy=40, ys=2 * M, ld_ys=40, place=3 * M, weight=4 * M, dys=5 * M, ld_dys=40, dweight=6 * M)
    a.update(change)
    return lib.psgd_expert_combine_backward(None, *a.values())


SHAPES = [(dict(tokens=-1), SHAPE), (dict(slots=0), SHAPE), (dict(cols=0), SHAPE), (dict(tokens=1 << 29, slots=4), SHAPE), (dict(dtype=2), INVALID), (dict(place=None), INVALID),
          (dict(place=7 * M + 4), ALIGN)]


@pytest.mark.parametrize("call,change,want", [(f, c, w) for f in (rows, combine, combine_backward) for c, w in SHAPES] + [
    (rows, dict(x=None), INVALID), (rows, dict(xs=None), INVALID), (rows, dict(ld_x=32), ALIGN), (rows, dict(ld_xs=44), ALIGN), (rows, dict(ld_x=BIG), SHAPE),
    (rows, dict(ld_xs=BIG), SHAPE), (rows, dict(x=M + 8), ALIGN), (rows, dict(xs=M + 8), ALIGN), (rows, dict(xs=M), INVALID), (rows, dict(xs=M + 5 * 160), INVALID),
    (rows, dict(xs=2 * M + 32), INVALID),
    (combine, dict(ys=None), INVALID), (combine, dict(y=None), INVALID), (combine, dict(ld_ys=32), ALIGN), (combine, dict(ld_y=44), ALIGN), (combine, dict(ld_y=BIG), SHAPE),
    (combine, dict(weight=M + 4), ALIGN), (combine, dict(y=M + 8), ALIGN), (combine, dict(y=M + 11 * 160), INVALID), (combine, dict(y=3 * M + 32), INVALID),
    (combine_backward, dict(dy=None), INVALID), (combine_backward, dict(dys=None), INVALID), (combine_backward, dict(ys=None), INVALID),
    (combine_backward, dict(ld_dy=36), ALIGN), (combine_backward, dict(ld_ys=32), ALIGN), (combine_backward, dict(ld_dys=BIG), SHAPE), (combine_backward, dict(dys=M), INVALID),
    (combine_backward, dict(dys=2 * M + 160), INVALID), (combine_backward, dict(dys=2 * M, ld_dys=48), INVALID), (combine_backward, dict(dweight=5 * M + 1904), INVALID),
    (combine_backward, dict(dweight=4 * M), INVALID), (combine_backward, dict(dweight=2 * M), INVALID)])
def test_rows_refuse(lib, call, change, want):
    assert call(lib, **change) == want


def test_rows_without_tokens(lib):
    assert rows(lib, tokens=0, x=None, place=None, xs=None) == OK
    assert combine(lib, tokens=0, ys=None, place=None, weight=None, y=None) == OK
    assert combine_backward(lib, tokens=0, dy=None, ys=None, place=None, weight=None, dys=None, dweight=None) == OK


def distill(lib, desc=None, grad=True, **change):
    a = dict(workspace=M, stream=None, x=M, w=2 * M, top=12, index=4 * M, teacher=5 * M, t_dtype=F32, ld=16, temperature=2.0, weight=6 * M, loss=7 * M, dx=8 * M, dw=9 * M,
             accumulate=0)
    assert not set(change) - set(a)
    a.update(change)
    if not grad:
        for k in ("weight", "dx", "dw", "accumulate"):
            a.pop(k)
    return (lib.psgd_head_distill_grad if grad else lib.psgd_head_distill)(C.byref(desc or head()), *a.values())


@pytest.mark.parametrize("change,want", [
    (dict(top=0), SHAPE), (dict(top=1025, ld=1032), SHAPE), (dict(ld=BIG), SHAPE), (dict(ld=11), ALIGN), (dict(index=M + 8), ALIGN), (dict(teacher=M + 4), ALIGN),
    (dict(index=None), INVALID), (dict(teacher=None), INVALID), (dict(t_dtype=2), INVALID), (dict(temperature=0.0), INVALID), (dict(temperature=-1.0), INVALID),
    (dict(temperature=float("nan")), INVALID), (dict(temperature=float("inf")), INVALID), (dict(temperature=1e-42), INVALID), (dict(temperature=1e-31), INVALID), (dict(temperature=1e31), INVALID), (dict(x=None), INVALID),
    (dict(loss=None), INVALID), (dict(workspace=M + 16), ALIGN),
    # 100 tokens: 99 rows of 16 entries and 12 more
    (dict(loss=4 * M + 99 * 128 + 80), INVALID), (dict(loss=5 * M + 99 * 64 + 32), INVALID)])
def test_distillation_refuses(lib, change, want):
    assert distill(lib, **change) == want
    assert distill(lib, grad=False, **change) == want
    if "top" in change:
        assert lib.psgd_head_distill_workspace_bytes(C.byref(head()), change["top"], 1) == 0


def test_distillation_refuses_as_the_head(lib):
    for change, want in ((dict(dtype=2), INVALID), (dict(d=0), SHAPE), (dict(tokens=-1), SHAPE), (dict(piece_tokens=-1), INVALID), (dict(ldx=60), ALIGN)):
        assert distill(lib, head(**change)) == want
    for k in ("dx", "dw"):
        assert distill(lib, **{k: None}) == INVALID
        assert distill(lib, **{k: 4 * M + 128}) == INVALID and distill(lib, **{k: 5 * M + 64}) == INVALID
    assert distill(lib, dx=M, desc=head(ldx=72)) == INVALID
    assert lib.psgd_head_distill_workspace_bytes(None, 5, 0) == 0


def test_distillation_workspace_is_bounded(lib):
    """Pieces of the tokens: lists and statistics exist for one piece at a time."""
    def size(tokens, top, grad, **change):
        return lib.psgd_head_distill_workspace_bytes(C.byref(head(tokens=tokens, vocab=64000, **change)), top, grad)

    assert 0 < size(1 << 14, 1024, 1, grad_dtype=BF16) < 1.3 * 2 ** 30 and size(1 << 18, 1024, 1, grad_dtype=BF16) < 1.4 * 2 ** 30
    assert size(1 << 22, 1024, 0) < 2.5 * 2 ** 30
    assert size(1 << 14, 64, 1, piece_tokens=256) < 2 ** 28 and size(0, 64, 1) > 0
    assert size(1000, 64, 1, piece_tokens=(1 << 63) - 1) == size(1000, 64, 1, piece_tokens=1000)


def test_binding_refuses_sizes():
    for make in (lambda: psgd.HeadDistill(10, 64, 100, 0), lambda: psgd.HeadDistill(10, 64, 100, 1025), lambda: psgd.HeadDistill(10, 0, 100, 5),
                 lambda: psgd.NormGrad(10, 16385), lambda: psgd.NormGrad(10, 10, 3), lambda: psgd.NormGrad(10, 10, F32, 7), lambda: psgd.ExpertSort(4, 0, 3),
                 lambda: psgd.ExpertSort(4, 2, 2000)):
        with pytest.raises(psgd.PsgdError):
            make()


def vec(n, dtype=torch.float32, device=0, shape=None):
    return OnGpu(torch.empty(shape or n, dtype=dtype), device)


def on(plan):
    def take(device):
        plan.workspace = OnGpu(plan.workspace.tensor if isinstance(plan.workspace, OnGpu) else plan.workspace, device)
        return plan
    return take


def expert_order(tokens, slots, experts, device=0):
    return psgd.ExpertOrder(vec(0, torch.int32, device, (tokens, slots)), vec(tokens * slots, torch.int32, device), vec(experts + 1, torch.int32, device))


def calls():
    """Every call of the binding, by the tensors it takes."""
    t, s, e, d = 6, 2, 5, 40
    m, v = (lambda r, c=d: lambda dev: matrix(r, c, device=dev)), (lambda n, dtype=torch.float32, shape=None: lambda dev: vec(n, dtype, dev, shape))
    o, w = (lambda dev: expert_order(t, s, e, dev)), v(0, shape=(t, s))
    plan = on(psgd.HeadDistill(t, d, 24, 5, F32, device="cpu"))
    entries = [v(0, torch.int64, (t, 5)), v(0, shape=(t, 5))]
    return {
        "distill": (lambda plan, x, w, i, k, l, stream: plan.loss(x, w, i, k, l, stream=stream), [plan, m(t), m(24), *entries, v(t)]),
        "distill_grad": (lambda plan, x, w, i, k, l, dx, dw, c, stream: plan.loss_grad(x, w, i, k, l, dx, dw, weight=c, stream=stream),
                         [plan, m(t), m(24), *entries, v(t), m(t), m(24), v(t)]),
        "norm": (lambda x, w, b, y, st, add, total, stream: psgd.norm(x, w, b, y, st, add=add, total=total, stream=stream),
                 [m(t), v(d), v(d), m(t), v(0, shape=(t, 2)), m(t), m(t)]),
        "norm_grad": (lambda plan, dy, x, w, st, dx, dw, db, past, stream: plan.run(dy, x, w, st, dx, dw, db, dtotal=past, stream=stream),
                      [on(psgd.NormGrad(t, d, F32, device="cpu")), m(t), m(t), v(d), v(0, shape=(t, 2)), m(t), v(d), v(d), m(t)]),
        "sort": (lambda plan, c, o, stream: plan.run(c, o, stream=stream), [on(psgd.ExpertSort(t, s, e, device="cpu")), v(0, torch.int64, (t, s)), o]),
        "rows": (lambda x, o, xs, stream: psgd.expert_rows(x, o, xs, stream=stream), [m(t), o, m(t * s)]),
        "combine": (lambda ys, o, y, w, stream: psgd.expert_combine(ys, o, y, weight=w, stream=stream), [m(t * s), o, m(t), w]),
        "combine_backward": (lambda dy, ys, o, dys, w, dw, stream: psgd.expert_combine_backward(dy, ys, o, dys, weight=w, dweight=dw, stream=stream),
                             [m(t), m(t * s), o, m(t * s), w, w]),
    }


class Enqueued(Exception):
    pass


@pytest.mark.parametrize("name", sorted(calls()))
def test_tensors_of_another_device(monkeypatch, name):
    """All tensors and the plan's workspace are on the device of the stream that the call goes to."""
    call, args = calls()[name]
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0, raising=False)

    def stop(*a):
        raise Enqueued                      # in the place of the library's result

    monkeypatch.setattr(psgd, "_check", stop)
    lib = psgd.load_library()
    for f in psgd.EXPORTS:
        if f.startswith(("psgd_norm", "psgd_expert", "psgd_head_distill")) and not f.endswith("_bytes"):
            monkeypatch.setattr(lib, f, lambda *a: 0)
    for stream, device in ((None, 0), (OnStream(0), 0), (OnStream(1), 1)):
        with pytest.raises(Enqueued):
            call(*[a(device) for a in args], stream)
        for i in range(len(args)):
            with pytest.raises(ValueError, match="cuda"):
                call(*[a(1 - device if j == i else device) for j, a in enumerate(args)], stream)


def test_binding_refuses_tensors():
    m, w, st = (lambda r, c=40, dtype=torch.float32: matrix(r, c, dtype)), vec(40), vec(0, shape=(6, 2))
    plan = psgd.HeadDistill(6, 40, 24, 5, F32, device="cpu")

    def entries(index=(6, 5), teacher=(6, 5), index_type=torch.int64, teacher_type=torch.float32):
        return (vec(0, index_type, 0, index) if isinstance(index, tuple) else OnGpu(index)), vec(0, teacher_type, 0, teacher)

    bad = [
        lambda: plan.loss(m(6), m(24), *entries(index=(6, 4)), vec(6)), lambda: plan.loss(m(6), m(24), *entries(teacher=(5, 5)), vec(6)),
        lambda: plan.loss(m(6), m(24), *entries(index_type=torch.int32), vec(6)), lambda: plan.loss(m(6), m(24), *entries(teacher_type=torch.float16), vec(6)),
        lambda: plan.loss(m(6), m(24), *entries(index=torch.empty((6, 8), dtype=torch.int64)[:, :5]), vec(6)),
        lambda: plan.loss(m(6), m(24), *entries(index=torch.empty((1, 5), dtype=torch.int64).expand(6, 5)), vec(6)),
        lambda: plan.loss(m(6), m(24), *entries(index=torch.empty((6, 10), dtype=torch.int64)[:, ::2]), vec(6)),
        lambda: plan.loss(m(6), m(24), *entries(), vec(5)), lambda: plan.loss(m(6), m(25), *entries(), vec(6)),
        lambda: psgd.HeadDistill(6, 40, 24, 5, F32, grad=False, device="cpu").loss_grad(m(6), m(24), *entries(), vec(6), m(6), m(24)),
        lambda: psgd.norm(m(6), w, None, m(5)), lambda: psgd.norm(m(6), w, None, m(6, dtype=torch.bfloat16)), lambda: psgd.norm(m(6), vec(39), None, m(6)),
        lambda: psgd.norm(m(6), w, vec(40, torch.bfloat16), m(6)), lambda: psgd.norm(m(6), w, None, m(6), vec(12)), lambda: psgd.norm(m(6), w, None, m(6), add=m(6)),
        lambda: psgd.norm(m(6), w, None, m(6), total=m(6)), lambda: psgd.norm(m(6), w, None, m(6), add=matrix(6, 41), total=m(6)),
        lambda: psgd.norm(m(6), vec(40, torch.float16), None, m(6)), lambda: psgd.norm(m(6, dtype=torch.float16), None, None, m(6)),
        lambda: psgd.NormGrad(6, 40, F32, device="cpu").run(m(6), m(6), vec(40, torch.bfloat16), st, m(6)),
        lambda: psgd.NormGrad(6, 40, F32, device="cpu").run(m(6), m(6), w, st, m(6), vec(40, torch.bfloat16)),
        lambda: psgd.NormGrad(6, 40, F32, device="cpu").run(m(6), m(6), w, vec(0, shape=(5, 2)), m(6)),
        lambda: psgd.ExpertOrder(vec(0, torch.int64, 0, (6, 2)), vec(12, torch.int32), vec(6, torch.int32)),
        lambda: psgd.ExpertOrder(vec(0, torch.int32, 0, (6, 2)), vec(11, torch.int32), vec(6, torch.int32)),
        lambda: psgd.ExpertSort(6, 2, 5, device="cpu").run(vec(0, torch.int32, 0, (6, 2)), expert_order(6, 2, 5)),
        lambda: psgd.ExpertSort(6, 2, 5, device="cpu").run(vec(0, torch.int64, 0, (6, 2)), expert_order(6, 2, 6)),
        lambda: psgd.expert_rows(m(6), expert_order(6, 2, 5), m(11)), lambda: psgd.expert_rows(m(5), expert_order(6, 2, 5), m(12)),
        lambda: psgd.expert_combine(m(12), expert_order(6, 2, 5), m(6), weight=vec(12)),
        lambda: psgd.expert_combine_backward(m(6), None, expert_order(6, 2, 5), m(12), dweight=vec(0, shape=(6, 2))),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail("call %d" % i)
