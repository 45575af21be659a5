"""What the Python binding of the training operators refuses before anything is enqueued; without a GPU: its tensors are stand-ins that
say they are on one."""
import pytest
import torch

from paper_2509_11254_amd import psgd


class OnGpu:
    """A tensor's shape, strides and type, on a GPU that is not there."""

    def __init__(self, tensor, device=0):
        self.tensor, self.index = tensor, device

    is_cuda = True
    device = property(lambda self: torch.device("cuda", self.index))

    def get_device(self):
        return self.index

    def data_ptr(self):
        return 1 << 20

    def __getattr__(self, name):
        return getattr(self.tensor, name)


def matrix(rows, cols, dtype=torch.float32, device=0):
    return OnGpu(torch.empty((rows, (cols + 15) // 16 * 16), dtype=dtype)[:, :cols], device)


def test_rows_that_lie_over_each_other():
    """An expanded row has stride 0, which the head's descriptor would take for d; any stride below the columns is refused."""
    x = torch.empty((1, 64))
    for t in (x.expand(5, 64), torch.empty(1000).as_strided((5, 64), (56, 1)), torch.empty((1, 1)).expand(5, 1)):
        with pytest.raises(ValueError, match="X"):
            psgd._matrix("X", OnGpu(t), *t.shape)
    for t, ld in ((torch.empty((5, 64)), 64), (torch.empty((5, 80))[:, :61], 80), (x, 64), (torch.empty((0, 64)), 64), (torch.empty((5, 8))[:, :1], 8)):
        assert psgd._matrix("X", OnGpu(t), *t.shape) == ld


class OnStream:
    cuda_stream = 0

    def __init__(self, index):
        self.device = torch.device("cuda", index)


def checkpoint(rows, cols, device=0):
    return psgd.Act8(OnGpu(torch.empty((rows, (cols + 15) // 16 * 16), dtype=torch.int8), device),
                     OnGpu(torch.empty((rows, -(-cols // 32)), dtype=torch.uint8), device), cols)


def calls():
    """Every call of the binding, by the tensors it takes."""
    f, t, d, v = psgd.PSGD_F32, 6, 40, 24
    head, wgrad = psgd.HeadLoss(t, d, v, f, device="cpu"), psgd.WeightGrad(t, v, d, f, device="cpu")

    def vectors(device):
        return dict(labels=OnGpu(torch.empty(t, dtype=torch.int64), device), loss=OnGpu(torch.empty(t), device))

    def on(plan):
        def take(device):
            plan.workspace = OnGpu(plan.workspace.tensor if isinstance(plan.workspace, OnGpu) else plan.workspace, device)
            return plan
        return take

    m, k = (lambda r, c: lambda dev: matrix(r, c, device=dev)), (lambda r, c: lambda dev: checkpoint(r, c, dev))
    lab, los = (lambda dev: vectors(dev)["labels"]), (lambda dev: vectors(dev)["loss"])
    return {
        "loss": (lambda plan, x, w, y, l, stream: plan.loss(x, w, y, l, stream=stream), [on(head), m(t, d), m(v, d), lab, los]),
        "loss_grad": (lambda plan, x, w, y, l, dx, dw, c, stream: plan.loss_grad(x, w, y, l, dx, dw, weight=c, stream=stream),
                      [on(head), m(t, d), m(v, d), lab, los, m(t, d), m(v, d), los]),
        "store": (lambda x, kept, stream: psgd.act_store(x, kept, stream=stream), [m(t, d), k(t, d)]),
        "restore": (lambda x, kept, stream: psgd.act_restore(kept, x, stream=stream), [m(t, d), k(t, d)]),
        "glu": (lambda g, u, h, kg, ku, stream: psgd.act_glu(g, u, h, kg, ku, stream=stream), [m(t, d)] * 3 + [k(t, d)] * 2),
        "glu_backward": (lambda kg, ku, dh, dg, du, stream: psgd.act_glu_backward(kg, ku, dh, dg, du, stream=stream),
                         [k(t, d)] * 2 + [m(t, d)] * 3),
        "wgrad": (lambda plan, dy, kept, g, stream: plan.run(dy, kept, g, stream=stream), [on(wgrad), m(t, v), k(t, d), m(v, d)]),
    }


class Enqueued(Exception):
    pass


@pytest.mark.parametrize("name", sorted(calls()))
def test_tensors_of_another_device(monkeypatch, name):
    """All tensors, checkpoints and the plan's workspace are on the device of the stream that the call goes to."""
    call, args = calls()[name]
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0, raising=False)

    def stop(*a):
        raise Enqueued                      # in the place of the library's result

    monkeypatch.setattr(psgd, "_check", stop)
    lib = psgd.load_library()
    for f in ("psgd_head_loss", "psgd_head_loss_grad", "psgd_act_store", "psgd_act_restore", "psgd_act_glu", "psgd_act_glu_backward", "psgd_act_wgrad"):
        monkeypatch.setattr(lib, f, lambda *a: 0)
    for stream, device in ((None, 0), (OnStream(0), 0), (OnStream(1), 1)):
        with pytest.raises(Enqueued):
            call(*[a(device) for a in args], stream)
        for i in range(len(args)):
            with pytest.raises(ValueError, match="cuda"):
                call(*[a(1 - device if j == i else device) for j, a in enumerate(args)], stream)
    with pytest.raises(ValueError, match="cuda"):
        call(*[a(1) for a in args], None)


def test_a_gated_unit_has_both_checkpoints_or_neither(monkeypatch):
    """up without a place for its checkpoint, and a checkpoint that would be left as it was."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    m, k = (lambda: matrix(6, 40)), (lambda: checkpoint(6, 40))
    for up, kept_up in ((m(), None), (None, k())):
        with pytest.raises(ValueError, match="up"):
            psgd.act_glu(m(), up, m(), k(), kept_up)
    for kept_up, dup in ((k(), None), (None, m())):
        with pytest.raises(ValueError, match="up"):
            psgd.act_glu_backward(k(), kept_up, m(), m(), dup)
