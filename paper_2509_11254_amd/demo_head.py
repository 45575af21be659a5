"""A gated unit and an output head trained with PowerSGD+ (Algorithm 2): where the gradients that the compressor takes come from.

    gate = x W_g^T, up = x W_u^T, h = silu(gate) * up, y = x + h W_d^T, loss = mean cross entropy of y W_o^T

x is a fixed table's row for each token, the label the next token of a made-up language: most often one particular successor,
else any token; a tenth of the labels is masked.  Several workers have a batch each; their gradients are averaged on the GPU by
psgd_compress, the compressed update goes to psgd_decompress_msgd.

Between the linear layers, which are torch's, every step is the library's: psgd_act_glu keeps gate and up in 8 bits, psgd_act_store
keeps x and h; psgd_head_loss_grad gives losses, dy and the head's gradient without logits in memory; psgd_act_glu_backward and
psgd_act_wgrad form the rest from the checkpoints.
"""
from __future__ import annotations

from typing import List

from . import psgd

NAMES = ("gate", "up", "down", "head")


class Model:
    """Weights in fp32 with bf16 copies, activations in bf16, gradients in bf16."""

    def __init__(self, tokens: int = 512, d: int = 256, hidden: int = 640, vocab: int = 1000, seed: int = 1):
        import torch
        self.tokens, self.d, self.hidden, self.vocab = tokens, d, hidden, vocab
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(seed)

        def randn(*shape, scale):
            return torch.randn(shape, generator=self.gen, device="cuda").mul_(scale)

        self.table = randn(vocab, d, scale=1.0).bfloat16()
        self.successor = torch.randperm(vocab, generator=self.gen, device="cuda")
        self.shapes = [(hidden, d), (hidden, d), (d, hidden), (vocab, d)]
        self.weights = [randn(*s, scale=s[1] ** -0.5) for s in self.shapes]
        self.kept_gate, self.kept_up, self.kept_h = (psgd.act_empty(tokens, hidden) for _ in range(3))
        self.kept_x = psgd.act_empty(tokens, d)
        self.head = psgd.HeadLoss(tokens, d, vocab)
        self.wgrad_in, self.wgrad_down = psgd.WeightGrad(tokens, hidden, d), psgd.WeightGrad(tokens, d, hidden)

    def batch(self):
        """Tokens and labels (the next tokens, -100 where masked)."""
        import torch
        x = torch.randint(0, self.vocab, (self.tokens,), generator=self.gen, device="cuda")
        other = torch.randint(0, self.vocab, (self.tokens,), generator=self.gen, device="cuda")
        u = torch.rand((self.tokens,), generator=self.gen, device="cuda")
        return x, torch.where(u < 0.1, -100, torch.where(u < 0.9, self.successor[x], other))

    def gradients(self, tokens, labels, out):
        """One forward and backward pass; the four weight gradients into out, the tokens' losses returned."""
        import torch
        gate_w, up_w, down_w, head_w = (w.bfloat16() for w in self.weights)
        x = self.table[tokens]
        gate, up = x @ gate_w.t(), x @ up_w.t()
        h = torch.empty_like(gate)
        psgd.act_glu(gate, up, h, self.kept_gate, self.kept_up)
        psgd.act_store(h, self.kept_h)
        psgd.act_store(x, self.kept_x)
        y = x + h @ down_w.t()
        del gate, up, h, x              # the backward pass takes the checkpoints
        loss, dy = torch.empty(self.tokens, device="cuda"), torch.empty_like(y)
        self.head.loss_grad(y, head_w, labels, loss, dy, out[3])
        self.wgrad_down.run(dy, self.kept_h, out[2])
        dh = dy @ down_w
        dgate, dup = torch.empty_like(dh), torch.empty_like(dh)
        psgd.act_glu_backward(self.kept_gate, self.kept_up, dh, dgate, dup)
        self.wgrad_in.run(dgate, self.kept_x, out[0])
        self.wgrad_in.run(dup, self.kept_x, out[1])
        return loss


def run(steps: int = 200, workers: int = 2, rank: int = 16, tau: int = 20, mu: float = 0.9, eta: float = 0.5, seed: int = 1) -> List[float]:
    """Mean losses of the counted tokens, step by step."""
    import torch
    model = Model(seed=seed)
    comp = psgd.Compressor([(r, c, rank, psgd.PSGD_BF16) for r, c in model.shapes], workers)
    grads = [[torch.empty(s, dtype=torch.bfloat16, device="cuda") for _ in range(workers)] for s in model.shapes]
    errors = [torch.zeros(s, device="cuda") for s in model.shapes]
    moments = [torch.zeros(s, device="cuda") for s in model.shapes]
    q = [torch.randn((min(s), rank), generator=model.gen, device="cuda") for s in model.shapes]
    p = [torch.zeros((max(s), rank), device="cuda") for s in model.shapes]
    losses = []
    for t in range(steps):
        total, counted = 0.0, 0
        for i in range(workers):
            tokens, labels = model.batch()
            loss = model.gradients(tokens, labels, [g[i] for g in grads])
            total, counted = total + loss.sum(), counted + (labels >= 0).sum()
        (comp.compress_refresh if t % tau == 0 else comp.compress)(grads, errors, q, p)
        comp.decompress_msgd(None, None, moments, model.weights, mu, eta)
        losses.append(total / counted)
    return [float(x) for x in losses]


if __name__ == "__main__":
    for t, x in enumerate(run()):
        if t % 20 == 0:
            print("step %4d  loss %.4f" % (t, x))
