"""A block of experts and an output head that learn a teacher's distribution with PowerSGD+ (Algorithm 2).

    a = norm(x), r = a W_r^T, each token's `slots` largest of r with the weights softmax(these)
    expert e: h = silu(a W_g,e^T) * (a W_u,e^T), o = h W_d,e^T;   y = norm(x + sum over the token's experts of weight * o)
    loss = mean divergence of softmax(y W_o^T / T) from the teacher's distribution, of which the largest logits are known

x is a fixed table's row for each token, the teacher a fixed table of logits; a tenth of the tokens is masked.  Several workers have a batch
each; their gradients are averaged on the GPU by psgd_compress, the compressed update goes to psgd_decompress_msgd.

Between the linear layers, which are torch's, every step is the library's: psgd_norm and its gradients, psgd_expert_sort, _rows and _combine
with theirs, psgd_act_glu and psgd_act_store on the rows of all experts at once, psgd_act_wgrad on each expert's rows, psgd_head_distill_grad.
"""
from __future__ import annotations

from typing import List

from . import psgd


class Model:
    """Weights in fp32 with bf16 copies, activations in bf16, gradients of matrices in bf16, of the norms in fp32."""

    def __init__(self, tokens: int = 512, d: int = 256, hidden: int = 320, experts: int = 4, slots: int = 2, vocab: int = 1000, top: int = 16,
                 temperature: float = 1.0, seed: int = 1):
        import torch
        self.tokens, self.d, self.hidden, self.experts, self.slots, self.vocab = tokens, d, hidden, experts, slots, vocab
        self.temperature = temperature
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(seed)

        def randn(*shape, scale):
            return torch.randn(shape, generator=self.gen, device="cuda").mul_(scale)

        self.table = randn(vocab, d, scale=1.0).bfloat16()
        self.teacher, self.words = randn(vocab, vocab, scale=3.0).topk(top, 1)
        # gate, up and down of each expert, the router, the head
        self.shapes = [(hidden, d), (hidden, d), (d, hidden)] * experts + [(experts, d), (vocab, d)]
        self.weights = [randn(*s, scale=s[1] ** -0.5) for s in self.shapes]
        # weight and bias of both norms
        self.vectors = [torch.ones(d, device="cuda") if i % 2 == 0 else torch.zeros(d, device="cuda") for i in range(4)]
        self.sort, self.order = psgd.ExpertSort(tokens, slots, experts), psgd.expert_order_empty(tokens, slots, experts)
        rows = tokens * slots
        self.kept_gate, self.kept_up, self.kept_h = (psgd.act_empty(rows, hidden) for _ in range(3))
        self.kept_a = psgd.act_empty(rows, d)
        self.head = psgd.HeadDistill(tokens, d, vocab, top)
        self.norm_grad = psgd.NormGrad(tokens, d, psgd.PSGD_BF16, psgd.PSGD_F32)

    def batch(self):
        """Tokens and the teacher's entries for them (-1 where masked)."""
        import torch
        x = torch.randint(0, self.vocab, (self.tokens,), generator=self.gen, device="cuda")
        masked = torch.rand((self.tokens, 1), generator=self.gen, device="cuda") < 0.1
        return x, torch.where(masked, -1, self.words[x]), self.teacher[x]

    def gradients(self, tokens, index, teacher, out, vectors):
        """One forward and backward pass; the matrices' gradients into out, the norms' into vectors, the tokens' losses returned."""
        import torch
        w = [m.bfloat16() for m in self.weights]
        gate_w, up_w, down_w, router_w, head_w = w[:-2:3], w[1:-2:3], w[2:-2:3], w[-2], w[-1]
        t, d, rows, bf16 = self.tokens, self.d, self.tokens * self.slots, torch.bfloat16

        def empty(n, cols):
            return torch.empty((n, cols), dtype=bf16, device="cuda")

        x = self.table[tokens]
        a, stats = empty(t, d), torch.empty((t, 2), device="cuda")
        psgd.norm(x, self.vectors[0], self.vectors[1], a, stats)
        best, choice = (a.float() @ router_w.float().t()).topk(self.slots, 1)
        weight = torch.softmax(best, 1)
        self.sort.run(choice, self.order)
        first = self.order.offsets.tolist()             # (which rows are whose: torch's products want to know)
        parts = [slice(first[e], first[e + 1]) for e in range(self.experts)]
        xs, gate, up, h, o = empty(rows, d), empty(rows, self.hidden), empty(rows, self.hidden), empty(rows, self.hidden), empty(rows, d)
        psgd.expert_rows(a, self.order, xs)
        psgd.act_store(xs, self.kept_a)
        for e, p in enumerate(parts):
            torch.mm(xs[p], gate_w[e].t(), out=gate[p])
            torch.mm(xs[p], up_w[e].t(), out=up[p])
        psgd.act_glu(gate, up, h, self.kept_gate, self.kept_up)
        psgd.act_store(h, self.kept_h)
        for e, p in enumerate(parts):
            torch.mm(h[p], down_w[e].t(), out=o[p])
        mixed, total, y, stats_y = empty(t, d), empty(t, d), empty(t, d), torch.empty((t, 2), device="cuda")
        psgd.expert_combine(o, self.order, mixed, weight=weight)
        psgd.norm(x, self.vectors[2], self.vectors[3], y, stats_y, add=mixed, total=total)
        del xs, gate, up, h, x, mixed           # the backward pass takes the checkpoints

        loss = torch.empty(t, device="cuda")
        self.head.loss_grad(y, head_w, index, teacher, loss, y, out[-1], temperature=self.temperature)       # (dy in the place of y)
        self.norm_grad.run(y, total, self.vectors[2], stats_y, y, vectors[2], vectors[3])
        dweight, do = torch.empty_like(weight), o
        psgd.expert_combine_backward(y, o, self.order, do, weight=weight, dweight=dweight)                   # (in the place of o)
        dh, dxs = empty(rows, self.hidden), empty(rows, d)
        for e, p in enumerate(parts):
            torch.mm(do[p], down_w[e], out=dh[p])
        dgate, dup = empty(rows, self.hidden), empty(rows, self.hidden)
        psgd.act_glu_backward(self.kept_gate, self.kept_up, dh, dgate, dup)
        for e, p in enumerate(parts):
            n = p.stop - p.start
            torch.addmm(torch.mm(dgate[p], gate_w[e]), dup[p], up_w[e], out=dxs[p])
            into, down = psgd.WeightGrad(n, self.hidden, d), psgd.WeightGrad(n, d, self.hidden)
            into.run(dgate[p], self._part(self.kept_a, p), out[3 * e])
            into.run(dup[p], self._part(self.kept_a, p), out[3 * e + 1])
            down.run(do[p], self._part(self.kept_h, p), out[3 * e + 2])
        da = empty(t, d)
        psgd.expert_combine(dxs, self.order, da)
        # the softmax over the chosen, and the router
        dbest = weight * (dweight - (weight * dweight).sum(1, keepdim=True))
        dr = torch.zeros((t, self.experts), device="cuda").scatter_(1, choice, dbest)
        out[-2].copy_(dr.t() @ a.float())
        da += (dr @ router_w.float()).bfloat16()
        self.norm_grad.run(da, self.table[tokens], self.vectors[0], stats, da, vectors[0], vectors[1])
        return loss

    @staticmethod
    def _part(kept, p):
        return psgd.Act8(kept.codes[p], kept.scales[p], kept.cols)


def run(steps: int = 200, workers: int = 2, rank: int = 16, tau: int = 20, mu: float = 0.9, eta: float = 0.5, seed: int = 1) -> List[float]:
    """Mean losses of the counted tokens, step by step."""
    import torch
    model = Model(seed=seed)
    comp = psgd.Compressor([(r, c, min(rank, r, c), psgd.PSGD_BF16) for r, c in model.shapes], workers)
    grads = [[torch.empty(s, dtype=torch.bfloat16, device="cuda") for _ in range(workers)] for s in model.shapes]
    vectors = [[torch.empty_like(v) for v in model.vectors] for _ in range(workers)]
    errors, moments = ([torch.zeros(s, device="cuda") for s in model.shapes] for _ in range(2))
    ranks = [min(rank, *s) for s in model.shapes]
    q = [torch.randn((min(s), r), generator=model.gen, device="cuda") for s, r in zip(model.shapes, ranks)]
    p = [torch.zeros((max(s), r), device="cuda") for s, r in zip(model.shapes, ranks)]
    losses = []
    for t in range(steps):
        total, counted = 0.0, 0
        for i in range(workers):
            tokens, index, teacher = model.batch()
            loss = model.gradients(tokens, index, teacher, [g[i] for g in grads], vectors[i])
            total, counted = total + loss.sum(), counted + (index >= 0).any(1).sum()
        (comp.compress_refresh if t % tau == 0 else comp.compress)(grads, errors, q, p)
        comp.decompress_msgd(None, None, moments, model.weights, mu, eta)
        for v, g in zip(model.vectors, zip(*vectors)):
            v -= 0.1 * eta * sum(g) / workers
        losses.append(total / counted)
    return [float(x) for x in losses]


if __name__ == "__main__":
    for t, x in enumerate(run()):
        if t % 20 == 0:
            print("step %4d  loss %.4f" % (t, x))
