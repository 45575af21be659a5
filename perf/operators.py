"""The operators of a training step that stand on either side of the compressor's gradients, as cases that can be timed
and compared: the loss at the output head with the gradients it starts the backward pass with, activations kept in 8 bits
for the backward pass, and the weight gradients formed from them -- the matrices that psgd_compress takes.

Keys of a case:
  op      "head"   softmax cross entropy of X W^T against labels, without logits in memory; with grad, dX and dW as well
          "round"  an activation stored as an 8-bit checkpoint and restored
          "glu"    h = act(gate) * up (or act(gate)) with 8-bit checkpoints of its inputs, and the backward pass from them
          "wgrad"  G = dY^T X from dY and the 8-bit checkpoint of X
  dtype   "bf16" or "f32": activations, weights of the head and their gradients;  gtype: dW of the head, G of wgrad
  tokens  rows;  d, vocab: the head's matrix is vocab x d;  cols: features of an activation;  out, inp: G is out x inp
  masked  part of the tokens whose label is -100 (prompt and padding);  weights: per-token weights in place of the mean
  pad     elements by which the rows of the activations are longer than their columns, on top of the rounding up to 8

8-bit checkpoints: each row is cut into groups of 32 columns.  A group has a power of two 2^e as its scale, the smallest
with max|x| <= 127 * 2^e, and each element a whole number round(x / 2^e), ties to even.
"""
import math

import torch

own = False

GROUP = 32
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _head(tokens, d, vocab, dtype="bf16", gtype=None, grad=True, masked=0.0, weights=False, pad=0):
    return {"op": "head", "tokens": tokens, "d": d, "vocab": vocab, "dtype": dtype, "gtype": gtype or dtype, "grad": grad,
            "masked": masked, "weights": weights, "pad": pad}


def _round(tokens, cols, dtype="bf16", pad=0):
    return {"op": "round", "tokens": tokens, "cols": cols, "dtype": dtype, "pad": pad}


def _glu(tokens, cols, dtype="bf16", act="silu", gated=True, pad=0):
    return {"op": "glu", "tokens": tokens, "cols": cols, "dtype": dtype, "act": act, "gated": gated, "pad": pad}


def _wgrad(tokens, out, inp, dtype="bf16", gtype=None, pad=0):
    return {"op": "wgrad", "tokens": tokens, "out": out, "inp": inp, "dtype": dtype, "gtype": gtype or dtype, "pad": pad}


def listed():
    named = {
        # the head of a large model on a batch of packed sequences, prompts masked: the largest matrix products there are
        "head_8192x4096x64000_bf16": _head(8192, 4096, 64000, masked=0.1),
        # a middling model and batch, mean over all tokens
        "head_4096x2048x32000_bf16": _head(4096, 2048, 32000),
        # a short batch, odd vocabulary, weighted tokens, padded rows: the head's weight is most of the traffic
        "head_200x1024x10007_bf16": _head(200, 1024, 10007, masked=0.3, weights=True, pad=24),
        # fp32 training of a small model, odd sizes everywhere, most tokens masked
        "head_777x515x10007_f32": _head(777, 515, 10007, dtype="f32", masked=0.5),
        # scoring of a text: losses alone
        "loss_2048x4096x32000_bf16": _head(2048, 4096, 32000, grad=False),
        # scoring of one token
        "loss_1x4096x32000_bf16": _head(1, 4096, 32000, grad=False),
        # the checkpoint of a wide hidden layer
        "round_16384x11008_bf16": _round(16384, 11008),
        # a small one with odd sizes: launches and little else
        "round_37x515_f32": _round(37, 515, dtype="f32", pad=5),
        # the gated unit of a large model's block, forward and backward
        "glu_8192x11008_bf16": _glu(8192, 11008),
        # a plain activation between two small linear layers
        "glu_128x2050_f32": _glu(128, 2050, dtype="f32", act="gelu", gated=False),
        # the weight gradient of a large block's linear layer
        "wgrad_8192x11008x4096_bf16": _wgrad(8192, 11008, 4096),
        # one of few outputs from many tokens, gradient in fp32: the contraction is all there is to split
        "wgrad_9001x256x1032_bf16_f32": _wgrad(9001, 256, 1032, gtype="f32"),
    }
    return [{"name": name, **case} for name, case in named.items()]


def _log_uniform(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    most = work(listed()[0])
    while True:
        op = rng.choice(["head", "head", "round", "glu", "wgrad", "wgrad"])
        dtype = "bf16" if rng.random() < 0.75 else "f32"
        size = lambda low, high: _log_uniform(rng, low, high) if rng.random() < 0.5 else max(low, _log_uniform(rng, low, high) // 64 * 64)  # noqa: E731
        pad = rng.choice([0, 0, 8, 40])
        tokens = _log_uniform(rng, 1, 16384)
        if op == "head":
            case = _head(tokens, size(64, 4096), size(300, 64000), dtype, rng.choice([dtype, dtype, "f32"]), rng.random() < 0.7,
                         rng.choice([0.0, 0.1, 0.5, 0.9]), rng.random() < 0.3, pad)
        elif op == "round":
            case = _round(tokens, size(33, 11008), dtype, pad)
        elif op == "glu":
            case = _glu(tokens, size(33, 11008), dtype, rng.choice(["silu", "silu", "gelu"]), rng.random() < 0.7, pad)
        else:
            case = _wgrad(tokens, size(64, 11008), size(64, 11008), dtype, rng.choice([dtype, "f32"]), pad)
        w = work(case)
        # fp32 costs several times as much a product;  3072 is left out: no configuration here has it
        if w["flops"] * (6 if dtype == "f32" else 1) <= most["flops"] and w["bytes"] <= most["bytes"] and 3072 not in case.values():
            return case


def work(case):
    sx = 2 if case["dtype"] == "bf16" else 4
    t = case["tokens"]
    if case["op"] == "head":
        sg, d, v = 2 if case["gtype"] == "bf16" else 4, case["d"], case["vocab"]
        counted = max(1, round(t * (1.0 - case["masked"])))
        move = (counted * d + v * d) * sx + 12 * t
        if not case["grad"]:
            return {"bytes": move, "flops": 2 * counted * d * v}
        return {"bytes": move + t * d * sx + v * d * sg, "flops": 6 * counted * d * v}
    if case["op"] == "wgrad":
        sg, o, i = 2 if case["gtype"] == "bf16" else 4, case["out"], case["inp"]
        return {"bytes": t * (o * sx + i + -(-i // GROUP)) + o * i * sg, "flops": 2 * t * o * i}
    n, kept = t * case["cols"], t * (case["cols"] + -(-case["cols"] // GROUP))
    if case["op"] == "round":
        return {"bytes": 2 * n * sx + 2 * kept, "flops": 4 * n}
    inputs = 2 if case["gated"] else 1
    return {"bytes": n * sx * (inputs + 1) + n * sx * (1 + inputs) + 2 * inputs * kept, "flops": 30 * n}


# ---- inputs ----------------------------------------------------------------------------------------------------------

def _rows(x, dtype, pad=0):
    """The values in rows that are a multiple of 8 elements (plus pad, rounded likewise) apart, as a view of the columns."""
    rows, cols = x.shape
    ld = (cols + pad + 7) // 8 * 8
    buf = torch.zeros((rows, ld), dtype=dtype, device=x.device)
    buf[:, :cols] = x
    return buf[:, :cols]


def _empty(rows, cols, dtype):
    return torch.zeros((rows, (cols + 7) // 8 * 8), dtype=dtype, device="cuda")[:, :cols]


def _activations(rows, cols, gen):
    """Unit normal, with a few channels twenty times as large, as activations of trained networks have."""
    scale = torch.where(torch.rand(cols, generator=gen, device="cuda") < 0.01, 20.0, 1.0)
    return torch.randn((rows, cols), generator=gen, device="cuda") * scale


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op, t, dtype = case["op"], case["tokens"], TYPES[case["dtype"]]
    state = {"case": case}
    if op == "head":
        d, v = case["d"], case["vocab"]
        w = torch.randn((v, d), generator=gen, device="cuda").mul_(d ** -0.5)
        labels = torch.randint(0, v, (t,), generator=gen, device="cuda")
        # some tokens are as good as known, most are not: the label's logit is raised by 0 to 12
        sure = 12.0 * torch.rand((t, 1), generator=gen, device="cuda") ** 2
        x = torch.randn((t, d), generator=gen, device="cuda") + sure * w[labels]
        labels = torch.where(torch.rand(t, generator=gen, device="cuda") < case["masked"], -100, labels)
        state |= {"x": _rows(x, dtype, case["pad"]), "w": _rows(w, dtype), "labels": labels, "weight": None}
        if case["weights"]:
            state["weight"] = torch.rand(t, generator=gen, device="cuda").div_(t)
    elif op == "round":
        state["x"] = _rows(_activations(t, case["cols"], gen), dtype, case["pad"])
    elif op == "glu":
        state["gate"] = _rows(_activations(t, case["cols"], gen), dtype, case["pad"])
        state["up"] = _rows(_activations(t, case["cols"], gen), dtype, case["pad"]) if case["gated"] else None
        state["dh"] = _rows(torch.randn((t, case["cols"]), generator=gen, device="cuda").mul_(1e-3), dtype, case["pad"])
    else:
        state["dy"] = _rows(torch.randn((t, case["out"]), generator=gen, device="cuda").mul_(1e-3), dtype, case["pad"])
        x = _activations(t, case["inp"], gen).to(dtype)
        codes, scales = _quantise(x.float())
        ldc = (case["inp"] + 15) // 16 * 16
        state["codes"] = torch.zeros((t, ldc), dtype=torch.int8, device="cuda")
        state["codes"][:, :case["inp"]] = codes
        state["scales"] = scales
    if own:
        _plan(state)
    return state


def _plan(state):
    """What a program keeps beside its data: output buffers, checkpoints, the plan with its workspace."""
    from paper_2509_11254_amd import psgd
    case = state["case"]
    op, t, dtype = case["op"], case["tokens"], TYPES[case["dtype"]]
    code = lambda name: psgd.PSGD_BF16 if case[name] == "bf16" else psgd.PSGD_F32  # noqa: E731
    state["psgd"] = psgd
    if op == "head":
        d, v = case["d"], case["vocab"]
        state["loss"] = torch.zeros(t, device="cuda")
        state["plan"] = psgd.HeadLoss(t, d, v, code("dtype"), code("gtype"), grad=case["grad"])
        if case["grad"]:
            state["dx"], state["dw"] = _empty(t, d, dtype), _empty(v, d, TYPES[case["gtype"]])
    elif op == "round":
        state["kept"] = psgd.act_empty(t, case["cols"])
        state["y"] = _empty(t, case["cols"], dtype)
    elif op == "glu":
        state["kept_gate"], state["kept_up"] = psgd.act_empty(t, case["cols"]), psgd.act_empty(t, case["cols"])
        state["h"], state["dgate"], state["dup"] = (_empty(t, case["cols"], dtype), _empty(t, case["cols"], dtype),
                                                    _empty(t, case["cols"], dtype))
        state["act"] = psgd.PSGD_SILU if case["act"] == "silu" else psgd.PSGD_GELU
    else:
        state["kept"] = psgd.Act8(state["codes"], state["scales"], case["inp"])
        state["plan"] = psgd.WeightGrad(t, case["out"], case["inp"], code("dtype"), code("gtype"))
        state["g"] = _empty(case["out"], case["inp"], TYPES[case["gtype"]])


# ---- one pass --------------------------------------------------------------------------------------------------------

def run(state):
    case = state["case"]
    if own:
        return {"head": _own_head, "round": _own_round, "glu": _own_glu, "wgrad": _own_wgrad}[case["op"]](state)
    return {"head": _plain_head, "round": _plain_round, "glu": _plain_glu, "wgrad": _plain_wgrad}[case["op"]](state)


def _own_head(s):
    if not s["case"]["grad"]:
        s["plan"].loss(s["x"], s["w"], s["labels"], s["loss"])
        return {"loss": s["loss"]}
    s["plan"].loss_grad(s["x"], s["w"], s["labels"], s["loss"], s["dx"], s["dw"], weight=s["weight"])
    return {"loss": s["loss"], "dx": s["dx"], "dw": s["dw"]}


def _own_round(s):
    s["psgd"].act_store(s["x"], s["kept"])
    s["psgd"].act_restore(s["kept"], s["y"])
    return {"y": s["y"]}


def _own_glu(s):
    if s["case"]["gated"]:
        s["psgd"].act_glu(s["gate"], s["up"], s["h"], s["kept_gate"], s["kept_up"], act=s["act"])
        s["psgd"].act_glu_backward(s["kept_gate"], s["kept_up"], s["dh"], s["dgate"], s["dup"], act=s["act"])
        return {"h": s["h"], "dgate": s["dgate"], "dup": s["dup"]}
    s["psgd"].act_glu(s["gate"], None, s["h"], s["kept_gate"], None, act=s["act"])
    s["psgd"].act_glu_backward(s["kept_gate"], None, s["dh"], s["dgate"], None, act=s["act"])
    return {"h": s["h"], "dgate": s["dgate"]}


def _own_wgrad(s):
    s["plan"].run(s["dy"], s["kept"], s["g"])
    return {"g": s["g"]}


def _quantise(x):
    """Whole numbers (rows x cols, int8) and scales (rows x groups, uint8: e + 127) of fp32 values."""
    rows, cols = x.shape
    groups = -(-cols // GROUP)
    g = torch.nn.functional.pad(x, (0, groups * GROUP - cols)).view(rows, groups, GROUP)
    most = g.abs().amax(2)
    fraction, exponent = torch.frexp(most)                   # most = fraction * 2^exponent, fraction in [1/2, 1)
    e = torch.where(fraction <= 127.0 / 128.0, exponent - 7, exponent - 6).clamp(-126, 121)
    codes = torch.round(torch.ldexp(g, -e.unsqueeze(2))).clamp(-127, 127)
    scales = torch.where(most > 0, e + 127, 0).to(torch.uint8)
    return codes.view(rows, groups * GROUP)[:, :cols].to(torch.int8), scales


def _values(codes, scales):
    """The fp32 values that whole numbers and scales stand for."""
    power = torch.ldexp(torch.ones((), device=codes.device), scales.int() - 127)
    return codes.float() * power.repeat_interleave(GROUP, 1)[:, :codes.shape[1]]


def _plain_head(s):
    x, w, labels = s["x"].float(), s["w"].float(), s["labels"]
    counted = labels >= 0
    at = labels.clamp(min=0).unsqueeze(1)
    logits = x @ w.t()
    most = logits.amax(1, keepdim=True)
    lse = most + torch.log(torch.exp(logits - most).sum(1, keepdim=True))
    loss = torch.where(counted, (lse - logits.gather(1, at)).squeeze(1), 0.0)
    if not s["case"]["grad"]:
        return {"loss": loss}
    weight = s["weight"] if s["weight"] is not None else torch.ones_like(loss) / counted.sum().clamp(min=1)
    p = torch.exp(logits - lse)
    p.scatter_add_(1, at, torch.full_like(lse, -1.0))
    p *= torch.where(counted, weight, 0.0).unsqueeze(1)
    return {"loss": loss, "dx": (p @ w).to(s["x"].dtype), "dw": (p.t() @ x).to(TYPES[s["case"]["gtype"]])}


def _plain_round(s):
    return {"y": _values(*_quantise(s["x"].float())).to(s["x"].dtype)}


def _normal(x):
    """The standard normal distribution function and its density."""
    return 0.5 * (1.0 + torch.erf(x * math.sqrt(0.5))), torch.exp(-0.5 * x * x) * (1.0 / math.sqrt(2.0 * math.pi))


def _act(x, act):
    return x / (1.0 + torch.exp(-x)) if act == "silu" else x * _normal(x)[0]


def _slope(x, act):
    if act == "silu":
        sig = 1.0 / (1.0 + torch.exp(-x))
        return sig * (1.0 + x * (1.0 - sig))
    cdf, density = _normal(x)
    return cdf + x * density


def _plain_glu(s):
    act, dtype, dh = s["case"]["act"], s["gate"].dtype, s["dh"].float()
    gate = s["gate"].float()
    gate8 = _values(*_quantise(gate))
    if not s["case"]["gated"]:
        return {"h": _act(gate, act).to(dtype), "dgate": (dh * _slope(gate8, act)).to(dtype)}
    up = s["up"].float()
    up8 = _values(*_quantise(up))
    return {"h": (_act(gate, act) * up).to(dtype), "dgate": (dh * up8 * _slope(gate8, act)).to(dtype),
            "dup": (dh * _act(gate8, act)).to(dtype)}


def _plain_wgrad(s):
    x = _values(s["codes"][:, :s["case"]["inp"]], s["scales"])
    return {"g": (s["dy"].float().t() @ x).to(TYPES[s["case"]["gtype"]])}


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------

def _exact_kept(x):
    """What an 8-bit checkpoint of x stands for, in 64 bits, group by group of 32 columns."""
    x = x.double()
    rows, cols = x.shape
    short = -cols % GROUP
    g = torch.cat([x, x.new_zeros((rows, short))], 1).reshape(rows, -1, GROUP)
    most = g.abs().max(2, keepdim=True).values
    e = torch.ceil(torch.log2(torch.where(most > 0, most, 1.0) / 127.0))
    # the logarithm may be off by its last bit where most is 127 times a power of two: the definition decides
    e = torch.where(most > 127.0 * 2.0 ** e, e + 1, torch.where(most <= 127.0 * 2.0 ** (e - 1), e - 1, e)).clamp(-126, 121)
    return (torch.round(g / 2.0 ** e).clamp(-127, 127) * 2.0 ** e).reshape(rows, -1)[:, :cols]


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "round":
        return {"y": _exact_kept(s["x"])}
    if case["op"] == "wgrad":
        scale = (2.0 ** (s["scales"].double() - 127.0)).repeat_interleave(GROUP, 1)[:, :case["inp"]]
        return {"g": torch.mm(s["dy"].double().t().contiguous(), s["codes"][:, :case["inp"]].double() * scale)}
    if case["op"] == "glu":
        return _exact_glu(case, s)
    x, w, labels = s["x"].double(), s["w"].double(), s["labels"]
    keep = (labels >= 0).nonzero().squeeze(1)
    xk, at = x[keep], labels[keep]
    logits = torch.mm(xk, w.t())
    lse = torch.logsumexp(logits, 1)
    loss = torch.zeros(x.shape[0], dtype=torch.float64, device="cuda")
    loss[keep] = lse - logits[torch.arange(len(keep), device="cuda"), at]
    if not case["grad"]:
        return {"loss": loss}
    p = torch.exp_(logits.sub_(lse.unsqueeze(1)))
    p[torch.arange(len(keep), device="cuda"), at] -= 1.0
    p *= s["weight"].double()[keep].unsqueeze(1) if s["weight"] is not None else 1.0 / max(1, len(keep))
    dx = torch.zeros_like(x)
    dx[keep] = torch.mm(p, w)
    return {"loss": loss, "dx": dx, "dw": torch.mm(p.t(), xk)}


def _exact_glu(case, s):
    def value(x):
        return x * torch.special.ndtr(x) if case["act"] == "gelu" else x * torch.sigmoid(x)

    def slope(x):
        if case["act"] == "gelu":
            return torch.special.ndtr(x) + x * torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)
        return torch.sigmoid(x) + x * torch.sigmoid(x) * torch.sigmoid(-x)

    gate, dh = s["gate"].double(), s["dh"].double()
    gate8 = _exact_kept(gate)
    if not case["gated"]:
        return {"h": value(gate), "dgate": dh * slope(gate8)}
    up = s["up"].double()
    return {"h": value(gate) * up, "dgate": dh * _exact_kept(up) * slope(gate8), "dup": dh * value(gate8)}
