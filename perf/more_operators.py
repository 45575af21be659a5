"""Operators of a training step that stand beside the output head's loss, the gated units and their checkpoints, as cases that can be timed and
compared: layer norms, distillation from a teacher's top logits at the output head, and tokens sorted by expert and back.

Keys of a case:
  op      "norm"      y = (s - mean) / sqrt(variance + eps) * weight + bias of s = x, or s = x + add; with grad, the backward pass as well
          "distill"   Kullback-Leibler divergence of softmax(X W^T / T) from a teacher's distribution, of which the largest logits are known, without
                      logits in memory; with grad, dX and dW as well
          "dispatch"  tokens sorted by the experts they chose, their rows laid out in that order, and the gradient of the rows
          "combine"   the experts' rows brought back to their tokens and added up with weights, forward and backward
  dtype   "bf16" or "f32": activations, their gradients, weights of the head;  gtype: dW of the head, gradients of the norm's weight and bias
  wtype   the norm's weight and bias
  rows, cols: an activation;  add: with a second addend, and in the backward pass a gradient that comes past the norm
  tokens, d, vocab, top: the head's matrix is vocab x d, a teacher's entries are tokens x top;  ttype: the teacher's logits
  ragged  part of the entries that a token lacks (index -1);  masked: part of the tokens without any (prompt and padding)
  weights per-token weights in place of the mean;  temperature: T
  slots, experts: each token chooses `slots` of `experts`;  dropped: part of the choices that are -1;  skew: how unequal the experts are
  pad     elements by which the rows of the activations are longer than their columns, on top of the rounding up to 8
"""
import math

import torch

own = False

EPS = 1e-5
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _norm(rows, cols, dtype="bf16", wtype=None, gtype=None, grad=True, add=False, pad=0):
    return {"op": "norm", "rows": rows, "cols": cols, "dtype": dtype, "wtype": wtype or dtype, "gtype": gtype or dtype, "grad": grad,
            "add": add, "pad": pad}


def _distill(tokens, d, vocab, top, dtype="bf16", gtype=None, ttype="f32", grad=True, temperature=1.0, ragged=0.0, masked=0.0, weights=False, pad=0):
    return {"op": "distill", "tokens": tokens, "d": d, "vocab": vocab, "top": top, "dtype": dtype, "gtype": gtype or dtype, "ttype": ttype,
            "grad": grad, "temperature": temperature, "ragged": ragged, "masked": masked, "weights": weights, "pad": pad}


def _dispatch(tokens, cols, slots, experts, dtype="bf16", dropped=0.0, skew=1.0, pad=0):
    return {"op": "dispatch", "tokens": tokens, "cols": cols, "slots": slots, "experts": experts, "dtype": dtype, "dropped": dropped,
            "skew": skew, "pad": pad}


def _combine(tokens, cols, slots, experts, dtype="bf16", dropped=0.0, skew=1.0, pad=0):
    return _dispatch(tokens, cols, slots, experts, dtype, dropped, skew, pad) | {"op": "combine"}


def listed():
    named = {
        # the residual stream of a large model's block on a batch of packed sequences: added up, normalised, and the way back
        "norm_16384x4096_bf16_add": _norm(16384, 4096, add=True),
        # a small model in fp32, odd width
        "norm_1000x515_f32": _norm(1000, 515, dtype="f32", pad=5),
        # the last norm of one token that is scored: a launch and little else
        "norm_1x4096_bf16_forward": _norm(1, 4096, wtype="f32", grad=False),
        # the head of a large model against a teacher's 64 largest logits, prompts masked: the largest matrix products there are
        "distill_8192x4096x64000_top64_bf16": _distill(8192, 4096, 64000, 64, masked=0.1),
        # a middling model and batch at a higher temperature, teachers that stop at a part of the probability
        "distill_2048x2048x32000_top20_bf16": _distill(2048, 2048, 32000, 20, ttype="bf16", temperature=2.0, ragged=0.3),
        # a short batch, odd vocabulary, weighted tokens, padded rows, dW in fp32
        "distill_200x1024x10007_top100_bf16_f32": _distill(200, 1024, 10007, 100, gtype="f32", masked=0.3, weights=True, pad=24),
        # fp32 training of a small model, odd sizes everywhere
        "distill_333x515x10007_top8_f32": _distill(333, 515, 10007, 8, dtype="f32", masked=0.5),
        # one token scored against its teacher
        "distill_1x4096x32000_top64_bf16_forward": _distill(1, 4096, 32000, 64, grad=False),
        # many small experts, eight to a token, on a large batch
        "dispatch_16384x2048_8of64_bf16": _dispatch(16384, 2048, 8, 64),
        # few large experts on a short batch, some choices over an expert's capacity and dropped
        "dispatch_200x1032_2of8_f32": _dispatch(200, 1032, 2, 8, dtype="f32", dropped=0.1, skew=3.0),
        "combine_16384x2048_8of64_bf16": _combine(16384, 2048, 8, 64),
        "combine_333x515_3of16_bf16": _combine(333, 515, 3, 16, dropped=0.1, skew=3.0, pad=8),
    }
    return [{"name": name, **case} for name, case in named.items()]


def _log_uniform(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    most = {what: max(work(case)[what] for case in listed()) for what in ("bytes", "flops")}
    while True:
        op = rng.choice(["norm", "norm", "distill", "distill", "dispatch", "combine"])
        dtype = "bf16" if rng.random() < 0.75 else "f32"
        size = lambda low, high: _log_uniform(rng, low, high) if rng.random() < 0.5 else max(low, _log_uniform(rng, low, high) // 64 * 64)  # noqa: E731
        pad = rng.choice([0, 0, 8, 40])
        tokens = _log_uniform(rng, 1, 16384)
        if op == "norm":
            case = _norm(tokens, size(33, 11008), dtype, rng.choice([dtype, "f32"]), rng.choice([dtype, "f32"]), rng.random() < 0.7,
                         rng.random() < 0.5, pad)
        elif op == "distill":
            vocab = size(300, 64000)
            case = _distill(tokens, size(64, 4096), vocab, _log_uniform(rng, 1, 200), dtype, rng.choice([dtype, dtype, "f32"]),
                            rng.choice(["f32", "bf16"]), rng.random() < 0.7, rng.choice([1.0, 1.0, 0.5, 2.0, 4.0]), rng.choice([0.0, 0.3]),
                            rng.choice([0.0, 0.1, 0.5, 0.9]), rng.random() < 0.3, pad)
        else:
            experts = _log_uniform(rng, 2, 256)
            make = _dispatch if op == "dispatch" else _combine
            case = make(tokens, size(33, 8192), min(experts, _log_uniform(rng, 1, 16)), experts, dtype, rng.choice([0.0, 0.1]),
                        rng.choice([1.0, 3.0]), pad)
        w = work(case)
        # fp32 costs several times as much a product
        if w["flops"] * (6 if dtype == "f32" else 1) <= most["flops"] and w["bytes"] <= most["bytes"]:
            return case


def work(case):
    size = lambda name: 2 if case[name] == "bf16" else 4  # noqa: E731
    sx, op = size("dtype"), case["op"]
    if op == "norm":
        n, one, more = case["rows"] * case["cols"] * sx, case["cols"], 1 if case["add"] else 0
        move = n * (2 + 2 * more) + 2 * one * size("wtype")
        if case["grad"]:            # dy, s, the gradient past the norm; dx
            move += n * (3 + more) + one * (size("wtype") + 2 * size("gtype")) + 16 * case["rows"]
        return {"bytes": move, "flops": case["rows"] * one * (22 if case["grad"] else 8)}
    if op == "distill":
        t, d, v = case["tokens"], case["d"], case["vocab"]
        counted = max(1, round(t * (1.0 - case["masked"])))
        move = (counted * d + v * d) * sx + t * case["top"] * (8 + size("ttype")) + 4 * t
        if not case["grad"]:
            return {"bytes": move, "flops": 2 * counted * d * v}
        return {"bytes": move + t * d * sx + v * d * size("gtype"), "flops": 6 * counted * d * v}
    entries = case["tokens"] * case["slots"]
    row, kept = case["cols"] * sx, max(1, round(entries * (1.0 - case["dropped"])))
    if op == "dispatch":            # choices in, places and order out; rows out, gradients of rows in
        return {"bytes": 16 * entries + 2 * (case["tokens"] + kept) * row, "flops": kept * case["cols"]}
    return {"bytes": 2 * (case["tokens"] + kept) * row + kept * row + 12 * entries, "flops": 5 * kept * case["cols"]}


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


def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


def _activations(rows, cols, gen):
    """A residual stream: unit normal, a few channels twenty times as large and away from zero, as in trained networks."""
    large = torch.rand(cols, generator=gen, device="cuda") < 0.01
    return _randn(gen, rows, cols) * torch.where(large, 20.0, 1.0) + torch.where(large, 30.0, 0.2) * _randn(gen, cols)


def _choices(case, gen):
    """Each token's experts, all different, the likely ones more often; -1: dropped."""
    t, e = case["tokens"], case["experts"]
    favour = case["skew"] * torch.rand(e, generator=gen, device="cuda")
    noise = -torch.log(-torch.log(torch.rand((t, e), generator=gen, device="cuda").clamp(1e-7, 1 - 1e-7)))
    choice = (favour + noise).topk(case["slots"], 1).indices
    return torch.where(torch.rand(choice.shape, generator=gen, device="cuda") < case["dropped"], -1, choice).contiguous()


def _teacher(case, gen):
    """Indices, all different in a token, low ones (frequent words) more often; logits that fall off; -1 where there is no entry."""
    t, v = case["tokens"], case["vocab"]
    k = min(case["top"], v)
    u = torch.rand((t, k), generator=gen, device="cuda") ** 3
    index = (u * (v - k + 1)).long().clamp(0, v - k).sort(1).values + torch.arange(k, device="cuda")
    index = index.gather(1, torch.rand((t, k), generator=gen, device="cuda").argsort(1))
    fall = 2.0 * torch.log1p(torch.arange(k, device="cuda").float())
    logits = 20.0 + 4.0 * _randn(gen, t, 1) - fall * (0.5 + torch.rand((t, 1), generator=gen, device="cuda")) + 0.3 * _randn(gen, t, k)
    first = index[:, :1].clone()
    # a token keeps its first entries, as many as hold a part of the probability
    left = torch.ceil(k * (1.0 - case["ragged"] * 2 * torch.rand((t, 1), generator=gen, device="cuda"))).clamp(min=1)
    gone = torch.arange(k, device="cuda") >= left
    index = torch.where(gone | (torch.rand((t, 1), generator=gen, device="cuda") < case["masked"]), -1, index)
    return index, logits.to(TYPES[case["ttype"]]), first


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op, dtype = case["op"], TYPES[case["dtype"]]
    state = {"case": case}
    if op == "norm":
        rows, cols = case["rows"], case["cols"]
        state["x"] = _rows(_activations(rows, cols, gen), dtype, case["pad"])
        state["add"] = _rows(_randn(gen, rows, cols), dtype, case["pad"]) if case["add"] else None
        state["weight"] = (1.0 + 0.2 * _randn(gen, cols)).to(TYPES[case["wtype"]])
        state["bias"] = (0.1 * _randn(gen, cols)).to(TYPES[case["wtype"]])
        if case["grad"]:
            state["dy"] = _rows(_randn(gen, rows, cols).mul_(1e-3), dtype, case["pad"])
            state["dtotal"] = _rows(_randn(gen, rows, cols).mul_(1e-3), dtype, case["pad"]) if case["add"] else None
    elif op == "distill":
        t, d, v = case["tokens"], case["d"], case["vocab"]
        w = _randn(gen, v, d).mul_(d ** -0.5)
        index, teacher, first = _teacher(case, gen)
        # a student that knows the teacher's first word of some tokens well
        x = _randn(gen, t, d) + 12.0 * torch.rand((t, 1), generator=gen, device="cuda") ** 2 * w[first[:, 0]]
        state |= {"x": _rows(x, dtype, case["pad"]), "w": _rows(w, dtype), "index": index, "teacher": teacher, "weight": None}
        if case["weights"]:
            state["weight"] = torch.rand(t, generator=gen, device="cuda").div_(t)
    else:
        t, slots, cols = case["tokens"], case["slots"], case["cols"]
        state["choice"] = _choices(case, gen)
        if op == "dispatch":
            state["x"] = _rows(_activations(t, cols, gen), dtype, case["pad"])
            state["dxs"] = _rows(_randn(gen, t * slots, cols).mul_(1e-3), dtype)
        else:
            state["ys"] = _rows(_randn(gen, t * slots, cols), dtype)
            state["dy"] = _rows(_randn(gen, t, cols).mul_(1e-3), dtype, case["pad"])
            state["weight"] = torch.softmax(2.0 * _randn(gen, t, slots), 1)
            state["place"], state["order"], state["offsets"] = _sorted(state["choice"], case["experts"])
    if own:
        _plan(state)
    return state


def _plan(state):
    """What a program keeps beside its data: output buffers, statistics, the plan with its workspace."""
    from paper_2509_11254_amd import psgd
    case = state["case"]
    op, dtype = case["op"], TYPES[case["dtype"]]
    code = lambda name: psgd.PSGD_BF16 if case[name] == "bf16" else psgd.PSGD_F32  # noqa: E731
    state["psgd"] = psgd
    if op == "norm":
        rows, cols = case["rows"], case["cols"]
        state["y"] = _empty(rows, cols, dtype)
        state["total"] = _empty(rows, cols, dtype) if case["add"] else None
        state["stats"] = torch.zeros((rows, 2), device="cuda") if case["grad"] else None
        if case["grad"]:
            state["plan"] = psgd.NormGrad(rows, cols, code("dtype"), code("wtype"), code("gtype"))
            state["dx"] = _empty(rows, cols, dtype)
            state["dweight"], state["dbias"] = (torch.zeros(cols, dtype=TYPES[case["gtype"]], device="cuda") for _ in range(2))
    elif op == "distill":
        t, d, v = case["tokens"], case["d"], case["vocab"]
        state["loss"] = torch.zeros(t, device="cuda")
        state["plan"] = psgd.HeadDistill(t, d, v, state["index"].shape[1], code("dtype"), code("gtype"), grad=case["grad"])
        if case["grad"]:
            state["dx"], state["dw"] = _empty(t, d, dtype), _empty(v, d, TYPES[case["gtype"]])
    else:
        t, slots, cols = case["tokens"], case["slots"], case["cols"]
        if op == "dispatch":
            state["sorted"] = psgd.expert_order_empty(t, slots, case["experts"])
            state["plan"] = psgd.ExpertSort(t, slots, case["experts"])
            state["xs"], state["dx"] = _empty(t * slots, cols, dtype), _empty(t, cols, dtype)
        else:
            state["sorted"] = psgd.ExpertOrder(state["place"], state["order"], state["offsets"])
            state["y"], state["dys"] = _empty(t, cols, dtype), _empty(t * slots, cols, dtype)
            state["dweight"] = torch.zeros((t, slots), device="cuda")


# ---- one pass --------------------------------------------------------------------------------------------------------

def run(state):
    op = state["case"]["op"]
    if own:
        return {"norm": _own_norm, "distill": _own_distill, "dispatch": _own_dispatch, "combine": _own_combine}[op](state)
    return {"norm": _plain_norm, "distill": _plain_distill, "dispatch": _plain_dispatch, "combine": _plain_combine}[op](state)


def _own_norm(s):
    s["psgd"].norm(s["x"], s["weight"], s["bias"], s["y"], s["stats"], eps=EPS, add=s["add"], total=s["total"])
    out = {"y": s["y"]}
    if s["case"]["add"]:
        out["total"] = s["total"]
    if s["case"]["grad"]:
        s["plan"].run(s["dy"], s["x"] if s["add"] is None else s["total"], s["weight"], s["stats"], s["dx"], s["dweight"], s["dbias"],
                      dtotal=s["dtotal"])
        out |= {"dx": s["dx"], "dweight": s["dweight"], "dbias": s["dbias"]}
    return out


def _own_distill(s):
    case = s["case"]
    if not case["grad"]:
        s["plan"].loss(s["x"], s["w"], s["index"], s["teacher"], s["loss"], temperature=case["temperature"])
        return {"loss": s["loss"]}
    s["plan"].loss_grad(s["x"], s["w"], s["index"], s["teacher"], s["loss"], s["dx"], s["dw"], temperature=case["temperature"],
                        weight=s["weight"])
    return {"loss": s["loss"], "dx": s["dx"], "dw": s["dw"]}


def _own_dispatch(s):
    s["plan"].run(s["choice"], s["sorted"])
    s["psgd"].expert_rows(s["x"], s["sorted"], s["xs"])
    s["psgd"].expert_combine(s["dxs"], s["sorted"], s["dx"])
    return {"place": s["sorted"].place, "order": s["sorted"].order, "offsets": s["sorted"].offsets, "xs": s["xs"], "dx": s["dx"]}


def _own_combine(s):
    s["psgd"].expert_combine(s["ys"], s["sorted"], s["y"], weight=s["weight"])
    s["psgd"].expert_combine_backward(s["dy"], s["ys"], s["sorted"], s["dys"], weight=s["weight"], dweight=s["dweight"])
    return {"y": s["y"], "dys": s["dys"], "dweight": s["dweight"]}


def _plain_norm(s):
    case, dtype = s["case"], s["x"].dtype
    x = s["x"].float()
    out = {}
    if case["add"]:
        out["total"] = (x + s["add"].float()).to(dtype)
        x = out["total"].float()
    mean = x.mean(1, keepdim=True)
    x = x - mean
    r = 1.0 / torch.sqrt((x * x).mean(1, keepdim=True) + EPS)
    x = x * r
    w = s["weight"].float()
    out["y"] = (x * w + s["bias"].float()).to(dtype)
    if case["grad"]:
        dy = s["dy"].float()
        g = dy * w
        dx = r * (g - g.mean(1, keepdim=True) - x * (g * x).mean(1, keepdim=True))
        if case["add"]:
            dx = dx + s["dtotal"].float()
        g_type = TYPES[case["gtype"]]
        out |= {"dx": dx.to(dtype), "dweight": (dy * x).sum(0).to(g_type), "dbias": dy.sum(0).to(g_type)}
    return out


def _plain_distill(s):
    case = s["case"]
    x, w, index, inverse = s["x"].float(), s["w"].float(), s["index"], 1.0 / case["temperature"]
    there = index >= 0
    counted = there.any(1)
    # (a token without entries has one of its own, so that no row is empty)
    z = torch.where(there, s["teacher"].float() * inverse, -math.inf)
    z = torch.where(counted.unsqueeze(1), z, 0.0)
    z = z - z.amax(1, keepdim=True)
    log_q = z - torch.log(torch.exp(z).sum(1, keepdim=True))
    q = torch.where(there, torch.exp(log_q), 0.0)
    at = index.clamp(min=0)
    logits = x @ w.t()
    logits *= inverse
    most = logits.amax(1, keepdim=True)
    lse = most + torch.log(torch.exp(logits - most).sum(1, keepdim=True))
    log_p = logits.gather(1, at) - lse
    loss = torch.where(there, q * (torch.where(there, log_q, 0.0) - log_p), 0.0).sum(1)
    if not case["grad"]:
        return {"loss": loss}
    weight = s["weight"] if s["weight"] is not None else torch.ones_like(loss) / counted.sum().clamp(min=1)
    p = torch.exp_(logits.sub_(lse))
    p.scatter_add_(1, at, -q)
    p *= torch.where(counted, weight, 0.0).unsqueeze(1) * inverse
    return {"loss": loss, "dx": (p @ w).to(s["x"].dtype), "dw": (p.t() @ x).to(TYPES[case["gtype"]])}


def _sorted(choice, experts):
    """Where each choice's row goes (-1: dropped), which choice each row is (-1 behind the last), and each expert's first row."""
    flat = choice.reshape(-1)
    key = torch.where(flat >= 0, flat, experts)
    key, order = torch.sort(key, stable=True)
    rows = torch.arange(len(flat), device="cuda")
    place = torch.empty_like(order)
    place[order] = torch.where(key < experts, rows, -1)
    offsets = torch.searchsorted(key, torch.arange(experts + 1, device="cuda"))
    return place.int().view(choice.shape), torch.where(key < experts, order, -1).int(), offsets.int()


def _back(rows, place, weight):
    """Each token's sum of its rows, in 32 bits."""
    there = place >= 0
    picked = rows[place.clamp(min=0).long().view(-1)].float().view(*place.shape, rows.shape[1])
    return (picked * torch.where(there, weight, 0.0).unsqueeze(2)).sum(1)


def _plain_dispatch(s):
    case = s["case"]
    place, order, offsets = _sorted(s["choice"], case["experts"])
    token = order.clamp(min=0).long() // case["slots"]
    xs = torch.where((order >= 0).unsqueeze(1), s["x"][token], 0.0)
    dx = _back(s["dxs"], place, torch.ones((), device="cuda"))
    return {"place": place, "order": order, "offsets": offsets, "xs": xs, "dx": dx.to(s["x"].dtype)}


def _plain_combine(s):
    place, weight, dtype = s["place"], s["weight"], s["ys"].dtype
    y = _back(s["ys"], place, weight).to(dtype)
    order, slots = s["order"].long(), s["case"]["slots"]
    there = (order >= 0).unsqueeze(1)
    dy = s["dy"][order.clamp(min=0) // slots].float()
    dys = torch.where(there, dy * weight.view(-1)[order.clamp(min=0)].unsqueeze(1), 0.0).to(dtype)
    dots = (dy * s["ys"].float()).sum(1)
    dweight = torch.where(place >= 0, dots[place.clamp(min=0).long()], 0.0)
    return {"y": y, "dys": dys, "dweight": dweight}


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------

def exact(case, seed):
    return {"norm": _exact_norm, "distill": _exact_distill, "dispatch": _exact_dispatch, "combine": _exact_combine}[case["op"]](case, prepare(case, seed))


def _exact_norm(case, s):
    out = {}
    x = s["x"].double()
    if case["add"]:
        out["total"] = x + s["add"].double()
        x = out["total"].to(s["x"].dtype).double()         # what is normalised is the sum as it is kept
    w = s["weight"].double()
    sd = torch.sqrt(x.var(1, unbiased=False, keepdim=True) + EPS)
    unit = (x - x.mean(1, keepdim=True)) / sd
    out["y"] = torch.addcmul(s["bias"].double(), unit, w)
    if case["grad"]:
        dy, n = s["dy"].double(), case["cols"]
        g = dy * w
        out["dx"] = (n * g - g.sum(1, keepdim=True) - unit * (g * unit).sum(1, keepdim=True)) / (n * sd)
        if case["add"]:
            out["dx"] += s["dtotal"].double()
        out["dweight"], out["dbias"] = (dy * unit).sum(0), dy.sum(0)
    return out


def _exact_distill(case, s):
    x, w, index = s["x"].double(), s["w"].double(), s["index"]
    keep = (index >= 0).any(1).nonzero().squeeze(1)
    index, teacher = index[keep], s["teacher"][keep].double() / case["temperature"]
    teacher[index < 0] = -math.inf
    q = torch.softmax(teacher, 1)
    log_p = torch.mm(x[keep], w.t()).div_(case["temperature"])
    log_p -= torch.logsumexp(log_p, 1, keepdim=True)
    loss = torch.zeros(x.shape[0], dtype=torch.float64, device="cuda")
    cross = (q * log_p.gather(1, index.clamp(min=0))).sum(1)
    loss[keep] = torch.special.xlogy(q, q).sum(1) - cross
    if not case["grad"]:
        return {"loss": loss}
    d = log_p.exp_()
    d.scatter_add_(1, index.clamp(min=0), -q)
    c = s["weight"].double()[keep] if s["weight"] is not None else torch.full((len(keep),), 1.0 / max(1, len(keep)), dtype=torch.float64, device="cuda")
    d *= (c / case["temperature"]).unsqueeze(1)
    dx = torch.zeros_like(x)
    dx[keep] = torch.mm(d, w)
    return {"loss": loss, "dx": dx, "dw": torch.mm(d.t(), x[keep])}


def _exact_sum(case, rows, place, weight):
    total = torch.zeros((case["tokens"], case["cols"]), dtype=torch.float64, device="cuda")
    for slot in range(case["slots"]):
        t = (place[:, slot] >= 0).nonzero().squeeze(1)
        total[t] += weight[t, slot].double().unsqueeze(1) * rows[place[t, slot].long()].double()
    return total


def _exact_dispatch(case, s):
    # (whole numbers have no other value than the plain form's)
    place, order, offsets = _sorted(s["choice"], case["experts"])
    xs = torch.zeros((case["tokens"] * case["slots"], case["cols"]), dtype=torch.float64, device="cuda")
    n = int(offsets[-1])
    xs[:n] = s["x"].double()[order[:n].long() // case["slots"]]
    return {"place": place, "order": order, "offsets": offsets, "xs": xs,
            "dx": _exact_sum(case, s["dxs"], place, torch.ones((case["tokens"], case["slots"]), device="cuda"))}


def _exact_combine(case, s):
    place, weight = s["place"], s["weight"].double()
    dy, dys = s["dy"].double(), torch.zeros(s["ys"].shape, dtype=torch.float64, device="cuda")
    dweight = torch.zeros_like(weight)
    for slot in range(case["slots"]):
        t = (place[:, slot] >= 0).nonzero().squeeze(1)
        rows = place[t, slot].long()
        dys[rows] = weight[t, slot].unsqueeze(1) * dy[t]
        dweight[t, slot] = (dy[t] * s["ys"][rows].double()).sum(1)
    return {"y": _exact_sum(case, s["ys"], place, weight), "dys": dys, "dweight": dweight}
