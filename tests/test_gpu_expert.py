"""Tokens sorted by expert, their rows, and the experts' rows back at their tokens, against plain implementations."""
import pytest
import torch

from paper_2509_11254_amd import psgd
from test_gpu_act import CODE, DT, UNIT, padded

pytestmark = pytest.mark.gpu

# (tokens, slots, experts): one choice, one expert, fewer choices than a wavefront, one workgroup's border, several workgroups, all experts there may be
SIZES = [(1, 1, 1), (1, 8, 8), (5, 3, 2), (63, 1, 7), (64, 2, 1024), (513, 2, 16), (1024, 8, 64), (1025, 8, 64), (3000, 7, 33), (20000, 8, 128), (40000, 10, 1000),
         (7, 1000, 3)]


def choices(tokens, slots, experts, seed, outside=0.2, skew=2.0):
    gen = torch.Generator().manual_seed(seed)
    c = (experts * torch.rand((tokens, slots), generator=gen) ** skew).long().clamp(max=experts - 1)
    off = torch.rand((tokens, slots), generator=gen) < outside
    other = torch.where(torch.rand((tokens, slots), generator=gen) < 0.5, -1, experts)
    other = torch.where(torch.rand((tokens, slots), generator=gen) < 0.1, 2 ** 40, other)
    return torch.where(off, other, c)


def plain_sort(choice, experts):
    flat = choice.reshape(-1).tolist()
    by = _by_expert(flat, experts)
    rows = [i for e in range(experts) for i in by[e]]
    place = [-1] * len(flat)
    for j, i in enumerate(rows):
        place[i] = j
    offsets = [0]
    for e in range(experts):
        offsets.append(offsets[-1] + len(by[e]))
    return (torch.tensor(place, dtype=torch.int32).view(choice.shape), torch.tensor(rows + [-1] * (len(flat) - len(rows)), dtype=torch.int32),
            torch.tensor(offsets, dtype=torch.int32))


def _by_expert(flat, experts):
    by = [[] for _ in range(experts)]
    for i, e in enumerate(flat):
        if 0 <= e < experts:
            by[e].append(i)
    return by


def sort(choice, experts):
    order = psgd.expert_order_empty(*choice.shape, experts)
    for t in (order.place, order.order, order.offsets):
        t.fill_(-7)
    plan = psgd.ExpertSort(*choice.shape, experts)
    plan.workspace.fill_(0xFF)
    plan.run(choice.cuda(), order)
    return order


def check_sort(order, choice, experts):
    place, rows, offsets = plain_sort(choice, experts)
    assert torch.equal(order.offsets.cpu(), offsets) and torch.equal(order.place.cpu(), place) and torch.equal(order.order.cpu(), rows)


@pytest.mark.parametrize("outside", [0.0, 0.2, 1.1])
@pytest.mark.parametrize("tokens,slots,experts", SIZES)
def test_sort(tokens, slots, experts, outside):
    choice = choices(tokens, slots, experts, 1, outside)
    check_sort(sort(choice, experts), choice, experts)


@pytest.mark.parametrize("tokens,experts", [(200, 5), (9000, 64)])
def test_sort_where_all_choose_one(tokens, experts):
    choice = torch.full((tokens, 2), experts - 1)
    check_sort(sort(choice, experts), choice, experts)


def test_sort_of_very_many():
    """24 million choices, against torch's stable sort; and rows of the most tokens that a launch goes through more than once."""
    tokens, slots, experts = 3000001, 8, 60
    choice = torch.randint(-2, experts + 2, (tokens, slots), device="cuda")
    order = sort(choice, experts)
    flat = choice.view(-1)
    key, want = torch.sort(torch.where((flat >= 0) & (flat < experts), flat, experts), stable=True)
    n = int((key < experts).sum())
    assert torch.equal(order.offsets.long(), torch.searchsorted(key, torch.arange(experts + 1, device="cuda"))) and int(order.offsets[-1]) == n
    assert torch.equal(order.order[:n].long(), want[:n]) and (order.order[n:] == -1).all()
    assert torch.equal(order.place.view(-1)[want[:n]].long(), torch.arange(n, device="cuda")) and (order.place.view(-1)[want[n:]] == -1).all()
    x = torch.arange(tokens, device="cuda").float()[:, None].expand(tokens, 8).contiguous()
    xs, y = torch.full((tokens * slots, 8), -1.0, device="cuda"), torch.empty_like(x)
    psgd.expert_rows(x, order, xs)
    assert torch.equal(xs[:n, 7], (want[:n] // slots).float()) and (xs[n:] == -1).all()
    psgd.expert_combine(xs, order, y)
    # (whole numbers below 2^24 times at most eight: exact in 32 bits or rounded once per sum)
    there = ((choice >= 0) & (choice < experts)).sum(1)
    assert ((y[:, 0].double() - there.double() * x[:, 0].double()).abs() <= slots * 2.0 ** -24 * 8 * tokens).all()


def test_sort_no_tokens():
    order = psgd.expert_order_empty(0, 2, 5)
    order.offsets.fill_(9)
    psgd.ExpertSort(0, 2, 5).run(torch.empty((0, 2), dtype=torch.int64, device="cuda"), order)
    assert (order.offsets == 0).all()
    e = torch.empty((0, 40), device="cuda")
    psgd.expert_rows(e, order, e.clone())
    psgd.expert_combine(e, order, e.clone())
    psgd.expert_combine_backward(e, e.clone(), order, e.clone(), dweight=torch.empty((0, 2), device="cuda"))


# (tokens, slots, experts, cols): one piece, odd columns, several rounds of pieces
ROWS = [(1, 1, 1, 1), (1, 8, 16, 4096), (5, 3, 2, 31), (40, 2, 8, 515), (130, 5, 4, 2056), (17, 9, 30, 5000), (1000, 4, 64, 72), (3, 2, 4, 20001),
        (301, 3, 20, 64), (77, 6, 9, 128), (50, 2, 4, 131), (65, 4, 8, 512), (33, 2, 4, 257)]


def rows_of(n, cols, dtype, seed, extra=8):
    return padded(torch.randn((n, cols), generator=torch.Generator().manual_seed(seed), dtype=torch.float64), DT[dtype], extra)


@pytest.mark.parametrize("outside", [0.0, 0.3, 1.1])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,slots,experts,cols", ROWS)
def test_rows(tokens, slots, experts, cols, dtype, outside):
    choice = choices(tokens, slots, experts, 2, outside)
    order = sort(choice, experts)
    x, _ = rows_of(tokens, cols, dtype, 3)
    xs, buf = rows_of(tokens * slots, cols, dtype, 4, 16)
    before = buf.clone()
    psgd.expert_rows(x, order, xs)
    n, rows = int(order.offsets[-1]), order.order.cpu().long()
    assert torch.equal(xs[:n].cpu(), x.cpu()[rows[:n] // slots])
    # rows behind the last and what lies behind the columns are as they were
    assert torch.equal(buf.view(torch.uint8)[n:], before.view(torch.uint8)[n:]) and buf[:, cols:].isnan().all()


@pytest.mark.parametrize("weighted", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,slots,experts,cols", ROWS)
def test_combine_and_its_gradients(tokens, slots, experts, cols, dtype, weighted):
    choice = choices(tokens, slots, experts, 5, 0.3)
    order = sort(choice, experts)
    n, place = int(order.offsets[-1]), order.place.cpu().long()
    ys, ys_buf = rows_of(tokens * slots, cols, dtype, 6)
    ys_buf[n:] = float("nan")               # rows behind the last reach no result
    weight = torch.randn((tokens, slots), generator=torch.Generator().manual_seed(7)).cuda() if weighted else None
    if weighted:
        weight[order.place < 0] = float("nan")          # nor do weights of choices that do not count
    y, y_buf = padded(torch.full((tokens, cols), float("nan")), DT[dtype], 16)
    psgd.expert_combine(ys, order, y, weight=weight)
    there = place >= 0
    w = torch.where(there, weight.double().cpu() if weighted else torch.ones(place.shape, dtype=torch.float64), 0.0)
    picked = torch.where(there[:, :, None], ys.double().cpu()[place.clamp(min=0)], 0.0)
    want, terms = (picked * w[:, :, None]).sum(1), (picked * w[:, :, None]).abs().sum(1)
    assert ((y.double().cpu() - want).abs() <= slots * 2.0 ** -24 * terms + UNIT[dtype] * 1.01 * want.abs()).all()
    assert (y.cpu()[~there.any(1)] == 0).all() and y_buf[:, cols:].isnan().all()

    dy, _ = rows_of(tokens, cols, dtype, 8)
    for with_dots, in_place in ((True, False), (False, False), (True, True)):
        if in_place:
            out, out_buf, before = ys, ys_buf, ys_buf.clone()
        else:
            out, out_buf = rows_of(tokens * slots, cols, dtype, 9, 16)
            before = out_buf.clone()
        dots = torch.full((tokens, slots), float("nan"), device="cuda") if with_dots else None
        psgd.expert_combine_backward(dy, ys if with_dots else None, order, out, weight=weight, dweight=dots)
        dy64 = dy.double().cpu()
        rows = order.order.cpu().long()[:n]
        want = dy64[rows // slots] * w.view(-1)[rows][:, None]
        assert ((out[:n].double().cpu() - want).abs() <= (UNIT[dtype] + 2.0 ** -24) * 1.01 * want.abs()).all()
        assert torch.equal(out_buf.view(torch.uint8)[n:], before.view(torch.uint8)[n:]) and out_buf[:, cols:].isnan().all()
        if with_dots:
            terms = dy64[:, None, :] * picked
            # a lane adds up a 64th of the columns, then 6 steps over the lanes
            bound = (cols / 64 + 32) * 2.0 ** -24 * terms.abs().sum(2)
            assert ((dots.double().cpu() - terms.sum(2)).abs() <= bound).all() and (dots.cpu()[~there] == 0).all()


def test_the_gradient_of_the_rows():
    """<Xs', G> = <X, combine(G)> for any X and G: the one is the other's transpose."""
    tokens, slots, experts, cols = 100, 4, 9, 136
    order = sort(choices(tokens, slots, experts, 10), experts)
    x, _ = rows_of(tokens, cols, "f32", 11)
    g, _ = rows_of(tokens * slots, cols, "f32", 12)
    xs, dx = torch.zeros_like(g), torch.empty_like(x)
    psgd.expert_rows(x, order, xs)
    psgd.expert_combine(g, order, dx)
    a, b = (xs.double() * g.double()).sum(), (x.double() * dx.double()).sum()
    assert abs(a - b) <= slots * 2.0 ** -24 * (xs.double() * g.double()).abs().sum()


def test_gradients_against_differences():
    """combine is linear in the rows and in the weights: a difference of any size is its derivative."""
    tokens, slots, experts, cols = 40, 3, 5, 72
    order = sort(choices(tokens, slots, experts, 13), experts)
    ys, dy = rows_of(tokens * slots, cols, "f32", 14)[0], rows_of(tokens, cols, "f32", 15)[0]
    weight = torch.randn((tokens, slots), generator=torch.Generator().manual_seed(16)).cuda()
    dys, dw = torch.zeros_like(ys), torch.empty_like(weight)
    psgd.expert_combine_backward(dy, ys, order, dys, weight=weight, dweight=dw)

    def total(ys, weight):
        y = torch.empty_like(dy)
        psgd.expert_combine(ys, order, y, weight=weight)
        return float((y.double() * dy.double()).sum())

    v, u = rows_of(tokens * slots, cols, "f32", 17)[0], torch.randn((tokens, slots), generator=torch.Generator().manual_seed(18)).cuda()
    size = tokens * slots * cols * 20.0
    assert abs(total(ys + v, weight) - total(ys - v, weight) - 2 * float((dys.double() * v.double()).sum())) <= 2.0 ** -22 * size
    assert abs(total(ys, weight + u) - total(ys, weight - u) - 2 * float((dw.double() * u.double()).sum())) <= 2.0 ** -22 * size


def test_places_outside_the_rows_count_for_none():
    order = sort(torch.zeros((6, 2), dtype=torch.int64), 1)
    order.place[2, 1], order.place[3, 0] = 12, -2 ** 31
    x, _ = rows_of(6, 40, "f32", 19)
    xs = torch.full((12, 40), 5.0, device="cuda")
    psgd.expert_rows(x, order, xs)
    y = torch.empty((6, 40), device="cuda")
    psgd.expert_combine(xs, order, y)
    assert (xs[5] == 5).all() and (xs[6] == 5).all() and torch.equal(y[2], x[2]) and torch.equal(y[3], x[3])


def test_in_a_graph_and_on_another_stream():
    tokens, slots, experts, cols = 3000, 4, 40, 264
    choice = choices(tokens, slots, experts, 20).cuda()
    order, plan = psgd.expert_order_empty(tokens, slots, experts), psgd.ExpertSort(tokens, slots, experts)
    x, dy = rows_of(tokens, cols, "bf16", 21)[0], rows_of(tokens, cols, "bf16", 22)[0]
    weight = torch.rand((tokens, slots), device="cuda")
    xs, dys = torch.zeros((tokens * slots, cols), dtype=torch.bfloat16, device="cuda"), torch.zeros((tokens * slots, cols), dtype=torch.bfloat16, device="cuda")
    y, dw = torch.zeros((tokens, cols), dtype=torch.bfloat16, device="cuda"), torch.zeros((tokens, slots), device="cuda")
    out = [order.place, order.order, order.offsets, xs, dys, y, dw]

    def step(stream=None):
        plan.run(choice, order, stream=stream)
        psgd.expert_rows(x, order, xs, stream=stream)
        psgd.expert_combine(xs, order, y, weight=weight, stream=stream)
        psgd.expert_combine_backward(dy, xs, order, dys, weight=weight, dweight=dw, stream=stream)

    def results(run):
        for t in out:
            t.fill_(0)
        torch.cuda.synchronize()
        run()
        torch.cuda.synchronize()
        return [t.clone() for t in out]

    results(step)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph):
        step()
    for seed in (23, 24, 25):
        choice.copy_(choices(tokens, slots, experts, seed, 0.1 * (seed - 22)))
        got = [results(graph.replay), results(step), results(lambda: step(side))]
        assert all(torch.equal(a, b) for other in got[1:] for a, b in zip(got[0], other))


def test_more_than_4_gib():
    tokens, slots, experts, cols = 40000, 8, 16, 8200
    choice = choices(tokens, slots, experts, 26, 0.0).cuda()
    order = sort(choice, experts)
    x = torch.randn((tokens, cols), device="cuda").bfloat16()
    xs = torch.empty((tokens * slots, cols), dtype=torch.bfloat16, device="cuda")
    psgd.expert_rows(x, order, xs)
    rows = order.order.long()
    for at in range(0, tokens * slots, 40000):
        assert torch.equal(xs[at:at + 40000], x[rows[at:at + 40000] // slots])
    # every row of a token is the token's: weights of eighths make it again, exactly
    y = torch.empty_like(x)
    psgd.expert_combine(xs, order, y, weight=torch.full((tokens, slots), 0.125, device="cuda"))
    assert torch.equal(y, x)
