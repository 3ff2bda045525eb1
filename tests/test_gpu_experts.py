"""Tokens sorted by expert, their rows, the weighted sum and its gradients against
the definitions in 64 bits, element by element."""
import pytest
import torch

import paper_2106_08846_gb300 as bsr

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
U = 2.0 ** -24   # half a step of fp32
SIZES = [  # N, k, E, D, align, share of dropped choices
    (1, 1, 1, 1, 1, 0.0), (1, 2, 8, 1024, 1, 0.0), (1, 8, 8, 770, 128, 0.0), (3, 2, 5, 2, 16, 0.5), (31, 4, 64, 63, 1, 0.1),
    (100, 1, 3, 64, 7, 0.0), (129, 2, 1024, 128, 128, 0.0), (300, 3, 4, 771, 128, 1.0), (1000, 2, 16, 516, 64, 0.2),
    (2100, 2, 7, 1028, 128, 0.0), (4097, 8, 33, 40, 1, 0.05), (20000, 4, 1000, 24, 3, 0.0), (700, 64, 64, 8, 1024, 0.0), (64, 2, 8, 5000, 1, 0.1)]


def choices(N, k, E, drop, seed=0):
    g = torch.Generator().manual_seed(1009 * N + 31 * E + k + seed)
    x = torch.randint(0, E, (N, k), generator=g, dtype=torch.int32)   # (an expert twice, too)
    x[:, 0] = x[:, 0] % max(1, E // 3)                                # some experts' runs are long, some empty
    bad = torch.randint(0, 4, (N, k), generator=g)
    wrong = torch.tensor([-1, E, -2 ** 31, 2 ** 31 - 1])[bad].int()
    return torch.where(torch.rand(N, k, generator=g) < drop, wrong, x)


def by_hand(x, E, align, rows):
    """offsets, place and source, choice by choice."""
    N, k = x.shape
    runs = [[] for _ in range(E)]
    for p, e in enumerate(x.reshape(-1).tolist()):
        if 0 <= e < E:
            runs[e].append(p)
    offsets, place, source = [0], torch.full((N * k,), -1, dtype=torch.int32), torch.full((rows,), -1, dtype=torch.int32)
    for run in runs:
        o = offsets[-1]
        if run:
            at = torch.tensor(run)
            place[at] = torch.arange(o, o + len(run), dtype=torch.int32)
            source[o:o + len(run)] = at.int()
        offsets.append(o + -(-len(run) // align) * align)
    return torch.tensor(offsets, dtype=torch.int32), place.view(N, k), source


def guarded(rows, D, dtype):
    buf = torch.full((rows * D + 64,), 7.0, dtype=dtype, device="cuda")
    return buf, buf[32:32 + rows * D].view(rows, D)


def unharmed(buf):
    return bool((buf[:32] == 7).all() and (buf[-32:] == 7).all())


def draw(N, D, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(17 * N + D + seed)
    return torch.randn(N, D, device="cuda", generator=g).to(DT[dtype])


def uniform(N, k):
    # (a generator of its own: a capture in another test may have left the default one unusable)
    return torch.rand(N, k, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3))


def make(N, k, E, align, drop):
    x = choices(N, k, E, drop)
    order = bsr.ExpertOrder(N, k, E, align)
    for t in (order.offsets, order.place, order.source):
        t.fill_(77)
    bsr.bsr_expert_order(x.cuda(), E, align, order=order)
    return x, order, by_hand(x, E, align, order.rows)


@pytest.mark.parametrize("N,k,E,D,align,drop", SIZES)
def test_order(N, k, E, D, align, drop):
    x, order, (offsets, place, source) = make(N, k, E, align, drop)
    assert torch.equal(order.offsets.cpu(), offsets)
    assert torch.equal(order.place.cpu(), place)
    assert torch.equal(order.source.cpu(), source)
    assert int(order.used) == int(offsets[-1]) <= order.rows
    again = bsr.bsr_expert_order(x.cuda(), E, align)
    assert all(torch.equal(getattr(order, f), getattr(again, f)) for f in ("offsets", "place", "source"))


def test_order_of_a_million_choices_and_one_expert():
    for N, k, E in ((1 << 19, 2, 1), (1 << 18, 4, 1024)):
        x = torch.randint(0, E, (N, k), dtype=torch.int32, device="cuda", generator=torch.Generator(device="cuda").manual_seed(5))
        order = bsr.bsr_expert_order(x, E, 128)
        flat = x.view(-1).long()
        pairs = torch.sort(flat, stable=True).indices
        counts = torch.bincount(flat, minlength=E)
        runs = (counts + 127) // 128 * 128
        assert torch.equal(order.offsets[1:].long(), runs.cumsum(0)) and int(order.offsets[0]) == 0
        first = torch.cat((counts.new_zeros(1), counts.cumsum(0)))[:-1]
        row = order.offsets[:-1].long()[flat[pairs]] + torch.arange(N * k, device="cuda") - first[flat[pairs]]
        assert torch.equal(order.place.view(-1)[pairs].long(), row)
        source = torch.full((order.rows,), -1, dtype=torch.int32, device="cuda")
        source[row] = pairs.int()
        assert torch.equal(order.source, source)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,k,E,D,align,drop", SIZES)
def test_rows_and_back(N, k, E, D, align, drop, dtype):
    x, order, (offsets, place, source) = make(N, k, E, align, drop)
    X, R, used = draw(N, D, dtype), order.rows, int(offsets[-1])
    buf, Xs = guarded(R, D, DT[dtype])
    bsr.bsr_expert_rows(X, order, Xs=Xs)
    want = torch.full_like(Xs, 7.0)
    want[:used] = 0
    sent = (source >= 0).cuda()
    want[sent] = X[(source.cuda()[sent] // k).long()]
    assert torch.equal(Xs, want) and unharmed(buf)

    Ys, w = draw(R, D, dtype, 1), uniform(N, k) - 0.2
    Ys[~sent] = float("nan")   # rows that no choice has are not read
    at = place.cuda().clamp(min=0).long()
    has = (place >= 0).cuda().unsqueeze(2)
    picked = torch.where(has, Ys[at].double(), torch.zeros((), dtype=torch.double, device="cuda"))
    half = 2.0 ** -8 if dtype == "bf16" else U
    for weights in (None, w):
        buf, Y = guarded(N, D, DT[dtype])
        bsr.bsr_expert_sum(Ys, order, weights, Y=Y)
        terms = picked if weights is None else picked * weights.double().unsqueeze(2)
        S, size = terms.sum(1), terms.abs().sum(1)
        # a rounding to 24 bits for each choice, then one to the result's type
        assert ((Y.double() - S).abs() <= half * S.abs() + 2 * k * U * size).all() and unharmed(buf)

    dY = draw(N, D, dtype, 2)
    buf, dYs = guarded(R, D, DT[dtype])
    got = bsr.bsr_expert_sum_backward(Ys, order, w, dY, dYs=dYs)
    pair = source.cuda()[sent].long()
    want = torch.full(dYs.shape, 7.0, dtype=torch.double, device="cuda")
    want[:used] = 0
    want[sent] = dY[pair // k].double() * w.view(-1)[pair].double().unsqueeze(1)
    # (one product of fp32, rounded twice)
    assert ((dYs.double() - want).abs() <= (half + 2 * U) * want.abs()).all() and unharmed(buf)
    terms = picked * dY.double().unsqueeze(1)
    # a lane's D / 32 products (runs of eight) in turn, then five sums of lanes
    bound = (D / 32 + 8 + 5) * U * terms.abs().sum(2)
    assert ((got["dweights"].double() - terms.sum(2)).abs() <= bound).all()
    plain = bsr.bsr_expert_sum_backward(None, order, None, dY, dYs=torch.zeros_like(dYs))
    assert set(plain) == {"dYs"}
    assert torch.equal(plain["dYs"], bsr.bsr_expert_rows(dY, order, Xs=torch.zeros_like(dYs)))


def test_gradients_against_differences():
    N, k, E, D = 9, 2, 4, 12
    x, order, _ = make(N, k, E, 4, 0.2)
    X, w, dY = draw(N, D, "f32"), uniform(N, k), draw(N, D, "f32", 1)

    def out(X, w):   # every expert doubles its rows and adds up with the weights
        Ys = 2 * bsr.bsr_expert_rows(X, order, Xs=torch.zeros(order.rows, D, device="cuda"))
        return Ys, float((bsr.bsr_expert_sum(Ys, order, w).double() * dY.double()).sum())

    Ys, _ = out(X, w)
    g = bsr.bsr_expert_sum_backward(Ys, order, w, dY, dYs=torch.zeros_like(Ys))
    dX = bsr.bsr_expert_sum(2 * g["dYs"], order)
    for v, d, other in ((X, dX, "w"), (w, g["dweights"], "X")):
        way = torch.randn(v.shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
        step = 0.5   # (linear in each: differences of any step are the derivative)
        hi, lo = (out(v + s * way, w)[1] if other == "w" else out(X, v + s * way)[1] for s in (step, -step))
        size = float((d.double().abs() * way.double().abs()).sum()) + abs(hi) + abs(lo)
        # sums of at most 2 N k D terms, each rounded a few times
        assert abs((hi - lo) / (2 * step) - float((d.double() * way.double()).sum())) <= 16 * U * size * N


def test_rows_beyond_32_bits():
    N, k, E, D = 40000, 2, 8, 32768   # 2.6e9 values
    x = choices(N, k, E, 0.0)
    order = bsr.bsr_expert_order(x.cuda(), E, 1)
    X = torch.arange(N, device="cuda").remainder(61).to(torch.bfloat16).unsqueeze(1).expand(N, D).contiguous()
    Xs = bsr.bsr_expert_rows(X, order)
    assert torch.equal(Xs[:, ::4096].cpu(), X[:, ::4096].cpu()[(order.source // k).long().cpu()])
    assert torch.equal(Xs[-1], X[int(order.source[-1]) // k])
    Y = bsr.bsr_expert_sum(Xs, order)
    assert torch.equal(Y[:, ::4096], 2 * X[:, ::4096]) and torch.equal(Y[-1], 2 * X[-1])
    g = bsr.bsr_expert_sum_backward(Xs, order, torch.ones(N, k, device="cuda"), X, dYs=torch.empty_like(Xs))
    assert torch.equal(g["dYs"], Xs)
    # exact in fp32: a lane's 1024 products are whole numbers below 2^22, and equal for all lanes
    want = D * X[:, :1].double() ** 2
    assert torch.equal(g["dweights"].double(), want.expand(N, k))


def test_streams_and_a_captured_graph():
    N, k, E, D = 500, 2, 8, 768
    xs = [choices(N, k, E, 0.1, seed).cuda() for seed in (0, 1)]
    X, w = draw(N, D, "bf16"), uniform(N, k)
    order, x = bsr.ExpertOrder(N, k, E, 16), xs[0].clone()
    Xs, Y = torch.zeros(order.rows, D, dtype=torch.bfloat16, device="cuda"), torch.empty_like(X)

    def layer(stream=None):
        bsr.bsr_expert_order(x, E, 16, order=order, stream=stream)
        bsr.bsr_expert_rows(X, order, Xs=Xs, stream=stream)
        bsr.bsr_expert_sum(Xs, order, w, Y=Y, stream=stream)
        return bsr.bsr_expert_sum_backward(Xs, order, w, X, dYs=Xs.clone() if stream is None else None, stream=stream)

    layer()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = layer()
    for choice in (xs[1], xs[0]):
        x.copy_(choice)
        graph.replay()
        got = [t.clone() for t in (order.place, Y, held["dweights"])]
        layer()
        for a, b in zip(got, (order.place, Y, bsr.bsr_expert_sum_backward(Xs, order, w, X)["dweights"])):
            assert torch.equal(a, b)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    Y.zero_()
    side.wait_stream(torch.cuda.current_stream())
    g = layer(side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(Y, got[1]) and torch.equal(g["dweights"], got[2])


def test_nobody_is_sent_and_invalid_orders():
    """All choices dropped; and places and sources that are no rows, which are left out."""
    N, k, E, D = 40, 2, 6, 64
    X = draw(N, D, "bf16")
    order = bsr.bsr_expert_order(torch.full((N, k), -1, dtype=torch.int32, device="cuda"), E, 16)
    assert int(order.used) == 0 and (order.place == -1).all() and (order.source == -1).all()
    Xs = torch.full((order.rows, D), 7.0, dtype=torch.bfloat16, device="cuda")
    assert (bsr.bsr_expert_rows(X, order, Xs=Xs) == 7).all()
    assert (bsr.bsr_expert_sum(Xs, order, uniform(N, k)) == 0).all()
    g = bsr.bsr_expert_sum_backward(Xs, order, uniform(N, k), X, dYs=Xs.clone())
    assert (g["dYs"] == 7).all() and (g["dweights"] == 0).all()
    with pytest.raises(bsr.BsrError):   # (not in place)
        bsr.bsr_expert_sum_backward(Xs, order, uniform(N, k), X, dYs=Xs)
    bsr.bsr_expert_order(torch.zeros(N, k, dtype=torch.int32, device="cuda"), E, 16, order=order)
    order.place[3, 1], order.place[4, 0] = order.rows, -5
    order.offsets[E] = 2 ** 31 - 1
    bsr.bsr_expert_rows(X, order, Xs=Xs)
    assert (bsr.bsr_expert_sum(Xs, order)[4] == X[4]).all()


def test_no_tokens():
    order = bsr.bsr_expert_order(torch.empty(0, 2, dtype=torch.int32, device="cuda"), 4, 128)
    assert order.rows == 0 and order.offsets.tolist() == [0] * 5
    X = torch.empty(0, 16, device="cuda")
    assert bsr.bsr_expert_rows(X, order).shape == bsr.bsr_expert_sum(X, order).shape == (0, 16)
