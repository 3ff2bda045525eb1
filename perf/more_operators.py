"""The measured work of the operators of expert layers and of 8-bit products:
tokens sorted by expert and added up again with the router's weights
(``bsr_expert_order``, ``bsr_expert_rows``, ``bsr_expert_sum`` and its backward
pass), and matrix products of 8-bit floating-point operands with a scale for each
block of 128 (``bsr_fp8_quantize``, ``bsr_fp8_product``), plain and for the runs of
rows of many experts.

Sizes are those of the repository's workloads (768, 1024 and 4096 features, 128
to 16384 tokens), with single tokens, small batches and ragged sizes beside
them; ``draw`` varies all of them.

A case is a dict of plain values:
  kind      "rows", "sum", "sum_backward", "quantize", "linear", "linear_backward",
            "experts" or "experts_backward"
  N         tokens
  dtype     "f32" or "bf16": the tensors' type on both sides
 expert layers:
  k, E      experts of a token, and of the layer
  align     each expert's rows start at a multiple of it
  drop      share of the tokens' choices that are dropped (expert -1)
 sorting and adding up:
  D         features
  weights   whether the sum has weights
 8-bit products:
  K, M      features that are summed over, and of the result ("quantize": K)
  fmt       "e4m3" or "e5m2": the format of X, or of the gradient
  bias      whether the result has a bias
"""
import torch

own = False

_TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
_BLOCK = 128
_MOST = {"e4m3": 448.0, "e5m2": 57344.0}
_FORMAT = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}


def _case(name, kind, N, dtype, **more):
    c = dict(kind=kind, N=N, dtype=dtype, **more)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token of a served request on its way to its experts: latency
        _case("rows_bf16_n1", "rows", 1, "bf16", D=1024, k=2, E=8, align=1, drop=0.0),
        # a large batch of BERT-large width over many experts, runs aligned for the weights' gradients
        _case("rows_bf16_n16384", "rows", 16384, "bf16", D=1024, k=4, E=64, align=128, drop=0.0),
        # a ragged batch, some choices dropped by the experts' capacity, an odd number of features
        _case("sum_f32_n1000", "sum", 1000, "f32", D=770, k=2, E=8, align=1, drop=0.1, weights=True),
        # a large batch back from its experts
        _case("sum_bf16_n16384", "sum", 16384, "bf16", D=1024, k=4, E=64, align=128, drop=0.0, weights=True),
        # its training step
        _case("sum_bwd_bf16_n16384", "sum_backward", 16384, "bf16", D=1024, k=2, E=16, align=128, drop=0.0, weights=True),
        # activations of a large training batch for the product and for the weights' gradient
        _case("quantize_bf16_n16384", "quantize", 16384, "bf16", K=1024, fmt="e4m3"),
        # one token of a served request: reading the weights is the work
        _case("linear_bf16_n1", "linear", 1, "bf16", K=1024, M=4096, fmt="e4m3", bias=False),
        # a ragged batch with odd sizes in fp32
        _case("linear_f32_n999", "linear", 999, "f32", K=770, M=2050, fmt="e4m3", bias=True),
        # a large batch
        _case("linear_bf16_n16384", "linear", 16384, "bf16", K=1024, M=4096, fmt="e4m3", bias=False),
        # a large training step: the gradients of the input and of the weight
        _case("linear_bwd_bf16_n8192", "linear_backward", 8192, "bf16", K=1024, M=4096, fmt="e5m2"),
        # a batch through an expert layer's products: sorted, quantised, every run with its expert's weight
        _case("experts_bf16_n4096", "experts", 4096, "bf16", K=1024, M=4096, fmt="e4m3", bias=False, k=2, E=16, align=128,
              drop=0.0),
        # its training step: the gradients of the rows and of every expert's weight
        _case("experts_bwd_bf16_n4096", "experts_backward", 4096, "bf16", K=768, M=2048, fmt="e4m3", k=2, E=8, align=128,
              drop=0.0),
    ]


def draw(rng):
    """Another case of the same ranges: 1 to 16384 tokens, 64 to 4096 features that
    are sorted, 128 to 4096 by 128 to 1536 of a product, 1 to 8 of 2 to 64 experts,
    odd sizes among them."""
    def log_int(lo, hi):
        return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))

    def size(lo, hi):   # mostly multiples of 64, as models have; some of 8, some odd
        n, p = log_int(lo, hi), rng.random()
        step = 64 if p < 0.6 else 8 if p < 0.85 else 1
        return max(lo, n - n % step)

    kind = rng.choice(("rows", "sum", "sum_backward", "quantize", "linear", "linear_backward", "experts", "experts_backward"))
    dtype = rng.choice(("f32", "bf16"))
    N = log_int(1, 16384)
    E = log_int(2, 64)
    es, bytes_most = 4 if dtype == "f32" else 2, 160000000
    route = dict(k=min(E, rng.choice((1, 2, 2, 4, 8))), E=E, align=rng.choice((1, 16, 128)), drop=rng.choice((0.0, 0.0, 0.1)))
    if kind in ("rows", "sum", "sum_backward"):
        D = size(64, 4096)
        N = max(1, min(N, bytes_most // (es * D * (2 * route["k"] + 1))))
        if kind != "rows":
            route["weights"] = rng.random() < 0.75
        return _case(None, kind, N, dtype, D=D, **route)
    K, M, fmt = size(128, 1536), size(128, 4096), rng.choice(("e4m3", "e4m3", "e5m2"))
    if kind == "quantize":
        return _case(None, kind, N, dtype, K=K, fmt=fmt)
    most = 16384 * 4096 * 1024
    if kind.startswith("linear"):
        N = max(1, min(N, most // (K * M * (2 if kind == "linear_backward" else 1)), bytes_most // (es * (2 * K + M))))
        bias = {} if kind == "linear_backward" else dict(bias=rng.random() < 0.5)
        return _case(None, kind, N, dtype, K=K, M=M, fmt=fmt, **bias)
    N = max(1, min(N, 4096, most // (2 * K * M * route["k"]), bytes_most // (es * (2 * K + M) * route["k"])))
    route["E"] = max(route["k"], min(route["E"], max(2, 16 * 4096 * 1024 // (K * M))))
    if kind == "experts_backward":
        return _case(None, kind, N, dtype, K=K, M=M, fmt=fmt, **dict(route, align=128))
    return _case(None, kind, N, dtype, K=K, M=M, fmt=fmt, bias=rng.random() < 0.5, **route)


# ---- inputs

def _rows_at_most(c):
    """Rows that the sorted tokens may take."""
    pairs = c["N"] * c["k"]
    return (pairs + min(c["E"], pairs) * (c["align"] - 1)) // c["align"] * c["align"]


def _inputs(case, seed):
    """What a case reads, but the weights in 8 bits; a router's choices favour some experts."""
    gen = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(*shape, std=1.0):
        return torch.randn(*shape, device="cuda", generator=gen) * std

    c, dt, s = case, _TORCH[case["dtype"]], {}
    kind, N = c["kind"], c["N"]
    if "E" in c:
        logits = normal(N, c["E"]) + normal(c["E"], std=0.7)
        s["experts"] = logits.topk(c["k"], 1).indices.int()
        if c["drop"]:
            s["experts"][torch.rand(N, c["k"], device="cuda", generator=gen) < c["drop"]] = -1
    R = _rows_at_most(c) if "E" in c else N
    if kind == "rows":
        s["X"] = normal(N, c["D"]).to(dt)
    elif kind in ("sum", "sum_backward"):
        s["Ys"] = normal(R, c["D"]).to(dt)
        s["weights"] = torch.rand(N, c["k"], device="cuda", generator=gen) if c["weights"] else None
        if kind == "sum_backward":
            s["dY"] = normal(N, c["D"], std=0.1).to(dt)
    else:   # features differ in their size, as activations' do
        wide = torch.exp(normal(c["K"], std=0.7))
        rows = R if kind == "experts_backward" else N
        s["X"] = (normal(rows, c["K"]) * wide).to(dt)
        if kind != "quantize":
            each = (c["E"],) if "E" in c else ()
            s["W"] = normal(*each, c["M"], c["K"], std=0.02).to(dt)
            s["bias"] = normal(*each, c["M"], std=0.02) if c.get("bias") else None
        if kind.endswith("backward"):   # gradients of different tokens differ in their size
            s["dY"] = (normal(rows, c["M"], std=0.01) * torch.exp(normal(rows, 1))).to(dt)
    if kind in ("sum", "sum_backward", "experts_backward"):
        s["order"] = _plain_order(s["experts"], c)
    if kind == "experts_backward":   # rows that nobody was sent to are zeros
        used = s["order"]["source"].unsqueeze(1) >= 0
        s["X"], s["dY"] = (torch.where(used, t, torch.zeros_like(t)) for t in (s["X"], s["dY"]))
    return s


def prepare(case, seed):
    """The inputs, the weights in 8 bits, and the buffers that a program keeps for the outputs."""
    c, s, kind = case, _inputs(case, seed), case["kind"]
    s["case"] = c
    dt = _TORCH[c["dtype"]]
    R = _rows_at_most(c) if "E" in c else c["N"]

    def zeros(*shape):
        return torch.zeros(*shape, dtype=dt, device="cuda")

    if kind in ("rows", "experts"):
        s["Xs"] = zeros(R, c["D"] if kind == "rows" else c["K"])
    if kind == "sum":
        s["Y"] = zeros(c["N"], c["D"])
    if kind == "sum_backward":
        s["dYs"] = zeros(R, c["D"])
    if kind in ("linear", "experts"):
        s["Y"] = zeros(R, c["M"])
    if kind.endswith("backward") and "W" in s:
        s["dX"], s["dW"] = zeros(R, c["K"]), torch.zeros_like(s["W"])
    if own:
        _own_prepare(s, c)
    elif "W" in s:
        s["W"] = _plain_values(s["W"], "e4m3", 128)
    return s


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"rows": _own_rows, "sum": _own_sum, "sum_backward": _own_sum_backward, "quantize": _own_quantize,
                "linear": _own_linear, "linear_backward": _own_linear_backward, "experts": _own_experts,
                "experts_backward": _own_experts_backward}[kind](state, state["case"])
    return {"rows": _plain_rows, "sum": _plain_sum, "sum_backward": _plain_sum_backward, "quantize": _plain_quantize,
            "linear": _plain_linear, "linear_backward": _plain_linear_backward, "experts": _plain_experts,
            "experts_backward": _plain_experts_backward}[kind](state, state["case"])


# ---- the framework's operators

def _own_prepare(s, c):
    """A layer's weights are quantised once; the order of a backward pass is the forward pass's."""
    import paper_2106_08846_gb300 as bsr
    if "W" in s:
        form = "columns" if c["kind"].endswith("backward") else "rows"
        s["W"] = bsr.bsr_fp8_quantize(s["W"], tile=128, form=form)
    if "order" in s:
        s["order"] = bsr.bsr_expert_order(s["experts"], c["E"], align=c["align"])
    elif "E" in c:   # the arrays that a program keeps
        s["order"] = bsr.ExpertOrder(c["N"], c["k"], c["E"], c["align"], "cuda")


def _own_rows(s, c):
    import paper_2106_08846_gb300 as bsr
    order = bsr.bsr_expert_order(s["experts"], c["E"], align=c["align"], order=s["order"])
    Xs = bsr.bsr_expert_rows(s["X"], order, Xs=s["Xs"])
    return {"offsets": order.offsets, "place": order.place, "source": order.source, "Xs": Xs}


def _own_sum(s, c):
    import paper_2106_08846_gb300 as bsr
    return {"Y": bsr.bsr_expert_sum(s["Ys"], s["order"], s["weights"], Y=s["Y"])}


def _own_sum_backward(s, c):
    import paper_2106_08846_gb300 as bsr
    return bsr.bsr_expert_sum_backward(s["Ys"], s["order"], s["weights"], s["dY"], dYs=s["dYs"])


def _own_quantize(s, c):
    import paper_2106_08846_gb300 as bsr
    x, t = bsr.bsr_fp8_quantize(s["X"], fmt=c["fmt"], form="both")
    return {"q": x.q, "scale": x.scale, "qt": t.q, "scale_t": t.scale}


def _own_linear(s, c):
    import paper_2106_08846_gb300 as bsr
    return {"Y": bsr.bsr_fp8_product(bsr.bsr_fp8_quantize(s["X"], fmt=c["fmt"]), s["W"], s["bias"], Y=s["Y"])}


def _own_linear_backward(s, c):
    import paper_2106_08846_gb300 as bsr
    d, dt = bsr.bsr_fp8_quantize(s["dY"], fmt=c["fmt"], form="both")
    xt = bsr.bsr_fp8_quantize(s["X"], form="columns")
    return {"dX": bsr.bsr_fp8_product(d, s["W"], Y=s["dX"]), "dW": bsr.bsr_fp8_product(dt, xt, Y=s["dW"])}


def _own_experts(s, c):
    import paper_2106_08846_gb300 as bsr
    order = bsr.bsr_expert_order(s["experts"], c["E"], align=c["align"], order=s["order"])
    Xs = bsr.bsr_fp8_quantize(bsr.bsr_expert_rows(s["X"], order, Xs=s["Xs"]), fmt=c["fmt"], used=order.used)
    Y = bsr.bsr_fp8_product(Xs, s["W"], s["bias"], offsets=order.offsets, Y=s["Y"])
    return {"offsets": order.offsets, "Y": Y}


def _own_experts_backward(s, c):
    import paper_2106_08846_gb300 as bsr
    o = s["order"]
    d, dt = bsr.bsr_fp8_quantize(s["dY"], fmt=c["fmt"], form="both", used=o.used)
    xt = bsr.bsr_fp8_quantize(s["X"], form="columns", used=o.used)
    return {"dX": bsr.bsr_fp8_product(d, s["W"], offsets=o.offsets, Y=s["dX"]),
            "dW": bsr.bsr_fp8_product(dt, xt, offsets=o.offsets, over="columns", Y=s["dW"])}


# ---- their plain forms: 32 bits, rounded once at the end

def _plain_order(experts, c):
    """Offsets of the experts' runs, the row of every choice and the choice of every row."""
    flat, E, R = experts.reshape(-1).long(), c["E"], _rows_at_most(c)
    kept = flat >= 0
    counts = torch.zeros(E + 1, dtype=torch.long, device="cuda").index_add_(0, torch.where(kept, flat, E), torch.ones_like(flat))[:E]
    runs = (counts + c["align"] - 1) // c["align"] * c["align"]
    zero = torch.zeros(1, dtype=torch.long, device="cuda")
    offsets, first = torch.cat((zero, runs.cumsum(0))), torch.cat((zero, counts.cumsum(0)))
    pairs = torch.sort(torch.where(kept, flat, E), stable=True).indices
    e = torch.where(kept, flat, E)[pairs]
    row = torch.where(e < E, offsets[e] + torch.arange(flat.numel(), device="cuda") - first[e], -1)
    place = torch.empty_like(flat)
    place[pairs] = row
    source = torch.full((R + 1,), -1, dtype=torch.long, device="cuda")
    source[torch.where(row >= 0, row, R)] = pairs
    return {"offsets": offsets.int(), "place": place.view(experts.shape).int(), "source": source[:R].int()}


def _plain_sorted(s, c, order):
    """The tokens' rows in the experts' order, 0 where nobody was sent to."""
    token = order["source"].clamp(min=0).long() // c["k"]
    return s["X"].float()[token] * (order["source"] >= 0).unsqueeze(1)


def _plain_rows(s, c):
    order = _plain_order(s["experts"], c)
    return dict(order, Xs=_plain_sorted(s, c, order).to(s["X"].dtype))


def _plain_sum(s, c):
    place = s["order"]["place"]
    picked = s["Ys"].float()[place.clamp(min=0).long()] * (place >= 0).unsqueeze(2)
    if s["weights"] is not None:
        picked = picked * s["weights"].unsqueeze(2)
    return {"Y": picked.sum(1).to(s["Ys"].dtype)}


def _plain_sum_backward(s, c):
    place, source = s["order"]["place"], s["order"]["source"]
    dY, pair = s["dY"].float(), source.clamp(min=0).long()
    rows = dY[pair // c["k"]] * (source >= 0).unsqueeze(1)
    if s["weights"] is None:
        return {"dYs": rows.to(s["Ys"].dtype)}
    rows = rows * s["weights"].reshape(-1)[pair].unsqueeze(1)
    picked = s["Ys"].float()[place.clamp(min=0).long()] * (place >= 0).unsqueeze(2)
    return {"dYs": rows.to(s["Ys"].dtype), "dweights": (picked * dY.unsqueeze(1)).sum(2)}


def _plain_quantized(x, fmt, tile):
    """The 8-bit values of the last two axes' blocks of `tile` x 128 and the power of
    two of each block. (The border between two powers in 64 bits.)"""
    R, C = x.shape[-2:]
    x = torch.nn.functional.pad(x.float(), (0, -C % _BLOCK, 0, -R % tile))
    x = x.view(*x.shape[:-2], -1, tile, x.shape[-1] // _BLOCK, _BLOCK)
    most = x.abs().amax((-3, -1), keepdim=True).double() / _MOST[fmt]
    m, e = torch.frexp(most)
    e = torch.where(m == 0.5, e - 1, e).clamp(min=-126)
    scale = torch.where(most > 0, torch.ldexp(torch.ones_like(most), e), torch.ones_like(most)).float()
    q = (x / scale).to(_FORMAT[fmt])
    return q.flatten(-2).flatten(-3, -2)[..., :R, :], scale.squeeze(-1).squeeze(-2).transpose(-1, -2)


def _plain_values(x, fmt, tile):
    """What the 8-bit form of x stands for."""
    q, scale = _plain_quantized(x, fmt, tile)
    whole = scale.transpose(-1, -2).repeat_interleave(tile, -2).repeat_interleave(_BLOCK, -1)
    return (q.float() * whole[..., :q.shape[-2], :])[..., :x.shape[-1]]


def _plain_quantize(s, c):
    q, scale = _plain_quantized(s["X"], c["fmt"], 1)
    qt, scale_t = _plain_quantized(s["X"].transpose(0, 1), c["fmt"], 1)
    return {"q": q, "scale": scale, "qt": qt, "scale_t": scale_t}


def _plain_linear(s, c):
    Y = _plain_values(s["X"], c["fmt"], 1) @ s["W"].T
    return {"Y": (Y if s["bias"] is None else Y + s["bias"]).to(s["X"].dtype)}


def _plain_linear_backward(s, c):
    dX = _plain_values(s["dY"], c["fmt"], 1) @ s["W"]
    dW = _plain_values(s["dY"].T, c["fmt"], 1) @ _plain_values(s["X"].T, "e4m3", 1).T
    return {"dX": dX.to(s["X"].dtype), "dW": dW.to(s["X"].dtype)}


def _plain_experts(s, c):
    order = _plain_order(s["experts"], c)
    X = _plain_values(_plain_sorted(s, c, order).to(s["X"].dtype), c["fmt"], 1)
    at = order["offsets"].tolist()
    for e in range(c["E"]):
        Y = X[at[e]:at[e + 1]] @ s["W"][e].T
        s["Y"][at[e]:at[e + 1]] = Y if s["bias"] is None else Y + s["bias"][e]
    return {"offsets": order["offsets"], "Y": s["Y"]}


def _plain_experts_backward(s, c):
    d, dt = _plain_values(s["dY"], c["fmt"], 1), _plain_values(s["dY"].T, c["fmt"], 1)
    xt = _plain_values(s["X"].T, "e4m3", 1)
    at = s["order"]["offsets"].tolist()
    for e in range(c["E"]):
        run = slice(at[e], at[e + 1])
        s["dX"][run] = d[run] @ s["W"][e]
        s["dW"][e] = dt[:, run] @ xt[:, run].T
    return {"dX": s["dX"], "dW": s["dW"]}


# ---- what they cannot do without, and their values in 64 bits

def work(case):
    c, es, N = case, 4 if case["dtype"] == "f32" else 2, case["N"]
    kind = c["kind"]
    pairs = N * c["k"] if "E" in c else N
    if kind in ("rows", "sum", "sum_backward"):
        D = c["D"]
        if kind == "rows":   # the choices and X in, the order (two ways) and the rows out
            return {"bytes": es * (N + pairs) * D + 12 * pairs + 4 * (c["E"] + 1), "flops": pairs}
        weights = 4 * pairs if c["weights"] else 0
        if kind == "sum":
            return {"bytes": es * (N + pairs) * D + 4 * pairs + weights, "flops": 2 * pairs * D}
        rows = 2 * pairs if c["weights"] else pairs   # (without weights the rows themselves are not read)
        return {"bytes": es * (N + rows) * D + 4 * pairs + 2 * weights, "flops": 3 * pairs * D}
    K = c["K"]
    if kind == "quantize":
        return {"bytes": (es + 2) * N * K + 4 * N * K // 64, "flops": 4 * N * K}
    M = c["M"]
    weights = M * K * min(c["E"], pairs) if "E" in c else M * K
    bias = 4 * weights // K if c.get("bias") else 0
    order = 12 * pairs if kind == "experts" else 0
    if kind.endswith("backward"):   # dY, X and the weights in, dX and dW out
        out = es * (M * K * c["E"] if "E" in c else M * K)
        return {"bytes": es * pairs * (M + 2 * K) + weights + out, "flops": 4 * pairs * M * K}
    return {"bytes": es * (N * K + pairs * M) + weights + bias + order, "flops": 2 * pairs * M * K}


def _exact_power(block, fmt, rows):
    """The exponent of a block's scale; rows 1: of each row's."""
    top = block.abs().amax(1, keepdim=True) if rows == 1 else block.abs().max()
    m, e = torch.frexp(top / _MOST[fmt])
    return torch.where(m == 0.5, e - 1, e).clamp(min=-126)


def _exact_blocks(x, fmt, rows, cols):
    """x with every block of rows x cols rounded to the format at its block's power of two."""
    bits, least = {"e4m3": (3, -6), "e5m2": (2, -14)}[fmt]
    out = torch.empty_like(x)
    for i in [slice(None)] if rows == 1 else [slice(i, i + rows) for i in range(0, x.shape[0], rows)]:
        for j in range(0, x.shape[1], cols):
            block = x[i, j:j + cols]
            power = _exact_power(block, fmt, rows)
            y = block * torch.exp2(-power.double())
            step = torch.exp2((torch.frexp(y).exponent - 1).clamp(min=least).double() - bits)
            out[i, j:j + cols] = torch.round(y / step) * step * torch.exp2(power.double())
    return out


def _exact_order(experts, c):
    """Every expert's choices behind one another, by hand."""
    def whole(v, shape):
        return torch.tensor(v, dtype=torch.int32, device="cuda").view(shape)

    flat, runs, offsets = experts.reshape(-1).tolist(), [[] for _ in range(c["E"])], [0]
    place, source = [-1] * len(flat), [-1] * _rows_at_most(c)
    for pair, e in enumerate(flat):
        if e >= 0:
            runs[e].append(pair)
    for run in runs:
        for rank, pair in enumerate(run):
            place[pair] = offsets[-1] + rank
            source[offsets[-1] + rank] = pair
        offsets.append(offsets[-1] + -(-len(run) // c["align"]) * c["align"])
    return whole(offsets, -1), whole(place, experts.shape), whole(source, -1)


def exact(case, seed):
    """The definitions in double precision."""
    c, s, kind = case, _inputs(case, seed), case["kind"]
    if kind == "quantize":
        out = {}
        for t, x in (("", s["X"].double()), ("t", s["X"].double().T.contiguous())):
            power = torch.stack([_exact_power(b, c["fmt"], 1)[:, 0] for b in x.split(_BLOCK, 1)])
            scale = torch.exp2(power.double())
            whole = scale.T.repeat_interleave(_BLOCK, 1)
            out["q" + t] = torch.zeros_like(whole)
            out["q" + t][:, :x.shape[1]] = _exact_blocks(x, c["fmt"], 1, _BLOCK) / whole[:, :x.shape[1]]
            out["scale_t" if t else "scale"] = scale
        return out
    if "E" in c:
        offsets, place, source = _exact_order(s["experts"], c)
        sent = source >= 0
        token = torch.div(source, c["k"], rounding_mode="floor").long()
    if kind == "rows":
        Xs = torch.zeros(source.numel(), c["D"], dtype=torch.double, device="cuda")
        Xs[sent] = s["X"].double()[token[sent]]
        return {"offsets": offsets, "place": place, "source": source, "Xs": Xs}
    if kind in ("sum", "sum_backward"):
        # as the product with the matrix of the weights: choice j of token n
        w = torch.ones(c["N"], c["k"], device="cuda") if s["weights"] is None else s["weights"]
        Ys = s["Ys"].double()
        if kind == "sum":
            Y = torch.zeros(c["N"], c["D"], dtype=torch.double, device="cuda")
            Y.index_add_(0, token[sent], Ys[sent] * w.double().reshape(-1)[source[sent].long()].unsqueeze(1))
            return {"Y": Y}
        dYs, dw, rows = torch.zeros_like(Ys), torch.zeros(c["N"] * c["k"], dtype=torch.double, device="cuda"), s["dY"].double()
        dYs[sent] = rows[token[sent]] * w.double().reshape(-1)[source[sent].long()].unsqueeze(1)
        dw[source[sent].long()] = torch.linalg.vecdot(Ys[sent], rows[token[sent]])
        return {"dYs": dYs} if s["weights"] is None else {"dYs": dYs, "dweights": dw.view(c["N"], c["k"])}
    W = s["W"].double()
    W = torch.stack([_exact_blocks(w, "e4m3", 128, 128) for w in W]) if "E" in c else _exact_blocks(W, "e4m3", 128, 128)
    X = s["X"].double()
    if kind == "linear":
        Y = _exact_blocks(X, c["fmt"], 1, 128) @ W.T
        return {"Y": Y if s["bias"] is None else Y + s["bias"].double()}
    if kind == "experts":
        Y = torch.zeros(source.numel(), c["M"], dtype=torch.double, device="cuda")
        rows = torch.where(sent.unsqueeze(1), X[token.clamp(min=0)], torch.zeros(1, dtype=torch.double, device="cuda"))
        rows = _exact_blocks(rows, c["fmt"], 1, 128)
        for e, (i, j) in enumerate(zip(offsets.tolist(), offsets.tolist()[1:])):
            Y[i:j] = rows[i:j] @ W[e].T
            if s["bias"] is not None:
                Y[i:j] += s["bias"][e].double()
        return {"offsets": offsets, "Y": Y}
    dY = s["dY"].double()
    d, dt, xt = (_exact_blocks(dY, c["fmt"], 1, 128), _exact_blocks(dY.T.contiguous(), c["fmt"], 1, 128),
                 _exact_blocks(X.T.contiguous(), "e4m3", 1, 128))
    if kind == "linear_backward":
        return {"dX": d @ W, "dW": dt @ xt.T}
    dX, dW = torch.zeros_like(X), torch.zeros_like(W)
    for e, (i, j) in enumerate(zip(offsets.tolist(), offsets.tolist()[1:])):
        dX[i:j], dW[e] = d[i:j] @ W[e], dt[:, i:j] @ xt[:, i:j].T
    return {"dX": dX, "dW": dW}
