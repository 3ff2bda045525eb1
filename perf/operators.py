"""The measured work of the operators beside the block-sparse product: the
residual step between two blocks of a transformer layer (``bsr_residual_norm``
and its backward pass) and the gated feed-forward block (``bsr_gated`` and its
backward pass).

Sizes are those of the repository's workloads (768, 1024 and 4096 features, 128
to 16384 tokens), with single tokens, small batches and ragged sizes beside
them; ``draw`` varies all of them.

A case is a dict of plain values:
  kind      "norm", "norm_backward", "gated" or "gated_backward"
  N         tokens
  dtype     "f32" or "bf16": the block's type (y, z, gate; X, weights, H)
 norms:
  D         features
  stream    the residual stream's type
  post, pre "none", "layer" or "rms": the norms after and before the block
  gate      tokens that share a row of the gate (0: no gate)
  scale     whether there is a residual scale for each feature
  alpha     factor of the incoming stream
  bias      whether the norms add a bias
 gated blocks:
  F, K      features of the block and of its input
  act       "silu", "gelu", "gelu_tanh", "relu" or "sigmoid"
  bias      whether the projections add a bias
"""
import math

import torch

own = False

_TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
_EPS = 1e-5


def _norm(name, kind, N, D, dtype, stream, post, pre, gate=0, scale=False, alpha=1.0, bias=True):
    c = dict(kind=kind, N=N, D=D, dtype=dtype, stream=stream, post=post, pre=pre, gate=gate, scale=scale, alpha=alpha,
             bias=bias)
    return dict(c, name=name) if name else c


def _gated(name, kind, N, F, K, dtype, act, bias):
    c = dict(kind=kind, N=N, F=F, K=K, dtype=dtype, act=act, bias=bias)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token of a served request between two blocks: latency
        _norm("norm_bf16_n1", "norm", 1, 1024, "bf16", "bf16", "rms", "rms", scale=True, bias=False),
        # a short sentence, BERT-base width, norms before and after the block
        _norm("norm_f32_n128", "norm", 128, 768, "f32", "f32", "layer", "layer", scale=True),
        # a large batch of BERT-large width with a gate for each sequence of 512 tokens
        _norm("norm_bf16_n16384", "norm", 16384, 1024, "bf16", "bf16", "rms", "rms", gate=512, bias=False),
        # a ragged batch's training step, post-norm scaled by feature, a stream that is scaled down
        _norm("norm_bwd_f32_n1000", "norm_backward", 1000, 768, "f32", "f32", "layer", "layer", scale=True, alpha=0.75),
        # a large training batch: bf16 block on an fp32 stream, gate for each sequence
        _norm("norm_bwd_mixed_n16384", "norm_backward", 16384, 1024, "bf16", "f32", "rms", "layer", gate=512, scale=True),
        # one token of a served request: reading the weights is the work
        _gated("gated_bf16_n1", "gated", 1, 4096, 1024, "bf16", "silu", False),
        # a handful of tokens in fp32
        _gated("gated_f32_n5", "gated", 5, 4096, 1024, "f32", "gelu", True),
        # a short sentence
        _gated("gated_bf16_n128", "gated", 128, 2048, 768, "bf16", "silu", True),
        # a ragged batch in fp32
        _gated("gated_f32_n1000", "gated", 1000, 2048, 768, "f32", "gelu_tanh", True),
        # a large batch
        _gated("gated_bf16_n8192", "gated", 8192, 4096, 1024, "bf16", "silu", False),
        # a small training step with odd sizes
        _gated("gated_bwd_f32_n999", "gated_backward", 999, 2050, 770, "f32", "gelu", True),
        # a large training step
        _gated("gated_bwd_bf16_n8192", "gated_backward", 8192, 4096, 1024, "bf16", "silu", True),
    ]


def draw(rng):
    """Another case of the same ranges: 1 to 16384 tokens (8192 for gated
    blocks), 64 to 4096 features of a stream, 128 to 4096 by 128 to 1536 of a
    gated block, odd sizes among them."""
    def log_int(lo, hi):
        return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))

    def size(lo, hi):   # mostly multiples of 64, as models have; some of 8, some odd
        n, p = log_int(lo, hi), rng.random()
        step = 64 if p < 0.6 else 8 if p < 0.85 else 1
        n = max(lo, n - n % step)
        return n + 64 if n == 3072 else n

    kind = rng.choice(("norm", "norm_backward", "gated", "gated_backward"))
    dtype = rng.choice(("f32", "bf16"))
    if kind.startswith("norm"):
        N, D = log_int(1, 16384), size(64, 4096)
        N = max(1, min(N, 16384 * 1024 // D))
        stream = "f32" if dtype == "f32" or rng.random() < 0.4 else "bf16"
        post, pre = rng.choice((("layer", "layer"), ("rms", "rms"), ("none", "rms"), ("none", "layer"), ("layer", "none"),
                                ("rms", "layer")))
        gate = rng.choice((0, 0, 1, log_int(2, 1024)))
        return _norm(None, kind, N, D, dtype, stream, post, pre, gate, rng.random() < 0.5, rng.choice((1.0, 0.75)),
                     rng.random() < 0.5)
    F, K, N = size(128, 4096), size(128, 1536), log_int(1, 8192)
    most = 12 * 8192 * 4096 * 1024
    N = max(1, min(N, most // ((12 if kind == "gated_backward" else 4) * F * K)))
    act = rng.choice(("silu", "gelu", "gelu_tanh", "relu", "sigmoid"))
    return _gated(None, kind, N, F, K, dtype, act, rng.random() < 0.5)


def _gate_rows(case):
    return -(-case["N"] // case["gate"]) if case["gate"] else 0


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(*shape, std=1.0, mean=0.0):
        return torch.randn(*shape, device="cuda", generator=gen) * std + mean

    dt, N = _TORCH[case["dtype"]], case["N"]
    s = {}
    if case["kind"].startswith("norm"):
        D, st = case["D"], _TORCH[case["stream"]]
        features = normal(D, std=0.5)   # features of a stream differ in their means
        s["y"] = (normal(N, D) + 0.3 * features).to(dt)
        s["h"] = (normal(N, D, std=2.0) + features).to(st)
        s["gate"] = normal(_gate_rows(case), D, std=0.5, mean=0.5).to(dt) if case["gate"] else None
        s["scale"] = normal(D, std=0.2, mean=0.6) if case["scale"] else None
        for side in ("post", "pre"):
            has = case[side] != "none"
            s[side + "_w"] = normal(D, std=0.1, mean=1.0) if has else None
            s[side + "_b"] = normal(D, std=0.1) if has and case["bias"] else None
        if case["kind"] == "norm_backward":
            s["dh_out"] = normal(N, D, std=0.1).to(st)
            s["dz"] = normal(N, D, std=0.1).to(dt) if case["pre"] != "none" else None
        return s
    F, K = case["F"], case["K"]
    s["X"] = normal(N, K).to(dt)
    s["Wg"], s["Wu"] = (normal(F, K, std=0.02).to(dt) for _ in range(2))
    s["bg"], s["bu"] = (normal(F, std=0.02) if case["bias"] else None for _ in range(2))
    if case["kind"] == "gated_backward":
        s["dH"] = normal(N, F, std=0.1).to(dt)
    return s


def prepare(case, seed):
    """The inputs, and the buffers that a program keeps for the outputs."""
    s = dict(_inputs(case, seed), case=case)
    like = torch.empty_like
    if case["kind"] == "norm":
        s["h_out"] = like(s["h"])
        s["z"] = like(s["y"]) if case["pre"] != "none" else None
    elif case["kind"] == "norm_backward":
        s["dy"], s["dh"] = like(s["y"]), like(s["h"])
    elif case["kind"] == "gated":
        s["H"] = torch.empty(case["N"], case["F"], dtype=s["X"].dtype, device="cuda")
    else:
        s["dX"], s["dWg"], s["dWu"] = like(s["X"]), like(s["Wg"]), like(s["Wu"])
    return s


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"norm": _own_norm, "norm_backward": _own_norm_backward, "gated": _own_gated,
                "gated_backward": _own_gated_backward}[kind](state, state["case"])
    return {"norm": _plain_norm, "norm_backward": _plain_norm_backward, "gated": _plain_gated,
            "gated_backward": _plain_gated_backward}[kind](state, state["case"])


# ---- the framework's operators

def _own_norm(s, c):
    import paper_2106_08846_gb300 as bsr
    h_out, z = bsr.bsr_residual_norm(s["y"], s["h"], gate=s["gate"], gate_tokens=c["gate"], scale=s["scale"],
                                     alpha=c["alpha"], post=c["post"], post_w=s["post_w"], post_b=s["post_b"], pre=c["pre"],
                                     pre_w=s["pre_w"], pre_b=s["pre_b"], eps=_EPS, h_out=s["h_out"], z=s["z"])
    return {"h_out": h_out} if z is None else {"h_out": h_out, "z": z}


def _own_norm_backward(s, c):
    import paper_2106_08846_gb300 as bsr
    return bsr.bsr_residual_norm_backward(s["y"], s["h"], s["dh_out"], s["dz"], gate=s["gate"], gate_tokens=c["gate"],
                                          scale=s["scale"], alpha=c["alpha"], post=c["post"], post_w=s["post_w"],
                                          post_b=s["post_b"], pre=c["pre"], pre_w=s["pre_w"], pre_b=s["pre_b"], eps=_EPS,
                                          dy=s["dy"], dh=s["dh"])


def _own_gated(s, c):
    import paper_2106_08846_gb300 as bsr
    return {"H": bsr.bsr_gated(s["X"], s["Wg"], s["Wu"], s["bg"], s["bu"], act=c["act"], H=s["H"])}


def _own_gated_backward(s, c):
    import paper_2106_08846_gb300 as bsr
    return bsr.bsr_gated_backward(s["X"], s["Wg"], s["Wu"], s["bg"], s["bu"], s["dH"], act=c["act"], dX=s["dX"],
                                  dWg=s["dWg"], dWu=s["dWu"])


# ---- their plain forms: 32 bits, rounded once at the end

def _f32(t):
    return None if t is None else t.float()


def _plain_stats(x, how):
    """Normalised rows and the factor 1 / deviation."""
    if how == "layer":
        x = x - x.mean(1, keepdim=True)
    r = torch.rsqrt((x * x).mean(1, keepdim=True) + _EPS)
    return x * r, r


def _plain_affine(xh, w, b):
    return xh * w if b is None else xh * w + b


def _plain_gate_rows(s, c):
    """The gate's row of each token."""
    return torch.arange(c["N"], device="cuda") // c["gate"]


def _plain_norm(s, c):
    t = _f32(s["y"])
    if c["post"] != "none":
        t = _plain_affine(_plain_stats(t, c["post"])[0], s["post_w"], s["post_b"])
    if c["gate"]:
        t = t * _f32(s["gate"])[_plain_gate_rows(s, c)]
    if c["scale"]:
        t = t * s["scale"]
    h = c["alpha"] * _f32(s["h"]) + t
    out = {"h_out": h.to(s["h"].dtype)}
    if c["pre"] != "none":
        out["z"] = _plain_affine(_plain_stats(h, c["pre"])[0], s["pre_w"], s["pre_b"]).to(s["y"].dtype)
    return out


def _plain_norm_grad(g, xh, r, how):
    """The gradient of a norm's input; g that of the normalised rows."""
    d = g - xh * (g * xh).mean(1, keepdim=True)
    if how == "layer":
        d = d - g.mean(1, keepdim=True)
    return d * r


def _plain_norm_backward(s, c):
    """Of the stream that the forward pass returned (here "h")."""
    out, dH = {}, _f32(s["dh_out"])
    if c["pre"] != "none":
        hh, r = _plain_stats(_f32(s["h"]), c["pre"])
        dz = _f32(s["dz"])
        dH = dH + _plain_norm_grad(dz * s["pre_w"], hh, r, c["pre"])
        out["dpre_w"] = (dz * hh).sum(0)
        if c["bias"]:
            out["dpre_b"] = dz.sum(0)
    out["dh"] = (c["alpha"] * dH).to(s["h"].dtype)
    y = t = _f32(s["y"])
    if c["post"] != "none":
        yh, r = _plain_stats(y, c["post"])
        t = _plain_affine(yh, s["post_w"], s["post_b"])
    dt = dH
    if c["gate"]:
        rows = _plain_gate_rows(s, c)
        gate = _f32(s["gate"])[rows]
        each = t * dH if s["scale"] is None else t * dH * s["scale"]
        whole = torch.zeros(_gate_rows(c) * c["gate"], c["D"], device="cuda")
        whole[:c["N"]] = each
        out["dgate"] = whole.view(-1, c["gate"], c["D"]).sum(1).to(s["gate"].dtype)
        dt = dt * gate
    if c["scale"]:
        out["dscale"] = (t * dt).sum(0)
        dt = dt * s["scale"]
    if c["post"] != "none":
        out["dpost_w"] = (dt * yh).sum(0)
        if c["bias"]:
            out["dpost_b"] = dt.sum(0)
        dt = _plain_norm_grad(dt * s["post_w"], yh, r, c["post"])
    out["dy"] = dt.to(s["y"].dtype)
    return out


def _plain_act(g, act, slope=False):
    """The activation, and with `slope` its derivative too."""
    if act == "relu":
        a = torch.where(g > 0, g, torch.zeros_like(g))
        return (a, (g > 0).to(g.dtype)) if slope else a
    if act in ("silu", "sigmoid"):
        p = 1 / (1 + torch.exp(-g))
        a = p if act == "sigmoid" else g * p
        if not slope:
            return a
        return (a, p * (1 - p)) if act == "sigmoid" else (a, p * (1 + g * (1 - p)))
    if act == "gelu":
        p = 0.5 * (1 + torch.erf(g * math.sqrt(0.5)))
        if not slope:
            return g * p
        return g * p, p + g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)
    k = math.sqrt(2 / math.pi)
    th = torch.tanh(k * (g + 0.044715 * g * g * g))
    if not slope:
        return 0.5 * g * (1 + th)
    return 0.5 * g * (1 + th), 0.5 * (1 + th) + 0.5 * g * (1 - th * th) * k * (1 + 3 * 0.044715 * g * g)


def _plain_project(X, W, b):
    P = X @ W.T
    return P if b is None else P + b


def _plain_gated(s, c):
    X = _f32(s["X"])
    G = _plain_project(X, _f32(s["Wg"]), s["bg"])
    U = _plain_project(X, _f32(s["Wu"]), s["bu"])
    return {"H": (_plain_act(G, c["act"]) * U).to(s["X"].dtype)}


def _plain_gated_backward(s, c):
    X, Wg, Wu, dH = (_f32(s[k]) for k in ("X", "Wg", "Wu", "dH"))
    a, slope = _plain_act(_plain_project(X, Wg, s["bg"]), c["act"], slope=True)
    dG = dH * _plain_project(X, Wu, s["bu"]) * slope
    dU = dH * a
    dt = s["X"].dtype
    out = {"dX": (dG @ Wg + dU @ Wu).to(dt), "dWg": (dG.T @ X).to(dt), "dWu": (dU.T @ X).to(dt)}
    if c["bias"]:
        out["dbg"], out["dbu"] = dG.sum(0), dU.sum(0)
    return out


# ---- what they cannot do without, and their values in 64 bits

def work(case):
    es, N = 4 if case["dtype"] == "f32" else 2, case["N"]
    if case["kind"].startswith("norm"):
        D, ss = case["D"], 4 if case["stream"] == "f32" else 2
        norms = [case[side] != "none" for side in ("post", "pre")]
        params = 4 * D * (sum(norms) * (2 if case["bias"] else 1) + case["scale"])
        gate = _gate_rows(case) * D * es
        if case["kind"] == "norm":   # y, h -> h_out, z
            rows = N * D * (es + 2 * ss + (es if norms[1] else 0))
            return {"bytes": rows + gate + params, "flops": N * D * (3 + 6 * sum(norms))}
        # y, dh_out (with a pre norm h_out and dz) -> dy, dh, and every parameter's gradient
        rows = N * D * (2 * es + 2 * ss + ((es + ss) if norms[1] else 0))
        return {"bytes": rows + 2 * (gate + params), "flops": N * D * (8 + 16 * sum(norms))}
    F, K = case["F"], case["K"]
    bias = 8 * F if case["bias"] else 0
    if case["kind"] == "gated":
        return {"bytes": es * (N * K + 2 * F * K + N * F) + bias, "flops": 4 * N * F * K}
    return {"bytes": es * (2 * N * K + 4 * F * K + N * F) + 2 * bias, "flops": 12 * N * F * K}


def _exact_rows(x, how, w, b):
    if how == "none":
        return x
    m = x.mean(-1, keepdim=True) if how == "layer" else 0.0
    out = (x - m) / ((x - m).pow(2).mean(-1, keepdim=True) + _EPS).sqrt() * w
    return out if b is None else out + b


def exact(case, seed):
    """The definitions in double precision; gradients by automatic differentiation."""
    s = {k: None if v is None else v.double() for k, v in _inputs(case, seed).items()}
    back = case["kind"].endswith("backward")
    if case["kind"].startswith("norm"):
        N, D = case["N"], case["D"]

        def joined(y, gate, scale, w, b):
            t = _exact_rows(y, case["post"], w, b)
            if scale is not None:
                t = t * scale
            return t if gate is None else t * gate.repeat_interleave(case["gate"], 0)[:N]

        if not back:
            h = case["alpha"] * s["h"] + joined(s["y"], s["gate"], s["scale"], s["post_w"], s["post_b"])
            z = _exact_rows(h, case["pre"], s["pre_w"], s["pre_b"])
            return {"h_out": h} if case["pre"] == "none" else {"h_out": h, "z": z}
        # first the stream that was returned, then the two that made it
        leaves = {"dh": s["h"], "dpre_w": s["pre_w"], "dpre_b": s["pre_b"]}
        dH, out = s["dh_out"], {}
        if case["pre"] != "none":
            leaves = {k: v.requires_grad_() for k, v in leaves.items() if v is not None}
            z = _exact_rows(s["h"], case["pre"], s["pre_w"], s["pre_b"])
            out = dict(zip(leaves, torch.autograd.grad(z, list(leaves.values()), s["dz"])))
            dH = dH + out["dh"]
        out["dh"] = case["alpha"] * dH
        leaves = {"dy": s["y"], "dgate": s["gate"], "dscale": s["scale"], "dpost_w": s["post_w"], "dpost_b": s["post_b"]}
        leaves = {k: v.requires_grad_() for k, v in leaves.items() if v is not None}
        t = joined(s["y"], s["gate"], s["scale"], s["post_w"], s["post_b"])
        return dict(out, **dict(zip(leaves, torch.autograd.grad(t, list(leaves.values()), dH))))
    act = {"silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu, "relu": torch.relu, "sigmoid": torch.sigmoid,
           "gelu_tanh": lambda g: torch.nn.functional.gelu(g, approximate="tanh")}[case["act"]]
    dH = s.pop("dH", None)
    if back:
        s = {k: None if v is None else v.requires_grad_() for k, v in s.items()}
    linear = torch.nn.functional.linear
    H = act(linear(s["X"], s["Wg"], s["bg"])) * linear(s["X"], s["Wu"], s["bu"])
    if not back:
        return {"H": H}
    leaves = {"d" + k: v for k, v in s.items() if v is not None}
    return dict(zip(leaves, torch.autograd.grad(H, list(leaves.values()), dH)))
