"""bsr_residual_norm and its backward pass against the definitions in 64 bits,
element by element, and the gradients against differences of the forward pass."""
import ctypes

import pytest
import torch

import paper_2106_08846_gb300 as bsr

pytestmark = pytest.mark.gpu
U = 2.0 ** -24   # half an fp32 unit in the last place, relative
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def make(N, D, block, stream, post, pre, gate=0, scale=False, bias=True, weight=True, seed=0, mean=0.5):
    g = torch.Generator(device="cuda").manual_seed(1000 * N + D + seed)

    def normal(*shape, std=1.0, m=0.0):
        return torch.randn(*shape, generator=g, device="cuda") * std + m

    s = dict(y=normal(N, D, m=mean).to(DT[block]), h=normal(N, D, std=2.0, m=-mean).to(DT[stream]),
             dh_out=normal(N, D).to(DT[stream]), dz=normal(N, D).to(DT[block]) if pre != "none" else None)
    p = dict(post=post, pre=pre, alpha=0.75, eps=1e-5,
             gate=normal(-(-N // gate), D, m=0.5).to(DT[block]) if gate else None, gate_tokens=gate or 1,
             scale=normal(D, std=0.3, m=0.7) if scale else None)
    for side, how in (("post", post), ("pre", pre)):
        p[side + "_w"] = normal(D, std=0.2, m=1.0) if how != "none" and weight else None
        p[side + "_b"] = normal(D, std=0.2) if how != "none" and bias else None
    return s, p


def f64(t, like):
    return torch.zeros_like(like, dtype=torch.float64) if t is None else t.double()


def ones(t, D):
    return torch.ones(D, dtype=torch.float64, device="cuda") if t is None else t.double()


def zeros(t, D):
    return torch.zeros(D, dtype=torch.float64, device="cuda") if t is None else t.double()


def stats(x, how, eps):
    """Normalised rows, 1 / deviation, and how much a unit of rounding grows in them: the
    mean's rounding is relative to the mean of |x|, and comes divided by the deviation."""
    m = x.mean(1, keepdim=True) if how == "layer" else 0.0
    r = 1 / ((x - m).square().mean(1, keepdim=True) + eps).sqrt()
    return (x - m) * r, r, 1 + (x.abs().mean(1, keepdim=True) * r if how == "layer" else 0.0)


def gate_rows(p, N, D):
    if p["gate"] is None:
        return torch.ones(N, D, dtype=torch.float64, device="cuda")
    return p["gate"].double()[torch.arange(N, device="cuda") // p["gate_tokens"]]


def reference(s, p):
    """(h', z) in 64 bits and the magnitudes that their roundings are relative to."""
    y, h = s["y"].double(), f64(s["h"], s["y"])
    N, D = y.shape
    t, mt = y, y.abs()
    if p["post"] != "none":
        yh, _, grow = stats(y, p["post"], p["eps"])
        w, b = ones(p["post_w"], D), zeros(p["post_b"], D)
        t, mt = yh * w + b, (yh.abs() + grow) * w.abs() + b.abs()
    gs = gate_rows(p, N, D) * ones(p["scale"], D)
    h2, mh = p["alpha"] * h + gs * t, (p["alpha"] * h).abs() + gs.abs() * mt
    if p["pre"] == "none":
        return h2, mh, None, None
    hh, r, grow = stats(h2, p["pre"], p["eps"])
    w, b = ones(p["pre_w"], D), zeros(p["pre_b"], D)
    # the error of h' itself comes in divided by the deviation, in the row and in its statistics
    mz = w.abs() * (hh.abs() + grow + r * mh + (1 + hh.abs()) * r * mh.mean(1, keepdim=True)) + b.abs()
    return h2, mh, hh * w + b, mz


def close(got, want, mag, factor, rounds):
    """|got - want| <= factor U mag, and half a unit of bf16 where the value is rounded to it."""
    bound = factor * U * mag + (2.0 ** -8 * want.abs() + 1e-30 if rounds else 0.0)
    bad = (got.double() - want).abs() > bound
    assert torch.isfinite(got).all()
    assert not bad.any(), (int(bad.sum()), got.double()[bad][:3], want[bad][:3], bound[bad][:3])


def check_forward(s, p, **more):
    h_out, z = bsr.bsr_residual_norm(s["y"], s["h"], **p, **more)
    h2, mh, zz, mz = reference(s, p)
    # sums run over at most 16 + 5 + 32 additions in sequence and their tree: 64 roundings; a handful more a value
    close(h_out, h2, mh, 128, h_out.dtype == torch.bfloat16)
    if zz is not None:
        close(z, zz, mz, 128, z.dtype == torch.bfloat16)
    else:
        assert z is None
    return h_out, z


TYPES = [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")]
NORMS = [("none", "rms"), ("layer", "none"), ("layer", "layer"), ("rms", "rms"), ("none", "none"), ("rms", "layer")]


@pytest.mark.parametrize("block,stream", TYPES)
@pytest.mark.parametrize("D", [1, 8, 31, 64, 100, 768, 1024, 1193, 4096, 4104, 8200, 16384, 16383])
def test_forward_widths(D, block, stream):
    for k, (post, pre) in enumerate(NORMS):
        check_forward(*make(5, D, block, stream, post, pre, gate=(0, 1, 2)[k % 3], scale=k % 2 == 0, bias=k % 2 == 1, seed=k))


@pytest.mark.parametrize("block,stream", TYPES)
@pytest.mark.parametrize("N", [1, 2, 7, 33, 1000, 5000])
def test_forward_tokens(N, block, stream):
    check_forward(*make(N, 768, block, stream, "rms", "layer", gate=max(1, N // 3), scale=True))
    check_forward(*make(N, 96, block, stream, "layer", "rms", gate=512))


def test_forward_without_stream_and_plain_norm():
    s, p = make(9, 320, "bf16", "bf16", "none", "layer")
    s["h"] = None
    check_forward(s, p)
    # z alone, through the C function: a plain norm
    s, p = make(9, 320, "f32", "f32", "none", "rms", weight=False, bias=False)
    z = torch.empty_like(s["y"])
    c = bsr.bsrlib._ResidualNorm(320, 0, 0, 0, 0, 2, 0.0, 1e-5, 1.0)
    assert bsr.load().bsr_residual_norm(c, s["y"].data_ptr(), None, None, None, z.data_ptr(), 9, None) == 0
    want = torch.nn.functional.rms_norm(s["y"].double(), (320,), eps=1e-5)
    close(z, want, want.abs() + 1, 128, False)


def test_forward_in_place_on_a_stream_and_without_tokens():
    s, p = make(300, 768, "bf16", "bf16", "rms", "rms", gate=100)
    h1, z1 = bsr.bsr_residual_norm(s["y"], s["h"], **p)
    y, h = s["y"].clone(), s["h"].clone()
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    h2, z2 = bsr.bsr_residual_norm(y, h, **p, h_out=h, z=y, stream=other)
    other.synchronize()
    assert h2 is h and z2 is y and torch.equal(h1, h) and torch.equal(z1, y)
    s, p = make(0, 768, "bf16", "f32", "rms", "rms")
    h_out, z = bsr.bsr_residual_norm(s["y"], s["h"], **p)
    assert h_out.shape == z.shape == (0, 768)


def test_parameters_on_odd_addresses_and_large_means():
    s, p = make(40, 768, "f32", "f32", "layer", "layer", scale=True, mean=100.0)
    want = check_forward(s, p)
    for k in ("scale", "post_w", "pre_b"):   # 4-byte aligned only
        at = torch.empty(769, device="cuda")
        at[1:] = p[k]
        p[k] = at[1:]
    got = check_forward(s, p)
    h2, mh, _, _ = reference(s, p)
    close(got[0], want[0].double(), mh, 256, False)


def test_a_bad_row_leaves_the_others_alone():
    s, p = make(64, 768, "bf16", "f32", "layer", "rms", gate=16)
    clean = bsr.bsr_residual_norm(s["y"], s["h"], **p)
    s["y"][5, 7], s["h"][9, 0], s["y"][11, 3] = float("nan"), float("inf"), float("-inf")
    got = bsr.bsr_residual_norm(s["y"], s["h"], **p)
    rows = torch.tensor([n for n in range(64) if n not in (5, 9, 11)], device="cuda")
    for a, b in zip(clean, got):
        assert torch.equal(a[rows], b[rows])
    assert torch.isnan(got[1][5]).all() and torch.isnan(got[1][11]).all() and torch.isinf(got[0][9, 0])


# ---- backward

def reference_backward(s, p, h_out):
    """{name: (value, magnitude of its terms)} in 64 bits; for sums the sums of both."""
    y = s["y"].double()
    N, D = y.shape
    dH, m = f64(s["dh_out"], y), f64(s["dh_out"], y).abs()
    out = {}

    def norm_grad(g, mg, xh, r, grow, how):
        mean = lambda v: v.mean(1, keepdim=True)  # noqa: E731
        d = r * (g - (mean(g) if how == "layer" else 0.0) - xh * mean(g * xh))
        x = xh.abs() + grow   # a normalised value's own roundings
        return d, r * (mg + mean(mg) + x * mean(mg * x)) * grow

    if p["pre"] != "none":
        hh, r, grow = stats(h_out.double(), p["pre"], p["eps"])
        dz, w = s["dz"].double(), ones(p["pre_w"], D)
        out["dpre_w"] = (dz * hh).sum(0), (dz.abs() * (hh.abs() + grow)).sum(0)
        out["dpre_b"] = dz.sum(0), dz.abs().sum(0)
        d, md = norm_grad(dz * w, (dz * w).abs(), hh, r, grow, p["pre"])
        dH, m = dH + d, m + md
    out["dh"] = p["alpha"] * dH, abs(p["alpha"]) * m
    t, mt, w = y, y.abs(), ones(p["post_w"], D)
    if p["post"] != "none":
        yh, r, grow = stats(y, p["post"], p["eps"])
        b = zeros(p["post_b"], D)
        t, mt = yh * w + b, (yh.abs() + grow) * w.abs() + b.abs()
    gate, sc = gate_rows(p, N, D), ones(p["scale"], D)
    rows = torch.arange(N, device="cuda") // p["gate_tokens"]
    R = -(-N // p["gate_tokens"])
    add = lambda v: torch.zeros(R, D, dtype=torch.float64, device="cuda").index_add_(0, rows, v)  # noqa: E731
    out["dgate"] = add(sc * t * dH), add(sc.abs() * mt * m)
    out["dscale"] = (gate * t * dH).sum(0), (gate.abs() * mt * m).sum(0)
    dt, mdt = gate * sc * dH, (gate * sc).abs() * m
    if p["post"] != "none":
        out["dpost_w"] = (dt * yh).sum(0), (mdt * (yh.abs() + grow)).sum(0)
        out["dpost_b"] = dt.sum(0), mdt.sum(0)
        dt, mdt = norm_grad(dt * w, mdt * w.abs(), yh, r, grow, p["post"])
    out["dy"] = dt, mdt
    return out


def check_backward(s, p, **more):
    h_out = bsr.bsr_residual_norm(s["y"], s["h"], **p)[0]
    got = bsr.bsr_residual_norm_backward(s["y"], h_out, s["dh_out"], s["dz"], **p, **more)
    want = reference_backward(s, p, h_out)
    given = {"dy", "dh"} | {"d" + k for k in ("gate", "scale", "post_w", "post_b", "pre_w", "pre_b") if p[k] is not None}
    assert set(got) == given
    N = s["y"].shape[0]
    for k in sorted(given):
        v, m = want[k]
        assert got[k].shape == v.shape
        # a value: two norms' sums of up to 64 roundings each and those of the formula; a sum: as many more as terms
        close(got[k], v, m, 512 + (N if k not in ("dy", "dh") else 0), got[k].dtype == torch.bfloat16)
    return got


@pytest.mark.parametrize("block,stream", TYPES)
@pytest.mark.parametrize("D", [1, 8, 31, 64, 768, 1193, 4096, 4104, 16384, 16383])
def test_backward_widths(D, block, stream):
    for k, (post, pre) in enumerate(NORMS):
        check_backward(*make(5, D, block, stream, post, pre, gate=(0, 1, 2)[k % 3], scale=k % 2 == 0, bias=k % 2 == 1, seed=k))


@pytest.mark.parametrize("block,stream", TYPES)
@pytest.mark.parametrize("N,gate", [(1, 1), (2, 7), (7, 3), (33, 0), (1000, 1), (1000, 999), (5000, 512), (5000, 2), (5000, 0)])
def test_backward_tokens(N, gate, block, stream):
    check_backward(*make(N, 768, block, stream, "rms", "layer", gate=gate, scale=True))
    check_backward(*make(N, 72, block, stream, "layer", "rms", gate=gate, scale=N % 2 == 0))


@pytest.mark.parametrize("block,stream", TYPES)
@pytest.mark.parametrize("D,gate", [(4104, 0), (5120, 30), (8192, 1), (8191, 16), (8200, 0), (12288, 64), (16384, 1), (16383, 50)])
def test_backward_wide_rows(D, gate, block, stream):
    # several rows to each group of threads that works on them
    check_backward(*make(200, D, block, stream, "layer", "rms", gate=gate, scale=True))
    check_backward(*make(151, D, block, stream, "rms", "layer", gate=gate, bias=False))


@pytest.mark.parametrize("block,stream", TYPES)
def test_gate_rows_longer_than_the_tokens_left(block, stream):
    # a last row of fewer tokens than the others, and one row for far more tokens than there are
    for N, gate in ((600, 512), (1030, 1024), (50, 2**63 - 1)):
        args = make(N, 264, block, stream, "rms", "layer", gate=gate, scale=True)
        check_forward(*args)
        check_backward(*args)


def test_backward_repeats_to_the_bit_and_in_place_on_a_stream():
    s, p = make(3000, 768, "bf16", "f32", "rms", "layer", gate=700, scale=True)
    h_out = bsr.bsr_residual_norm(s["y"], s["h"], **p)[0]
    one = bsr.bsr_residual_norm_backward(s["y"], h_out, s["dh_out"], s["dz"], **p)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    y, dh = s["y"].clone(), s["dh_out"].clone()
    other.wait_stream(torch.cuda.current_stream())
    two = bsr.bsr_residual_norm_backward(y, h_out, dh, s["dz"], **p, dy=y, dh=dh, stream=other)
    other.synchronize()
    assert two["dy"] is y and two["dh"] is dh
    for k in one:
        assert torch.equal(one[k], two[k]), k


def test_backward_without_tokens_and_without_some_gradients():
    s, p = make(0, 768, "bf16", "bf16", "rms", "layer", gate=4, scale=True)
    got = bsr.bsr_residual_norm_backward(s["y"], s["h"], s["dh_out"], s["dz"], **p)
    for k in ("dscale", "dpost_w", "dpost_b", "dpre_w", "dpre_b"):
        assert got[k].shape == (768,) and not got[k].any()
    # dh_out None: only z is read downstream
    s, p = make(50, 768, "f32", "f32", "rms", "rms")
    s["dh_out"] = None
    check_backward(s, p)
    # the C function leaves out what is NULL
    c = bsr.bsrlib._ResidualNorm(768, 0, 0, 0, 2, 0, 1e-5, 0.0, 1.0, None, p["post_w"].data_ptr())
    s, _ = make(50, 768, "f32", "f32", "rms", "none")
    dy = torch.empty_like(s["y"])
    assert bsr.load().bsr_residual_norm_backward(c, s["y"].data_ptr(), None, None, s["dh_out"].data_ptr(), None, dy.data_ptr(),
                                                 None, None, 50, torch.empty(1 << 22, device="cuda").data_ptr(), 1 << 24,
                                                 None) == 0
    yh, r, grow = stats(s["y"].double(), "rms", 1e-5)
    g = s["dh_out"].double() * p["post_w"].double()
    want = r * (g - yh * (g * yh).mean(1, keepdim=True))
    close(dy, want, r * (g.abs() + yh.abs() * (g * yh).abs().mean(1, keepdim=True)), 512, False)


@pytest.mark.parametrize("post,pre,gate", [("layer", "rms", 3), ("rms", "layer", 1), ("none", "layer", 0), ("layer", "none", 100)])
def test_gradients_against_differences(post, pre, gate):
    """(L(x + e v) - L(x - e v)) / 2e of L = sum h' dh' + sum z dz against <gradient, v>."""
    s, p = make(24, 96, "f32", "f32", post, pre, gate=gate, scale=True)
    h_out = bsr.bsr_residual_norm(s["y"], s["h"], **p)[0]
    grads = bsr.bsr_residual_norm_backward(s["y"], h_out, s["dh_out"], s["dz"], **p)
    g = torch.Generator(device="cuda").manual_seed(5)

    def L(s, p):
        h2, z = bsr.bsr_residual_norm(s["y"], s["h"], **p)
        v = (h2.double() * s["dh_out"].double()).sum()
        return float(v if z is None else v + (z.double() * s["dz"].double()).sum())

    e = 2.0 ** -8
    for name, grad in grads.items():
        x = (s if name in ("dy", "dh") else p)[name[1:]]
        v = torch.randn(x.shape, generator=g, device="cuda")
        out = []
        for sign in (1, -1):
            where, moved = (dict(s), dict(p)), x + sign * e * v
            where[0 if name in ("dy", "dh") else 1][name[1:]] = moved
            out.append(L(*where))
        want = float((grad.double() * v.double()).sum())
        # the third derivative's share, and the outputs' roundings (2^-24 each of about 4600 terms of order 1) over 2e
        assert abs((out[0] - out[1]) / (2 * e) - want) <= 2e-3 * float(grad.double().norm() * v.double().norm()) + 0.01, name


def test_refusals_on_the_device():
    L = bsr.load()
    from paper_2106_08846_gb300.bsrlib import BSR_ERR_ALIGNMENT, BSR_ERR_CAPACITY, BSR_ERR_INVALID_ARG, _ResidualNorm
    y, h, z = (torch.zeros(4, 64, device="cuda") for _ in range(3))
    ws = torch.zeros(1 << 16, device="cuda")
    c = _ResidualNorm(64, 0, 0, 0, 0, 2, 0.0, 1e-5, 1.0)
    P = lambda t, off=0: t.data_ptr() + off  # noqa: E731
    assert L.bsr_residual_norm(c, P(y, 4), None, None, None, P(z), 2, None) == BSR_ERR_ALIGNMENT
    assert L.bsr_residual_norm(c, P(y), None, None, P(y), P(z), 4, None) == BSR_ERR_INVALID_ARG      # h_out on y
    assert L.bsr_residual_norm(c, P(y), P(h), None, P(h, 256), P(z), 3, None) == BSR_ERR_INVALID_ARG  # h_out across h
    assert L.bsr_residual_norm(c, P(y), P(h), None, P(z), P(z), 4, None) == BSR_ERR_INVALID_ARG      # both outputs
    host = torch.zeros(4, 64).pin_memory()
    assert L.bsr_residual_norm(c, host.data_ptr(), None, None, None, P(z), 4, None) == BSR_ERR_INVALID_ARG
    n = ctypes.c_size_t(0)
    assert L.bsr_residual_norm_workspace(c, 4, ctypes.byref(n)) == 0 and n.value > 0
    args = (c, P(y), P(h), None, None, P(y), P(z), None, None, 4)
    assert L.bsr_residual_norm_backward(*args, P(ws), n.value - 1, None) == BSR_ERR_CAPACITY
    assert L.bsr_residual_norm_backward(*args, None, n.value, None) == BSR_ERR_INVALID_ARG
    assert L.bsr_residual_norm_backward(*args, P(y), n.value, None) == BSR_ERR_INVALID_ARG
    for bad in (dict(y=y.t()), dict(h=h.double()), dict(h=h[:2]), dict(gate=y, gate_tokens=4), dict(pre="batch"),
                dict(scale=torch.zeros(63, device="cuda"))):
        with pytest.raises((TypeError, ValueError)):
            bsr.bsr_residual_norm(**dict(dict(y=y, h=h), **bad))
    torch.cuda.synchronize()
