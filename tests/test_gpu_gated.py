"""bsr_gated and its backward pass against the definitions in 64 bits, element by
element, and the gradients against differences of the forward pass."""
import ctypes
import math

import pytest
import torch

import paper_2106_08846_gb300 as bsr
from paper_2106_08846_gb300 import bsrlib

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
ACTS = ["silu", "gelu", "gelu_tanh", "relu", "sigmoid"]
SUM = 1e-5             # a sum of products: this times the sum of their sizes, as for the block-sparse product
FUN = 2.0 ** -20       # an activation or its derivative: this times 1 + |g|
CURVE = {"silu": 0.51, "gelu": 0.81, "gelu_tanh": 0.82, "relu": 0.0, "sigmoid": 0.1}   # largest |act''|


def make(N, F, K, dtype, bias=True, seed=0, wide=1.0):
    g = torch.Generator(device="cuda").manual_seed(7919 * N + 31 * F + K + seed)
    normal = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    dt = DT[dtype]
    s = dict(X=normal(N, K).to(dt), Wg=(normal(F, K) * wide / math.sqrt(K)).to(dt), Wu=(normal(F, K) / math.sqrt(K)).to(dt),
             bg=normal(F) * 0.3 if bias else None, bu=normal(F) * 0.3 if bias else None)
    return s, normal(N, F).to(dt)


def act64(g, act):
    """act, act' and act'' bounds in 64 bits."""
    if act == "silu":
        p = torch.sigmoid(g)
        return g * p, p * (1 + g * (1 - p))
    if act == "sigmoid":
        p = torch.sigmoid(g)
        return p, p * (1 - p)
    if act == "relu":
        return g.clamp(min=0), (g > 0).double()
    if act == "gelu":
        p = 0.5 * torch.erfc(-g / math.sqrt(2))
        return g * p, p + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    k = math.sqrt(2 / math.pi)
    th = torch.tanh(k * (g + 0.044715 * g ** 3))
    return 0.5 * g * (1 + th), 0.5 * (1 + th) + 0.5 * g * (1 - th * th) * k * (1 + 3 * 0.044715 * g * g)


def project(X, W, b):
    P, m = X.double() @ W.double().T, X.double().abs() @ W.double().abs().T
    return (P, m) if b is None else (P + b.double(), m + b.double().abs())


def near(got, want, bound, dtype, roundings):
    """Element by element, and the 2-norm: a sum's error of 5e-6 of it, and per rounding to bf16 (2^-9 at most, 1.7e-3 on average)."""
    assert got.dtype == dtype and got.shape == want.shape and torch.isfinite(got).all()
    if dtype == torch.bfloat16:
        bound = bound + 2.0 ** -8 * want.abs() + 1e-30
    err = (got.double() - want).abs()
    assert not (err > bound).any(), (int((err > bound).sum()), float(err.max()), got.double()[err > bound][:3], want[err > bound][:3])
    size = float(want.norm())
    if size > 1e-6 * math.sqrt(want.numel()) and want.numel() > 1000:
        assert float(err.norm()) <= (5e-6 + 2.4e-3 * roundings) * size, float(err.norm()) / size


def call(s, act, dtype, dH=None, stream=None):
    """Through the C functions, with a workspace of NaNs of the size asked for and
    outputs between guards; returns {name: output}."""
    lib = bsr.load()
    (N, K), F = s["X"].shape, s["Wg"].shape[0]
    dt = bsrlib.dtype_code(DT[dtype])
    n = ctypes.c_size_t(0)
    assert lib.bsr_gated_workspace(N, F, K, dt, int(dH is not None), ctypes.byref(n)) == 0
    ws = torch.full((n.value + 64,), 0xff, dtype=torch.uint8, device="cuda")
    shapes = {"H": (N, F, DT[dtype])} if dH is None else {
        "dX": (N, K, DT[dtype]), "dWg": (F, K, DT[dtype]), "dWu": (F, K, DT[dtype])}
    if dH is not None and s["bg"] is not None:
        shapes.update(dbg=(1, F, torch.float32), dbu=(1, F, torch.float32))
    held, out = [], {}
    for k, (a, b, t) in shapes.items():
        buf = torch.full((a * b + 64,), 7.0, dtype=t, device="cuda")
        held.append((buf, a * b))
        out[k] = buf[32:32 + a * b].view(a, b)
    P = lambda t: None if t is None else t.data_ptr()  # noqa: E731
    q = torch.cuda.current_stream().cuda_stream if stream is None else stream.cuda_stream
    tail = (N, F, K, dt, bsrlib._ACT[act], ws.data_ptr() if n.value else None, n.value, q)
    ins = [P(s[k]) for k in ("X", "Wg", "Wu", "bg", "bu")]
    if dH is None:
        assert lib.bsr_gated(*ins, P(out["H"]), *tail) == 0
    else:
        assert lib.bsr_gated_backward(*ins, P(dH), *[P(out.get(k)) for k in ("dX", "dWg", "dWu", "dbg", "dbu")], *tail) == 0
    torch.cuda.synchronize()
    assert (ws[n.value:] == 0xff).all()
    for buf, size in held:
        assert (buf[:32] == 7).all() and (buf[32 + size:] == 7).all()
    return out


def check_forward(s, act, dtype):
    H = call(s, act, dtype)["H"]
    (G, mG), (U, mU) = project(s["X"], s["Wg"], s["bg"]), project(s["X"], s["Wu"], s["bu"])
    a, _ = act64(G, act)
    # |act'| <= 1.13 for all of them
    bound = 1.13 * SUM * mG * (U.abs() + SUM * mU) + a.abs() * SUM * mU + FUN * (1 + G.abs()) * U.abs()
    near(H, a * U, bound, DT[dtype], 1)
    return H


def check_backward(s, dH, act, dtype):
    got = call(s, act, dtype, dH)
    X, Wg, Wu, d = (t.double() for t in (s["X"], s["Wg"], s["Wu"], dH))
    (G, mG), (U, mU) = project(s["X"], s["Wg"], s["bg"]), project(s["X"], s["Wu"], s["bu"])
    a, slope = act64(G, act)
    dG, dU = d * U * slope, d * a
    # their errors: of the sums, of the functions, where relu' may fall on its other side, and (bf16) of their rounding
    eU = d.abs() * (1.13 * SUM * mG + FUN * (1 + G.abs()))
    eG = d.abs() * (1.13 * SUM * mU + (U.abs() + SUM * mU) * (CURVE[act] * SUM * mG + FUN * (1 + G.abs())))
    if act == "relu":
        eG = eG + torch.where(G.abs() <= SUM * mG, d.abs() * (U.abs() + SUM * mU), torch.zeros_like(G))
    sums = {"dbg": (dG.sum(0, keepdim=True), eG.sum(0) + SUM * dG.abs().sum(0)),
            "dbu": (dU.sum(0, keepdim=True), eU.sum(0) + SUM * dU.abs().sum(0))}
    if dtype == "bf16":
        eG, eU = eG + 2.0 ** -9 * (dG.abs() + eG), eU + 2.0 ** -9 * (dU.abs() + eU)
    want = {"dX": (dG @ Wg + dU @ Wu, (eG + SUM * dG.abs()) @ Wg.abs() + (eU + SUM * dU.abs()) @ Wu.abs()),
            "dWg": (dG.T @ X, (eG + SUM * dG.abs()).T @ X.abs()), "dWu": (dU.T @ X, (eU + SUM * dU.abs()).T @ X.abs())}
    if s["bg"] is not None:
        want.update(sums)
    assert set(want) == set(got)
    for k, (v, bound) in want.items():
        f32 = dtype == "f32" or k in ("dbg", "dbu")
        near(got[k], v, bound, torch.float32 if f32 else torch.bfloat16, 0 if f32 else 2)
    return got


SIZES = [(1, 1, 1), (1, 64, 64), (2, 100, 72), (3, 8, 7), (5, 257, 130), (7, 1000, 96), (8, 512, 768), (9, 130, 1023),
         (16, 2050, 1024), (17, 96, 64), (31, 64, 520), (33, 72, 264), (64, 1024, 256), (65, 40, 1032), (100, 300, 770),
         (127, 128, 128), (128, 256, 768), (129, 136, 72), (255, 64, 65), (256, 512, 512), (257, 1030, 200), (600, 384, 640),
         (1000, 771, 96)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,F,K", SIZES)
def test_forward_sizes(N, F, K, dtype):
    check_forward(make(N, F, K, dtype, bias=(N + F) % 2 == 0)[0], ACTS[(N + F + K) % 5], dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,F,K", SIZES)
def test_backward_sizes(N, F, K, dtype):
    check_backward(*make(N, F, K, dtype, bias=(N + F) % 2 == 0), ACTS[(N + F + K) % 5], dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N", [4, 300])
@pytest.mark.parametrize("act", ACTS)
def test_activations_over_their_range(act, N, dtype):
    # G to about +-40: the exponentials overflow and vanish there
    s, dH = make(N, 384, 256, dtype, wide=10.0)
    check_forward(s, act, dtype)
    check_backward(s, dH, act, dtype)


@pytest.mark.parametrize("N", [2, 4000])
def test_gelu_on_a_grid(N):
    # G is x itself and U is 1. Phi: 7.5e-8 of the formula, and a few roundings of values below 1
    x = torch.linspace(-12, 12, N, device="cuda")[:, None].contiguous()
    W, none, one = torch.ones(32, 1, device="cuda"), torch.zeros(32, device="cuda"), torch.ones(32, device="cuda")
    H = bsr.bsr_gated(x, W, W * 0, none, one, act="gelu").double()
    want, slope = act64(x.double(), "gelu")
    assert ((H - want).abs() <= 4e-7 * x.abs() + 2.0 ** -22 * want.abs()).all()
    got = bsr.bsr_gated_backward(x, W, W * 0, none, one, torch.ones(N, 32, device="cuda"), act="gelu")
    assert ((got["dX"].double() / 32 - slope).abs() <= 4e-7 * (1 + x.abs()) + SUM * slope.abs()).all()


@pytest.mark.parametrize("dtype,N,F,K", [("bf16", 4096, 2048, 768), ("f32", 2048, 1024, 768), ("bf16", 2500, 4096, 1024)])
def test_many_tiles(dtype, N, F, K):
    s, dH = make(N, F, K, dtype)
    check_forward(s, "silu", dtype)
    check_backward(s, dH, "silu", dtype)


def test_long_sums_in_fp32():
    # sums of one sign, where an accumulator that drops bits drifts
    s, dH = make(200, 128, 4096, "f32")
    s = {k: v.abs() if v is not None else v for k, v in s.items()}
    check_forward(s, "relu", "f32")
    s, dH = make(6000, 64, 64, "f32")
    s = {k: v.abs() if v is not None else v for k, v in s.items()}
    check_backward(s, dH.abs(), "relu", "f32")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N", [6, 300])
def test_a_bad_token_leaves_the_others_alone(N, dtype):
    s, _ = make(N, 200, 136, dtype)
    clean = call(s, "gelu", dtype)["H"].clone()
    s["X"][1, 3], s["X"][4, 0] = float("nan"), float("inf")
    got = call(s, "gelu", dtype)["H"]
    rows = torch.tensor([n for n in range(N) if n not in (1, 4)], device="cuda")
    assert torch.equal(clean[rows], got[rows])
    assert torch.isnan(got[1]).all() and not torch.isfinite(got[4]).any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_bias_gradients_of_features_that_are_not_finite(dtype):
    s, dH = make(40, 96, 64, dtype)
    dH = dH.abs() + 0.5
    s["bg"][3] = float("inf")
    got = bsr.bsr_gated_backward(s["X"], s["Wg"], s["Wu"], s["bg"], s["bu"], dH, act="relu")
    assert got["dbu"][3] == float("inf")   # sum of dH relu(inf)
    U = project(s["X"], s["Wu"], s["bu"])[0]
    want = (dH.double() * U)[:, 3].sum()
    assert abs(float(got["dbg"][3]) - float(want)) <= SUM * 40 * float((dH.double() * (U.abs() + 10)).max())
    if dtype == "bf16":   # weights: every token's G is -inf, and relu of it 0 (fp32 parts give NaN)
        s, dH = make(40, 96, 64, dtype)
        s["X"], s["Wg"][5, 7] = s["X"].abs() + 0.5, -float("inf")
        got = bsr.bsr_gated_backward(s["X"], s["Wg"], s["Wu"], s["bg"], s["bu"], dH, act="relu")
        assert got["dbg"][5] == 0 and got["dbu"][5] == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N", [3, 700])
def test_repeats_to_the_bit_on_another_stream(N, dtype):
    s, dH = make(N, 520, 328, dtype)
    one = dict(call(s, "silu", dtype), **call(s, "silu", dtype, dH))
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    two = {"H": bsr.bsr_gated(s["X"], s["Wg"], s["Wu"], s["bg"], s["bu"], act="silu", stream=other)}
    two.update(bsr.bsr_gated_backward(s["X"], s["Wg"], s["Wu"], s["bg"], s["bu"], dH, act="silu", stream=other))
    other.synchronize()
    for k in one:
        assert torch.equal(one[k].view(two[k].shape), two[k]), k


def test_weights_are_read_as_they_are():
    s, dH = make(40, 256, 128, "bf16")
    check_forward(s, "silu", "bf16")
    s["Wg"].neg_()
    s["X"].mul_(0.5)
    check_forward(s, "silu", "bf16")
    check_backward(s, dH, "silu", "bf16")


def test_without_tokens_and_without_some_gradients():
    s, dH = make(0, 72, 40, "bf16")
    assert bsr.bsr_gated(s["X"], s["Wg"], s["Wu"]).shape == (0, 72)
    got = bsr.bsr_gated_backward(s["X"], s["Wg"], s["Wu"], s["bg"], s["bu"], dH)
    assert got["dX"].shape == (0, 40)
    for k in ("dWg", "dWu", "dbg", "dbu"):
        assert not got[k].any()
    s, dH = make(50, 72, 40, "f32")
    whole = call(s, "silu", "f32", dH)
    lib, n = bsr.load(), ctypes.c_size_t(0)
    assert lib.bsr_gated_workspace(50, 72, 40, 0, 1, ctypes.byref(n)) == 0
    ws = torch.empty(n.value, dtype=torch.uint8, device="cuda")
    for some in (("dX",), ("dWg", "dWu"), ("dbu",)):
        out = {k: torch.empty_like(whole[k]) for k in some}
        P = lambda t: None if t is None else t.data_ptr()  # noqa: E731
        assert lib.bsr_gated_backward(*[P(s[k]) for k in ("X", "Wg", "Wu", "bg", "bu")], P(dH),
                                      *[P(out.get(k)) for k in ("dX", "dWg", "dWu", "dbg", "dbu")], 50, 72, 40, 0, 0,
                                      ws.data_ptr(), n.value, torch.cuda.current_stream().cuda_stream) == 0
        torch.cuda.synchronize()
        for k in some:
            assert torch.equal(out[k], whole[k]), k


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh", "sigmoid"])
def test_gradients_against_differences(act):
    """(L(x + e v) - L(x - e v)) / 2e of L = sum H dH against <gradient, v>."""
    s, dH = make(40, 96, 64, "f32")
    grads = bsr.bsr_gated_backward(s["X"], s["Wg"], s["Wu"], s["bg"], s["bu"], dH, act=act)
    g, e = torch.Generator(device="cuda").manual_seed(5), 2.0 ** -8

    def L(s):
        return float((bsr.bsr_gated(s["X"], s["Wg"], s["Wu"], s["bg"], s["bu"], act=act).double() * dH.double()).sum())

    for name, grad in grads.items():
        x = s[name[1:]]
        v = torch.randn(x.shape, generator=g, device="cuda")
        up, down = (L(dict(s, **{name[1:]: x + sign * e * v})) for sign in (1, -1))
        want = float((grad.double() * v.double()).sum())
        # the third derivative's share, and the outputs' roundings (2^-24 each of about 3800 terms of order 1) over 2e
        assert abs((up - down) / (2 * e) - want) <= 2e-3 * float(grad.double().norm() * v.double().norm()) + 0.01, name


def test_refusals_on_the_device():
    lib = bsr.load()
    s, dH = make(20, 64, 64, "bf16")
    n = ctypes.c_size_t(0)
    assert lib.bsr_gated_workspace(20, 64, 64, 1, 1, ctypes.byref(n)) == 0 and n.value > 0
    ws, H = torch.empty(n.value + 16, dtype=torch.uint8, device="cuda"), torch.empty(20, 64, dtype=torch.bfloat16, device="cuda")
    X, Wg, Wu, W, h = (t.data_ptr() for t in (s["X"], s["Wg"], s["Wu"], ws, H))
    big = 1 << 30

    def forward(X=X, H=h, ws=W):
        return lib.bsr_gated(X, Wg, Wu, None, None, H, 20, 64, 64, 1, 0, ws, big, None)

    assert forward(X=X + 2) == forward(H=h + 8) == bsrlib.BSR_ERR_ALIGNMENT
    assert forward(H=X) == forward(H=Wu) == bsrlib.BSR_ERR_INVALID_ARG
    assert forward(X=s["X"].cpu().pin_memory().data_ptr()) == bsrlib.BSR_ERR_INVALID_ARG
    args = (X, Wg, Wu, None, None, dH.data_ptr(), h, None, None, None, None, 20, 64, 64, 1, 0)
    assert lib.bsr_gated_backward(*args, W, n.value - 1, None) == bsrlib.BSR_ERR_CAPACITY
    assert lib.bsr_gated_backward(*args, None, n.value, None) == bsrlib.BSR_ERR_INVALID_ARG
    assert lib.bsr_gated_backward(*args, W + 8, n.value, None) == bsrlib.BSR_ERR_ALIGNMENT
    assert lib.bsr_gated_backward(*args, h, n.value, None) == bsrlib.BSR_ERR_INVALID_ARG
    for bad in (dict(X=s["X"].float()), dict(Wu=s["Wu"].t()), dict(Wu=s["Wu"][:32]), dict(act="swish"),
                dict(bg=torch.zeros(64, device="cuda", dtype=torch.bfloat16)), dict(H=H[:4])):
        with pytest.raises((TypeError, ValueError)):
            bsr.bsr_gated(**dict(dict(X=s["X"], Wg=s["Wg"], Wu=s["Wu"]), **bad))
    torch.cuda.synchronize()
