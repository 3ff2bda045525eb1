"""Operands in 8-bit floating point against the rounding rule in 64 bits, bit by
bit, and their products against sums in 64 bits, element by element."""
import pytest
import torch

import paper_2106_08846_gb300 as bsr
from paper_2106_08846_gb300.bsrlib import BSR_OK

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
FMT = {"e4m3": (3, -6, 448.0), "e5m2": (2, -14, 57344.0)}   # bits, exponent of the least normal value, largest value
U = 2.0 ** -24


def normal(*shape, seed=0, wide=0.0):
    g = torch.Generator(device="cuda").manual_seed(seed + 7 * shape[-1] + 3 * shape[0])
    x = torch.randn(*shape, device="cuda", generator=g)
    return x * torch.exp(wide * torch.randn(shape[-1], device="cuda", generator=g)) if wide else x


def quantized(x, tile, fmt):
    """q and scale of x [R, C] (finite and other values) from the rule, in 64 bits."""
    bits, least, most = FMT[fmt]
    R, C = x.shape
    RB, KB = -(-R // tile), -(-C // 128)
    X = torch.zeros(RB * tile, KB * 128, dtype=torch.double, device="cuda")
    X[:R, :C] = x.double()
    blocks = X.view(RB, tile, KB, 128)
    size = torch.where(blocks.isfinite(), blocks.abs(), torch.zeros_like(blocks)).amax((1, 3))
    m, e = torch.frexp(size / most)
    e = torch.where(m == 0.5, e - 1, e).clamp(min=-126)
    e = torch.where(size == 0, torch.zeros_like(e), e).double()
    y = blocks * torch.exp2(-e).view(RB, 1, KB, 1)
    step = torch.exp2((torch.frexp(torch.where(y.isfinite(), y, torch.zeros_like(y))).exponent - 1).clamp(min=least).double() - bits)
    q = torch.where(y.isfinite(), torch.round(y / step) * step, torch.full_like(y, float("nan")))
    return q.reshape(RB * tile, KB * 128)[:R], torch.exp2(e).T


def same(m, q, scale):
    assert m.scale.dtype == torch.float32 and torch.equal(m.scale.double(), scale)
    got = m.q.double()
    assert torch.equal(got.isnan(), q.isnan()) and torch.equal(got.nan_to_num(), q.nan_to_num())
    assert torch.equal(torch.signbit(m.q.float()) & ~got.isnan(), torch.signbit(q) & ~q.isnan())


def check_exponents(m, rows=None, blocks=None):
    """A byte for each row and block, in the order that include/bsr.h gives."""
    rows, blocks = m.rows if rows is None else rows, -(-m.cols // 128) if blocks is None else blocks
    r, b = torch.arange(rows, device="cuda").view(-1, 1), torch.arange(blocks, device="cuda")
    runs = -(-m.rows // 128)
    at = ((b // 4) * runs + r // 128) * 512 + (r % 32) * 16 + (r // 32 % 4) * 4 + b % 4
    want = 127 + torch.log2(m.scale.double()).round().long()[:blocks, :].repeat_interleave(m.tile, 1)[:, :rows].T
    assert torch.equal(m.exponent.view(-1)[at.reshape(-1)].long().view(rows, blocks), want)


def filled(m):
    m.q.view(torch.uint8).fill_(0x55)
    m.scale.fill_(-7.0)
    return m


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("tile", [1, 128])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("R,C", [(1, 1), (1, 1024), (3, 130), (127, 128), (128, 127), (129, 72), (200, 770), (1000, 513), (257, 2052)])
def test_quantize(R, C, dtype, tile, fmt):
    x = normal(R, C, wide=2.0).to(DT[dtype])
    x[R // 2, : (C + 1) // 2] = 0
    rows, columns = (filled(bsr.Fp8Matrix(r, c, tile, fmt)) for r, c in ((R, C), (C, R)))
    got = bsr.bsr_fp8_quantize(x, tile, fmt, "both", out=(rows, columns))
    assert got == (rows, columns)
    same(rows, *quantized(x, tile, fmt))
    same(columns, *quantized(x.T, tile, fmt))
    check_exponents(rows)
    check_exponents(columns)
    for form, of in (("rows", rows), ("columns", columns)):
        one = bsr.bsr_fp8_quantize(x, tile, fmt, form)
        assert torch.equal(one.q.view(torch.uint8), of.q.view(torch.uint8)) and torch.equal(one.scale, of.scale)


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_quantize_borders(dtype, fmt):
    """Largest values at and beside a border between two scales, halves between two
    values, subnormal blocks, and what is not finite."""
    most, dt = FMT[fmt][2], DT[dtype]
    x = torch.zeros(24, 256, device="cuda")
    x[:, :128] = normal(24, 128, seed=1)
    for r, big in enumerate((most, most * (1 + torch.finfo(dt).eps), most * (1 - torch.finfo(dt).eps), 2 * most, most / 2, 1.0,
                             3.4028234663852886e38 if dtype == "f32" else 3.3895313892515355e38, 1e-38, 1e-40, 2.0 ** -126)):
        x[r, 5] = -big
    x[8, :] *= 1e-39
    x[8, 5] = 1e-40
    x[10, :128] = torch.arange(128, device="cuda") * (most / 128)          # ties between values
    x[11, :128] = torch.arange(128, device="cuda") * (most / 1024) * 1.0625
    x[12, 3], x[13, 4], x[14, 4] = float("nan"), float("inf"), -float("inf")
    x[15, :128] = float("inf")
    x[16, :] = 0.0
    x[17, :] = -0.0
    x = x.to(dt)
    for tile in (1, 128):
        rows, columns = bsr.bsr_fp8_quantize(x, tile, fmt, "both")
        same(rows, *quantized(x, tile, fmt))
        same(columns, *quantized(x.T, tile, fmt))


@pytest.mark.parametrize("used", [-5, 0, 1, 100, 128, 200, 300, 1000])
def test_quantize_rows_in_use(used):
    R, C = 300, 200
    x = normal(R, C).to(torch.bfloat16)
    n = max(0, min(used, R))
    x[n:] = float("nan")
    rows, columns = (filled(bsr.Fp8Matrix(r, c, 1)) for r, c in ((R, C), (C, R)))
    bsr.bsr_fp8_quantize(x, form="both", used=torch.tensor([used], dtype=torch.int32, device="cuda"), out=(rows, columns))
    x[n:] = 0
    q, scale = quantized(x, 1, "e4m3")
    assert torch.equal(rows.q[:n].double(), q[:n]) and torch.equal(rows.scale[:, :n].double(), scale[:, :n])
    assert (rows.q[n:].view(torch.uint8) == 0x55).all() and (rows.scale[:, n:] == -7).all()
    q, scale = quantized(x.T, 1, "e4m3")
    whole = -(-n // 128)
    assert torch.equal(columns.q[:, :128 * whole].double(), q[:, :128 * whole]) and torch.equal(columns.scale[:whole].double(), scale[:whole])
    assert (columns.q[:, 128 * whole:].view(torch.uint8) == 0x55).all() and (columns.scale[whole:] == -7).all()
    check_exponents(rows, rows=n)
    check_exponents(columns, blocks=whole)


def test_quantize_a_batch():
    x = normal(3, 130, 200).to(torch.bfloat16)
    rows, columns = bsr.bsr_fp8_quantize(x, 128, form="both")
    for i in range(3):
        one, turned = bsr.bsr_fp8_quantize(x[i].contiguous(), 128, form="both")
        for of, m in ((rows, one), (columns, turned)):
            assert torch.equal(of.q[i].view(torch.uint8), m.q.view(torch.uint8)) and torch.equal(of.scale[i], m.scale)


def values(m):
    """What the 8-bit values stand for, in 64 bits."""
    s = m.scale.double().transpose(-1, -2).repeat_interleave(m.tile, -2).repeat_interleave(128, -1)
    return (m.q.double() * s[..., :m.rows, :])[..., :m.cols]


def near(got, A, B, bias=None):
    """Every element: a block's 128 products and the accumulator are added with 24 bits of the largest
    one or more (132 half steps, of two halves where they are cut off), then a rounding for each block's scale, sum and the bias."""
    Y, size = A @ B.T, A.abs() @ B.abs().T
    if bias is not None:
        Y, size = Y + bias.double(), size + bias.double().abs()
    bound = (132 + 2 * (A.shape[1] // 128 + 4)) * U * size
    if got.dtype == torch.bfloat16:
        bound = bound + 2.0 ** -8 * Y.abs()
    err = (got.double() - Y).abs()
    assert torch.isfinite(got).all() and not (err > bound).any(), (int((err > bound).sum()), float((err / size.clamp(min=1e-300)).max()))


def guarded(dtype, *shape):
    n = 1
    for d in shape:
        n *= d
    buf = torch.full((n + 64,), 7.0, dtype=DT[dtype], device="cuda")
    return buf, buf[32:32 + n].view(*shape)


SIZES = [(1, 1, 1), (1, 4096, 1024), (2, 64, 128), (3, 130, 127), (5, 1000, 2000), (8, 1024, 8192), (16, 769, 384), (17, 64, 129), (31, 33, 4096),
         (33, 2048, 768), (64, 1024, 4096), (127, 128, 256), (128, 256, 768), (129, 384, 200), (257, 1000, 513), (300, 770, 2050), (512, 100, 16384), (999, 2050, 770),
         (1500, 4096, 1024), (4100, 257, 300)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,M,K", SIZES)
def test_product(N, M, K, dtype):
    x, w = normal(N, K, wide=1.0), normal(M, K, seed=1) / K ** 0.5
    for bias, fa, fb, ta, tb in ((False, "e4m3", "e4m3", 1, 128), (True, "e5m2", "e4m3", 1, 1), (True, "e4m3", "e5m2", 128, 128)):
        a, b = bsr.bsr_fp8_quantize(x, ta, fa), bsr.bsr_fp8_quantize(w, tb, fb)
        v = normal(M, seed=2) if bias else None
        buf, Y = guarded(dtype, N, M)
        bsr.bsr_fp8_product(a, b, v, Y=Y)
        near(Y, values(a), values(b), v)
        assert (buf[:32] == 7).all() and (buf[-32:] == 7).all()
        again = bsr.bsr_fp8_product(a, b, v, dtype=DT[dtype])
        assert torch.equal(again, Y)
    assert bsr.bsr_check_status() == BSR_OK


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("K", [1024, 1152, 16384, 20000, 65536])
def test_long_sums_of_one_sign(K, dtype):
    """The accumulators lose bits always towards zero, at most 2^-23 of the sum with each 32 columns: 2^-18 of it in the 1024
    that fp32 results have of them, 2^-14 in the 16384 of bf16 ones; `near` has 148 2^-24 and 2^-8."""
    a, b = bsr.bsr_fp8_quantize(normal(300, K).abs()), bsr.bsr_fp8_quantize(normal(200, K, seed=1).abs(), 128)
    near(bsr.bsr_fp8_product(a, b, dtype=DT[dtype]), values(a), values(b))
    near(bsr.bsr_fp8_product(b, a, dtype=DT[dtype]), values(b), values(a))


RUNS = [(1, 64, 128, [0, 1]), (300, 130, 200, [0, 0, 100, 100, 257, 300]), (1000, 1024, 768, [0, 256, 256, 768, 896]),
        (777, 2050, 513, [5, 5, 6, 300, 301, 700]), (5000, 512, 256, [0, 4000, 4001, 4128, 4999]), (64, 256, 1024, list(range(0, 65, 4))),
        (2000, 300, 384, [0] * 20 + [1999] + [2000] * 43), (40, 1024, 2048, [0, 1, 3, 4, 5, 9, 40]), (50, 64, 128, [7, 7, 7]),
        (300, 128, 3000, [0, 129, 300])]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("R,M,K,at", RUNS)
def test_runs_of_rows(R, M, K, at, dtype):
    E = len(at) - 1
    x, w = normal(R, K, wide=1.0), normal(E, M, K, seed=1) / K ** 0.5
    offsets = torch.tensor(at, dtype=torch.int32, device="cuda")
    for bias, fa, tb in ((False, "e4m3", 128), (True, "e5m2", 1)):
        a, b = bsr.bsr_fp8_quantize(x, 1, fa), bsr.bsr_fp8_quantize(w, tb)
        v = normal(E, M, seed=2) if bias else None
        buf, Y = guarded(dtype, R, M)
        bsr.bsr_fp8_product(a, b, v, offsets=offsets, Y=Y)
        A, B = values(a), values(b)
        for e in range(E):
            run = slice(at[e], at[e + 1])
            near(Y[run], A[run], B[e], None if v is None else v[e])
        assert (Y[:at[0]] == 7).all() and (Y[at[-1]:] == 7).all() and (buf[:32] == 7).all() and (buf[-32:] == 7).all()
    assert bsr.bsr_check_status() == BSR_OK


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,M,R,at", [(1, 1, 128, [0, 128]), (130, 64, 640, [0, 0, 256, 384, 384]), (513, 770, 1024, [0, 128, 128, 1024]),
                                      (1024, 768, 2000, [0, 512, 1920, 2048]), (256, 4096, 4096, [128 * i for i in range(33)]),
                                      (64, 64, 8192, [0, 8192, 8192])])
def test_runs_of_columns(N, M, R, at, dtype):
    E = len(at) - 1
    d, x = normal(R, N, wide=1.0), normal(R, M, seed=1)
    for fmt, tile in (("e5m2", 1), ("e4m3", 128)):
        a, b = bsr.bsr_fp8_quantize(d, 1, fmt, "columns"), bsr.bsr_fp8_quantize(x, tile, form="columns")
        buf, Y = guarded(dtype, E, N, M)
        bsr.bsr_fp8_product(a, b, offsets=torch.tensor(at, dtype=torch.int32, device="cuda"), over="columns", Y=Y)
        A, B = values(a), values(b)
        for e in range(E):
            near(Y[e], A[:, at[e]:at[e + 1]], B[:, at[e]:at[e + 1]])   # (no columns: zeros)
        assert (buf[:32] == 7).all() and (buf[-32:] == 7).all()
    assert bsr.bsr_check_status() == BSR_OK


def test_offsets_out_of_range_touch_nothing_else():
    """Offsets that do not ascend or lie outside are clamped to the rows and columns that there are."""
    R, M, K = 300, 200, 256
    a, b = bsr.bsr_fp8_quantize(normal(R, K)), bsr.bsr_fp8_quantize(normal(3, M, K), 128)
    buf, Y = guarded("f32", R, M)
    bsr.bsr_fp8_product(a, b, offsets=torch.tensor([-9, 100, 50, 2 ** 31 - 1], dtype=torch.int32, device="cuda"), Y=Y)
    assert (buf[:32] == 7).all() and (buf[-32:] == 7).all()
    near(Y[:50], values(a)[:50], values(b)[0])
    c = bsr.bsr_fp8_quantize(normal(R, K), form="columns")
    out = bsr.bsr_fp8_product(c, c, offsets=torch.tensor([-128, 128, 0, 2 ** 31 - 1], dtype=torch.int32, device="cuda"), over="columns")
    near(out[0], values(c)[:, :128], values(c)[:, :128])
    assert (out[1] == 0).all()
    near(out[2], values(c), values(c))
    assert bsr.bsr_check_status() == BSR_OK


def test_values_that_are_not_finite():
    N, M, K = 70, 200, 300
    x, w = normal(N, K), normal(M, K, seed=1)
    x[3, 5], x[68, 299], w[7, 131], w[199, 0] = float("nan"), float("inf"), -float("inf"), float("nan")
    a, b = bsr.bsr_fp8_quantize(x), bsr.bsr_fp8_quantize(w, 128)
    Y = bsr.bsr_fp8_product(a, b, dtype=torch.float32)
    want = torch.zeros(N, M, dtype=torch.bool, device="cuda")
    want[[3, 68]] = True
    want[:, [7, 199]] = True
    assert torch.equal(Y.isnan(), want)
    ok, cols = ~want[:, 0], ~want[0]
    near(Y[ok][:, cols], values(a)[ok], values(b)[cols])


def test_no_rows_and_no_columns():
    w = bsr.bsr_fp8_quantize(normal(64, 128), 128)
    assert bsr.bsr_fp8_product(bsr.bsr_fp8_quantize(torch.empty(0, 128, device="cuda")), w).shape == (0, 64)
    none = bsr.bsr_fp8_quantize(torch.empty(0, 96, device="cuda"), form="columns")   # a batch of no tokens
    other = bsr.bsr_fp8_quantize(torch.empty(0, 300, device="cuda"), form="columns")
    for dtype in DT.values():
        Y = torch.full((96, 300), 7.0, dtype=dtype, device="cuda")
        bsr.bsr_fp8_product(none, other, Y=Y)
        assert (Y == 0).all()
        v = normal(300)
        assert torch.equal(bsr.bsr_fp8_product(none, other, v, dtype=dtype), v.to(dtype).expand(96, 300))


def test_layer_gradients_against_differences():
    """Y = X W' with both in 8 bits: dX and dW of what the 8-bit values stand for."""
    N, M, K = 200, 96, 160
    x, w, dy = normal(N, K), normal(M, K, seed=1) / K ** 0.5, normal(N, M, seed=2)
    (a, at), (b, bt), (d, dt) = (bsr.bsr_fp8_quantize(t, tile, form="both") for t, tile in ((x, 1), (w, 128), (dy, 1)))
    dX = bsr.bsr_fp8_product(d, bt, dtype=torch.float32)
    dW = bsr.bsr_fp8_product(dt, at, dtype=torch.float32)
    near(dX, values(d), values(b).T)   # (a weight's two forms are the same values)
    near(dW, values(dt), values(at))
    # along a direction: (<dy, Y(x + t v)> - <dy, Y(x - t v)>) / 2 t, with directions and steps that 8 bits hold
    A, B, G = values(a), values(b), values(d)
    v = torch.sign(normal(N, K, seed=3)).double()
    diff = ((G * ((A + v) @ B.T)).sum() - (G * ((A - v) @ B.T)).sum()) / 2
    size = (G.abs() @ B.abs()).sum()
    assert abs(float(diff - (dX.double() * v).sum())) <= float(144 * U * size)


def test_streams_and_a_captured_graph():
    N, M, K = 400, 512, 768
    x, w = normal(N, K).to(torch.bfloat16), normal(M, K, seed=1)
    b = bsr.bsr_fp8_quantize(w, 128)
    a, Y = bsr.Fp8Matrix(N, K), torch.empty(N, M, dtype=torch.bfloat16, device="cuda")

    def layer(stream=None):
        bsr.bsr_fp8_quantize(x, out=a, stream=stream)
        bsr.bsr_fp8_product(a, b, Y=Y, stream=stream)

    layer()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer()
    for seed in (5, 6):
        x.copy_(normal(N, K, seed=seed))
        graph.replay()
        got = Y.clone()
        near(got, values(a), values(b))
        layer()
        assert torch.equal(got, Y)
    side = torch.cuda.Stream()
    Y.zero_()
    side.wait_stream(torch.cuda.current_stream())
    made = bsr.bsr_fp8_product(bsr.bsr_fp8_quantize(x, stream=side), b, stream=side)
    layer(side.cuda_stream)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, Y) and torch.equal(made, Y)
    assert bsr.bsr_check_status() == BSR_OK


def test_two_graphs_and_a_call_that_needs_a_workspace():
    """Sums that are split: their parts' memory is each call's own."""
    N, M, K = 64, 1024, 4096
    a, b = bsr.bsr_fp8_quantize(normal(N, K)), bsr.bsr_fp8_quantize(normal(M, K, seed=1), 128)
    c, d = bsr.bsr_fp8_quantize(normal(N, K, seed=2)), bsr.bsr_fp8_quantize(normal(M, K, seed=3), 128)
    want = [bsr.bsr_fp8_product(a, b), bsr.bsr_fp8_product(c, d)]
    near(want[0], values(a), values(b))
    graphs, got = [], []
    for x, w in ((a, b), (c, d)):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            got.append(bsr.bsr_fp8_product(x, w))
    streams = [torch.cuda.Stream() for _ in graphs]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        eager = bsr.bsr_fp8_product(a, d)
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    near(eager, values(a), values(d))
    assert bsr.bsr_check_status() == BSR_OK


def test_other_devices_memory_and_the_host_are_refused():
    a, b = bsr.bsr_fp8_quantize(normal(8, 128)), bsr.bsr_fp8_quantize(normal(8, 128))
    with pytest.raises(bsr.BsrError):
        bsr.bsr_fp8_product(a, b, Y=torch.empty(8, 8))
    with pytest.raises(bsr.BsrError):
        bsr.bsr_fp8_product(a, b, offsets=torch.tensor([0, 128], dtype=torch.int32), over="columns")
    with pytest.raises(bsr.BsrError):
        bsr.bsr_fp8_quantize(torch.zeros(8, 128), out=a)
    with pytest.raises(bsr.BsrError):   # rows that do not start on 16 bytes
        bsr.bsr_fp8_quantize(torch.zeros(8 * 128 + 1, device="cuda")[1:].view(8, 128), out=a)


def test_beyond_32_bits():
    R, K = 70000, 32768   # 2.3e9 values
    x = torch.ones(R, K, dtype=torch.bfloat16, device="cuda")
    x[-1, -1], x[-3, 0] = 3.0, 2.0
    rows, columns = bsr.bsr_fp8_quantize(x, form="both")
    assert float(rows.q[-1, -1].float()) * float(rows.scale[-1, -1]) == 3 and float(columns.q[-1, R - 1].float()) * float(columns.scale[-1, -1]) == 3
    w = torch.ones(64, K, device="cuda")
    Y = bsr.bsr_fp8_product(rows, bsr.bsr_fp8_quantize(w, 128), dtype=torch.float32)
    assert Y[-1].eq(K + 2).all() and Y[-3].eq(K + 1).all() and Y[:-3].eq(K).all()
    d = bsr.bsr_fp8_quantize(torch.ones(R, 64, device="cuda"), form="columns")
    dW = bsr.bsr_fp8_product(d, columns, dtype=torch.float32)   # a product of 64 x 32768 over 70000
    assert dW[:, -1].eq(R + 2).all() and dW[:, 0].eq(R + 1).all() and dW[:, 1:-1].eq(R).all()
    del x, rows, columns
    few, many = torch.ones(R, 128, device="cuda"), torch.ones(K, 128, device="cuda")
    few[-1] = 2
    many[-1] = 3
    Y = bsr.bsr_fp8_product(bsr.bsr_fp8_quantize(few), bsr.bsr_fp8_quantize(many, 128))   # 2.3e9 results
    assert Y[-1, :-1].eq(256).all() and float(Y[-1, -1]) == 768 and Y[:-1, -1].eq(384).all() and Y[::999, :-1].eq(128).all()
