"""A layer of experts in 8 bits, forward and backward, step by step: each result against double
precision on the same 8-bit values and the same inputs of the step, so that nothing but
accumulation and the rounding of results is left."""
import importlib.util
import os

import pytest
import torch

import paper_2106_08846_gb300 as bsr
from tests.test_gpu_fp8 import U, near, quantized

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BF16 = 2.0 ** -8   # half a step


def example():
    spec = importlib.util.spec_from_file_location("expert_layer", os.path.join(ROOT, "examples", "expert_layer.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def in_8_bits(x, tile, fmt):
    q, scale = quantized(x, tile, fmt)
    whole = scale.T.repeat_interleave(tile, 0).repeat_interleave(128, 1)
    return (q * whole[:q.shape[0]])[:, :x.shape[1]]


def close(got, want, bound):
    err = (got.double() - want).abs()
    assert (err <= bound).all(), float((err / bound).max())


def norm_close(got, want, bound):
    err = float((got.double() - want).norm())
    assert err <= float(bound), (err, float(bound))


@pytest.mark.parametrize("N,D,E,k", [(1, 256, 4, 2), (37, 256, 40, 2), (500, 768, 8, 2), (1000, 512, 3, 1)])
def test_every_step(N, D, E, k):
    layer, g = example().Experts(D, E, k), torch.Generator(device="cuda").manual_seed(1)
    normal = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    x, h, dh2, dz = normal(N, D).to(torch.bfloat16), normal(N, D), 0.1 * normal(N, D), (0.1 * normal(N, D)).to(torch.bfloat16)
    chosen = normal(N, E).topk(k, 1)
    experts, weights = chosen.indices.int(), torch.softmax(chosen.values, 1)
    h2, z, saved = layer.forward(x, h, experts, weights)
    grads = layer.backward(saved, dh2, dz)
    order, _, Ys, _, y, _ = saved

    # ---- every choice has a row, each expert's from a multiple of 128 on
    at, place = order.offsets.tolist(), order.place.long()
    pairs = torch.arange(N * k, device="cuda")
    assert torch.equal(order.source[place.view(-1)].long(), pairs)
    for e in range(E):
        rows = place[experts == e]
        assert at[e] % 128 == 0 and rows.numel() <= at[e + 1] - at[e] < rows.numel() + 128
        assert ((rows >= at[e]) & (rows < at[e + 1])).all()
    used = at[E]
    sent = torch.zeros(used, D, dtype=torch.double, device="cuda")
    sent[place.view(-1)] = x.double()[pairs // k]

    # ---- forward
    W = [in_8_bits(layer.W[e], 128, "e4m3") for e in range(E)]
    A = in_8_bits(sent, 1, "e4m3")
    for e in range(E):
        near(Ys[at[e]:at[e + 1]], A[at[e]:at[e + 1]], W[e])
    w = weights.double()
    terms = Ys.double()[place] * w.unsqueeze(2)
    close(y, terms.sum(1), BF16 * terms.sum(1).abs() + 2 * k * U * terms.abs().sum(1))
    p = {n: layer.norms[n].double() for n in ("post_w", "pre_w", "scale")}
    over = lambda t: (t.square().mean(1, keepdim=True) + 1e-5).rsqrt()  # noqa: E731
    yhat = y.double() * over(y.double())
    c = p["scale"] * p["post_w"] * yhat
    sums = (D + 16) * U   # a sum over a row's features and what is done with it, in fp32
    close(h2, h.double() + c, 2 * U * (h.double().abs() + c.abs()) + sums * c.abs())
    hhat = h2.double() * over(h2.double())
    close(z, hhat * p["pre_w"], (BF16 + sums) * (hhat * p["pre_w"]).abs())

    # ---- what the layer adds, from its inputs in 8 bits at once: the rows' and the sum's rounding to bf16, each
    # felt twice (in the value and in the norm), the rows' together up to twice as long as their sum
    exact = torch.zeros(used, D, dtype=torch.double, device="cuda")
    for e in range(E):
        exact[at[e]:at[e + 1]] = A[at[e]:at[e + 1]] @ W[e].T
    whole = (exact[place] * w.unsqueeze(2)).sum(1)
    add = p["scale"] * p["post_w"] * whole * over(whole)
    norm_close(h2.double() - h.double(), add, 2 * BF16 * 3 * add.norm())

    # ---- backward: the norms
    u = dz.double() * p["pre_w"]
    dh = dh2.double() + over(h2.double()) * (u - hhat * (u * hhat).mean(1, keepdim=True))
    dh_size = dh2.double().norm() + 2 * (over(h2.double()) * u).norm()
    norm_close(grads["h"], dh, 2 * sums * dh_size)
    v = dh * p["scale"] * p["post_w"]
    dy = over(y.double()) * (v - yhat * (v * yhat).mean(1, keepdim=True))
    r = bsr.bsr_residual_norm_backward(y, h2, dh2, dz, **layer.norms)
    size = (over(y.double()) * (v.abs() + 2 * sums * dh_size * (p["scale"] * p["post_w"]).abs())).norm()
    norm_close(r["dy"], dy, BF16 * dy.norm() + 4 * sums * size)
    for name, t in (("post_w", dh * p["scale"] * yhat), ("scale", dh * p["post_w"] * yhat), ("pre_w", dz.double() * hhat)):
        norm_close(grads[name], t.sum(0), (N + 2 * D + 32) * U * t.abs().sum(0).norm() + 2 * sums * dh_size * float(N) ** 0.5)

    # ---- the sum's gradients, then the experts' products
    dY = r["dy"].double()
    t = Ys.double()[place] * dY.unsqueeze(1)
    close(grads["weights"], t.sum(2), (D / 32 + 13) * U * t.abs().sum(2))
    dYs = bsr.bsr_expert_sum_backward(Ys, order, weights, r["dy"])["dYs"][:used].double()
    want = torch.zeros_like(dYs)
    want[place.view(-1)] = (dY.unsqueeze(1) * w.unsqueeze(2)).view(-1, D)
    close(dYs, want, (BF16 + 2 * U) * want.abs() + 1e-300)
    d = in_8_bits(dYs, 1, "e5m2")
    drows = torch.zeros_like(d)
    for e in range(E):
        run = slice(at[e], at[e + 1])
        drows[run] = d[run] @ W[e]
        near(grads["W"][e], in_8_bits(dYs[run].T, 1, "e5m2"), in_8_bits(sent[run].T, 1, "e4m3"))
    dx = drows[place].sum(1)
    each = drows[place].abs().sum(1)
    size = torch.zeros_like(d)
    for e in range(E):
        size[at[e]:at[e + 1]] = d[at[e]:at[e + 1]].abs() @ W[e].abs()
    # each expert's row is rounded to bf16, then their sum
    close(grads["x"], dx, BF16 * (dx.abs() + 1.01 * each) + 1.01 * (132 + 2 * (D // 128 + 4)) * U * size[place].sum(1) + 1e-300)
    assert bsr.bsr_check_status() == bsr.bsrlib.BSR_OK
