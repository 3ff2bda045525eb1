"""A layer of experts in 8 bits, forward and backward: the tokens sorted by expert,
each expert's weight on its run of rows in one product, the results added up with the
router's weights and to the residual stream with its norms. Checks every result
against double precision and prints what a pass takes.

    python examples/expert_layer.py [tokens] [features] [experts] [experts of a token]
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2106_08846_gb300 as bsr  # noqa: E402


class Experts:
    """E weights [D, D] in 8 bits, as they lie for the forward pass and transposed for
    the gradient, and the norms of the residual step behind them."""

    def __init__(self, D, E, k, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.E, self.k = E, k
        self.W = (torch.randn(E, D, D, device="cuda", generator=g) * D ** -0.5).to(torch.bfloat16)
        self.w, self.wt = bsr.bsr_fp8_quantize(self.W, tile=128, form="both")
        ones = lambda: 1 + 0.1 * torch.randn(D, device="cuda", generator=g)  # noqa: E731
        self.norms = dict(post="rms", post_w=ones(), pre="rms", pre_w=ones(), scale=0.5 * ones())

    def forward(self, x, h, experts, weights):
        """The stream after the layer, its norm, and what the backward pass needs; runs start at
        multiples of 128 for the sums over rows of the weights' gradients."""
        order = bsr.bsr_expert_order(experts, self.E, align=128)
        rows = bsr.bsr_expert_rows(x, order)
        a, at = bsr.bsr_fp8_quantize(rows, form="both", used=order.used)
        Ys = bsr.bsr_fp8_product(a, self.w, offsets=order.offsets)
        y = bsr.bsr_expert_sum(Ys, order, weights)
        h2, z = bsr.bsr_residual_norm(y, h, **self.norms)
        return h2, z, (order, at, Ys, weights, y, h2)

    def backward(self, saved, dh2, dz):
        """Gradients of x, h, the router's weights, the experts' and the norms'."""
        order, at, Ys, weights, y, h2 = saved
        r = bsr.bsr_residual_norm_backward(y, h2, dh2, dz, **self.norms)
        s = bsr.bsr_expert_sum_backward(Ys, order, weights, r["dy"])
        d, dt = bsr.bsr_fp8_quantize(s["dYs"], fmt="e5m2", form="both", used=order.used)
        drows = bsr.bsr_fp8_product(d, self.wt, offsets=order.offsets)
        dW = bsr.bsr_fp8_product(dt, at, offsets=order.offsets, over="columns", dtype=torch.float32)
        grads = {"x": bsr.bsr_expert_sum(drows, order), "h": r["dh"], "weights": s["dweights"], "W": dW}
        grads.update({n: r["d" + n] for n in ("post_w", "pre_w", "scale")})
        return grads


def double_precision(layer, x, h, experts, weights, dh2, dz):
    """The same from the definitions, by automatic differentiation, and the size of what
    the weights' gradients are sums of: the sums themselves cancel, since the norm behind
    them does not see a token's results scaled (with one expert a token they are zero)."""
    leaves = {"x": x, "h": h, "weights": weights, "W": layer.W, **{n: layer.norms[n] for n in ("post_w", "pre_w", "scale")}}
    v = {n: t.double().requires_grad_() for n, t in leaves.items()}
    rms = lambda t: t / (t.square().mean(1, keepdim=True) + 1e-5).sqrt()  # noqa: E731
    rows = torch.zeros(*experts.shape, x.shape[1], dtype=torch.double, device="cuda")
    for e in range(layer.E):
        at = (experts == e).nonzero(as_tuple=True)
        rows = rows.index_put(at, v["x"][at[0]] @ v["W"][e].T)
    y = (rows * v["weights"].unsqueeze(2)).sum(1)
    h2 = v["h"] + v["scale"] * rms(y) * v["post_w"]
    z = rms(h2) * v["pre_w"]
    *grads, dy = torch.autograd.grad([h2, z], [*v.values(), y], [dh2.double(), dz.double()])
    return h2, z, dict(zip(v, grads)), float((rows.norm(dim=2) * dy.norm(dim=1, keepdim=True)).norm().detach())


def run(N=4096, D=1024, E=16, k=2):
    """The error of each result (2-norms; the router's weights' gradient: of what it sums), and the milliseconds of a forward and backward pass."""
    layer, g = Experts(D, E, k), torch.Generator(device="cuda").manual_seed(1)
    normal = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    x, h, dh2, dz = normal(N, D).to(torch.bfloat16), normal(N, D), 0.1 * normal(N, D), (0.1 * normal(N, D)).to(torch.bfloat16)
    chosen = normal(N, E).topk(k, 1)
    experts, weights = chosen.indices.int(), torch.softmax(chosen.values, 1)
    h2, z, saved = layer.forward(x, h, experts, weights)
    grads = layer.backward(saved, dh2, dz)
    assert bsr.bsr_check_status() == bsr.bsrlib.BSR_OK
    want_h, want_z, want, size = double_precision(layer, x, h, experts, weights, dh2, dz)
    error = lambda p, q, of=None: float((p.double() - q.detach()).norm()) / (of or float(q.detach().norm()))  # noqa: E731
    errors = {"h_out": error(h2, want_h), "z": error(z, want_z)}
    errors.update({"d" + n: error(grads[n], want[n], size if n == "weights" else None) for n in want})
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    begin.record()
    for _ in range(10):
        h2, z, saved = layer.forward(x, h, experts, weights)
        layer.backward(saved, dh2, dz)
    end.record()
    torch.cuda.synchronize()
    return errors, begin.elapsed_time(end) / 10


if __name__ == "__main__":
    sizes = [int(v) for v in sys.argv[1:5]]
    found, ms = run(*sizes)
    for name, e in found.items():
        print(f"{name:10s} error {e:.1e}")
    print(f"forward and backward: {ms:.3f} ms")
