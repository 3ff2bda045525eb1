"""The feed-forward half of a transformer layer on a pruned model, forward and
backward: the pruned output projection of the attention block, the residual step
with its norms, the gated block, the pruned down projection and the next residual
step. Checks every result against double precision and prints what a pass takes.

    python examples/feed_forward_layer.py [tokens] [features] [inner features]
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2106_08846_gb300 as bsr  # noqa: E402

F32 = torch.float32


def pruned(rows, cols, gen, sparsity=0.8, block=16):
    """A bf16 weight of which whole 16 x 16 blocks are removed, dense and as two BSR
    operators: of the weight, for the product, and of its transpose, for the product
    that takes a gradient back."""
    W = torch.randn(rows, cols, device="cuda", generator=gen) * (1 - sparsity) ** -0.5 * cols ** -0.5
    keep = torch.rand(rows // block, 1, cols // block, 1, device="cuda", generator=gen) > sparsity
    W = (W.view(rows // block, block, cols // block, block) * keep).view(rows, cols).to(torch.bfloat16)
    handles = []
    for w in (W, W.t().contiguous()):
        handles.append(bsr.bsr_create(*bsr.bsr_from_dense(w, block, block), block, block, *w.shape))
    return W, handles


class Layer:
    """Weights of the half layer: bf16 blocks on an fp32 residual stream."""

    def __init__(self, D, F, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.Wo, self.o = pruned(D, D, g)
        self.Wd, self.d = pruned(D, F, g)
        self.Wg, self.Wu = ((torch.randn(F, D, device="cuda", generator=g) * D ** -0.5).to(torch.bfloat16) for _ in range(2))
        ones = lambda: 1 + 0.1 * torch.randn(D, device="cuda", generator=g)  # noqa: E731
        self.norms = [dict(post="rms", post_w=ones(), pre="rms", pre_w=ones(), scale=0.5 * ones()) for _ in range(2)]
        self.bias = 0.1 * torch.randn(D, device="cuda", generator=g)

    def forward(self, a, h):
        """The stream after the layer, its norm (the next block's input), and what
        the backward pass needs; a: the attention's output, h: the stream."""
        y1 = self.o[0].spmm(a, self.bias)
        h1, z1 = bsr.bsr_residual_norm(y1, h, **self.norms[0])
        H = bsr.bsr_gated(z1, self.Wg, self.Wu, act="silu")
        y2 = self.d[0].spmm(H)
        h2, z2 = bsr.bsr_residual_norm(y2, h1, **self.norms[1])
        return h2, z2, (y1, h1, z1, y2, h2)

    def backward(self, saved, dh2, dz2):
        """Gradients of a, of the stream that came in and of the dense parameters."""
        y1, h1, z1, y2, h2 = saved
        r2 = bsr.bsr_residual_norm_backward(y2, h2, dh2, dz2, **self.norms[1])
        dH = self.d[1].spmm(r2["dy"])
        g = bsr.bsr_gated_backward(z1, self.Wg, self.Wu, None, None, dH, act="silu")
        r1 = bsr.bsr_residual_norm_backward(y1, h1, r2["dh"], g["dX"], **self.norms[0])
        grads = {"a": self.o[1].spmm(r1["dy"]), "h": r1["dh"], "Wg": g["dWg"], "Wu": g["dWu"]}
        for k, r in enumerate((r1, r2)):
            grads.update({f"{n}{k}": r["d" + n] for n in ("post_w", "pre_w", "scale")})
        return grads


def double_precision(layer, a, h, dh2, dz2):
    """The same from the definitions, by automatic differentiation."""
    leaves = {"a": a, "h": h, "Wg": layer.Wg, "Wu": layer.Wu}
    for k, p in enumerate(layer.norms):
        leaves.update({f"{n}{k}": p[n] for n in ("post_w", "pre_w", "scale")})
    v = {k: t.double().requires_grad_() for k, t in leaves.items()}

    def step(y, h, k):
        rms = lambda x: x / (x.square().mean(1, keepdim=True) + 1e-5).sqrt()  # noqa: E731
        h = h + v[f"scale{k}"] * rms(y) * v[f"post_w{k}"]
        return h, rms(h) * v[f"pre_w{k}"]

    h1, z1 = step(v["a"] @ layer.Wo.double().T + layer.bias.double(), v["h"], 0)
    H = torch.nn.functional.silu(z1 @ v["Wg"].T) * (z1 @ v["Wu"].T)
    h2, z2 = step(H @ layer.Wd.double().T, h1, 1)
    grads = torch.autograd.grad([h2, z2], list(v.values()), [dh2.double(), dz2.double()])
    return h2, z2, dict(zip(v, grads))


def run(N=4096, D=1024, F=4096):
    """The 2-norm error of each result, and the milliseconds of a forward and backward pass."""
    layer, g = Layer(D, F), torch.Generator(device="cuda").manual_seed(1)
    normal = lambda: torch.randn(N, D, device="cuda", generator=g)  # noqa: E731
    a, h, dh2, dz2 = normal().to(torch.bfloat16), normal(), 0.1 * normal(), (0.1 * normal()).to(torch.bfloat16)
    h2, z2, saved = layer.forward(a, h)
    grads = layer.backward(saved, dh2, dz2)
    assert bsr.bsr_check_status() == bsr.bsrlib.BSR_OK
    want_h, want_z, want = double_precision(layer, a, h, dh2, dz2)
    error = lambda x, y: float((x.double() - y.detach()).norm() / y.detach().norm())  # noqa: E731
    errors = {"h_out": error(h2, want_h), "z": error(z2, want_z), **{"d" + k: error(grads[k], want[k]) for k in want}}
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    begin.record()
    for _ in range(10):
        h2, z2, saved = layer.forward(a, h)
        layer.backward(saved, dh2, dz2)
    end.record()
    torch.cuda.synchronize()
    return errors, begin.elapsed_time(end) / 10


if __name__ == "__main__":
    sizes = [int(v) for v in sys.argv[1:4]]
    found, ms = run(*sizes)
    for name, e in found.items():
        print(f"{name:10s} error {e:.1e}")
    print(f"forward and backward: {ms:.3f} ms")
