"""A layer of experts in 8-bit integers, trained and then served.

    y_t = sum over the token's experts e of p_te silu(x_t Wu_e^T) Wd_e^T

Weights are kept in binary32 and converted after every step, as they lie and each transposed, so that the products forwards and backwards read 8-bit
integers with a scale for each channel.  Tokens are converted on their way to their experts (a scale for each token, or, transposed for the
gradients of the weights, for each channel of an expert's tokens); what flows between the products is bfloat16.  The router's choice is
plain torch and is not trained here.  Serving replays one captured graph for a fixed number of tokens.

    python examples/i8_experts.py [--tokens 2048] [--width 512] [--hidden 700] [--experts 8] [--each 2] [--steps 40]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
import paper_2508_03984_amd as oz  # noqa: E402


class Weights:
    """`experts` matrices of rows x cols, one below the other, in binary32, and their conversions: `as_is` for products over their columns, `turned` over their rows."""

    def __init__(self, experts, rows, cols, gen):
        self.experts, self.rows, self.cols = experts, rows, cols
        self.master = torch.randn(experts * rows, cols, device="cuda", generator=gen) * cols ** -0.5
        self.grad = torch.empty_like(self.master)
        self.as_is, self.turned = oz.I8.empty(experts * rows, cols), oz.I8.empty(experts * cols, rows)
        self.convert()

    def convert(self):
        oz.oz2_i8_quantize(self.experts, self.rows, self.cols, self.master, self.cols, self.as_is, self.turned)


class Routes:
    """Which experts have which tokens: rows in the order of experts, the token of each, where each expert's begin, and the weight of each in its token's sum."""

    def __init__(self, logits, each):
        tokens, experts = logits.shape
        weight, expert = torch.softmax(logits.float(), 1).topk(each, dim=1)
        expert, order = torch.sort(expert.flatten(), stable=True)
        self.index = (order // each).int()
        self.weight = weight.flatten()[order].unsqueeze(1)
        self.offsets = torch.searchsorted(expert, torch.arange(experts + 1, device=logits.device)).int()
        self.rows = tokens * each


class Experts:
    def __init__(self, experts, width, hidden, seed=0):
        self.experts, self.width, self.hidden = experts, width, hidden
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.up, self.down = Weights(experts, hidden, width, gen), Weights(experts, width, hidden, gen)

    def weights(self):
        return (self.up, self.down)

    def forward(self, x, routes, keep=None):
        """y of x (tokens x width); `keep`, a dictionary, receives what the backward pass needs."""
        r, e, w, f, off = routes.rows, self.experts, self.width, self.hidden, routes.offsets
        turned = oz.oz2_i8_grouped_cols(r, e)
        x8, h8 = oz.I8.empty(r, w), oz.I8.empty(r, f)
        xt8, ht8 = (oz.I8.empty(w, turned, e), oz.I8.empty(f, turned, e)) if keep is not None else (None, None)
        z, out = x.new_empty(r, f), x.new_empty(r, w)
        oz.oz2_i8_quantize_grouped(r, w, x, x.shape[0], w, routes.index, e, off, x8, xt8)
        oz.oz2_i8_grouped_gemm(r, f, w, e, off, 1.0, x8, self.up.as_is, 0.0, z, f)
        h = torch.nn.functional.silu(z)
        oz.oz2_i8_quantize_grouped(r, f, h, r, f, None, e, off, h8, ht8)
        oz.oz2_i8_grouped_gemm(r, w, f, e, off, 1.0, h8, self.down.as_is, 0.0, out, w)
        if keep is not None:
            keep.update(z=z, xt8=xt8, ht8=ht8)
        return torch.zeros(x.shape, device="cuda").index_add_(0, routes.index, out * routes.weight).to(x.dtype)

    def backward(self, dy, routes, kept):
        """The gradient of x; those of the weights in their `grad`."""
        r, e, w, f, off = routes.rows, self.experts, self.width, self.hidden, routes.offsets
        turned = oz.oz2_i8_grouped_cols(r, e)
        d8, dt8, g8, gt8 = oz.I8.empty(r, w), oz.I8.empty(w, turned, e), oz.I8.empty(r, f), oz.I8.empty(f, turned, e)
        d = (dy[routes.index] * routes.weight).to(dy.dtype)
        dh, dx = dy.new_empty(r, f), dy.new_empty(r, w)
        oz.oz2_i8_quantize_grouped(r, w, d, r, w, None, e, off, d8, dt8)
        oz.oz2_i8_grouped_grad(w, f, r, e, off, 1.0, dt8, kept["ht8"], 0.0, self.down.grad, f)
        oz.oz2_i8_grouped_gemm(r, f, w, e, off, 1.0, d8, self.down.turned, 0.0, dh, f)
        z = kept["z"].float()
        p = torch.sigmoid(z)
        dz = (dh * p * (1 + z * (1 - p))).to(dy.dtype)
        oz.oz2_i8_quantize_grouped(r, f, dz, r, f, None, e, off, g8, gt8)
        oz.oz2_i8_grouped_grad(f, w, r, e, off, 1.0, gt8, kept["xt8"], 0.0, self.up.grad, w)
        oz.oz2_i8_grouped_gemm(r, w, f, e, off, 1.0, g8, self.up.turned, 0.0, dx, w)
        return torch.zeros(dy.shape, device="cuda").index_add_(0, routes.index, dx.float()).to(dy.dtype)


def train(layer, teacher, router, tokens, each, steps, rate=2e-3, tell=None):
    """Fits the layer to `teacher`, a function from x and routes to y.  The losses of all steps."""
    params = [torch.nn.Parameter(w.master) for w in layer.weights()]       # the same memory as the weights'
    adam = torch.optim.Adam(params, lr=rate)
    gen = torch.Generator(device="cuda").manual_seed(1)
    losses = []
    for step in range(steps):
        x = torch.randn(tokens, layer.width, device="cuda", generator=gen).bfloat16()
        routes, kept = Routes(x.float() @ router, each), {}
        off = layer.forward(x, routes, kept).float() - teacher(x, routes)
        losses.append(off.square().mean())
        layer.backward((off * (2 / layer.width)).bfloat16(), routes, kept)
        for p, w in zip(params, layer.weights()):
            p.grad = w.grad / tokens
        adam.step()
        for w in layer.weights():
            w.convert()
        if tell and step % 10 == 9:
            tell(f"step {step + 1}: loss {losses[-1].item():.4f}")
    return [float(v) for v in losses]


class Server:
    """`tokens` tokens at a time as one captured graph that is replayed: the router's choice, too, is on the device."""

    def __init__(self, layer, router, tokens, each):
        self.x = torch.zeros(tokens, layer.width, dtype=torch.bfloat16, device="cuda")
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            layer.forward(self.x, Routes(self.x.float() @ router, each))
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            self.y = layer.forward(self.x, Routes(self.x.float() @ router, each))

    def __call__(self, x):
        self.x.copy_(x)
        self.graph.replay()
        return self.y


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("tokens", 2048), ("width", 512), ("hidden", 700), ("experts", 8), ("each", 2), ("steps", 40)):
        ap.add_argument("--" + name, type=int, default=value)
    o = ap.parse_args()
    layer, other = Experts(o.experts, o.width, o.hidden), Experts(o.experts, o.width, o.hidden, seed=5)
    router = torch.randn(o.width, o.experts, device="cuda") * o.width ** -0.5
    losses = train(layer, lambda x, routes: other.forward(x, routes).float(), router, o.tokens, o.each, o.steps, tell=lambda s: print(s, flush=True))
    print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f}")
    server = Server(layer, router, 4, o.each)
    for _ in range(3):
        y = server(torch.randn(4, o.width, device="cuda").bfloat16())
    torch.cuda.synchronize()
    print(f"served: {tuple(y.shape)}, finite: {bool(y.isfinite().all())}")


if __name__ == "__main__":
    main()
