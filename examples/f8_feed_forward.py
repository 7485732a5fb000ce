"""A gated feed-forward block in 8-bit floating point, trained and then served.

    y = (silu(x Wg^T) * (x Wu^T)) Wd^T

Weights are kept in binary32 and converted after every step, whole blocks of 128 x 128 at once, as they lie and transposed, so that the products
forwards and backwards read the same numbers.  What flows between the layers is bfloat16 and is converted by rows (blocks of 1 x 128) where a
product reads it: once as it lies, for the product over its columns, and in training transposed as well, for the gradient of the weights, whose
sums go over the tokens.  Serving replays one captured graph per token.

    python examples/f8_feed_forward.py [--tokens 2048] [--width 512] [--hidden 1400] [--steps 60] [--serve 32]
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
import paper_2508_03984_amd as oz  # noqa: E402

SILU = 0


class Weight:
    """rows x cols in binary32, and its conversions: `as_is` for products over its columns, `turned` over its rows."""

    def __init__(self, rows, cols):
        self.rows, self.cols = rows, cols
        self.master = torch.zeros(rows, cols, device="cuda")
        self.grad = torch.empty(rows, cols, device="cuda")
        self.as_is, self.turned = oz.F8.empty(rows, cols, 128), oz.F8.empty(cols, rows, 128)

    def convert(self):
        oz.oz2_f8_quantize(self.rows, self.cols, self.master, self.cols, self.as_is, self.turned)


class Activations:
    """Memory for a number of tokens: what the forward pass leaves for the backward pass, and their conversions."""

    def __init__(self, m, width, hidden, train):
        def half(*shape):
            return torch.empty(*shape, dtype=torch.bfloat16, device="cuda")

        up = (hidden + 127) // 128 * 128
        wide = up + hidden
        self.m, self.h, self.y = m, half(m, hidden), half(m, width)
        self.x8, self.h8 = oz.F8.empty(m, width), oz.F8.empty(m, hidden)
        self.z = self.xt8 = self.ht8 = None
        if train:
            self.z, self.dh = half(m, wide), half(m, hidden)
            self.xt8, self.ht8 = oz.F8.empty(width, m), oz.F8.empty(hidden, m)
            self.dy8, self.dyt8 = oz.F8.empty(m, width), oz.F8.empty(width, m)
            self.d8, self.dt8 = oz.F8.empty(m, wide), oz.F8.empty(wide, m)


class FeedForward:
    def __init__(self, width, hidden, seed=0):
        self.width, self.hidden = width, hidden
        self.up = (hidden + 127) // 128 * 128                 # the rows of Wu begin at a whole block
        self.gate_up, self.down = Weight(self.up + hidden, width), Weight(width, hidden)
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.gate_up.master[:hidden].normal_(0, width ** -0.5, generator=gen)
        self.gate_up.master[self.up:].normal_(0, width ** -0.5, generator=gen)
        self.down.master.normal_(0, hidden ** -0.5, generator=gen)
        # The products' memory, kept between calls and where it is: what a captured graph holds stays valid when later calls need more.  Training
        # and all servers of the block share it, so their calls and replays are ordered, on one stream or by events.
        self.ctx = oz.oz2_create()
        self.convert()

    def close(self):
        """Frees the products' memory.  No graph that was captured with the block may run after it."""
        oz.oz2_destroy(self.ctx)

    def weights(self):
        return (self.gate_up, self.down)

    def convert(self):
        for w in self.weights():
            w.convert()

    def forward(self, x, a):
        """y of x (tokens x width), in a.y."""
        w, f, m = self.width, self.hidden, a.m
        oz.oz2_f8_quantize(m, w, x, w, a.x8, a.xt8)
        oz.oz2_ctx_f8_gated(self.ctx, m, f, w, SILU, a.x8, self.gate_up.as_is, a.h, f, a.z, self.up + f if a.z is not None else 0)
        oz.oz2_f8_quantize(m, f, a.h, f, a.h8, a.ht8)
        oz.oz2_ctx_f8_gemm(self.ctx, m, w, f, 1.0, a.h8, self.down.as_is, 0.0, a.y, w)
        return a.y

    def backward(self, dy, a, dx=None):
        """The weights' gradients, and that of x in `dx` if it is given, from the gradient of y."""
        w, f, m, wide = self.width, self.hidden, a.m, self.up + self.hidden
        oz.oz2_f8_quantize(m, w, dy, w, a.dy8, a.dyt8)
        oz.oz2_ctx_f8_gemm(self.ctx, w, f, m, 1.0, a.dyt8, a.ht8, 0.0, self.down.grad, f)
        oz.oz2_ctx_f8_gemm(self.ctx, m, f, w, 1.0, a.dy8, self.down.turned, 0.0, a.dh, f)
        oz.oz2_f8_gated_grad(m, f, SILU, a.z, wide, a.dh, f, a.d8, a.dt8)
        oz.oz2_ctx_f8_gemm(self.ctx, wide, w, m, 1.0, a.dt8, a.xt8, 0.0, self.gate_up.grad, w)
        if dx is not None:
            oz.oz2_ctx_f8_gemm(self.ctx, m, w, wide, 1.0, a.d8, self.gate_up.turned, 0.0, dx, w)


def train(block, teacher, tokens, steps, rate=2e-3, tell=None):
    """Fits the block to `teacher`, a function from x to y.  The losses of all steps."""
    params = [torch.nn.Parameter(w.master) for w in block.weights()]       # the same memory as the weights'
    adam = torch.optim.Adam(params, lr=rate)
    a = Activations(tokens, block.width, block.hidden, True)
    gen = torch.Generator(device="cuda").manual_seed(1)
    losses = []
    for step in range(steps):
        x = torch.randn(tokens, block.width, device="cuda", generator=gen).bfloat16()
        off = block.forward(x, a).float() - teacher(x)
        losses.append(off.square().mean())
        block.backward((off * (2 / block.width)).bfloat16(), a)
        for p, w in zip(params, block.weights()):
            p.grad = w.grad / tokens
        adam.step()
        block.convert()
        if tell and step % 10 == 9:
            tell(f"step {step + 1}: loss {losses[-1].item():.4f}")
    return [float(v) for v in losses]


class Server:
    """One token at a time, or `tokens` of them, as one captured graph that is replayed: fill `x`, call, read `y`."""

    def __init__(self, block, tokens=1):
        self.x = torch.zeros(tokens, block.width, dtype=torch.bfloat16, device="cuda")
        self.a = Activations(tokens, block.width, block.hidden, False)
        self.y = self.a.y
        block.forward(self.x, self.a)                         # memory is allocated before the capture, not in it
        torch.cuda.synchronize()
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            block.forward(self.x, self.a)

    def __call__(self, x):
        self.x.copy_(x)
        self.graph.replay()
        return self.y


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", type=int, default=2048)
    ap.add_argument("--width", type=int, default=512)
    ap.add_argument("--hidden", type=int, default=1400)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--serve", type=int, default=32)
    o = ap.parse_args()
    block, other = FeedForward(o.width, o.hidden), FeedForward(o.width, o.hidden, seed=5)
    memory = Activations(o.tokens, o.width, o.hidden, False)
    losses = train(block, lambda x: other.forward(x, memory).float(), o.tokens, o.steps, tell=lambda s: print(s, flush=True))
    print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f}")
    server = Server(block)
    x = torch.randn(o.serve, 1, o.width, device="cuda").bfloat16()
    server(x[0])
    torch.cuda.synchronize()
    began = time.perf_counter()
    for t in x:
        server(t)
    torch.cuda.synchronize()
    print(f"{(time.perf_counter() - began) / o.serve * 1e6:.1f} us per token")
    block.close()
    other.close()


if __name__ == "__main__":
    main()
