"""The 8-bit floating-point products of feed-forward layers, as cases that can be timed and compared.

A matrix in 8 bits is E4M3 numbers (`torch.float8_e4m3fn`) with one power of two per block (`torch.float8_e8m0fnu`): the
smallest 2^s, s >= -126, with max|x| <= 448 * 2^s over the block's elements, 2^0 for a block of zeros.  A block is 128
elements of one row, or 128 x 128 elements; blocks at the edges are smaller.  The operators ("op" of a case):

  quantize   rows x cols numbers of `dtype` into that form, as they are ("as_is"), transposed ("transposed": blocks run
             along the rows of the transpose), or both from one call
  product    C = A B^T for A: m x k, B: n x k in that form, C of type `dtype`.  A has blocks of one row; B of 128 rows
             (`b_rows` 128: a weight) or of one (`b_rows` 1: both factors are activations or their gradients)
  gated      H = act(X Wg^T) * (X Wu^T) for X: m x k with blocks of one row and Wg, Wu: f x k with blocks of 128 rows.  The two
             weights are one matrix, Wu's rows from f rounded up to 128 on.  `train`: also Z = X W^T, for the gradient; H
             and Z are of type `dtype`
  gradient   the backward pass of gated: from Z and dH the gradients D of Z in 8 bits with blocks of one row, as they are and
             transposed, then dX = D W and dW = D^T X
"""
from __future__ import annotations

import math

import torch

own = False

MODES = {"as_is": (True, False), "transposed": (False, True), "both": (True, True)}
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
MOST = 2 * 8192 * 16384 * 16384                                # operations of the largest product


def listed():
    return [
        # a batch of single tokens on its way into a product
        {"name": "quantize_64x8192", "op": "quantize", "rows": 64, "cols": 8192, "dtype": "bf16", "block_rows": 1, "mode": "as_is"},
        # activations of no round size, for a product and for the gradient of the weight
        {"name": "quantize_1500x1111", "op": "quantize", "rows": 1500, "cols": 1111, "dtype": "f32", "block_rows": 1, "mode": "both"},
        # a weight after an optimizer step, for the products forward and backward
        {"name": "quantize_16384x8192", "op": "quantize", "rows": 16384, "cols": 8192, "dtype": "bf16", "block_rows": 128, "mode": "both"},
        # one token through a square layer: the weight is read once
        {"name": "product_1x8192x8192", "op": "product", "m": 1, "n": 8192, "k": 8192, "b_rows": 128, "dtype": "bf16"},
        # a small layer of no round size
        {"name": "product_500x300x777", "op": "product", "m": 500, "n": 300, "k": 777, "b_rows": 128, "dtype": "f16"},
        # the gradient of a small weight over many tokens: a long contraction and few outputs
        {"name": "product_1536x1000x40000", "op": "product", "m": 1536, "n": 1000, "k": 40000, "b_rows": 1, "dtype": "bf16"},
        # a large layer over a large batch
        {"name": "product_8192x16384x16384", "op": "product", "m": 8192, "n": 16384, "k": 16384, "b_rows": 128, "dtype": "bf16"},
        # four tokens of a decoder through the block
        {"name": "gated_4x16384x4096", "op": "gated", "m": 4, "f": 16384, "k": 4096, "act": "silu", "train": False, "dtype": "bf16"},
        # a prompt of no round size through a block of no round size
        {"name": "gated_1000x1500x1111", "op": "gated", "m": 1000, "f": 1500, "k": 1111, "act": "gelu", "train": False, "dtype": "f16"},
        # a training batch
        {"name": "gated_8192x8192x4096", "op": "gated", "m": 8192, "f": 8192, "k": 4096, "act": "silu", "train": True, "dtype": "bf16"},
        # the gradients of a small block
        {"name": "gradient_777x1000x500", "op": "gradient", "m": 777, "f": 1000, "k": 500, "act": "gelu", "dtype": "f16"},
        # the gradients of the training batch
        {"name": "gradient_8192x8192x4096", "op": "gradient", "m": 8192, "f": 8192, "k": 4096, "act": "silu", "dtype": "bf16"},
    ]


def draw(rng):
    def size(lo, hi):
        return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))

    op = rng.choice(("quantize", "product", "product", "gated", "gated", "gradient"))
    while True:
        if op == "quantize":
            c = {"rows": size(1, 16384), "cols": size(16, 16384), "dtype": rng.choice(("bf16", "f16", "f32")),
                 "block_rows": rng.choice((1, 128)), "mode": rng.choice(("as_is", "transposed", "both"))}
            fits = c["rows"] * c["cols"] <= 16384 * 8192 // (2 if c["dtype"] == "f32" else 1)
        elif op == "product":
            c = {"m": size(1, 16384), "n": size(16, 16384), "k": size(32, 40000), "b_rows": rng.choice((1, 128)),
                 "dtype": rng.choice(("bf16", "f16"))}
            fits = True
        elif op == "gated":
            c = {"m": size(1, 8192), "f": size(16, 16384), "k": size(32, 8192), "act": rng.choice(("silu", "gelu")),
                 "train": rng.choice((False, True)), "dtype": rng.choice(("bf16", "f16"))}
            fits = True
        else:
            c = {"m": size(16, 8192), "f": size(16, 8192), "k": size(32, 4096), "act": rng.choice(("silu", "gelu")),
                 "dtype": rng.choice(("bf16", "f16"))}
            fits = True
        c = {"op": op, **c}
        if fits and work(c)["flops"] <= MOST:
            return c


def _up(f):
    return -(-f // 128) * 128                                  # first row of Wu


# ------------------------------------------------------------------ the plain form
def _blocks(x, block_rows):
    """x, filled up with zeros, as (blocks of rows, rows of a block, blocks of columns, 128)."""
    r, c = x.shape
    rb, cb = -(-r // block_rows), -(-c // 128)
    full = x.new_zeros(rb * block_rows, cb * 128)
    full[:r, :c] = x
    return full.view(rb, block_rows, cb, 128)


def _power(s):
    """2^s for whole s in -126 .. 127, exactly: the bits of a binary32 number."""
    return ((s.int() + 127) << 23).view(torch.float32)


def _quantize(x, block_rows):
    """(E4M3 numbers, E8M0 scales) of x."""
    b = _blocks(x.float(), block_rows)
    frac, exp = torch.frexp(b.abs().amax(dim=(1, 3)))           # max = frac 2^exp, 448 = 0.875 * 2^9
    s = torch.where(frac == 0, 0, (exp - 9 + (frac > 0.875).int()).clamp(min=-126))
    q = (b * _power(-s)[:, None, :, None]).reshape(b.shape[0] * block_rows, -1)[: x.shape[0], : x.shape[1]]
    return q.to(torch.float8_e4m3fn).contiguous(), (s + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _numbers(q, scale, block_rows):
    """The numbers that a matrix in 8 bits stands for."""
    s = scale.float().repeat_interleave(block_rows, 0)[: q.shape[0]].repeat_interleave(128, 1)[:, : q.shape[1]]
    return q.float() * s


def _act(g, kind):
    if kind == "silu":
        return g / (1 + torch.exp(-g))
    return 0.5 * g * (1 + torch.tanh(0.7978845608028654 * (g + 0.044715 * g * g * g)))


def _act_slope(g, kind):
    if kind == "silu":
        p = 1 / (1 + torch.exp(-g))
        return p * (1 + g * (1 - p))
    t = torch.tanh(0.7978845608028654 * (g + 0.044715 * g * g * g))
    return 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * 0.7978845608028654 * (1 + 3 * 0.044715 * g * g)


def _run_plain(st):
    c = st["case"]
    if c["op"] == "quantize":
        got = {}
        if "as_is" in st["out"]:
            got["as_is"] = _quantize(st["x"], c["block_rows"])
        if "transposed" in st["out"]:
            got["transposed"] = _quantize(st["x"].t(), c["block_rows"])
        return got
    dtype = DTYPES[c["dtype"]]
    if c["op"] == "product":
        return (_numbers(*st["a"]) @ _numbers(*st["b"]).t()).to(dtype)
    f, up = c["f"], _up(c["f"])
    if c["op"] == "gated":
        z = _numbers(*st["x"]) @ _numbers(*st["w"]).t()
        h = _act(z[:, :f], c["act"]) * z[:, up:]
        return (h.to(dtype), z[:, :f].to(dtype), z[:, up:].to(dtype)) if c["train"] else h.to(dtype)
    g, u, dh = st["z"][:, :f].float(), st["z"][:, up:].float(), st["dh"].float()
    d = torch.zeros(c["m"], up + f, device=g.device)
    d[:, :f] = dh * u * _act_slope(g, c["act"])
    d[:, up:] = dh * _act(g, c["act"])
    dx = _numbers(*_quantize(d, 1), 1) @ _numbers(*st["wt"]).t()
    dw = _numbers(*_quantize(d.t(), 1), 1) @ _numbers(*st["xt"]).t()
    return dx.to(dtype), dw.to(dtype)


# ------------------------------------------------------------------ the framework's calls
def _run_own(st):
    import paper_2508_03984_amd as oz
    c, out = st["case"], st["out"]
    if c["op"] == "quantize":
        oz.oz2_f8_quantize(c["rows"], c["cols"], st["x"], st["x"].stride(0), out.get("as_is"), out.get("transposed"))
        return {name: (m.q, m.scale) for name, m in out.items()}
    if c["op"] == "product":
        oz.oz2_f8_gemm(c["m"], c["n"], c["k"], 1.0, st["a"], st["b"], 0.0, out["c"], c["n"])
        return out["c"]
    f, up, act = c["f"], _up(c["f"]), oz.OZ2_ACT_SILU if c["act"] == "silu" else oz.OZ2_ACT_GELU
    if c["op"] == "gated":
        oz.oz2_f8_gated(c["m"], f, c["k"], act, st["x"], st["w"], out["h"], f, out.get("z"), up + f)
        return (out["h"], out["z"][:, :f], out["z"][:, up:]) if c["train"] else out["h"]
    oz.oz2_f8_gated_grad(c["m"], f, act, st["z"], up + f, st["dh"], f, out["d"], out["dt"])
    oz.oz2_f8_gemm(c["m"], c["k"], up + f, 1.0, out["d"], st["wt"], 0.0, out["dx"], c["k"])
    oz.oz2_f8_gemm(up + f, c["k"], c["m"], 1.0, out["dt"], st["xt"], 0.0, out["dw"], c["k"])
    return out["dx"], out["dw"]


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------------------------ inputs
def _activations(gen, rows, cols):
    """Numbers of a spread that differs between the columns; the last of several rows is padding, all zero."""
    x = torch.randn(rows, cols, device="cuda", generator=gen) * torch.exp(0.5 * torch.randn(cols, device="cuda", generator=gen))
    if rows > 4:
        x[-1] = 0
    return x


def _weight(gen, rows, cols):
    return torch.randn(rows, cols, device="cuda", generator=gen) * cols ** -0.5


def _stacked(gen, f, k):
    w = _weight(gen, _up(f) + f, k)
    w[f:_up(f)] = 0
    return w


def _inputs(case, seed):
    """What the operator reads: numbers, or pairs of E4M3 numbers and scales with their rows of a block."""
    gen = torch.Generator("cuda").manual_seed(int(seed))
    c = case
    if c["op"] == "quantize":
        x = _activations(gen, c["rows"], c["cols"]) if c["block_rows"] == 1 else _weight(gen, c["rows"], c["cols"])
        return {"x": x.to(DTYPES[c["dtype"]])}
    if c["op"] == "product":
        b = _activations(gen, c["n"], c["k"]) if c["b_rows"] == 1 else _weight(gen, c["n"], c["k"])
        return {"a": (*_quantize(_activations(gen, c["m"], c["k"]), 1), 1), "b": (*_quantize(b, c["b_rows"]), c["b_rows"])}
    m, f, k, dtype = c["m"], c["f"], c["k"], DTYPES[c["dtype"]]
    x, w = _activations(gen, m, k), _stacked(gen, f, k)
    if c["op"] == "gated":
        return {"x": (*_quantize(x, 1), 1), "w": (*_quantize(w, 128), 128)}
    z = torch.randn(m, _up(f) + f, device="cuda", generator=gen) * 1.5
    dh = torch.randn(m, f, device="cuda", generator=gen) * 1e-3
    dh[-1] = 0
    return {"z": z.to(dtype), "dh": dh.to(dtype), "wt": (*_quantize(w.t(), 128), 128), "xt": (*_quantize(x.t(), 1), 1)}


def prepare(case, seed):
    c, st, out = case, _inputs(case, seed), {}
    if c["op"] == "quantize":
        out = {name: None for name, asked in zip(("as_is", "transposed"), MODES[c["mode"]]) if asked}
    if own:                                                     # the handles and the buffers that a program keeps
        import paper_2508_03984_amd as oz
        st = {name: oz.F8.of(*v) if isinstance(v, tuple) else v for name, v in st.items()}
        new = lambda *shape: torch.empty(*shape, device="cuda", dtype=DTYPES[c["dtype"]])  # noqa: E731
        if c["op"] == "quantize":
            shape = {"as_is": (c["rows"], c["cols"]), "transposed": (c["cols"], c["rows"])}
            out = {name: oz.F8.empty(*shape[name], c["block_rows"]) for name in out}
        elif c["op"] == "product":
            out["c"] = new(c["m"], c["n"])
        elif c["op"] == "gated":
            m, f, up = c["m"], c["f"], _up(c["f"])
            out["h"] = new(m, f)
            if c["train"]:
                out["z"] = new(m, up + f)
        else:
            m, wide = c["m"], _up(c["f"]) + c["f"]
            out = {"d": oz.F8.empty(m, wide, 1), "dt": oz.F8.empty(wide, m, 1), "dx": new(m, c["k"]), "dw": new(wide, c["k"])}
    return {"case": dict(case), "out": out, **st}


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c, size = case, {"bf16": 2, "f16": 2, "f32": 4}[case["dtype"]]

    def bytes8(rows, cols, block_rows):
        return rows * cols + -(-rows // block_rows) * -(-cols // 128)

    if c["op"] == "quantize":
        r, k, b = c["rows"], c["cols"], c["block_rows"]
        as_is, transposed = MODES[c["mode"]]
        forms = as_is + transposed
        return {"bytes": size * r * k + as_is * bytes8(r, k, b) + transposed * bytes8(k, r, b), "flops": (1 + 2 * forms) * r * k}
    if c["op"] == "product":
        m, n, k = c["m"], c["n"], c["k"]
        return {"bytes": bytes8(m, k, 1) + bytes8(n, k, c["b_rows"]) + size * m * n, "flops": 2 * m * n * k}
    m, f, k = c["m"], c["f"], c["k"]
    if c["op"] == "gated":
        made = size * m * f * (3 if c["train"] else 1)
        return {"bytes": bytes8(m, k, 1) + 2 * bytes8(f, k, 128) + made, "flops": 4 * m * f * k}
    read = 3 * size * m * f + 2 * bytes8(f, k, 128) + bytes8(k, m, 1)
    return {"bytes": read + size * (m * k + 2 * f * k), "flops": 8 * m * f * k}


# ------------------------------------------------------------------ the definition in 64 bits
def _exact_power(s):
    """2^s: the bits of a binary64 number (a power function may be off by its last bit)."""
    return ((s.long() + 1023) * 2 ** 52).view(torch.float64)


def _exact_quantize(x, block_rows):
    r, k = x.shape
    rb, kb = math.ceil(r / block_rows), math.ceil(k / 128)
    q = torch.nn.functional.pad(x, (0, kb * 128 - k, 0, rb * block_rows - r)).unflatten(1, (kb, 128)).unflatten(0, (rb, block_rows))
    top = q.abs().amax(3).amax(1)
    s = torch.log2(top.clamp(min=2.0 ** -300) / 448).ceil()
    s = torch.where(top <= 448 * _exact_power(s - 1), s - 1, s)  # the logarithm is rounded
    s = torch.where(top > 448 * _exact_power(s), s + 1, s)
    scale = _exact_power(torch.where(top == 0, torch.zeros_like(s), s.clamp(min=-126)))
    q = q / scale[:, None, :, None]
    size = q.abs().clamp(min=2.0 ** -6)
    e = torch.log2(size).floor()
    e = torch.where(size < _exact_power(e), e - 1, e)
    step = _exact_power(e - 3)
    q = (q / step).round() * step                               # ties to even
    return q.flatten(2).flatten(0, 1)[:r, :k], scale


def _exact_numbers(q, scale, block_rows):
    r, k = q.shape
    rows = torch.arange(r, device=q.device) // block_rows
    cols = torch.arange(k, device=q.device) // 128
    return q.double() * scale.double()[rows][:, cols]


def exact(case, seed):
    c, st = case, _inputs(case, seed)
    if c["op"] == "quantize":
        x, got = st["x"].double(), {}
        as_is, transposed = MODES[c["mode"]]
        if as_is:
            got["as_is"] = _exact_quantize(x, c["block_rows"])
        if transposed:
            got["transposed"] = _exact_quantize(x.t(), c["block_rows"])
        return got
    if c["op"] == "product":
        return _exact_numbers(*st["a"]) @ _exact_numbers(*st["b"]).t()
    f, up = c["f"], _up(c["f"])

    def act(g):
        return g * torch.sigmoid(g) if c["act"] == "silu" else g * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3))

    if c["op"] == "gated":
        x, w = _exact_numbers(*st["x"]), _exact_numbers(*st["w"])
        g, u = x @ w[:f].t(), x @ w[up:].t()
        h = act(g) * u
        return (h, g, u) if c["train"] else h
    g, u, dh = st["z"][:, :f].double().requires_grad_(), st["z"][:, up:].double().requires_grad_(), st["dh"].double()
    dg, du = torch.autograd.grad((act(g) * u * dh).sum(), (g, u))
    gap = torch.zeros(c["m"], up - f, dtype=torch.float64, device=g.device)
    d = torch.cat((dg, gap, du), 1)
    dx = _exact_numbers(*_exact_quantize(d, 1), 1) @ _exact_numbers(*st["wt"]).t()
    dw = _exact_numbers(*_exact_quantize(d.t(), 1), 1) @ _exact_numbers(*st["xt"]).t()
    return dx, dw
