"""Products in 8-bit integers with a scale for each token and channel, alone and grouped by expert, as cases that can be timed and compared.

A matrix in 8-bit integers is whole numbers q of -127 .. 127 (`torch.int8`) and one binary32 number for each row: s = max|x| / 127 over the
row, rounded to binary32, 2^-126 at least; q is the whole number next to x / s, ties to even.  The operators ("op" of a case):

  quantize   `batch` matrices of rows x cols numbers of `dtype` into that form, as they are ("as_is"), each transposed ("transposed": a scale
             belongs to a column of the matrix), or both from one call
  dispatch   the same of tokens on their way to experts.  Row r of what is written is token index[r] (a row of zeros where the index is -1), rows
             offsets[g] .. offsets[g + 1] - 1 belong to expert g.  Transposed, the rows of an expert lie side by side from column
             offsets[g] / 128 * 128 + 128 g on (the quotient rounded down), with a scale for each expert and column
  product    C = A B^T for A: m x k, B: n x k in that form, C of type `dtype`
  grouped    row r of C is A's row r times the transpose of its expert's weight, n x k; the weights are one matrix of groups * n rows
  gradient   the backward pass of grouped: from dY (rows x n of `dtype`) its forms in 8-bit integers, as it is and transposed, then dX = dY W by
             expert, and dW = dY^T X of each expert (the rest in 8-bit integers from before)
"""
from __future__ import annotations

import math

import torch

own = False

MODES = {"as_is": (True, False), "transposed": (False, True), "both": (True, True)}
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
MOST = 2 * 8192 * 16384 * 16384                                # operations of the largest product
MOST_NUMBERS = 16384 * 8192                                    # of the largest conversion
MOST_WEIGHTS = 64 * 4096 * 4096                                # of all experts


def listed():
    return [
        # a batch of single tokens on its way into a product
        {"name": "quantize_64x8192", "op": "quantize", "batch": 1, "rows": 64, "cols": 8192, "dtype": "bf16", "mode": "as_is"},
        # the weights of eight experts after an optimizer step, for the products forward and backward
        {"name": "quantize_8x4096x2048", "op": "quantize", "batch": 8, "rows": 4096, "cols": 2048, "dtype": "f32", "mode": "both"},
        # a training batch on its way to two of eight experts each
        {"name": "dispatch_8192x4096_2of8", "op": "dispatch", "tokens": 8192, "each": 2, "cols": 4096, "groups": 8, "spare": 0, "dtype": "bf16",
         "mode": "both"},
        # a prompt of no round size on its way to eight of 64 experts each, in a buffer with rows to spare
        {"name": "dispatch_333x1111_8of64", "op": "dispatch", "tokens": 333, "each": 8, "cols": 1111, "groups": 64, "spare": 100, "dtype": "f16",
         "mode": "as_is"},
        # one token through a square layer: the weight is read once
        {"name": "product_1x8192x8192", "op": "product", "m": 1, "n": 8192, "k": 8192, "dtype": "bf16"},
        # a small layer of no round size
        {"name": "product_500x300x777", "op": "product", "m": 500, "n": 300, "k": 777, "dtype": "f16"},
        # a large layer over a large batch
        {"name": "product_8192x16384x16384", "op": "product", "m": 8192, "n": 16384, "k": 16384, "dtype": "bf16"},
        # a token through eight of 64 experts: their weights are read once
        {"name": "grouped_1x4096x2048_8of64", "op": "grouped", "tokens": 1, "each": 8, "n": 4096, "k": 2048, "groups": 64, "spare": 0, "dtype": "bf16"},
        # a prompt of no round size through four of 24 experts of no round size
        {"name": "grouped_333x1500x1111_4of24", "op": "grouped", "tokens": 333, "each": 4, "n": 1500, "k": 1111, "groups": 24, "spare": 50, "dtype": "f16"},
        # a large batch through eight of 64 experts
        {"name": "grouped_8192x4096x4096_8of64", "op": "grouped", "tokens": 8192, "each": 8, "n": 4096, "k": 4096, "groups": 64, "spare": 0, "dtype": "bf16"},
        # the gradients of a few small experts over a batch of no round size
        {"name": "gradient_777x1000x500_2of5", "op": "gradient", "tokens": 777, "each": 2, "n": 1000, "k": 500, "groups": 5, "spare": 30, "dtype": "f16"},
        # the gradients of a training batch
        {"name": "gradient_8192x4096x2048_2of8", "op": "gradient", "tokens": 8192, "each": 2, "n": 4096, "k": 2048, "groups": 8, "spare": 0,
         "dtype": "bf16"},
    ]


def draw(rng):
    def size(lo, hi):
        return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))

    def experts(tokens):
        groups = size(2, 128)
        return {"tokens": size(1, tokens), "each": rng.randint(1, min(8, groups)), "groups": groups, "spare": rng.choice((0, 0, size(1, 500)))}

    op = rng.choice(("quantize", "dispatch", "product", "product", "grouped", "grouped", "gradient"))
    while True:
        dtype = rng.choice(("bf16", "f16", "f32"))
        if op == "quantize":
            c = {"batch": rng.choice((1, 1, size(2, 64))), "rows": size(1, 16384), "cols": size(16, 16384), "mode": rng.choice(tuple(MODES))}
            fits = c["batch"] * c["rows"] * c["cols"] <= MOST_NUMBERS // (2 if dtype == "f32" else 1)
        elif op == "dispatch":
            c = {**experts(16384), "cols": size(16, 16384), "mode": rng.choice(tuple(MODES))}
            fits = _rows(c) * c["cols"] <= MOST_NUMBERS // 2
        elif op == "product":
            c = {"m": size(1, 16384), "n": size(16, 16384), "k": size(32, 40000)}
            fits = True
        elif op == "grouped":
            c = {**experts(8192), "n": size(16, 8192), "k": size(32, 8192)}
            fits = c["groups"] * c["n"] * c["k"] <= MOST_WEIGHTS and _rows(c) * max(c["n"], c["k"]) <= 2 * MOST_NUMBERS
        else:
            c = {**experts(8192), "n": size(16, 4096), "k": size(32, 4096)}
            fits = c["groups"] * c["n"] * c["k"] <= MOST_WEIGHTS // 8 and _rows(c) * max(c["n"], c["k"]) <= MOST_NUMBERS
        c = {"op": op, **c, "dtype": dtype}
        if fits and work(c)["flops"] <= MOST:
            return c


def _rows(c):
    """Rows of the experts' matrices: a token's for each of its experts, and some to spare behind the last one."""
    return c["tokens"] * c["each"] + c["spare"]


def _wide(rows, groups):
    """Columns of a matrix that is transposed by experts."""
    return rows // 128 * 128 + 128 * groups


# ------------------------------------------------------------------ the plain form
def _scales(top):
    return (top / 127).clamp(min=2.0 ** -126)


def _whole(x, scale):
    """The whole numbers next to x / scale: in 64 bits, since 32 put some quotients beside a half onto it."""
    return torch.round(x.double() / scale.double()).to(torch.int8)


def _quantize(x):
    """(whole numbers, scales) of the rows of x."""
    s = _scales(x.float().abs().amax(-1))
    return _whole(x, s[..., None]), s


def _places(st):
    """Of each row that an expert has: its expert, and its column where rows lie side by side."""
    off = st["offsets"].long()
    lengths = off[1:] - off[:-1]
    expert = torch.repeat_interleave(torch.arange(lengths.numel(), device=off.device), lengths, output_size=st["used"])
    first = off[:-1] // 128 * 128 + 128 * torch.arange(lengths.numel(), device=off.device)
    return expert, first[expert] + torch.arange(st["used"], device=off.device) - off[expert]


def _quantize_grouped(st, x, mode):
    """What the experts get of x (a row for each of theirs)."""
    got, rows, (as_is, transposed) = {}, _rows(st["case"]), MODES[mode]
    x, groups, cols = x.float(), st["case"]["groups"], x.shape[1]
    if as_is:
        q, s = _quantize(x)
        got["as_is"] = torch.cat((q, q.new_zeros(rows - st["used"], cols))), torch.cat((s, s.new_zeros(rows - st["used"])))
    if transposed:
        expert, place = _places(st)
        s = _scales(x.new_zeros(groups, cols).index_reduce_(0, expert, x.abs(), "amax"))
        q = torch.zeros(cols, _wide(rows, groups), dtype=torch.int8, device=x.device)
        q[:, place] = _whole(x, s[expert]).t()
        got["transposed"] = q, s
    return got


def _product(a, b):
    return (a[0].float() @ b[0].float().t()) * a[1][:, None] * b[1]


def _grouped(st, a, b, n, dtype):
    """By expert: a's rows, in order, with b's rows from expert * n on."""
    out = torch.zeros(a[0].shape[0], n, dtype=dtype, device=a[0].device)
    for g, (lo, hi) in enumerate(st["bounds"]):
        if lo < hi:
            out[lo:hi] = _product((a[0][lo:hi], a[1][lo:hi]), (b[0][g * n:(g + 1) * n], b[1][g * n:(g + 1) * n])).to(dtype)
    return out


def _run_plain(st):
    c = st["case"]
    dtype = DTYPES[c["dtype"]]
    if c["op"] == "quantize":
        got, x = {}, st["x"].view(c["batch"], c["rows"], c["cols"])
        if "as_is" in st["out"]:
            got["as_is"] = tuple(v.flatten(0, 1) for v in _quantize(x))
        if "transposed" in st["out"]:
            got["transposed"] = tuple(v.flatten(0, 1).contiguous() for v in _quantize(x.mT))
        return got
    if c["op"] == "dispatch":
        index = st["index"][: st["used"]].long()
        return _quantize_grouped(st, st["x"][index.clamp(min=0)] * (index >= 0)[:, None], c["mode"])
    if c["op"] == "product":
        return _product(st["a"], st["b"]).to(dtype)
    if c["op"] == "grouped":
        return _grouped(st, st["a"], st["b"], c["n"], dtype)
    n, k = c["n"], c["k"]
    d = _quantize_grouped(st, st["dy"][: st["used"]], "both")
    dx = _grouped(st, d["as_is"], st["wt"], k, dtype)
    dw = torch.zeros(c["groups"] * n, k, dtype=dtype, device=dx.device)
    for g, (lo, hi) in enumerate(st["bounds"]):
        first = lo // 128 * 128 + 128 * g
        part = slice(first, first + hi - lo)
        dw[g * n:(g + 1) * n] = _product((d["transposed"][0][:, part], d["transposed"][1][g]), (st["xt"][0][:, part], st["xt"][1][g])).to(dtype)
    return dx, dw


# ------------------------------------------------------------------ the framework's calls
def _run_own(st):
    import paper_2508_03984_amd as oz
    c, out = st["case"], st["out"]
    if c["op"] == "quantize":
        oz.oz2_i8_quantize(c["batch"], c["rows"], c["cols"], st["x"], c["cols"], out.get("as_is"), out.get("transposed"))
        return {name: (m.q, m.scale) for name, m in out.items()}
    if c["op"] == "product":
        oz.oz2_i8_gemm(c["m"], c["n"], c["k"], 1.0, st["a"], st["b"], 0.0, out["c"], c["n"])
        return out["c"]
    rows, groups, off = _rows(c), c["groups"], st["offsets"]
    if c["op"] == "dispatch":
        oz.oz2_i8_quantize_grouped(rows, c["cols"], st["x"], c["tokens"], c["cols"], st["index"], groups, off, out.get("as_is"), out.get("transposed"))
        return {name: (m.q, m.scale) for name, m in out.items()}
    n, k = c["n"], c["k"]
    if c["op"] == "grouped":
        oz.oz2_i8_grouped_gemm(rows, n, k, groups, off, 1.0, st["a"], st["b"], 0.0, out["c"], n)
        return out["c"]
    oz.oz2_i8_quantize_grouped(rows, n, st["dy"], rows, n, None, groups, off, out["d"], out["dt"])
    oz.oz2_i8_grouped_gemm(rows, k, n, groups, off, 1.0, out["d"], st["wt"], 0.0, out["dx"], k)
    oz.oz2_i8_grouped_grad(n, k, rows, groups, off, 1.0, out["dt"], st["xt"], 0.0, out["dw"], k)
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


def _weight8(gen, rows, cols):
    """A weight in 8-bit integers: normal numbers, whose largest is about 3.5 of their deviations in a row."""
    q = (torch.randn(rows, cols, device="cuda", generator=gen) * 36).round_().clamp_(-127, 127).to(torch.int8)
    return q, cols ** -0.5 / 36 * torch.exp(0.2 * torch.randn(rows, device="cuda", generator=gen))


def _routed(gen, c):
    """Which experts have which tokens: `each` different ones a token, some experts more sought than others, rows in the order of experts."""
    liking = 0.7 * torch.randn(c["groups"], device="cuda", generator=gen)
    chance = torch.rand(c["tokens"], c["groups"], device="cuda", generator=gen).clamp_(min=1e-7)
    expert = (liking - torch.log(-torch.log(chance))).topk(c["each"], dim=1).indices.flatten()
    order = torch.sort(expert, stable=True).indices
    count = torch.zeros(c["groups"] + 1, dtype=torch.int64, device="cuda").index_add_(0, expert + 1, torch.ones_like(expert))
    index = torch.full((_rows(c),), -1, dtype=torch.int32, device="cuda")
    index[: order.numel()] = (order // c["each"]).int()
    if c["tokens"] > 4:
        index[: order.numel()][order % 97 == 96] = -1           # places that stayed empty
    offsets = count.cumsum(0)
    bounds = offsets.tolist()
    return {"index": index, "offsets": offsets.int(), "bounds": list(zip(bounds[:-1], bounds[1:])), "used": order.numel()}


def _inputs(case, seed):
    """What the operator reads: numbers, or pairs of whole numbers and scales."""
    gen = torch.Generator("cuda").manual_seed(int(seed))
    c = case
    dtype = DTYPES[c["dtype"]]
    if c["op"] == "quantize":
        return {"x": _activations(gen, c["batch"] * c["rows"], c["cols"]).to(dtype)}
    if c["op"] == "product":
        return {"a": _quantize(_activations(gen, c["m"], c["k"])), "b": _weight8(gen, c["n"], c["k"])}
    st = {"case": dict(c), **_routed(gen, c)}
    rows, groups = _rows(c), c["groups"]
    if c["op"] == "dispatch":
        return {**st, "x": _activations(gen, c["tokens"], c["cols"]).to(dtype)}
    if c["op"] == "grouped":
        return {**st, "a": _quantize(_activations(gen, rows, c["k"])), "b": _weight8(gen, groups * c["n"], c["k"])}
    dy = torch.randn(rows, c["n"], device="cuda", generator=gen) * 1e-3
    dy[-1] = 0
    xt = _quantize_grouped(st, _activations(gen, rows, c["k"])[: st["used"]], "transposed")["transposed"]
    return {**st, "dy": dy.to(dtype), "xt": xt, "wt": _weight8(gen, groups * c["k"], c["n"])}


def prepare(case, seed):
    c, st, out = case, _inputs(case, seed), {}
    if c["op"] in ("quantize", "dispatch"):
        out = {name: None for name, asked in zip(("as_is", "transposed"), MODES[c["mode"]]) if asked}
    if own:                                                     # the handles and the buffers that a program keeps
        import paper_2508_03984_amd as oz
        st = {name: oz.I8.of(*v) if isinstance(v, tuple) else v for name, v in st.items()}
        new = lambda *shape: torch.zeros(*shape, device="cuda", dtype=DTYPES[c["dtype"]])  # noqa: E731

        def empty(rows, cols, groups=1):
            m = oz.I8.empty(rows, cols, groups)
            m.q.zero_()
            m.scale.zero_()
            return m

        if c["op"] == "quantize":
            shape = {"as_is": (c["batch"] * c["rows"], c["cols"]), "transposed": (c["batch"] * c["cols"], c["rows"])}
            out = {name: empty(*shape[name]) for name in out}
        elif c["op"] == "dispatch":
            rows, groups = _rows(c), c["groups"]
            shape = {"as_is": (rows, c["cols"]), "transposed": (c["cols"], _wide(rows, groups), groups)}
            out = {name: empty(*shape[name]) for name in out}
        elif c["op"] == "product":
            out["c"] = new(c["m"], c["n"])
        elif c["op"] == "grouped":
            out["c"] = new(_rows(c), c["n"])
        else:
            rows, n, k, groups = _rows(c), c["n"], c["k"], c["groups"]
            out = {"d": empty(rows, n), "dt": empty(n, _wide(rows, groups), groups), "dx": new(rows, k), "dw": new(groups * n, k)}
    return {"case": dict(case), **st, "out": out}


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c, size = case, {"bf16": 2, "f16": 2, "f32": 4}[case["dtype"]]
    if c["op"] == "quantize":
        numbers, forms = c["batch"] * c["rows"] * c["cols"], sum(MODES[c["mode"]])
        as_is, transposed = MODES[c["mode"]]
        return {"bytes": (size + forms) * numbers + 4 * c["batch"] * (as_is * c["rows"] + transposed * c["cols"]), "flops": (1 + 2 * forms) * numbers}
    if c["op"] == "product":
        m, n, k = c["m"], c["n"], c["k"]
        return {"bytes": (m + n) * (k + 4) + size * m * n, "flops": 2 * m * n * k}
    slots, groups = c["tokens"] * c["each"], c["groups"]
    if c["op"] == "dispatch":
        as_is, transposed = MODES[c["mode"]]
        numbers, forms = slots * c["cols"], as_is + transposed
        scales = 4 * (as_is * slots + transposed * groups * c["cols"])
        return {"bytes": size * c["tokens"] * c["cols"] + forms * numbers + scales + 4 * slots, "flops": (1 + 2 * forms) * numbers}
    n, k, sought = c["n"], c["k"], min(groups, slots)           # experts that have tokens, at most
    if c["op"] == "grouped":
        return {"bytes": slots * (k + 4) + sought * n * (k + 4) + size * slots * n, "flops": 2 * slots * n * k}
    read = size * slots * n + sought * k * (n + 4) + slots * k + 4 * sought * k
    return {"bytes": read + size * (slots * k + groups * n * k), "flops": 4 * slots * n * k}


# ------------------------------------------------------------------ the definition in 64 bits
def _exact_quantize(x):
    """By rows: the scale is the binary32 number next to max|x| / 127, then the whole number whose distance to x / scale is least, the even one of two."""
    scale = torch.maximum(x.abs().max(-1).values / 127, torch.tensor(2.0 ** -126, dtype=torch.float64, device=x.device)).float().double()
    t = (x / scale.unsqueeze(-1)).abs_()
    q = torch.floor(t)
    t -= q
    q += (t > 0.5) | ((t == 0.5) & (q % 2 == 1))
    return torch.copysign(q, x).to(torch.int8), scale


def _exact_numbers(q, scale):
    return q.double() * scale.double().unsqueeze(-1)


def _exact_grouped(c, st, x):
    """Both forms of the experts' rows; x: a row for each."""
    rows, cols, groups = _rows(c), x.shape[1], c["groups"]
    q, s = torch.zeros(rows, cols, dtype=torch.int8, device=x.device), torch.zeros(rows, dtype=torch.float64, device=x.device)
    q[: x.shape[0]], s[: x.shape[0]] = _exact_quantize(x)
    tq = torch.zeros(cols, _wide(rows, groups), dtype=torch.int8, device=x.device)
    ts = torch.full((groups, cols), 2.0 ** -126, dtype=torch.float64, device=x.device)
    for g, (lo, hi) in enumerate(st["bounds"]):
        first = (lo >> 7 << 7) + (g << 7)
        if hi > lo:
            tq[:, first:first + hi - lo], ts[g] = _exact_quantize(x[lo:hi].t())
    return {"as_is": (q, s), "transposed": (tq, ts)}


def exact(case, seed):
    c, st = case, _inputs(case, seed)
    if c["op"] == "quantize":
        x, got = st["x"].double().unflatten(0, (c["batch"], c["rows"])), {}
        if MODES[c["mode"]][0]:
            q, s = _exact_quantize(x)
            got["as_is"] = q.reshape(-1, c["cols"]), s.reshape(-1)
        if MODES[c["mode"]][1]:
            q, s = _exact_quantize(x.transpose(1, 2))
            got["transposed"] = q.reshape(-1, c["rows"]), s.reshape(-1)
        return got
    if c["op"] == "dispatch":
        full = torch.cat((st["x"].double(), torch.zeros(1, c["cols"], dtype=torch.float64, device="cuda")))
        both = _exact_grouped(c, st, full[st["index"][: st["used"]].long()])         # (row -1 is the one of zeros)
        return {name: both[name] for name, asked in zip(("as_is", "transposed"), MODES[c["mode"]]) if asked}
    if c["op"] == "product":
        return _exact_numbers(*st["a"]) @ _exact_numbers(*st["b"]).t()
    rows, n, k = _rows(c), c["n"], c["k"]

    def by_expert(a, b, n):
        out = torch.zeros(rows, n, dtype=torch.float64, device="cuda")
        for g, (lo, hi) in enumerate(st["bounds"]):
            out[lo:hi] = _exact_numbers(a[0][lo:hi], a[1][lo:hi]) @ _exact_numbers(b[0][g * n:g * n + n], b[1][g * n:g * n + n]).t()
        return out

    if c["op"] == "grouped":
        return by_expert(st["a"], st["b"], n)
    d = _exact_grouped(c, st, st["dy"][: st["used"]].double())
    dw = torch.zeros(c["groups"], n, k, dtype=torch.float64, device="cuda")
    for g, (lo, hi) in enumerate(st["bounds"]):
        part = slice((lo >> 7 << 7) + (g << 7), (lo >> 7 << 7) + (g << 7) + hi - lo)
        dw[g] = _exact_numbers(d["transposed"][0][:, part], d["transposed"][1][g]) @ _exact_numbers(st["xt"][0][:, part], st["xt"][1][g]).t()
    return by_expert(d["as_is"], st["wt"], k), dw.reshape(-1, k)
