"""The library's operators in microscaled 4-bit floating point (MX: E2M1 elements, one power-of-two scale per 32
neighbours of a row): their workloads, each as a program that quantises, serves or trains calls it.

A microscaled matrix is two byte arrays.  Row r of q holds the elements, two to a byte, the lower column in the lower
four bits; row r of s holds one exponent (biased by 127) per 32 columns; the columns are padded with zeros to a multiple
of 128.  The operators:

  quantize   X -> its microscaled form, X^T's, or both, and back to values (what the 4 bits stand for)
  gemm       C = A * B^T, or C += A * B^T, both operands microscaled
  apply      Y = X * W^T (grad 0) or Y = X * W (grad 1), W microscaled and X in ordinary floating point
  step       a linear layer's training step: X, W and dY quantised in both forms, Y = X W^T, dX = dY W, dW = dY^T X
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
MOST = 8192               # the largest dimension of a product


def _quantize(name, dtype, rows, cols, forms):
    return {"name": name, "op": "quantize", "dtype": dtype, "rows": rows, "cols": cols, "forms": forms}


def _gemm(name, dtype, m, n, k, onto=0):
    return {"name": name, "op": "gemm", "dtype": dtype, "m": m, "n": n, "k": k, "onto": onto}


def _apply(name, dtype, m, n, k, grad=0):
    return {"name": name, "op": "apply", "dtype": dtype, "m": m, "n": n, "k": k, "grad": grad}


def _step(name, m, n, k):
    return {"name": name, "op": "step", "dtype": "bf16", "m": m, "n": n, "k": k}


def listed():
    return [
        # one token's activations on their way into a product: latency only
        _quantize("quantize_1x4096_bf16", "bf16", 1, 4096, "rows"),
        # a ragged batch, columns that no block divides, both forms
        _quantize("quantize_both_1000x1801_f16", "f16", 1000, 1801, "both"),
        # a large weight matrix in single precision, both forms: bandwidth
        _quantize("quantize_both_8192x8192_f32", "f32", 8192, 8192, "both"),
        # one token through a microscaled layer
        _gemm("gemm_1x8192x8192_bf16", "bf16", 1, 8192, 8192),
        # the E of the extralarge 3mm, added onto a gradient in single precision
        _gemm("gemm_onto_1600x1800x2000_f32", "f32", 1600, 1800, 2000, onto=1),
        # a long batch through a square layer: the largest product
        _gemm("gemm_8192x8192x8192_bf16", "bf16", 8192, 8192, 8192),
        # one token against microscaled weights, activations as they are
        _apply("apply_1x16384x4096_bf16", "bf16", 1, 16384, 4096),
        # a batch of sequences, one token each
        _apply("apply_48x8192x8192_f16", "f16", 48, 8192, 8192),
        # a prompt
        _apply("apply_4096x8192x8192_bf16", "bf16", 4096, 8192, 8192),
        # the gradient of a prompt through frozen weights
        _apply("apply_grad_2048x8192x8192_bf16", "bf16", 2048, 8192, 8192, grad=1),
        # the same, ragged and in single precision
        _apply("apply_grad_333x2200x1801_f32", "f32", 333, 2200, 1801, grad=1),
        # forward and backward of a layer
        _step("step_4096x8192x4096_bf16", 4096, 8192, 4096),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("quantize", "gemm", "apply", "apply", "step"))
    dtype = rng.choice(("f32", "bf16", "f16"))
    if op == "quantize":
        rows = _log_uniform(rng, 1, MOST)
        return {"op": op, "dtype": dtype, "rows": rows, "cols": _log_uniform(rng, 32, MOST), "forms": rng.choice(("rows", "columns", "both"))}
    n, k = (_log_uniform(rng, 128, MOST) for _ in range(2))
    if op == "step":
        return {"op": op, "dtype": "bf16", "m": _log_uniform(rng, 64, 4096), "n": n, "k": min(k, 4096)}
    if op == "gemm":
        return {"op": op, "dtype": dtype, "m": _log_uniform(rng, 1, MOST), "n": n, "k": k, "onto": rng.choice((0, 0, 1))}
    return {"op": op, "dtype": dtype, "m": _log_uniform(rng, 1, 4096), "n": n, "k": k, "grad": rng.choice((0, 0, 1))}


# ---------------------------------------------------------------- the plain form, in 32 bits
def _padded(cols):
    return -(-cols // 128) * 128


def _power(e):
    """2^e in 32 bits from its exponent field, e from -126 to 127 (-127: zero).  torch.ldexp goes by pow, which is a rounding off
    at some exponents, and that moves values that lie half way between two elements."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _plain_quantize(x):
    """(q, s) of the rows of x."""
    rows, cols = x.shape
    b = torch.nn.functional.pad(x.float(), (0, _padded(cols) - cols)).view(rows, -1, 32)
    most = b.abs().amax(-1, keepdim=True)
    shared = (torch.frexp(most).exponent - 3).clamp(-127, 127)
    shared = torch.where(most == 0, torch.full_like(shared, -127), shared)
    v = b.abs() * _power(-shared)
    code = torch.signbit(b).to(torch.uint8) * 8
    for at, ties_up in ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        code += (v >= at) if ties_up else (v > at)
    code = code.view(rows, -1)
    return code[:, 0::2] | (code[:, 1::2] << 4), (shared.view(rows, -1) + 127).to(torch.uint8)


def _plain_values(q, s, cols):
    """What (q, s) stands for, in 32 bits."""
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float32, device=q.device)
    table = torch.cat((table, -table))
    code = torch.stack((q & 15, q >> 4), -1).view(q.shape[0], -1, 32).int()
    v = table[code] * _power(s.int().unsqueeze(-1) - 127)
    return v.view(q.shape[0], -1)[:, :cols]


def _plain_run(st):
    op, dtype = st["op"], st["dtype"]
    if op == "quantize":
        x, cols, rows = st["x"], st["x"].shape[1], st["x"].shape[0]
        out = {}
        if st["forms"] != "columns":
            out["rows"] = _plain_values(*_plain_quantize(x), cols).to(dtype)
        if st["forms"] != "rows":
            out["columns"] = _plain_values(*_plain_quantize(x.t()), rows).to(dtype)
        return out
    if op == "gemm":
        c = _plain_values(*st["a"], st["k"]) @ _plain_values(*st["b"], st["k"]).t()
        return (c + st["c"].float() if st["onto"] else c).to(dtype)
    if op == "apply":
        w = _plain_values(*st["w"], st["k"])
        return (st["x"].float() @ (w if st["grad"] else w.t())).to(dtype)
    x, w, dy = st["x"], st["w"], st["dy"]
    (m, k), n = x.shape, w.shape[0]
    y = _plain_values(*_plain_quantize(x), k) @ _plain_values(*_plain_quantize(w), k).t()
    dx = _plain_values(*_plain_quantize(dy), n) @ _plain_values(*_plain_quantize(w.t()), n).t()
    dw = _plain_values(*_plain_quantize(dy.t()), m) @ _plain_values(*_plain_quantize(x.t()), m).t()
    return {"y": y.to(dtype), "dx": dx.to(dtype), "dw": dw}


# ---------------------------------------------------------------- the library's calls
def _own_run(st):
    from paper_2309_07235_amd import binding as B

    op, dtype = st["op"], st["dtype"]
    if op == "quantize":
        x = st["x"]
        rows, cols = x.shape
        q = B.mx4_empty(rows, cols) if st["forms"] != "columns" else None
        qt = B.mx4_empty(cols, rows) if st["forms"] != "rows" else None
        B.mx4_quantize(x, q, qt)
        out = {}
        if q is not None:
            out["rows"] = torch.empty_like(x)
            B.mx4_dequantize(q, out["rows"])
        if qt is not None:
            out["columns"] = torch.empty((cols, rows), dtype=dtype, device=x.device)
            B.mx4_dequantize(qt, out["columns"])
        return out
    if op == "gemm":
        a, b = (B.Mx4(*st[i], st["k"]) for i in ("a", "b"))
        c = st["c"].clone() if st["onto"] else torch.empty((a.rows, b.rows), dtype=dtype, device=st["a"][0].device)
        B.mx4_gemm(1 if st["onto"] else 0, a, b, c)
        return c
    if op == "apply":
        x, w = st["x"], B.Mx4(*st["w"], st["k"])
        y = torch.empty((x.shape[0], w.cols if st["grad"] else w.rows), dtype=dtype, device=x.device)
        B.mx4_apply(st["grad"], x, w, y)
        return y
    x, w, dy = st["x"], st["w"], st["dy"]
    (m, k), n = x.shape, w.shape[0]
    forms = {}
    for name, t in (("x", x), ("w", w), ("dy", dy)):
        forms[name] = B.mx4_empty(*t.shape), B.mx4_empty(t.shape[1], t.shape[0])
        B.mx4_quantize(t, *forms[name])
    y, dx = torch.empty_like(dy), torch.empty_like(x)
    dw = torch.empty(w.shape, dtype=torch.float32, device=w.device)
    B.mx4_gemm(0, forms["x"][0], forms["w"][0], y)
    B.mx4_gemm(0, forms["dy"][0], forms["w"][1], dx)
    B.mx4_gemm(0, forms["dy"][1], forms["x"][1], dw)
    return {"y": y, "dx": dx, "dw": dw}


# ---------------------------------------------------------------- inputs
def _normal(gen, rows, cols, scale):
    return torch.randn(rows, cols, dtype=torch.float32, device="cuda", generator=gen).mul_(scale)


def _activations(gen, rows, cols, scale=1.0):
    """Normal values with some channels much larger than the rest, as between a model's layers."""
    x = _normal(gen, rows, cols, scale)
    return x.mul_(torch.randn(cols, device="cuda", generator=gen).mul_(0.7).exp_())


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op, dtype = case["op"], DTYPES[case["dtype"]]
    st = {"op": op, "dtype": dtype, **{i: case[i] for i in ("k", "forms", "onto", "grad") if i in case}}
    if op == "quantize":
        st["x"] = _activations(gen, case["rows"], case["cols"]).to(dtype)
        return st
    m, n, k = case["m"], case["n"], case["k"]
    w = _normal(gen, n, k, 0.02)
    if op == "gemm":
        st["a"], st["b"] = _plain_quantize(_activations(gen, m, k)), _plain_quantize(w)
        st["c"] = _normal(gen, m, n, 1.0).to(dtype) if case["onto"] else None
    elif op == "apply":
        st["w"] = _plain_quantize(w)
        st["x"] = _activations(gen, m, n if case["grad"] else k).to(dtype)
    else:
        st["x"], st["w"] = _activations(gen, m, k).to(dtype), w.to(dtype)
        st["dy"] = _activations(gen, m, n, 1e-3).to(dtype)
    return st


def run(st):
    if own:
        return _own_run(st)
    return _plain_run(st)


# ---------------------------------------------------------------- the definition, in 64 bits
def _exact_round(x):
    """The values that the microscaled form of x's rows stands for: to the nearest step of the binade, ties to even."""
    rows, cols = x.shape
    b = torch.nn.functional.pad(x.double(), (0, -cols % 32)).reshape(rows, -1, 32)
    most = b.abs().amax(-1, keepdim=True)
    e = most.clamp_min(2.0 ** -200).log2().round()
    e = torch.where(torch.exp2(e) > most, e - 1, e)
    unit = torch.exp2((e - 2).clamp(-127, 127))
    v = b / unit
    step = torch.where(v.abs() < 2, 0.5, torch.where(v.abs() < 4, 1.0, 2.0).double())
    return (((v / step).round() * step).clamp(-6, 6) * unit).view(rows, -1)[:, :cols]


def _exact_values(q, s, cols):
    """What (q, s) stands for: sign, two bits of exponent, one of mantissa."""
    code = torch.stack((q.bitwise_and(15), q.bitwise_right_shift(4)), 2).flatten(1).long()
    e, half = (code >> 1) & 3, (code & 1).double() / 2
    v = torch.where(e == 0, half, torch.exp2((e - 1).double()) * (1 + half)) * (1 - 2 * (code >> 3)).double()
    return (v.view(q.shape[0], -1, 32) * torch.exp2(s.double() - 127).unsqueeze(2)).flatten(1)[:, :cols]


def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    if op == "quantize":
        x = st["x"].double()
        out = {}
        if case["forms"] != "columns":
            out["rows"] = _exact_round(x)
        if case["forms"] != "rows":
            out["columns"] = _exact_round(x.t())
        return out
    if op == "gemm":
        c = torch.mm(_exact_values(*st["a"], st["k"]), _exact_values(*st["b"], st["k"]).t())
        return c + st["c"].double() if case["onto"] else c
    if op == "apply":
        w = _exact_values(*st["w"], st["k"])
        return torch.mm(st["x"].double(), w if case["grad"] else w.t())
    x, w, dy = st["x"], st["w"], st["dy"]
    return {"y": torch.mm(_exact_round(x), _exact_round(w).t()), "dx": torch.mm(_exact_round(dy), _exact_round(w.t()).t()),
            "dw": torch.mm(_exact_round(dy.t()), _exact_round(x.t()).t())}


# ---------------------------------------------------------------- what a pass cannot do without
def _micro(rows, cols):
    return rows * (cols / 2 + -(-cols // 32))


def work(case):
    size = DTYPES[case["dtype"]].itemsize
    if case["op"] == "quantize":  # X read; each form written, read again and written as values
        r, c, forms = case["rows"], case["cols"], case["forms"]
        total = size * r * c
        if forms != "columns":
            total += 2 * _micro(r, c) + size * r * c
        if forms != "rows":
            total += 2 * _micro(c, r) + size * r * c
        return {"bytes": total, "flops": 0}
    m, n, k = case["m"], case["n"], case["k"]
    flops = 2.0 * m * n * k
    if case["op"] == "gemm":
        return {"bytes": _micro(m, k) + _micro(n, k) + size * m * n * (2 if case["onto"] else 1), "flops": flops}
    if case["op"] == "apply":
        return {"bytes": size * m * (n + k) + _micro(n, k), "flops": flops}
    return {"bytes": 2 * (m * k + n * k + m * n) + 2 * (m * n + m * k) + 4 * n * k, "flops": 3 * flops}
