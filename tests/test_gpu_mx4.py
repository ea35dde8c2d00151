"""The microscaled operators against a plain implementation in 64 bits."""
import numpy as np
import pytest

from tests import mx4_oracle as O
from tests.gpu_util import announce, to_host

pytestmark = pytest.mark.gpu

TYPES = ["float32", "bfloat16", "float16"]
# half a step of the type, relative; and half the smallest step (fp32 and bf16: below anything tested)
HALF = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
TINY = {"float32": 2.0 ** -150, "bfloat16": 2.0 ** -134, "float16": 2.0 ** -25}


@pytest.fixture(scope="module")
def B():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2309_07235_amd import binding
    return binding


def put(x, dtype, pad=0):
    """x (float64) as a device matrix of dtype, inside a larger one of NaN: `pad` elements before and behind every row."""
    import torch
    dt = getattr(torch, dtype)
    full = torch.full((x.shape[0] + 1, x.shape[1] + 2 * pad), float("nan"), dtype=dt, device="cuda")
    view = full[:x.shape[0], pad:pad + x.shape[1]]
    view.copy_(torch.from_numpy(np.ascontiguousarray(x)).to(dt))
    return full, view


def f64(t):
    return to_host(t.double())


def micro(B, codes, scales, cols, pad=0):
    """A microscaled matrix on the device, rows `pad` blocks of 16 (4) bytes longer than they have to be, that room filled with 0xff."""
    import torch
    q = torch.full((codes.shape[0], codes.shape[1] // 2 + 16 * pad), 255, dtype=torch.uint8, device="cuda")
    s = torch.full((codes.shape[0], scales.shape[1] + 4 * pad), 255, dtype=torch.uint8, device="cuda")
    q[:, :codes.shape[1] // 2] = torch.from_numpy(O.pack(codes)).cuda()
    s[:, :scales.shape[1]] = torch.from_numpy(scales).cuda()
    return B.Mx4(q, s, cols)


def check_form(form, x, pad):
    """form holds the microscaled form of x (float64), padding included, and nothing behind it was written."""
    codes, scales = O.quantize(x)
    q, s = to_host(form.q), to_host(form.s)
    assert np.array_equal(s[:, :scales.shape[1]], scales)
    assert np.array_equal(q[:, :codes.shape[1] // 2], O.pack(codes))
    if pad:
        assert (q[:, codes.shape[1] // 2:] == 0xA5).all() and (s[:, scales.shape[1]:] == 0xA5).all()


def room(B, rows, cols, pad):
    import torch
    wide = O.padded(cols)
    return B.Mx4(torch.full((rows, wide // 2 + 16 * pad), 0xA5, dtype=torch.uint8, device="cuda"),
                 torch.full((rows, wide // 32 + 4 * pad), 0xA5, dtype=torch.uint8, device="cuda"), cols)


SHAPES = [(1, 1), (1, 4096), (3, 31), (5, 33), (2, 127), (7, 128), (127, 129), (129, 1), (33, 250), (130, 255), (257, 640)]


@pytest.mark.parametrize("forms", ["rows", "columns", "both"])
@pytest.mark.parametrize("dtype", TYPES)
def test_quantize(B, dtype, forms):
    rng = np.random.default_rng(5)
    for pad in (0, 1, 8):
        for rows, cols in SHAPES:
            announce(f"quantize {dtype} {forms} pad {pad} {rows} x {cols}")
            x = rng.standard_normal((rows, cols)) * np.exp2(rng.integers(-6, 7, (rows, cols)))
            _, xd = put(x, dtype, pad)
            x = f64(xd)
            q = room(B, rows, cols, pad) if forms != "columns" else None
            qt = room(B, cols, rows, pad) if forms != "rows" else None
            B.mx4_quantize(xd, q, qt)
            if q is not None:
                check_form(q, x, pad)
            if qt is not None:
                check_form(qt, x.T, pad)


@pytest.mark.parametrize("dtype", TYPES)
def test_quantize_special_values(B, dtype):
    """Every border between two elements and its neighbours, at the type's lowest, highest and middle exponents; zeros of both signs;
    blocks that hold an infinity or a NaN, whole blocks of the type's lowest value, subnormal ones."""
    import torch
    announce(f"quantize special {dtype}")
    info = torch.finfo(getattr(torch, dtype))
    rows = []
    top = int(np.log2(info.max))
    for e in (-149, -130, -127, -126, -24, -14, -13, -3, 0, 3, top - 3, top - 2):
        for border in (0.25, 0.5, 0.75, 1.0, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6, 7, 7.9):
            for off in (0.0, info.eps, -info.eps, 2.0 ** -7, -2.0 ** -7):
                rows.append([4.0 * 2.0 ** e, -border * (1 + off) * 2.0 ** e, border * (1 + off) * 2.0 ** e] + [0.0] * 29)
    rows += [[0.0] * 32, [-0.0] * 32, [-0.0, 1.0] * 16, [float(info.min)] * 32, [float(info.max)] * 32, [float(info.tiny)] * 32,
             [float(info.tiny) * float(info.eps)] * 32, [np.nan] + [1.0] * 31, [1.0] * 31 + [np.inf], [-np.inf] * 32, [1e-3] * 20 + [np.nan] * 12]
    x = np.array(rows)
    _, xd = put(x, dtype)
    x = f64(xd)
    q, qt = room(B, *x.shape, 1), room(B, x.shape[0], 32, 1)
    B.mx4_quantize(xd, q)
    check_form(q, x, 1)
    xt = xd.t().contiguous()
    B.mx4_quantize(xt, None, qt)  # the same blocks along the columns
    check_form(qt, x, 1)


@pytest.mark.parametrize("dtype", TYPES)
def test_dequantize_every_value(B, dtype):
    import torch
    announce(f"dequantize {dtype}")
    codes = np.tile(np.arange(16, dtype=np.uint8), (1, 8 * 256)).reshape(16, -1)
    scales = np.arange(256, dtype=np.uint8).repeat(4).reshape(16, -1)[:, ::1]
    codes = np.tile(np.arange(16, dtype=np.uint8), (16, scales.shape[1] * 2))
    for cols, pad in ((codes.shape[1], 0), (codes.shape[1] - 1, 1), (codes.shape[1] - 37, 3)):
        w = micro(B, codes, scales, cols, pad)
        full, y = put(np.zeros((16, cols)), dtype, pad)
        B.mx4_dequantize(w, y)
        with np.errstate(over="ignore"):
            want = torch.from_numpy(O.values(codes, scales)[:, :cols]).to(getattr(torch, dtype))
        assert np.array_equal(f64(y), to_host(want.double()), equal_nan=True)
        assert int(torch.isnan(full).sum()) == full.numel() - 16 * cols + int(torch.isnan(want).sum())


def bound(y, size, terms, dtype):
    """How far a sum of `terms` products may be from its value y in 64 bits: (terms - 1) additions of fp32, each off by at most a step
    2^-23 of the sum of magnitudes `size`, and the rounding to the result's type."""
    return terms * 2.0 ** -23 * size + HALF[dtype] * np.abs(y) * 1.0001 + TINY[dtype]


def rounded(y, dtype):
    import torch
    return to_host(torch.from_numpy(y).float().to(getattr(torch, dtype)).double())


def gemm_params(B):
    return [None] + [B.Mx4Params(t.tile_m, t.tile_n, s) for t in B.mx4_enumerate_tiles(B.DLA_KERNEL_MX4_GEMM) for s in (1, 3)]


GEMM_SHAPES = [(1, 1, 1), (1, 128, 384), (16, 17, 513), (15, 33, 129), (33, 31, 640), (65, 66, 400), (130, 259, 1100), (300, 270, 515)]


@pytest.mark.parametrize("op", [0, 1])
@pytest.mark.parametrize("dtype", TYPES)
def test_gemm_bit_for_bit(B, dtype, op):
    """Scales 2^-1 and 1: every partial sum is a multiple of 2^-4 below 2^16, exact in fp32 whatever the order.  The result is
    the exact one, rounded once; nothing around it is written."""
    import torch
    rng = np.random.default_rng(7)
    for m, n, k in GEMM_SHAPES:
        ac, as_ = O.random_codes(rng, m, k)
        bc, bs = O.random_codes(rng, n, k)
        exact = O.values(ac, as_) @ O.values(bc, bs).T
        c0 = rng.integers(-8, 9, (m, n)).astype(float)
        for i, p in enumerate(gemm_params(B)):
            if p is not None and p.splits > -(-k // 128):
                continue
            pad = i % 3
            announce(f"mx4_gemm op {op} {dtype} {m} x {n} x {k} {p}")
            a, b = micro(B, ac, as_, k, pad), micro(B, bc, bs, k, 2 - pad)
            full, c = put(c0, dtype, pad)
            B.mx4_gemm(op, a, b, c, p)
            want = rounded(exact + c0 if op else exact, dtype)
            assert np.array_equal(f64(c), want), (m, n, k, p)
            assert int(torch.isnan(full).sum()) == full.numel() - m * n


@pytest.mark.parametrize("dtype", TYPES)
def test_gemm_against_64_bits(B, dtype):
    rng = np.random.default_rng(8)
    for m, n, k in GEMM_SHAPES[1:] + [(2, 48, 9000), (70, 40, 4100)]:
        ac, as_ = O.random_codes(rng, m, k, 118, 131)
        bc, bs = O.random_codes(rng, n, k, 110, 125)
        av, bv = O.values(ac, as_), O.values(bc, bs)
        want, size = av @ bv.T, np.abs(av) @ np.abs(bv).T
        for p in gemm_params(B):
            if p is not None and p.splits > -(-k // 128):
                continue
            announce(f"mx4_gemm values {dtype} {m} x {n} x {k} {p}")
            _, c = put(np.zeros((m, n)), dtype)
            B.mx4_gemm(0, micro(B, ac, as_, k), micro(B, bc, bs, k), c, p)
            off = np.abs(f64(c) - want) - bound(want, size, k, dtype)
            assert off.max() <= 0, (m, n, k, p, off.max())


def test_gemm_nan_stays_in_its_row_and_extreme_scales(B):
    rng = np.random.default_rng(9)
    m, n, k = 70, 40, 700
    ac, as_ = O.random_codes(rng, m, k)
    bc, bs = O.random_codes(rng, n, k)
    as_[3, 5] = 255
    as_[69, 0] = 255
    ac[69, :32] = 0  # a NaN even where its elements are zero
    bs[11, 20] = 255
    as_[5, :22], bs[7, :22] = 254, 0  # 2^127 and 2^-127: the products are ordinary numbers
    with np.errstate(invalid="ignore", over="ignore"):
        want = O.values(ac, as_) @ O.values(bc, bs).T
    for p in gemm_params(B):
        announce(f"mx4_gemm nan {p}")
        _, c = put(np.zeros((m, n)), "float32")
        B.mx4_gemm(0, micro(B, ac, as_, k), micro(B, bc, bs, k), c, p)
        got = f64(c)
        rest = [i for i in range(m) if i != 5]  # (row 5 leaves fp32's range in the other columns)
        assert np.array_equal(np.isnan(got[rest]), np.isnan(want[rest])), p
        rest = [i for i in range(m) if i not in (3, 5, 69)]
        cols = [j for j in range(n) if j not in (7, 11)]
        assert np.array_equal(got[np.ix_(rest, cols)], want[np.ix_(rest, cols)])
        assert got[5, 7] == want[5, 7] and np.isfinite(got[5, 7])


def test_gemm_nothing_to_sum_and_empty_results(B):
    import torch
    announce("mx4_gemm k 0, m 0, n 0")
    a, b = B.mx4_empty(5, 0), B.mx4_empty(6, 0)
    for dtype in TYPES:
        full, c = put(np.ones((5, 6)), dtype, 1)
        B.mx4_gemm(1, a, b, c)
        assert (f64(c) == 1).all()
        B.mx4_gemm(0, a, b, c)
        assert (f64(c) == 0).all() and int(torch.isnan(full).sum()) == full.numel() - 30
    B.mx4_gemm(0, B.mx4_empty(0, 64), B.mx4_empty(6, 64), torch.empty((0, 6), device="cuda"))
    B.mx4_gemm(0, B.mx4_empty(6, 64), B.mx4_empty(0, 64), torch.empty((6, 0), device="cuda"))
    q = B.mx4_empty(0, 7)
    B.mx4_quantize(torch.empty((0, 7), device="cuda"), q, B.mx4_empty(7, 0))
    B.mx4_dequantize(q, torch.empty((0, 7), device="cuda"))
    y = torch.ones((3, 9), device="cuda")
    B.mx4_apply(1, torch.empty((3, 0), device="cuda"), B.mx4_empty(0, 9), y)
    assert (f64(y) == 0).all()


def apply_params(B, op, dtype):
    code = {"float32": B.DLA_F32, "bfloat16": B.DLA_BF16, "float16": B.DLA_F16}[dtype]
    return [None] + [B.Mx4Params(t.tile_m, t.tile_n, s) for t in B.mx4_enumerate_tiles(B.DLA_KERNEL_MX4_APPLY, op, code) for s in (1, 3)]


def legal_apply(B, op, p, terms):
    return p is None or p.splits <= -(-terms // 128)


APPLY_SHAPES = [(1, 1, 1), (1, 130, 512), (3, 384, 129), (16, 33, 640), (17, 400, 100), (40, 257, 390), (65, 70, 520), (130, 515, 270), (260, 300, 515)]


@pytest.mark.parametrize("op", [0, 1])
@pytest.mark.parametrize("dtype", TYPES)
def test_apply_bit_for_bit(B, dtype, op):
    """Integers up to 8 in X and scales 2^-1 and 1: every partial sum is exact in fp32; the result is rounded once."""
    import torch
    rng = np.random.default_rng(11)
    for m, n, k in APPLY_SHAPES:
        wc, ws = O.random_codes(rng, n, k)
        w = O.values(wc, ws)[:, :k]
        x = rng.integers(-8, 9, (m, k if op == 0 else n)).astype(float)
        exact = x @ (w.T if op == 0 else w)
        for i, p in enumerate(apply_params(B, op, dtype)):
            if not legal_apply(B, op, p, x.shape[1]):
                continue
            pad = (0, 1, 8)[i % 3]
            for dtype_y in (dtype, "float32") if i else TYPES:
                announce(f"mx4_apply op {op} {dtype} to {dtype_y} {m} x {n} x {k} pad {pad} {p}")
                _, xd = put(x, dtype, pad)
                full, y = put(np.zeros(exact.shape), dtype_y, pad)
                B.mx4_apply(op, xd, micro(B, wc, ws, k, i % 3), y, p)
                assert np.array_equal(f64(y), rounded(exact, dtype_y)), (m, n, k, p)
                assert int(torch.isnan(full).sum()) == full.numel() - exact.size


@pytest.mark.parametrize("op", [0, 1])
@pytest.mark.parametrize("dtype", TYPES)
def test_apply_against_64_bits(B, dtype, op):
    """X keeps all bits of its type: a result in fp32 is off by the additions' roundings alone (three products a term in fp32)."""
    rng = np.random.default_rng(12)
    terms = {"float32": 3, "bfloat16": 1, "float16": 2}[dtype]
    for m, n, k in APPLY_SHAPES[1:] + [(2, 1030, 4100), (70, 4100, 140)]:
        wc, ws = O.random_codes(rng, n, k, 115, 126)
        w = O.values(wc, ws)[:, :k]
        _, xd = put(rng.standard_normal((m, k if op == 0 else n)), dtype, 3)
        x = f64(xd)
        w = w.T if op == 0 else w
        want, size = x @ w, np.abs(x) @ np.abs(w)
        for p in apply_params(B, op, dtype):
            if not legal_apply(B, op, p, x.shape[1]):
                continue
            announce(f"mx4_apply values op {op} {dtype} {m} x {n} x {k} {p}")
            _, y = put(np.zeros(want.shape), "float32")
            B.mx4_apply(op, xd, micro(B, wc, ws, k), y, p)
            off = np.abs(f64(y) - want) - bound(want, size, terms * x.shape[1], "float32")
            assert off.max() <= 0, (m, n, k, p, off.max())


@pytest.mark.parametrize("op", [0, 1])
@pytest.mark.parametrize("dtype", TYPES)
def test_apply_infinities_nan_and_the_largest_values(B, dtype, op):
    """What is not finite in X reaches its row only, as in a product of real numbers; the type's largest and smallest values
    are kept whole; W's NaN blocks reach what they multiply."""
    import torch
    info = torch.finfo(getattr(torch, dtype))
    m, n, k = 67, 200, 330
    rng = np.random.default_rng(13)
    wc = rng.integers(1, 8, (n, O.padded(k))).astype(np.uint8)  # positive, no zeros
    wc[:, k:] = 0
    ws = np.full((n, wc.shape[1] // 32), 120, np.uint8)
    ws[:, -(-k // 32):] = 0
    ws[4, 2] = 255
    x = np.ones((m, k if op == 0 else n))
    x[1, 7], x[2, 7], x[3, 9] = np.inf, -np.inf, np.nan
    x[66, 0], x[66, -1] = np.inf, -np.inf
    x[5] = 0.0
    x[5, 100] = info.max
    x[6] = 0.0
    x[6, 100] = info.tiny
    x[8, -1] = np.nan
    _, xd = put(x, dtype, 1)
    x = f64(xd)
    w = O.values(wc, ws)[:, :k]
    with np.errstate(invalid="ignore"):
        want = x @ (w.T if op == 0 else w)
    for p in apply_params(B, op, dtype):
        if not legal_apply(B, op, p, x.shape[1]):
            continue
        announce(f"mx4_apply special op {op} {dtype} {p}")
        _, y = put(np.zeros(want.shape), "float32")
        B.mx4_apply(op, xd, micro(B, wc, ws, k), y, p)
        got = f64(y)
        over = np.abs(want) >= 2.0 ** 128
        got, ref = np.where(over, 0, got), np.where(over, 0, want)
        assert np.array_equal(np.isnan(got), np.isnan(ref)), p
        assert np.array_equal(np.isinf(got), np.isinf(ref)), p
        fine = np.isfinite(ref)
        assert (np.abs(got[fine] - ref[fine]) <= 2.0 ** -23 * 3 * x.shape[1] * np.abs(ref[fine])).all(), p


def test_apply_gradient_against_the_formula_and_differences(B):
    """loss = sum(g * (x W^T)): its gradient is g W (op 1), and the loss is linear in x, so a difference over any step is the gradient
    but for the roundings of the two losses (fp32 results, 64-bit sums)."""
    import torch
    announce("mx4_apply gradient")
    rng = np.random.default_rng(14)
    m, n, k = 9, 130, 200
    wc, ws = O.random_codes(rng, n, k, 121, 126)
    w = micro(B, wc, ws, k)
    wv = O.values(wc, ws)[:, :k]
    x = torch.from_numpy(rng.standard_normal((m, k))).float().cuda()
    g = torch.from_numpy(rng.standard_normal((m, n))).float().cuda()
    dx = torch.empty_like(x)
    B.mx4_apply(1, g, w, dx)
    gv = f64(g)
    size = np.abs(gv) @ np.abs(wv)
    assert (np.abs(f64(dx) - gv @ wv) <= bound(gv @ wv, size, 3 * n, "float32")).all()
    step = 4.0
    for i, j in ((0, 0), (8, 199), (3, 77), (5, 128)):
        loss, room_ = [], 0.0
        for sign in (1, -1):
            xs = x.clone()
            xs[i, j] = sign * step
            y = torch.empty((m, n), device="cuda")
            B.mx4_apply(0, xs, w, y)
            loss.append(float((gv * f64(y)).sum()))
            room_ += float((np.abs(gv) * bound(f64(y), np.abs(f64(xs)) @ np.abs(wv).T, 3 * k, "float32")).sum())
        assert abs((loss[0] - loss[1]) / (2 * step) - f64(dx)[i, j]) <= room_ / (2 * step) + bound(0, size[i, j], 3 * n, "float32")


def step_of_a_layer(B, x, w, dy, stream=None, into=None):
    """A training step of a linear layer in microscaled operands: y, dx, dw."""
    import torch
    (m, k), n = x.shape, w.shape[0]
    into = into if into is not None else {}
    if not into:
        for name, t in (("x", x), ("w", w), ("dy", dy)):
            into[name] = B.mx4_empty(*t.shape), B.mx4_empty(t.shape[1], t.shape[0])
        into["y"], into["dx"] = torch.empty((m, n), dtype=x.dtype, device="cuda"), torch.empty((m, k), dtype=x.dtype, device="cuda")
        into["dw"] = torch.empty((n, k), device="cuda")
    for name, t in (("x", x), ("w", w), ("dy", dy)):
        B.mx4_quantize(t, *into[name], stream=stream)
    B.mx4_gemm(0, into["x"][0], into["w"][0], into["y"], stream=stream)
    B.mx4_gemm(0, into["dy"][0], into["w"][1], into["dx"], stream=stream)
    B.mx4_gemm(0, into["dy"][1], into["x"][1], into["dw"], stream=stream)
    return into


@pytest.mark.parametrize("m,n,k", [(1, 96, 160), (77, 130, 259), (300, 515, 390)])
def test_the_operators_together_train_a_layer(B, m, n, k):
    import torch
    announce(f"mx4 layer {m} {n} {k}")
    rng = np.random.default_rng(15)
    x, w, dy = (put(rng.standard_normal(s), "bfloat16")[1].contiguous() for s in ((m, k), (n, k), (m, n)))
    got = step_of_a_layer(B, x, w, dy)

    def q(t):
        return O.values(*O.quantize(t))

    xv, wv, gv = f64(x), f64(w), f64(dy)
    for name, a, b, dtype in (("y", q(xv), q(wv), "bfloat16"), ("dx", q(gv), q(wv.T), "bfloat16"), ("dw", q(gv.T), q(xv.T), "float32")):
        want, size = a @ b.T, np.abs(a) @ np.abs(b).T
        assert (np.abs(f64(got[name]) - want) <= bound(want, size, a.shape[1], dtype)).all(), name
    # and what is quantised and read back is what the products multiplied
    back = torch.empty((m, k), device="cuda")
    B.mx4_dequantize(got["x"][0], back)
    assert np.array_equal(f64(back), q(xv)[:, :k])


def test_captured_and_replayed_between_eager_calls(B):
    """The step in a graph, replayed with other inputs in the same buffers and with eager work between: each time the eager result."""
    import torch
    announce("mx4 graph")
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)

    def fresh(s):
        return torch.randn(s, device="cuda", generator=gen).to(torch.bfloat16)

    shapes = ((40, 2100), (24, 2100), (40, 24))
    x, w, dy = (fresh(s) for s in shapes)
    into = step_of_a_layer(B, x, w, dy)
    yx = torch.empty((40, 24), dtype=torch.bfloat16, device="cuda")
    B.mx4_apply(0, x, into["w"][0], yx)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step_of_a_layer(B, x, w, dy, into=into)
        B.mx4_apply(0, x, into["w"][0], yx)
    for _ in range(3):
        for t in (x, w, dy):
            t.copy_(fresh(t.shape))
        graph.replay()
        torch.cuda.synchronize()
        got = {i: into[i].clone() for i in ("y", "dx", "dw")}
        eager = step_of_a_layer(B, x, w, dy)
        ye = torch.empty_like(yx)
        B.mx4_apply(0, x, eager["w"][0], ye)
        for i in got:
            assert torch.equal(got[i], eager[i]), i
        assert torch.equal(yx, ye)


def test_several_streams_at_once(B):
    """Calls on two streams that overlap, each with the workspace the binding takes for it: the results of calls one by one."""
    import torch
    announce("mx4 streams")
    gen = torch.Generator(device="cuda")
    gen.manual_seed(4)
    data = [[torch.randn(s, device="cuda", generator=gen).to(torch.bfloat16) for s in ((33, 4200), (50, 4200), (33, 50))] for _ in range(2)]
    want = [step_of_a_layer(B, *d) for d in data]
    streams = [torch.cuda.Stream() for _ in data]
    torch.cuda.synchronize()
    got = [None, None]
    for _ in range(5):
        for i, s in enumerate(streams):
            got[i] = step_of_a_layer(B, *data[i], stream=s, into=got[i])
    torch.cuda.synchronize()
    for w, g in zip(want, got):
        for i in ("y", "dx", "dw"):
            assert torch.equal(w[i], g[i]), i


def test_offsets_past_32_bits(B):
    """Rows 4 MB apart (the most that is taken), 1050 of them: operands, results and partial sums lie beyond 2^32 bytes."""
    import torch
    announce("mx4 long rows")
    m, n, k = 1050, 40, 300
    rng = np.random.default_rng(16)
    ac, as_ = O.random_codes(rng, m, k)
    bc, bs = O.random_codes(rng, n, k)
    exact = O.values(ac, as_) @ O.values(bc, bs).T
    big = torch.zeros(m << 22, dtype=torch.uint8, device="cuda").view(m, 1 << 22)
    a = B.Mx4(big[:, :192], big[:, 1024:1036], k)
    a.q.copy_(torch.from_numpy(O.pack(ac)).cuda())
    a.s.copy_(torch.from_numpy(as_).cuda())
    b = micro(B, bc, bs, k)
    for p in gemm_params(B):
        c = torch.zeros((m, n), device="cuda")
        B.mx4_gemm(0, a, b, c, p)
        assert np.array_equal(f64(c), exact), p
        ct = torch.zeros((n, m), device="cuda")
        B.mx4_gemm(0, b, a, ct, p)
        assert np.array_equal(f64(ct), exact.T), p
    for p in apply_params(B, 0, "bfloat16"):
        x = rng.integers(-4, 5, (20, k)).astype(float)
        y = torch.zeros((20, m), device="cuda")
        B.mx4_apply(0, put(x, "bfloat16")[1], a, y, p)
        assert np.array_equal(f64(y), x @ O.values(ac, as_)[:, :k].T), p
    for p in apply_params(B, 1, "bfloat16"):
        x = rng.integers(-4, 5, (20, m)).astype(float)
        y = torch.zeros((20, k), device="cuda")
        B.mx4_apply(1, put(x, "bfloat16")[1], a, y, p)
        assert np.array_equal(f64(y), x @ O.values(ac, as_)[:, :k]), p
    del a, big
    wide = torch.zeros((3, 1 << 30), dtype=torch.float32, device="cuda")  # rows 4 GB apart
    x = wide[:, 5:305]
    x.copy_(torch.from_numpy(rng.standard_normal((3, 300))).float())
    q, qt = room(B, 3, 300, 1), room(B, 300, 3, 1)
    B.mx4_quantize(x, q, qt)
    check_form(q, f64(x), 1)
    check_form(qt, f64(x).T, 1)
    y = wide[:, 1000:1300]
    B.mx4_dequantize(q, y)
    codes, scales = O.quantize(f64(x))
    assert np.array_equal(f64(y), O.values(codes, scales)[:, :300])
    w = micro(B, codes, scales, 300)
    z = wide[:, 2000:2003]
    B.mx4_apply(0, x, w, z)
    xv, wv = f64(x), O.values(codes, scales)[:, :300]
    assert (np.abs(f64(z) - xv @ wv.T) <= bound(xv @ wv.T, np.abs(xv) @ np.abs(wv).T, 900, "float32")).all()


@pytest.mark.parametrize("kernel,op,shape,dtype", [("mx4_gemm", 1, (70, 200, 900), "f32"), ("mx4_apply", 0, (9, 300, 700), "f16"),
                                                   ("mx4_apply", 1, (40, 700, 130), "bf16")])
def test_search_over_the_schedules(B, capsys, tmp_path, kernel, op, shape, dtype):
    import json

    from paper_2309_07235_amd import tune
    announce(f"search {kernel} op {op} {shape} {dtype}")
    db = tmp_path / "perf.csv"
    assert tune.main(["--kernel", kernel, "--op", str(op), "--shape", *map(str, shape), "--dtype", dtype, "--evals", "8", "--strategy", "random",
                      "--from-default", "--db", str(db)]) == 0
    out = json.loads(capsys.readouterr().out.strip().splitlines()[-1])
    rows = db.read_text().strip().splitlines()
    assert len(rows) == 9 and out["kernel"] == kernel and out["evaluations"] == 8
    assert 0.0 < out["best_runtime_ms"] <= float(rows[1].split(",")[-2]) + 1e-3
    assert len(out["best"]["tile"]) == 2 and out["best"]["splits"] >= 1


@pytest.mark.parametrize("dtype", TYPES)
def test_gemm_onto_aligned_rows_that_end_anywhere(B, dtype):
    """C in rows of whole 16 bytes, its last columns and rows inside a lane's run, a wave's part, a tile.  All sums are exact."""
    import torch
    rng = np.random.default_rng(17)
    k = 200
    for m, n in ((1, 1), (2, 3), (33, 5), (64, 8), (70, 9), (130, 131), (257, 63), (100, 260), (300, 193)):
        ac, as_ = O.random_codes(rng, m, k)
        bc, bs = O.random_codes(rng, n, k)
        c0 = rng.integers(-8, 9, (m, n)).astype(float)
        want = rounded(O.values(ac, as_) @ O.values(bc, bs).T + c0, dtype)
        a, b = micro(B, ac, as_, k), micro(B, bc, bs, k)
        for tile in ((128, 128), (256, 256), (16, 32)):
            announce(f"mx4_gemm onto {dtype} {m} x {n} tile {tile}")
            full = torch.full((m + 2, (n + 7) // 8 * 8 + 16), float("nan"), dtype=getattr(torch, dtype), device="cuda")
            c = full[1:m + 1, 8:8 + n]
            assert c.data_ptr() % 16 == 0 and c.stride(0) % 8 == 0
            c.copy_(torch.from_numpy(c0).to(c.dtype))
            B.mx4_gemm(1, a, b, c, B.Mx4Params(*tile, 1))
            assert np.array_equal(f64(c), want)
            assert int(torch.isnan(full).sum()) == full.numel() - m * n


@pytest.mark.parametrize("dtype", TYPES)
def test_few_rows_by_many_columns(B, dtype):
    """At and above the four rows that have a kernel of their own, with more and fewer workgroups than compute units."""
    rng = np.random.default_rng(18)
    for m, n, k in ((2, 8200, 260), (4, 8200, 128), (5, 8200, 130), (4, 100, 1000), (5, 60, 900), (17, 4200, 384)):
        wc, ws = O.random_codes(rng, n, k)
        xc, xs = O.random_codes(rng, m, k)
        w, xv = micro(B, wc, ws, k), O.values(xc, xs)[:, :k]
        wv = O.values(wc, ws)[:, :k]
        x = rng.integers(-8, 9, (m, k)).astype(float)
        for tile in ((16, 32), (0, 0)):
            announce(f"few rows {dtype} {m} x {n} x {k} tile {tile}")
            p = B.Mx4Params(*tile, 1 if tile[0] else 0)
            _, y = put(np.zeros((m, n)), dtype)
            B.mx4_apply(0, put(x, dtype)[1], w, y, p)
            assert np.array_equal(f64(y), rounded(x @ wv.T, dtype))
            B.mx4_gemm(0, micro(B, xc, xs, k), w, y, p)
            assert np.array_equal(f64(y), rounded(xv @ wv.T, dtype))


def test_profile_counts_the_products(B):
    import torch
    announce("mx4 profile")
    w, y = B.mx4_empty(50, 300), torch.empty((9, 50), device="cuda")
    x = torch.ones((50, 300), device="cuda")
    B.mx4_quantize(x, w)
    a = B.mx4_empty(9, 300)
    B.mx4_quantize(x[:9], a)
    B.profile_enable(True)
    try:
        B.mx4_gemm(0, a, w, y)
        B.mx4_apply(0, x[:9], w, y)
    finally:
        B.profile_enable(False)
    ms, calls, flops = B.profile_read(B.PHASE_GEMM)
    assert calls == 2 and ms > 0 and flops == 2 * 2 * 9 * 50 * 300
    assert (f64(y) == 300).all()


def test_quantize_rows_of_many_tiles(B):
    """64 tiles of columns and more a row, of which groups go to one cache; the last group is not whole."""
    rng = np.random.default_rng(19)
    for rows, cols in ((1, 8192), (130, 8065), (129, 8200), (300, 10000)):
        announce(f"quantize wide {rows} x {cols}")
        x = rng.standard_normal((rows, cols)) * np.exp2(rng.integers(-6, 7, (rows, cols)))
        _, xd = put(x, "bfloat16")
        q, qt = room(B, rows, cols, 1), room(B, cols, rows, 1)
        B.mx4_quantize(xd, q, qt)
        check_form(q, f64(xd), 1)
        check_form(qt, f64(xd).T, 1)


@pytest.mark.parametrize("op", [0, 1])
@pytest.mark.parametrize("dtype", TYPES)
def test_apply_subnormal_x(B, dtype, op):
    """The type's smallest values count: multiples of its smallest step (fp32: of 2^-133, the least that the terms hold), products
    and sums of which fp32 holds exactly with weights of 2^2 and more."""
    import torch
    rng = np.random.default_rng(20)
    step = {"float32": 2.0 ** -133, "bfloat16": 2.0 ** -133, "float16": 2.0 ** -24}[dtype]
    m, n, k = 33, 70, 200
    wc, ws = O.random_codes(rng, n, k, 131, 133)
    wv = O.values(wc, ws)[:, :k]
    x = rng.integers(-100, 101, (m, n if op else k)) * step
    _, xd = put(x, dtype)
    assert np.array_equal(f64(xd), x)
    want = x @ (wv if op else wv.T)
    w = micro(B, wc, ws, k)
    for rows in (m, 3):
        for p in apply_params(B, op, dtype):
            if not legal_apply(B, op, p, x.shape[1]):
                continue
            announce(f"mx4_apply subnormal {dtype} op {op} {rows} rows {p}")
            y = torch.empty((rows, want.shape[1]), device="cuda")
            B.mx4_apply(op, xd[:rows], w, y, p)
            assert np.array_equal(f64(y), want[:rows]), p


@pytest.mark.parametrize("op", [0, 1])
@pytest.mark.parametrize("dtype", TYPES)
def test_apply_smallest_weights(B, dtype, op):
    """Weights at and next to the least scale, 2^-127, some of them subnormal in bf16; all sums are exact in fp32."""
    import torch
    rng = np.random.default_rng(21)
    m, n, k = 20, 70, 200
    wc, ws = O.random_codes(rng, n, k, 0, 3)
    wv = O.values(wc, ws)[:, :k]
    x = rng.integers(-8, 9, (m, n if op else k)).astype(float)
    want = x @ (wv if op else wv.T)
    w = micro(B, wc, ws, k)
    for rows in (m, 3):
        for p in apply_params(B, op, dtype):
            if not legal_apply(B, op, p, x.shape[1]):
                continue
            announce(f"mx4_apply smallest weights {dtype} op {op} {rows} rows {p}")
            y = torch.empty((rows, want.shape[1]), device="cuda")
            B.mx4_apply(op, put(x[:rows], dtype)[1], w, y, p)
            assert np.array_equal(f64(y), want[:rows]), p


@pytest.mark.parametrize("op", [0, 1])
@pytest.mark.parametrize("dtype", TYPES)
def test_apply_keeps_every_bit_of_x(B, dtype, op):
    """A row of X holds one value, an odd integer of all the type's bits, at a term of its own; weights are powers of two.  Each result is
    one product, exact in fp32: a term of X that is lost, or read from another place, changes its last bits."""
    import torch
    rng = np.random.default_rng(22)
    bits = {"float32": 24, "bfloat16": 8, "float16": 11}[dtype]
    most, out, terms = 130, 70, 390
    n, k = (terms, out) if op else (out, terms)
    wc, ws = O.random_codes(rng, n, k, 118, 131)
    wc[:, :k] = rng.choice(np.array([1, 2, 4, 6, 9, 10, 12, 14], np.uint8), (n, k))
    assert (np.log2(np.abs(O.VALUES[[1, 2, 4, 6]])) == [-1, 0, 1, 2]).all()
    wv = O.values(wc, ws)[:, :k]
    at = (np.arange(most) * 3 + rng.integers(0, 3, most)) % terms
    at[[0, 1, 2]] = terms - 1, 0, terms - 2
    x = np.zeros((most, terms))
    x[np.arange(most), at] = (2 ** (bits - 1) + 2 * rng.integers(0, 2 ** (bits - 2), most) + 1) * np.where(rng.integers(0, 2, most), 1.0, -1.0) * 2.0 ** -bits
    want = x @ (wv if op else wv.T)
    w = micro(B, wc, ws, k)
    for rows, pad in ((3, 0), (16, 1), (33, 8), (most, 0)):
        _, xd = put(x[:rows], dtype, pad)
        assert np.array_equal(f64(xd), x[:rows])
        for p in apply_params(B, op, dtype):
            if not legal_apply(B, op, p, terms):
                continue
            announce(f"mx4_apply every bit {dtype} op {op} {rows} rows {p}")
            y = torch.empty((rows, out), device="cuda")
            B.mx4_apply(op, xd, w, y, p)
            assert np.array_equal(f64(y), want[:rows]), p


@pytest.mark.parametrize("op", [0, 1])
@pytest.mark.parametrize("dtype", TYPES)
def test_apply_largest_weights(B, dtype, op):
    """Weights up to 6 * 2^127, past fp32's own range, in blocks of some rows beside ordinary and NaN ones: where X brings the results back
    into the range they are what they are, exactly (sums of multiples of 2^104 below 2^119, of 2^-23 below 2^-9 beside them), whichever
    tile computes them, and zeros of X stay zeros."""
    import torch
    rng = np.random.default_rng(23)
    m, n, k = 300, 290, 300
    wc, ws = O.random_codes(rng, n, k, 125, 127)
    big = rng.choice(n, 40, replace=False)
    ws[big, :-(-k // 32)] = rng.integers(252, 255, (40, -(-k // 32)))
    ws[big[3], 4] = 255
    wv = O.values(wc, ws)[:, :k]
    x = rng.integers(-8, 9, (m, n if op else k)) * 2.0 ** -20
    x[7] = 0.0
    if op:  # a row of Y is made of rows of W that are all large or all ordinary
        x[::2, big] = 0.0
        x[1::2, np.setdiff1d(np.arange(n), big)] = 0.0
    want = x @ (wv if op else wv.T)
    w = micro(B, wc, ws, k)
    for rows in (m, 40, 3):
        _, xd = put(x[:rows], dtype, rows % 2)
        assert np.array_equal(f64(xd), x[:rows])
        for i, p in enumerate(apply_params(B, op, dtype)):
            if not legal_apply(B, op, p, x.shape[1]):
                continue
            for dtype_y in ("float32", TYPES[1 + i % 2]):
                announce(f"mx4_apply largest weights {dtype} to {dtype_y} op {op} {rows} rows {p}")
                full, y = put(np.zeros((rows, want.shape[1])), dtype_y, i % 3)
                B.mx4_apply(op, xd, w, y, p)
                assert np.array_equal(f64(y), rounded(want[:rows], dtype_y), equal_nan=True), p
                assert int(torch.isnan(full).sum()) == full.numel() - y.numel() + int(np.isnan(want[:rows]).sum())


@pytest.mark.parametrize("op", [0, 1])
@pytest.mark.parametrize("dtype", TYPES)
def test_apply_rows_at_every_alignment(B, dtype, op):
    """X at each place inside 32 bytes, its rows apart by each remainder of 32 bytes: what a row's first access may be aligned to.
    Integers up to 8 and scales 2^-1 and 1, so every sum is exact."""
    import torch
    rng = np.random.default_rng(24)
    m, n, k = 5, 96, 104
    wc, ws = O.random_codes(rng, n, k)
    wv = O.values(wc, ws)[:, :k]
    w = micro(B, wc, ws, k)
    terms, out = (n, k) if op else (k, n)
    dt = getattr(torch, dtype)
    per = 32 // dt.itemsize
    x = rng.integers(-8, 9, (m, terms)).astype(float)
    want = rounded(x @ (wv if op else wv.T), dtype)
    for first in range(per):
        for more in range(per):
            ldx = terms + per + more
            full = torch.full((m * ldx + first,), float("nan"), dtype=dt, device="cuda")
            xd = full[first:].view(m, ldx)[:, :terms]
            xd.copy_(torch.from_numpy(x).to(dt))
            assert xd.data_ptr() % 32 == first * dt.itemsize and xd.stride(0) == ldx
            y = torch.empty((m, out), dtype=dt, device="cuda")
            announce(f"mx4_apply alignment {dtype} op {op} first {first} ldx {ldx}")
            B.mx4_apply(op, xd, w, y)
            assert np.array_equal(f64(y), want), (first, ldx)


def test_quantize_widths_about_64_tiles(B):
    """Rows of 61 to 67 and of 126 to 131 tiles: the numbers about a multiple of 64 at which the order of the tiles changes."""
    rng = np.random.default_rng(25)
    for tiles in (61, 62, 63, 64, 65, 66, 67, 126, 128, 130, 131):
        rows, cols = (150, tiles * 128 - 5) if tiles < 100 else (129, tiles * 128)
        announce(f"quantize {rows} x {cols}, {tiles} tiles a row")
        x = rng.standard_normal((rows, cols)) * np.exp2(rng.integers(-6, 7, (rows, cols)))
        _, xd = put(x, "float32")
        q, qt = room(B, rows, cols, 1), room(B, cols, rows, 1)
        B.mx4_quantize(xd, q, qt)
        check_form(q, f64(xd), 1)
        check_form(qt, f64(xd).T, 1)
