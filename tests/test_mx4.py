"""Host-side checks of the microscaled operators: refusals before any GPU work, menus, schedules, and the oracle itself."""
import ctypes

import numpy as np
import pytest

from tests import mx4_oracle as O


@pytest.fixture(scope="module")
def B():
    from paper_2309_07235_amd import binding
    return binding


FAKE = ctypes.c_void_p(0x1000)  # never dereferenced: every call below fails or ends before any GPU work
ODD = ctypes.c_void_p(0x1001)


def test_oracle_by_hand():
    x = np.zeros((1, 40))
    x[0, :9] = [6, 5, -2.5, 3.5, 0.25, 0.75, -0.1, 7.9, 1.75]
    x[0, 32:34] = [0.0625, -0.046875]
    codes, scales = O.quantize(x)
    assert list(scales[0]) == [127, 121, 0, 0]
    assert list(codes[0, :9]) == [7, 6, 8 + 4, 6, 0, 2, 8, 7, 4]
    assert list(codes[0, 32:34]) == [6, 8 + 5]
    assert O.pack(codes)[0, 0] == 0x67
    v = O.values(codes, scales)
    assert list(v[0, :5]) == [6, 4, -2, 4, 0] and v[0, 32] == 0.0625 and v[0, 33] == -0.046875


def test_quantize_refusals(B):
    f = B.lib.mx4_quantize

    def call(x=FAKE, ldx=200, rows=8, cols=200, dt=B.DLA_BF16, q=FAKE, ldq=128, s=FAKE, lds=8, qt=FAKE, ldqt=64, st=FAKE, ldst=4):
        return f(x, ldx, rows, cols, dt, q, ldq, s, lds, qt, ldqt, st, ldst, None)

    assert call(x=None) == -1 and call(x=ODD) == -1
    assert call(ldx=199) == -2
    assert call(rows=-1) == -3
    assert call(cols=-1) == -4
    for dt in (B.DLA_F64, 4, -1):
        assert call(dt=dt) == -5
    assert call(q=None) == -6 and call(q=ctypes.c_void_p(0x1008)) == -6
    assert call(ldq=112) == -7 and call(ldq=136) == -7
    assert call(s=None) == -8 and call(s=ctypes.c_void_p(0x1002)) == -8
    assert call(lds=4) == -9 and call(lds=10) == -9
    assert call(qt=None) == -10 and call(ldqt=48) == -11 and call(st=None) == -12 and call(ldst=0) == -13 and call(ldst=6) == -13
    assert call(q=None, s=None, qt=None, st=None) == -6
    assert call(ldq=(1 << 22) + 16) == B.DLA_ERR_TOO_LARGE
    assert call(rows=1 << 31) == B.DLA_ERR_TOO_LARGE
    assert call(rows=0, x=None, q=None, s=None, qt=None, st=None) == 0
    assert call(cols=0, x=None) == 0


def test_dequantize_refusals(B):
    f = B.lib.mx4_dequantize

    def call(q=FAKE, ldq=128, s=FAKE, lds=8, rows=8, cols=200, dt=B.DLA_F32, y=FAKE, ldy=200):
        return f(q, ldq, s, lds, rows, cols, dt, y, ldy, None)

    assert call(q=None) == -1 and call(ldq=64) == -2 and call(s=None) == -3 and call(lds=4) == -4
    assert call(rows=-1) == -5 and call(cols=-1) == -6 and call(dt=B.DLA_F64) == -7
    assert call(y=None) == -8 and call(y=ctypes.c_void_p(0x1002)) == -8 and call(ldy=100) == -9
    assert call(rows=0, q=None, s=None, y=None) == 0


def test_gemm_refusals(B):
    f = B.lib.mx4_gemm

    def call(op=0, a=FAKE, lda=128, sa=FAKE, ldsa=8, b=FAKE, ldb=128, sb=FAKE, ldsb=8, c=FAKE, ldc=9, m=8, n=9, k=200, dt=B.DLA_F32, p=None,
             ws=FAKE, wsb=1 << 20):
        return f(op, a, lda, sa, ldsa, b, ldb, sb, ldsb, c, ldc, m, n, k, dt, ctypes.byref(p) if p else None, ws, wsb, None)

    assert call(op=2) == -1 and call(a=None) == -2 and call(lda=64) == -3 and call(sa=None) == -4 and call(ldsa=4) == -5
    assert call(b=None) == -6 and call(ldb=64) == -7 and call(sb=None) == -8 and call(ldsb=4) == -9
    assert call(c=None) == -10 and call(ldc=8) == -11 and call(m=-1) == -12 and call(n=-1) == -13 and call(k=-1) == -14
    assert call(dt=B.DLA_F64) == -15
    assert call(m=1 << 31) == B.DLA_ERR_TOO_LARGE
    for bad in ((17, 16, 0), (16, 0, 0), (-16, 16, 0), (0, 0, -1), (0, 0, 33), (0, 0, 3)):  # 200 terms are two steps: no three splits
        assert call(p=B.Mx4Params(*bad)) == B.DLA_ERR_UNSUPPORTED_PARAMS, bad
    two = B.Mx4Params(0, 0, 2)
    need = B.lib.mx4_gemm_workspace_bytes(8, 9, 200, ctypes.byref(two))
    assert need >= 2 * 8 * 9 * 4
    assert call(p=two, ws=None, wsb=need) == B.DLA_ERR_WORKSPACE
    assert call(p=two, wsb=need - 1) == B.DLA_ERR_WORKSPACE
    assert call(p=two, ws=ctypes.c_void_p(0x1010), wsb=need) == B.DLA_ERR_WORKSPACE
    assert call(m=0, a=None, sa=None, c=None) == 0 and call(n=0, b=None, sb=None, c=None, ldc=1) == 0
    assert call(op=1, k=0, a=None, sa=None, b=None, sb=None) == 0  # nothing to add


def test_apply_refusals(B):
    f = B.lib.mx4_apply

    def call(op=0, x=FAKE, ldx=200, dt=B.DLA_BF16, w=FAKE, ldw=128, sw=FAKE, ldsw=8, y=FAKE, ldy=200, dt_y=B.DLA_F32, m=8, n=9, k=200, p=None,
             ws=FAKE, wsb=1 << 40):
        return f(op, x, ldx, dt, w, ldw, sw, ldsw, y, ldy, dt_y, m, n, k, ctypes.byref(p) if p else None, ws, wsb, None)

    for op in (0, 1):
        assert call(op=op, x=None) == -2 and call(op=op, ldx=8) == -3 and call(op=op, dt=B.DLA_F64) == -4
        assert call(op=op, w=None) == -5 and call(op=op, ldw=64) == -6 and call(op=op, sw=None) == -7 and call(op=op, ldsw=4) == -8
        assert call(op=op, y=None) == -9 and call(op=op, ldy=8) == -10 and call(op=op, dt_y=7) == -11
        assert call(op=op, m=-1) == -12 and call(op=op, n=-1) == -13 and call(op=op, k=-1) == -14
        assert call(op=op, p=B.Mx4Params(16, 17, 0)) == B.DLA_ERR_UNSUPPORTED_PARAMS
        assert call(op=op, p=B.Mx4Params(0, 0, 3)) == B.DLA_ERR_UNSUPPORTED_PARAMS
        assert call(op=op, m=0, x=None, w=None, sw=None, y=None) == 0
    assert call(op=2) == -1
    assert call(n=1 << 31) == B.DLA_ERR_TOO_LARGE


def test_menus_and_default_schedules(B):
    for kernel in (B.DLA_KERNEL_MX4_GEMM, B.DLA_KERNEL_MX4_APPLY):
        for op in (0, 1):
            tiles = [(t.tile_m, t.tile_n) for t in B.mx4_enumerate_tiles(kernel, op)]
            assert tiles and len(set(tiles)) == len(tiles)
            for m, n, k in ((1, 1, 1), (1, 4096, 4096), (8192, 8192, 8192), (300, 70, 9000)):
                d = B.mx4_default_params(kernel, op, m, n, k)
                assert (d.tile_m, d.tile_n) in tiles and 1 <= d.splits <= 32
            out = B.Mx4Params()
            r = ctypes.byref(out)
            for pos, args in ((1, (2, op, 1, 1, 1, 1)), (2, (kernel, 2, 1, 1, 1, 1)), (3, (kernel, op, 0, 1, 1, 1)), (4, (kernel, op, 1, 0, 1, 1)),
                              (5, (kernel, op, 1, 1, 0, 1)), (6, (kernel, op, 1, 1, 1, 0))):
                assert B.lib.mx4_default_params(*args, r) == -pos
            assert B.lib.mx4_default_params(kernel, op, 1, 1, 1, 1, None) == -7
    assert B.lib.mx4_enumerate_tiles(0, 0, 1, None, 0) == B.lib.mx4_enumerate_tiles(3, 2, 1, None, 0) == B.lib.mx4_enumerate_tiles(3, 0, 0, None, 0) == 0
    assert [B.lib.mx4_padded(c) for c in (-1, 0, 1, 128, 129)] == [0, 0, 128, 128, 256]


def test_binding_refuses_shapes_and_types(B):
    import torch
    u8 = torch.uint8
    w = B.Mx4(torch.zeros((4, 64), dtype=u8), torch.zeros((4, 4), dtype=u8), 100)
    with pytest.raises(ValueError):
        B.mx4_quantize(torch.zeros((4, 100)))
    with pytest.raises(ValueError):
        B.mx4_quantize(torch.zeros((4, 100)), B.Mx4(w.q, w.s, 99))
    with pytest.raises(ValueError):
        B.mx4_dequantize(w, torch.zeros((4, 99)))
    with pytest.raises(ValueError):
        B.mx4_gemm(0, w, B.Mx4(w.q, w.s, 101), torch.zeros((4, 4)))
    with pytest.raises(ValueError):
        B.mx4_apply(0, torch.zeros((3, 99)), w, torch.zeros((3, 4)))
    with pytest.raises(ValueError):
        B.mx4_apply(2, torch.zeros((3, 100)), w, torch.zeros((3, 4)))
    with pytest.raises(ValueError):  # too few columns for 129 with their padding
        B.mx4_dequantize(B.Mx4(w.q, w.s, 129), torch.zeros((4, 129)))
    with pytest.raises(ValueError):  # host memory
        B.mx4_dequantize(w, torch.zeros((4, 100)))
    with pytest.raises(TypeError):
        B.mx4_apply(0, torch.zeros((3, 100), dtype=torch.float64), w, torch.zeros((3, 4)))


def test_rows_that_share_their_memory_are_refused(B):
    """A broadcast matrix has row stride 0: one of one column would otherwise pass for a packed column."""
    import torch
    u8 = torch.uint8
    one = torch.zeros((1, 1))
    assert B._leading(one.expand(5, 1), "x") == 0 and B._leading(torch.zeros((1, 7)).expand(5, 7), "x") == 0
    assert B._leading(one, "x") == 1 and B._leading(torch.zeros((0, 3)), "x") == 3 and B._leading(torch.zeros((1, 0)), "x") == 1
    assert B.lib.mx4_quantize(FAKE, 0, 5, 1, B.DLA_F32, FAKE, 64, FAKE, 4, None, 0, None, 0, None) == -2
    shared = B.Mx4(torch.zeros((1, 64), dtype=u8).expand(4, 64), torch.zeros((4, 4), dtype=u8), 100)
    assert shared._args()[1] == 0
    assert B.lib.mx4_dequantize(FAKE, 0, FAKE, 4, 4, 100, B.DLA_F32, FAKE, 100, None) == -2
    with pytest.raises(ValueError):  # every other byte of a buffer
        B._mx4_workspace(0, one.device, torch.zeros(512, dtype=u8)[::2], None)
    with pytest.raises(ValueError):  # columns that are not neighbours
        B.Mx4(torch.zeros((4, 128), dtype=u8)[:, ::2], torch.zeros((4, 4), dtype=u8), 100)
    with pytest.raises(ValueError):
        B.Mx4(torch.zeros((4, 64), dtype=torch.int8), torch.zeros((4, 4), dtype=u8), 100)
    with pytest.raises(ValueError):
        B.Mx4(torch.zeros((4, 64), dtype=u8), torch.zeros((3, 4), dtype=u8), 100)


def test_launches_of_too_many_threads_are_refused(B):
    """A launch has fewer than 2^32 threads.  (Without a GPU a call that gets as far as its launch fails with another code.)"""
    big = 1 << 22
    assert B.lib.mx4_quantize(FAKE, big, big, big, B.DLA_BF16, FAKE, big // 2, FAKE, big // 32, None, 0, None, 0, None) == B.DLA_ERR_TOO_LARGE
    assert B.lib.mx4_quantize(FAKE, big, big, big, B.DLA_BF16, None, 0, None, 0, FAKE, big // 2, FAKE, big // 32, None) == B.DLA_ERR_TOO_LARGE
    for dt in (B.DLA_F32, B.DLA_F16):
        assert B.lib.mx4_dequantize(FAKE, 1 << 17, FAKE, 1 << 13, 1 << 18, 1 << 18, dt, FAKE, 1 << 18, None) == B.DLA_ERR_TOO_LARGE
    n, one = 1 << 20, B.Mx4Params(16, 32, 1)
    args = (FAKE, 64, FAKE, 4, FAKE, 64, FAKE, 4, FAKE, n, n, n, 128, B.DLA_BF16)
    assert B.lib.mx4_gemm(0, *args, ctypes.byref(one), None, 0, None) == B.DLA_ERR_TOO_LARGE
    two, m = B.Mx4Params(256, 256, 2), 1 << 18  # the tiles alone would do, joining their 2^36 values would not
    args = (FAKE, 128, FAKE, 8, FAKE, 128, FAKE, 8, FAKE, m, m, m, 256, B.DLA_BF16)
    assert B.lib.mx4_gemm(0, *args, ctypes.byref(two), FAKE, 1 << 60, None) == B.DLA_ERR_TOO_LARGE
    assert B.lib.mx4_gemm(0, FAKE, 64, FAKE, 4, FAKE, 64, FAKE, 4, FAKE, n, n, n, 0, B.DLA_BF16, None, None, 0, None) == B.DLA_ERR_TOO_LARGE
    wide = 1 << 21  # terms
    many = 1 << 28
    assert B.lib.mx4_apply(0, FAKE, wide, B.DLA_F32, FAKE, wide // 2, FAKE, wide // 32, FAKE, 1, B.DLA_F32, many, 1, wide, None, FAKE, 1 << 60,
                           None) == B.DLA_ERR_TOO_LARGE
    assert B.lib.mx4_apply(0, FAKE, 2 * wide, B.DLA_F32, FAKE, wide, FAKE, wide // 16, FAKE, 1, B.DLA_F32, 1, 1, 2 * wide, None, FAKE, 1 << 60,
                           None) == B.DLA_ERR_TOO_LARGE


@pytest.mark.parametrize("kernel,op,m,n,k,dtype", [("mx4_gemm", 0, 100, 300, 5000, "f32"), ("mx4_gemm", 1, 8192, 8192, 8192, "bf16"),
                                                   ("mx4_apply", 0, 1, 4096, 16384, "f16"), ("mx4_apply", 1, 333, 2200, 1801, "f32"),
                                                   ("mx4_apply", 1, 5, 1, 200, "bf16")])
def test_search_space_holds_the_default_and_legal_schedules_only(B, kernel, op, m, n, k, dtype):
    from paper_2309_07235_amd import tune
    space, default = tune.mx4_space(kernel, op, m, n, k, dtype)
    assert space.decode(space.encode(default)) == default and space.is_legal(space.encode(default))
    dt = {"f32": B.DLA_F32, "bf16": B.DLA_BF16, "f16": B.DLA_F16}[dtype]
    out = B.Mx4Params()
    for i in range(len(space.values[0])):
        for j in range(len(space.values[1])):
            if not space.is_legal((i, j)):
                continue
            c = space.decode((i, j))
            p = B.Mx4Params(*c["tile"], c["splits"])
            if kernel == "mx4_gemm":  # (a legal schedule's parts, or none)
                need = B.lib.mx4_gemm_workspace_bytes(m, n, k, ctypes.byref(p))
            else:
                need = B.lib.mx4_apply_workspace_bytes(op, FAKE, n if op else k, dt, m, n, k, ctypes.byref(p))
            parts = c["splits"] * m * (k if op and kernel == "mx4_apply" else n) * 4 if c["splits"] > 1 else 0
            assert need >= parts, c
    assert len(space.features(space.encode(default))) == 3


def test_every_tile_is_the_choice_for_some_sizes(B):
    """Nothing in the menus that no call without a schedule reaches."""
    for kernel in (B.DLA_KERNEL_MX4_GEMM, B.DLA_KERNEL_MX4_APPLY):
        for op in (0, 1) if kernel == B.DLA_KERNEL_MX4_APPLY else (0,):
            for dt in (B.DLA_F32, B.DLA_BF16, B.DLA_F16):
                left = {(t.tile_m, t.tile_n) for t in B.mx4_enumerate_tiles(kernel, op, dt)}
                for m in (1, 2, 8, 16, 17, 24, 32, 33, 40, 48, 50, 64, 65, 96, 128, 200, 256, 400, 512, 700, 1024, 2048, 4096, 8192):
                    for n in (64, 128, 256, 500, 1024, 2048, 4096, 8192, 16384):
                        for k in (64, 128, 512, 1024, 2048, 4096, 8192):
                            d = B.mx4_default_params(kernel, op, m, n, k, dt)
                            left.discard((d.tile_m, d.tile_n))
                assert not left, (kernel, op, dt, left)


def test_apply_workspace_follows_how_x_lies(B):
    """X that a kernel takes as it lies needs no copy; any other needs room for one, which the call insists on."""
    m, n, k = 64, 512, 256
    query, f = B.lib.mx4_apply_workspace_bytes, B.lib.mx4_apply

    def need(op, x, ldx, dt, terms_n=n, terms_k=k):
        return query(op, x, ldx, dt, m, terms_n, terms_k, ctypes.byref(one))

    for op in (0, 1):
        for tile in ((16, 32), (128, 128)) if op == 0 else ((128, 128),):
            one = B.Mx4Params(*tile, 1)
            terms = n if op else k
            assert need(op, FAKE, terms, B.DLA_BF16) == 0
            assert need(op, ctypes.c_void_p(0x1002), terms, B.DLA_BF16) >= m * terms * 2
            assert need(op, FAKE, terms + 1, B.DLA_BF16) >= m * terms * 2
            assert need(op, FAKE, terms, B.DLA_F32) >= m * terms * 6
            assert (need(op, FAKE, terms, B.DLA_F16) == 0) == (tile == (16, 32))  # two bf16 terms for the other
            got = need(op, FAKE, terms + 1, B.DLA_BF16)
            args = (op, FAKE, terms + 1, B.DLA_BF16, FAKE, k // 2, FAKE, k // 32, FAKE, max(n, k), B.DLA_F32, m, n, k, ctypes.byref(one))
            assert f(*args, None, got, None) == B.DLA_ERR_WORKSPACE
            assert f(*args, FAKE, got - 1, None) == B.DLA_ERR_WORKSPACE
            assert f(*args, ctypes.c_void_p(0x1080), got, None) == B.DLA_ERR_WORKSPACE
    one = B.Mx4Params(128, 128, 1)
    assert need(0, FAKE, k - 8, B.DLA_BF16, n, k - 8) >= m * (k - 8) * 2  # no whole steps
    assert query(2, FAKE, k, B.DLA_BF16, m, n, k, None) == query(0, FAKE, k, B.DLA_F64, m, n, k, None) == query(0, FAKE, k, B.DLA_BF16, 0, n, k, None) == 0


def test_padded_columns_are_the_librarys(B):
    for cols in (-1000, -200, -128, -1, 0, 1, 127, 128, 129, 1801, 1 << 30, (1 << 30) + 1):
        assert B.mx4_padded(cols) == B.lib.mx4_padded(cols), cols
    assert B.mx4_padded(-200) == 0 and B.mx4_padded(129) == 256


def test_one_row_in_a_buffer_of_any_width(B):
    """One token's microscaled form in the front of a longer buffer: nothing lies behind its row, so the buffer's width is no leading
    dimension that the library could refuse (no multiple of 16 or 4 bytes, longer than 2^22)."""
    import torch
    u8 = torch.uint8
    for per_q, per_s, cols in ((71, 5, 100), (64, 4, 128), (200, 9, 129), ((1 << 22) + 16, (1 << 22) + 4, 300)):
        q, lds = B.Mx4(torch.zeros((1, per_q), dtype=u8), torch.zeros((1, per_s), dtype=u8), cols)._args()[1::2]
        assert (q, lds) == (B.mx4_padded(cols) // 2, B.mx4_padded(cols) // 32)
        # the checks let it pass: the call ends at the next one, the missing result
        assert B.lib.mx4_dequantize(FAKE, q, FAKE, lds, 1, cols, B.DLA_F32, None, cols, None) == -8
