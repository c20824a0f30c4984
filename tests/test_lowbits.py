"""Microscaled 4-bit matrices and 8-bit checkpoints without a GPU: the oracle's own pins, layouts, sizes, refusals."""
import ctypes as C

import numpy as np
import pytest

from oracle import lowbits as ref
from paper_2102_04782_amd import binding as daq


def test_oracle_nearest_codes_against_a_search_over_all_codes():
    rng = np.random.default_rng(0)
    x = (rng.standard_normal((40, 96)) * np.exp2(rng.integers(-20, 20, (40, 1)))).astype(np.float32)
    codes, byte = ref.mx4_codes(x)
    v = ref.mx4_values(codes, byte, 96)
    s = np.repeat(np.exp2(byte - 127.0), 32, axis=1)
    grid = np.concatenate((ref.GRID, -ref.GRID))
    best = np.abs(x[:, :, None].astype(np.float64) - grid * s[:, :, None]).min(axis=2)
    assert np.array_equal(np.abs(x - v), best)                       # no code is nearer
    top = np.abs(x.reshape(40, 3, 32)).max(axis=2)
    assert np.all(top < 8 * np.exp2(byte - 127.0)) and np.all(top >= 4 * np.exp2(byte - 127.0))


def test_oracle_ties_go_to_the_even_code():
    middle = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    x = np.zeros((1, 32), np.float32)
    x[0, :7], x[0, 7:14], x[0, 31] = middle, -middle, 6.0
    codes, byte = ref.mx4_codes(x)
    assert byte[0, 0] == 127 and list(codes[0, 0, :7]) == [0, 2, 2, 4, 4, 6, 6] and list(codes[0, 0, 7:14] - 8) == [0, 2, 2, 4, 4, 6, 6]


def test_oracle_stochastic_codes_bracket_are_unbiased_and_cut_nothing_off():
    rng = np.random.default_rng(1)
    row = rng.standard_normal(64).astype(np.float32)
    x = np.repeat(row[None], 6000, axis=0)
    codes, byte = ref.mx4_codes(x, True, 12345)
    s = np.repeat(np.exp2(byte - 127.0), 32, axis=1)
    v = ref.mx4_values(codes, byte, 64)
    assert np.all(np.abs(x) <= 6 * s) and np.all(np.abs(x).reshape(6000, 2, 32).max(axis=2) > 3 * s[:, ::32])
    t = np.abs(row) / s[0]
    gap = np.where(t < 2, 0.5, np.where(t < 4, 1.0, 2.0)) * s[0]
    assert np.all(np.abs(v - x) < gap)
    # the mean of 6000 draws of a two-valued variable of spread `gap`: six deviations of at most gap / (2 sqrt 6000), and the 2^-16 of the draws
    assert np.all(np.abs(v.mean(axis=0) - row) <= gap * (6 / (2 * np.sqrt(6000)) + 2.0 ** -16))
    d = ref.draws(64, 33, 7)
    assert d.min() >= 0 and d.max() < 65536 and np.unique(d).size > 2000 and not np.array_equal(d, ref.draws(64, 33, 8))


def test_oracle_checkpoint_codes():
    rng = np.random.default_rng(2)
    x = (rng.standard_normal((30, 70)) * np.exp2(rng.integers(-30, 30, (30, 1)))).astype(np.float32)
    codes, byte = ref.ckpt8_codes(x)
    v = ref.ckpt8_values(codes, byte, 30, 70)
    s = np.repeat(np.exp2(byte - 127.0), 32, axis=1)[:, :70]
    over = np.abs(x) > 127.5 * s
    assert np.all(np.abs(v - x)[~over] <= 0.5 * s[~over]) and np.all(np.abs(v - x)[over] <= s[over]) and np.abs(codes).max() <= 127
    again, byte2 = ref.ckpt8_codes(v)
    assert np.array_equal(ref.ckpt8_values(again, byte2, 30, 70), v)         # what was saved is saved as it is


@pytest.mark.parametrize("fn", ["silu", "gelu"])
def test_oracle_slopes_against_differences(fn):
    x = np.linspace(-9, 9, 401)
    h = 1e-5
    want = (ref.act(x + h, fn)[0] - ref.act(x - h, fn)[0]) / (2 * h)
    # second-order differences: h^2 / 6 times a third derivative below 2, and rounding of 9 * 2^-53 / h
    assert np.all(np.abs(ref.act(x, fn)[1] - want) <= h * h + 2e-10)


@pytest.mark.parametrize("rows,cols", [(1, 1), (31, 33), (32, 256), (33, 257), (100, 1000)])
def test_layouts_hold_what_the_oracle_packs(rows, cols):
    codes, byte = ref.mx4_codes(np.ones((rows, cols), np.float32))
    L = daq.layout_mx4(rows, cols)
    assert L.bytes == ref.mx4_buffer(codes, byte).size and L.bytes % 256 == 0 and L.off_scales == L.row_blocks * L.groups * 4096
    for parts in (1, 2):
        codes, byte = ref.ckpt8_codes(np.ones((rows, parts * cols), np.float32), parts)
        L = daq.layout_ckpt8(rows, cols, parts)
        assert L.bytes == ref.ckpt8_buffer(codes, byte).size and L.bytes % 256 == 0 and L.pitch % 32 == 0 and L.pitch - cols < 32


def test_sizes_of_no_rows_and_of_too_many():
    assert daq.layout_mx4(0, 5).bytes == 0 and daq.layout_ckpt8(0, 5).bytes == 0
    for fn, sizes, code in [("daq_layout_mx4", (-1, 4), daq.ERR_INVALID_ARG), ("daq_layout_mx4", (4, -1), daq.ERR_INVALID_ARG),
                            ("daq_layout_mx4", (1 << 31, 4), daq.ERR_UNSUPPORTED), ("daq_layout_mx4", (1 << 30, 1 << 30), daq.ERR_UNSUPPORTED)]:
        assert getattr(daq.lib(), fn)(*sizes, C.byref(daq.Mx4Layout())) == code
    for sizes, code in [((4, 0, 1), daq.ERR_INVALID_ARG), ((4, 4, 3), daq.ERR_INVALID_ARG), ((4, 4, 0), daq.ERR_INVALID_ARG), ((-1, 4, 1), daq.ERR_INVALID_ARG),
                        ((1, 1 << 31, 1), daq.ERR_UNSUPPORTED), ((1, 1 << 30, 2), daq.ERR_UNSUPPORTED), ((1 << 20, 1 << 21, 1), daq.ERR_UNSUPPORTED)]:
        assert daq.lib().daq_layout_ckpt8(*sizes, C.byref(daq.Ckpt8Layout())) == code
    assert daq.lib().daq_layout_mx4(1, 1, None) == daq.ERR_INVALID_ARG and daq.lib().daq_layout_ckpt8(1, 1, 1, None) == daq.ERR_INVALID_ARG
    assert daq.layout_mx4(1 << 20, 1 << 14).bytes == (1 << 34) // 2 + (1 << 34) // 32      # offsets beyond 32 bits


def test_refusals_come_before_any_launch():
    L, a, odd, n = daq.lib(), 1 << 20, (1 << 20) + 2, C.c_size_t(0)   # addresses that are never read: there is no GPU here
    INV, WS, UNS = daq.ERR_INVALID_ARG, daq.ERR_WORKSPACE, daq.ERR_UNSUPPORTED
    q = lambda src=a, dt=0, r=4, c=40, ld=40, tr=0, mode=0, dst=a: L.daq_mx4_quantize(src, dt, r, c, ld, tr, mode, 0, dst, None)
    assert q(src=None) == q(dst=None) == q(src=a + 2) == q(dst=a + 128) == q(ld=39) == q(c=0) == q(r=-1) == q(mode=2) == q(dt=2) == INV
    assert q(src=a + 1, dt=1) == INV and q(r=1 << 20, c=1 << 12, ld=1 << 12, mode=1) == UNS
    assert q(r=0) == q(r=0, tr=1) == daq.OK
    v = lambda src=a, r=4, c=40, dst=a, dt=0, ld=40: L.daq_mx4_dequantize(src, r, c, dst, dt, ld, None)
    assert v(src=None) == v(dst=None) == v(src=a + 16) == v(dst=odd) == v(ld=39) == v(dt=3) == v(r=-1) == v(c=-1) == INV and v(r=0) == v(c=0) == daq.OK
    m = lambda M=4, N=8, K=40, A=a, B=a, D=a, dt=0, ld=8, ws=None, wn=0: L.daq_mx4_matmul(M, N, K, A, B, D, dt, ld, ws, wn, None)
    assert m(A=None) == m(B=None) == m(D=None) == m(A=a + 16) == m(B=a + 16) == m(D=odd) == m(ld=7) == m(N=0) == m(K=0) == m(M=-1) == m(dt=9) == INV
    assert m(K=1 << 28) == UNS and m(M=1 << 31) == UNS and m(M=0) == daq.OK
    assert L.daq_mx4_matmul_workspace(4, 0, 4, C.byref(n)) == L.daq_mx4_matmul_workspace(4, 4, 4, None) == INV
    li = lambda M=64, N=8, K=40, X=a, xd=0, ldx=40, mode=0, W=a, Y=a, yd=0, ldy=8, ws=a, wn=1 << 30: L.daq_mx4_linear(M, N, K, X, xd, ldx, mode, 0, W, Y, yd, ldy, ws, wn, None)
    assert li(X=None) == li(W=None) == li(Y=None) == li(ldx=39) == li(ldy=7) == li(xd=2) == li(yd=2) == li(mode=3) == li(X=odd) == li(N=0) == INV
    assert L.daq_mx4_linear_workspace(4, 4, 4, 2, 0, C.byref(n)) == L.daq_mx4_linear_workspace(4, 4, 4, 0, 2, C.byref(n)) == INV
    assert L.daq_mx4_linear_workspace(1, 8192, 2048, 1, 0, C.byref(n)) == daq.OK and n.value == 0          # one token: one launch
    assert L.daq_mx4_linear_workspace(4096, 4096, 4096, 0, 0, C.byref(n)) == daq.OK and n.value >= 4096 * 4096 // 2
    big = dict(M=4096, N=4096, K=4096, ldx=4096, ldy=4096)
    assert li(ws=None, wn=0, **big) == li(ws=a, wn=n.value - 1, **big) == li(ws=a + 16, **big) == WS and li(M=0) == daq.OK
    for fn in (lambda x=a, dt=0, r=4, c=40, p=2, ld=80, k=a: L.daq_ckpt8_save(x, dt, r, c, p, ld, k, None),
               lambda x=a, dt=0, r=4, c=40, p=2, ld=80, k=a: L.daq_ckpt8_restore(k, r, c, p, x, dt, ld, None)):
        assert fn(x=None) == fn(k=None) == fn(k=a + 64) == fn(x=odd) == fn(dt=2) == fn(p=3) == fn(ld=79) == fn(c=0) == fn(r=-1) == INV and fn(r=0) == daq.OK
    f = lambda h=a, dt=0, r=4, c=40, ldh=80, act=0, gated=1, y=a, ldy=40, k=a: L.daq_ckpt8_act_forward(h, dt, r, c, ldh, act, gated, y, ldy, k, None)
    assert f(h=None) == f(y=None) == f(k=None) == f(h=odd) == f(y=odd) == f(k=a + 32) == f(ldh=79) == f(ldy=39) == f(act=2) == f(dt=2) == f(c=0) == INV
    assert f(r=0) == daq.OK
    b = lambda dy=a, dt=0, r=4, c=40, ld=40, k=a, act=0, gated=1, dh=a, ldh=80, yk=None: L.daq_ckpt8_act_backward(dy, dt, r, c, ld, k, act, gated, dh, ldh, yk, None)
    assert b(dy=None) == b(dh=None) == b(k=None) == b(dy=odd) == b(dh=odd) == b(k=a + 32) == b(yk=a + 32) == b(ld=39) == b(ldh=79) == b(act=-1) == b(dt=2) == INV
    assert b(r=0) == daq.OK
    g = lambda M=4, N=8, K=40, dy=a, dt=0, ld=8, x=a, dW=a, ldw=40, ws=a, wn=1 << 30: L.daq_ckpt8_weight_grad(M, N, K, dy, dt, ld, x, dW, ldw, 0, ws, wn, None)
    assert g(dy=None) == g(x=None) == g(dW=None) == g(dy=odd) == g(dW=odd) == g(x=a + 32) == g(ld=7) == g(ldw=39) == g(N=0) == g(K=0) == g(M=-1) == g(dt=2) == INV and g(M=1 << 24) == UNS
    assert L.daq_ckpt8_weight_grad_workspace(4, 4, 4, 5, 4, 0, C.byref(n)) == L.daq_ckpt8_weight_grad_workspace(4, 4, 4, 0, 4, -1, C.byref(n)) == INV
    assert L.daq_ckpt8_weight_grad_workspace(64, 64, 64, 1, 64, 0, C.byref(n)) == daq.OK and n.value == 0
    assert L.daq_ckpt8_weight_grad_workspace(2048, 2048, 64, 1, 2048, 0, C.byref(n)) == daq.OK and n.value > 0
    assert g(M=2048, N=2048, K=64, dt=1, ld=2048, ldw=64, ws=None, wn=0) == g(M=2048, N=2048, K=64, dt=1, ld=2048, ldw=64, wn=n.value - 1) == WS


def test_oracle_gelu_keeps_its_tail():
    """Far below zero against the continued fraction Phi(-t) = phi(t) / (t + 1 / (t + 2 / (t + 3 / ...))).  With u = 2^-53: t / sqrt 2 is off by two
    units, which erfc makes t^2 + 1 times as many of; t^2 / 2 by one, which the exponential makes t^2 / 2 times as many of; the functions and the
    fraction are good to 16 units together.  The slope is a difference whose terms are at most 5/4 of it."""
    t = np.linspace(3, 30, 271)
    f = t.copy()
    for k in range(400, 0, -1):
        f = t + k / f
    phi = np.exp(-t * t / 2) / np.sqrt(2 * np.pi)
    y, slope = ref.act(-t, "gelu")
    rel = (3 * t * t + 18) * 2.0 ** -53
    assert np.all(np.abs(y + t * phi / f) <= rel * t * phi / f)
    assert np.all(np.abs(slope - (phi / f - t * phi)) <= 2 * rel * t * phi)


def test_launches_of_too_many_threads_are_refused_before_the_first():
    """A launch takes fewer than 2^32 threads along an axis.  Where a call makes several, none is made: there is no GPU here to make one."""
    L, a, n, UNS = daq.lib(), 1 << 20, C.c_size_t(0), daq.ERR_UNSUPPORTED
    assert L.daq_mx4_quantize(a, 0, 1 << 29, 1, 1, 0, 0, 0, a, None) == L.daq_mx4_quantize(a, 1, 1, 1 << 30, 1 << 30, 1, 1, 0, a, None) == UNS
    assert L.daq_mx4_dequantize(a, 1 << 29, 1, a, 0, 1, None) == UNS
    for rows, parts in ((1 << 30, 1), (1 << 29, 2)):
        assert L.daq_ckpt8_save(a, 1, rows, 1, parts, parts, a, None) == L.daq_ckpt8_restore(a, rows, 1, parts, a, 0, parts, None) == UNS
    assert L.daq_ckpt8_act_forward(a, 0, 1 << 30, 1, 1, 0, 0, a, 1, a, None) == L.daq_ckpt8_act_backward(a, 0, 1 << 30, 1, 1, a, 1, 0, a, 1, None, None) == UNS
    wide = 65535 * 2048 + 1                                       # along the other axis workgroups are counted
    assert L.daq_ckpt8_save(a, 1, 1, wide, 1, wide, a, None) == L.daq_ckpt8_restore(a, 1, wide, 1, a, 1, wide, None) == UNS
    assert L.daq_ckpt8_act_forward(a, 1, 1, wide, wide, 0, 0, a, wide, a, None) == UNS
    M = N = 1 << 20
    assert L.daq_mx4_matmul(M, N, 4096, a, a, a, 0, N, None, 0, None) == UNS
    assert L.daq_mx4_linear(M, N, 4096, a, 0, 4096, 0, 0, a, a, 0, N, a, 1 << 40, None) == UNS
    for dtype in (0, 1):
        assert L.daq_ckpt8_weight_grad(1, N, M, a, dtype, N, a, a, M, 0, a, 1 << 60, None) == UNS
    assert L.daq_ckpt8_weight_grad(0, 1 << 17, 1 << 17, None, 0, 0, None, a, 1 << 17, 0, None, 0, None) == UNS
    assert L.daq_ckpt8_weight_grad(0, 1 << 17, 1 << 17, None, 0, 0, None, a, 1 << 17, 1, None, 0, None) == daq.OK      # nothing to launch
    # one row: a launch whose workgroups quantize it, while there are few enough of them
    for N, one_launch in (((1 << 28) - 32, True), (1 << 28, False)):
        assert L.daq_mx4_linear_workspace(1, N, 64, 1, 0, C.byref(n)) == daq.OK and (n.value == 0) == one_launch


def test_a_layout_belongs_to_its_caller():
    for fn, sizes in ((daq.layout_mx4, (70, 300)), (daq.layout_ckpt8, (70, 300, 2))):
        first = fn(*sizes)
        want, first.bytes, first.off_scales = (first.bytes, first.off_scales), 256, 0
        again = fn(*sizes)
        assert (again.bytes, again.off_scales) == want
    assert daq.alloc_mx4(70, 300, device="cpu").buf.numel() == daq.layout_mx4(70, 300).bytes
    assert daq.alloc_ckpt8(70, 300, 2, device="cpu").buf.numel() == daq.layout_ckpt8(70, 300, 2).bytes


def test_packed_buffers_off_the_gpu_are_refused(monkeypatch):
    """As weights read from a file are: their host addresses must not get to a kernel."""
    def reached(stream):
        raise RuntimeError("reached the call")

    monkeypatch.setattr(daq, "_stream", reached)
    q, c = daq.alloc_mx4(40, 70, device="cpu"), daq.alloc_ckpt8(40, 70, device="cpu")
    for call in (lambda: daq.mx4_dequantize(q), lambda: daq.mx4_matmul(q, q), lambda: daq.ckpt8_restore(c)):
        with pytest.raises(AssertionError):
            call()
