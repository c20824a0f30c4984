"""8-bit floating point matrices, routing and experts' products without a GPU: the oracle's own pins, layouts, sizes, refusals."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import fp8 as ref
from paper_2102_04782_amd import binding as daq


def test_oracle_codes_are_the_published_format():
    """A sign, four exponent and three mantissa bits with bias 7, largest value 448, smallest 2^-9: the library's own type of that name."""
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).to(torch.float64).numpy()
    assert np.array_equal(every[:127], ref.GRID) and np.array_equal(every[128:255], -ref.GRID) and np.isnan(every[127]) and np.isnan(every[255])


def test_oracle_nearest_codes_against_a_search_over_all_codes():
    rng = np.random.default_rng(0)
    x = (rng.standard_normal((20, 300)) * np.exp2(rng.integers(-20, 20, (20, 1)))).astype(np.float32)
    codes, byte = ref.quantize(x)
    v, s = ref.values(codes, byte), np.repeat(np.exp2(byte - 127.0), 128, axis=1)[:, :300]
    grid = np.concatenate((ref.GRID, -ref.GRID))
    best = np.abs(x[:, :, None].astype(np.float64) - grid * s[:, :, None]).min(axis=2)
    assert np.array_equal(np.abs(x - v), best)                        # no code is nearer
    top = np.stack([np.abs(x[:, b:b + 128]).max(1) for b in range(0, 300, 128)], 1)
    assert np.all(top <= 448 * np.exp2(byte - 127.0)) and np.all(top > 224 * np.exp2(byte - 127.0))      # nothing cut off, no smaller scale


def test_oracle_ties_go_to_the_even_code():
    middle = (ref.GRID[1:] + ref.GRID[:-1]) / 2
    code = ref.nearest(middle)
    assert np.all(code % 2 == 0) and np.all(np.abs(ref.GRID[code] - middle) == (ref.GRID[1:] - ref.GRID[:-1]) / 2)


def test_oracle_weights_have_the_values_of_their_transposes():
    w = np.random.default_rng(1).standard_normal((300, 200))
    codes, byte = ref.quantize_weights(w)
    assert np.array_equal(ref.values(codes, byte).T, ref.values(*ref.transposed_weights(codes, byte)))
    ct, bt = ref.quantize_weights(w.T)
    assert np.array_equal(ct, codes.T) and np.array_equal(ref.values(ct, bt).T, ref.values(codes, byte))


def test_oracle_scale_bytes():
    for top, byte in ((0.0, 1), (2.0 ** -140, 1), (448 * 2.0 ** -126, 1), (449 * 2.0 ** -126, 2), (1.0, 119), (1.75, 119), (1.7500001, 120), (448.0, 127), (448.5, 128),
                      (float(np.finfo(np.float32).max), 247), (np.inf, 255), (np.nan, 255)):
        assert ref.scale_byte(top) == byte, top


def test_oracle_route_by_hand():
    l = np.log(np.array([[1.0, 2.0, 4.0, 1.0], [1.0, 1.0, 1.0, 1.0]]))
    w, c = ref.route(l, 2, "softmax", renormalize=False)
    assert np.allclose(w, [[0.5, 0.25], [0.25, 0.25]]) and c.tolist() == [[2, 1], [0, 1]]
    w, c = ref.route(l, 2, "softmax", bias=[0.3, 0, 0, 0.6])                     # scores 1/8 1/4 1/2 1/8, with the bias .425 .25 .5 .725
    assert c.tolist() == [[3, 2], [3, 0]] and np.allclose(w, [[0.2, 0.8], [0.5, 0.5]])
    w, c = ref.route(np.array([[3.0, -3.0, 1.0, 1.0]]), 2, "sigmoid", groups=2, top_groups=1)    # .95 + .05 against .73 + .73
    assert c.tolist() == [[2, 3]] and np.allclose(w, 0.5)
    w, c = ref.route(np.array([[-np.inf, 0.0, -np.inf], [-np.inf] * 3, [np.nan, 1, 2]]), 2, "softmax")
    assert c.tolist() == [[1, -1], [-1, -1], [-1, -1]] and w[0].tolist() == [1.0, 0.0] and w[1].tolist() == [0.0, 0.0] and np.isnan(w[2]).all()


@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalize", [True, False])
def test_oracle_route_gradient_against_differences(kind, renormalize):
    """Central differences of step h = 2^-17 in 64 bits: off by h^2 of a third derivative below 8, and 2^-52 / h."""
    rng = np.random.default_rng(0)
    x, g, h = rng.standard_normal((6, 9)), rng.standard_normal((6, 3)), 2.0 ** -17
    _, c = ref.route(x, 3, kind, renormalize=renormalize, scale=1.5)
    grad = ref.route_backward(g, x, c, kind, renormalize, 1.5)

    def loss(v):
        s = np.take_along_axis(ref.scores(v, kind), c, 1)
        return (1.5 * (s / s.sum(1, keepdims=True) if renormalize else s) * g).sum()

    for t in range(6):
        for e in range(9):
            d = np.zeros_like(x)
            d[t, e] = h
            assert abs((loss(x + d) - loss(x - d)) / (2 * h) - grad[t, e]) < 2.0 ** -29 * (1 + np.abs(g).sum())


def test_oracle_plan_by_hand():
    counts, table, rows, place = ref.plan(np.array([[1, 0], [1, -1], [3, 1]]), 4)
    assert counts.tolist() == [1, 3, 0, 1] and table.tolist() == [[0, 1, 4, 4, 5], [0, 1, 2, 2, 3], [0, 1, 2, 2, 3], [0, 1, 2, 2, 3]]
    assert rows.tolist() == [1, 0, 2, 5, 4, -1] and place.tolist() == [[1, 0], [2, -1], [4, 3]]


@pytest.mark.parametrize("rows,cols", [(0, 5), (1, 1), (3, 128), (129, 513), (70, 1024), (5, 0)])
def test_layouts(rows, cols):
    L = daq.layout_fp8(rows, cols)
    assert L.pitch == -(-cols // 128) * 128 and L.off_scales % 256 == 0 and L.off_scales >= rows * L.pitch and L.bytes % 256 == 0
    assert L.bytes - L.off_scales >= -(-cols // 512) * rows * 4
    if rows and cols:
        codes, byte = ref.quantize(np.ones((rows, cols)))
        assert ref.buffer(codes, byte)[0].size == L.bytes
    L.bytes = 0
    assert daq.alloc_fp8(rows, cols, device="cpu").buf.numel() == daq.layout_fp8(rows, cols).bytes      # a layout is its caller's to change


def test_sizes_of_layouts_and_plans():
    for sizes, code in (((-1, 4), daq.ERR_INVALID_ARG), ((4, -1), daq.ERR_INVALID_ARG), ((1 << 31, 4), daq.ERR_UNSUPPORTED), ((1 << 30, 1 << 30), daq.ERR_UNSUPPORTED)):
        assert daq.lib().daq_layout_fp8(*sizes, C.byref(daq.Fp8Layout())) == code
    assert daq.lib().daq_layout_fp8(1, 1, None) == daq.ERR_INVALID_ARG
    assert daq.layout_fp8(1 << 20, 1 << 14).off_scales == 1 << 34                               # offsets beyond 32 bits
    rng = np.random.default_rng(0)
    for _ in range(200):      # whatever the choice is, its blocks of 128 (and the tiles of 256 and 64) fit
        T, k, E = int(rng.integers(1, 300)), int(rng.integers(1, 6)), int(rng.integers(1, 40))
        c = rng.integers(-1, E, (T, k)) if rng.random() < 0.5 else np.minimum(rng.geometric(0.5, (T, k)) - 1, E - 1)
        _, table, _, _ = ref.plan(c, E)
        assert table[2, E] * 128 <= daq.experts_columns(T, k, E) == ref.columns(T, k, E)
    n = C.c_int64(0)
    L = daq.lib()
    assert L.daq_experts_columns(4, 2, 1025, C.byref(n)) == L.daq_experts_columns(1 << 28, 1, 4, C.byref(n)) == daq.ERR_UNSUPPORTED
    assert L.daq_experts_columns(4, 0, 4, C.byref(n)) == L.daq_experts_columns(-1, 1, 4, C.byref(n)) == L.daq_experts_columns(4, 2, 4, None) == daq.ERR_INVALID_ARG


def test_refusals_come_before_any_launch():
    L, a, odd, n = daq.lib(), 1 << 20, (1 << 20) + 2, C.c_size_t(0)      # addresses that are never read: there is no GPU here
    INV, WS, UNS, OK = daq.ERR_INVALID_ARG, daq.ERR_WORKSPACE, daq.ERR_UNSUPPORTED, daq.OK
    q = lambda src=a, dt=0, r=4, c=40, ld=40, br=a, bc=a: L.daq_fp8_quantize(src, dt, r, c, ld, br, bc, None)
    assert q(src=None) == q(br=None, bc=None) == q(src=odd) == q(br=a + 128) == q(bc=a + 128) == q(ld=39) == q(c=0) == q(r=-1) == q(dt=2) == INV
    assert q(src=a + 1, dt=1) == INV and q(r=0) == q(r=0, br=None, bc=None) == OK
    assert q(r=(1 << 31) - 1, c=512, ld=512, bc=None) == q(r=1 << 22, c=1 << 18, ld=1 << 18) == UNS           # launches of 2^32 threads
    w = lambda src=a, dt=0, e=2, r=4, c=40, ld=40, st=160, d=a, t=a: L.daq_fp8_quantize_weights(src, dt, e, r, c, ld, st, d, t, None)
    assert w(src=None) == w(d=None, t=None) == w(src=odd) == w(d=a + 8) == w(t=a + 8) == w(ld=39) == w(c=0) == w(r=0) == w(e=-1) == w(dt=3) == w(st=-1) == INV
    assert w(e=0) == OK and w(e=1 << 30, r=4) == UNS
    v = lambda src=a, r=4, c=40, dst=a, dt=0, ld=40: L.daq_fp8_dequantize(src, r, c, dst, dt, ld, None)
    assert v(src=None) == v(dst=None) == v(src=a + 16) == v(dst=odd) == v(ld=39) == v(dt=3) == v(r=-1) == v(c=-1) == INV and v(r=0) == v(c=0) == OK
    m = lambda M=4, N=8, K=40, A=a, B=a, D=a, dt=0, ld=8, acc=0, ws=a, wn=1 << 40: L.daq_fp8_matmul(M, N, K, A, B, D, dt, ld, acc, ws, wn, None)
    assert m(A=None) == m(B=None) == m(D=None) == m(A=a + 16) == m(B=a + 16) == m(D=odd) == m(ld=7) == m(N=0) == m(K=-1) == m(M=-1) == m(dt=9) == INV
    assert m(dt=1, acc=1) == INV and m(M=0) == OK
    assert m(K=1 << 23) == m(M=1 << 31) == m(N=1 << 31, ld=1 << 31) == UNS
    assert m(M=1 << 20, N=1 << 20, K=128, ld=1 << 20) == UNS                                                      # tiles of a launch
    assert L.daq_fp8_matmul_workspace(4, 0, 4, 0, C.byref(n)) == L.daq_fp8_matmul_workspace(4, 4, 4, 0, None) == L.daq_fp8_matmul_workspace(4, 4, 4, 2, C.byref(n)) == INV
    li = lambda M=64, N=8, K=40, X=a, xd=0, ldx=40, W=a, Y=a, yd=0, ldy=8, ws=a, wn=1 << 40: L.daq_fp8_linear(M, N, K, X, xd, ldx, W, Y, yd, ldy, ws, wn, None)
    assert li(X=None) == li(W=None) == li(Y=None) == li(ldx=39) == li(ldy=7) == li(xd=2) == li(yd=2) == li(X=odd) == li(N=0) == li(K=0) == li(W=a + 64) == INV
    assert li(M=0) == OK
    assert L.daq_fp8_linear_workspace(1, 8192, 4096, 1, 1, C.byref(n)) == OK and n.value == 0                     # one token: one launch
    assert L.daq_fp8_linear_workspace(4096, 4096, 4096, 0, 0, C.byref(n)) == OK and n.value >= 4096 * 4096
    big = dict(M=4096, N=4096, K=4096, ldx=4096, ldy=4096)
    assert li(ws=None, wn=0, **big) == li(ws=a, wn=n.value - 1, **big) == li(ws=a + 16, **big) == WS
    o = lambda s=0, k=2, g=1, t=1, r=1, sc=1.0: C.byref(daq.RouteOpts(s, k, g, t, r, sc))
    r = lambda T=4, E=8, l=a, dt=0, ld=8, b=None, op=None, w=a, c=a: L.daq_route(T, E, l, dt, ld, b, op or o(), w, c, None)
    assert r(l=None) == r(l=odd) == r(dt=2) == r(ld=7) == r(b=odd) == r(w=None) == r(w=odd) == r(c=None) == r(c=odd) == r(E=0) == r(T=-1) == INV
    for bad in (o(s=2), o(k=0), o(k=9), o(g=3), o(g=0), o(g=4, t=5), o(g=4, t=0), o(g=4, t=1, k=3), o(sc=float("nan")), o(sc=float("inf"))):
        assert r(op=bad) == INV
    assert L.daq_route(4, 8, a, 0, 8, None, None, a, a, None) == INV
    assert r(E=1025, ld=1025) == r(E=64, ld=64, op=o(k=33)) == r(E=130, ld=130, op=o(g=65, t=2)) == r(T=1 << 28) == UNS and r(T=0) == OK
    rb = lambda T=4, E=8, g=a, l=a, dt=0, ld=8, c=a, op=None, d=a, ldd=8: L.daq_route_backward(T, E, g, l, dt, ld, c, op or o(), d, ldd, None)
    assert rb(g=None) == rb(g=odd) == rb(l=None) == rb(c=None) == rb(d=None) == rb(d=odd) == rb(ld=7) == rb(ldd=7) == rb(op=o(k=9)) == INV and rb(T=0) == OK
    p = lambda T=4, k=2, E=8, c=a, n_=a, t=a, rw=a, pl=a, ws=a, wn=1 << 40: L.daq_experts_plan(T, k, E, c, n_, t, rw, pl, ws, wn, None)
    assert p(c=None) == p(n_=None) == p(t=None) == p(rw=None) == p(pl=None) == p(c=odd) == p(n_=odd) == p(t=odd) == p(rw=odd) == p(pl=odd) == p(k=0) == p(E=0) == p(T=-1) == INV
    assert p(E=1025) == p(T=1 << 28) == UNS
    assert L.daq_experts_plan_workspace(100000, 8, 64, C.byref(n)) == OK and n.value > 0
    assert p(T=100000, k=8, E=64, ws=None, wn=0) == p(T=100000, k=8, E=64, wn=n.value - 1) == p(T=100000, k=8, E=64, ws=a + 4) == WS
    e = lambda T=4, k=2, E=8, t=a, rw=a, pl=a: C.byref(daq.Experts(T, k, E, t, rw, pl))
    bad_plans = (None, e(T=-1), e(k=0), e(E=0), e(E=1025), e(T=1 << 28), e(t=None), e(rw=None), e(pl=None), e(t=odd), e(rw=odd), e(pl=odd))
    x = lambda pl=None, src=a, dt=0, c=40, ld=40, s=0, br=a, bc=a: L.daq_experts_quantize(pl or e(), src, dt, c, ld, s, br, bc, None)
    assert x(src=None) == x(src=odd) == x(dt=2) == x(c=0) == x(ld=39) == x(br=None, bc=None) == x(br=a + 1) == x(bc=a + 1) == INV and x(e(T=0)) == OK
    mm = lambda pl=None, N=8, K=40, A=a, s=0, W=a, Y=a, dt=0, ld=8: L.daq_experts_matmul(pl or e(), N, K, A, s, W, Y, dt, ld, None)
    assert mm(N=0) == mm(K=0) == mm(A=None) == mm(W=None) == mm(Y=None) == mm(A=a + 1) == mm(W=a + 1) == mm(Y=odd) == mm(dt=2) == mm(ld=7) == INV
    assert mm(e(T=0)) == OK and mm(N=1 << 30, ld=1 << 30) == mm(K=1 << 23) == mm(e(T=1 << 20, k=1), K=1 << 13) == UNS      # (taken rows beyond one descriptor)
    el = lambda pl=None, N=8, K=40, X=a, xd=0, ldx=40, s=0, W=a, Y=a, yd=0, ldy=8, ws=a, wn=1 << 40: L.daq_experts_linear(pl or e(), N, K, X, xd, ldx, s, W, Y, yd, ldy, ws, wn, None)
    assert el(X=None) == el(X=odd) == el(xd=2) == el(yd=2) == el(ldx=39) == el(ldy=7) == el(W=None) == el(Y=None) == INV and el(e(T=0)) == OK
    many = e(T=4096, k=4)
    assert L.daq_experts_linear_workspace(many, 512, 512, 1, 0, C.byref(n)) == OK and n.value >= 4096 * 512
    big = dict(pl=many, N=512, K=512, ldx=512, ldy=512)
    assert el(ws=None, wn=0, **big) == el(wn=n.value - 1, **big) == el(ws=a + 4, **big) == WS
    wg = lambda pl=None, N=8, K=40, dy=a, x_=a, d=a, dt=0, ld=40, st=320, acc=0: L.daq_experts_weight_grad(pl or e(), N, K, dy, x_, d, dt, ld, st, acc, None)
    assert wg(N=0) == wg(K=0) == wg(dy=None) == wg(x_=None) == wg(d=None) == wg(dy=a + 1) == wg(x_=a + 1) == wg(d=odd) == wg(dt=2) == wg(ld=39) == wg(st=319) == wg(dt=1, acc=1) == INV
    assert wg(e(T=0), acc=1) == OK
    cb = lambda pl=None, y=a, dt=0, c=40, ldy=40, w_=a, out=a, ldo=40: L.daq_experts_combine(pl or e(), y, dt, c, ldy, w_, out, ldo, None)
    assert cb(y=None) == cb(out=None) == cb(y=odd) == cb(out=odd) == cb(w_=odd) == cb(dt=2) == cb(c=0) == cb(ldy=39) == cb(ldo=39) == INV and cb(e(T=0)) == OK
    cc = lambda pl=None, d=a, dt=0, c=40, ldo=40, y=a, ldy=40, w_=a, dy=a, lddy=40, dw=a: L.daq_experts_combine_backward(pl or e(), d, dt, c, ldo, y, ldy, w_, dy, lddy, dw, None)
    assert cc(d=None) == cc(d=odd) == cc(y=None) == cc(y=odd) == cc(dy=None) == cc(dy=odd) == cc(w_=odd) == cc(dw=odd) == cc(ldo=39) == cc(ldy=39) == cc(lddy=39) == cc(c=0) == INV
    for b in bad_plans:
        none = b is None
        for fn in ((lambda: L.daq_experts_quantize(b, a, 0, 40, 40, 0, a, a, None)), (lambda: L.daq_experts_matmul(b, 8, 40, a, 0, a, a, 0, 8, None)),
                   (lambda: L.daq_experts_linear(b, 8, 40, a, 0, 40, 0, a, a, 0, 8, a, 1 << 40, None)), (lambda: L.daq_experts_weight_grad(b, 8, 40, a, a, a, 0, 40, 320, 0, None)),
                   (lambda: L.daq_experts_combine(b, a, 0, 40, 40, a, a, 40, None)), (lambda: L.daq_experts_combine_backward(b, a, 0, 40, 40, a, 40, a, a, 40, a, None))):
            assert fn() == INV, none


def test_weight_gradients_without_tokens_read_the_table():
    L, a, odd = daq.lib(), 1 << 20, (1 << 20) + 2
    for table in (None, odd):
        plan = C.byref(daq.Experts(0, 2, 8, table, None, None))
        assert L.daq_experts_weight_grad(plan, 8, 40, None, None, a, 0, 40, 320, 0, None) == daq.ERR_INVALID_ARG
        assert L.daq_experts_weight_grad(plan, 8, 40, None, None, a, 0, 40, 320, 1, None) == daq.OK      # (adds nothing)


def test_buffers_off_the_gpu_are_refused(monkeypatch):
    """As weights read from a file are: their host addresses must not get to a kernel."""
    def reached(stream):
        raise RuntimeError("reached the call")

    monkeypatch.setattr(daq, "_stream", reached)
    q, x = daq.alloc_fp8(40, 70, device="cpu"), torch.zeros(4, 70)
    plan = daq.alloc_plan(4, 2, 4, device="cpu")
    ids = torch.zeros(4, 2, dtype=torch.int32)
    for call in (lambda: daq.fp8_quantize(x), lambda: daq.fp8_quantize_both(x), lambda: daq.fp8_quantize_weights(x), lambda: daq.fp8_dequantize(q), lambda: daq.fp8_matmul(q, q),
                 lambda: daq.fp8_linear(x, q), lambda: daq.route(x, 2), lambda: daq.route_backward(torch.zeros(4, 2), x, ids), lambda: daq.experts_plan(ids, 4),
                 lambda: daq.experts_quantize(x, plan), lambda: daq.experts_matmul(q, q, plan), lambda: daq.experts_linear(x, q, plan),
                 lambda: daq.experts_combine(torch.zeros(8, 70), plan), lambda: daq.experts_combine_backward(x, torch.zeros(8, 70), plan)):
        with pytest.raises(AssertionError):
            call()


def test_choices_of_forms():
    """Sizes that the measured rules are about."""
    L, n = daq.lib(), C.c_size_t(0)
    for M, K, one in ((1, 4096, True), (1, 16384, True), (1, 16385, False), (4, 4096, True), (4, 8192, False), (32, 512, True), (33, 128, False)):
        assert L.daq_fp8_linear_workspace(M, 2048, K, 1, 1, C.byref(n)) == daq.OK and (n.value == 0) == one, (M, K)
    assert L.daq_fp8_linear_workspace(1, 1 << 15, 128, 1, 1, C.byref(n)) == daq.OK and n.value > 0           # columns enough to fill the CUs with tiles
