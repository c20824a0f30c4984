"""Microscaled 4-bit products and 8-bit checkpoints on the GPU, through the binding, against the oracle in 64 bits.

Codes, scales and whole buffers are compared byte for byte.  Sums: every product is exact, each fp32 addition is off by at most 2^-23 of the
magnitudes added so far (to nearest or cut off), so a sum of n terms by at most n * 2^-23 * sum |products|; the matrix instructions add 64
(4-bit) or 16 (bfloat16) products as trees, so n counts steps, with ten additions inside and behind them.  A bfloat16 result adds 2^-8 of itself."""
import numpy as np
import pytest
import torch

from oracle import lowbits as ref
from paper_2102_04782_amd import binding as daq

pytestmark = pytest.mark.gpu

DT = [torch.float32, torch.bfloat16]
SIZES = [(1, 1), (1, 31), (3, 32), (31, 33), (32, 64), (33, 255), (64, 256), (65, 257), (7, 1000), (300, 130), (257, 515)]


def _x(rows, cols, dtype, seed, spread=6):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * torch.exp2(torch.randint(-spread, spread + 1, (rows, cols), generator=g).float())
    if rows > 1 and cols > 40:
        x[1, :32] = 0                                # a block of zeros
        x[0, 32:40] = 0.25 * torch.arange(8)          # ties, once the block's scale is a power of two above them
        x[0, 40:min(cols, 64)] = 1.0
    return x.to(dtype)


def _strided(x, dev, pad=5, first=3):
    """x inside a wider matrix of other values: rows start at any element."""
    wide = torch.full((x.shape[0], x.shape[1] + pad), 7.0, dtype=x.dtype, device=dev)
    v = wide[:, first:first + x.shape[1]]
    v.copy_(x)
    return v


def _np(t):
    return t.detach().cpu().to(torch.float64).numpy()


def _mx4(x, **kw):
    codes, byte = ref.mx4_codes(_np(x), **kw)
    return codes, byte


def _values(x, **kw):
    codes, byte = _mx4(x, **kw)
    return ref.mx4_values(codes, byte, x.shape[0] if kw.get("transpose") else x.shape[1])


def _saved(x, parts=1):
    codes, byte = ref.ckpt8_codes(_np(x), parts)
    return ref.ckpt8_values(codes, byte, x.shape[0], x.shape[1] // parts, parts)


@pytest.mark.parametrize("transpose", [False, True])
@pytest.mark.parametrize("stochastic", [False, True])
@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("rows,cols", SIZES)
def test_mx4_codes_scales_and_padding(rows, cols, dtype, stochastic, transpose):
    x = _x(rows, cols, dtype, rows * 1000 + cols)
    for src in (x.cuda(), _strided(x, "cuda")):
        out = daq.alloc_mx4(*((cols, rows) if transpose else (rows, cols)))
        out.buf.fill_(0xA5)                           # every byte, padding included, must come from the call
        q = daq.mx4_quantize(src, transpose=transpose, mode=daq.ROUND_STOCHASTIC if stochastic else daq.ROUND_NEAREST, seed=(5 << 40) + 77, out=out)
        codes, byte = _mx4(x, stochastic=stochastic, seed=(5 << 40) + 77, transpose=transpose)
        got, want = q.buf.cpu().numpy(), ref.mx4_buffer(codes, byte)
        off = daq.layout_mx4(q.rows, q.cols).off_scales
        assert np.array_equal(got[off:], want[off:])
        # a code of zero may carry either sign
        same = got[:off] == want[:off]
        lo, hi = got[:off] & 15, got[:off] >> 4
        zero = lambda a, b: (a == b) | ((a & 7 == 0) & (b & 7 == 0))
        assert np.all(same | (zero(lo, want[:off] & 15) & zero(hi, want[:off] >> 4)))
        for to in DT:
            v = daq.mx4_dequantize(q, dtype=to)
            assert np.array_equal(_np(v), ref.mx4_values(codes, byte, q.cols))


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("stochastic", [False, True])
def test_mx4_extremes(dtype, stochastic):
    x = torch.zeros(9, 96, dtype=dtype)
    big = torch.finfo(dtype).max
    x[0, 0], x[0, 33], x[1, 5] = big, -big, 2.0 ** -126
    x[2, 7], x[2, 40] = 2.0 ** -133, 2.0 ** -128          # below the normal range
    x[3, 3], x[4, 50], x[5, 70] = float("nan"), float("inf"), float("-inf")
    x[6] = torch.tensor([2.0 ** -129 * (i % 13) for i in range(96)])
    x[7, 31], x[7, 0] = 3.0, 6.0
    x[8, :8] = torch.tensor([6.0, 6.5, 7.0, 7.5, 5.0, 4.999, 1e-30, -7.9])
    for transpose in (False, True):
        q = daq.mx4_quantize(x.cuda(), transpose=transpose, mode=int(stochastic), seed=3)
        codes, byte = _mx4(x, stochastic=stochastic, seed=3, transpose=transpose)
        for to in DT:
            # (2^128, which stochastic rounding can make of the largest values, is an infinity in either type)
            with np.errstate(over="ignore"):
                want = ref.mx4_values(codes, byte, q.cols).astype(np.float32)
            assert np.array_equal(_np(daq.mx4_dequantize(q, dtype=to)), want, equal_nan=True)


MATMUL = [(1, 1, 1), (1, 33, 65), (1, 512, 2048), (2, 70, 300), (5, 64, 256), (13, 100, 1030), (32, 256, 512), (33, 129, 64), (40, 2049, 96), (64, 64, 4096),
          (100, 260, 700), (255, 257, 513), (256, 256, 256), (300, 600, 320), (513, 511, 1024), (1030, 770, 200)]


def _bound(steps, absolute, exact, dtype):
    return (steps + 10) * 2.0 ** -23 * absolute + (2.0 ** -8 * np.abs(exact) if dtype == torch.bfloat16 else 0) + 1e-40


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("M,N,K", MATMUL)
def test_mx4_matmul(M, N, K, dtype):
    a, b = _x(M, K, torch.bfloat16, M + K), _x(N, K, torch.float32, N + 3 * K)
    va, vb = _values(a), _values(b)
    exact, absolute = va @ vb.T, np.abs(va) @ np.abs(vb).T
    qa, qb = daq.mx4_quantize(a.cuda()), daq.mx4_quantize(b.cuda())
    wide = torch.full((M, N + 7), 55.0, dtype=dtype, device="cuda")
    for out in (torch.full((M, N), float("nan"), dtype=dtype, device="cuda"), wide[:, 3:3 + N]):
        got = _np(daq.mx4_matmul(qa, qb, out=out))
        assert np.all(np.abs(got - exact) <= _bound(-(-K // 64), absolute, exact, dtype))
    assert bool((wide[:, :3] == 55).all()) and bool((wide[:, 3 + N:] == 55).all())     # nothing beside the result


@pytest.mark.parametrize("stochastic", [False, True])
@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("M,N,K", MATMUL)
def test_mx4_linear(M, N, K, dtype, stochastic):
    x, w = _x(M, K, dtype, M + 2 * K), _x(N, K, torch.bfloat16, N + 5 * K)
    vx, vw = _values(x, stochastic=stochastic, seed=9), _values(w)
    exact, absolute = vx @ vw.T, np.abs(vx) @ np.abs(vw).T
    qw = daq.mx4_quantize(w.cuda())
    for src in (x.cuda(), _strided(x, "cuda")):
        for to in DT:
            got = _np(daq.mx4_linear(src, qw, mode=int(stochastic), seed=9, dtype=to))
            assert np.all(np.abs(got - exact) <= _bound(-(-K // 64), absolute, exact, to))


def test_mx4_linear_data_gradient_is_the_product_with_the_weights_by_columns():
    dy, w = _x(70, 200, torch.float32, 1), _x(200, 330, torch.bfloat16, 2)
    vy, vw = _values(dy, stochastic=True, seed=4), _values(w, transpose=True)       # vw [330, 200]
    exact, absolute = vy @ vw.T, np.abs(vy) @ np.abs(vw).T
    got = _np(daq.mx4_linear(dy.cuda(), daq.mx4_quantize(w.cuda(), transpose=True), mode=daq.ROUND_STOCHASTIC, seed=4))
    assert got.shape == (70, 330) and np.all(np.abs(got - exact) <= _bound(4, absolute, exact, torch.float32))


@pytest.mark.parametrize("M", [1, 3, 40, 300])
def test_mx4_linear_keeps_a_bad_row_to_itself(M):
    x, w = _x(M, 300, torch.bfloat16, 11), _x(150, 300, torch.bfloat16, 12)
    w[149, 299] = float("inf")
    x[0, 7] = float("nan")
    got = _np(daq.mx4_linear(x.cuda(), daq.mx4_quantize(w.cuda())))
    assert np.isnan(got[0]).all() and np.isnan(got[:, 149]).all() and np.isfinite(got[1:, :149]).all()


def test_no_rows():
    w = daq.mx4_quantize(_x(64, 96, torch.bfloat16, 1).cuda())
    x = torch.empty(0, 96, dtype=torch.bfloat16, device="cuda")
    assert daq.mx4_linear(x, w).shape == (0, 64)
    assert daq.mx4_dequantize(daq.mx4_quantize(x)).shape == (0, 96)
    assert daq.mx4_dequantize(daq.mx4_quantize(x, transpose=True)).shape == (96, 0)
    assert daq.ckpt8_restore(daq.ckpt8_save(x)).shape == (0, 96)
    y, c = daq.ckpt8_act_forward(x, daq.ACT_SILU, gated=True)
    assert y.shape == (0, 48) and daq.ckpt8_act_backward(y, c, daq.ACT_SILU).shape == (0, 96)
    dy = torch.empty(0, 40, dtype=torch.bfloat16, device="cuda")
    assert bool((daq.ckpt8_weight_grad(dy, daq.ckpt8_save(x)) == 0).all())
    kept = torch.full((40, 96), 3.0, device="cuda")
    daq.ckpt8_weight_grad(dy, daq.ckpt8_save(x), out=kept, accumulate=True)
    assert bool((kept == 3).all())


@pytest.mark.parametrize("parts", [1, 2])
@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("rows,cols", SIZES + [(3, 5000)])
def test_ckpt8_codes_scales_and_padding(rows, cols, dtype, parts):
    x = _x(rows, parts * cols, dtype, rows + cols)
    codes, byte = ref.ckpt8_codes(_np(x), parts)
    n, L = rows * parts, daq.layout_ckpt8(rows, cols, parts)
    want = ref.ckpt8_buffer(codes, byte)
    for src in (x.cuda(), _strided(x, "cuda")):
        c = daq.alloc_ckpt8(rows, cols, parts)
        c.buf.fill_(0xA5)
        daq.ckpt8_save(src, parts, out=c)
        got = c.buf.cpu().numpy()
        assert np.array_equal(got[:n * L.pitch], want[:n * L.pitch])
        assert np.array_equal(got[L.off_scales:L.off_scales + n * L.pitch // 32], want[L.off_scales:L.off_scales + n * L.pitch // 32])
        wide = torch.full((rows, parts * cols + 9), 55.0, dtype=dtype, device="cuda")
        for out in (torch.empty_like(src), wide[:, 4:4 + parts * cols]):
            assert np.array_equal(_np(daq.ckpt8_restore(c, out=out)), ref.ckpt8_values(codes, byte, rows, cols, parts))
        assert bool((wide[:, :4] == 55).all()) and bool((wide[:, 4 + parts * cols:] == 55).all())


@pytest.mark.parametrize("dtype", DT)
def test_ckpt8_extremes(dtype):
    x = torch.zeros(7, 96, dtype=dtype)
    big = torch.finfo(dtype).max
    x[0, 0], x[0, 33], x[1, 5] = big, -big, 2.0 ** -126
    x[2, 7], x[2, 40] = 2.0 ** -133, 2.0 ** -128
    x[3, 3], x[4, 50], x[5, 70] = float("nan"), float("inf"), float("-inf")
    x[6, :9] = torch.tensor([127.0, 127.5, -127.5, 127.75, 0.5, 1.5, -2.5, 126.5, -0.5])
    assert np.array_equal(_np(daq.ckpt8_restore(daq.ckpt8_save(x.cuda()))), _saved(x), equal_nan=True)


ACTS = [("silu", daq.ACT_SILU), ("gelu", daq.ACT_GELU)]


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("name,act", ACTS)
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 32), (5, 31), (33, 100), (64, 257), (3, 4100)])
def test_act_forward_and_backward(rows, cols, name, act, dtype, gated):
    """fp32 formulas: the exponential and the error function are good to some units in the last place, their sums and products to a unit
    each; x times an error of the sigmoid or of Phi (an absolute one, at most 8 * 2^-24) bounds f, and as much times 1 + |x| its slope."""
    parts = 2 if gated else 1
    h, dy = _x(rows, parts * cols, dtype, rows + cols, 2), _x(rows, cols, dtype, rows + cols + 1, 2)
    one = 2.0 ** -8 if dtype == torch.bfloat16 else 0.0
    eps = 8 * 2.0 ** -24
    hv, hs, d = _np(h), _saved(h, parts), _np(dy)
    f, _ = ref.act(hv[:, :cols], name)
    fs, slope = ref.act(hs[:, :cols], name)
    u, us = (hv[:, cols:], hs[:, cols:]) if gated else (1.0, 1.0)
    for strided in (False, True):
        src = _strided(h, "cuda") if strided else h.cuda()
        y, kept = daq.ckpt8_act_forward(src, act, gated=gated)
        assert y.dtype == dtype and np.all(np.abs(_np(y) - f * u) <= eps * np.abs(hv[:, :cols] * u) + one * np.abs(f * u) + 1e-37)
        assert np.array_equal(_np(daq.ckpt8_restore(kept)), hs)
        wide = torch.full((rows, parts * cols + 6), 55.0, dtype=dtype, device="cuda")
        yk = daq.alloc_ckpt8(rows, cols)
        dh = daq.ckpt8_act_backward(_strided(dy, "cuda") if strided else dy.cuda(), kept, act, out=wide[:, 2:2 + parts * cols], y_ckpt=yk)
        got, want = _np(dh), d * us * slope
        tol = eps * np.abs(d * us) * (1 + np.abs(hs[:, :cols])) ** 2
        assert np.all(np.abs(got[:, :cols] - want) <= tol + one * np.abs(want) + 1e-37)
        if gated:
            assert np.all(np.abs(got[:, cols:] - d * fs) <= eps * np.abs(d * hs[:, :cols]) + one * np.abs(d * fs) + 1e-37)
        assert bool((wide[:, :2] == 55).all()) and bool((wide[:, 2 + parts * cols:] == 55).all())
        # the output saved again: within a code of what the oracle's value is, and the same gradient without it
        ycodes, ybyte = ref.ckpt8_codes(fs * us)
        step = np.repeat(np.exp2(ybyte - 127.0), 32, axis=1)[:, :cols]
        assert np.all(np.abs(_np(daq.ckpt8_restore(yk)) - fs * us) <= 1.01 * step + eps * np.abs(hs[:, :cols] * us))
        again = daq.ckpt8_act_backward(dy.cuda(), kept, act)
        assert torch.equal(again, dh)


@pytest.mark.parametrize("name,act", ACTS)
def test_act_gradient_against_differences(name, act):
    """(f(x + h) - f(x - h)) / 2h of the forward pass at points that 8 bits hold exactly; h = 2^-6: h^2 / 6 times a third derivative below 2,
    and fp32 rounding of f over h."""
    codes = torch.arange(-127, 128, dtype=torch.float32)
    x = torch.zeros(8, 32)
    x.view(-1)[:255] = codes / 16
    x[:, 31] = 127 / 16                                  # the scale of every block
    x, one = x.cuda(), torch.ones(8, 32, device="cuda")
    h = 2.0 ** -6
    up, _ = daq.ckpt8_act_forward(x + h, act)
    down, _ = daq.ckpt8_act_forward(x - h, act)
    _, kept = daq.ckpt8_act_forward(x, act)
    assert torch.equal(daq.ckpt8_restore(kept), x)
    slope = daq.ckpt8_act_backward(one, kept, act)
    assert float((slope - (up - down) / (2 * h)).abs().max()) <= h * h / 3 + 16 * 8 * 2.0 ** -24 / h


WGRAD = [(1, 1, 1), (1, 40, 70), (7, 33, 31), (16, 32, 32), (64, 128, 256), (100, 130, 260), (257, 300, 129), (1000, 64, 64), (513, 520, 400), (2048, 96, 1000)]


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("M,N,K", WGRAD)
def test_weight_grad(M, N, K, dtype):
    dy, x = _x(M, N, dtype, M + N), _x(M, K, torch.bfloat16, M + 7 * K)
    xs, d = _saved(x), _np(dy)
    exact, absolute = d.T @ xs, np.abs(d.T) @ np.abs(xs)
    kept = daq.ckpt8_save(x.cuda())
    bound = _bound((3 if dtype == torch.float32 else 1) * -(-M // 16), absolute, exact, torch.float32)
    for src in (dy.cuda(), _strided(dy, "cuda")):
        got = daq.ckpt8_weight_grad(src, kept)
        assert np.all(np.abs(_np(got) - exact) <= bound)
        wide = torch.full((N, K + 5), 2.0, device="cuda")
        daq.ckpt8_weight_grad(src, kept, out=wide[:, 1:1 + K], accumulate=True)
        assert bool((wide[:, 0] == 2).all()) and bool((wide[:, 1 + K:] == 2).all())
        assert np.all(np.abs(_np(wide[:, 1:1 + K]) - 2 - exact) <= bound + 2.0 ** -22 * (2 + np.abs(exact)))
        assert torch.equal(got, daq.ckpt8_weight_grad(src, kept))       # the same bits every time


def test_weight_grad_against_differences():
    """The loss sum(dy * (x^ w^T)) is linear in the weights: a step in one of them changes it by its gradient."""
    g = torch.Generator().manual_seed(3)
    x = daq.ckpt8_save(torch.randn(50, 40, generator=g).cuda())
    xs, dy = daq.ckpt8_restore(x).double(), torch.randn(50, 24, generator=g).cuda()
    dW, w = daq.ckpt8_weight_grad(dy, x), torch.randn(24, 40, generator=g).cuda().double()
    loss = lambda w: float((dy.double() * (xs @ w.t().contiguous())).sum())
    for n, k in [(0, 0), (5, 31), (23, 39), (11, 32)]:
        up, down = w.clone(), w.clone()
        up[n, k] += 0.5
        down[n, k] -= 0.5
        assert abs(loss(up) - loss(down) - float(dW[n, k])) <= 14 * 2.0 ** -23 * float((dy[:, n].abs().double() * xs[:, k].abs()).sum()) + 1e-9


@pytest.mark.parametrize("dtype", DT)
def test_weight_grad_keeps_what_is_not_finite_to_itself(dtype):
    dy, x = _x(100, 40, dtype, 1), _x(100, 70, torch.bfloat16, 2)
    dy[3, 5], dy[99, 39], x[50, 33] = float("nan"), float("inf"), float("inf")
    got = _np(daq.ckpt8_weight_grad(dy.cuda(), daq.ckpt8_save(x.cuda())))
    bad = np.zeros((40, 70), bool)
    bad[5] = bad[39] = True
    bad[:, 32:64] = True
    assert np.isnan(got[5]).all() and np.isnan(got[:, 32:64]).all() and not np.isfinite(got[39]).any() and np.isfinite(got[~bad]).all()


def test_calls_on_another_stream():
    side = torch.cuda.Stream()
    x, w = _x(200, 512, torch.bfloat16, 1).cuda(), _x(300, 512, torch.bfloat16, 2).cuda()
    dy = _x(200, 300, torch.bfloat16, 3).cuda()
    want = daq.mx4_linear(x, daq.mx4_quantize(w)), daq.ckpt8_weight_grad(dy, daq.ckpt8_save(x))
    out, dW = torch.empty_like(want[0]), torch.empty_like(want[1])
    qw, kept = daq.alloc_mx4(300, 512), daq.alloc_ckpt8(200, 512)
    ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    daq.mx4_quantize(w, out=qw, stream=side)
    daq.mx4_linear(x, qw, out=out, workspace=ws, stream=side)
    daq.ckpt8_save(x, out=kept, stream=side)
    daq.ckpt8_weight_grad(dy, kept, out=dW, workspace=ws, stream=side)
    side.synchronize()
    assert torch.equal(out, want[0]) and torch.equal(dW, want[1])


# sizes of the larger forms: the reference runs in fp64 on the GPU, on the values the packed operands hold (compared with the oracle above)
@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("M,N,K", [(2100, 2050, 260), (4100, 4097, 520), (2300, 3900, 1030), (5000, 4000, 64), (16500, 40, 300)])
def test_mx4_matmul_large(M, N, K, dtype):
    a, b = daq.mx4_quantize(_x(M, K, torch.bfloat16, 5).cuda()), daq.mx4_quantize(_x(N, K, torch.bfloat16, 6).cuda())
    va, vb = daq.mx4_dequantize(a).double(), daq.mx4_dequantize(b).double()
    exact, absolute = va @ vb.t().contiguous(), va.abs() @ vb.t().abs().contiguous()
    got = daq.mx4_matmul(a, b, dtype=dtype).double()
    bound = (-(-K // 64) + 10) * 2.0 ** -23 * absolute + (2.0 ** -8 * exact.abs() if dtype == torch.bfloat16 else 0)
    assert bool(((got - exact).abs() <= bound).all())


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("M,N,K,pad", [(700, 4104, 4100, 0), (130, 4112, 4096, 8), (4099, 520, 1000, 16), (5000, 264, 96, 0), (64, 2048, 2080, 8), (20000, 40, 33, 24)])
def test_weight_grad_large(M, N, K, pad, dtype):
    """Rows of dY that begin at 16-byte places, in a matrix of their own or (pad) in a wider one."""
    wide = _x(M, N + pad, dtype, 7).cuda()
    dy, kept = wide[:, pad:], daq.ckpt8_save(_x(M, K, torch.bfloat16, 8).cuda())
    xs = daq.ckpt8_restore(kept).double()
    d = dy.double().t().contiguous()
    exact, absolute = d @ xs, d.abs() @ xs.abs()
    got = daq.ckpt8_weight_grad(dy, kept)
    steps = (3 if dtype == torch.float32 else 1) * -(-M // 16)
    assert bool(((got.double() - exact).abs() <= (steps + 10) * 2.0 ** -23 * absolute + 1e-40).all())
    assert torch.equal(got, daq.ckpt8_weight_grad(dy, kept))


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("M,N,K,pad", [(300, 1, 70, 0), (9001, 70, 33, 0), (4100, 65, 129, 2), (17, 1030, 1000, 1), (271, 2, 2, 0), (3001, 610, 1101, 2), (5001, 520, 400, 8),
                                       (40, 1500, 1400, 0), (300, 1101, 1090, 1), (2050, 1032, 1000, 0)])
def test_weight_grad_forms(M, N, K, pad, dtype):
    """Both sides of the sizes at which the products stop reading their operands as they are, and added to what is there."""
    wide = _x(M, N + pad, dtype, 11).cuda()
    dy, kept = wide[:, pad:], daq.ckpt8_save(_x(M, K, torch.bfloat16, 12).cuda())
    xs = daq.ckpt8_restore(kept).double()
    d = dy.double().t().contiguous()
    exact, absolute = d @ xs, d.abs() @ xs.abs()
    got = daq.ckpt8_weight_grad(dy, kept)
    steps = (3 if dtype == torch.float32 else 1) * -(-M // 16)
    assert bool(((got.double() - exact).abs() <= (steps + 10) * 2.0 ** -23 * absolute + 1e-40).all())
    kept_out = torch.full((N, K + 3), 2.0, device="cuda")
    daq.ckpt8_weight_grad(dy, kept, out=kept_out[:, 1:1 + K], accumulate=True)
    assert torch.equal(kept_out[:, 1:1 + K], got + 2) and bool((kept_out[:, 0] == 2).all()) and bool((kept_out[:, 1 + K:] == 2).all())


def test_offsets_beyond_32_bits():
    """More than 2^31 elements, twice as many bytes: the last rows are what they are alone."""
    rows, cols, tail = 66000, 32800, 40
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    x.normal_()
    last = x[-tail:].contiguous()
    assert torch.equal(daq.ckpt8_restore(daq.ckpt8_save(x), dtype=torch.bfloat16)[-tail:], daq.ckpt8_restore(daq.ckpt8_save(last), dtype=torch.bfloat16))
    q = daq.mx4_quantize(x)
    assert torch.equal(daq.mx4_dequantize(q, dtype=torch.bfloat16)[-tail:], daq.mx4_dequantize(daq.mx4_quantize(last), dtype=torch.bfloat16))
    del q
    w = daq.mx4_quantize(x[:64].contiguous())
    assert torch.equal(daq.mx4_linear(x, w)[-tail:], daq.mx4_linear(last, w))
    qt = daq.mx4_dequantize(daq.mx4_quantize(x, transpose=True), dtype=torch.bfloat16)      # blocks of 32 rows: 66000 = 2062 * 32 + 16
    assert torch.equal(qt[:, -16:], daq.mx4_dequantize(daq.mx4_quantize(x[-16:].contiguous(), transpose=True), dtype=torch.bfloat16))
    del qt
    y, kept = daq.ckpt8_act_forward(x, daq.ACT_SILU, gated=True)
    y1, kept1 = daq.ckpt8_act_forward(last, daq.ACT_SILU, gated=True)
    assert torch.equal(y[-tail:], y1)
    assert torch.equal(daq.ckpt8_act_backward(y, kept, daq.ACT_SILU)[-tail:], daq.ckpt8_act_backward(y1, kept1, daq.ACT_SILU))
    dy = torch.zeros(rows, 8, dtype=torch.bfloat16, device="cuda")
    dy[-tail:] = 1
    got, want = daq.ckpt8_weight_grad(dy, daq.ckpt8_save(x)), daq.ckpt8_weight_grad(dy[-tail:].contiguous(), daq.ckpt8_save(last))
    assert bool(((got - want).abs() <= 13 * 2.0 ** -23 * daq.ckpt8_restore(daq.ckpt8_save(last)).abs().sum(0)).all())


def test_a_captured_training_step_replays():
    """One graph of every operator, replayed with other work between, against the eager calls on the same inputs."""
    from paper_2102_04782_amd.feed_forward import FeedForward

    block = FeedForward(320, 480, seed=4)
    x, dy = _x(300, 320, torch.bfloat16, 1, 1).cuda(), _x(300, 320, torch.bfloat16, 2, 1).cuda()

    def step():
        y, saved = block.forward(x)
        return (y, *block.backward(dy, saved, seed=5))

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for i in range(4):
        x.copy_(_x(300, 320, torch.bfloat16, 10 + i, 1))
        dy.copy_(_x(300, 320, torch.bfloat16, 20 + i, 1))
        want = [t.clone() for t in step()]
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_feed_forward_block_against_its_definition():
    """The block's outputs and gradients, in fp64, from the values that its packed weights and checkpoints hold.  Each value of the
    chain below was rounded once to bfloat16 (2^-8) and, going into a product, to 4 bits like the oracle's: the products are compared one
    by one, on the values the block itself passes on."""
    from paper_2102_04782_amd.feed_forward import FeedForward

    block = FeedForward(160, 224, seed=6)
    x, dy = _x(90, 160, torch.bfloat16, 3, 1).cuda(), _x(90, 160, torch.bfloat16, 4, 1).cuda()
    y, saved = block.forward(x)
    dx, dw_in, dw_out = block.backward(dy, saved, seed=7)
    w_in, w_out = _values(block.w_in.cpu()), _values(block.w_out.cpu())
    h = _values(x.cpu()) @ w_in.T
    a = ref.act(h[:, :224], "silu")[0] * h[:, 224:]
    hs = _np(daq.ckpt8_restore(saved.h))
    assert np.array_equal(_np(daq.ckpt8_restore(saved.x)), _saved(x.cpu()))
    # h was rounded to bfloat16 and then to 8 bits: half a step of a 64th of its block's largest value at most (a whole one at the very top)
    top = np.repeat(np.abs(h).reshape(90, -1, 32).max(axis=2), 32, axis=1)
    assert np.all(np.abs(hs - h) <= (2.0 ** -8 + 2.0 ** -6) * top + 1e-6)
    # the output against exact products of unrounded activations: 4-bit rounding of a moves each by an eighth of its magnitude or, among the
    # small ones of a block, by a quarter of an element; the block's rms error stays below a fifth of the output's
    want = a @ w_out.T
    assert np.linalg.norm(_np(y) - want) <= 0.2 * np.linalg.norm(want)
    # gradients of the weights: exact in what was kept
    da = _values(dy.cpu(), stochastic=True, seed=14) @ _values(block.w_out.cpu(), transpose=True).T
    f, slope = ref.act(hs[:, :224], "silu")
    a8 = f * hs[:, 224:]
    got, exact = _np(dw_out), _np(dy).T @ a8
    assert np.linalg.norm(got - exact) <= 2.0 ** -6 * np.linalg.norm(exact)
    dh = np.concatenate((da * hs[:, 224:] * slope, da * f), axis=1)
    exact = dh.T @ _saved(x.cpu())
    assert np.linalg.norm(_np(dw_in) - exact) <= 2.0 ** -6 * np.linalg.norm(exact)      # (da and dh rounded to bfloat16)
    exact = dh @ w_in
    assert np.linalg.norm(_np(dx) - exact) <= 0.35 * np.linalg.norm(exact)                # dh in 4 bits, stochastically; w by columns


def test_the_example_learns(capsys):
    from paper_2102_04782_amd import feed_forward

    feed_forward.main(steps=41)
    said = [float(l.split()[-1]) for l in capsys.readouterr().out.splitlines() if l.startswith("step")]
    assert said[-1] < 0.75 * said[0]


def test_results_and_workspaces_of_another_stream():
    """Nothing is given: what a call allocates belongs to its stream, also while the current stream takes and fills memory of the same sizes."""
    side = torch.cuda.Stream()
    x, w, dy = _x(500, 1024, torch.bfloat16, 1).cuda(), _x(700, 1024, torch.bfloat16, 2).cuda(), _x(500, 700, torch.float32, 3).cuda()
    h = _x(500, 1400, torch.bfloat16, 4).cuda()
    y, kept = daq.ckpt8_act_forward(h, daq.ACT_GELU, gated=True)
    want = (daq.mx4_linear(x, daq.mx4_quantize(w)), daq.ckpt8_weight_grad(dy, daq.ckpt8_save(x)), y, daq.ckpt8_act_backward(y, kept, daq.ACT_GELU))
    torch.cuda.synchronize()
    for _ in range(20):
        a = daq.mx4_linear(x, daq.mx4_quantize(w, stream=side), stream=side)
        b = daq.ckpt8_weight_grad(dy, daq.ckpt8_save(x, stream=side), stream=side)
        c, k = daq.ckpt8_act_forward(h, daq.ACT_GELU, gated=True, stream=side)
        d = daq.ckpt8_act_backward(c, k, daq.ACT_GELU, stream=side)
        for n in (1 << 18, 1 << 20, 3 << 20):
            torch.empty(n, dtype=torch.uint8, device="cuda").fill_(0xEE)
        side.synchronize()
        assert all(torch.equal(p, q) for p, q in zip((a, b, c, d), want))


@pytest.mark.parametrize("gated", [False, True])
def test_gelu_keeps_its_tail(gated):
    """Relative to the value itself where Phi(x) is far below one.  With u = 2^-24: x / sqrt 2 is off by 1.5 u (its constant and its rounding), which
    the complementary error function makes x^2 + 1 times as much of, its own error is 32 u at most, and six products and sums follow; the
    exponential's argument is off by 1.5 u of x^2 / 2.  Where the function leaves the normal range, by one of the smallest normal values."""
    u = 2.0 ** -24
    x = torch.cat((torch.linspace(-9, -3, 40 * 64), -torch.tensor([9.5, 10, 11, 12, 12.5, 13, 14, 20, 40, 1e4] * 6 + [9.0] * 4))).view(41, 64)
    parts = 2 if gated else 1
    h = torch.cat([x, torch.linspace(0.5, 3, x.numel()).view_as(x)][:parts], 1)
    dy = torch.linspace(-2, 1, x.numel()).view_as(x)
    y, kept = daq.ckpt8_act_forward(h.cuda(), daq.ACT_GELU, gated=gated)
    hv, hs, d = _np(h), _saved(h, parts), _np(dy)
    up, us = (hv[:, 64:], hs[:, 64:]) if gated else (1.0, 1.0)

    def bound(x, size):
        with np.errstate(over="ignore"):
            return (1.5 * x * x + 40) * u * size

    want = ref.act(hv[:, :64], "gelu")[0] * up
    assert np.all(np.abs(_np(y) - want) <= bound(hv[:, :64], np.abs(want)) + np.abs(hv[:, :64] * up) * 2.0 ** -126)
    yk = daq.alloc_ckpt8(41, 64)
    dh = _np(daq.ckpt8_act_backward(dy.cuda(), kept, daq.ACT_GELU, y_ckpt=yk))
    g = hs[:, :64]
    f, slope = ref.act(g, "gelu")
    density = np.exp(-g * g / 2) / np.sqrt(2 * np.pi)
    terms = np.abs(slope - g * density) + np.abs(g) * density
    assert np.all(np.abs(dh[:, :64] - d * us * slope) <= np.abs(d * us) * (bound(g, terms) + (1 + np.abs(g)) * 2.0 ** -126) + 2.0 ** -126)
    if gated:
        assert np.all(np.abs(dh[:, 64:] - d * f) <= bound(g, np.abs(d * f)) + np.abs(d * g) * 2.0 ** -126 + 2.0 ** -126)
    step = np.repeat(np.exp2(ref.ckpt8_codes(f * us)[1] - 127.0), 32, axis=1)
    assert np.all(np.abs(_np(daq.ckpt8_restore(yk)) - f * us) <= 1.01 * step)


def test_packed_buffers_are_looked_at_before_a_launch():
    """A buffer on the host, one of fewer bytes than its sizes need, one whose bytes are not in a row; a workspace on the host or not in a row."""
    x, dy = _x(40, 300, torch.bfloat16, 1).cuda(), _x(40, 50, torch.bfloat16, 2).cuda()
    w, h, kept = daq.mx4_quantize(_x(50, 300, torch.bfloat16, 3).cuda()), daq.ckpt8_save(dy), daq.ckpt8_save(x)

    def broken(q):
        for buf in (q.buf.cpu(), q.buf[:-1], q.buf[:1].expand(q.buf.numel()), torch.empty(2 * q.buf.numel(), dtype=torch.uint8, device="cuda")[::2]):
            yield type(q)(buf, *[getattr(q, f) for f in ("rows", "cols", "parts") if hasattr(q, f)])

    calls = [(w, lambda q: daq.mx4_dequantize(q)), (w, lambda q: daq.mx4_linear(x, q)), (w, lambda q: daq.mx4_matmul(q, w)), (w, lambda q: daq.mx4_matmul(w, q)),
             (w, lambda q: daq.mx4_quantize(_x(50, 300, torch.bfloat16, 3).cuda(), out=q)), (h, lambda q: daq.ckpt8_restore(q)), (h, lambda q: daq.ckpt8_save(dy, out=q)),
             (h, lambda q: daq.ckpt8_act_forward(dy, daq.ACT_SILU, ckpt=q)), (h, lambda q: daq.ckpt8_act_backward(dy, q, daq.ACT_SILU)),
             (h, lambda q: daq.ckpt8_act_backward(dy, h, daq.ACT_SILU, y_ckpt=q)), (kept, lambda q: daq.ckpt8_weight_grad(dy, q))]
    for good, call in calls:
        call(good)
        for q in broken(good):
            with pytest.raises(AssertionError):
                call(q)
    for ws in (torch.empty(1 << 20, dtype=torch.uint8), torch.empty(1, dtype=torch.uint8, device="cuda").expand(1 << 20)):
        for call in (lambda: daq.mx4_linear(x, w, workspace=ws), lambda: daq.mx4_matmul(w, w, workspace=ws), lambda: daq.ckpt8_weight_grad(dy, kept, workspace=ws)):
            with pytest.raises(AssertionError):
                call()
    torch.cuda.synchronize()


# weight gradients on tiles, by form (few_bits_plans.hip holds that they are of it); first: the column of a wider matrix at which dY begins
LARGE_TILES = [(700, 4103, 4100, 0, 0), (700, 4104, 4100, 1, 8), (600, 4096, 8200, 0, 0), (9000, 2049, 2100, 0, 0), (6000, 1536, 1300, 0, 0), (1111, 3000, 900, 0, 0)]


@pytest.mark.parametrize("M,N,K,first,pad", LARGE_TILES)
def test_weight_grad_on_tiles(M, N, K, first, pad):
    wide = _x(M, N + pad, torch.bfloat16, 21).cuda()
    dy, kept = wide[:, first:first + N], daq.ckpt8_save(_x(M, K, torch.bfloat16, 22).cuda())
    xs = daq.ckpt8_restore(kept).double()
    d = dy.double().t().contiguous()
    exact, absolute = d @ xs, d.abs() @ xs.abs()
    got = daq.ckpt8_weight_grad(dy, kept)
    assert bool(((got.double() - exact).abs() <= (-(-M // 16) + 10) * 2.0 ** -23 * absolute + 1e-40).all())
    out = torch.full((N, K + 3), 2.0, device="cuda")
    daq.ckpt8_weight_grad(dy, kept, out=out[:, 1:1 + K], accumulate=True)
    assert torch.equal(out[:, 1:1 + K], got + 2) and bool((out[:, 0] == 2).all()) and bool((out[:, 1 + K:] == 2).all())


@pytest.mark.parametrize("dtype,M,N,K", [(torch.float32, 300, 1101, 1090), (torch.float32, 3001, 610, 1101), (torch.float32, 700, 4103, 4100),
                                         (torch.bfloat16, 300, 1101, 1090), (torch.bfloat16, 3001, 610, 1101), (torch.bfloat16, 1111, 3000, 900),
                                         (torch.bfloat16, 2050, 1032, 1000), (torch.bfloat16, 700, 4103, 4100), (torch.bfloat16, 700, 4104, 4100),
                                         (torch.bfloat16, 9000, 2049, 2100), (torch.bfloat16, 6000, 1536, 1300)])
def test_weight_grad_on_tiles_keeps_what_is_not_finite_to_itself(dtype, M, N, K):
    """In the first and last columns, where reads pass a row's end, and in the first and last tokens, where they pass the last row's."""
    dy, x = _x(M, N, dtype, 31), _x(M, K, torch.bfloat16, 32)
    dy[0, 0], dy[M - 1, N - 1], dy[M // 2, N // 2], x[M - 1, K - 1] = float("nan"), float("inf"), float("-inf"), float("inf")
    got = daq.ckpt8_weight_grad(dy.cuda(), daq.ckpt8_save(x.cuda()))
    k0 = (K - 1) // 32 * 32
    bad = torch.zeros(N, K, dtype=torch.bool, device="cuda")
    bad[[0, N // 2, N - 1]] = True
    bad[:, k0:] = True
    assert bool(got[0].isnan().all()) and bool(got[:, k0:].isnan().all()) and not bool(got[bad].isfinite().any()) and bool(got[~bad].isfinite().all())


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("name,act", ACTS)
def test_large_activations_are_their_parts(name, act, dtype, gated):
    """From 48 MiB on the kernels pass the caches by: every value and every code as of the two halves, which do not (and are compared with
    the oracle at their small sizes).  Rows of any length that begin at any element."""
    parts, cols = (2, 1003) if gated else (1, 1003)
    rows = (51 << 20) // (parts * cols * (2 if dtype == torch.bfloat16 else 4)) + 1
    half = rows // 2 + 3
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    h = torch.randn(rows, parts * cols + 3, generator=g, device="cuda").mul_(3).to(dtype)[:, 1:1 + parts * cols]
    dy = torch.randn(rows, cols + 1, generator=g, device="cuda").to(dtype)[:, :cols]

    def run(rs):
        y, kept = daq.ckpt8_act_forward(h[rs], act, gated=gated)
        yk = daq.alloc_ckpt8(*y.shape)
        dh = daq.ckpt8_act_backward(dy[rs], kept, act, y_ckpt=yk)
        assert torch.equal(daq.ckpt8_act_backward(dy[rs], kept, act), dh)
        return y, dh, daq.ckpt8_restore(kept), daq.ckpt8_restore(yk), daq.ckpt8_restore(kept, dtype=torch.bfloat16)

    whole = run(slice(None))
    for rs in (slice(0, half), slice(half, rows)):
        for a, b in zip(whole, run(rs)):
            assert bool(b.isfinite().all()) and torch.equal(a[rs], b)
    saved = daq.ckpt8_save(h, parts)
    assert torch.equal(daq.ckpt8_restore(saved), whole[2])
    for rs in (slice(0, half), slice(half, rows)):
        assert torch.equal(daq.ckpt8_restore(daq.ckpt8_save(h[rs], parts)), whole[2][rs])


def test_feed_forward_block_product_by_product(monkeypatch):
    """Every call of a training step against the oracle on the values that the block passes to it: products elementwise from their own operands, in
    the rounding and with the draws that each is meant to have, and both gradients of the weights."""
    from paper_2102_04782_amd import feed_forward as ff

    products, grads = [], []
    linear, weight_grad = daq.mx4_linear, daq.ckpt8_weight_grad

    def recording_linear(x, w, mode=daq.ROUND_NEAREST, seed=0, **kw):
        out = linear(x, w, mode=mode, seed=seed, **kw)
        products.append((x.clone(), w, mode, seed, out.clone()))
        return out

    def recording_grad(dy, x, **kw):
        out = weight_grad(dy, x, **kw)
        grads.append((dy.clone(), daq.ckpt8_restore(x), out.clone()))
        return out

    monkeypatch.setattr(ff.daq, "mx4_linear", recording_linear)
    monkeypatch.setattr(ff.daq, "ckpt8_weight_grad", recording_grad)
    block = ff.FeedForward(160, 224, seed=6)
    x, dy = _x(90, 160, torch.bfloat16, 3, 1).cuda(), _x(90, 160, torch.bfloat16, 4, 1).cuda()
    y, saved = block.forward(x)
    dx, dw_in, dw_out = block.backward(dy, saved, seed=7)

    w_in, w_out = block.w_in.cpu(), block.w_out.cpu()
    by = [(block.q_in, _values(w_in)), (block.q_out, _values(w_out)), (block.q_out_t, _values(w_out, transpose=True)), (block.q_in_t, _values(w_in, transpose=True))]
    assert len(products) == 4 and len(grads) == 2
    for i, ((a, w, mode, seed, out), (packed, vw)) in enumerate(zip(products, by)):
        assert w is packed and mode == (daq.ROUND_NEAREST if i < 2 else daq.ROUND_STOCHASTIC)
        va = _values(a.cpu(), stochastic=i >= 2, seed=seed)
        exact, absolute = va @ vw.T, np.abs(va) @ np.abs(vw).T
        assert out.dtype == torch.bfloat16 and np.all(np.abs(_np(out) - exact) <= _bound(-(-a.shape[1] // 64), absolute, exact, torch.bfloat16))
    assert products[2][3] != products[3][3]                                  # draws of their own
    (x0, *_, h), (a, *_, y0), (dy0, *_, da), (dh, *_, dx0) = products
    assert all(torch.equal(p, q) for p, q in ((x0, x), (y0, y), (dy0, dy), (dx0, dx)))
    want_a, kept = daq.ckpt8_act_forward(h, daq.ACT_SILU, gated=True)        # (compared with the oracle above)
    a8 = daq.alloc_ckpt8(90, 224)
    want_dh = daq.ckpt8_act_backward(da, kept, daq.ACT_SILU, y_ckpt=a8)
    assert torch.equal(a, want_a) and torch.equal(dh, want_dh)
    for (d, xs, out), (want_d, want_x, want_out) in zip(grads, ((dh, _saved(x.cpu()), dw_in), (dy, _np(daq.ckpt8_restore(a8)), dw_out))):
        assert torch.equal(d, want_d) and np.array_equal(_np(xs), want_x) and torch.equal(out, want_out)
        exact, absolute = _np(d).T @ want_x, np.abs(_np(d)).T @ np.abs(want_x)
        assert np.all(np.abs(_np(out) - exact) <= _bound(-(-90 // 16), absolute, exact, torch.float32))
