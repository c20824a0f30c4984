"""8-bit floating point matrices and their products on the GPU, through the binding, against the oracle in 64 bits.

Codes, scales and whole buffers are compared byte for byte.  Sums in fp32 (results in fp32, through bfloat16): every product is exact, each addition is
off by at most 2^-23 of the magnitudes added so far (to nearest or cut off), so a sum of n terms by at most n * 2^-23 * sum |products|; the matrix
instructions add 16 products as trees, so n counts these, with ten additions inside and behind them.  Results in bfloat16: the 8-bit instructions add
eight products at a time, each cut off at a multiple of 2^-13 of a power of two that the largest does not fall below, so seven of them lose at most
7 * 2^-13 of it; with the additions that follow as above, and 2^-8 of itself for the rounding."""
import numpy as np
import pytest
import torch

from oracle import fp8 as ref
from paper_2102_04782_amd import binding as daq

pytestmark = pytest.mark.gpu

DT = [torch.float32, torch.bfloat16]
SIZES = [(1, 1), (1, 127), (3, 128), (2, 129), (17, 511), (16, 512), (33, 513), (127, 64), (128, 130), (129, 255), (7, 1000), (300, 130), (257, 1029)]


def _x(rows, cols, dtype, seed, spread=6):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * torch.exp2(torch.randint(-spread, spread + 1, (rows, cols), generator=g).float())
    if rows > 2 and cols > 130:
        x[1, :128] = 0                                            # a block of zeros
        x[0, :128] = 0
        x[0, :64] = (torch.arange(64) + 0.5) * 0.5                # ties, once the block's scale is a power of two
        x[0, 64] = 256.0
        x[2, :32] = torch.arange(32) * 2.0 ** -10                 # below the codes' normal range
        x[2, 32:128] = 0
        x[2, 33] = 448.0
    return x.to(dtype)


def _strided(x, dev="cuda", pad=5, first=3):
    """x inside a wider matrix of other values: rows start at any element."""
    wide = torch.full((x.shape[0], x.shape[1] + pad), 7.0, dtype=x.dtype, device=dev)
    v = wide[:, first:first + x.shape[1]]
    v.copy_(x)
    return v


def _np(t):
    return t.detach().cpu().to(torch.float64).numpy()


def _filled(rows, cols):
    q = daq.alloc_fp8(rows, cols)
    q.buf.fill_(0xA5)
    return q


def _same(q, codes, byte):
    """Every byte of a packed matrix; a code of zero may carry either sign."""
    want, known = ref.buffer(codes, byte)
    got = q.buf.cpu().numpy()
    assert got.size == want.size
    off = daq.layout_fp8(q.rows, q.cols).off_scales
    assert np.array_equal(got[off:][known[off:]], want[off:][known[off:]])
    g, w = got[:off][known[:off]], want[:off][known[:off]]
    assert np.all((g == w) | ((g & 127 == 0) & (w & 127 == 0)))


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("rows,cols", SIZES)
def test_codes_scales_and_padding(rows, cols, dtype):
    x = _x(rows, cols, dtype, rows * 1000 + cols)
    by_rows, by_columns = ref.quantize(_np(x)), ref.quantize(_np(x).T)
    for src in (x.cuda(), _strided(x)):
        _same(daq.fp8_quantize(src, out=_filled(rows, cols)), *by_rows)
        _same(daq.fp8_quantize(src, columns=True, out=_filled(cols, rows)), *by_columns)
        r, c = daq.fp8_quantize_both(src, _filled(rows, cols), _filled(cols, rows))
        _same(r, *by_rows)
        _same(c, *by_columns)
        for to in DT:
            assert np.array_equal(_np(daq.fp8_dequantize(r, dtype=to)), ref.values(*by_rows))
            assert np.array_equal(_np(daq.fp8_dequantize(c, dtype=to)), ref.values(*by_columns))


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("count,rows,cols", [(1, 1, 1), (1, 128, 128), (2, 129, 127), (3, 70, 300), (5, 256, 640), (2, 300, 1030)])
def test_weights_by_tiles_and_their_transposes(count, rows, cols, dtype):
    w = _x(count * rows, cols, dtype, rows + cols).view(count, rows, cols)
    parts = [ref.quantize_weights(_np(w[e])) for e in range(count)]
    turned = [ref.transposed_weights(*p) for p in parts]
    stack = lambda ps: (np.concatenate([p[0] for p in ps]), np.concatenate([p[1] for p in ps]))
    wide = torch.full((count, rows + 2, cols + 3), 9.0, dtype=dtype, device="cuda")[:, 1:1 + rows, 2:2 + cols]
    wide.copy_(w)
    for src in (w.cuda(), wide):
        q, t = daq.fp8_quantize_weights(src, _filled(count * rows, cols), _filled(count * cols, rows))
        _same(q, *stack(parts))
        _same(t, *stack(turned))
        alone, none = daq.fp8_quantize_weights(src, transposed=False)
        assert none is None
        _same(alone, *stack(parts))
    if count == 1:
        _same(daq.fp8_quantize_weights(w[0].cuda())[0], *parts[0])


@pytest.mark.parametrize("dtype", DT)
def test_extremes(dtype):
    x = torch.zeros(12, 300, dtype=dtype)
    big = torch.finfo(dtype).max
    x[0, 0], x[0, 200], x[1, 5] = big, -big, 2.0 ** -126
    x[2, 7], x[2, 40] = 2.0 ** -133, 2.0 ** -128                  # below the normal range
    x[3, 3], x[4, 150], x[5, 299] = float("nan"), float("inf"), float("-inf")
    x[6] = torch.tensor([2.0 ** -133 * (i % 13) for i in range(300)])
    x[7, 31], x[7, 0], x[7, 129] = 448.0, 449.0, 464.0
    x[8, :8] = torch.tensor([448.0, 450.0, 456.0, 460.0, 464.0, 5.0, 1e-30, -447.9])
    x[9, 0], x[9, 1], x[10, 140], x[10, 130] = 448 * 2.0 ** -126, 2.0 ** -130, 450 * 2.0 ** -126, 3 * 2.0 ** -133
    for m, q in ((_np(x), daq.fp8_quantize(x.cuda())), (_np(x).T, daq.fp8_quantize(x.cuda(), columns=True))):
        codes, byte = ref.quantize(m)
        _same(q, codes, byte)
        with np.errstate(over="ignore"):                           # (2^128, which rounding can make of the largest values, is an infinity in either type)
            v = ref.values(codes, byte).astype(np.float32)
        assert np.array_equal(_np(daq.fp8_dequantize(q)), v, equal_nan=True)
        got = _np(daq.fp8_dequantize(q, dtype=torch.bfloat16))
        with np.errstate(invalid="ignore"):
            assert np.all((got == v) | (np.isnan(got) & np.isnan(v)) | (np.abs(got - v) <= 2.0 ** -134))   # half a step of the smallest
    w = x.cuda()
    q, t = daq.fp8_quantize_weights(w)
    codes, byte = ref.quantize_weights(_np(x))
    _same(q, codes, byte)
    _same(t, *ref.transposed_weights(codes, byte))


def test_all_codes_and_all_ties():
    """Every code, every middle between two codes, and what lies a little beside it."""
    g = ref.GRID
    mid = (g[1:] + g[:-1]) / 2
    v = np.concatenate((g, mid, np.nextafter(mid.astype(np.float32), np.float32(0)), np.nextafter(mid.astype(np.float32), np.float32(1e9))))
    v = np.concatenate((v, -v)).astype(np.float32)
    x = np.zeros((-(-v.size // 127), 128), np.float32)
    x[:, 0] = 448
    x[:, 1:].flat[:v.size] = v
    for shift in (-100, 0, 37):
        t = torch.from_numpy(x * np.float32(2.0) ** shift)
        codes, byte = ref.quantize(_np(t))
        assert np.all(byte == 127 + shift)
        _same(daq.fp8_quantize(t.cuda()), codes, byte)
        _same(daq.fp8_quantize(t.t().contiguous().cuda(), columns=True), codes, byte)


MATMUL = [(1, 1, 1), (1, 33, 130), (1, 512, 2048), (2, 70, 300), (5, 64, 256), (13, 100, 1030), (16, 2049, 512), (17, 256, 513), (32, 256, 512), (33, 129, 64),
          (40, 2049, 96), (64, 64, 4096), (65, 130, 8200), (100, 260, 700), (255, 257, 513), (256, 256, 256), (300, 600, 320), (513, 511, 1024), (1030, 770, 200),
          (2050, 2100, 300), (4100, 3900, 129)]


def _bound(K, absolute, exact, dtype):
    return (-(-K // 16) + 10) * 2.0 ** -23 * absolute + (7 * 2.0 ** -13 * absolute + 2.0 ** -8 * np.abs(exact) if dtype == torch.bfloat16 else 0) + 1e-40


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("M,N,K", MATMUL)
def test_matmul(M, N, K, dtype):
    a, b = _x(M, K, torch.bfloat16, M + K), _x(N, K, torch.float32, N + 3 * K)
    va, vb = ref.values(*ref.quantize(_np(a))), ref.values(*ref.quantize(_np(b)))
    exact, absolute = va @ vb.T, np.abs(va) @ np.abs(vb).T
    qa, qb = daq.fp8_quantize(a.cuda()), daq.fp8_quantize(b.cuda())
    wide = torch.full((M, N + 7), 55.0, dtype=dtype, device="cuda")
    for out in (torch.full((M, N), float("nan"), dtype=dtype, device="cuda"), wide[:, 3:3 + N]):
        got = _np(daq.fp8_matmul(qa, qb, out=out))
        assert np.all(np.abs(got - exact) <= _bound(K, absolute, exact, dtype))
    assert bool((wide[:, :3] == 55).all()) and bool((wide[:, 3 + N:] == 55).all())     # nothing beside the result
    if dtype == torch.float32:
        start = torch.randn(M, N, device="cuda")
        got = _np(daq.fp8_matmul(qa, qb, out=start.clone(), accumulate=True))
        want = exact + _np(start)
        assert np.all(np.abs(got - want) <= _bound(K, absolute, exact, dtype) + 2.0 ** -23 * np.abs(want))


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("M,N,K", MATMUL)
def test_linear(M, N, K, dtype):
    x, w = _x(M, K, dtype, M + 2 * K), _x(N, K, torch.bfloat16, N + 5 * K)
    vx, vw = ref.values(*ref.quantize(_np(x))), ref.values(*ref.quantize_weights(_np(w)))
    exact, absolute = vx @ vw.T, np.abs(vx) @ np.abs(vw).T
    qw, _ = daq.fp8_quantize_weights(w.cuda())
    for src in (x.cuda(), _strided(x)):
        for to in DT:
            got = _np(daq.fp8_linear(src, qw, dtype=to))
            assert np.all(np.abs(got - exact) <= _bound(K, absolute, exact, to))


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("M,N,K", [(1, 40, 70), (129, 200, 330), (600, 513, 257), (1500, 130, 700)])
def test_gradients_of_a_layer(M, N, K, dtype):
    x, w, dy = _x(M, K, dtype, 1), _x(N, K, torch.bfloat16, 2), _x(M, N, dtype, 3)
    qw, qt = daq.fp8_quantize_weights(w.cuda())
    (_, xc), (dr, dc) = daq.fp8_quantize_both(x.cuda()), daq.fp8_quantize_both(dy.cuda())
    vw, vd = ref.values(*ref.quantize_weights(_np(w))), ref.values(*ref.quantize(_np(dy)))
    got, want = _np(daq.fp8_matmul(dr, qt, dtype=torch.float32)), vd @ vw
    assert np.all(np.abs(got - want) <= _bound(N, np.abs(vd) @ np.abs(vw), want, torch.float32))
    cd, cx = ref.values(*ref.quantize(_np(dy).T)), ref.values(*ref.quantize(_np(x).T))
    got, want = _np(daq.fp8_matmul(dc, xc, dtype=torch.float32)), cd @ cx.T
    assert np.all(np.abs(got - want) <= _bound(M, np.abs(cd) @ np.abs(cx).T, want, torch.float32))


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("M,N,K", [(3, 40, 300), (20, 130, 700), (200, 300, 600), (600, 300, 513), (2100, 2050, 513), (4352, 4096, 300)])
def test_what_is_not_finite_reaches_its_sums_only(M, N, K, dtype):
    x, w = torch.randn(M, K), torch.randn(N, K)
    x[M // 2, 140], w[N - 2, 5], w[1, K - 1] = float("nan"), float("inf"), float("-inf")
    got = daq.fp8_matmul(daq.fp8_quantize(x.cuda()), daq.fp8_quantize(w.cuda()), dtype=dtype).float().cpu()
    bad = torch.zeros(M, N, dtype=torch.bool)
    bad[M // 2], bad[:, N - 2], bad[:, 1] = True, True, True
    assert torch.equal(torch.isnan(got), bad) and bool(torch.isfinite(got[~bad]).all())
    if M <= 32:                                                           # rows quantized on the way
        got = daq.fp8_linear(x.cuda(), daq.fp8_quantize(w.cuda()), dtype=dtype).float().cpu()
        assert torch.equal(torch.isnan(got), bad) and bool(torch.isfinite(got[~bad]).all())


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("M,N,K", [(2, 40, 300), (70, 70, 300), (300, 600, 320)])
def test_scales_far_apart(M, N, K, dtype):
    """Operands near the ends of the range that a product in bfloat16 keeps: 2^-117 times 2^110, and 2^60 times 2^60."""
    for ea, eb in ((-117, 110), (100, -105), (60, 60), (-60, -60)):
        a, b = torch.randn(M, K) * 2.0 ** ea, torch.randn(N, K) * 2.0 ** eb
        va, vb = ref.values(*ref.quantize(_np(a))), ref.values(*ref.quantize(_np(b)))
        exact, absolute = va @ vb.T, np.abs(va) @ np.abs(vb).T
        got = _np(daq.fp8_matmul(daq.fp8_quantize(a.cuda()), daq.fp8_quantize(b.cuda()), dtype=dtype))
        assert np.all(np.abs(got - exact) <= _bound(K, absolute, exact, dtype))


def test_nothing_to_do_and_nothing_to_sum():
    w, _ = daq.fp8_quantize_weights(torch.randn(40, 70, device="cuda"))
    assert daq.fp8_linear(torch.empty(0, 70, device="cuda"), w).shape == (0, 40)
    a, b = daq.fp8_quantize(torch.empty(0, 40, device="cuda"), columns=True), daq.fp8_quantize(torch.empty(0, 70, device="cuda"), columns=True)
    assert (a.rows, a.cols, b.rows, b.cols) == (40, 0, 70, 0)
    out = torch.full((40, 70), 3.0, device="cuda")
    assert bool((daq.fp8_matmul(a, b, out=out, accumulate=True) == 3).all())
    assert bool((daq.fp8_matmul(a, b, out=out) == 0).all())


@pytest.mark.parametrize("M,N,K", [(4352, 4096, 100), (4100, 4104, 200), (4352, 4096, 300), (4097, 4352, 640), (2304, 8192, 1100)])
def test_large_products_go_from_tile_to_tile(M, N, K):
    """More tiles than CUs, rows of whole 16-byte pieces, one stage to nine: results whose stores are still under way when the next tile begins."""
    a, b = _x(M, K, torch.bfloat16, M + K), _x(N, K, torch.bfloat16, N + 3 * K)
    va, vb = ref.values(*ref.quantize(_np(a))), ref.values(*ref.quantize(_np(b)))
    exact, absolute = va @ vb.T, np.abs(va) @ np.abs(vb).T
    qa, qb = daq.fp8_quantize(a.cuda()), daq.fp8_quantize(b.cuda())
    wide = torch.full((M + 3, N + 16), 55.0, dtype=torch.bfloat16, device="cuda")
    for out in (torch.full((M, N), float("nan"), dtype=torch.bfloat16, device="cuda"), wide[1:1 + M, 8:8 + N]):
        got = _np(daq.fp8_matmul(qa, qb, out=out))
        assert np.all(np.abs(got - exact) <= _bound(K, absolute, exact, torch.bfloat16))
    assert bool((wide[:, :8] == 55).all()) and bool((wide[:, 8 + N:] == 55).all()) and bool((wide[0] == 55).all()) and bool((wide[1 + M:] == 55).all())


def test_results_that_pass_the_caches_by():
    """192 MiB of results: the same values as of two halves."""
    a, b = daq.fp8_quantize(torch.randn(12800, 256, device="cuda")), daq.fp8_quantize(torch.randn(8192, 256, device="cuda"))
    half = daq.fp8_quantize(daq.fp8_dequantize(b)[4096:].contiguous())
    whole = daq.fp8_matmul(a, b)
    assert torch.equal(whole[:, 4096:], daq.fp8_matmul(a, half))


@pytest.mark.parametrize("M,N,K", [(64, 64, 8192), (130, 70, 5000), (512, 512, 8192), (300, 1000, 4096), (128, 300, 16384)])
def test_sums_in_parts(M, N, K):
    """Few tiles and a long axis: parts of it, added up in their order."""
    a, b = _x(M, K, torch.float32, 1, 2), _x(N, K, torch.float32, 2, 2)
    va, vb = ref.values(*ref.quantize(_np(a))), ref.values(*ref.quantize(_np(b)))
    exact, absolute = va @ vb.T, np.abs(va) @ np.abs(vb).T
    qa, qb = daq.fp8_quantize(a.cuda()), daq.fp8_quantize(b.cuda())
    assert daq._few_ws_bytes("daq_fp8_matmul_workspace", M, N, K, daq.FP32) > 0
    for to in DT:
        first = daq.fp8_matmul(qa, qb, dtype=to)
        assert np.all(np.abs(_np(first) - exact) <= _bound(K, absolute, exact, to))
        assert torch.equal(first, daq.fp8_matmul(qa, qb, dtype=to))
    start = torch.randn(M, N, device="cuda")
    want = exact + _np(start)
    assert np.all(np.abs(_np(daq.fp8_matmul(qa, qb, out=start, accumulate=True)) - want) <= _bound(K, absolute, exact, torch.float32) + 2.0 ** -23 * np.abs(want))


def test_offsets_beyond_32_bits():
    """4.4 GB of codes, 8.8 GB of elements, 5 GB of results: the first and the last rows against those of small matrices."""
    rows, K = 540001, 8192
    x = torch.empty(rows, K, dtype=torch.bfloat16, device="cuda")
    x.view(-1)[:1 << 20].normal_()
    x.view(-1)[1 << 20:] = 0.5
    ends = torch.cat((torch.arange(40), torch.arange(rows - 40, rows))).cuda()
    x[ends] = torch.randn(80, K, device="cuda").bfloat16()
    w, _ = daq.fp8_quantize_weights(torch.randn(72, K, device="cuda"))
    q, small = daq.fp8_quantize(x), daq.fp8_quantize(x[ends].contiguous())
    va, vb = _np(daq.fp8_dequantize(small)), _np(daq.fp8_dequantize(w))
    exact, absolute = va @ vb.T, np.abs(va) @ np.abs(vb).T
    for to in DT:
        got = daq.fp8_matmul(q, w, dtype=to)[ends].double()
        assert np.all(np.abs(_np(got) - exact) <= _bound(K, absolute, exact, to))
        assert torch.equal(got, daq.fp8_linear(x, w, dtype=to)[ends].double())
    assert torch.equal(daq.fp8_dequantize(q, dtype=torch.bfloat16)[ends], daq.fp8_dequantize(small, dtype=torch.bfloat16))
    c = daq.fp8_quantize(x, columns=True)
    assert c.rows == K and c.cols == rows
    byte = daq.layout_fp8(K, rows)
    last = c.buf[(K - 1) * byte.pitch:(K - 1) * byte.pitch + rows][ends]
    tail = daq.fp8_quantize(x[rows - rows % 128:].contiguous(), columns=True)      # the last block of tokens
    assert torch.equal(last[40:], tail.buf[(K - 1) * 128:(K - 1) * 128 + rows % 128][-40:]) or rows % 128 < 40
    del x, q, c
    # results of more than 2^32 bytes
    a, b = daq.fp8_quantize(torch.randn(70000, 128, device="cuda")), daq.fp8_quantize(torch.randn(36000, 128, device="cuda"))
    out = daq.fp8_matmul(a, b)
    ends = torch.cat((torch.arange(40), torch.arange(70000 - 40, 70000))).cuda()
    va, vb = _np(daq.fp8_dequantize(a)[ends]), _np(daq.fp8_dequantize(b))
    exact, absolute = va @ vb.T, np.abs(va) @ np.abs(vb).T
    assert np.all(np.abs(_np(out[ends]) - exact) <= _bound(128, absolute, exact, torch.bfloat16))


@pytest.mark.parametrize("M,K,ld", [(12300, 8193, 8256), (24577, 4160, 4160), (25000, 4100, 4100)])
def test_large_sources(M, K, ld):
    """Sources of 96 Mi elements and more, whose rows begin with a line or do not: the same buffers as of their parts."""
    x = torch.randn(M, ld, device="cuda", dtype=torch.bfloat16)[:, :K]
    by_rows, by_columns = daq.fp8_quantize_both(x)
    L, pitch = daq.layout_fp8(M, K), daq.layout_fp8(M, K).pitch
    for one, other in ((daq.fp8_quantize(x), by_rows), (daq.fp8_quantize(x, columns=True), by_columns)):
        lay = daq.layout_fp8(one.rows, one.cols)
        for first, n in ((0, one.rows * lay.pitch), (lay.off_scales, -(-one.cols // 512) * one.rows * 4)):
            assert torch.equal(one.buf[first:first + n], other.buf[first:first + n])
    C = daq.layout_fp8(K, M)
    codes, codes_t = by_rows.buf[:M * pitch].view(M, pitch), by_columns.buf[:K * C.pitch].view(K, C.pitch)
    scales = by_rows.buf[L.off_scales:L.off_scales + -(-K // 512) * M * 4].view(-1, M, 4)
    for first in (0, 4096, M // 128 * 128 - 256):                          # whole blocks of rows
        part = x[first:first + 256].contiguous()
        n, P = part.shape[0], daq.layout_fp8(part.shape[0], K)
        q, qc = daq.fp8_quantize_both(part)
        assert torch.equal(q.buf[:n * P.pitch].view(n, -1), codes[first:first + n])
        assert torch.equal(q.buf[P.off_scales:P.off_scales + -(-K // 512) * n * 4].view(-1, n, 4), scales[:, first:first + n])
        assert torch.equal(qc.buf[:K * n].view(K, n), codes_t[:, first:first + n])


@pytest.mark.parametrize("M,N", [(2, 5), (70, 40), (300, 270)])
def test_the_longest_sums(M, N):
    """K = 2^23 - 128.  Products are multiples of 1/2, equal ones side by side, and their sums below 2^23 (of the first row: multiples of 64 below 2^24): fp32 holds
    every sum on the way, in any order, so results in fp32 are exact and those in bfloat16 are off by their rounding.  The last row's cancel."""
    K = (1 << 23) - 128
    a = torch.full((M, K), 0.5, device="cuda", dtype=torch.bfloat16)
    a[0] = 0
    a[0, -128:] = 448.0
    a[-1, 1::2] = -0.5
    b = torch.ones(N, K, device="cuda", dtype=torch.bfloat16)
    b[:, -128:] = torch.arange(1, N + 1, device="cuda")[:, None].to(torch.bfloat16)
    last = daq.fp8_dequantize(daq.fp8_quantize(b[:, -128:].contiguous()))[:, 0].double() * 128
    want = (0.5 * (K - 128) + 0.5 * last).expand(M, N).clone()
    want[0] = 448 * last
    want[-1] = 0
    qa, qb = daq.fp8_quantize(a), daq.fp8_quantize(b)
    assert torch.equal(daq.fp8_matmul(qa, qb, dtype=torch.float32).double(), want)
    assert bool(((daq.fp8_matmul(qa, qb).double() - want).abs() <= 2.0 ** -8 * want).all())
