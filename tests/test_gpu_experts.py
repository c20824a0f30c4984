"""Routing, the order of the rows by expert, experts' products and their sums on the GPU, through the binding, against the oracle in 64 bits.

Choices, orders and 8-bit buffers are compared exactly.  Weights are computed in 64 bits and rounded once: 2^-24 of themselves, and a little for
the library's exponential (2^-50).  Products: the bounds of the products of whole matrices."""
import numpy as np
import pytest
import torch

from oracle import fp8 as ref
from paper_2102_04782_amd import binding as daq
from test_gpu_fp8 import DT, _bound, _filled, _np, _same, _strided, _x

pytestmark = pytest.mark.gpu

KIND = {"softmax": daq.SCORES_SOFTMAX, "sigmoid": daq.SCORES_SIGMOID}


def _logits(T, E, dtype, seed, masked=True):
    g = torch.Generator().manual_seed(seed)
    l = torch.randn(T, E, generator=g) * 2
    if masked and T > 4:
        l[T // 2] = -torch.inf                                            # a padded token
        l[T // 3, torch.randperm(E, generator=g)[:E * 3 // 4]] = -torch.inf   # some experts switched off
        l[T // 4] = -torch.inf
        l[T // 4, E // 2] = 0.5                                           # a single one left
    if T > 8:
        l[1] = 0.25                                                       # all equal
        l[2, ::2] = l[2, 0]                                               # ties
        l[3] = torch.finfo(dtype).min                                     # the type's lowest value
        l[4, 0] = torch.finfo(dtype).min
    return l.to(dtype)


ROUTES = [(1, 1, 1, 1, 1), (1, 4, 2, 1, 1), (5, 60, 4, 1, 1), (17, 64, 6, 8, 3), (33, 65, 1, 1, 1), (40, 128, 32, 1, 1), (9, 129, 5, 3, 2), (130, 160, 6, 8, 3),
          (100, 256, 8, 8, 4), (64, 250, 7, 1, 1), (31, 384, 8, 64, 10), (20, 512, 16, 4, 1), (12, 1024, 8, 1, 1), (13, 1000, 31, 8, 8), (70, 32, 4, 32, 5)]


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("T,E,k,groups,top", ROUTES)
def test_route(T, E, k, groups, top, kind, dtype):
    logits = _logits(T, E, dtype, T + E)
    g = torch.Generator().manual_seed(E)
    for bias in (None, 0.1 * torch.randn(E, generator=g)):
        if bias is not None and E > 8:
            bias[3], bias[5] = -torch.inf, bias[4]
        for renormalize, scale in ((True, 1.0), (False, 2.5), (True, 0.5)):
            want, chosen = ref.route(_np(logits), k, kind, None if bias is None else _np(bias), groups, top, renormalize, scale)
            for src in (logits.cuda(), _strided(logits)):
                w, e = daq.route(src, k, KIND[kind], None if bias is None else bias.cuda(), groups, top, renormalize, scale)
                assert np.array_equal(_np(e), chosen)
                assert np.all(np.abs(_np(w) - want) <= (2.0 ** -24 + 2.0 ** -48) * np.abs(want) + 2.0 ** -149)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (3, 4, 2), (33, 60, 4), (64, 256, 8), (20, 1000, 16), (9, 1024, 32)])
def test_route_backward(T, E, k, kind, dtype):
    """fp32: the chosen ones' part is computed in 64 bits; the softmax over all experts in 32, where a sum of E / 64 + 6 terms and an exponential, off by 2^-22, make
    each score off by less than (E / 64 + 20) * 2^-24 of itself, and the sum of k products the same of the magnitudes that it adds."""
    logits = _logits(T, E, dtype, 3 * T + E)
    g = torch.randn(T, k, generator=torch.Generator().manual_seed(T))
    for renormalize, scale in ((True, 1.0), (False, 2.5), (True, 0.5)):
        _, chosen = ref.route(_np(logits), k, kind, renormalize=renormalize)
        want = ref.route_backward(_np(g), _np(logits), chosen, kind, renormalize, scale)
        s = ref.scores(_np(logits), kind)
        ds = np.where(chosen >= 0, np.abs(_np(g)) * scale, 0)
        size = np.abs(want) + s * (ds.sum(1, keepdims=True) if not renormalize else 0)
        if renormalize:                                                    # shares of the chosen ones, and the difference of a place's own and the mean
            take = np.where(chosen >= 0, np.take_along_axis(s, np.maximum(chosen, 0), 1), 0)
            total = take.sum(1, keepdims=True)
            share = np.divide(take, total, out=np.zeros_like(take), where=total > 0)
            size = np.abs(want)
            for j in range(k):
                rows = np.arange(T)[chosen[:, j] >= 0]
                size[rows, chosen[rows, j]] += (share[:, j] * (ds * share).sum(1))[rows] * 2.0 ** -24
            # the oracle's own sums in 64 bits: where they cancel, an expert that was not chosen has k roundings of s * sum |g| / total instead of zero
            size += (2.0 ** -24 * s * np.divide(ds.sum(1, keepdims=True), total, out=np.zeros_like(total), where=total > 0))
        bound = (E / 64 + k + 30) * 2.0 ** -24 * size + (2.0 ** -8 * np.abs(want) if dtype == torch.bfloat16 else 0) + 1e-37
        for src in (logits.cuda(), _strided(logits)):
            got = _np(daq.route_backward(g.cuda(), src, torch.from_numpy(chosen).int().cuda(), KIND[kind], renormalize, scale))
            assert np.all(np.abs(got - want) <= bound)


@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalize", [True, False])
def test_route_gradient_against_differences(kind, renormalize):
    """A step of 2^-10 along random directions: the difference quotient of the weights (in 64 bits, by the oracle) is off by some 2^-20 of the
    third derivative, here below 2^-14 of the gradients' sizes."""
    logits = _logits(40, 32, torch.float32, 5, masked=False)[8:]
    g = torch.randn(32, 4, generator=torch.Generator().manual_seed(1))
    w, chosen = daq.route(logits.cuda(), 4, KIND[kind], renormalize=renormalize)
    grad = _np(daq.route_backward(g.cuda(), logits.cuda(), chosen, KIND[kind], renormalize))
    x, c = _np(logits), _np(chosen).astype(int)

    def loss(v):
        s = np.take_along_axis(ref.scores(v, kind), c, 1)
        return ((s / s.sum(1, keepdims=True) if renormalize else s) * _np(g)).sum(1)

    rng = np.random.default_rng(0)
    for _ in range(8):
        d = rng.standard_normal(x.shape)
        h = 2.0 ** -10
        quotient = (loss(x + h * d) - loss(x - h * d)) / (2 * h)
        assert np.all(np.abs((grad * d).sum(1) - quotient) <= 2.0 ** -14 * (np.abs(_np(g)).sum(1) + 1))


def test_route_of_what_is_no_number():
    logits = torch.randn(8, 40)
    logits[1, 3], logits[2, 7], logits[5, 0] = float("nan"), float("inf"), float("nan")
    for kind in ("softmax", "sigmoid"):
        want, chosen = ref.route(_np(logits), 4, kind)
        w, e = daq.route(logits.cuda(), 4, KIND[kind])
        assert np.array_equal(_np(e), chosen) and np.array_equal(np.isnan(_np(w)), np.isnan(want))
        assert bool((e[1] == -1).all()) and bool(torch.isnan(w[1]).all()) and (int(e[2, 0]) == 7) == (kind == "sigmoid")
        grad = daq.route_backward(torch.ones(8, 4, device="cuda"), logits.cuda(), e, KIND[kind], renormalize=False)
        assert bool((grad[1] == 0).all()) and bool(torch.isfinite(grad[3]).all())
        y = torch.ones(32, 16, device="cuda")
        out = daq.experts_combine(y, daq.experts_plan(e, 40), w)
        assert np.array_equal(np.isnan(_np(out)[:, 0]), np.isnan(want[:, 0]))
    bias = torch.zeros(40)
    bias[6] = float("nan")
    assert bool((daq.route(torch.randn(3, 40).cuda(), 4, bias=bias.cuda())[1] == -1).all())


def test_scores_that_32_bits_do_not_tell_apart():
    """Sigmoids next to one another: the order is that of 64 bits."""
    g = torch.Generator().manual_seed(0)
    base = 3 + torch.randn(200, 1, generator=g)
    logits = base + torch.randint(-3, 4, (200, 64), generator=g) * 2.0 ** -22
    bias = torch.randint(-2, 3, (64,), generator=g) * 2.0 ** -26
    for kind in ("softmax", "sigmoid"):
        want, chosen = ref.route(_np(logits), 8, kind, _np(bias), 4, 2)
        w, e = daq.route(logits.cuda(), 8, KIND[kind], bias.cuda(), 4, 2)
        assert np.array_equal(_np(e), chosen)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E", [60, 100, 256, 512, 1000])
def test_zeros_of_both_signs_are_equals(E, kind, dtype):
    logits = torch.full((6, E), -1.0)
    logits[:, 1::7] = -0.0
    logits[:, 3::7] = 0.0
    logits[1] = -0.0
    logits[2] = 0.0
    logits[2, :8] = -0.0
    for groups in (1, 4):
        _, want = ref.route(_np(logits), 8, kind, None, groups, min(groups, 2), True, 1.0)
        _, e = daq.route(logits.to(dtype).cuda(), 8, KIND[kind], None, groups, min(groups, 2))
        assert np.array_equal(_np(e), want) and want[2].tolist() == list(range(8))


def _chosen(T, k, E, seed, none=0.1, skew=1.0):
    g = torch.Generator().manual_seed(seed)
    score = torch.randn(T, E, generator=g) + skew * torch.randn(E, generator=g)
    c = torch.topk(score, k, dim=1).indices.int() if k <= E else torch.randint(0, E, (T, k), generator=g).int()
    return torch.where(torch.rand(T, k, generator=g) < none, torch.full_like(c, -1), c)


PLANS = [(1, 1, 1), (1, 8, 64), (3, 2, 5), (64, 1, 7), (65, 3, 16), (300, 4, 33), (1000, 2, 64), (1024, 1, 1024), (1025, 4, 300), (2049, 2, 5), (5000, 8, 256), (40000, 8, 1024)]


@pytest.mark.parametrize("T,k,E", PLANS)
def test_plan(T, k, E):
    for none, skew in ((0.0, 1.0), (0.3, 4.0), (1.0, 0.0)):
        c = _chosen(T, k, E, T + E, none, skew)
        if none == 0.3 and T * k > 3:
            c.view(-1)[0], c.view(-1)[-1] = E, -7                          # no expert of this plan
        counts, table, rows, place = ref.plan(torch.where((c >= 0) & (c < E), c, -1).numpy(), E)
        out = daq.alloc_plan(T, k, E)
        for t in (out.counts, out.table, out.rows, out.place):
            t.fill_(-99)
        p = daq.experts_plan(c.cuda(), E, out=out)
        assert np.array_equal(_np(p.counts), counts) and np.array_equal(_np(p.table), table)
        assert np.array_equal(_np(p.rows), rows) and np.array_equal(_np(p.place), place)


def test_plan_of_many_rounds():
    """More slots than 256 workgroups take in one round."""
    c = torch.randint(-1, 37, (150000, 2), generator=torch.Generator().manual_seed(2)).int().cuda()
    p = daq.experts_plan(c, 37)
    flat = c.view(-1).long()
    key = torch.where(flat < 0, 37, flat)
    order = torch.sort(key, stable=True).indices
    n = int((flat >= 0).sum())
    assert torch.equal(p.rows[:n].long(), order[:n]) and bool((p.rows[n:] == -1).all())
    assert torch.equal(p.counts.long(), torch.bincount(key, minlength=38)[:37])
    assert torch.equal(p.place.view(-1)[order[:n]].long(), torch.arange(n, device="cuda")) and bool((p.place.view(-1)[flat < 0] == -1).all())


EXPERTS = [(1, 1, 1, 1, 1), (1, 6, 64, 100, 300), (3, 2, 5, 33, 70), (40, 2, 4, 130, 257), (70, 3, 16, 64, 128), (200, 4, 8, 300, 130), (515, 2, 3, 260, 513), (1200, 1, 3, 513, 100),
           (700, 4, 5, 1030, 129)]


def _values_of(w):
    return np.stack([ref.values(*ref.quantize_weights(_np(m))) for m in w])


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("T,k,E,N,K", EXPERTS)
def test_products_of_experts(T, k, E, N, K, dtype):
    c = _chosen(T, k, E, T + N)
    plan = daq.experts_plan(c.cuda(), E)
    counts, table, rows, place = ref.plan(c.numpy(), E)
    total = int(counts.sum())
    expert = np.repeat(np.arange(E), counts)
    w = _x(E * N, K, torch.bfloat16, N + K).view(E, N, K)
    vw = _values_of(w)
    qw, qt = daq.fp8_quantize_weights(w.cuda())
    # rows taken by their tokens
    x = _x(T, K, dtype, T + K)
    vx = ref.values(*ref.quantize(_np(x)))[rows[:total] // k]
    exact = np.einsum("pk,pnk->pn", vx, vw[expert]) if total * N * K < 3e7 else np.stack([vw[e] @ v for e, v in zip(expert, vx)]).reshape(total, N)
    absolute = np.stack([np.abs(vw[e]) @ np.abs(v) for e, v in zip(expert, vx)]).reshape(total, N)
    for to in DT:
        wide = torch.full((T * k, N + 6), 7.0, dtype=to, device="cuda")
        for src in (x.cuda(), _strided(x)):
            y = daq.experts_linear(src, qw, plan, out=wide[:, 2:2 + N])
            assert np.all(np.abs(_np(y)[:total] - exact) <= _bound(K, absolute, exact, to))
            assert bool((wide[:, :2] == 7).all()) and bool((wide[:, 2 + N:] == 7).all()) and bool((wide[total:] == 7).all())
        again = daq.experts_matmul(daq.fp8_quantize(x.cuda()), qw, plan, dtype=to)
        assert torch.equal(again[:total], y[:total])
    # rows in the order of the plan, times the transposed weights
    d = _x(T * k, N, dtype, 5 + N)
    vd = ref.values(*ref.quantize(_np(d)))[:total]
    exact = np.stack([v @ vw[e] for e, v in zip(expert, vd)]).reshape(total, K)
    absolute = np.stack([np.abs(v) @ np.abs(vw[e]) for e, v in zip(expert, vd)]).reshape(total, K)
    for to in DT:
        dx = daq.experts_linear(d.cuda(), qt, plan, sorted_rows=True, dtype=to)
        assert np.all(np.abs(_np(dx)[:total] - exact) <= _bound(N, absolute, exact, to))


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("T,k,E,N,K", EXPERTS)
def test_gradients_of_experts(T, k, E, N, K, dtype):
    c = _chosen(T, k, E, 2 * T + N)
    plan = daq.experts_plan(c.cuda(), E)
    counts, table, rows, place = ref.plan(c.numpy(), E)
    total, ends = int(counts.sum()), np.cumsum(counts)
    x, dy = _x(T, K, dtype, 7), _x(T * k, N, dtype, 8)
    columns = daq.experts_columns(T, k, E)
    assert columns == ref.columns(T, k, E)
    for src in (x.cuda(), _strided(x)):
        xr, xc = daq.experts_quantize(src, plan, by_rows=_filled(T, K), by_columns=_filled(K, columns))
        _same(xr, *ref.quantize(_np(x)))
    dr, dc = daq.experts_quantize(dy.cuda(), plan, sorted_rows=True)
    _same(dr, *ref.quantize(_np(dy)))
    # the columns, expert by expert
    layout = daq.layout_fp8(K, columns)
    buf = xc.buf.cpu().numpy()
    want, absolute = np.zeros((E, N, K)), np.zeros((E, N, K))
    for e in range(E):
        n, first, b0 = counts[e], ends[e] - counts[e], table[2, e]
        if n == 0:
            continue
        cx, bx = ref.quantize(_np(x)[rows[first:first + n] // k].T)
        cd, bd = ref.quantize(_np(dy)[first:first + n].T)
        for col in range(K):
            at = col * layout.pitch + b0 * 128
            got = buf[at:at + bx.shape[1] * 128]
            assert np.all((got[:n] == cx[col]) | ((got[:n] & 127 == 0) & (cx[col] & 127 == 0))) and np.all(got[n:] == 0)
            assert all(buf[layout.off_scales + (((b0 + b) // 4) * K + col) * 4 + (b0 + b) % 4] == bx[col, b] for b in range(bx.shape[1]))
        vx, vd = ref.values(cx, bx), ref.values(cd, bd)
        want[e], absolute[e] = vd @ vx.T, np.abs(vd) @ np.abs(vx).T
    longest = max(int(counts.max()), 1)
    for to in DT:
        wide = torch.full((E, N + 1, K + 5), 3.0, dtype=to, device="cuda")
        got = _np(daq.experts_weight_grad(dc, xc, plan, out=wide[:, :N, 2:2 + K]))
        assert np.all(np.abs(got - want) <= _bound(longest, absolute, want, to))
        assert bool((wide[:, N] == 3).all()) and bool((wide[:, :, :2] == 3).all()) and bool((wide[:, :, 2 + K:] == 3).all())
    start = torch.randn(E, N, K, device="cuda")
    got = _np(daq.experts_weight_grad(dc, xc, plan, out=start.clone(), accumulate=True))
    sum_ = want + _np(start)
    assert np.all(np.abs(got - sum_) <= _bound(longest, absolute, want, torch.float32) + 2.0 ** -23 * np.abs(sum_))


COMBINE = [(1, 1, 1, 1), (3, 8, 64, 5121), (5, 2, 4, 7), (33, 3, 5, 64), (100, 4, 8, 1000), (64, 32, 40, 257), (300, 5, 16, 2049)]


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("weighted", [True, False])
@pytest.mark.parametrize("T,k,E,D", COMBINE)
def test_combine(T, k, E, D, weighted, dtype):
    """k products and sums: k * 2^-23 of the magnitudes; a dot product of D terms over 64 lanes (D / 64 + 8) of them."""
    c = _chosen(T, k, E, T + D)
    plan = daq.experts_plan(c.cuda(), E)
    _, _, rows, place = ref.plan(c.numpy(), E)
    total = int((c >= 0).sum())
    g = torch.Generator().manual_seed(D)
    y, d = _x(T * k, D, dtype, 1), _x(T, D, dtype, 2)
    w = torch.softmax(torch.randn(T, k, generator=g), 1)
    there = place >= 0
    rows_of = np.where(there[:, :, None], _np(y)[np.maximum(place, 0)], 0)
    fw = _np(w) if weighted else np.ones((T, k))
    ulp = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    want, absolute = np.einsum("tk,tkd->td", fw, rows_of), np.einsum("tk,tkd->td", np.abs(fw), np.abs(rows_of))
    kw = {"weights": w.cuda()} if weighted else {}
    y_nan = y.clone()
    y_nan[total:] = float("nan")                                           # behind the order's last row nothing is read
    wide = torch.full((T, D + 4), 5.0, dtype=dtype, device="cuda")
    for src in (y_nan.cuda(), _strided(y_nan)):
        out = _np(daq.experts_combine(src, plan, out=wide[:, 1:1 + D], **kw))
        assert np.all(np.abs(out - want) <= k * 2.0 ** -23 * absolute + ulp * np.abs(want) + 1e-40)
        assert bool((wide[:, :1] == 5).all()) and bool((wide[:, 1 + D:] == 5).all())
    dv = _np(d)
    want_dw = np.where(there, np.einsum("td,tkd->tk", dv, rows_of), 0)
    bound_dw = (D / 64 + 8) * 2.0 ** -23 * np.einsum("td,tkd->tk", np.abs(dv), np.abs(rows_of)) + 1e-40
    want_dy = (fw[:, :, None] * dv[:, None, :]).reshape(T * k, D)[rows[:total]]
    for src in (d.cuda(), _strided(d)):
        dy = torch.full((T * k, D + 3), 9.0, dtype=dtype, device="cuda")
        got, dw = daq.experts_combine_backward(src, y_nan.cuda(), plan, out=dy[:, 2:2 + D], **kw)
        assert np.all(np.abs(_np(dw) - want_dw) <= bound_dw)
        assert np.all(np.abs(_np(got)[:total] - want_dy) <= (2.0 ** -24 + (ulp if dtype == torch.bfloat16 else 0)) * np.abs(want_dy) + 1e-40)
        assert bool((dy[total:] == 9).all()) and bool((dy[:, :2] == 9).all()) and bool((dy[:, 2 + D:] == 9).all())
        only, none = daq.experts_combine_backward(src, None, plan, **kw)
        assert none is None and torch.equal(only[:total], got[:total])


def test_no_tokens_and_no_rows():
    empty = torch.empty(0, 2, dtype=torch.int32, device="cuda")
    plan = daq.experts_plan(empty, 5)
    assert plan.counts.tolist() == [0] * 5 and int(plan.table.abs().sum()) == 0
    w, t = daq.fp8_quantize_weights(torch.randn(5, 40, 70, device="cuda"))
    assert daq.experts_linear(torch.empty(0, 70, device="cuda"), w, plan).shape == (0, 40)
    assert daq.experts_combine(torch.empty(0, 9, device="cuda"), plan).shape == (0, 9)
    _, xc = daq.experts_quantize(torch.empty(0, 70, device="cuda"), plan)
    _, dc = daq.experts_quantize(torch.empty(0, 40, device="cuda"), plan, sorted_rows=True)
    assert bool((daq.experts_weight_grad(dc, xc, plan) == 0).all())
    assert daq.route(torch.empty(0, 5, device="cuda"), 2)[0].shape == (0, 2)
    # tokens, none of which has an expert
    plan = daq.experts_plan(torch.full((6, 2), -1, dtype=torch.int32, device="cuda"), 5)
    y = torch.full((12, 40), 4.0, device="cuda")
    assert bool((daq.experts_linear(torch.randn(6, 70, device="cuda"), w, plan, out=y) == 4).all())
    assert bool((daq.experts_combine(y, plan) == 0).all())
    _, xc = daq.experts_quantize(torch.randn(6, 70, device="cuda"), plan)
    _, dc = daq.experts_quantize(torch.randn(12, 40, device="cuda"), plan, sorted_rows=True)
    assert bool((daq.experts_weight_grad(dc, xc, plan) == 0).all())


def test_the_same_bits_every_time():
    c = _chosen(700, 4, 16, 1, none=0.05)
    w, t = daq.fp8_quantize_weights(torch.randn(16, 300, 400, device="cuda"))
    x, d = torch.randn(700, 400, device="cuda").bfloat16(), torch.randn(2800, 300, device="cuda").bfloat16()

    def once():
        plan = daq.experts_plan(c.cuda(), 16)
        n = int(plan.counts.sum())
        _, xc = daq.experts_quantize(x, plan)
        _, dc = daq.experts_quantize(d, plan, sorted_rows=True)
        y = daq.experts_linear(x, w, plan)[:n]
        full = torch.zeros(2800, 300, device="cuda", dtype=torch.bfloat16)
        full[:n] = y
        return plan.rows, y, daq.experts_weight_grad(dc, xc, plan), daq.experts_combine(full, plan, torch.ones(700, 4, device="cuda"))

    first = once()
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(first, once()))


@pytest.mark.parametrize("E,k", [(40, 3), (300, 12), (520, 20)])
@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
def test_router_of_many_tokens(E, k, kind):
    """Tokens enough for a wave to take several backwards; their number leaves the last wave some."""
    T = 8197
    logits = torch.randn(T, E, generator=torch.Generator().manual_seed(E))
    logits[77] = -torch.inf
    g = torch.randn(T, k, generator=torch.Generator().manual_seed(k))
    for renormalize in (True, False):
        s = ref.scores(_np(logits), kind)
        chosen = np.argsort(-np.where(np.isneginf(_np(logits)), -np.inf, _np(logits)), axis=1, kind="stable")[:, :k]
        chosen[77] = -1
        w, e = daq.route(logits.cuda(), k, KIND[kind], renormalize=renormalize)
        assert np.array_equal(_np(e), chosen)
        take = np.where(chosen >= 0, np.take_along_axis(s, np.maximum(chosen, 0), 1), 0)
        total = np.where(chosen[:, :1] >= 0, take.sum(1, keepdims=True), 1.0) if renormalize else np.ones((T, 1))
        assert np.all(np.abs(_np(w) - take / total) <= (2.0 ** -24 + 2.0 ** -48) * take / total + 2.0 ** -149)
        want = ref.route_backward(_np(g), _np(logits), chosen, kind, renormalize)
        got = _np(daq.route_backward(g.cuda(), logits.cuda(), e, KIND[kind], renormalize))
        size = np.abs(want) + s * np.abs(_np(g)).sum(1, keepdims=True) * (1.0 if not renormalize else 2.0 ** -20 / total)
        assert np.all(np.abs(got - want) <= (E / 64 + k + 30) * 2.0 ** -24 * size + 1e-37)


@pytest.mark.parametrize("T", [5, 8200])
@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
def test_a_token_that_names_an_expert_twice(T, kind):
    """Each place counts, in the gradient, in the order of the rows and in the sum."""
    logits, g = torch.randn(T, 12, generator=torch.Generator().manual_seed(1)), torch.randn(T, 4, generator=torch.Generator().manual_seed(2))
    chosen = torch.randint(0, 12, (T, 4), generator=torch.Generator().manual_seed(3)).int()
    chosen[:, 2], chosen[1] = chosen[:, 0], 7
    for renormalize in (True, False):
        want = ref.route_backward(_np(g), _np(logits), _np(chosen).astype(int), kind, renormalize)
        got = _np(daq.route_backward(g.cuda(), logits.cuda(), chosen.cuda(), KIND[kind], renormalize))
        # the places of an expert are added in 32 bits: parts of up to its share of the chosen ones' scores, times the weights' gradients
        s = ref.scores(_np(logits), kind)
        share = s / np.take_along_axis(s, _np(chosen).astype(int), 1).sum(1, keepdims=True) if renormalize else s
        assert np.all(np.abs(got - want) <= 50 * 2.0 ** -24 * (np.abs(want) + share * np.abs(_np(g)).sum(1, keepdims=True)) + 1e-37)
    plan = daq.experts_plan(chosen.cuda(), 12)
    _, _, rows, place = ref.plan(chosen.numpy(), 12)
    assert np.array_equal(_np(plan.rows), rows) and np.array_equal(_np(plan.place), place)


def test_all_tokens_of_one_expert():
    """The longest run that a plan can have, among experts without rows; few experts' rows in a wide matrix."""
    c = torch.full((3000, 1), 5, dtype=torch.int32)
    plan = daq.experts_plan(c.cuda(), 64)
    assert plan.counts[5] == 3000 and plan.table[1, -1] == 12 and plan.table[2, -1] == 24
    x, w = torch.randn(3000, 256), torch.randn(64, 512, 256)
    qw, _ = daq.fp8_quantize_weights(w.cuda())
    got = _np(daq.experts_linear(x.cuda(), qw, plan, dtype=torch.float32))
    vx, vw = ref.values(*ref.quantize(_np(x))), ref.values(*ref.quantize_weights(_np(w[5])))
    assert np.all(np.abs(got - vx @ vw.T) <= _bound(256, np.abs(vx) @ np.abs(vw).T, vx @ vw.T, torch.float32))
    few = torch.tensor([[63], [0], [63]], dtype=torch.int32).cuda()
    got = _np(daq.experts_linear(x[:3].cuda(), qw, daq.experts_plan(few, 64), dtype=torch.float32))
    for p, (t, e) in enumerate(((1, 0), (0, 63), (2, 63))):
        vw = ref.values(*ref.quantize_weights(_np(w[e])))
        assert np.all(np.abs(got[p] - vw @ vx[t]) <= _bound(256, np.abs(vw) @ np.abs(vx[t]), vw @ vx[t], torch.float32))


@pytest.mark.parametrize("sorted_rows", [False, True])
def test_large_products_of_experts(sorted_rows):
    """Tiles of 256 x 256 of uneven experts, more of them than CUs, rows of whole 16-byte pieces; and their gradients."""
    T, k, E, N, K = 9000, 2, 10, 2048, 264
    c = _chosen(T, k, E - 1, 3, none=0.02, skew=0.3)                       # the last one has no rows
    plan = daq.experts_plan(c.cuda(), E)
    counts, table, rows, place = ref.plan(c.numpy(), E)
    total, ends = int(counts.sum()), np.cumsum(counts)
    a = torch.randn(T * k if sorted_rows else T, K, generator=torch.Generator().manual_seed(1)).bfloat16()
    w = torch.randn(E, N, K, generator=torch.Generator().manual_seed(2)).bfloat16()
    qw, _ = daq.fp8_quantize_weights(w.cuda())
    va = ref.values(*ref.quantize(_np(a)))
    out = torch.full((T * k, N), 7.0, dtype=torch.bfloat16, device="cuda")
    y = _np(daq.experts_linear(a.cuda(), qw, plan, sorted_rows=sorted_rows, out=out))
    d = torch.randn(T * k, N, generator=torch.Generator().manual_seed(3)).bfloat16()
    _, ac = daq.experts_quantize(a.cuda(), plan, sorted_rows=sorted_rows)
    _, dc = daq.experts_quantize(d.cuda(), plan, sorted_rows=True)
    grads = {to: _np(daq.experts_weight_grad(dc, ac, plan, dtype=to)) for to in DT}
    for e in range(E):
        here = slice(ends[e] - counts[e], ends[e])
        r = va[here] if sorted_rows else va[rows[here] // k]
        vw = ref.values(*ref.quantize_weights(_np(w[e])))
        assert np.all(np.abs(y[here] - r @ vw.T) <= _bound(K, np.abs(r) @ np.abs(vw).T, r @ vw.T, torch.bfloat16))
        r = _np(a)[here] if sorted_rows else _np(a)[rows[here] // k]
        vd, vx = ref.values(*ref.quantize(_np(d)[here].T)), ref.values(*ref.quantize(r.T))
        for to in DT:
            assert np.all(np.abs(grads[to][e] - vd @ vx.T) <= _bound(int(counts[e]), np.abs(vd) @ np.abs(vx).T, vd @ vx.T, to))
    assert bool((out[total:] == 7).all())


@pytest.mark.parametrize("D,ld", [(4096, 4096), (4090, 4096), (4100, 4100)])
def test_sums_of_many_rows(D, ld):
    """256 MiB and more of experts' rows, some of them behind the last one, the rows' ends inside a lane's eight columns too."""
    T, k, E = 8400, 4, 8
    plan = daq.experts_plan(_chosen(T, k, E, 5).cuda(), E)
    y, dout = torch.randn(T * k, ld, device="cuda", dtype=torch.bfloat16)[:, :D], torch.randn(T, D, device="cuda", dtype=torch.bfloat16)
    w = torch.rand(T, k, device="cuda")
    dy = torch.full((T * k, ld), 7.0, device="cuda", dtype=torch.bfloat16)
    out = daq.experts_combine(y, plan, w)
    _, dw = daq.experts_combine_backward(dout, y, plan, w, out=dy[:, :D])
    n = int(plan.counts.sum())
    assert bool((dy[n:] == 7).all()) and bool((dy[:, D:] == 7).all())
    for first in range(0, T, 1050):                                        # in parts: 64 bits take memory
        part = slice(first, first + 1050)
        place, there = plan.place[part].long(), plan.place[part] >= 0
        rows = torch.where(there[..., None], y[place.clamp(min=0)].double(), 0.0)
        terms = w[part].double()[..., None] * rows
        want, size = terms.sum(1), terms.abs().sum(1)
        assert bool(((out[part].double() - want).abs() <= 2.0 ** -8 * want.abs() + (k + 1) * 2.0 ** -24 * size * (1 + 2.0 ** -8)).all())
        d = dout[part].double()[:, None]
        assert bool((((rows * d).sum(2) - dw[part].double()).abs() <= (-(-D // 512) * 8 + 7) * 2.0 ** -24 * (rows * d).abs().sum(2)).all())
        g = w[part].double()[..., None] * d
        assert bool(((dy[place.clamp(min=0)][:, :, :D].double() - g).abs() <= (2.0 ** -8 + 2.0 ** -23) * g.abs())[there].all())
