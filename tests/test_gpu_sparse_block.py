"""The sparse feed-forward block on the GPU: every call it makes, forwards and backwards, against the oracle in 64 bits on the values that the block passes
to it; the whole of it in another form, on another stream and in a graph."""
import numpy as np
import pytest
import torch

from oracle import fp8 as ref
from paper_2102_04782_amd import binding as daq
from paper_2102_04782_amd.experts import SparseFeedForward
from test_gpu_fp8 import _bound, _np

pytestmark = pytest.mark.gpu


def _held(q):
    """The values of a matrix by rows, from its bytes by the layout's formulas."""
    L, buf = daq.layout_fp8(q.rows, q.cols), q.buf.cpu().numpy()
    codes = buf[:q.rows * L.pitch].reshape(q.rows, L.pitch)[:, :q.cols]
    byte = np.array([[buf[L.off_scales + ((b // 4) * q.rows + r) * 4 + b % 4] for b in range(-(-q.cols // 128))] for r in range(q.rows)], np.int64)
    return ref.values(codes, byte.reshape(q.rows, -1))


def _close(got, want, absolute, terms, dtype):
    got = _np(got)[:want.shape[0]]
    assert np.all(np.abs(got - want) <= _bound(terms, absolute, want, dtype))


class Calls:
    """Stands in for the binding and keeps what went through it."""

    def __init__(self):
        self.made = []

    def __getattr__(self, name):
        real = getattr(daq, name)
        if not callable(real) or isinstance(real, type):
            return real

        def call(*a, **k):
            out = real(*a, **k)
            self.made.append((name, a, k, out.clone() if torch.is_tensor(out) else out))     # (what the block adds to it comes later)
            return out

        return call


@pytest.fixture
def calls(monkeypatch):
    from paper_2102_04782_amd import experts

    c = Calls()
    monkeypatch.setattr(experts, "daq", c)
    return c


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,d,f,E,k,groups,top", [(1, 130, 64, 4, 2, 1, 1), (37, 200, 130, 8, 3, 4, 2), (150, 256, 96, 6, 2, 1, 1)])
def test_every_call_of_the_block(calls, T, d, f, E, k, groups, top, dtype):
    block = SparseFeedForward(d, f, E, k, groups, top, seed=5)
    block.bias = 0.05 * torch.randn(E, generator=torch.Generator().manual_seed(1)).cuda()
    x = torch.randn(T, d, generator=torch.Generator().manual_seed(2)).to(dtype).cuda()
    calls.made.clear()
    y, saved = block.forward(x)
    g = block.backward(torch.randn(T, d, generator=torch.Generator().manual_seed(3)).to(dtype).cuda(), saved)
    counts, table, rows, place = ref.plan(_np(saved.chosen).astype(int), E)
    assert np.array_equal(_np(saved.plan.counts), counts) and np.array_equal(_np(saved.plan.place), place)
    total, expert, ends = int(counts.sum()), np.repeat(np.arange(E), counts), np.cumsum(counts)
    seen = set()
    for name, a, kw, out in calls.made:
        seen.add(name)
        if name == "fp8_linear":
            vx, vw = ref.values(*ref.quantize(_np(a[0]))), _held(a[1])
            _close(out, vx @ vw.T, np.abs(vx) @ np.abs(vw).T, d, torch.float32)
        elif name == "route":
            w, c = ref.route(_np(a[0]), k, "sigmoid", _np(kw["bias"]), groups, top)
            assert np.array_equal(_np(out[1]), c) and np.all(np.abs(_np(out[0]) - w) <= 2.0 ** -23 * np.abs(w))
        elif name == "experts_matmul":
            A, w = _held(a[0]), _held(a[1]).reshape(E, -1, a[1].cols)
            A = A[:total] if kw.get("sorted_rows") else A[rows[:total] // k]
            want = np.stack([w[e] @ v for e, v in zip(expert, A)])
            _close(out, want, np.stack([np.abs(w[e]) @ np.abs(v) for e, v in zip(expert, A)]), a[0].cols, dtype)
        elif name == "experts_combine":
            w = _np(a[2]) if len(a) > 2 else np.ones((T, k))
            r = _np(a[0])[place]
            want, absolute = np.einsum("tk,tkd->td", w, r), np.einsum("tk,tkd->td", np.abs(w), np.abs(r))
            assert np.all(np.abs(_np(out) - want) <= k * 2.0 ** -23 * absolute + (2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24) * np.abs(want) + 1e-40)
        elif name == "experts_combine_backward":
            want = np.einsum("td,tkd->tk", _np(a[0]), _np(a[1])[place])
            size = np.einsum("td,tkd->tk", np.abs(_np(a[0])), np.abs(_np(a[1])[place]))
            assert np.all(np.abs(_np(out[1]) - want) <= (d / 64 + 8) * 2.0 ** -23 * size)
            want = (_np(a[3])[:, :, None] * _np(a[0])[:, None]).reshape(T * k, d)[rows]
            assert np.all(np.abs(_np(out[0]) - want) <= (2.0 ** -24 + (2.0 ** -8 if dtype == torch.bfloat16 else 0)) * np.abs(want) + 1e-40)
        elif name == "route_backward":
            want = ref.route_backward(_np(a[0]), _np(a[1]), _np(a[2]).astype(int), "sigmoid")
            s, own = ref.scores(_np(a[1]), "sigmoid"), np.abs(_np(a[0])).sum(1, keepdims=True)
            assert np.all(np.abs(_np(out) - want) <= 2.0 ** -23 * (np.abs(want) + s * own * 2.0 ** -20) + 1e-40)
        elif name == "fp8_matmul":
            va, vb = _held(a[0]), _held(a[1])
            _close(out, va @ vb.T, np.abs(va) @ np.abs(vb).T, a[0].cols, out.dtype)
        elif name == "experts_weight_grad":
            va, vb = _held(a[0]), _held(a[1])
            for e in range(E):
                span = slice(table[2, e] * 128, table[2, e + 1] * 128)
                with np.errstate(invalid="ignore"):
                    want, size = va[:, span] @ vb[:, span].T, np.abs(va[:, span]) @ np.abs(vb[:, span]).T
                _close(out[e], want, size, counts[e] + 128, torch.float32)
        elif name in ("experts_quantize", "fp8_quantize", "fp8_quantize_both"):
            if name == "experts_quantize":
                assert np.array_equal(_held(out[0])[:total], ref.values(*ref.quantize(_np(a[0])))[:total])
                v, r = _held(out[1]), _np(a[0])[:total] if kw.get("sorted_rows") else _np(a[0])[rows[:total] // k]
                for e in range(E):
                    n, first = counts[e], ends[e] - counts[e]
                    if n:
                        assert np.array_equal(v[:, table[2, e] * 128:][:, :n], ref.values(*ref.quantize(r[first:first + n].T)))
    assert {"fp8_linear", "route", "experts_plan", "experts_quantize", "experts_matmul", "experts_combine", "experts_combine_backward", "experts_weight_grad",
            "route_backward", "fp8_matmul", "fp8_quantize", "fp8_quantize_both"} <= seen
    assert g.w_in.shape == block.w_in.shape and g.w_out.shape == block.w_out.shape and g.w_router.shape == block.w_router.shape and g.x.shape == x.shape
    # served: the same products, of rows quantized on the way
    assert torch.equal(block.serve(x), y)


def test_the_block_runs_and_its_gradients_are_those_of_each_update():
    from paper_2102_04782_amd import experts

    experts.main(d=64, f=32, experts=4, picks=2, tokens=96, steps=2)
    block = SparseFeedForward(64, 32, 4, 2)
    x = torch.randn(50, 64, device="cuda").bfloat16()
    y, s = block.forward(x)
    g = block.backward(torch.ones_like(y), s)
    before = block.w_in.clone()
    block.update(g, 0.5)
    assert torch.equal(block.w_in, before - 0.5 * g.w_in) and not torch.equal(block.forward(x)[0], y)
    bias = block.bias.clone()
    block.balance(s.plan, 0.25)
    assert torch.equal(block.bias - bias, 0.25 * torch.sign(s.plan.counts.float().mean() - s.plan.counts.float()))


@pytest.mark.parametrize("T,dtype", [(2, torch.bfloat16), (300, torch.bfloat16), (300, torch.float32)])
def test_a_step_in_a_graph_replays_with_other_tokens(T, dtype):
    """Forwards and backwards captured into one graph: every replay against the eager result on the same tokens, the experts' rows another number each time."""
    block = SparseFeedForward(256, 128, 8, 2, seed=4)
    x, dout = torch.zeros(T, 256, dtype=dtype, device="cuda"), torch.zeros(T, 256, dtype=dtype, device="cuda")

    def step():
        y, s = block.forward(x)
        g = block.backward(dout, s)
        return y, g.x, g.w_router, g.w_in, g.w_out, s.plan.counts

    x.normal_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for n in range(4):
        x.normal_(generator=torch.Generator(device="cuda").manual_seed(n))
        dout.normal_(generator=torch.Generator(device="cuda").manual_seed(100 + n))
        graph.replay()
        torch.cuda.synchronize()
        kept = [t.clone() for t in captured]
        for a, b in zip(kept, step()):
            assert torch.equal(a, b)


def test_another_stream_than_the_current_one():
    block = SparseFeedForward(256, 128, 8, 2, seed=4)
    x = torch.randn(200, 256, device="cuda").bfloat16()
    want = block.forward(x)[0]
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    w, e = daq.route(daq.fp8_linear(x, block.q_router, dtype=torch.float32, stream=st), 2, bias=block.bias, stream=st, **block.form)
    plan = daq.experts_plan(e, 8, stream=st)
    xq, xc = daq.experts_quantize(x, plan, stream=st)
    a, _ = daq.ckpt8_act_forward(daq.experts_matmul(xq, block.q_in, plan, stream=st), daq.ACT_SILU, gated=True, stream=st)
    y = daq.experts_linear(a, block.q_out, plan, sorted_rows=True, stream=st)
    out = daq.experts_combine(y, plan, w, stream=st)
    st.synchronize()
    assert torch.equal(out, want)


def test_two_calls_at_once_on_two_streams():
    """Workspaces belong to their calls: the same products on two streams, their launches one among the other."""
    a = [torch.randn(700, 1000, device="cuda") for _ in range(2)]
    w = [daq.fp8_quantize_weights(torch.randn(600, 1000, device="cuda"))[0] for _ in range(2)]
    want = [daq.fp8_linear(a[i], w[i]) for i in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for _ in range(10):
        for i in range(2):
            got[i].append(daq.fp8_linear(a[i], w[i], stream=streams[i]))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want[i]) for i in range(2) for o in got[i])


def test_two_graphs_in_turn():
    """Sums in parts and plans of many workgroups, whose workspaces are each graph's own: replayed in turn on other inputs, with eager calls between."""
    def step(a, b, chosen):
        qa, qb = daq.fp8_quantize(a), daq.fp8_quantize(b)
        plan = daq.experts_plan(chosen, 24)
        return daq.fp8_matmul(qa, qb), daq.fp8_matmul(qa, qb, dtype=torch.float32), plan.counts, plan.table, plan.rows, plan.place

    graphs = []
    for _ in range(2):
        ins = (torch.randn(130, 5000, device="cuda"), torch.randn(70, 5000, device="cuda"), torch.zeros(9000, 4, dtype=torch.int32, device="cuda"))
        step(*ins)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs = step(*ins)
        graphs.append((ins, graph, outs))
    for n in range(3):
        for seed, (ins, _, _) in enumerate(graphs):
            g = torch.Generator(device="cuda").manual_seed(10 * n + seed)
            ins[0].normal_(generator=g)
            ins[1].normal_(generator=g)
            ins[2].random_(-1, 24, generator=g)
        for _, graph, _ in graphs:
            graph.replay()
        torch.cuda.synchronize()
        kept = [[t.clone() for t in outs] for _, _, outs in graphs]
        for (ins, _, _), got in zip(graphs, kept):
            assert all(torch.equal(a, b) for a, b in zip(got, step(*ins)))
