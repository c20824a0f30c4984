"""Experts' rows taken by their tokens at the end of what a descriptor reaches: 2^32 - 256 bytes of codes."""
import numpy as np
import pytest
import torch

from oracle import fp8 as ref
from paper_2102_04782_amd import binding as daq
from test_gpu_fp8 import DT, _bound, _np

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens,K,N", [((1 << 22) - 1, 1024, 72), ((1 << 22) - 1, 1024, 520), ((1 << 25) - 2, 100, 8)])
def test_rows_at_the_end_of_a_descriptor(tokens, K, N):
    """The first and the last tokens' rows, on tiles of every size, among millions of others of the same experts."""
    E = 4
    x = torch.full((tokens, K), 0.5, device="cuda", dtype=torch.bfloat16)
    ends = torch.cat((torch.arange(40), torch.arange(tokens - 40, tokens)))
    x[ends.cuda()] = torch.randn(80, K, device="cuda").bfloat16()
    w = torch.randn(E, N, K, generator=torch.Generator().manual_seed(1))
    qw, _ = daq.fp8_quantize_weights(w.cuda())
    chosen = (torch.arange(tokens, device="cuda", dtype=torch.int32) * 7 % E).view(-1, 1)
    plan = daq.experts_plan(chosen, E)
    at, e = plan.place[ends.cuda(), 0].long(), chosen[ends.cuda(), 0].tolist()
    vx = ref.values(*ref.quantize(_np(x[ends.cuda()])))
    vw = np.stack([ref.values(*ref.quantize_weights(_np(m))) for m in w])
    exact, absolute = np.einsum("tk,tnk->tn", vx, vw[e]), np.einsum("tk,tnk->tn", np.abs(vx), np.abs(vw[e]))
    qx = daq.fp8_quantize(x)
    for to in DT:
        got = _np(daq.experts_matmul(qx, qw, plan, dtype=to)[at])
        assert np.all(np.abs(got - exact) <= _bound(K, absolute, exact, to))
        assert np.array_equal(got, _np(daq.experts_linear(x, qw, plan, dtype=to)[at]))
