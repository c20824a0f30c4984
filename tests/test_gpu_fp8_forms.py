"""Products of few rows on either side of the sizes from which on they take tiles."""
import numpy as np
import pytest
import torch

from paper_2102_04782_amd import binding as daq
from test_gpu_fp8 import DT, _bound, _np, _x

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N,K", [(4096, 4096), (4096, 4224), (4096, 8192), (8000, 8300), (12288, 4096)])
def test_few_rows_of_wide_layers(N, K):
    w = daq.fp8_quantize(_x(N, K, torch.bfloat16, N).cuda())
    vw = daq.fp8_dequantize(w).double()
    for M in (1, 8, 9, 16, 17, 31, 32, 33):
        x = _x(M, K, torch.bfloat16, M + K).cuda()
        q = daq.fp8_quantize(x)
        v = daq.fp8_dequantize(q).double()
        exact, absolute = _np(v @ vw.T), _np(v.abs() @ vw.abs().T)
        for to in DT:
            first = daq.fp8_matmul(q, w, dtype=to)
            assert np.all(np.abs(_np(first) - exact) <= _bound(K, absolute, exact, to)), (M, to)
            assert torch.equal(first, daq.fp8_linear(x, w, dtype=to))
