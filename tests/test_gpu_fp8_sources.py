"""Sources on either side of the sizes from which on, and up to which, they are read past the caches: the same codes and scales, whichever way."""
import pytest
import torch

from paper_2102_04782_amd import binding as daq

pytestmark = pytest.mark.gpu


def _equal(a, b):
    """The defined bytes of two packed matrices of one size."""
    L = daq.layout_fp8(a.rows, a.cols)
    for first, n in ((0, a.rows * L.pitch), (L.off_scales, -(-a.cols // 512) * a.rows * 4)):
        assert torch.equal(a.buf[first:first + n], b.buf[first:first + n])


@pytest.mark.parametrize("rows,cols", [(12287, 8192), (12288, 8192), (20479, 8192), (20480, 8192), (49151, 8192), (49152, 8192)])
def test_sources_around_the_sizes_that_pass_the_caches(rows, cols):
    """96, 160 and 384 Mi elements and a row less, in one call and in two; rows that begin off a line are never read past the caches."""
    x = torch.randn(rows, cols, device="cuda", dtype=torch.bfloat16)
    by_rows, by_columns = daq.fp8_quantize_both(x)
    _equal(daq.fp8_quantize(x), by_rows)
    _equal(daq.fp8_quantize(x, columns=True), by_columns)
    wide = torch.empty(rows, cols + 1, device="cuda", dtype=torch.bfloat16)[:, 1:]
    wide.copy_(x)
    del x
    _equal(daq.fp8_quantize(wide), by_rows)
    _equal(daq.fp8_quantize(wide, columns=True), by_columns)


@pytest.mark.parametrize("tokens", [12288, 20480])
def test_rows_of_experts_around_the_sizes_that_pass_the_caches(tokens):
    """96 and 160 Mi elements in the order of their experts; taken by their tokens they are read as they come."""
    plan = daq.experts_plan(torch.topk(torch.randn(tokens, 8, device="cuda"), 2, dim=1).indices.int(), 8)
    x = torch.randn(tokens, 4096, device="cuda", dtype=torch.bfloat16)
    in_order = x[plan.rows.long() // 2]
    _, by_token = daq.experts_quantize(x, plan)
    by_rows, by_columns = daq.experts_quantize(in_order, plan, sorted_rows=True)
    _equal(daq.fp8_quantize(in_order), by_rows)
    # the blocks that the experts have (those behind them are left as they were)
    blocks = int(plan.table[2, -1])
    L = daq.layout_fp8(4096, by_columns.cols)
    codes = lambda q: q.buf[:4096 * L.pitch].view(4096, L.pitch)[:, :blocks * 128]
    assert torch.equal(codes(by_columns), codes(by_token))
    scales = lambda q: q.buf[L.off_scales:L.off_scales + -(-by_columns.cols // 512) * 4096 * 4].view(-1, 4096, 4).transpose(1, 2).reshape(-1, 4096)[:blocks]
    assert torch.equal(scales(by_columns), scales(by_token))
