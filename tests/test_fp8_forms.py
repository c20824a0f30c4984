"""Forms of 8-bit products, by the workspaces that they ask for: the few-rows form needs none, tiles need one at the
sizes here, for the parts of the summed axis."""
import ctypes as C

from paper_2102_04782_amd import binding as daq


def test_few_rows_of_wide_layers_take_tiles():
    """Where these were measured to be faster, by rows, elements of the weights and type of the result."""
    L, n = daq.lib(), C.c_size_t(0)
    for M, N, K, few in ((1, 8192, 8192, (1, 1)), (8, 8192, 8192, (1, 1)), (9, 8192, 8192, (0, 1)), (16, 4096, 8192, (1, 1)), (16, 4096, 8320, (0, 1)), (17, 8192, 8192, (0, 0)),
                         (24, 4096, 4096, (1, 1)), (24, 4096, 4224, (0, 1)), (32, 4096, 8192, (0, 1)), (32, 4096, 8320, (0, 0)), (24, 2300, 5130, (1, 1)), (33, 4096, 4096, (0, 0))):
        for dtype, want in zip((daq.BF16, daq.FP32), few):
            assert L.daq_fp8_matmul_workspace(M, N, K, dtype, C.byref(n)) == daq.OK
            assert (n.value == 0) == bool(want), (M, N, K, dtype)
