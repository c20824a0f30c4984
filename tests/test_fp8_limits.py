"""Limits of the 8-bit floating point layers, the router and the experts' products: what goes beyond them is refused before anything is launched.
Addresses are never read: every call here is refused."""
import ctypes as C

from paper_2102_04782_amd import binding as daq

A, UNS = 1 << 20, daq.ERR_UNSUPPORTED


def test_routers_of_more_tokens_than_a_launch_takes():
    """A workgroup of 256 threads takes 4 tokens (backwards 4, 8 or 16 of them), and a launch fewer than 2^32 threads."""
    L = daq.lib()

    def forward(T, E=8, k=2, dtype=daq.FP32):
        return L.daq_route(T, E, A, dtype, E, None, C.byref(daq.RouteOpts(0, k, 1, 1, 1, 1.0)), A, A, None)

    def backward(T, E=8, k=2, dtype=daq.FP32):
        return L.daq_route_backward(T, E, A, A, dtype, E, A, C.byref(daq.RouteOpts(0, k, 1, 1, 1, 1.0)), A, E, None)

    for dtype in (daq.FP32, daq.BF16):
        for T in ((1 << 26) - 3, 1 << 26, (1 << 28) - 1, 1 << 28):
            assert forward(T, dtype=dtype) == UNS, T
        for T, k in (((1 << 28) - 1, 2), ((1 << 28) - 15, 16), ((1 << 27) - 7, 17), (1 << 27, 32), (1 << 28, 2)):
            assert backward(T, 64, k, dtype) == UNS, (T, k)


def test_layers_whose_product_is_too_large_are_refused_as_it_is():
    """The product's limits are those of the call that quantizes X on the way to it: nothing is launched before they are known."""
    L, n = daq.lib(), C.c_size_t(0)
    M = N = 1 << 20                                        # more tiles than can be counted
    for dtype in (daq.FP32, daq.BF16):
        for x_dtype in (daq.FP32, daq.BF16):
            assert L.daq_fp8_matmul(M, N, 128, A, A, A, dtype, N, 0, A, 1 << 60, None) == UNS
            assert L.daq_fp8_matmul_workspace(M, N, 128, dtype, C.byref(n)) == UNS and n.value == 0
            assert L.daq_fp8_linear(M, N, 128, A, x_dtype, 128, A, A, dtype, N, A, 1 << 60, None) == UNS
            assert L.daq_fp8_linear_workspace(M, N, 128, x_dtype, dtype, C.byref(n)) == UNS and n.value == 0
    assert L.daq_fp8_matmul(M, N, 0, None, None, A, daq.FP32, N, 0, None, 0, None) == UNS
    plan = C.byref(daq.Experts(1 << 20, 8, 64, A, A, A))
    for sorted_rows, K in ((0, 128), (1, 512)):
        for dtype in (daq.FP32, daq.BF16):
            assert L.daq_experts_matmul(plan, 1 << 17, K, A, sorted_rows, A, A, dtype, 1 << 17, None) == UNS
            assert L.daq_experts_linear(plan, 1 << 17, K, A, daq.BF16, K, sorted_rows, A, A, dtype, 1 << 17, A, 1 << 60, None) == UNS
