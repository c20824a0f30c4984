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


def test_the_longest_sums_and_the_farthest_rows():
    """K up to 2^23 - 128 (columns of an experts' weight gradient as well), rows taken by their tokens up to 2^32 - 256 bytes of codes."""
    L, n = daq.lib(), C.c_size_t(0)
    most = (1 << 23) - 128
    for dtype in (daq.FP32, daq.BF16):
        assert L.daq_fp8_matmul_workspace(4, 8, most, dtype, C.byref(n)) == daq.OK
        assert L.daq_fp8_linear_workspace(4, 8, most, dtype, dtype, C.byref(n)) == daq.OK
        for K in (most + 1, 1 << 23):
            assert L.daq_fp8_matmul_workspace(4, 8, K, dtype, C.byref(n)) == UNS and n.value == 0
            assert L.daq_fp8_matmul(4, 8, K, A, A, A, dtype, 8, 0, A, 1 << 60, None) == UNS
            assert L.daq_fp8_linear(4, 8, K, A, dtype, K, A, A, dtype, 8, A, 1 << 60, None) == UNS
            for sorted_rows in (0, 1):
                assert L.daq_experts_matmul(C.byref(daq.Experts(4, 2, 8, A, A, A)), 8, K, A, sorted_rows, A, A, dtype, 8, None) == UNS
    # weight gradients: as many rows of one expert, or one more
    for tokens, fits in ((most, True), (most + 1, False)):
        plan = daq.Experts(tokens, 1, 1, A, A, A)
        columns = C.c_int64(0)
        assert L.daq_experts_columns(tokens, 1, 1, C.byref(columns)) == daq.OK and (columns.value <= most) == fits
        if not fits:
            assert L.daq_experts_weight_grad(C.byref(plan), 8, 40, A, A, A, daq.FP32, 40, 320, 0, None) == UNS
    for tokens, K, fits in (((1 << 22) - 1, 1024, True), (1 << 22, 1024, False), (1 << 25, 1, False), ((1 << 25) - 2, 1, True)):
        plan = daq.Experts(tokens, 1, 4, A, A, A)
        assert L.daq_experts_linear_workspace(C.byref(plan), 8, K, daq.BF16, 0, C.byref(n)) == (daq.OK if fits else UNS)
        assert L.daq_experts_linear_workspace(C.byref(plan), 8, K, daq.BF16, 1, C.byref(n)) == daq.OK
        if not fits:
            assert L.daq_experts_linear(C.byref(plan), 8, K, A, daq.BF16, K, 0, A, A, daq.BF16, 8, A, 1 << 60, None) == UNS
