// Products of microscaled 4-bit matrices, D[m][n] = sum over k of A[m][k] * B[n][k], and linear layers on them.
//
// The matrix instruction of 32 x 32 x 64 takes of each operand a block of 32 elements a lane (16 bytes and a scale byte): lane l has
// row l % 32 and block l / 32 of the 64 columns.  The packed layout holds operands in that order, so a wave loads a 32 x 64 tile
// as one contiguous KiB and the scale bytes of four tiles as one contiguous 256 bytes.  B goes in as the instruction's first
// operand, so that a lane holds four neighbouring columns of a row of D at a time.
#include "tile_product.h"

namespace daq {

namespace {

struct MatmulArgs {
    const uint8_t* a;       // codes
    const uint8_t* a_scales;
    const uint8_t* b;
    const uint8_t* b_scales;
    int64_t M, N;
    int a_blocks, b_blocks;   // row blocks of 32
    int groups;               // 256 columns each
    int steps;                // 64 columns each, of the ones that hold an element
    void* d;
    int64_t ldd;
    int bf16;
};

// Tiles of 32 RB WR x 32 CB WC results, a workgroup each.  Workgroup b runs on XCD b % 8; an XCD takes an eighth of the tiles, in bands
// of four row tiles, so that the 32 it holds at a time share twelve panels of the operands in its L2.
template <int WR, int WC, int RB, int CB>
__global__ __launch_bounds__(64 * WR * WC, 1) void k_mx4_tiles(MatmulArgs p, int tiles_m, int tiles_n, int per_xcd) {
    using Product = TileProduct<WR, WC, RB, CB, true>;
    extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
    const int64_t t = (int64_t)(blockIdx.x % kXcd) * per_xcd + blockIdx.x / kXcd;
    if (t >= (int64_t)tiles_m * tiles_n) return;
    const int64_t band = t / (4 * tiles_n);
    const int rest = (int)(t - band * 4 * tiles_n), high = min(4, tiles_m - (int)band * 4);
    const int tm = (int)band * 4 + rest % high, tn = rest / high;
    const TileOperand r{p.a, p.a_scales, p.a_blocks, p.groups * 4}, c{p.b, p.b_scales, p.b_blocks, p.groups * 4};
    Product prod;
    prod.run(r, c, tm * WR * RB, tn * WC * CB, 0, p.groups, p.groups, lds, lds + Product::kStageBytes);
    const int wave = threadIdx.x / kWave;
    const int64_t m0 = ((int64_t)tm * WR + wave / WC) * RB * 32, n0 = ((int64_t)tn * WC + wave % WC) * CB * 32;
    if (p.bf16) {
        prod.store(true, lds, [&](int row, int col, u32x4 v) {
            const int64_t m = m0 + row, n = n0 + col;
            if (m >= p.M || n >= p.N) return;
            uint16_t* z = static_cast<uint16_t*>(p.d) + m * p.ldd + n;
            if (n + 8 <= p.N) {
                *reinterpret_cast<u32x4_a2*>(z) = v;
            } else {
#pragma unroll
                for (int i = 0; i < 7; ++i)
                    if (n + i < p.N) z[i] = (uint16_t)(v[i / 2] >> (16 * (i & 1)));
            }
        });
    } else {
        prod.store(false, lds, [&](int row, int col, u32x4 v) {
            const int64_t m = m0 + row, n = n0 + col;
            if (m >= p.M || n >= p.N) return;
            uint32_t* z = static_cast<uint32_t*>(p.d) + m * p.ldd + n;
            if (n + 4 <= p.N) {
                *reinterpret_cast<u32x4_a4*>(z) = v;
            } else {
#pragma unroll
                for (int i = 0; i < 3; ++i)
                    if (n + i < p.N) z[i] = v[i];
            }
        });
    }
}

template <int WR, int WC, int RB, int CB>
daq_status launch_tiles(const MatmulArgs& p, hipStream_t st) {
    using Product = TileProduct<WR, WC, RB, CB, true>;
    const int64_t tm = ceil_div(p.a_blocks, WR * RB), tn = ceil_div(p.b_blocks, WC * CB), per = ceil_div(tm * tn, kXcd);
    if (!grid_ok(per * kXcd)) return DAQ_ERR_UNSUPPORTED;
    const auto kernel = k_mx4_tiles<WR, WC, RB, CB>;
    if (!allow_lds((const void*)kernel, Product::kLdsBytes)) return DAQ_ERR_HIP;
    DAQ_LAUNCH("mx4_tiles", st,
               hipLaunchKernelGGL(kernel, dim3((unsigned)(per * kXcd)), dim3(64 * WR * WC), Product::kLdsBytes, st, p, (int)tm, (int)tn, (int)per));
    return DAQ_OK;
}

}  // namespace

// What the packed operands, the sizes and the result have to be.
static daq_status matmul_check(int64_t M, int64_t N, int64_t K, const void* B, const void* D, int dtype, int64_t ldd) {
    if (!dtype_ok(dtype)) return DAQ_ERR_INVALID_ARG;
    daq_status rc = matrix_size(M, K);
    if (rc == DAQ_OK) rc = matrix_size(N, K);
    if (rc == DAQ_OK) rc = matrix_size(M, N > 0 ? N : 1);
    if (rc != DAQ_OK) return rc;
    if (N <= 0) return DAQ_ERR_INVALID_ARG;
    if (M > 0 && (!B || !aligned256(B) || !D || !elem_aligned(D, dtype) || ldd < N)) return DAQ_ERR_INVALID_ARG;
    return DAQ_OK;
}

static daq_status mx4_matmul(int64_t M, int64_t N, int64_t K, const uint8_t* A, const uint8_t* B, void* D, int dtype, int64_t ldd,
                             hipStream_t st) {
    daq_mx4_layout la, lb;
    daq_layout_mx4(M, K, &la);
    daq_layout_mx4(N, K, &lb);
    const MatmulArgs p{A, A + la.off_scales, B, B + lb.off_scales, M, N, la.row_blocks, lb.row_blocks, la.groups,
                       (int)ceil_div(K, 64), D, ldd, dtype == DAQ_BF16};
    const int64_t big = ceil_div(la.row_blocks, 8) * ceil_div(lb.row_blocks, 8);
    return big >= 160 ? launch_tiles<2, 4, 4, 2>(p, st) : launch_tiles<2, 2, 2, 2>(p, st);
}

}  // namespace daq

using namespace daq;

extern "C" daq_status daq_mx4_matmul_workspace(int64_t M, int64_t N, int64_t K, size_t* bytes) {
    if (!bytes) return DAQ_ERR_INVALID_ARG;
    *bytes = 0;
    const daq_status rc = matrix_size(M, K);
    if (rc != DAQ_OK) return rc;
    return N > 0 ? matrix_size(N, K) : DAQ_ERR_INVALID_ARG;
}

extern "C" daq_status daq_mx4_matmul(int64_t M, int64_t N, int64_t K, const uint8_t* A, const uint8_t* B, void* D, daq_dtype dtype,
                                     int64_t ldd, void* workspace, size_t workspace_bytes, void* stream) {
    const daq_status rc = matmul_check(M, N, K, B, D, dtype, ldd);
    if (rc != DAQ_OK) return rc;
    if (M == 0) return DAQ_OK;
    if (!A || !aligned256(A)) return DAQ_ERR_INVALID_ARG;
    return mx4_matmul(M, N, K, A, B, D, dtype, ldd, (hipStream_t)stream);
}

extern "C" daq_status daq_mx4_linear_workspace(int64_t M, int64_t N, int64_t K, size_t* bytes) {
    size_t product = 0;
    const daq_status rc = daq_mx4_matmul_workspace(M, N, K, &product);
    if (!bytes) return DAQ_ERR_INVALID_ARG;
    *bytes = 0;
    if (rc != DAQ_OK) return rc;
    daq_mx4_layout L;
    daq_layout_mx4(M, K, &L);
    *bytes = (size_t)L.bytes + product;
    return DAQ_OK;
}

extern "C" daq_status daq_mx4_linear(int64_t M, int64_t N, int64_t K, const void* X, daq_dtype x_dtype, int64_t ldx, daq_round mode,
                                     uint64_t seed, const uint8_t* W, void* Y, daq_dtype y_dtype, int64_t ldy, void* workspace,
                                     size_t workspace_bytes, void* stream) {
    daq_status rc = matmul_check(M, N, K, W, Y, y_dtype, ldy);
    if (rc == DAQ_OK) rc = mx4_quantize_check(X, x_dtype, M, K, ldx, mode);
    if (rc != DAQ_OK) return rc;
    if (M == 0) return DAQ_OK;
    size_t need = 0;
    rc = daq_mx4_linear_workspace(M, N, K, &need);
    if (rc != DAQ_OK) return rc;
    if (need > 0 && (!workspace || workspace_bytes < need || !aligned256(workspace))) return DAQ_ERR_WORKSPACE;
    uint8_t* xq = static_cast<uint8_t*>(workspace);
    rc = mx4_quantize(X, x_dtype, M, K, ldx, false, mode == DAQ_ROUND_STOCHASTIC, seed, xq, (hipStream_t)stream);
    if (rc != DAQ_OK) return rc;
    return mx4_matmul(M, N, K, xq, W, Y, y_dtype, ldy, (hipStream_t)stream);
}
