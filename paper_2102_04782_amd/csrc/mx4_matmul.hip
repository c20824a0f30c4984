// Products of microscaled 4-bit matrices, D[m][n] = sum over k of A[m][k] * B[n][k], and linear layers on them.
//
// The matrix instruction of 32 x 32 x 64 takes of each operand a block of 32 elements a lane (16 bytes and a scale byte): lane l has
// row l % 32 and block l / 32 of the 64 columns.  The packed layout holds operands in that order, so a wave loads a 32 x 64 tile
// as one contiguous KiB and the scale bytes of four tiles as one contiguous 256 bytes.  B goes in as the instruction's first
// operand, so that a lane holds four neighbouring columns of a row of D at a time.
#include "lowbits.h"

namespace daq {

namespace {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));

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

// One step: cbsz / blgp 4 say 4-bit elements; S picks the byte of the scale words.
template <int S>
__device__ __forceinline__ v16f mfma4(v4i x, v4i y, v16f c, int sx, int sy) {
    const v8i a = {x[0], x[1], x[2], x[3], 0, 0, 0, 0}, b = {y[0], y[1], y[2], y[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 4, 4, S, sx, S, sy);
}

// Four columns of row m of D from column n on.
__device__ __forceinline__ void store4(const MatmulArgs& p, int64_t m, int64_t n, float a, float b, float c, float d) {
    if (m >= p.M || n >= p.N) return;
    const int left = (int)min(p.N - n, (int64_t)4);
    if (p.bf16) {
        uint16_t* z = static_cast<uint16_t*>(p.d) + m * p.ldd + n;
        const uint32_t w0 = pack_bf16(a, b), w1 = pack_bf16(c, d);
        if (left == 4) {
            *reinterpret_cast<u32x2_a2*>(z) = u32x2_a2{w0, w1};
        } else {
            z[0] = (uint16_t)w0;
            if (left > 1) z[1] = (uint16_t)(w0 >> 16);
            if (left > 2) z[2] = (uint16_t)w1;
        }
    } else {
        float* z = static_cast<float*>(p.d) + m * p.ldd + n;
        if (left == 4) {
            *reinterpret_cast<u32x4_a4*>(z) = u32x4_a4{__float_as_uint(a), __float_as_uint(b), __float_as_uint(c), __float_as_uint(d)};
        } else {
            z[0] = a;
            if (left > 1) z[1] = b;
            if (left > 2) z[2] = c;
        }
    }
}

// A wave takes 64 x 64 results, operands straight from memory.
__global__ __launch_bounds__(256) void k_mx4_matmul(MatmulArgs p) {
    const int lane = threadIdx.x % kWave;
    const int64_t wave = (int64_t)blockIdx.x * 4 + threadIdx.x / kWave;
    const int tiles_n = (p.b_blocks + 1) / 2;
    const int64_t tm = wave / tiles_n;
    const int tn = (int)(wave - tm * tiles_n);
    if (tm * 2 >= p.a_blocks) return;
    const uint8_t *a[2], *b[2], *sa[2], *sb[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int64_t ra = min(tm * 2 + i, (int64_t)p.a_blocks - 1), rb = min(tn * 2 + i, p.b_blocks - 1);
        a[i] = p.a + ra * p.groups * 4096 + lane * 16;
        b[i] = p.b + rb * p.groups * 4096 + lane * 16;
        sa[i] = p.a_scales + ra * p.groups * 256 + lane * 4;
        sb[i] = p.b_scales + rb * p.groups * 256 + lane * 4;
    }
    v16f acc[2][2] = {};
    for (int g = 0; g < p.groups; ++g) {
        int wa[2], wb[2];
        v4i va[2][4], vb[2][4];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            wa[i] = *reinterpret_cast<const int*>(sa[i] + (int64_t)g * 256);
            wb[i] = *reinterpret_cast<const int*>(sb[i] + (int64_t)g * 256);
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                va[i][s] = *reinterpret_cast<const v4i*>(a[i] + ((int64_t)g * 4 + s) * 1024);
                vb[i][s] = *reinterpret_cast<const v4i*>(b[i] + ((int64_t)g * 4 + s) * 1024);
            }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                acc[i][j] = mfma4<0>(vb[j][0], va[i][0], acc[i][j], wb[j], wa[i]);
                acc[i][j] = mfma4<1>(vb[j][1], va[i][1], acc[i][j], wb[j], wa[i]);
                acc[i][j] = mfma4<2>(vb[j][2], va[i][2], acc[i][j], wb[j], wa[i]);
                acc[i][j] = mfma4<3>(vb[j][3], va[i][3], acc[i][j], wb[j], wa[i]);
            }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                store4(p, (tm * 2 + i) * 32 + lane % 32, ((int64_t)tn * 2 + j) * 32 + q * 8 + (lane / 32) * 4, acc[i][j][4 * q], acc[i][j][4 * q + 1],
                       acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
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
    const int64_t waves = ceil_div(la.row_blocks, 2) * ceil_div(lb.row_blocks, 2), blocks = ceil_div(waves, 4);
    if (!grid_ok(blocks)) return DAQ_ERR_UNSUPPORTED;
    DAQ_LAUNCH("mx4_matmul", st, hipLaunchKernelGGL(k_mx4_matmul, dim3((unsigned)blocks), dim3(256), 0, st, p));
    return DAQ_OK;
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
