// Weight gradient of a linear layer from its input saved in 8 bits, dW[n][k] = sum over m of dY[m][n] * X^[m][k].
//
// A decoded code is an integer of at most seven bits times a power of two, so X^ is exact in bfloat16 and the products run on the
// bfloat16 matrix cores with fp32 sums.  An fp32 gradient is the sum of three bfloat16 values of eight bits each.
#include "lowbits.h"

namespace daq {

namespace {

typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef uint16_t v8u __attribute__((ext_vector_type(8)));

struct WgradArgs {
    const void* dy;
    int64_t lddy;
    const uint8_t* codes;
    const uint8_t* scales;
    int64_t pitch;
    int64_t M, N, K;
    float* dw;
    int64_t ldw;
    int accumulate;
};

// x = hi + mid + lo, each the leading eight bits of what is left (a value that is not finite stays whole).
__device__ __forceinline__ void split3(float x, uint16_t& hi, uint16_t& mid, uint16_t& lo) {
    const uint32_t h = __float_as_uint(x) & 0xFFFF0000u;
    hi = (uint16_t)(h >> 16);
    const bool finite = (h & 0x7F800000u) != 0x7F800000u;
    const float r = finite ? x - bits_as<float>(h) : 0.0f;
    const uint32_t m = __float_as_uint(r) & 0xFFFF0000u;
    mid = (uint16_t)(m >> 16);
    lo = (uint16_t)(__float_as_uint(r - bits_as<float>(m)) >> 16);
    if (!finite && x != x) hi |= 0x40;   // a NaN of low bits only
}

template <typename T>
__global__ __launch_bounds__(256) void k_ckpt8_wgrad(WgradArgs p) {
    const int lane = threadIdx.x % kWave;
    const int64_t wave = (int64_t)blockIdx.x * 4 + threadIdx.x / kWave;
    const int64_t tiles_k = (p.K + 31) / 32, tn = wave / tiles_k, tk = wave - tn * tiles_k;
    if (tn * 32 >= p.N) return;
    const int64_t n = tn * 32 + lane % 32, k = tk * 32 + lane % 32;
    const T* dy = static_cast<const T*>(p.dy) + min(n, p.N - 1);
    const uint8_t* code = p.codes + k;                        // inside the row's padding at least
    const uint8_t* scale = p.scales + tk;
    v16f acc = {};
    for (int64_t m0 = 0; m0 < p.M; m0 += 16) {
        v8u hi, mid, lo, x;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int64_t m = m0 + (lane / 32) * 8 + j;
            const bool in = m < p.M;
            const int64_t r = in ? m : 0;
            const float xv = (float)(int8_t)code[r * p.pitch] * scale_of(scale[r * (p.pitch / kMxBlock)]);
            x[j] = in ? (uint16_t)(__float_as_uint(xv) >> 16) : (uint16_t)0;
            if constexpr (sizeof(T) == 4) {
                uint16_t a, b, c;
                split3(dy[r * p.lddy], a, b, c);
                hi[j] = in ? a : (uint16_t)0;
                mid[j] = in ? b : (uint16_t)0;
                lo[j] = in ? c : (uint16_t)0;
            } else {
                hi[j] = in ? dy[r * p.lddy] : (uint16_t)0;
            }
        }
        const v8bf xb = __builtin_bit_cast(v8bf, x);
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, hi), xb, acc, 0, 0, 0);
        if constexpr (sizeof(T) == 4) {
            acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, mid), xb, acc, 0, 0, 0);
            acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, lo), xb, acc, 0, 0, 0);
        }
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int64_t row = tn * 32 + 8 * (i / 4) + 4 * (lane / 32) + i % 4;
        if (row < p.N && k < p.K) {
            float* z = p.dw + row * p.ldw + k;
            *z = p.accumulate ? *z + acc[i] : acc[i];
        }
    }
}

}  // namespace

}  // namespace daq

using namespace daq;

static daq_status wgrad_size(int64_t M, int64_t N, int64_t K) {
    if (N <= 0) return DAQ_ERR_INVALID_ARG;
    daq_status rc = matrix_size(M, K);
    if (rc == DAQ_OK) rc = matrix_size(M, N);
    if (rc == DAQ_OK) rc = matrix_size(N, K);
    return rc;
}

extern "C" daq_status daq_ckpt8_weight_grad_workspace(int64_t M, int64_t N, int64_t K, daq_dtype dtype, size_t* bytes) {
    if (!bytes) return DAQ_ERR_INVALID_ARG;
    *bytes = 0;
    if (!dtype_ok(dtype)) return DAQ_ERR_INVALID_ARG;
    return wgrad_size(M, N, K);
}

extern "C" daq_status daq_ckpt8_weight_grad(int64_t M, int64_t N, int64_t K, const void* dY, daq_dtype dtype, int64_t lddy,
                                            const uint8_t* x_ckpt, float* dW, int64_t ldw, int32_t accumulate, void* workspace,
                                            size_t workspace_bytes, void* stream) {
    if (!dtype_ok(dtype)) return DAQ_ERR_INVALID_ARG;
    const daq_status rc = wgrad_size(M, N, K);
    if (rc != DAQ_OK) return rc;
    if (!dW || !elem_aligned(dW, DAQ_FP32) || ldw < K) return DAQ_ERR_INVALID_ARG;
    if (M > 0 && (!dY || !elem_aligned(dY, dtype) || lddy < N || !x_ckpt || !aligned256(x_ckpt))) return DAQ_ERR_INVALID_ARG;
    daq_ckpt8_layout L;
    daq_layout_ckpt8(M, K, 1, &L);
    const WgradArgs p{dY, lddy, x_ckpt, x_ckpt + L.off_scales, L.pitch, M, N, K, dW, ldw, accumulate};
    const int64_t blocks = ceil_div(ceil_div(N, 32) * ceil_div(K, 32), 4);
    if (!grid_ok(blocks)) return DAQ_ERR_UNSUPPORTED;
    hipStream_t st = (hipStream_t)stream;
    if (dtype == DAQ_BF16) DAQ_LAUNCH("ckpt8_wgrad", st, hipLaunchKernelGGL(k_ckpt8_wgrad<uint16_t>, dim3((unsigned)blocks), dim3(256), 0, st, p));
    else DAQ_LAUNCH("ckpt8_wgrad", st, hipLaunchKernelGGL(k_ckpt8_wgrad<float>, dim3((unsigned)blocks), dim3(256), 0, st, p));
    return DAQ_OK;
}
