// The weighted sum of the rows that a token's experts made, and its gradients.
#include "fp8_block.h"

namespace daq {

namespace {

struct CombineArgs {
    int64_t tokens, cols, ldy, ldo, lddy;
    int picks, chunks;        // of columns, of a workgroup each
    const int32_t* place;
    const float* weights;
    float* dweights;
};

__device__ __forceinline__ float element(const Eight<float>& v, int i) { return bits_as<float>(v.w[i]); }
__device__ __forceinline__ float element(const Eight<uint16_t>& v, int i) { return (i & 1) ? bf16_hi(v.w[i / 2]) : bf16_lo(v.w[i / 2]); }
template <bool PAST = false, typename T>
__device__ __forceinline__ void load_some(const T* p, int64_t left, Eight<T>& v) {
    if (left >= 8) load8<PAST>(p, v);
    else load8(p, (int)max(left, (int64_t)0), v);
}

// Eight columns of a token a lane; the rows of four places are asked for before the first is added.  Bound: memory; 16384 x 4096 bfloat16, 4 places,
// 671 MB in 108 us, 6.2 TB/s; rows of 1024 26 us, 6.5, of 512 14, 5.9, of 128 10.2, 2.1 (16 of a
// workgroup's 256 threads have columns then).
template <typename T, bool PAST>
__global__ __launch_bounds__(256) void k_combine(const T* y, T* out, CombineArgs p) {
    const int64_t t = blockIdx.x / p.chunks, c = (int64_t)(blockIdx.x - t * p.chunks) * 2048 + threadIdx.x * 8, left = p.cols - c;
    if (left <= 0) return;
    const int32_t* place = p.place + t * p.picks;
    const float* weights = p.weights ? p.weights + t * p.picks : nullptr;
    float sum[8] = {};
    for (int j0 = 0; j0 < p.picks; j0 += 4) {
        Eight<T> v[4];
        float w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int j = j0 + i, row = j < p.picks ? place[j] : -1;
            w[i] = j < p.picks ? weights ? weights[j] : 1.f : 0.f;
            load_some<PAST>(y + (int64_t)max(row, 0) * p.ldy + c, row >= 0 ? left : 0, v[i]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] = fmaf(w[i], element(v[i], e), sum[e]);
    }
    store8(out + t * p.ldo + c, (int)min(left, (int64_t)8), sum);
}

// A wave a place of a token: the row's gradient, and the dot product that is its weight's.  Bound: memory; 16384 x 4096 bfloat16, 4 places, 1.21 GB in 202 us,
// 6 TB/s; rows of 512 26 us, 5.9, of 128 19, 2.0 (a token's gradient is read once from memory, its other places find it in L2).
// PAST: bfloat16 (past_caches).
template <typename T, bool DW, bool PAST>
__global__ __launch_bounds__(256) void k_combine_back(const T* dout, const T* y, T* dy, CombineArgs p) {
    const int lane = threadIdx.x % kWave;
    const int64_t slot = (int64_t)blockIdx.x * 4 + threadIdx.x / kWave;
    if (slot >= p.tokens * p.picks) return;
    const int64_t t = slot / p.picks;
    const int row = p.place[slot];
    if (row < 0) {
        if (DW && lane == 0) p.dweights[slot] = 0.f;
        return;
    }
    const float w = p.weights ? p.weights[slot] : 1.f;
    float dot = 0.f;
    for (int64_t c = lane * 8; c < p.cols; c += 512) {
        Eight<T> d, v;
        load_some(dout + t * p.ldo + c, p.cols - c, d);
        if (DW) load_some<PAST>(y + (int64_t)row * p.ldy + c, p.cols - c, v);
        float z[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float x = element(d, e);
            z[e] = w * x;
            if (DW) dot = fmaf(x, element(v, e), dot);
        }
        T* to = dy + (int64_t)row * p.lddy + c;
        if (PAST && p.cols - c >= 8)
            __builtin_nontemporal_store(u32x4{pack_bf16(z[0], z[1]), pack_bf16(z[2], z[3]), pack_bf16(z[4], z[5]), pack_bf16(z[6], z[7])}, reinterpret_cast<u32x4*>(to));
        else store8(to, (int)min(p.cols - c, (int64_t)8), z);
    }
    if (DW) {
#pragma unroll
        for (int d = 1; d < kWave; d *= 2) dot += __shfl_xor(dot, d);
        if (lane == 0) p.dweights[slot] = dot;
    }
}

// Experts' rows in bfloat16 that are more than the caches hold and begin with a line are read, and their gradients written, past them, so that the tokens' rows stay.
// us without and with, 4 places, forward and backward one after the other: 16384 x 4096 382 to 399 and 343 to 359, 8192 x 4096 188 and 177, 6144 x 4096 no difference,
// 4096 x 4096 81 and 93, 16384 x 4099 414 and 417; fp32 16384 x 4096 743 to 774 and 790.
bool past_caches(const void* y, int64_t rows, int64_t cols, int64_t ld) {
    return rows * cols * 2 >= (int64_t)256 << 20 && (uintptr_t)y % 128 == 0 && ld * 2 % 128 == 0;
}
daq_status launch_combine(const void* y, int dtype, void* out, const CombineArgs& p, hipStream_t st) {
    const dim3 grid((unsigned)(p.tokens * p.chunks));
    auto launch = [&](auto kernel, auto* from, auto* to) -> daq_status {
        DAQ_LAUNCH("combine", st, hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, from, to, p));
        return DAQ_OK;
    };
    if (dtype == DAQ_FP32) return launch(k_combine<float, false>, static_cast<const float*>(y), static_cast<float*>(out));
    return launch(past_caches(y, p.tokens * p.picks, p.cols, p.ldy) ? k_combine<uint16_t, true> : k_combine<uint16_t, false>, static_cast<const uint16_t*>(y), static_cast<uint16_t*>(out));
}
daq_status launch_combine_back(const void* dout, const void* y, int dtype, void* dy, const CombineArgs& p, hipStream_t st) {
    const int64_t rows = p.tokens * p.picks;
    const dim3 grid((unsigned)ceil_div(rows, 4));
    auto launch = [&](auto kernel, auto* of_out, auto* from, auto* to) -> daq_status {
        DAQ_LAUNCH("combine_back", st, hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, of_out, from, to, p));
        return DAQ_OK;
    };
    if (dtype == DAQ_FP32)
        return launch(p.dweights ? k_combine_back<float, true, false> : k_combine_back<float, false, false>, static_cast<const float*>(dout), static_cast<const float*>(y), static_cast<float*>(dy));
    const bool past = past_caches(dy, rows, p.cols, p.lddy) && (!p.dweights || past_caches(y, rows, p.cols, p.ldy));
    return launch(past ? p.dweights ? k_combine_back<uint16_t, true, true> : k_combine_back<uint16_t, false, true>
                       : p.dweights ? k_combine_back<uint16_t, true, false> : k_combine_back<uint16_t, false, false>,
                  static_cast<const uint16_t*>(dout), static_cast<const uint16_t*>(y), static_cast<uint16_t*>(dy));
}
daq_status combine_check(const daq_experts* plan, int dtype, int64_t cols) {
    if (!plan_ok(plan) || !dtype_ok(dtype) || cols <= 0) return DAQ_ERR_INVALID_ARG;
    return matrix_size(plan_slots(*plan), cols);
}
bool a4(const void* p) { return ((uintptr_t)p & 3u) == 0; }

}  // namespace

}  // namespace daq

using namespace daq;

extern "C" daq_status daq_experts_combine(const daq_experts* plan, const void* y, daq_dtype dtype, int64_t cols, int64_t ldy, const float* weights,
                                          void* out, int64_t ldo, void* stream) {
    const daq_status rc = combine_check(plan, dtype, cols);
    if (rc != DAQ_OK || plan->tokens == 0) return rc;
    if (!y || !elem_aligned(y, dtype) || !out || !elem_aligned(out, dtype) || ldy < cols || ldo < cols || !a4(weights)) return DAQ_ERR_INVALID_ARG;
    const int64_t chunks = ceil_div(cols, 2048);
    if (!grid_ok(plan->tokens * chunks, 256)) return DAQ_ERR_UNSUPPORTED;
    const CombineArgs p{plan->tokens, cols, ldy, ldo, 0, plan->picks, (int)chunks, plan->place, weights, nullptr};
    return launch_combine(y, dtype, out, p, (hipStream_t)stream);
}

extern "C" daq_status daq_experts_combine_backward(const daq_experts* plan, const void* dout, daq_dtype dtype, int64_t cols, int64_t ldo,
                                                   const void* y, int64_t ldy, const float* weights, void* dy, int64_t lddy, float* dweights,
                                                   void* stream) {
    const daq_status rc = combine_check(plan, dtype, cols);
    if (rc != DAQ_OK || plan->tokens == 0) return rc;
    if (!dout || !elem_aligned(dout, dtype) || !dy || !elem_aligned(dy, dtype) || ldo < cols || lddy < cols || !a4(weights) || !a4(dweights)) return DAQ_ERR_INVALID_ARG;
    if (dweights && (!y || !elem_aligned(y, dtype) || ldy < cols)) return DAQ_ERR_INVALID_ARG;
    if (!grid_ok(ceil_div(plan_slots(*plan), 4), 256)) return DAQ_ERR_UNSUPPORTED;
    const CombineArgs p{plan->tokens, cols, ldy, ldo, lddy, plan->picks, 0, plan->place, weights, dweights};
    return launch_combine_back(dout, y, dtype, dy, p, (hipStream_t)stream);
}
