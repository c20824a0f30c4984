// Matrices saved in 8 bits, and activation layers that keep their input so.
//
// All of it is bound by memory: a thread takes 8 elements, 16 bytes of a bfloat16 row, and four neighbours share a block's largest
// magnitude by lane exchanges.  Measured (us; TB/s of what is read and written, the Infinity Cache keeping part of it): 32768 x 8192 saved
// 134 (6.1) and restored 116 (7.0); gated, 16384 x 8192, forward 157 (6.9: h read, y and the codes written), backward 175 (6.2), 10 more with
// y saved again (0.14 GB).  Small matrices 3 to 5 us.  Exponentials and Phi are fp32; f' shares them with f.
#include <type_traits>

#include "lowbits.h"

namespace daq {

namespace {

constexpr int kBlock = 256;
constexpr int kPer = 8;                         // elements of a thread; four neighbouring threads hold a block
constexpr int kLanes = kMxBlock / kPer;

// Matrices of 48 MiB and more pass the caches by (NT); the codes are read so too but written into them.  us with and without, bfloat16:
// 32768 x 8192 saved and restored 256 and 316; gated, 16384 x 8192, forward and backward 335 and 432 (with the codes' stores past the caches
// as well 281 and 371).  Between a producer and a consumer of the matrices, gated of 34 MB 64.7 and 62.3 for the whole, 67 MB 114 and
// 116, 134 MB 214 and 228, 268 MB 429 and 473.
constexpr int64_t kPassBytes = 2 * kStreamBytes;

// How the rows of a launch are dealt out: `tpr` threads (a power of two, at most a workgroup) to a row, several rows to a workgroup
// where they are short, several workgroups to a row (blockIdx.y) where they are long.
struct Rows {
    int64_t rows;
    int64_t units;     // of kPer elements, of a row; a multiple of kLanes
    int shift;         // tpr = 1 << shift
    __device__ bool place(int64_t& row, int64_t& unit) const {
        const int tpr = 1 << shift;
        row = ((int64_t)blockIdx.x << (8 - shift)) + (threadIdx.x >> shift);
        unit = (int64_t)blockIdx.y * tpr + (threadIdx.x & (tpr - 1));
        return row < rows && unit < units;     // (the threads of a block of elements stay together)
    }
};
bool rows_grid(int64_t rows, int64_t pitch, Rows& r, dim3& grid) {
    r.rows = rows;
    r.units = pitch / kPer;
    r.shift = 2;
    while (r.shift < 8 && ((int64_t)1 << r.shift) < r.units) ++r.shift;
    const int64_t x = ceil_div(rows, (int64_t)1 << (8 - r.shift)), y = ceil_div(r.units, (int64_t)1 << r.shift);
    if (!grid_ok(x, kBlock) || y > 65535) return false;
    grid = dim3((unsigned)x, (unsigned)y);
    return true;
}

// kPer elements from column c on, as fp32; those behind the last column are zero.
template <bool NT>
__device__ __forceinline__ void load_unit(const float* p, int64_t left, float (&v)[kPer]) {
    if (left >= kPer) {
#pragma unroll
        for (int i = 0; i < kPer / 4; ++i) {
            const u32x4_a4* at = reinterpret_cast<const u32x4_a4*>(p + 4 * i);
            const u32x4_a4 q = NT ? __builtin_nontemporal_load(at) : *at;
#pragma unroll
            for (int j = 0; j < 4; ++j) v[4 * i + j] = bits_as<float>(q[j]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < kPer; ++i) v[i] = i < left ? p[i] : 0.0f;
    }
}
template <bool NT>
__device__ __forceinline__ void load_unit(const uint16_t* p, int64_t left, float (&v)[kPer]) {
    if (left >= kPer) {
#pragma unroll
        for (int k = 0; k < kPer / 8; ++k) {
            const u32x4_a2* at = reinterpret_cast<const u32x4_a2*>(p + 8 * k);
            const u32x4_a2 q = NT ? __builtin_nontemporal_load(at) : *at;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[8 * k + 2 * i] = bf16_lo(q[i]);
                v[8 * k + 2 * i + 1] = bf16_hi(q[i]);
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < kPer; ++i) v[i] = i < left ? bits_as<float>((uint32_t)p[i] << 16) : 0.0f;
    }
}
template <bool NT>
__device__ __forceinline__ void store_unit(float* p, int64_t left, const float (&v)[kPer]) {
    if (left >= kPer) {
#pragma unroll
        for (int i = 0; i < kPer / 4; ++i) {
            const u32x4_a4 q = {__float_as_uint(v[4 * i]), __float_as_uint(v[4 * i + 1]), __float_as_uint(v[4 * i + 2]), __float_as_uint(v[4 * i + 3])};
            u32x4_a4* at = reinterpret_cast<u32x4_a4*>(p + 4 * i);
            if constexpr (NT) __builtin_nontemporal_store(q, at);
            else *at = q;
        }
    } else {
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            if (i < left) p[i] = v[i];
    }
}
template <bool NT>
__device__ __forceinline__ void store_unit(uint16_t* p, int64_t left, const float (&v)[kPer]) {
    uint32_t w[kPer / 2];
#pragma unroll
    for (int i = 0; i < kPer / 2; ++i) w[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
    if (left >= kPer) {
#pragma unroll
        for (int i = 0; i < kPer / 8; ++i) {
            const u32x4_a2 q = {w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]};
            u32x4_a2* at = reinterpret_cast<u32x4_a2*>(p + 8 * i);
            if constexpr (NT) __builtin_nontemporal_store(q, at);
            else *at = q;
        }
    } else {
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            if (i < left) p[i] = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
    }
}

// The largest of four neighbouring threads.
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, true));   // lane ^ 1
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, true));   // lane ^ 2
}

// A checkpoint's row of one part.
struct Saved {
    uint8_t* codes;
    uint8_t* scales;
    int64_t pitch;
    __host__ __device__ uint8_t* code(int64_t part_row, int64_t unit) const { return codes + part_row * pitch + unit * kPer; }
    __host__ __device__ uint8_t* scale(int64_t part_row, int64_t unit) const { return scales + part_row * (pitch / kMxBlock) + unit / kLanes; }
};

__device__ __forceinline__ void save_unit(const Saved& to, int64_t part_row, int64_t unit, const float (&v)[kPer]) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) top = max(top, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    const uint32_t byte = scale_byte<6>(quad_max(top));
    const float inv = byte == 255u ? 0.0f : inverse_scale(byte);
    uint32_t c[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        // adding 1.5 * 2^23 rounds to an integer, ties to even, which is then the low byte in two's complement
        const float t = fminf(fmaxf(v[i] * inv, -127.0f), 127.0f);
        c[i] = __float_as_uint(t + 12582912.0f);
    }
    u32x2 w;
#pragma unroll
    for (int i = 0; i < kPer / 4; ++i)
        w[i] = (c[4 * i] & 255u) | ((c[4 * i + 1] & 255u) << 8) | ((c[4 * i + 2] & 255u) << 16) | (c[4 * i + 3] << 24);
    *reinterpret_cast<u32x2*>(to.code(part_row, unit)) = w;
    if (unit % kLanes == 0) *to.scale(part_row, unit) = (uint8_t)byte;
}
template <bool NT>
__device__ __forceinline__ void read_unit(const Saved& from, int64_t part_row, int64_t unit, float (&v)[kPer]) {
    const u32x2* at = reinterpret_cast<const u32x2*>(from.code(part_row, unit));
    const u32x2 w = NT ? __builtin_nontemporal_load(at) : *at;
    const float s = scale_of(*from.scale(part_row, unit));
#pragma unroll
    for (int i = 0; i < kPer; ++i) v[i] = (float)(int8_t)(w[i / 4] >> (8 * (i % 4))) * s;
}

struct SaveArgs {
    const void* src;
    void* dst;
    int64_t ld, cols;
    int parts;
    Saved ckpt;
};

// The parts are rows of their own here.
template <typename T, bool NT>
__global__ __launch_bounds__(kBlock) void k_ckpt8_save(Rows rows, SaveArgs p) {
    int64_t row, unit;
    if (!rows.place(row, unit)) return;
    const int64_t r = p.parts == 1 ? row : row >> 1, part = p.parts == 1 ? 0 : row & 1, c = unit * kPer;
    float v[kPer];
    load_unit<NT>(static_cast<const T*>(p.src) + r * p.ld + part * p.cols + c, p.cols - c, v);
    save_unit(p.ckpt, row, unit, v);
}

template <typename T, bool NT>
__global__ __launch_bounds__(kBlock) void k_ckpt8_restore(Rows rows, SaveArgs p) {
    int64_t row, unit;
    if (!rows.place(row, unit)) return;
    const int64_t r = p.parts == 1 ? row : row >> 1, part = p.parts == 1 ? 0 : row & 1, c = unit * kPer;
    float v[kPer];
    read_unit<NT>(p.ckpt, row, unit, v);
    store_unit<NT>(static_cast<T*>(p.dst) + r * p.ld + part * p.cols + c, p.cols - c, v);
}

// Phi(x) from e = exp(-x^2 / 2).  0.5 (1 + erf) cancels far below zero (4 % at -5 in fp32, nothing left at -5.6), so Phi(-t) is taken as e * Q(t) for
// t >= 0, Q(t) = exp(t^2 / 2) * erfc(t / sqrt 2) / 2, and Phi(t) as 1 - e * Q(t).  Q is s * (polynomial of s) of s = 1 / (1 + 0.36 t), fitted here by
// least squares at Chebyshev points with weights that even out the relative error, for t up to 14.5 (e has left fp32 there): 2e-8 off, and
// 4.4 * 2^-24 with the roundings of its evaluation.  Plain GELU of 16384 x 8192 bfloat16, forward + backward: 118 + 119 us; with the library's
// erff 133 + 144, with its erfcf, which keeps the tail too, 188 + 210.
__device__ __forceinline__ float normal_cdf(float x, float e) {
    const float s = __builtin_amdgcn_rcpf(__builtin_fmaf(0.36f, fabsf(x), 1.0f));
    constexpr float c[10] = {0.14360565f, 0.14397098f, 0.121114075f, 0.11191071f, -0.053047687f, 0.21752816f, -0.3696232f, 0.25836864f, -0.08439457f, 0.010567232f};
    float q = c[9];
#pragma unroll
    for (int i = 8; i >= 0; --i) q = __builtin_fmaf(q, s, c[i]);
    q = q * s * e;
    return x < 0.0f ? q : 1.0f - q;
}

// f(x), and f'(x) where `slope` is asked for.
__device__ __forceinline__ float act_value(int act, float x, float* slope) {
    if (act == DAQ_ACT_SILU) {
        const float s = 1.0f / (1.0f + __expf(-x));
        if (slope) *slope = s * (1.0f + x * (1.0f - s));
        return x * s;
    }
    const float e = __expf(-0.5f * x * x), cdf = normal_cdf(x, e);
    if (slope) *slope = cdf + x * (0.39894228f * e);
    return x * cdf;
}

struct ActArgs {
    const void* in;      // h, or dy
    int64_t ld_in;
    void* out;           // y, or dh
    int64_t ld_out;
    int64_t cols;
    Saved ckpt;
    Saved y;             // backward: y saved again, where asked for
};

template <typename T, int ACT, bool GATED, bool NT>
__global__ __launch_bounds__(kBlock) void k_ckpt8_act_forward(Rows rows, ActArgs p) {
    int64_t row, unit;
    if (!rows.place(row, unit)) return;
    const int64_t c = unit * kPer;
    const T* h = static_cast<const T*>(p.in) + row * p.ld_in + c;
    float g[kPer], u[kPer], y[kPer];
    load_unit<NT>(h, p.cols - c, g);
    if constexpr (GATED) load_unit<NT>(h + p.cols, p.cols - c, u);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        y[i] = act_value(ACT, g[i], nullptr);
        if constexpr (GATED) y[i] *= u[i];
    }
    store_unit<NT>(static_cast<T*>(p.out) + row * p.ld_out + c, p.cols - c, y);
    save_unit(p.ckpt, GATED ? 2 * row : row, unit, g);
    if constexpr (GATED) save_unit(p.ckpt, 2 * row + 1, unit, u);
}

template <typename T, int ACT, bool GATED, bool SAVE, bool NT>
__global__ __launch_bounds__(kBlock) void k_ckpt8_act_backward(Rows rows, ActArgs p) {
    int64_t row, unit;
    if (!rows.place(row, unit)) return;
    const int64_t c = unit * kPer;
    float dy[kPer], g[kPer], u[kPer], y[kPer];
    load_unit<NT>(static_cast<const T*>(p.in) + row * p.ld_in + c, p.cols - c, dy);
    read_unit<NT>(p.ckpt, GATED ? 2 * row : row, unit, g);
    if constexpr (GATED) read_unit<NT>(p.ckpt, 2 * row + 1, unit, u);
    float dg[kPer], du[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        float slope;
        const float f = act_value(ACT, g[i], &slope);
        if constexpr (GATED) {
            dg[i] = dy[i] * u[i] * slope;
            du[i] = dy[i] * f;
            y[i] = f * u[i];
        } else {
            dg[i] = dy[i] * slope;
            y[i] = f;
        }
    }
    T* dh = static_cast<T*>(p.out) + row * p.ld_out + c;
    store_unit<NT>(dh, p.cols - c, dg);
    if constexpr (GATED) store_unit<NT>(dh + p.cols, p.cols - c, du);
    if constexpr (SAVE) save_unit(p.y, row, unit, y);
}

Saved saved_at(const uint8_t* ckpt, int64_t rows, int64_t cols, int parts) {
    daq_ckpt8_layout L;
    daq_layout_ckpt8(rows, cols, parts, &L);
    uint8_t* base = const_cast<uint8_t*>(ckpt);
    return Saved{base, base + L.off_scales, L.pitch};
}

template <typename T, int ACT, bool GATED, bool NT>
daq_status act_backward(const Rows& rows, const dim3& grid, const ActArgs& p, hipStream_t st) {
    if (p.y.codes)
        DAQ_LAUNCH("ckpt8_act_backward", st, hipLaunchKernelGGL((k_ckpt8_act_backward<T, ACT, GATED, true, NT>), grid, dim3(kBlock), 0, st, rows, p));
    else
        DAQ_LAUNCH("ckpt8_act_backward", st, hipLaunchKernelGGL((k_ckpt8_act_backward<T, ACT, GATED, false, NT>), grid, dim3(kBlock), 0, st, rows, p));
    return DAQ_OK;
}
template <typename T, int ACT, bool GATED, bool NT>
daq_status act_forward(const Rows& rows, const dim3& grid, const ActArgs& p, hipStream_t st) {
    DAQ_LAUNCH("ckpt8_act_forward", st, hipLaunchKernelGGL((k_ckpt8_act_forward<T, ACT, GATED, NT>), grid, dim3(kBlock), 0, st, rows, p));
    return DAQ_OK;
}
// f(type, act, gated, streaming) with one of the sixteen combinations as constants.
template <typename F>
daq_status act_pick(int dtype, int act, bool gated, bool nt, F f) {
    auto with_nt = [&](auto t, auto a, auto g) { return nt ? f(t, a, g, std::true_type{}) : f(t, a, g, std::false_type{}); };
    auto with_gate = [&](auto t, auto a) { return gated ? with_nt(t, a, std::true_type{}) : with_nt(t, a, std::false_type{}); };
    auto with_act = [&](auto t) {
        return act == DAQ_ACT_SILU ? with_gate(t, std::integral_constant<int, DAQ_ACT_SILU>{}) : with_gate(t, std::integral_constant<int, DAQ_ACT_GELU>{});
    };
    return dtype == DAQ_BF16 ? with_act(uint16_t{}) : with_act(float{});
}

// The sizes of a matrix of `parts` parts.
daq_status parts_size(int64_t rows, int64_t cols, int parts) {
    if (parts != 1 && parts != 2) return DAQ_ERR_INVALID_ARG;
    if (cols <= 0) return DAQ_ERR_INVALID_ARG;
    if (cols >= (int64_t)1 << 31) return DAQ_ERR_UNSUPPORTED;
    return matrix_size(rows, cols * parts);
}
// A pointer of a matrix whose rows hold `width` elements.
bool matrix_ok(const void* p, int dtype, int64_t width, int64_t ld) { return p && elem_aligned(p, dtype) && ld >= width; }
bool ckpt_ok(const void* p) { return p && aligned256(p); }

}  // namespace

}  // namespace daq

using namespace daq;

extern "C" daq_status daq_layout_ckpt8(int64_t rows, int64_t cols, int32_t parts, daq_ckpt8_layout* out) {
    if (!out) return DAQ_ERR_INVALID_ARG;
    *out = daq_ckpt8_layout{};
    const daq_status rc = parts_size(rows, cols, parts);
    if (rc != DAQ_OK) return rc;
    out->pitch = round_up(cols, kMxBlock);
    out->off_scales = round_up(rows * parts * out->pitch, 256);
    out->bytes = out->off_scales + round_up(rows * parts * (out->pitch / kMxBlock), 256);
    return DAQ_OK;
}

static daq_status save_or_restore(bool save, const void* src, void* dst, int dtype, int64_t rows, int64_t cols, int parts, int64_t ld,
                                  const uint8_t* ckpt, hipStream_t st) {
    if (!dtype_ok(dtype)) return DAQ_ERR_INVALID_ARG;
    const daq_status rc = parts_size(rows, cols, parts);
    if (rc != DAQ_OK) return rc;
    if (rows == 0) return DAQ_OK;
    if (!matrix_ok(save ? src : dst, dtype, cols * parts, ld) || !ckpt_ok(ckpt)) return DAQ_ERR_INVALID_ARG;
    const SaveArgs p{src, dst, ld, cols, parts, saved_at(ckpt, rows, cols, parts)};
    Rows r;
    dim3 grid;
    if (!rows_grid(rows * parts, p.ckpt.pitch, r, grid)) return DAQ_ERR_UNSUPPORTED;
    auto launch = [&](auto t, auto n) -> daq_status {
        using T = decltype(t);
        constexpr bool NT = decltype(n)::value;
        if (save) DAQ_LAUNCH("ckpt8_save", st, hipLaunchKernelGGL((k_ckpt8_save<T, NT>), grid, dim3(kBlock), 0, st, r, p));
        else DAQ_LAUNCH("ckpt8_restore", st, hipLaunchKernelGGL((k_ckpt8_restore<T, NT>), grid, dim3(kBlock), 0, st, r, p));
        return DAQ_OK;
    };
    const bool nt = rows * cols * parts * dtype_size(dtype) >= kPassBytes;
    if (dtype == DAQ_BF16) return nt ? launch(uint16_t{}, std::true_type{}) : launch(uint16_t{}, std::false_type{});
    return nt ? launch(float{}, std::true_type{}) : launch(float{}, std::false_type{});
}

extern "C" daq_status daq_ckpt8_save(const void* src, daq_dtype dtype, int64_t rows, int64_t cols, int32_t parts, int64_t ld,
                                     uint8_t* ckpt, void* stream) {
    return save_or_restore(true, src, nullptr, dtype, rows, cols, parts, ld, ckpt, (hipStream_t)stream);
}

extern "C" daq_status daq_ckpt8_restore(const uint8_t* ckpt, int64_t rows, int64_t cols, int32_t parts, void* dst, daq_dtype dtype,
                                        int64_t ld, void* stream) {
    return save_or_restore(false, nullptr, dst, dtype, rows, cols, parts, ld, ckpt, (hipStream_t)stream);
}

extern "C" daq_status daq_ckpt8_act_forward(const void* h, daq_dtype dtype, int64_t rows, int64_t cols, int64_t ldh, daq_act act,
                                            int32_t gated, void* y, int64_t ldy, uint8_t* ckpt, void* stream) {
    if (!dtype_ok(dtype) || (act != DAQ_ACT_SILU && act != DAQ_ACT_GELU)) return DAQ_ERR_INVALID_ARG;
    const int parts = gated ? 2 : 1;
    const daq_status rc = parts_size(rows, cols, parts);
    if (rc != DAQ_OK) return rc;
    if (rows == 0) return DAQ_OK;
    if (!matrix_ok(h, dtype, cols * parts, ldh) || !matrix_ok(y, dtype, cols, ldy) || !ckpt_ok(ckpt)) return DAQ_ERR_INVALID_ARG;
    const ActArgs p{h, ldh, y, ldy, cols, saved_at(ckpt, rows, cols, parts), Saved{}};
    Rows r;
    dim3 grid;
    if (!rows_grid(rows, p.ckpt.pitch, r, grid)) return DAQ_ERR_UNSUPPORTED;
    const bool nt = rows * cols * parts * dtype_size(dtype) >= kPassBytes;
    return act_pick(dtype, act, gated != 0, nt, [&](auto t, auto a, auto g, auto n) {
        return act_forward<decltype(t), decltype(a)::value, decltype(g)::value, decltype(n)::value>(r, grid, p, (hipStream_t)stream);
    });
}

extern "C" daq_status daq_ckpt8_act_backward(const void* dy, daq_dtype dtype, int64_t rows, int64_t cols, int64_t lddy, const uint8_t* ckpt,
                                             daq_act act, int32_t gated, void* dh, int64_t lddh, uint8_t* y_ckpt, void* stream) {
    if (!dtype_ok(dtype) || (act != DAQ_ACT_SILU && act != DAQ_ACT_GELU)) return DAQ_ERR_INVALID_ARG;
    const int parts = gated ? 2 : 1;
    const daq_status rc = parts_size(rows, cols, parts);
    if (rc != DAQ_OK) return rc;
    if (rows == 0) return DAQ_OK;
    if (!matrix_ok(dy, dtype, cols, lddy) || !matrix_ok(dh, dtype, cols * parts, lddh) || !ckpt_ok(ckpt) || !aligned256(y_ckpt))
        return DAQ_ERR_INVALID_ARG;
    const ActArgs p{dy, lddy, dh, lddh, cols, saved_at(ckpt, rows, cols, parts), y_ckpt ? saved_at(y_ckpt, rows, cols, 1) : Saved{}};
    Rows r;
    dim3 grid;
    if (!rows_grid(rows, p.ckpt.pitch, r, grid)) return DAQ_ERR_UNSUPPORTED;
    const bool nt = rows * cols * parts * dtype_size(dtype) >= kPassBytes;
    return act_pick(dtype, act, gated != 0, nt, [&](auto t, auto a, auto g, auto n) {
        return act_backward<decltype(t), decltype(a)::value, decltype(g)::value, decltype(n)::value>(r, grid, p, (hipStream_t)stream);
    });
}
