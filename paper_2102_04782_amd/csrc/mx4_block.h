// A block of 32 elements to microscaled 4 bits, in the registers of one lane.
#pragma once

#include "lowbits.h"

namespace daq {

namespace {

// The bits of |x| of the largest of a block, as fp32 bits.
__device__ __forceinline__ uint32_t top_of(const uint32_t (&v)[32]) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 32; ++i) m = max(m, v[i] & 0x7FFFFFFFu);
    return m;
}
__device__ __forceinline__ uint32_t top_of(const uint32_t (&v)[16]) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) m = max_pairs(m, v[i] & 0x7FFF7FFFu);
    return max(m << 16, m & 0xFFFF0000u);
}

// 32 elements to 16 bytes of codes, the nearest ones: the conversion instructions round ties to even and stop at 6.
__device__ __forceinline__ u32x4 nearest_codes(const uint32_t (&v)[32], uint32_t byte) {
    const float s = scale_of(byte);
    u32x4 c;
#pragma unroll
    for (int d = 0; d < 4; ++d) {
        uint32_t w = 0;
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, bits_as<float>(v[8 * d]), bits_as<float>(v[8 * d + 1]), s, 0);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, bits_as<float>(v[8 * d + 2]), bits_as<float>(v[8 * d + 3]), s, 1);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, bits_as<float>(v[8 * d + 4]), bits_as<float>(v[8 * d + 5]), s, 2);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, bits_as<float>(v[8 * d + 6]), bits_as<float>(v[8 * d + 7]), s, 3);
        c[d] = w;
    }
    return c;
}
__device__ __forceinline__ u32x4 nearest_codes(const uint32_t (&v)[16], uint32_t byte) {
    const float s = scale_of(byte);
    u32x4 c;
#pragma unroll
    for (int d = 0; d < 4; ++d) {
        uint32_t w = 0;
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, bits_as<bf16x2>(v[4 * d]), s, 0);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, bits_as<bf16x2>(v[4 * d + 1]), s, 1);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, bits_as<bf16x2>(v[4 * d + 2]), s, 2);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, bits_as<bf16x2>(v[4 * d + 3]), s, 3);
        c[d] = w;
    }
    return c;
}
// The code of one element in the upper four bits, stochastically, from the complement V = 65535 - U of its draw.  With t = |x| * 2^-e, at most
// 6, as a fixed-point number of 29 places, or from t = 2 on as the bits of the float themselves moved there, the bits from 28 on count
// the elements up to t and the 16 below them are the fraction of the step to the next, so that adding V there carries exactly if the
// fraction is above U.
__device__ __forceinline__ uint32_t stochastic_code(float x, float up, uint32_t v16) {
    const float t = fabsf(x) * up;                                            // t * 2^29
    const uint32_t bits = (__float_as_uint(t) << 6) - (uint32_t)((252u + 58u) << 28);
    const uint32_t w = (t < 1073741824.0f ? (uint32_t)t : bits) + (v16 << 12);
    return (w & 0x7FFFFFFFu) | (__float_as_uint(x) & 0x80000000u);
}
__device__ __forceinline__ float elem_f32(const uint32_t (&v)[32], int i) { return bits_as<float>(v[i]); }
__device__ __forceinline__ float elem_f32(const uint32_t (&v)[16], int i) { return (i & 1) ? bf16_hi(v[i / 2]) : bf16_lo(v[i / 2]); }
__device__ __forceinline__ void scale_up(uint32_t (&v)[32], float f) {
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = __float_as_uint(bits_as<float>(v[i]) * f);
}
__device__ __forceinline__ void scale_up(uint32_t (&v)[16], float f) {
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = pack_bf16(bf16_lo(v[i]) * f, bf16_hi(v[i]) * f);
}
// draw(i): the complement of element i's draw, asked for from the last one on.  v is used up.
template <int W, typename F>
__device__ __forceinline__ u32x4 stochastic_codes(uint32_t (&v)[W], uint32_t byte, F draw) {
    // 2^(156 - byte) exceeds fp32 for the smallest scales: such elements are brought up by 2^64 first (exactly, also from below the normal
    // range); a block of zeros, of scale byte 1, is so too
    uint32_t from = byte;
    if (__any(byte < 29u)) {
        const bool tiny = byte < 29u;
        scale_up(v, tiny ? 0x1p64f : 1.0f);
        from += tiny ? 64u : 0u;
    }
    const float up = bits_as<float>((283u - from) << 23);
    u32x4 c;
#pragma unroll
    for (int d = 0; d < 4; ++d) {
        uint32_t w = 0;
#pragma unroll
        for (int i = 7; i >= 0; --i) w = __builtin_amdgcn_alignbit(w, stochastic_code(elem_f32(v, 8 * d + i), up, draw(8 * d + i)), 28);
        c[d] = w;
    }
    return byte == 255u ? u32x4{0, 0, 0, 0} : c;
}

// A block of a row.
__device__ __forceinline__ void load_block(const float* p, uint32_t (&v)[32]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const u32x4_a4 q = *reinterpret_cast<const u32x4_a4*>(p + 4 * i);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[4 * i + j] = q[j];
    }
}
__device__ __forceinline__ void load_block(const uint16_t* p, uint32_t (&v)[16]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const u32x4_a2 q = *reinterpret_cast<const u32x4_a2*>(p + 8 * i);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[4 * i + j] = q[j];
    }
}
// n of its 32 elements are there, the others are zero.
__device__ __forceinline__ void load_block(const float* p, int n, uint32_t (&v)[32]) {
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = i < n ? __float_as_uint(p[i]) : 0u;
}
__device__ __forceinline__ void load_block(const uint16_t* p, int n, uint32_t (&v)[16]) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const uint32_t lo = 2 * i < n ? p[2 * i] : 0u, hi = 2 * i + 1 < n ? p[2 * i + 1] : 0u;
        v[i] = lo | (hi << 16);
    }
}
template <typename T> struct Words;
template <> struct Words<float> { static constexpr int kBlock = 32; };
template <> struct Words<uint16_t> { static constexpr int kBlock = 16; };

}  // namespace

}  // namespace daq
