// Blocks of 128 elements to 8-bit floating point, in the registers of the lanes that hold them: eight elements of a row a lane.
#pragma once

#include "fp8.h"

namespace daq {

namespace {

// Eight neighbouring elements as they lie in memory.
template <typename T>
struct Eight {
    static constexpr int kWords = (int)sizeof(T) * 2;
    uint32_t w[kWords];
};
// PAST: past the caches, which keep what they have.
template <bool PAST = false>
__device__ __forceinline__ void load8(const uint16_t* p, Eight<uint16_t>& v) {
    const u32x4_a2* from = reinterpret_cast<const u32x4_a2*>(p);
    const u32x4 q = PAST ? __builtin_nontemporal_load(from) : *from;
#pragma unroll
    for (int i = 0; i < 4; ++i) v.w[i] = q[i];
}
template <bool PAST = false>
__device__ __forceinline__ void load8(const float* p, Eight<float>& v) {
    const u32x4_a4* from = reinterpret_cast<const u32x4_a4*>(p);
    const u32x4 a = PAST ? __builtin_nontemporal_load(from) : *from, b = PAST ? __builtin_nontemporal_load(from + 1) : from[1];
#pragma unroll
    for (int i = 0; i < 4; ++i) v.w[i] = a[i], v.w[4 + i] = b[i];
}
// The first `left` of them (any number), zeros behind.
__device__ __forceinline__ void load8(const uint16_t* p, int left, Eight<uint16_t>& v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v.w[i] = (2 * i < left ? (uint32_t)p[2 * i] : 0u) | (2 * i + 1 < left ? (uint32_t)p[2 * i + 1] << 16 : 0u);
}
__device__ __forceinline__ void load8(const float* p, int left, Eight<float>& v) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v.w[i] = i < left ? __float_as_uint(p[i]) : 0u;
}

// Eight results of a row, or the first `left` of them.
__device__ __forceinline__ void store8(float* z, int left, const float (&v)[8]) {
    if (left >= 8) {
        *reinterpret_cast<u32x4_a4*>(z) = __builtin_bit_cast(u32x4, f32x4{v[0], v[1], v[2], v[3]});
        *reinterpret_cast<u32x4_a4*>(z + 4) = __builtin_bit_cast(u32x4, f32x4{v[4], v[5], v[6], v[7]});
    } else {
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (i < left) z[i] = v[i];
    }
}
__device__ __forceinline__ void store8(uint16_t* z, int left, const float (&v)[8]) {
    if (left >= 8) {
        *reinterpret_cast<u32x4_a2*>(z) = u32x4{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
    } else {
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (i < left) z[i] = (uint16_t)(pack_bf16(v[i], 0.f) & 0xFFFFu);
    }
}

// Magnitudes are compared as integers: NaN and infinity are the largest.  Of fp32 one a word, of bfloat16 two.
__device__ __forceinline__ uint32_t larger(const uint16_t*, uint32_t m, uint32_t w) { return max_pairs(m, w & 0x7FFF7FFFu); }
__device__ __forceinline__ uint32_t larger(const float*, uint32_t m, uint32_t w) { return max(m, w & 0x7FFFFFFFu); }
// The fp32 bits of the largest of a word's magnitudes.
__device__ __forceinline__ uint32_t top_bits(const uint16_t*, uint32_t m) { return max(m << 16, m & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t top_bits(const float*, uint32_t m) { return m; }
template <typename T>
__device__ __forceinline__ uint32_t top_of(const Eight<T>& v) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < Eight<T>::kWords; ++i) m = larger((const T*)nullptr, m, v.w[i]);
    return top_bits((const T*)nullptr, m);
}

// The largest of 16 neighbouring lanes, to all of them.
__device__ __forceinline__ uint32_t max16(uint32_t m) {
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xB1, 0xF, 0xF, true));    // lanes 1 0 3 2
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4E, 0xF, 0xF, true));    // lanes 2 3 0 1
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x141, 0xF, 0xF, true));   // 7 .. 0 of each eight
    return max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x140, 0xF, 0xF, true));   // 15 .. 0
}

typedef short i16x2 __attribute__((ext_vector_type(2)));
// Two elements to the lower or upper half of a word of codes: the conversion divides by the scale and rounds to the nearest, ties to even.
template <bool UP>
__device__ __forceinline__ uint32_t codes2(uint32_t w, float a, float b, float s) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(__builtin_bit_cast(i16x2, w), a, b, s, UP));
}
template <bool UP>
__device__ __forceinline__ uint32_t codes2(uint32_t w, uint32_t pair, float s) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(__builtin_bit_cast(i16x2, w), bits_as<bf16x2>(pair), s, UP));
}
constexpr uint32_t kNanCodes = 0x7F7F7F7Fu;

__device__ __forceinline__ u32x2 codes8(const Eight<float>& v, uint32_t byte) {
    const float s = scale_of(byte);
    u32x2 c;
#pragma unroll
    for (int d = 0; d < 2; ++d) {
        c[d] = codes2<false>(0, bits_as<float>(v.w[4 * d]), bits_as<float>(v.w[4 * d + 1]), s);
        c[d] = codes2<true>(c[d], bits_as<float>(v.w[4 * d + 2]), bits_as<float>(v.w[4 * d + 3]), s);
        if (byte == 255u) c[d] = kNanCodes;
    }
    return c;
}
__device__ __forceinline__ u32x2 codes8(const Eight<uint16_t>& v, uint32_t byte) {
    const float s = scale_of(byte);
    u32x2 c;
#pragma unroll
    for (int d = 0; d < 2; ++d) {
        c[d] = codes2<false>(0, v.w[2 * d], s);
        c[d] = codes2<true>(c[d], v.w[2 * d + 1], s);
        if (byte == 255u) c[d] = kNanCodes;
    }
    return c;
}
// Column j of eight columns of four rows: the four codes in a word.
__device__ __forceinline__ uint32_t codes_down(const Eight<float> (&v)[4], int j, uint32_t byte) {
    const float s = scale_of(byte);
    uint32_t c = codes2<false>(0, bits_as<float>(v[0].w[j]), bits_as<float>(v[1].w[j]), s);
    c = codes2<true>(c, bits_as<float>(v[2].w[j]), bits_as<float>(v[3].w[j]), s);
    return byte == 255u ? kNanCodes : c;
}
__device__ __forceinline__ uint32_t codes_down(const Eight<uint16_t> (&v)[4], int j, uint32_t byte) {
    const float s = scale_of(byte);
    const uint32_t pick = (j & 1) ? 0x07060302u : 0x05040100u;   // the upper or lower halves of two words
    uint32_t c = codes2<false>(0, __builtin_amdgcn_perm(v[1].w[j / 2], v[0].w[j / 2], pick), s);
    c = codes2<true>(c, __builtin_amdgcn_perm(v[3].w[j / 2], v[2].w[j / 2], pick), s);
    return byte == 255u ? kNanCodes : c;
}

}  // namespace

}  // namespace daq
