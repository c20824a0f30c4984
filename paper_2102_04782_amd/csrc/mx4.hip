// Microscaled 4-bit matrices: layout, quantization along rows and along columns, and back.
#include "lowbits.h"

namespace daq {

namespace {

struct PackArgs {
    const void* src;
    int64_t ld;
    int64_t rows, cols;      // of src
    uint8_t* codes;
    uint8_t* scales;
    int64_t row_blocks;      // of the packed matrix
    int groups;
    uint32_t key;            // of the random words
    uint32_t half;           // random words of a row of src
};

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
// The code of one element, stochastically.  t = |x| * 2^-e is at most 6; with p = 0, 1, 2 for t < 2, < 4, more, the elements
// around it are 2^(p-1) apart and have the codes n + 2p, n = t / 2^(p-1): so the code is floor(t * 2^(1-p) + V * 2^-16) + 2p with
// V = 65535 - U, evaluated on t * 2^(17-p) cut off to an integer.
__device__ __forceinline__ uint32_t stochastic_code(float x, float inv, uint32_t u16) {
    const float t = fabsf(x) * inv;
    const int e = (int)(__float_as_uint(t) >> 23) - 127;
    const int p = min(max(e, 0), 2);
    const uint32_t n = (uint32_t)(t * bits_as<float>((uint32_t)(144 - p) << 23));
    return (((n + (65535u - u16)) >> 16) + 2u * (uint32_t)p) | ((__float_as_uint(x) >> 28) & 8u);
}
__device__ __forceinline__ float elem_f32(const uint32_t (&v)[32], int i) { return bits_as<float>(v[i]); }
__device__ __forceinline__ float elem_f32(const uint32_t (&v)[16], int i) { return (i & 1) ? bf16_hi(v[i / 2]) : bf16_lo(v[i / 2]); }
// word(i): the random word of element i, half(i): which half of it
template <int W, typename F>
__device__ __forceinline__ u32x4 stochastic_codes(const uint32_t (&v)[W], uint32_t byte, F draw) {
    if (byte == 255u) return u32x4{0, 0, 0, 0};
    const float inv = inverse_scale(byte);
    u32x4 c;
#pragma unroll
    for (int d = 0; d < 4; ++d) {
        uint32_t w = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) w |= stochastic_code(elem_f32(v, 8 * d + i), inv, draw(8 * d + i)) << (4 * i);
        c[d] = w;
    }
    return c;
}

// A block of a row: n of its 32 elements are there, the others are zero.
__device__ __forceinline__ void load_block(const float* p, int n, uint32_t (&v)[32]) {
    if (n >= 32) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const u32x4_a4 q = *reinterpret_cast<const u32x4_a4*>(p + 4 * i);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[4 * i + j] = q[j];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = i < n ? __float_as_uint(p[i]) : 0u;
    }
}
__device__ __forceinline__ void load_block(const uint16_t* p, int n, uint32_t (&v)[16]) {
    if (n >= 32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const u32x4_a2 q = *reinterpret_cast<const u32x4_a2*>(p + 8 * i);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[4 * i + j] = q[j];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const uint32_t lo = 2 * i < n ? p[2 * i] : 0u, hi = 2 * i + 1 < n ? p[2 * i + 1] : 0u;
            v[i] = lo | (hi << 16);
        }
    }
}
template <typename T> struct Words;
template <> struct Words<float> { static constexpr int kBlock = 32; };
template <> struct Words<uint16_t> { static constexpr int kBlock = 16; };

// Blocks along the rows of src.  A wave takes 32 rows x 256 columns, a lane four blocks of one row (lane / 32 says which of
// the two blocks of each 64 columns), so that codes leave as whole KiB and the four scale bytes as one word.
template <typename T, bool SR>
__global__ __launch_bounds__(256) void k_mx4_rows(PackArgs p) {
    const int lane = threadIdx.x % kWave;
    const int64_t wave = (int64_t)blockIdx.x * 4 + threadIdx.x / kWave;
    const int64_t rb = wave / p.groups;
    const int g = (int)(wave - rb * p.groups);
    if (rb >= p.row_blocks) return;
    const int half = lane / 32, r32 = lane % 32;
    const int64_t r = rb * 32 + r32;
    const bool there = r < p.rows;
    const T* row = static_cast<const T*>(p.src) + (there ? r : 0) * p.ld;
    uint32_t word = 0;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
        const int64_t c0 = (int64_t)g * kMxGroup + s * 64 + half * 32;
        const int64_t left = there ? p.cols - c0 : 0;
        u32x4 codes = {0, 0, 0, 0};
        if (left > 0) {
            uint32_t v[Words<T>::kBlock];
            load_block(row + c0, (int)min(left, (int64_t)32), v);
            const uint32_t top = top_of(v);
            const uint32_t byte = SR ? scale_byte_whole(top) : scale_byte<2>(top);
            if constexpr (SR) {
                const uint32_t first = (uint32_t)r * p.half + (uint32_t)(c0 / 2);
                codes = stochastic_codes(v, byte, [&](int i) {
                    const uint32_t h = fmix32((first + (uint32_t)(i / 2)) ^ p.key);
                    return (i & 1) ? h & 0xFFFFu : h >> 16;
                });
            } else {
                codes = nearest_codes(v, byte);
            }
            word |= byte << (8 * s);
        }
        *reinterpret_cast<u32x4*>(p.codes + (((rb * p.groups + g) * 4 + s) * 2 + half) * 512 + r32 * 16) = codes;
    }
    *reinterpret_cast<uint32_t*>(p.scales + ((rb * p.groups + g) * 2 + half) * 128 + r32 * 4) = word;
}

// Blocks along the columns of src: rows of the packed matrix are columns of src.  A wave takes 64 columns x 256 rows, a lane
// two neighbouring columns of the 32 rows of a block (lane / 32 says which block of each 64 rows), so that src is read in
// pieces of 64 columns and each lane writes 32 bytes in a row.
template <typename T>
__device__ __forceinline__ void load_pair(const T* p, bool one, bool two, uint32_t& a, uint32_t& b);
template <>
__device__ __forceinline__ void load_pair<float>(const float* p, bool one, bool two, uint32_t& a, uint32_t& b) {
    if (two) {
        const u32x2_a4 q = *reinterpret_cast<const u32x2_a4*>(p);
        a = q[0];
        b = q[1];
    } else {
        a = one ? __float_as_uint(*p) : 0u;
        b = 0u;
    }
}
template <>
__device__ __forceinline__ void load_pair<uint16_t>(const uint16_t* p, bool one, bool two, uint32_t& a, uint32_t& b) {
    const uint32_t q = two ? *reinterpret_cast<const u32_a2*>(p) : one ? (uint32_t)*p : 0u;
    a = q & 0xFFFFu;
    b = q >> 16;
}

template <typename T, bool SR>
__global__ __launch_bounds__(256) void k_mx4_columns(PackArgs p) {
    const int lane = threadIdx.x % kWave;
    const int64_t wave = (int64_t)blockIdx.x * 4 + threadIdx.x / kWave;
    const int64_t pairs = (p.row_blocks + 1) / 2;   // pairs of row blocks of the packed matrix
    const int64_t g = wave / pairs;                 // neighbouring waves take neighbouring columns of src
    const int64_t rp = wave - g * pairs;
    if (g >= p.groups) return;
    const int half = lane / 32;
    const int64_t c = rp * 64 + (lane % 32) * 2;    // the two columns of src
    const bool one = c < p.cols, two = c + 1 < p.cols;
    const T* src = static_cast<const T*>(p.src) + (one ? c : 0);
    const int64_t rb = c / 32;
    const int r32 = (int)(c % 32);
    uint32_t words[2] = {0, 0};
#pragma unroll 1
    for (int s = 0; s < 4; ++s) {
        const int64_t r0 = g * kMxGroup + s * 64 + half * 32;
        uint32_t v[2][Words<T>::kBlock];
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                const bool in = r0 + i < p.rows;
                load_pair<T>(src + (in ? r0 + i : 0) * p.ld, one && in, two && in, v[0][i], v[1][i]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                uint32_t a[2], b[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const bool in = r0 + 2 * i + j < p.rows;
                    load_pair<T>(src + (in ? r0 + 2 * i + j : 0) * p.ld, one && in, two && in, a[j], b[j]);
                }
                v[0][i] = a[0] | (a[1] << 16);
                v[1][i] = b[0] | (b[1] << 16);
            }
        }
        u32x4 codes[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const uint32_t top = top_of(v[j]);
            const uint32_t byte = SR ? scale_byte_whole(top) : scale_byte<2>(top);
            if constexpr (SR) {
                const uint32_t first = (uint32_t)r0 * p.half + (uint32_t)(c / 2);
                codes[j] = stochastic_codes(v[j], byte, [&](int i) {
                    const uint32_t h = fmix32((first + (uint32_t)i * p.half) ^ p.key);
                    return j ? h & 0xFFFFu : h >> 16;
                });
            } else {
                codes[j] = nearest_codes(v[j], byte);
            }
            if (r0 < p.rows && (j ? two : one)) words[j] |= byte << (8 * s);   // (not of padding)
        }
        if (rb < p.row_blocks) {
            u32x4* to = reinterpret_cast<u32x4*>(p.codes + (((rb * p.groups + g) * 4 + s) * 2 + half) * 512 + r32 * 16);
            to[0] = codes[0];
            to[1] = codes[1];
        }
    }
    if (rb < p.row_blocks)
        *reinterpret_cast<u32x2*>(p.scales + ((rb * p.groups + g) * 2 + half) * 128 + r32 * 4) = u32x2{words[0], words[1]};
}

struct ValuesArgs {
    const uint8_t* codes;
    const uint8_t* scales;
    int64_t rows, cols, row_blocks;
    int groups;
    void* dst;
    int64_t ld;
};

// Waves and lanes as in k_mx4_rows.
template <typename T>
__global__ __launch_bounds__(256) void k_mx4_values(ValuesArgs p) {
    const int lane = threadIdx.x % kWave;
    const int64_t wave = (int64_t)blockIdx.x * 4 + threadIdx.x / kWave;
    const int64_t rb = wave / p.groups;
    const int g = (int)(wave - rb * p.groups);
    if (rb >= p.row_blocks) return;
    const int half = lane / 32, r32 = lane % 32;
    const int64_t r = rb * 32 + r32;
    if (r >= p.rows) return;
    const uint32_t word = *reinterpret_cast<const uint32_t*>(p.scales + ((rb * p.groups + g) * 2 + half) * 128 + r32 * 4);
    T* row = static_cast<T*>(p.dst) + r * p.ld;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
        const int64_t c0 = (int64_t)g * kMxGroup + s * 64 + half * 32;
        const int64_t left = p.cols - c0;
        if (left <= 0) break;
        const u32x4 codes = *reinterpret_cast<const u32x4*>(p.codes + (((rb * p.groups + g) * 4 + s) * 2 + half) * 512 + r32 * 16);
        const uint32_t byte = (word >> (8 * s)) & 255u;
        const float scale = scale_of(byte);
        const bool nan = byte == 255u;
        if constexpr (sizeof(T) == 4) {
            float v[32];
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                f32x2 q[4];
                q[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[d], scale, 0);
                q[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[d], scale, 1);
                q[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[d], scale, 2);
                q[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[d], scale, 3);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    v[8 * d + 2 * i] = nan ? scale : q[i][0];
                    v[8 * d + 2 * i + 1] = nan ? scale : q[i][1];
                }
            }
            if (left >= 32) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    *reinterpret_cast<u32x4_a4*>(row + c0 + 4 * i) =
                        u32x4_a4{__float_as_uint(v[4 * i]), __float_as_uint(v[4 * i + 1]), __float_as_uint(v[4 * i + 2]), __float_as_uint(v[4 * i + 3])};
            } else {
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    if (i < left) row[c0 + i] = v[i];
            }
        } else {
            uint32_t v[16];
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                v[4 * d] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[d], scale, 0));
                v[4 * d + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[d], scale, 1));
                v[4 * d + 2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[d], scale, 2));
                v[4 * d + 3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[d], scale, 3));
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = nan ? 0x7FC07FC0u : v[i];
            if (left >= 32) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    *reinterpret_cast<u32x4_a2*>(row + c0 + 8 * i) = u32x4_a2{v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]};
            } else {
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    if (i < left) row[c0 + i] = (uint16_t)(v[i / 2] >> (16 * (i & 1)));
            }
        }
    }
}

}  // namespace

daq_status mx4_quantize(const void* src, int dtype, int64_t rows, int64_t cols, int64_t ld, bool transpose, bool stochastic,
                        uint64_t seed, uint8_t* dst, hipStream_t st) {
    daq_mx4_layout L;
    const daq_status rc = transpose ? daq_layout_mx4(cols, rows, &L) : daq_layout_mx4(rows, cols, &L);
    if (rc != DAQ_OK) return rc;
    if (L.bytes == 0) return DAQ_OK;
    PackArgs p{src, ld, rows, cols, dst, dst + L.off_scales, L.row_blocks, L.groups, (uint32_t)round_keys(seed), (uint32_t)((cols + 1) / 2)};
    const int64_t waves = transpose ? ceil_div(L.row_blocks, 2) * L.groups : (int64_t)L.row_blocks * L.groups;
    if (!grid_ok(ceil_div(waves, 4))) return DAQ_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)ceil_div(waves, 4)), block(256);
#define DAQ_MX4_PACK(KERNEL, NAME)                                                                                          \
    do {                                                                                                                    \
        if (dtype == DAQ_BF16) {                                                                                            \
            if (stochastic) DAQ_LAUNCH(NAME, st, hipLaunchKernelGGL((KERNEL<uint16_t, true>), grid, block, 0, st, p));      \
            else DAQ_LAUNCH(NAME, st, hipLaunchKernelGGL((KERNEL<uint16_t, false>), grid, block, 0, st, p));                \
        } else {                                                                                                            \
            if (stochastic) DAQ_LAUNCH(NAME, st, hipLaunchKernelGGL((KERNEL<float, true>), grid, block, 0, st, p));         \
            else DAQ_LAUNCH(NAME, st, hipLaunchKernelGGL((KERNEL<float, false>), grid, block, 0, st, p));                   \
        }                                                                                                                   \
    } while (0)
    if (transpose) DAQ_MX4_PACK(k_mx4_columns, "mx4_columns");
    else DAQ_MX4_PACK(k_mx4_rows, "mx4_rows");
#undef DAQ_MX4_PACK
    return DAQ_OK;
}

daq_status mx4_quantize_check(const void* src, int dtype, int64_t rows, int64_t cols, int64_t ld, int mode) {
    if (!dtype_ok(dtype) || (mode != DAQ_ROUND_NEAREST && mode != DAQ_ROUND_STOCHASTIC)) return DAQ_ERR_INVALID_ARG;
    const daq_status rc = matrix_size(rows, cols);
    if (rc != DAQ_OK) return rc;
    if (rows > 0 && (!src || !elem_aligned(src, dtype) || ld < cols)) return DAQ_ERR_INVALID_ARG;
    // the counter of the random words holds 32 bits
    if (mode == DAQ_ROUND_STOCHASTIC && rows * cols > ((int64_t)1 << 31)) return DAQ_ERR_UNSUPPORTED;
    return DAQ_OK;
}

}  // namespace daq

using namespace daq;

extern "C" daq_status daq_layout_mx4(int64_t rows, int64_t cols, daq_mx4_layout* out) {
    if (!out) return DAQ_ERR_INVALID_ARG;
    if (rows < 0 || cols < 0) return DAQ_ERR_INVALID_ARG;
    *out = daq_mx4_layout{};
    if (rows == 0 || cols == 0) return DAQ_OK;   // (a transposed matrix of no rows has no columns)
    const daq_status rc = matrix_size(rows, cols);
    if (rc != DAQ_OK) return rc;
    const int64_t rb = ceil_div(rows, 32), groups = ceil_div(cols, kMxGroup);
    out->row_blocks = (int32_t)rb;
    out->groups = (int32_t)groups;
    out->off_scales = rb * groups * 4096;
    out->bytes = out->off_scales + rb * groups * 256;
    return DAQ_OK;
}

extern "C" daq_status daq_mx4_quantize(const void* src, daq_dtype dtype, int64_t rows, int64_t cols, int64_t ld, int32_t transpose,
                                       daq_round mode, uint64_t seed, uint8_t* dst, void* stream) {
    const daq_status rc = mx4_quantize_check(src, dtype, rows, cols, ld, mode);
    if (rc != DAQ_OK) return rc;
    if (rows > 0 && (!dst || !aligned256(dst))) return DAQ_ERR_INVALID_ARG;
    return mx4_quantize(src, dtype, rows, cols, ld, transpose != 0, mode == DAQ_ROUND_STOCHASTIC, seed, dst, (hipStream_t)stream);
}

extern "C" daq_status daq_mx4_dequantize(const uint8_t* src, int64_t rows, int64_t cols, void* dst, daq_dtype dtype, int64_t ld,
                                         void* stream) {
    if (!dtype_ok(dtype)) return DAQ_ERR_INVALID_ARG;
    if (rows >= 0 && cols == 0) return DAQ_OK;
    const daq_status rc = matrix_size(rows, cols);
    if (rc != DAQ_OK) return rc;
    if (rows == 0) return DAQ_OK;
    if (!src || !aligned256(src) || !dst || !elem_aligned(dst, dtype) || ld < cols) return DAQ_ERR_INVALID_ARG;
    daq_mx4_layout L;
    daq_layout_mx4(rows, cols, &L);
    const int64_t blocks = ceil_div((int64_t)L.row_blocks * L.groups, 4);
    if (!grid_ok(blocks)) return DAQ_ERR_UNSUPPORTED;
    const ValuesArgs p{src, src + L.off_scales, rows, cols, L.row_blocks, L.groups, dst, ld};
    hipStream_t st = (hipStream_t)stream;
    if (dtype == DAQ_BF16) DAQ_LAUNCH("mx4_values", st, hipLaunchKernelGGL(k_mx4_values<uint16_t>, dim3((unsigned)blocks), dim3(256), 0, st, p));
    else DAQ_LAUNCH("mx4_values", st, hipLaunchKernelGGL(k_mx4_values<float>, dim3((unsigned)blocks), dim3(256), 0, st, p));
    return DAQ_OK;
}
