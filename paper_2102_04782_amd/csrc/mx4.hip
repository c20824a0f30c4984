// Microscaled 4-bit matrices: layout, quantization along rows and along columns, and back.
//
// A block of 32 elements becomes 16 bytes of codes and a scale byte, so a bfloat16 matrix of 2 bytes an element is read once and 17/32
// of one are written.  Measured (us, and TB/s of what is read and written): 16384 x 8192 by rows 62-69 (5.2); 16384 x 4096 by rows 24.4,
// by columns 26.9 (6.4), stochastically 38.5 and 41 - there the vector instructions bound it, 17 an element, 5 of them the random word's;
// back to bfloat16 26.4.  Small matrices take the 3 us of a launch whose lanes wait for memory once: a lane has one block, and asks for
// all of it at a time (77 x 1000 3.3; with four blocks a lane, one after the other, 4.7).
#include <type_traits>

#include "mx4_block.h"

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

// Blocks along the rows of src.  A workgroup takes 32 rows x 256 columns, a wave 64 of the columns, a lane one block (lane / 32 says which
// of a row's two), so that codes leave as whole KiB; the scale bytes of the four waves make words on their way through LDS.
template <typename T, bool SR>
__global__ __launch_bounds__(256) void k_mx4_rows(PackArgs p) {
    __shared__ uint32_t words[64];
    const int lane = threadIdx.x % kWave, s = threadIdx.x / kWave;
    const int64_t rb = blockIdx.x / p.groups;
    const int g = (int)(blockIdx.x - rb * p.groups);
    const int half = lane / 32, r32 = lane % 32;
    const int64_t r = rb * 32 + r32, c = (int64_t)g * kMxGroup + s * 64 + half * 32, left = r < p.rows ? p.cols - c : 0;
    const T* from = static_cast<const T*>(p.src) + r * p.ld + c;
    uint32_t v[Words<T>::kBlock];
    if (left >= 32) load_block(from, v);
    else load_block(from, (int)max(left, (int64_t)0), v);
    const uint32_t top = top_of(v);
    const uint32_t byte = SR ? scale_byte_whole(top) : scale_byte<2>(top);
    u32x4 codes;
    if constexpr (SR) {
        const uint32_t first = (uint32_t)r * p.half + (uint32_t)(c / 2);
        uint32_t word = 0;
        codes = stochastic_codes(v, byte, [&](int i) {
            if (i & 1) word = ~fmix32((first + (uint32_t)(i / 2)) ^ p.key);   // (asked for from the last one on)
            return (i & 1) ? word & 0xFFFFu : word >> 16;
        });
    } else {
        codes = nearest_codes(v, byte);
    }
    *reinterpret_cast<u32x4*>(p.codes + ((blockIdx.x * 4 + s) * (int64_t)2 + half) * 512 + r32 * 16) = codes;
    reinterpret_cast<uint8_t*>(words)[lane * 4 + s] = (uint8_t)(left > 0 ? byte : 0u);
    __syncthreads();
    if (s == 0) *reinterpret_cast<uint32_t*>(p.scales + (int64_t)blockIdx.x * 256 + lane * 4) = words[lane];
}

// Blocks along the columns of src: rows of the packed matrix are columns of src.  A workgroup takes 64 columns x 256 rows, a wave 64 of the
// rows, a lane two neighbouring columns of the 32 rows of a block (lane / 32 says which of a column's two), so that src is read in
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
    __shared__ uint32_t words[128];
    const int lane = threadIdx.x % kWave, s = threadIdx.x / kWave;
    const int64_t pairs = (p.row_blocks + 1) / 2;   // pairs of row blocks of the packed matrix
    const int64_t g = blockIdx.x / pairs;           // neighbouring workgroups take neighbouring columns of src
    const int64_t rp = blockIdx.x - g * pairs;
    const int half = lane / 32;
    const int64_t c = rp * 64 + (lane % 32) * 2;    // the two columns of src
    const bool one = c < p.cols, two = c + 1 < p.cols;
    const int64_t r0 = g * kMxGroup + s * 64 + half * 32;
    const T* src = static_cast<const T*>(p.src) + (one ? c : 0);
    uint32_t v[2][Words<T>::kBlock];
    // inside the matrix every element is asked for before the first is used
    const bool whole = (rp + 1) * 64 <= p.cols && g * kMxGroup + s * 64 + 64 <= p.rows;   // the same for the wave
    auto load = [&](auto all) {
        constexpr bool kAll = decltype(all)::value;
        uint32_t a[32], b[32];
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            const bool in = kAll || r0 + i < p.rows;
            load_pair<T>(src + (in ? r0 + i : 0) * p.ld, kAll || (one && in), kAll || (two && in), a[i], b[i]);
        }
#pragma unroll
        for (int i = 0; i < Words<T>::kBlock; ++i) {
            v[0][i] = sizeof(T) == 4 ? a[i] : a[2 * i % 32] | (a[(2 * i + 1) % 32] << 16);
            v[1][i] = sizeof(T) == 4 ? b[i] : b[2 * i % 32] | (b[(2 * i + 1) % 32] << 16);
        }
    };
    if (whole) load(std::true_type{});
    else load(std::false_type{});
    u32x4 codes[2];
    uint32_t bytes[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const uint32_t top = top_of(v[j]);
        bytes[j] = SR ? scale_byte_whole(top) : scale_byte<2>(top);
        if constexpr (!SR) codes[j] = nearest_codes(v[j], bytes[j]);
    }
    if constexpr (SR) {   // the two columns of a row share a random word
        uint32_t w[32];
        const uint32_t first = (uint32_t)r0 * p.half + (uint32_t)(c / 2);
#pragma unroll
        for (int i = 0; i < 32; ++i) w[i] = ~fmix32((first + (uint32_t)i * p.half) ^ p.key);
        codes[0] = stochastic_codes(v[0], bytes[0], [&](int i) { return w[i] >> 16; });
        codes[1] = stochastic_codes(v[1], bytes[1], [&](int i) { return w[i] & 0xFFFFu; });
    }
    const int64_t rb = c / 32;
    if (rb < p.row_blocks) {
        u32x4* to = reinterpret_cast<u32x4*>(p.codes + (((rb * p.groups + g) * 4 + s) * 2 + half) * 512 + (c % 32) * 16);
        to[0] = codes[0];
        to[1] = codes[1];
    }
    uint8_t* mine = reinterpret_cast<uint8_t*>(words) + lane * 8 + s;
    mine[0] = (uint8_t)(r0 < p.rows && one ? bytes[0] : 0u);   // (no scale for padding)
    mine[4] = (uint8_t)(r0 < p.rows && two ? bytes[1] : 0u);
    __syncthreads();
    if (s == 0 && rb < p.row_blocks)
        *reinterpret_cast<u32x2*>(p.scales + ((rb * p.groups + g) * 2 + half) * 128 + (c % 32) * 4) = u32x2{words[lane * 2], words[lane * 2 + 1]};
}

struct ValuesArgs {
    const uint8_t* codes;
    const uint8_t* scales;
    int64_t rows, cols, row_blocks;
    int groups;
    void* dst;
    int64_t ld;
};

// Workgroups and waves as in k_mx4_rows; a lane takes a piece of 16 bytes of a row of dst, so that every store of the wave fills whole
// lines: 8 rows of 64 bfloat16, 4 rows of 64 fp32 at a time.
template <typename T>
__global__ __launch_bounds__(256) void k_mx4_values(ValuesArgs p) {
    constexpr int kPiece = 16 / sizeof(T), kAcross = 64 / kPiece, kRows = kWave / kAcross;
    const int lane = threadIdx.x % kWave, s = threadIdx.x / kWave;
    const int64_t rb = blockIdx.x / p.groups;
    const int g = (int)(blockIdx.x - rb * p.groups);
    const int col = (lane % kAcross) * kPiece, half = col / 32;
    const int64_t c = (int64_t)g * kMxGroup + s * 64 + col, left = p.cols - c;
    if (left <= 0) return;
    const uint8_t* codes = p.codes + ((blockIdx.x * 4 + s) * (int64_t)2 + half) * 512 + (col % 32) / 2;
    const uint8_t* scales = p.scales + (int64_t)blockIdx.x * 256 + half * 128 + s;
    uint32_t word[32 / kRows], byte[32 / kRows];
#pragma unroll
    for (int i = 0; i < 32 / kRows; ++i) {
        const int r32 = i * kRows + lane / kAcross;
        word[i] = kPiece == 8 ? *reinterpret_cast<const uint32_t*>(codes + r32 * 16) : (uint32_t)*reinterpret_cast<const uint16_t*>(codes + r32 * 16);
        byte[i] = scales[r32 * 4];
    }
#pragma unroll
    for (int i = 0; i < 32 / kRows; ++i) {
        const int64_t r = rb * 32 + i * kRows + lane / kAcross;
        if (r >= p.rows) return;
        const float scale = scale_of(byte[i]);
        const bool nan = byte[i] == 255u;
        u32x4 v;
        if constexpr (sizeof(T) == 4) {
            const f32x2 lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word[i], scale, 0), hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word[i], scale, 1);
            v = u32x4{__float_as_uint(lo[0]), __float_as_uint(lo[1]), __float_as_uint(hi[0]), __float_as_uint(hi[1])};
        } else {
            v[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word[i], scale, 0));
            v[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word[i], scale, 1));
            v[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word[i], scale, 2));
            v[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word[i], scale, 3));
        }
        if (nan) v = sizeof(T) == 4 ? u32x4{0x7FC00000u, 0x7FC00000u, 0x7FC00000u, 0x7FC00000u} : u32x4{0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u};
        T* z = static_cast<T*>(p.dst) + r * p.ld + c;
        if (left >= kPiece) {
            if constexpr (sizeof(T) == 4) *reinterpret_cast<u32x4_a4*>(z) = v;
            else *reinterpret_cast<u32x4_a2*>(z) = v;
        } else {
#pragma unroll
            for (int k = 0; k < kPiece - 1; ++k)
                if (k < left) {
                    if constexpr (sizeof(T) == 4) z[k] = bits_as<float>(v[k]);
                    else z[k] = (uint16_t)(v[k / 2] >> (16 * (k & 1)));
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
    const int64_t blocks = transpose ? ceil_div(L.row_blocks, 2) * L.groups : (int64_t)L.row_blocks * L.groups;
    if (!grid_ok(blocks, 256)) return DAQ_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)blocks), block(256);
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
    const int64_t blocks = (int64_t)L.row_blocks * L.groups;
    if (!grid_ok(blocks, 256)) return DAQ_ERR_UNSUPPORTED;
    const ValuesArgs p{src, src + L.off_scales, rows, cols, L.row_blocks, L.groups, dst, ld};
    hipStream_t st = (hipStream_t)stream;
    if (dtype == DAQ_BF16) DAQ_LAUNCH("mx4_values", st, hipLaunchKernelGGL(k_mx4_values<uint16_t>, dim3((unsigned)blocks), dim3(256), 0, st, p));
    else DAQ_LAUNCH("mx4_values", st, hipLaunchKernelGGL(k_mx4_values<float>, dim3((unsigned)blocks), dim3(256), 0, st, p));
    return DAQ_OK;
}
