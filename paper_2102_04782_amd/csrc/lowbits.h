// What the kernels of microscaled 4-bit matrices and 8-bit checkpoints share: blocks of 32 elements with a power-of-two scale.
#pragma once

#include "daq_internal.h"

namespace daq {

constexpr int kMxBlock = 32;       // elements that share a scale
constexpr int kMxGroup = 256;      // columns of an mx4 scale word group: four matrix instructions of 64
constexpr int64_t kMaxElems = (int64_t)1 << 40;

inline bool dtype_ok(int dtype) { return dtype == DAQ_FP32 || dtype == DAQ_BF16; }
inline int dtype_size(int dtype) { return dtype == DAQ_BF16 ? 2 : 4; }
inline bool elem_aligned(const void* p, int dtype) { return ((uintptr_t)p & (uintptr_t)(dtype_size(dtype) - 1)) == 0; }
inline bool aligned256(const void* p) { return ((uintptr_t)p & 255u) == 0; }
// DAQ_OK for sizes of a matrix that the entry points take (zero rows among them).
inline daq_status matrix_size(int64_t rows, int64_t cols) {
    if (rows < 0 || cols <= 0) return DAQ_ERR_INVALID_ARG;
    constexpr int64_t most = ((int64_t)1 << 31) - 1;
    if (rows > most || cols > most || rows * cols > kMaxElems) return DAQ_ERR_UNSUPPORTED;
    return DAQ_OK;
}
// Workgroups along the first axis of a grid: a launch takes fewer than 2^32 threads along one.
inline bool grid_ok(int64_t blocks, int threads) { return blocks * threads < ((int64_t)1 << 32); }

// mx4.hip: src to its packed form, and what its arguments have to be
daq_status mx4_quantize_check(const void* src, int dtype, int64_t rows, int64_t cols, int64_t ld, int mode);
daq_status mx4_quantize(const void* src, int dtype, int64_t rows, int64_t cols, int64_t ld, bool transpose, bool stochastic,
                        uint64_t seed, uint8_t* dst, hipStream_t st);

// mx4_matmul.hip: the form of a product (row blocks of 32 of either operand, groups of 256 along k), and whether a linear layer's
// workgroups quantize its rows themselves
enum class MatmulForm { kFew, kSmall, kBig };
MatmulForm matmul_form(int64_t a_blocks, int64_t b_blocks, int64_t groups);
bool raw_rows(int64_t M, int64_t K, int dtype, int mode);
// ckpt8_wgrad.hip: sizes of a weight gradient and where its workspace holds what
struct WgradPlan {
    int n_blocks, k_blocks, steps, parts;   // parts: of a value of dY
    bool few;                               // small products, no tiles: per_split is of 16 tokens then
    bool flat;                              // dY as it is, not in tiles
    bool big;                               // tiles of 256 x 256 instead of 128 x 128
    int splits, per_split;                  // parts of the tokens, and stages of one
    int64_t off_x, off_part, pitch, bytes;
};
WgradPlan wgrad_plan(int64_t M, int64_t N, int64_t K, int dtype, int64_t lddy, int dy_misaligned);

#if defined(__HIPCC__)
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
// Rows of any stride begin at any element: vectors of the alignment of one.
typedef uint32_t u32x4_a2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x2_a2 __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t u32_a2 __attribute__((aligned(2)));
typedef uint32_t u32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x2_a4 __attribute__((ext_vector_type(2), aligned(4)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

template <typename T> __device__ __forceinline__ T bits_as(uint32_t u) { return __builtin_bit_cast(T, u); }

// The larger of two pairs of unsigned 16-bit values.
__device__ __forceinline__ uint32_t max_pairs(uint32_t a, uint32_t b) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}
// The scale byte of a block from the bits of its largest magnitude (an integer maximum: NaN and infinity are the largest):
// 2^(floor(log2 a) - BELOW) as byte - 127, at least 1; 255 for a block with a NaN or an infinity.
template <int BELOW>
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
    const uint32_t e = top >> 23;
    return e >= 255u ? 255u : e > (uint32_t)BELOW ? e - BELOW : 1u;
}
// The same for 4-bit codes that must not be cut off: the smallest power of two of which the largest magnitude is at most 6.
__device__ __forceinline__ uint32_t scale_byte_whole(uint32_t top) {
    const uint32_t e = top >> 23, up = (top & 0x7FFFFFu) > 0x400000u ? 1u : 0u;
    return e >= 255u ? 255u : e + up > 2u ? e + up - 2u : 1u;
}
// 2^(byte - 127), NaN for 255; and 1 over it for bytes 1 .. 253.
__device__ __forceinline__ float scale_of(uint32_t byte) { return bits_as<float>(byte == 255u ? 0x7FC00000u : byte << 23); }
__device__ __forceinline__ float inverse_scale(uint32_t byte) { return bits_as<float>((254u - byte) << 23); }

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const bf16x2 p = {(__bf16)lo, (__bf16)hi};   // to nearest, ties to even
    return __builtin_bit_cast(uint32_t, p);
}
__device__ __forceinline__ float bf16_lo(uint32_t u) { return bits_as<float>(u << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t u) { return bits_as<float>(u & 0xFFFF0000u); }
#endif

}  // namespace daq
