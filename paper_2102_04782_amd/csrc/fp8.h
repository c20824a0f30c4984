// What the kernels of 8-bit floating point matrices and of experts' products share.
#pragma once

#include "lowbits.h"

namespace daq {

constexpr int kFp8Block = 128;     // elements that share a scale
constexpr int kFp8Group = 512;     // columns of a word of scale bytes
constexpr int64_t kFp8MaxK = ((int64_t)1 << 23) - kFp8Block;   // 256 rows of a product's operand stay within 32 bits
constexpr int kMaxExperts = 1024;
constexpr int64_t kMaxSlots = (int64_t)1 << 28;

// Rows of an experts' plan: what stands before every expert, [rows, tiles of 256, of 128, of 64][experts + 1].
enum { kTableRows = 0, kTable256 = 1, kTable128 = 2, kTable64 = 3 };
inline bool plan_ok(const daq_experts* p) {
    return p && p->tokens >= 0 && p->picks > 0 && p->experts > 0 && p->experts <= kMaxExperts && p->tokens < kMaxSlots / p->picks &&
           (p->tokens == 0 || (p->table && p->rows && p->place && !((uintptr_t)p->table & 3) && !((uintptr_t)p->rows & 3) && !((uintptr_t)p->place & 3)));
}
inline int64_t plan_slots(const daq_experts& p) { return p.tokens * p.picks; }
// At most so many row tiles of n rows have rows of one expert only.
inline int64_t most_tiles(const daq_experts& p, int64_t n) {
    const int64_t slots = plan_slots(p);
    return (slots + (n - 1) * std::min<int64_t>(p.experts, slots)) / n;
}

// fp8.hip: to 8 bits along the rows (checked sizes)
daq_status fp8_quantize_rows(const void* src, int dtype, int64_t rows, int64_t cols, int64_t ld, uint8_t* dst, hipStream_t st);
inline bool fp8_rows_grid_ok(int64_t rows, int64_t cols) { return grid_ok(ceil_div(rows, 16) * ceil_div(cols, kFp8Group), 256); }

#if defined(__HIPCC__)
// The scale byte of a block from the bits of its largest magnitude: the smallest power of two of which that is at most 448 = 1.75 * 2^8.
__device__ __forceinline__ uint32_t fp8_scale_byte(uint32_t top) {
    const uint32_t e = top >> 23, up = (top & 0x7FFFFFu) > 0x600000u ? 1u : 0u;
    return e >= 255u ? 255u : e + up > 8u ? e + up - 8u : 1u;
}
// The expert that tile t belongs to, `before` being the tiles before every expert (and in all): the number of experts whose tiles
// end at or before t.  The whole wave asks.
__device__ __forceinline__ int expert_of_tile(const int32_t* before, int experts, int t, int lane) {
    int e = 0;
    for (int first = 0; first < experts; first += kWave) {
        const bool past = first + lane < experts && before[first + lane + 1] <= t;
        const int n = __popcll(__ballot(past));
        e += n;
        if (n < kWave) break;
    }
    return __builtin_amdgcn_readfirstlane(e);
}
#endif

}  // namespace daq
