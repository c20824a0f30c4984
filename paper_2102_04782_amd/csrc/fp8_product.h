// What the kernels of 8-bit floating point products share: their arguments, and where a tile lies.
#pragma once

#include <type_traits>

#include "fp8_block.h"
#include "tile_product.h"

namespace daq {

struct Fp8Operand {
    const uint8_t* codes;
    const uint8_t* scales;
    int64_t rows, pitch;
};

struct ProductArgs {
    Fp8Operand a, b;
    int64_t M, N;             // of one product
    int stages;               // blocks of 128 of the summed axis
    void* d;
    int64_t ldd;
    int bf16, accumulate, stream;   // stream: results pass the caches by
    int tiles_m, tiles_n;     // (experts' rows: tiles_m is the most there can be)
    int splits, per_split;    // of the summed axis: part z, of per_split stages, goes to d + z * M * ldd
    // experts
    const int32_t* table;
    const int32_t* order;
    int experts, picks;       // picks: row p of the order is row order[p] / picks of A, 0: row p
    int64_t stride;           // from one expert's gradient to the next
};
enum class Of { kWhole, kExpertRows, kExpertWeights };

namespace {

// 32 x 32 x 64; the scale is the lowest byte of its word.
__device__ __forceinline__ v16f mfma8(v8i x, v8i y, v16f c, int sx, int sy) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, y, c, 0, 0, 0, sx, 0, sy);
}

// Eight codes to bfloat16, times the scale: exact, but what the scale takes beyond bfloat16's range.
__device__ __forceinline__ v4i in_bf16(int lo, int hi, float s) {
    const bf16x2 v[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s, true),
                         __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s, true)};
    return v4i{__builtin_bit_cast(int, v[0]), __builtin_bit_cast(int, v[1]), __builtin_bit_cast(int, v[2]), __builtin_bit_cast(int, v[3])};
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t bytes_of(const uint8_t* from, int64_t n) {
    return __builtin_amdgcn_make_buffer_rsrc((void*)from, 0, (int)(n < (int64_t)kTileReach ? (uint32_t)n : kTileReach), 0x00020000);
}

// The tiles of ROWS x COLS results that an XCD takes, numbered from 0: a run of them all; of experts' gradients, whose lengths differ, a run of every
// expert's, another XCD's for every expert.
template <int ROWS, Of OF>
struct TileCount {
    const int32_t* before;    // experts' rows: tiles before every expert
    int tiles_m, all, per_xcd, mine;    // all: of an expert's gradient; mine: of this XCD (host: all of a launch's are within 31 bits)
    __device__ __forceinline__ explicit TileCount(const ProductArgs& p) {
        constexpr int kTable = ROWS == 256 ? kTable256 : ROWS == 128 ? kTable128 : kTable64;
        before = OF == Of::kExpertRows ? p.table + kTable * (p.experts + 1) : nullptr;
        tiles_m = OF == Of::kExpertRows ? __builtin_amdgcn_readfirstlane(before[p.experts]) : p.tiles_m;
        all = tiles_m * p.tiles_n;
        per_xcd = (all + kXcd - 1) / kXcd;
        mine = OF == Of::kExpertWeights ? p.experts * per_xcd : max(0, min(per_xcd, all - xcd() * per_xcd));
    }
    static __device__ __forceinline__ int xcd() { return (int)(blockIdx.x % kXcd); }
};
// Workgroups of a launch with one for every tile.
template <Of OF>
int64_t tile_groups(const ProductArgs& p) { return round_up((int64_t)p.tiles_m * p.tiles_n, kXcd) * (OF == Of::kExpertWeights ? p.experts : 1); }

// A tile: rows a0 .. of A (a_end: the first that is not its product's), rows b0 .. of B, stages s0 .. s1 - 1, and its results, of which row
// a0, column c0 are the first.
struct Tile {
    int64_t a0, a_end, b0, b_end, c0;
    int s0, s1;
    uint8_t* d;
};
// The XCD's tile i, in bands of four row tiles, whose panels its L2 holds; false: there is none.  The whole wave asks.
template <int ROWS, int COLS, Of OF>
__device__ __forceinline__ bool tile_at(const ProductArgs& p, const TileCount<ROWS, OF>& n, int i, int part, Tile& w) {
    auto uniform = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
    if (i >= n.mine) return false;
    int e = 0, t = n.xcd() * n.per_xcd + i;
    if constexpr (OF == Of::kExpertWeights) {
        e = uniform((int)((uint32_t)i / (uint32_t)n.per_xcd));
        t = ((n.xcd() + e) % kXcd) * n.per_xcd + i - e * n.per_xcd;
        if (t >= n.all) return false;
    }
    const int band = uniform((int)((uint32_t)t / (4u * (uint32_t)p.tiles_n)));
    const int rest = t - band * 4 * p.tiles_n, high = min(4, n.tiles_m - band * 4);
    const int col = uniform((int)((uint32_t)rest / (uint32_t)high)), tm = band * 4 + rest - col * high, tn = col;
    w.a0 = (int64_t)tm * ROWS;
    w.a_end = p.M;
    w.c0 = w.b0 = (int64_t)tn * COLS;
    w.b_end = p.N;
    w.s0 = 0;
    w.s1 = p.stages;
    w.d = static_cast<uint8_t*>(p.d);
    if constexpr (OF == Of::kExpertRows) {
        e = expert_of_tile(n.before, p.experts, tm, threadIdx.x % kWave);
        w.a0 = uniform(p.table[e] + (tm - n.before[e]) * ROWS);
        w.a_end = uniform(p.table[e + 1]);
        w.b0 += (int64_t)e * p.N;
        w.b_end += (int64_t)e * p.N;
    } else if constexpr (OF == Of::kExpertWeights) {
        const int32_t* blocks = p.table + kTable128 * (p.experts + 1);
        w.s0 = uniform(blocks[e]);
        w.s1 = uniform(blocks[e + 1]);
        w.d += (int64_t)e * p.stride * (p.bf16 ? 2 : 4);
    } else {
        w.s0 = part * p.per_split;
        w.s1 = min(w.s0 + p.per_split, p.stages);
        w.d += (int64_t)part * p.M * p.ldd * 4;      // (parts are fp32)
    }
    return true;
}

// Eight neighbouring bfloat16 results, of which `left` are within the row.
__device__ __forceinline__ void put8(uint16_t* z, u32x4 v, int64_t left) {
    if (left >= 8) {
        *reinterpret_cast<u32x4_a2*>(z) = v;
    } else {
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (i < left) z[i] = (uint16_t)(v[i / 2] >> (16 * (i & 1)));
    }
}

}  // namespace

// fp8_large.hip: results in bfloat16 on tiles of 256 x 256; operands and sizes are checked, p.tiles_m and p.tiles_n set
daq_status fp8_large(Of of, ProductArgs p, hipStream_t st);
// fp8_few.hip: whole products or experts' rows in `tiles` row tiles of 64 (experts: at most so many), none of more than most_rows rows; x not NULL: A from X
// [..][K], quantized on the way
daq_status fp8_few(Of of, const ProductArgs& p, int64_t tiles, int64_t most_rows, const void* x, int x_dtype, int64_t ldx, int64_t K, hipStream_t st);

}  // namespace daq
