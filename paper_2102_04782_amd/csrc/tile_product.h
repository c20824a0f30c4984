// Products of operands that lie in the register order of the matrix cores: tiles of 32 rows x one instruction's depth, 16 bytes a
// lane, a contiguous KiB each; microscaled 4-bit tiles of 64 columns or bfloat16 tiles of 16.  Both take the 32 x 32 instruction
// the same 32 cycles, so one skeleton serves both.
#pragma once

#include <type_traits>

#include "lowbits.h"

namespace daq {

// One operand: tile (row block, step) is the KiB at tiles + (row block * steps + step) * 1024.  4-bit: the scale words of the four
// steps of a group are the 256 bytes at scales + (row block * groups + group) * 256, groups = steps / 4.
struct TileOperand {
    const uint8_t* tiles;
    const uint8_t* scales;
    int blocks;         // row blocks
    int steps;          // of a row block, a multiple of kStageSteps
};
constexpr int kStageSteps = 4;

namespace {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));

// cbsz / blgp 4 say 4-bit elements; S picks the byte of the scale words.
template <int S>
__device__ __forceinline__ v16f mfma4(v4i x, v4i y, v16f c, int sx, int sy) {
    const v8i a = {x[0], x[1], x[2], x[3], 0, 0, 0, 0}, b = {y[0], y[1], y[2], y[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 4, 4, S, sx, S, sy);
}
__device__ __forceinline__ v16f mfma16(v4i x, v4i y, v16f c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, x), __builtin_bit_cast(v8bf, y), c, 0, 0, 0);
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t bytes_from(const uint8_t* base) {
    return __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, (int)0xFFFFFF00u, 0x00020000);
}
// 16 or 4 bytes of every lane to consecutive places of LDS, without registers in between.
__device__ __forceinline__ void tile_to_lds(__amdgpu_buffer_rsrc_t src, uint32_t lane_off, uint32_t off, uint8_t* dst) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(src, (__attribute__((address_space(3))) void*)dst, 16, (int)lane_off, (int)off, 0, 0);
}
__device__ __forceinline__ void words_to_lds(__amdgpu_buffer_rsrc_t src, uint32_t lane_off, uint32_t off, uint8_t* dst) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(src, (__attribute__((address_space(3))) void*)dst, 4, (int)lane_off, (int)off, 0, 0);
}

// The results of a workgroup of WR x WC waves, each RB x CB tiles of 32 x 32: rows from row block `rb` of `r` on, columns from row block
// `cb` of `c` on, summed over the stages s0 .. s1 - 1.  A stage of both operands is asked for while the SLOTS - 1 before it are multiplied,
// straight into LDS, and the fragments of a step while the step before is multiplied, the first step of a stage among them:
// the barrier stands before the last step's products, when that step's fragments are in registers already.
// c_wrap: stages after which the second operand begins again.
template <int WR, int WC, int RB, int CB, bool MX, int SLOTS = 2>
struct TileProduct {
    static constexpr int kWaves = WR * WC;
    static constexpr int kTiles = WR * RB + WC * CB;               // of a step
    static constexpr int kScales = MX ? kTiles * 256 : 0;          // bytes of a stage
    static constexpr int kStageBytes = kTiles * kStageSteps * 1024 + kScales;
    static constexpr int kLdsBytes = SLOTS * kStageBytes;
    static constexpr int kShare = kTiles / kWaves;                    // operand row blocks that a wave fetches
    static constexpr int kAsks = kShare * (kStageSteps + (MX ? 1 : 0));   // requests of a wave for a stage

    static_assert(SLOTS == 2 || SLOTS == 4, "two or four stages in LDS");
    static_assert(kTiles % kWaves == 0, "every wave fetches the same number of row blocks");

    v16f acc[CB][RB];

    __device__ __forceinline__ void run(const TileOperand& r, const TileOperand& c, int rb, int cb, int s0, int s1, int c_wrap, uint8_t* lds) {
        run_on(r, c, rb, cb, s0, s1, c_wrap, lds, lds + kStageBytes, lds + (SLOTS - 2) * kStageBytes, lds + (SLOTS - 1) * kStageBytes);
    }
    // lds0 ..: the stages' places (the last two are not used where there are two).  They are arguments so that the compiler knows them
    // apart, and does not let a read of one wait for the requests into the others.
    __device__ __forceinline__ void run_on(const TileOperand& r, const TileOperand& c, int rb, int cb, int s0, int s1, int c_wrap,
                                           uint8_t* __restrict__ lds0, uint8_t* __restrict__ lds1, uint8_t* __restrict__ lds2, uint8_t* __restrict__ lds3) {
        const int lane = threadIdx.x % kWave;
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
        const int wr = wave / WC, wc = wave % WC;
        // what this wave fetches: row blocks wave * kShare .. of the rows' WR * RB and the columns' WC * CB
        __amdgpu_buffer_rsrc_t src[kShare], ssrc[kShare];
        bool of_c[kShare];
#pragma unroll
        for (int i = 0; i < kShare; ++i) {
            const int t = wave * kShare + i;
            of_c[i] = t >= WR * RB;
            const TileOperand& o = of_c[i] ? c : r;
            const int64_t b = min(of_c[i] ? cb + t - WR * RB : rb + t, o.blocks - 1);     // (blocks behind the last one are not stored)
            src[i] = bytes_from(o.tiles + b * o.steps * 1024);
            if constexpr (MX) ssrc[i] = bytes_from(o.scales + b * (o.steps / 4) * 256);
        }
        auto ask = [&](int s, uint8_t* to) {
#pragma unroll
            for (int i = 0; i < kShare; ++i) {
                const int st = of_c[i] ? (s >= 2 * c_wrap ? s - 2 * c_wrap : s >= c_wrap ? s - c_wrap : s) : s;
                uint8_t* at = to + (wave * kShare + i) * kStageSteps * 1024;
#pragma unroll
                for (int k = 0; k < kStageSteps; ++k) tile_to_lds(src[i], lane * 16, (uint32_t)(st * kStageSteps + k) * 1024u, at + k * 1024);
                if constexpr (MX) words_to_lds(ssrc[i], lane * 4, (uint32_t)st * 256u, to + kTiles * kStageSteps * 1024 + (wave * kShare + i) * 256);
            }
        };
        v4i fr[2][RB], fc[2][CB];
        int sr[2][RB], sc[2][CB];
        const int at_r = wr * RB * kStageSteps * 1024 + lane * 16, at_c = (WR * RB + wc * CB) * kStageSteps * 1024 + lane * 16;
        const int at_sr = kTiles * kStageSteps * 1024 + wr * RB * 256 + lane * 4, at_sc = kTiles * kStageSteps * 1024 + (WR * RB + wc * CB) * 256 + lane * 4;
        auto read = [&](const uint8_t* from, int k, int set, int sset) {
#pragma unroll
            for (int i = 0; i < CB; ++i) fc[set][i] = *reinterpret_cast<const v4i*>(from + at_c + (i * kStageSteps + k) * 1024);
#pragma unroll
            for (int i = 0; i < RB; ++i) fr[set][i] = *reinterpret_cast<const v4i*>(from + at_r + (i * kStageSteps + k) * 1024);
            if constexpr (MX) {
                if (k == 0) {
#pragma unroll
                    for (int i = 0; i < RB; ++i) sr[sset][i] = *reinterpret_cast<const int*>(from + at_sr + i * 256);
#pragma unroll
                    for (int i = 0; i < CB; ++i) sc[sset][i] = *reinterpret_cast<const int*>(from + at_sc + i * 256);
                }
            }
        };
        auto multiply = [&](auto step, int set, int sset) {
#pragma unroll
            for (int j = 0; j < CB; ++j)
#pragma unroll
                for (int i = 0; i < RB; ++i) {
                    if constexpr (MX) acc[j][i] = mfma4<decltype(step)::value>(fc[set][j], fr[set][i], acc[j][i], sc[sset][j], sr[sset][i]);
                    else acc[j][i] = mfma16(fc[set][j], fr[set][i], acc[j][i]);
                }
        };
#pragma unroll
        for (int j = 0; j < CB; ++j)
#pragma unroll
            for (int i = 0; i < RB; ++i) acc[j][i] = v16f{};
        if (s0 >= s1) return;
        const int last = s1 - 1;
        ask(s0, lds0);
        ask(min(s0 + 1, last), lds1);
        if constexpr (SLOTS == 4) {
            ask(min(s0 + 2, last), lds2);
            ask(min(s0 + 3, last), lds3);
        }
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"((SLOTS - 1) * kAsks) : "memory");
        __builtin_amdgcn_s_barrier();
        read(lds0, 0, 0, 0);
        // The reads of a step stand between the products of the step before, one each, from its beginning on: left to itself the compiler
        // moves them behind the last one, where every wave then waits for them.
        auto interleave = [&] {
#pragma unroll
            for (int i = 0; i < RB + CB; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);   // a matrix instruction
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);   // an LDS read
            }
            __builtin_amdgcn_sched_group_barrier(0x008, RB * CB, 0);
            __builtin_amdgcn_sched_barrier(0);
        };
        // as many stages a round as there are places, so that these and the register sets have numbers known here
        auto stage = [&](int s, uint8_t* here, uint8_t* next, int sset) {
            read(here, 1, 1, sset);
            multiply(std::integral_constant<int, 0>{}, 0, sset);
            interleave();
            read(here, 2, 0, sset);
            multiply(std::integral_constant<int, 1>{}, 1, sset);
            interleave();
            read(here, 3, 1, sset);
            multiply(std::integral_constant<int, 2>{}, 0, sset);
            interleave();
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((SLOTS - 2) * kAsks) : "memory");   // the next stage has landed, this one is read out
            __builtin_amdgcn_s_barrier();
            read(next, 0, 0, sset ^ 1);
            ask(min(s + SLOTS, last), here);
            multiply(std::integral_constant<int, 3>{}, 1, sset);
            interleave();
        };
        int s = s0;
        if constexpr (SLOTS == 2) {
            for (; s + 1 < s1; s += 2) {
                stage(s, lds0, lds1, 0);
                stage(s + 1, lds1, lds0, 1);
            }
            if (s < s1) stage(s, lds0, lds1, 0);
        } else {
            for (; s + 3 < s1; s += 4) {
                stage(s, lds0, lds1, 0);
                stage(s + 1, lds1, lds2, 1);
                stage(s + 2, lds2, lds3, 0);
                stage(s + 3, lds3, lds0, 1);
            }
            if (s < s1) stage(s, lds0, lds1, 0);
            if (s + 1 < s1) stage(s + 1, lds1, lds2, 1);
            if (s + 2 < s1) stage(s + 2, lds2, lds3, 0);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // the requests past the end have landed before LDS is put to other use
    }

    // Results leave in rows of 128 bytes (64 bfloat16 or 32 fp32 columns) so that whole lines are written: through the wave's share of
    // LDS, 16-byte pieces of a row in the order piece ^ row % 8, which keeps both sides off one another's banks.  put(row, column,
    // piece): row and column of the wave's tile.
    static_assert(kLdsBytes / kWaves >= RB * 32 * 128 && (CB % 2 == 0), "a wave's share holds its rows");
    template <typename Put>
    __device__ __forceinline__ void store(bool bf16, uint8_t* lds, Put put) const {
        const int lane = threadIdx.x % kWave;
        uint8_t* mine = lds + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave) * (RB * 32 * 128);
        __builtin_amdgcn_s_barrier();   // everybody has read the last stage
        auto out = [&](int col0, int per) {
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int k = 0; k < RB * 4; ++k) {
                const int row = k * 8 + lane / 8;
                const u32x4 v = *reinterpret_cast<const u32x4*>(mine + row * 128 + ((lane ^ row) & 7) * 16);
                put(row, col0 + (lane & 7) * per, v);
            }
            __builtin_amdgcn_wave_barrier();
        };
        const int m = lane % 32, h = lane / 32;
        if (bf16) {
#pragma unroll
            for (int j0 = 0; j0 < CB; j0 += 2) {
#pragma unroll
                for (int i = 0; i < RB; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j)
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const v16f& a = acc[j0 + j][i];
                            *reinterpret_cast<u32x2*>(mine + (i * 32 + m) * 128 + (((j * 4 + q) ^ m) & 7) * 16 + h * 8) =
                                u32x2{pack_bf16(a[4 * q], a[4 * q + 1]), pack_bf16(a[4 * q + 2], a[4 * q + 3])};
                        }
                out(j0 * 32, 8);
            }
        } else {
#pragma unroll
            for (int j = 0; j < CB; ++j) {
#pragma unroll
                for (int i = 0; i < RB; ++i)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const v16f& a = acc[j][i];
                        *reinterpret_cast<f32x4*>(mine + (i * 32 + m) * 128 + (((q * 2 + h) ^ m) & 7) * 16) = f32x4{a[4 * q], a[4 * q + 1], a[4 * q + 2], a[4 * q + 3]};
                    }
                out(j * 32, 4);
            }
        }
    }
};

}  // namespace

}  // namespace daq
