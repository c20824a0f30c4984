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
    int steps;          // of a row block, a multiple of kGroupSteps
    // Or, for the first operand of bfloat16 products (FLAT), not tiles but the matrix itself, its columns being the rows of the
    // product: row m of the sum's axis is `width` bytes at tiles + m * pitch, for m < depth.  16-byte aligned, pitch included.
    int64_t pitch, width, depth;
};
constexpr int kGroupSteps = 4;
constexpr uint32_t kTileReach = 0xFFFFFF00u;   // bytes that one descriptor reaches: of a row block's tiles, or of a stage's rows

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
    return __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, (int)kTileReach, 0x00020000);
}
// 16 or 4 bytes of every lane to consecutive places of LDS, without registers in between.
__device__ __forceinline__ void tile_to_lds(__amdgpu_buffer_rsrc_t src, uint32_t lane_off, uint32_t off, uint8_t* dst) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(src, (__attribute__((address_space(3))) void*)dst, 16, (int)lane_off, (int)off, 0, 0);
}
__device__ __forceinline__ void words_to_lds(__amdgpu_buffer_rsrc_t src, uint32_t lane_off, uint32_t off, uint8_t* dst) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(src, (__attribute__((address_space(3))) void*)dst, 4, (int)lane_off, (int)off, 0, 0);
}

// Results leave in rows of 128 bytes (64 bfloat16 or 32 fp32 columns) so that whole lines are written: through the wave's share of
// LDS, 16-byte pieces of a row in the order piece ^ row % 8, which keeps both sides off one another's banks.  put(row, column,
// piece): row and column of the wave's tile.  LDS holds RB * 4 KiB for every wave.
template <int RB, int CB, typename Put>
__device__ __forceinline__ void store_tiles(const v16f (&acc)[CB][RB], bool bf16, uint8_t* lds, Put put) {
    static_assert(CB % 2 == 0, "pairs of column blocks");
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

// The results of a workgroup of WR x WC waves, each RB x CB tiles of 32 x 32: rows from row block `rb` of `r` on, columns from row block
// `cb` of `c` on, summed over the stages s0 .. s1 - 1.  A stage, two steps of both operands, is asked for while the three before it are multiplied,
// straight into LDS, and the fragments of a step while the step before is multiplied, the first step of a stage among them:
// the barrier stands before the last step's products, when that step's fragments are in registers already.
// PARTS: the first operand is the sum of so many, whose tiles of a step follow one another, the leading one first; the others' products
// have sums of their own, which stay small, until the end.
template <int WR, int WC, int RB, int CB, bool MX, bool FLAT = false, int PARTS = 1>
struct TileProduct {
    static constexpr int kSteps = 2, kSlots = 4;                   // steps of a stage, stages in LDS
    static constexpr int kWaves = WR * WC;
    static constexpr int kTiles = WR * RB * PARTS + WC * CB;       // of a step
    static constexpr int kScales = MX ? kTiles * 256 : 0;          // bytes of a group's scale words, with the group's first stage
    static constexpr int kStageBytes = kTiles * kSteps * 1024 + kScales;
    static constexpr int kLdsBytes = kSlots * kStageBytes;
    static constexpr int kStrips = WR * RB * PARTS;                // of the first operand: strips of two tiles of a row block
    static constexpr int kShare = kTiles / kWaves;                 // strips that a wave fetches
    // whether stage i begins a group of scale words, and the requests of a wave for it
    static constexpr bool begins(int i) { return MX && i % (kGroupSteps / kSteps) == 0; }
    static constexpr int asks(int i) { return kShare * (kSteps + (begins(i) ? 1 : 0)); }

    // FLAT: a stage of the first operand lies in LDS as its 32 rows, 16-byte pieces of a row in the order piece ^ place(row): the fragment
    // reads, which transpose, take 64 bytes each of eight rows, four of them neighbours and four more eight on.
    static constexpr int kRowBytes = WR * RB * 64, kRowPieces = kRowBytes / 16, kRowsAsked = 1024 / kRowBytes;   // (a request is a KiB)
    static __device__ __forceinline__ int place(int row) { return ((row & 3) * 4 + (row & 8) * 2) & (kRowPieces - 1); }
    static_assert(!FLAT || (!MX && RB == 2 && kStrips % kShare == 0), "two row blocks to a wave, which fetches of one operand only");
    static_assert(kTiles % kWaves == 0, "every wave fetches the same number of strips");
    static_assert(PARTS == 1 || (!MX && !FLAT), "parts are of bfloat16 tiles");

    v16f acc[CB][RB];

    __device__ __forceinline__ void run(const TileOperand& r, const TileOperand& c, int rb, int cb, int s0, int s1, uint8_t* lds) {
        run_on(r, c, rb, cb, s0, s1, lds, lds + kStageBytes, lds + 2 * kStageBytes, lds + 3 * kStageBytes);
    }
    // lds0 ..: the stages' places.  They are arguments so that the compiler knows them apart, and does not let a read of one wait for the
    // requests into the others.
    __device__ __forceinline__ void run_on(const TileOperand& r, const TileOperand& c, int rb, int cb, int s0, int s1, uint8_t* __restrict__ lds0,
                                           uint8_t* __restrict__ lds1, uint8_t* __restrict__ lds2, uint8_t* __restrict__ lds3) {
        const int lane = threadIdx.x % kWave;
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
        const int wr = wave / WC, wc = wave % WC;
        // what this wave fetches: strips wave * kShare .. of the rows' kStrips and the columns' WC * CB
        __amdgpu_buffer_rsrc_t src[kShare], ssrc[kShare];
        bool of_c[kShare];
#pragma unroll
        for (int i = 0; i < kShare; ++i) {
            const int t = wave * kShare + i;
            of_c[i] = t >= kStrips;
            const TileOperand& o = of_c[i] ? c : r;
            const int64_t b = min(of_c[i] ? cb + t - kStrips : rb + t / PARTS, o.blocks - 1);     // (blocks behind the last one are not stored)
            if (!FLAT || of_c[i]) src[i] = bytes_from(o.tiles + (b * o.steps + (of_c[i] ? 0 : t % PARTS * kSteps)) * 1024);
            if constexpr (MX) ssrc[i] = bytes_from(o.scales + b * (o.steps / 4) * 256);
        }
        // FLAT: the rows of a stage that this wave asks for, request by request, and where in them a lane reads
        constexpr int kAskedRows = kShare * kSteps * kRowsAsked;
        uint32_t flat_off[kShare * kSteps];
        if constexpr (FLAT) {
#pragma unroll
            for (int k = 0; k < kShare * kSteps; ++k) {
                const int in = lane / kRowPieces, row = wave * kAskedRows + k * kRowsAsked + in;
                flat_off[k] = (uint32_t)(row * (int)r.pitch) + (uint32_t)((lane % kRowPieces) ^ place(row)) * 16u;
            }
        }
        auto ask = [&](int s, uint8_t* to, bool scales) {
            if (FLAT && !of_c[0]) {
                // rows behind the last one are beyond the descriptor's end and read as zeros
                const int64_t first = (int64_t)s * kSteps * 16 * r.pitch + (int64_t)rb * 64;
                const int64_t bytes = max((r.depth - 1) * r.pitch + r.width - first, (int64_t)0);
                const __amdgpu_buffer_rsrc_t rows = __builtin_amdgcn_make_buffer_rsrc((void*)(r.tiles + first), 0, (int)(uint32_t)min(bytes, (int64_t)kTileReach), 0x00020000);
#pragma unroll
                for (int k = 0; k < kShare * kSteps; ++k) tile_to_lds(rows, flat_off[k], 0, to + (wave * kShare * kSteps + k) * 1024);
                return;
            }
#pragma unroll
            for (int i = 0; i < kShare; ++i) {
                const uint32_t first = (uint32_t)s * (kSteps * 1024u) * (of_c[i] ? 1u : (uint32_t)PARTS);
                uint8_t* at = to + (wave * kShare + i) * kSteps * 1024;
#pragma unroll
                for (int k = 0; k < kSteps; ++k) tile_to_lds(src[i], lane * 16, first + k * 1024u, at + k * 1024);
                if (MX && scales) words_to_lds(ssrc[i], lane * 4, (uint32_t)s / (kGroupSteps / kSteps) * 256u, to + kTiles * kSteps * 1024 + (wave * kShare + i) * 256);
            }
        };
        v4i fr[2][PARTS][RB], fc[2][CB];
        int sr[2][RB], sc[2][CB];
        const int at_r = wr * RB * PARTS * kSteps * 1024 + lane * 16, at_c = (kStrips + wc * CB) * kSteps * 1024 + lane * 16;
        const int at_sr = kTiles * kSteps * 1024 + wr * RB * 256 + lane * 4, at_sc = kTiles * kSteps * 1024 + (WR * RB + wc * CB) * 256 + lane * 4;
        // FLAT: lane l takes column l % 16 of the 16 of its quarter wave and four rows at a time; the quarters are 16 columns and 8 rows apart
        int at_flat[RB];
        if constexpr (FLAT) {
            const int row = (lane / 32) * 8 + (lane % 16) / 4;
#pragma unroll
            for (int i = 0; i < RB; ++i) {
                const int piece = (wr * RB + i) * 4 + (lane / 16 & 1) * 2 + (lane & 3) / 2;
                at_flat[i] = row * kRowBytes + (piece ^ place(row)) * 16 + (lane & 1) * 8;
            }
        }
        // FLAT: the transposing reads are written out, with their wait, as the compiler would have each wait for the requests under way.  Waves
        // of 64 rows x 128 columns make few of them; 16384 x 8192 x 4096 takes as long with waves of 128 x 64, within what two runs differ by.
        auto read_flat = [&](const uint8_t* from, auto step, int set) {
            if constexpr (FLAT) {
                typedef short v4s __attribute__((ext_vector_type(4)));
                constexpr int kAt = decltype(step)::value * 16 * kRowBytes;
                const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const uint8_t*)from;
                v4s part[2 * RB];
                uint32_t at[RB];
#pragma unroll
                for (int i = 0; i < RB; ++i) at[i] = base + (uint32_t)at_flat[i];
                asm volatile(
                    "ds_read_b64_tr_b16 %0, %4 offset:%6\n\tds_read_b64_tr_b16 %1, %4 offset:%7\n\t"
                    "ds_read_b64_tr_b16 %2, %5 offset:%6\n\tds_read_b64_tr_b16 %3, %5 offset:%7\n\t"
                    "s_waitcnt lgkmcnt(0)"
                    : "=&v"(part[0]), "=&v"(part[1]), "=&v"(part[2]), "=&v"(part[3])
                    : "v"(at[0]), "v"(at[1]), "n"(kAt), "n"(kAt + 4 * kRowBytes)
                    : "memory");
#pragma unroll
                for (int i = 0; i < RB; ++i) fr[set][0][i] = __builtin_bit_cast(v4i, __builtin_shufflevector(part[2 * i], part[2 * i + 1], 0, 1, 2, 3, 4, 5, 6, 7));
            }
        };
        auto read = [&](const uint8_t* from, int k, int set, bool scales, int sset) {
#pragma unroll
            for (int i = 0; i < CB; ++i) fc[set][i] = *reinterpret_cast<const v4i*>(from + at_c + (i * kSteps + k) * 1024);
            if constexpr (!FLAT) {
#pragma unroll
                for (int i = 0; i < RB; ++i)
#pragma unroll
                    for (int q = 0; q < PARTS; ++q)
                        fr[set][q][i] = *reinterpret_cast<const v4i*>(from + at_r + ((i * kSteps + k) * PARTS + q) * 1024);
            }
            if constexpr (MX) {
                if (scales) {
#pragma unroll
                    for (int i = 0; i < RB; ++i) sr[sset][i] = *reinterpret_cast<const int*>(from + at_sr + i * 256);
#pragma unroll
                    for (int i = 0; i < CB; ++i) sc[sset][i] = *reinterpret_cast<const int*>(from + at_sc + i * 256);
                }
            }
        };
        v16f small[PARTS > 1 ? CB : 1][PARTS > 1 ? RB : 1];
        auto multiply = [&](auto step, int set, int sset) {
#pragma unroll
            for (int j = 0; j < CB; ++j)
#pragma unroll
                for (int i = 0; i < RB; ++i) {
                    if constexpr (MX) acc[j][i] = mfma4<decltype(step)::value>(fc[set][j], fr[set][0][i], acc[j][i], sc[sset][j], sr[sset][i]);
                    else acc[j][i] = mfma16(fc[set][j], fr[set][0][i], acc[j][i]);
                    if constexpr (PARTS > 1) {
#pragma unroll
                        for (int q = PARTS - 1; q > 0; --q) small[j][i] = mfma16(fc[set][j], fr[set][q][i], small[j][i]);
                    }
                }
        };
#pragma unroll
        for (int j = 0; j < CB; ++j)
#pragma unroll
            for (int i = 0; i < RB; ++i) {
                acc[j][i] = v16f{};
                if constexpr (PARTS > 1) small[j][i] = v16f{};
            }
        if (s0 >= s1) return;
        const int last = s1 - 1;
        ask(s0, lds0, true);
        ask(min(s0 + 1, last), lds1, begins(1));
        ask(min(s0 + 2, last), lds2, begins(2));
        ask(min(s0 + 3, last), lds3, begins(3));
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(asks(1) + asks(2) + asks(3)) : "memory");
        __builtin_amdgcn_s_barrier();
        read(lds0, 0, 0, true, 0);
        read_flat(lds0, std::integral_constant<int, 0>{}, 0);
        // The reads of a step stand between the products of the step before, one each, from its beginning on: left to itself the compiler
        // moves them behind the last one, where every wave then waits for them.  (FLAT: the written ones do follow the products, and the
        // wave that shares the SIMD multiplies meanwhile.)
        auto then = [&](const uint8_t* from, auto step, int set) {
            if constexpr (FLAT) {
                __builtin_amdgcn_sched_barrier(0);
                read_flat(from, step, set);
            } else {
#pragma unroll
                for (int i = 0; i < RB * CB * PARTS; ++i) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);   // a matrix instruction
                    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);   // an LDS read
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        };
        // as many stages a round as there are places, so that these, the register sets and the bytes of a scale word have numbers known here
        auto stage = [&](int s, uint8_t* here, uint8_t* next, auto index) {
            constexpr int kIndex = decltype(index)::value, kPer = kGroupSteps / kSteps, kScaleSet = kIndex / kPer & 1, kFirst = kIndex % kPer * kSteps;
            read(here, 1, 1, false, 0);
            multiply(std::integral_constant<int, kFirst>{}, 0, kScaleSet);
            then(here, std::integral_constant<int, 1>{}, 1);
            // the next stage has landed, this one is read out
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(asks(kIndex + 2) + asks(kIndex + 3)) : "memory");
            __builtin_amdgcn_s_barrier();
            read(next, 0, 0, begins(kIndex + 1), (kIndex + 1) / kPer & 1);
            ask(min(s + kSlots, last), here, begins(kIndex));
            multiply(std::integral_constant<int, kFirst + kSteps - 1>{}, 1, kScaleSet);
            then(next, std::integral_constant<int, 0>{}, 0);
        };
        int s = s0;
        for (; s + 3 < s1; s += 4) {
            stage(s, lds0, lds1, std::integral_constant<int, 0>{});
            stage(s + 1, lds1, lds2, std::integral_constant<int, 1>{});
            stage(s + 2, lds2, lds3, std::integral_constant<int, 2>{});
            stage(s + 3, lds3, lds0, std::integral_constant<int, 3>{});
        }
        if (s < s1) stage(s, lds0, lds1, std::integral_constant<int, 0>{});
        if (s + 1 < s1) stage(s + 1, lds1, lds2, std::integral_constant<int, 1>{});
        if (s + 2 < s1) stage(s + 2, lds2, lds3, std::integral_constant<int, 2>{});
        if constexpr (PARTS > 1) {
#pragma unroll
            for (int j = 0; j < CB; ++j)
#pragma unroll
                for (int i = 0; i < RB; ++i) acc[j][i] += small[j][i];
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // the requests past the end have landed before LDS is put to other use
    }

    static_assert(kLdsBytes / kWaves >= RB * 32 * 128, "a wave's share holds its rows");
    template <typename Put>
    __device__ __forceinline__ void store(bool bf16, uint8_t* lds, Put put) const {
        store_tiles<RB, CB>(acc, bf16, lds, put);
    }
};

}  // namespace

}  // namespace daq
