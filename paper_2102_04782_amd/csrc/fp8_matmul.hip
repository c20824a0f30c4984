// Products of 8-bit floating point matrices with a scale for every 128 elements, D[m][n] = sum over k of A[m][k] * B[n][k], whole ones and those of
// experts, whose rows, or whose share of the summed axis, a plan on the device tells.
//
// Results in bfloat16 take the 8-bit matrix instructions.  These add eight neighbouring products with what lies below 2^-13 of the largest cut off (measured), some
// 2^-16 of a result's magnitude: nothing beside bfloat16's rounding, but 200 times an fp32 sum's error.  Results in fp32 (EXACT) therefore
// decode to bfloat16, which holds code times scale exactly, and take those instructions at half the rate.
//
// The matrix instructions take codes and scale bytes as they are: 32 x 32 x 64 (tiles) or 16 x 16 x 128 (few rows), 32 bytes a lane of each operand
// and one scale for 32 of the summed axis.  As a block is 128 long and both operands are cut alike, which of a block's elements a
// lane holds does not matter, as long as it is the same of both.  B goes in as the first operand, so that a lane holds
// neighbouring columns of a row of D.
#include <cmath>

#include "fp8_product.h"

namespace daq {

namespace {

// Form of a product: edge of a workgroup's tile, and parts of the summed axis.
enum class Fp8Form { kFew, k64, k128, k256 };
struct Fp8Plan {
    Fp8Form form;
    int splits, per_split;   // stages of 128 of a part
};

Fp8Operand operand(const uint8_t* buf, int64_t rows, int64_t cols) {
    daq_fp8_layout L;
    daq_layout_fp8(rows, cols, &L);
    return {buf, buf + L.off_scales, rows, L.pitch};
}

// The results of a workgroup of WR x WC waves, each RB x CB tiles of 32 x 32, summed over the stages s0 .. s1 - 1 of 128.  A stage of both operands,
// 128 bytes of every row, goes straight to LDS, where the 16-byte piece j of a row lies at j ^ (row / 2 % 8): eight lanes ask for a row's line in
// that order, and the fragment reads of sixteen rows share no bank.  SLOTS stages are under way or being read.  Fragments are read a step
// (64 of a stage's 128) ahead into the registers that the products have just done with; the barrier stands between a stage's two steps, when this
// stage is read out and the next has landed.
template <int WR, int WC, int RB, int CB, int SLOTS, bool EXACT>
struct Fp8Product {
    static constexpr int kWaves = WR * WC, kRows = WR * RB * 32, kCols = WC * CB * 32;
    static constexpr int kCodes = (kRows + kCols) * 128, kStage = kCodes + (kRows + kCols) * 4;   // bytes of a stage, its scale words behind the codes
    static constexpr int kLdsBytes = SLOTS * kStage;
    static constexpr int kUnits = (kRows + kCols) / 64 / kWaves;   // of 64 rows, that a wave asks for
    static constexpr int kAsks = 9 * kUnits;              // requests of a wave for a stage: eight rows at a time, and the scale words of a unit
    static_assert((kRows + kCols) % (kWaves * 64) == 0 && kRows % (64 * kUnits) == 0, "a wave asks for rows of one operand");
    static_assert(SLOTS == 2 || SLOTS == 4, "the loop is written out for these");
    static_assert(kLdsBytes / kWaves >= RB * 32 * 128, "a wave's share holds its rows of results");

    v16f acc[CB][RB];

    // Rows a0 .. of A (a_end: the first that is not the tile's; rows behind it repeat the last) and b0 .. of B; `order`: of A's rows.
    __device__ __forceinline__ void run(const Fp8Operand& a, const Fp8Operand& b, int64_t a0, int64_t a_end, int64_t b0, int64_t b_end,
                                        const int32_t* order, int picks, int s0, int s1, uint8_t* lds) {
        run_on(a, b, a0, a_end, b0, b_end, order, picks, s0, s1, lds, lds + kStage, lds + 2 % SLOTS * kStage, lds + 3 % SLOTS * kStage);
    }
    // lds0 ..: the stages' places, as arguments so that the compiler knows them apart, and does not let a read of one wait for the requests
    // into the others.
    __device__ __forceinline__ void run_on(const Fp8Operand& a, const Fp8Operand& b, int64_t a0, int64_t a_end, int64_t b0, int64_t b_end,
                                           const int32_t* order, int picks, int s0, int s1, uint8_t* __restrict__ lds0, uint8_t* __restrict__ lds1,
                                           uint8_t* __restrict__ lds2, uint8_t* __restrict__ lds3) {
        const int lane = threadIdx.x % kWave;
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
        const int wr = wave / WC, wc = wave % WC;
        // what this wave asks for
        const bool of_b = wave >= kRows / 64 / kUnits;
        const Fp8Operand& o = of_b ? b : a;
        const bool gather = !of_b && order != nullptr;
        const int64_t first = of_b ? b0 + wave * kUnits * 64 - kRows : a0 + wave * kUnits * 64, end = of_b ? b_end : a_end;
        const int64_t base = gather ? 0 : min(first, end - 1);
        uint32_t off[8 * kUnits], soff[kUnits];
        auto row_of = [&](int i) {
            const int64_t r = min(first + i, end - 1);
            return (uint32_t)(gather ? (picks ? order[r] / picks : (int)r) : r - base);
        };
#pragma unroll
        for (int i = 0; i < 8 * kUnits; ++i) off[i] = row_of(i * 8 + lane / 8) * (uint32_t)o.pitch + (uint32_t)((lane % 8) ^ ((i * 4 + lane / 16) & 7)) * 16u;
#pragma unroll
        for (int u = 0; u < kUnits; ++u) soff[u] = row_of(u * 64 + lane) * 4u;
        // (a stage behind the last one is asked for through descriptors without an extent: LDS receives zeros)
        auto codes_of = [&](int s) { return bytes_of(o.codes + base * o.pitch, s < s1 ? (o.rows - base) * o.pitch : 0); };
        auto words_of = [&](int s) { return bytes_of(o.scales + ((int64_t)(s / 4) * o.rows + base) * 4, s < s1 ? (o.rows - base) * 4 : 0); };
        // request n of a stage: eight rows, or the words of a unit
        auto request = [&](int n, int s, __amdgpu_buffer_rsrc_t codes, __amdgpu_buffer_rsrc_t words, uint8_t* to) {
            if (n < 8 * kUnits) tile_to_lds(codes, off[n], (uint32_t)s * 128u, to + (wave * 8 * kUnits + n) * 1024);
            else words_to_lds(words, soff[n - 8 * kUnits], 0, to + kCodes + (wave * kUnits + n - 8 * kUnits) * 256);
        };
        auto ask = [&](int s, uint8_t* to) {
            const __amdgpu_buffer_rsrc_t codes = codes_of(s), words = words_of(s);
#pragma unroll
            for (int n = 0; n < kAsks; ++n) request(n, s, codes, words, to);
        };
        v8i fr[2][RB], fc[2][CB];
        int sr[RB], sc[CB];
        int at[2][2];     // of a lane in 32 rows: step and half of its 32 bytes
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int t = 0; t < 2; ++t) at[k][t] = (lane % 32) * 128 + ((k * 4 + lane / 32 * 2 + t) ^ (lane / 2 & 7)) * 16;
        auto fragment = [&](const uint8_t* from, int block, int k) {
            const v4i lo = *reinterpret_cast<const v4i*>(from + block * 4096 + at[k][0]), hi = *reinterpret_cast<const v4i*>(from + block * 4096 + at[k][1]);
            return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        };
        const int block_r = wr * RB, block_c = WR * RB + wc * CB;
        auto read = [&](const uint8_t* from, int k) {
#pragma unroll
            for (int j = 0; j < CB; ++j) fc[k][j] = fragment(from, block_c + j, k);
#pragma unroll
            for (int i = 0; i < RB; ++i) fr[k][i] = fragment(from, block_r + i, k);
        };
        int wr_next[RB], wc_next[CB];
        auto read_words = [&](const uint8_t* from) {
#pragma unroll
            for (int i = 0; i < RB; ++i) wr_next[i] = *reinterpret_cast<const int*>(from + kCodes + (block_r + i) * 128 + (lane % 32) * 4);
#pragma unroll
            for (int j = 0; j < CB; ++j) wc_next[j] = *reinterpret_cast<const int*>(from + kCodes + (block_c + j) * 128 + (lane % 32) * 4);
        };
        auto take_words = [&](int s) {      // the byte of stage s; EXACT: the scale itself
            auto of = [&](int w) { return EXACT ? __float_as_int(scale_of((uint32_t)w >> (s % 4 * 8) & 255u)) : w >> (s % 4 * 8); };
#pragma unroll
            for (int i = 0; i < RB; ++i) sr[i] = of(wr_next[i]);
#pragma unroll
            for (int j = 0; j < CB; ++j) sc[j] = of(wc_next[j]);
        };
        auto multiply = [&](int k) {
            if constexpr (EXACT) {             // in bfloat16, eight of a lane's 32 elements at a time
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    v4i x[CB];
#pragma unroll
                    for (int j = 0; j < CB; ++j) x[j] = in_bf16(fc[k][j][2 * q], fc[k][j][2 * q + 1], __int_as_float(sc[j]));
#pragma unroll
                    for (int i = 0; i < RB; ++i) {
                        const v4i y = in_bf16(fr[k][i][2 * q], fr[k][i][2 * q + 1], __int_as_float(sr[i]));
#pragma unroll
                        for (int j = 0; j < CB; ++j) acc[j][i] = mfma16(x[j], y, acc[j][i]);
                    }
                }
            } else {
#pragma unroll
                for (int i = 0; i < RB; ++i)
#pragma unroll
                    for (int j = 0; j < CB; ++j) acc[j][i] = mfma8(fc[k][j], fr[k][i], acc[j][i], sc[j], sr[i]);
            }
        };
#pragma unroll
        for (int j = 0; j < CB; ++j)
#pragma unroll
            for (int i = 0; i < RB; ++i) acc[j][i] = v16f{};
        if (s0 >= s1) return;
        ask(s0, lds0);
        ask(s0 + 1, lds1);
        if constexpr (SLOTS == 4) {
            ask(s0 + 2, lds2);
            ask(s0 + 3, lds3);
        }
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"((SLOTS - 1) * kAsks) : "memory");
        __builtin_amdgcn_s_barrier();
        read_words(lds0);
        read(lds0, 0);
        take_words(s0);
        // Reads and requests stand between the products, one each: left to itself the compiler moves them together, and they are waited for.
        auto between = [&](auto reads, auto requests) {
            if constexpr (!EXACT) {
#pragma unroll
                for (int i = 0; i < RB * CB; ++i) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);                          // a matrix instruction
                    __builtin_amdgcn_sched_group_barrier(0x100, decltype(reads)::value, 0);     // LDS reads
                    if constexpr (decltype(requests)::value > 0) __builtin_amdgcn_sched_group_barrier(0x020, decltype(requests)::value, 0);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        };
        constexpr int kReads = (2 * (RB + CB) + RB * CB - 1) / (RB * CB), kReadsAll = (3 * (RB + CB) + RB * CB - 1) / (RB * CB);
        auto stage = [&](int s, uint8_t* here, uint8_t* next) {
            read(here, 1);
            multiply(0);
            between(std::integral_constant<int, kReads>{}, std::integral_constant<int, 0>{});
            // the next stage has landed, this one is read out
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((SLOTS - 2) * kAsks) : "memory");
            __builtin_amdgcn_s_barrier();
            read(next, 0);
            read_words(next);
            ask(s + SLOTS, here);
            multiply(1);
            between(std::integral_constant<int, kReadsAll>{}, std::integral_constant<int, (kAsks + RB * CB - 1) / (RB * CB)>{});
            take_words(s + 1);
        };
        int s = s0;
        if constexpr (SLOTS == 4) {
            for (; s + 3 < s1; s += 4) {
                stage(s, lds0, lds1);
                stage(s + 1, lds1, lds2);
                stage(s + 2, lds2, lds3);
                stage(s + 3, lds3, lds0);
            }
            if (s < s1) stage(s, lds0, lds1);
            if (s + 1 < s1) stage(s + 1, lds1, lds2);
            if (s + 2 < s1) stage(s + 2, lds2, lds3);
        } else {
            for (; s + 1 < s1; s += 2) {
                stage(s, lds0, lds1);
                stage(s + 1, lds1, lds0);
            }
            if (s < s1) stage(s, lds0, lds1);
        }
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");   // the requests past the end have landed before LDS is put to other use
    }
};

// Tiles of kRows x kCols results, a workgroup each.  Workgroup b runs on XCD b % 8; an XCD takes an eighth of the tiles, in bands of four row
// tiles, whose panels its L2 holds.  Bound: too few tiles for the CUs (1111 x 1500 x 2030, fp32: 432 of 64 x 64, 19.1 us, where the bytes take 2 and the
// matrix cores 4), and LDS reads: a wave of a tile of 128 makes 32 products of a byte, of 64 21, of 256 64 (2048 x 4096 x 4096, bfloat16, 32.8 us, 2.1 PFLOP/s).
template <int WR, int WC, int RB, int CB, int SLOTS, bool EXACT, Of OF>
__global__ __launch_bounds__(64 * WR * WC, 1) void k_fp8_product(ProductArgs p) {
    using Product = Fp8Product<WR, WC, RB, CB, SLOTS, EXACT>;
    extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
    const TileCount<Product::kRows, OF> count(p);
    Tile tile;
    if (!tile_at<Product::kRows, Product::kCols, OF>(p, count, (int)(blockIdx.x / kXcd), blockIdx.y, tile)) return;
    if (OF == Of::kExpertWeights && tile.s0 == tile.s1 && p.accumulate) return;
    Product prod;
    prod.run(p.a, p.b, tile.a0, tile.a_end, tile.b0, tile.b_end, OF == Of::kExpertRows && p.picks ? p.order : nullptr, p.picks, tile.s0, tile.s1, lds);
    const int wave = threadIdx.x / kWave;
    const int64_t m0 = tile.a0 + wave / WC * RB * 32, c0 = tile.c0 + wave % WC * CB * 32;
    if (p.bf16) {
        store_tiles<RB, CB>(prod.acc, true, lds, [&](int row, int col, u32x4 v) {
            const int64_t m = m0 + row, n = c0 + col;
            if (m >= tile.a_end || n >= p.N) return;
            put8(reinterpret_cast<uint16_t*>(tile.d) + m * p.ldd + n, v, p.N - n);
        });
    } else {
        store_tiles<RB, CB>(prod.acc, false, lds, [&](int row, int col, u32x4 v) {
            const int64_t m = m0 + row, n = c0 + col;
            if (m >= tile.a_end || n >= p.N) return;
            float* z = reinterpret_cast<float*>(tile.d) + m * p.ldd + n;
            if (n + 4 <= p.N) {
                u32x4_a4* q = reinterpret_cast<u32x4_a4*>(z);
                if (p.accumulate) *q = __builtin_bit_cast(u32x4, __builtin_bit_cast(f32x4, (u32x4)*q) + __builtin_bit_cast(f32x4, v));
                else *q = v;
            } else {
#pragma unroll
                for (int i = 0; i < 3; ++i)
                    if (n + i < p.N) z[i] = p.accumulate ? z[i] + bits_as<float>(v[i]) : bits_as<float>(v[i]);
            }
        });
    }
}

// The parts of a product that was split along the summed axis, added in their order.
__global__ __launch_bounds__(256) void k_fp8_sum(const float* parts, int splits, int64_t M, int64_t N, void* d, int64_t ldd, int bf16, int accumulate) {
    const int64_t pieces = (N + 3) / 4, i = (int64_t)blockIdx.x * 256 + threadIdx.x, m = i / pieces, n = (i - m * pieces) * 4;
    if (m >= M) return;
    const int64_t pitch = pieces * 4;
    f32x4 v = {0, 0, 0, 0};
    for (int z = 0; z < splits; ++z) v += *reinterpret_cast<const f32x4*>(parts + (z * M + m) * pitch + n);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (n + j >= N) break;
        if (bf16) static_cast<uint16_t*>(d)[m * ldd + n + j] = (uint16_t)(pack_bf16(v[j], 0.f) & 0xFFFFu);
        else static_cast<float*>(d)[m * ldd + n + j] = accumulate ? static_cast<float*>(d)[m * ldd + n + j] + v[j] : v[j];
    }
}

int form_edge(Fp8Form form) { return form == Fp8Form::k256 ? 256 : form == Fp8Form::k128 ? 128 : 64; }
// Tiles are counted, and eight more of them and four bands, within 31 bits, and a launch has fewer than 2^32 threads (`experts` times so many tiles).
bool tiles_fit(Fp8Form form, int64_t tm, int64_t N, int64_t experts) {
    const int64_t tn = ceil_div(N, form_edge(form));
    return tm <= (0x7FFFFFFF - 64) / (4 * tn) && tm * tn + kXcd <= (0x7FFFFFFF - 64) / experts &&
           grid_ok(round_up(tm * tn, kXcd) * experts, form == Fp8Form::k64 ? 128 : 256);
}

template <int WR, int WC, int RB, int CB, int SLOTS, bool EXACT, Of OF>
daq_status launch_product(const ProductArgs& p, hipStream_t st) {
    using Product = Fp8Product<WR, WC, RB, CB, SLOTS, EXACT>;
    const int64_t tiles = tile_groups<OF>(p);
    const auto kernel = k_fp8_product<WR, WC, RB, CB, SLOTS, EXACT, OF>;
    if (!allow_lds((const void*)kernel, Product::kLdsBytes)) return DAQ_ERR_HIP;
    DAQ_LAUNCH("fp8_product", st, hipLaunchKernelGGL(kernel, dim3((unsigned)tiles, (unsigned)p.splits), dim3(64 * WR * WC), Product::kLdsBytes, st, p));
    return DAQ_OK;
}
template <Of OF>
daq_status launch_form(Fp8Form form, bool exact, ProductArgs p, hipStream_t st) {
    const int64_t tm = OF == Of::kExpertRows ? p.tiles_m : ceil_div(p.M, form_edge(form));
    if (!tiles_fit(form, tm, p.N, OF == Of::kExpertWeights ? p.experts : 1)) return DAQ_ERR_UNSUPPORTED;
    p.tiles_m = (int)tm;
    p.tiles_n = (int)ceil_div(p.N, form_edge(form));
    if (exact) return form == Fp8Form::k64 ? launch_product<2, 1, 1, 2, 4, true, OF>(p, st) : launch_product<2, 2, 2, 2, 2, true, OF>(p, st);
    if (form == Fp8Form::k64) return launch_product<2, 1, 1, 2, 4, false, OF>(p, st);
    if (form == Fp8Form::k128) {
        // a workgroup to a CU: four stages in LDS (512 x 8192 x 8192 39.4 us instead of 48); two to a CU: two each (2048 x 4096 x 4096 32.8 instead of 38)
        const int64_t tiles = (int64_t)p.tiles_m * p.tiles_n * (OF == Of::kExpertWeights ? p.experts : 1);
        return tiles <= 256 ? launch_product<2, 2, 2, 2, 4, false, OF>(p, st) : launch_product<2, 2, 2, 2, 2, false, OF>(p, st);
    }
    return fp8_large(OF, p, st);
}

}  // namespace

static bool few_fits(int64_t tiles, int64_t N) { return tiles <= 65535 && grid_ok(ceil_div(N, 16), 512); }
// Whether the workgroups of a product of few rows quantize these themselves: 16384 elements are 4 a thread.  us with it and in two launches: 1 x 8192 x 4096
// 10.1 and 13.0 with the weights from memory, 8.5 and 10.9 from the caches; 4 x 8192 x 8192 18.3 and 18.5, 8 x 8192 x 8192 24 and 19.3.
static bool fp8_raw_rows(int64_t rows, int64_t K) { return rows <= 64 && rows * round_up(K, kFp8Block) <= 16384; }

// us that a product of so many tiles of a form takes, by what was measured of each: a fixed time, and one for a stage, longer where more workgroups than one are
// on a CU.  E.g., bfloat16, 64, 128 and 256: 1111 x 1500 x 2030 9.7, 12.7, -; 1777 x 2080 x 4096 28.5, 21.1, 36.5; 2048 x 4096 x 4096 -, 32.8, 38.7;
// 2100 x 6000 x 3000 -, 51, 35.5; 512 x 8192 x 8192 -, 39.4, 66.9; fp32, 64 and 128: 1111 x 1500 x 2030 16.8, 18.8; 1777 x 2080 x 4096 53.5, 35.2.
static double fp8_cost(Fp8Form form, double tiles, double stages, bool exact) {
    switch (form) {
        case Fp8Form::k64: return std::ceil(tiles / 512) * (3 + stages * (exact ? (tiles <= 256 ? 0.53 : 0.8) : tiles <= 256 ? 0.24 : 0.4));
        case Fp8Form::k128: return tiles <= 256 ? 3 + stages * (exact ? 1.02 : 0.57) : std::ceil(tiles / 512) * (3 + stages * (exact ? 1.74 : 0.94));
        default: return exact ? 1e30 : std::ceil(tiles / 256) * (4 + stages * (tiles <= 128 ? 1.04 : 1.36));
    }
}
static Fp8Form least_cost(double t64, double t128, double t256, double stages, bool exact) {
    const double a = fp8_cost(Fp8Form::k64, t64, stages, exact), b = fp8_cost(Fp8Form::k128, t128, stages, exact), c = fp8_cost(Fp8Form::k256, t256, stages, exact);
    return a <= b && a <= c ? Fp8Form::k64 : b <= c ? Fp8Form::k128 : Fp8Form::k256;
}

// Up to 32 rows, while their tiles of 64 would not fill the CUs, the few-rows form, as long as the weights are no more elements than this: it takes longer with every row, tiles (parts of the
// summed axis among them) do not.  us of both, weights from memory:
//   bfloat16   8 rows 8192 x 8192 19.1 and 18.5, 12288 x 4096 15.5 and 13.9, 4096 x 14336 17.7 and 18.2;   16 rows 8192 x 4096 12.6 and 12.8, 4096 x 8192 12.8 and 12.6, 8192 x 8192 21.7
//              and 18.7, 12288 x 4096 17.3 and 14.1;   24 rows 4096 x 4096 9.6 and 10.7, 3000 x 5000 10.6 and 10.9, 5120 x 4096 14.9 and 12.5, 8192 x 8192 26.0 and 19.2
//   fp32       16 rows 8192 x 8192 22.0 and 22.9, 16000 x 4096 21.7 and 21.1;   24 rows 4096 x 4096 9.8 and 12.5, 8192 x 4096 15.9 and 16.7, 12288 x 4096 21.7 and 20.4, 8192 x 8192
//              26.7 and 23.3
static int64_t few_weights(int64_t M, bool exact) {
    constexpr int64_t mi = (int64_t)1 << 20;
    return M <= 8 ? kMaxElems : M <= 16 ? (exact ? kMaxElems : 32 * mi) : M <= 32 ? (exact ? 32 : 16) * mi : 0;
}
static Fp8Plan fp8_plan(int64_t M, int64_t N, int64_t K, bool exact) {
    Fp8Plan pl{};
    const int64_t stages = ceil_div(K, kFp8Block);
    auto tiles = [&](int64_t n) { return (double)ceil_div(M, n) * (double)ceil_div(N, n); };
    pl.form = N * K <= few_weights(M, exact) && few_fits(1, N) && ceil_div(N, 64) < 256 ? Fp8Form::kFew : least_cost(tiles(64), tiles(128), tiles(256), (double)stages, exact);
    pl.splits = 1;
    pl.per_split = (int)stages;
    if (pl.form == Fp8Form::kFew) return pl;
    // parts of the summed axis, of four stages or more, for what they and the launch that adds them up (at 3 TB/s) take less
    double least = fp8_cost(pl.form, tiles(form_edge(pl.form)), (double)stages, exact);
    for (const Fp8Form form : {Fp8Form::k64, Fp8Form::k128})
        for (int s = 2; s <= 16 && stages >= 4 * s; s *= 2) {
            const double cost = fp8_cost(form, tiles(form_edge(form)) * s, std::ceil((double)stages / s), exact) + 3.5 + s * (double)M * (double)N * 8 / 3e6;
            if (cost >= least) continue;
            least = cost;
            pl.form = form;
            pl.per_split = (int)ceil_div(stages, s);
            pl.splits = (int)ceil_div(stages, pl.per_split);
        }
    return pl;
}

static bool one_launch(int64_t M, int64_t N, int64_t K, int y_dtype) {
    return fp8_raw_rows(M, K) && fp8_plan(M, N, K, y_dtype == DAQ_FP32).form == Fp8Form::kFew;
}

// Workgroups of the launch that adds up a product's parts.
static int64_t sum_groups(int64_t M, int64_t N) { return ceil_div(M * ceil_div(N, 4), 256); }
// Whether the launches of a product can be made.
static bool product_fits(const Fp8Plan& pl, int64_t M, int64_t N) {
    return pl.form == Fp8Form::kFew || (tiles_fit(pl.form, ceil_div(M, form_edge(pl.form)), N, 1) && (pl.splits == 1 || grid_ok(sum_groups(M, N), 256)));
}
static daq_status product_sizes(int64_t M, int64_t N, int64_t K) {
    if (M < 0 || N <= 0 || K < 0) return DAQ_ERR_INVALID_ARG;
    daq_status rc = matrix_size(M, K > 0 ? K : 1);
    if (rc == DAQ_OK) rc = matrix_size(N, K > 0 ? K : 1);
    if (rc == DAQ_OK) rc = matrix_size(M, N);
    if (rc != DAQ_OK) return rc;
    return K > kFp8MaxK ? DAQ_ERR_UNSUPPORTED : DAQ_OK;
}
static daq_status result_check(const void* D, int dtype, int64_t N, int64_t ldd, int accumulate) {
    return !dtype_ok(dtype) || !D || !elem_aligned(D, dtype) || ldd < N || (accumulate && dtype != DAQ_FP32) ? DAQ_ERR_INVALID_ARG : DAQ_OK;
}

// X not NULL: A from X, in the call.
static daq_status fp8_matmul(int64_t M, int64_t N, int64_t K, const uint8_t* A, const void* X, int x_dtype, int64_t ldx, const uint8_t* B, void* D, int dtype,
                             int64_t ldd, int accumulate, void* ws, hipStream_t st) {
    const bool exact = dtype == DAQ_FP32;
    const Fp8Plan pl = fp8_plan(M, N, K, exact);
    ProductArgs p{};
    p.a = operand(A, M, K);
    p.b = operand(B, N, K);
    p.M = M;
    p.N = N;
    p.stages = (int)ceil_div(K, kFp8Block);
    p.splits = pl.splits;
    p.per_split = pl.per_split;
    if (pl.splits == 1) {
        p.d = D;
        p.ldd = ldd;
        p.bf16 = dtype == DAQ_BF16;
        p.accumulate = accumulate;
        if (pl.form == Fp8Form::kFew) return fp8_few(Of::kWhole, p, ceil_div(M, 64), std::min<int64_t>(M, 64), X, x_dtype, ldx, K, st);
        return launch_form<Of::kWhole>(pl.form, exact, p, st);
    }
    p.d = ws;
    p.ldd = round_up(N, 4);
    const daq_status rc = launch_form<Of::kWhole>(pl.form, exact, p, st);
    if (rc != DAQ_OK) return rc;
    DAQ_LAUNCH("fp8_sum", st, hipLaunchKernelGGL(k_fp8_sum, dim3((unsigned)sum_groups(M, N)), dim3(256), 0, st, static_cast<const float*>(ws), pl.splits, M, N, D, ldd, dtype == DAQ_BF16, accumulate));
    return DAQ_OK;
}

}  // namespace daq

using namespace daq;

extern "C" daq_status daq_fp8_matmul_workspace(int64_t M, int64_t N, int64_t K, daq_dtype dtype, size_t* bytes) {
    if (!bytes || !dtype_ok(dtype)) return DAQ_ERR_INVALID_ARG;
    *bytes = 0;
    const daq_status rc = product_sizes(M, N, K);
    if (rc != DAQ_OK || M == 0) return rc;
    const Fp8Plan pl = fp8_plan(M, N, K, dtype == DAQ_FP32);
    if (!product_fits(pl, M, N)) return DAQ_ERR_UNSUPPORTED;
    if (pl.splits > 1) *bytes = (size_t)round_up(pl.splits * M * round_up(N, 4) * 4, 256);
    return DAQ_OK;
}

extern "C" daq_status daq_fp8_matmul(int64_t M, int64_t N, int64_t K, const uint8_t* A, const uint8_t* B, void* D, daq_dtype dtype,
                                     int64_t ldd, int32_t accumulate, void* workspace, size_t workspace_bytes, void* stream) {
    size_t need = 0;
    daq_status rc = daq_fp8_matmul_workspace(M, N, K, dtype, &need);
    if (rc != DAQ_OK) return rc;
    if (accumulate && dtype != DAQ_FP32) return DAQ_ERR_INVALID_ARG;
    if (M == 0) return DAQ_OK;
    rc = result_check(D, dtype, N, ldd, accumulate);
    if (rc != DAQ_OK) return rc;
    if (K > 0 && (!A || !aligned256(A) || !B || !aligned256(B))) return DAQ_ERR_INVALID_ARG;
    if (need > 0 && (!workspace || workspace_bytes < need || !aligned256(workspace))) return DAQ_ERR_WORKSPACE;
    return fp8_matmul(M, N, K, A, nullptr, 0, 0, B, D, dtype, ldd, accumulate, workspace, (hipStream_t)stream);
}

extern "C" daq_status daq_fp8_linear_workspace(int64_t M, int64_t N, int64_t K, daq_dtype x_dtype, daq_dtype y_dtype, size_t* bytes) {
    if (!dtype_ok(x_dtype) || K <= 0) return DAQ_ERR_INVALID_ARG;
    size_t product = 0;
    const daq_status rc = daq_fp8_matmul_workspace(M, N, K, y_dtype, &product);
    if (!bytes) return DAQ_ERR_INVALID_ARG;
    *bytes = 0;
    if (rc != DAQ_OK || M == 0 || one_launch(M, N, K, y_dtype)) return rc;
    if (!fp8_rows_grid_ok(M, K)) return DAQ_ERR_UNSUPPORTED;
    daq_fp8_layout L;
    daq_layout_fp8(M, K, &L);
    *bytes = (size_t)L.bytes + product;
    return DAQ_OK;
}

extern "C" daq_status daq_fp8_linear(int64_t M, int64_t N, int64_t K, const void* X, daq_dtype x_dtype, int64_t ldx, const uint8_t* W, void* Y,
                                     daq_dtype y_dtype, int64_t ldy, void* workspace, size_t workspace_bytes, void* stream) {
    size_t need = 0;
    daq_status rc = daq_fp8_linear_workspace(M, N, K, x_dtype, y_dtype, &need);
    if (rc != DAQ_OK) return rc;
    if (M == 0) return DAQ_OK;
    rc = result_check(Y, y_dtype, N, ldy, 0);
    if (rc != DAQ_OK) return rc;
    if (!X || !elem_aligned(X, x_dtype) || ldx < K || !W || !aligned256(W)) return DAQ_ERR_INVALID_ARG;
    if (one_launch(M, N, K, y_dtype)) return fp8_matmul(M, N, K, nullptr, X, x_dtype, ldx, W, Y, y_dtype, ldy, 0, nullptr, (hipStream_t)stream);
    if (!workspace || workspace_bytes < need || !aligned256(workspace)) return DAQ_ERR_WORKSPACE;
    uint8_t* xq = static_cast<uint8_t*>(workspace);
    daq_fp8_layout L;
    daq_layout_fp8(M, K, &L);
    rc = fp8_quantize_rows(X, x_dtype, M, K, ldx, xq, (hipStream_t)stream);
    if (rc != DAQ_OK) return rc;
    return fp8_matmul(M, N, K, xq, nullptr, 0, 0, W, Y, y_dtype, ldy, 0, xq + L.bytes, (hipStream_t)stream);
}

// An expert has at most so many rows: a token may name one several times.
static int64_t most_rows(const daq_experts& plan) { return plan_slots(plan); }

// Experts of up to 32 rows take the few-rows form, by the tiles of 64 that they would be.  us of both, weights from memory, `each` rows of every expert:
//   64 tiles    4 of 1024 x 4096, bfloat16 each 1, 16, 32: 8.3 and 13.4, 9.8 and 13.7, 12.2 and 14.2
//   128 tiles   4 of 2048 x 4096, bfloat16 each 8, 16, 32: 13.0 and 14.4, 14.9 and 14.6, 19.2 and 15.2;  fp32 14.4 and 20.8, 15.5 and 21.0, 19.5 and 21.4
//   192 tiles   6 of 2048 x 2048, bfloat16 each 1, 4, 16: 10.7 and 10.1, 11.4 and 10.2, 13.4 and 10.5;  fp32 12.7 and 13.7, 13.2 and 13.9, 14.8 and 14.1
//   228 tiles   4 of 3600 x 4096, bfloat16 each 1, 4, 16: 20.5 and 17.4, 21.5 and 17.4, 25.1 and 17.7;  fp32 21.7 and 21.6, 22.5 and 21.7, 25.9 and 22.1
// Rows that its workgroups quantize themselves save a launch, which makes up for more than 128 tiles: 6 of 2048 x 2048, each 1, bfloat16 10.1 and 12.9, fp32 10.9 and 16.4, 4 of 4000 x 4096
// 19.3 and 20.9, 21.0 and 25.0.
static Fp8Form experts_form(const daq_experts& plan, int64_t N, int64_t K, bool exact) {
    const int64_t slots = plan_slots(plan), experts = std::min<int64_t>(slots, plan.experts), each = slots / experts, few_tiles = ceil_div(N, 64) * experts;
    const int64_t most = fp8_raw_rows(most_rows(plan), K) || (exact && each <= 4) ? 255 : exact || each <= 16 ? 128 : 64;
    if (each <= 32 && few_tiles <= most && most_tiles(plan, 64) <= 65535) return Fp8Form::kFew;
    const double active = (double)experts;
    auto tiles = [&](int64_t n) { return active * (double)ceil_div(each, n) * (double)ceil_div(N, n); };
    return least_cost(tiles(64), tiles(128), tiles(256), (double)ceil_div(K, kFp8Block), exact);
}
static bool experts_one_launch(const daq_experts& plan, int64_t N, int64_t K, int y_dtype) {
    return experts_form(plan, N, K, y_dtype == DAQ_FP32) == Fp8Form::kFew && fp8_raw_rows(most_rows(plan), K);
}

static int64_t experts_tiles(const daq_experts& plan, Fp8Form form) { return most_tiles(plan, form_edge(form)); }
static bool experts_fit(const daq_experts& plan, int64_t N, int64_t K, bool exact) {
    const Fp8Form form = experts_form(plan, N, K, exact);
    return form == Fp8Form::kFew || tiles_fit(form, experts_tiles(plan, form), N, 1);
}

// X not NULL: A from X, in the call.
static daq_status experts_product(const daq_experts& plan, int64_t N, int64_t K, const uint8_t* A, const void* X, int x_dtype, int64_t ldx, int sorted,
                                  const uint8_t* W, void* Y, int dtype, int64_t ldy, hipStream_t st) {
    const int64_t slots = plan_slots(plan);
    ProductArgs p{};
    p.a = operand(A, sorted ? slots : plan.tokens, K);
    p.b = operand(W, plan.experts * N, K);
    p.M = slots;
    p.N = N;
    p.stages = (int)ceil_div(K, kFp8Block);
    p.d = Y;
    p.ldd = ldy;
    p.bf16 = dtype == DAQ_BF16;
    p.splits = 1;
    p.table = plan.table;
    p.order = plan.rows;
    p.experts = plan.experts;
    p.picks = sorted ? 0 : plan.picks;
    const bool exact = dtype == DAQ_FP32;
    const Fp8Form form = experts_form(plan, N, K, exact);
    if (form == Fp8Form::kFew) return fp8_few(Of::kExpertRows, p, most_tiles(plan, 64), std::min<int64_t>(most_rows(plan), 64), X, x_dtype, ldx, K, st);
    p.tiles_m = (int)experts_tiles(plan, form);
    return launch_form<Of::kExpertRows>(form, exact, p, st);
}

// What the plan, the sizes, the weights and the result have to be.
static daq_status experts_check(const daq_experts* plan, int64_t N, int64_t K, int sorted) {
    if (!plan_ok(plan) || N <= 0 || K <= 0) return DAQ_ERR_INVALID_ARG;
    const int64_t slots = plan_slots(*plan), rows = sorted ? slots : plan->tokens;
    daq_status rc = matrix_size(rows, K);
    if (rc == DAQ_OK) rc = matrix_size(slots, N);
    if (rc == DAQ_OK) rc = N > (((int64_t)1 << 31) - 1) / plan->experts ? DAQ_ERR_UNSUPPORTED : matrix_size(plan->experts * N, K);
    if (rc != DAQ_OK) return rc;
    // rows that are taken in another order are read through one descriptor
    if (K > kFp8MaxK || (!sorted && rows * round_up(K, kFp8Block) > (int64_t)kTileReach)) return DAQ_ERR_UNSUPPORTED;
    return DAQ_OK;
}

extern "C" daq_status daq_experts_matmul(const daq_experts* plan, int64_t N, int64_t K, const uint8_t* A, int32_t sorted, const uint8_t* W, void* Y,
                                         daq_dtype dtype, int64_t ldy, void* stream) {
    daq_status rc = experts_check(plan, N, K, sorted);
    if (rc != DAQ_OK) return rc;
    if (!dtype_ok(dtype)) return DAQ_ERR_INVALID_ARG;
    if (plan->tokens == 0) return DAQ_OK;
    rc = result_check(Y, dtype, N, ldy, 0);
    if (rc != DAQ_OK) return rc;
    if (!A || !aligned256(A) || !W || !aligned256(W)) return DAQ_ERR_INVALID_ARG;
    return experts_product(*plan, N, K, A, nullptr, 0, 0, sorted, W, Y, dtype, ldy, (hipStream_t)stream);
}

extern "C" daq_status daq_experts_linear_workspace(const daq_experts* plan, int64_t N, int64_t K, daq_dtype x_dtype, int32_t sorted, size_t* bytes) {
    if (!bytes || !dtype_ok(x_dtype)) return DAQ_ERR_INVALID_ARG;
    *bytes = 0;
    const daq_status rc = experts_check(plan, N, K, sorted);
    if (rc != DAQ_OK || plan->tokens == 0) return rc;
    daq_fp8_layout L;
    daq_layout_fp8(sorted ? plan_slots(*plan) : plan->tokens, K, &L);
    *bytes = (size_t)L.bytes;
    return DAQ_OK;
}

extern "C" daq_status daq_experts_linear(const daq_experts* plan, int64_t N, int64_t K, const void* X, daq_dtype x_dtype, int64_t ldx, int32_t sorted,
                                         const uint8_t* W, void* Y, daq_dtype y_dtype, int64_t ldy, void* workspace, size_t workspace_bytes, void* stream) {
    size_t need = 0;
    daq_status rc = daq_experts_linear_workspace(plan, N, K, x_dtype, sorted, &need);
    if (rc != DAQ_OK) return rc;
    if (!dtype_ok(y_dtype)) return DAQ_ERR_INVALID_ARG;
    if (plan->tokens == 0) return DAQ_OK;
    rc = result_check(Y, y_dtype, N, ldy, 0);
    if (rc != DAQ_OK) return rc;
    if (!X || !elem_aligned(X, x_dtype) || ldx < K || !W || !aligned256(W)) return DAQ_ERR_INVALID_ARG;
    const int64_t rows = sorted ? plan_slots(*plan) : plan->tokens;
    if (experts_one_launch(*plan, N, K, y_dtype)) return experts_product(*plan, N, K, nullptr, X, x_dtype, ldx, sorted, W, Y, y_dtype, ldy, (hipStream_t)stream);
    if (!fp8_rows_grid_ok(rows, K) || !experts_fit(*plan, N, K, y_dtype == DAQ_FP32)) return DAQ_ERR_UNSUPPORTED;
    if (need > 0 && (!workspace || workspace_bytes < need || !aligned256(workspace))) return DAQ_ERR_WORKSPACE;
    rc = fp8_quantize_rows(X, x_dtype, rows, K, ldx, static_cast<uint8_t*>(workspace), (hipStream_t)stream);
    if (rc != DAQ_OK) return rc;
    return experts_product(*plan, N, K, static_cast<const uint8_t*>(workspace), nullptr, 0, 0, sorted, W, Y, y_dtype, ldy, (hipStream_t)stream);
}

extern "C" daq_status daq_experts_weight_grad(const daq_experts* plan, int64_t N, int64_t K, const uint8_t* dY, const uint8_t* X, void* dW,
                                              daq_dtype dtype, int64_t ldw, int64_t stride, int32_t accumulate, void* stream) {
    if (!plan_ok(plan) || N <= 0 || K <= 0 || !dtype_ok(dtype) || (accumulate && dtype != DAQ_FP32)) return DAQ_ERR_INVALID_ARG;
    const int64_t columns = most_tiles(*plan, 128) * 128;
    daq_status rc = matrix_size(N, std::max<int64_t>(columns, 1));
    if (rc == DAQ_OK) rc = matrix_size(K, std::max<int64_t>(columns, 1));
    if (rc == DAQ_OK) rc = matrix_size(N, K);
    if (rc != DAQ_OK) return rc;
    if (columns > kFp8MaxK || N * K > kMaxElems / plan->experts) return DAQ_ERR_UNSUPPORTED;
    if (!dW || !elem_aligned(dW, dtype) || ldw < K || stride < 0 || (plan->experts > 1 && stride < (N - 1) * ldw + K)) return DAQ_ERR_INVALID_ARG;
    if (plan->tokens == 0 && accumulate) return DAQ_OK;
    if (!plan->table || ((uintptr_t)plan->table & 3)) return DAQ_ERR_INVALID_ARG;      // (read without tokens too)
    if (plan->tokens > 0 && (!dY || !aligned256(dY) || !X || !aligned256(X))) return DAQ_ERR_INVALID_ARG;
    ProductArgs p{};
    p.a = operand(dY, N, columns);
    p.b = operand(X, K, columns);
    p.M = N;
    p.N = K;
    p.d = dW;
    p.ldd = ldw;
    p.accumulate = accumulate;
    p.bf16 = dtype == DAQ_BF16;
    p.splits = 1;
    p.table = plan->table;
    p.experts = plan->experts;
    p.stride = stride;
    const bool exact = dtype == DAQ_FP32;
    auto tiles = [&](int64_t n) { return (double)plan->experts * (double)ceil_div(N, n) * (double)ceil_div(K, n); };
    const Fp8Form form = least_cost(tiles(64), tiles(128), tiles(256), (double)ceil_div(plan_slots(*plan), kFp8Block * (int64_t)plan->experts), exact);
    return launch_form<Of::kExpertWeights>(form, exact, p, (hipStream_t)stream);
}
