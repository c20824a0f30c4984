// Products of microscaled 4-bit matrices, D[m][n] = sum over k of A[m][k] * B[n][k], and linear layers on them.
//
// The matrix instruction of 32 x 32 x 64 takes of each operand a block of 32 elements a lane (16 bytes and a scale byte): lane l has
// row l % 32 and block l / 32 of the 64 columns.  The packed layout holds operands in that order, so a wave loads a 32 x 64 tile
// as one contiguous KiB and the scale bytes of four tiles as one contiguous 256 bytes.  B goes in as the instruction's first
// operand, so that a lane holds four neighbouring columns of a row of D at a time.
#include <cmath>

#include "mx4_block.h"
#include "tile_product.h"

namespace daq {

namespace {

struct MatmulArgs {
    const uint8_t* a;       // codes
    const uint8_t* a_scales;
    const uint8_t* b;
    const uint8_t* b_scales;
    int64_t M, N;
    int a_blocks, b_blocks;   // row blocks of 32
    int groups;               // 256 columns each
    void* d;
    int64_t ldd;
    int bf16;
};

// Four columns of a row of D.
__device__ __forceinline__ void store4(const MatmulArgs& p, int64_t row, int64_t col, f32x4 v) {
    const int left = (int)min(p.N - col, (int64_t)4);
    if (p.bf16) {
        uint16_t* z = static_cast<uint16_t*>(p.d) + row * p.ldd + col;
        const u32x2_a2 w = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
        if (left == 4) *reinterpret_cast<u32x2_a2*>(z) = w;
        else
            for (int e = 0; e < left; ++e) z[e] = (uint16_t)(w[e / 2] >> (16 * (e & 1)));
    } else {
        float* z = static_cast<float*>(p.d) + row * p.ldd + col;
        if (left == 4) *reinterpret_cast<u32x4_a4*>(z) = __builtin_bit_cast(u32x4, v);
        else
            for (int e = 0; e < left; ++e) z[e] = v[e];
    }
}

// Tiles of 32 RB WR x 32 CB WC results, a workgroup each.  Workgroup b runs on XCD b % 8; an XCD takes an eighth of the tiles, in bands
// of four row tiles, so that the 32 it holds at a time share twelve panels of the operands in its L2.
// 16384 x 8192 x 8192 464-564 us, medians of traces 503 and 524, 4.3 PFLOP/s: the matrix cores are busy 72 % of the cycles, at the 1.3 to 1.6 GHz
// that the power limit leaves; a loop of the same instructions on registers alone makes 5.4-6.2.  128 x 128 tiles read twice as much LDS for the same
// products: 1777 x 2080 x 4096, 238 tiles, 12.7-16.1 us, median 14, 2.2 PFLOP/s.  Results that left as 8 bytes a lane took 554 us at the first size.
template <int WR, int WC, int RB, int CB>
__global__ __launch_bounds__(64 * WR * WC, 1) void k_mx4_tiles(MatmulArgs p, int tiles_m, int tiles_n, int per_xcd) {
    using Product = TileProduct<WR, WC, RB, CB, true>;
    extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
    const int64_t t = (int64_t)(blockIdx.x % kXcd) * per_xcd + blockIdx.x / kXcd;
    if (t >= (int64_t)tiles_m * tiles_n) return;
    const int64_t band = t / (4 * tiles_n);
    const int rest = (int)(t - band * 4 * tiles_n), high = min(4, tiles_m - (int)band * 4);
    const int tm = (int)band * 4 + rest % high, tn = rest / high;
    const TileOperand r{p.a, p.a_scales, p.a_blocks, p.groups * 4, 0, 0, 0}, c{p.b, p.b_scales, p.b_blocks, p.groups * 4, 0, 0, 0};
    Product prod;
    prod.run(r, c, tm * WR * RB, tn * WC * CB, 0, p.groups * (kGroupSteps / Product::kSteps), lds);
    const int wave = threadIdx.x / kWave;
    const int64_t m0 = ((int64_t)tm * WR + wave / WC) * RB * 32, n0 = ((int64_t)tn * WC + wave % WC) * CB * 32;
    if (p.bf16) {
        prod.store(true, lds, [&](int row, int col, u32x4 v) {
            const int64_t m = m0 + row, n = n0 + col;
            if (m >= p.M || n >= p.N) return;
            uint16_t* z = static_cast<uint16_t*>(p.d) + m * p.ldd + n;
            if (n + 8 <= p.N) {
                *reinterpret_cast<u32x4_a2*>(z) = v;
            } else {
#pragma unroll
                for (int i = 0; i < 7; ++i)
                    if (n + i < p.N) z[i] = (uint16_t)(v[i / 2] >> (16 * (i & 1)));
            }
        });
    } else {
        prod.store(false, lds, [&](int row, int col, u32x4 v) {
            const int64_t m = m0 + row, n = n0 + col;
            if (m >= p.M || n >= p.N) return;
            uint32_t* z = static_cast<uint32_t*>(p.d) + m * p.ldd + n;
            if (n + 4 <= p.N) {
                *reinterpret_cast<u32x4_a4*>(z) = v;
            } else {
#pragma unroll
                for (int i = 0; i < 3; ++i)
                    if (n + i < p.N) z[i] = v[i];
            }
        });
    }
}

template <int WR, int WC, int RB, int CB>
daq_status launch_tiles(const MatmulArgs& p, hipStream_t st) {
    using Product = TileProduct<WR, WC, RB, CB, true>;
    const int64_t tm = ceil_div(p.a_blocks, WR * RB), tn = ceil_div(p.b_blocks, WC * CB), per = ceil_div(tm * tn, kXcd);
    const auto kernel = k_mx4_tiles<WR, WC, RB, CB>;
    if (!allow_lds((const void*)kernel, Product::kLdsBytes)) return DAQ_ERR_HIP;
    DAQ_LAUNCH("mx4_tiles", st,
               hipLaunchKernelGGL(kernel, dim3((unsigned)(per * kXcd)), dim3(64 * WR * WC), Product::kLdsBytes, st, p, (int)tm, (int)tn, (int)per));
    return DAQ_OK;
}

// Small products: a workgroup has 32 x 32 results, and its waves share the groups of 256 along k, everything a wave needs asked for
// a group ahead, with no tile to wait for; the waves' sums meet in LDS.  What bounds it is the way of the weights, one after the other
// through each wave: 13 x 2048 x 8192 (8.9 MB of weights) 5.0 us, 1 x 8192 x 8192 (36 MB) 9.7 with its quantization, 3.7 TB/s.
// X: type of the rows: void for packed ones; otherwise every workgroup quantizes them itself, to the nearest codes, a block a thread, into
// LDS, while its first weights are on their way: a launch less, for rows of not many more blocks than a workgroup has threads.
struct FewArgs {
    MatmulArgs d;
    const void* x;
    int64_t ldx, K;
};

constexpr int kFewWaves = 8;
template <typename X>
__global__ __launch_bounds__(64 * kFewWaves) void k_mx4_few(FewArgs f) {
    constexpr bool kRaw = !std::is_void_v<X>;
    extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
    float* sums = reinterpret_cast<float*>(lds);       // [kFewWaves][32][32]
    uint8_t* xq = lds + kFewWaves * 4096;                 // raw: [group][step][half][row] codes, then [group][half][row] scale words
    const MatmulArgs& p = f.d;
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int cb = blockIdx.x;
    const uint8_t* b = p.b + (int64_t)cb * p.groups * 4096 + lane * 16;
    const uint8_t* sb = p.b_scales + (int64_t)cb * p.groups * 256 + lane * 4;
    const uint8_t* a = p.a + (int64_t)blockIdx.y * p.groups * 4096 + lane * 16;
    const uint8_t* sa = p.a_scales + (int64_t)blockIdx.y * p.groups * 256 + lane * 4;
    const int rows = (int)p.M;                         // (raw: at most 32)
    struct Group {
        v4i vb[4], va[4];
        int wb, wa;
    };
    auto load = [&](int g, Group& o) {
        o.wb = *reinterpret_cast<const int*>(sb + (int64_t)g * 256);
#pragma unroll
        for (int s = 0; s < 4; ++s) o.vb[s] = *reinterpret_cast<const v4i*>(b + ((int64_t)g * 4 + s) * 1024);
        if constexpr (!kRaw) {
            o.wa = *reinterpret_cast<const int*>(sa + (int64_t)g * 256);
#pragma unroll
            for (int s = 0; s < 4; ++s) o.va[s] = *reinterpret_cast<const v4i*>(a + ((int64_t)g * 4 + s) * 1024);
        }
    };
    Group cur, next;
    if (wave < p.groups) load(wave, cur);
    if constexpr (kRaw) {
        const int per_row = p.groups * 8;
        for (int t = threadIdx.x; t < rows * per_row; t += 64 * kFewWaves) {
            const int row = t / per_row, blk = t - row * per_row;
            const int64_t left = f.K - (int64_t)blk * 32;
            u32x4 codes = {0, 0, 0, 0};
            uint32_t byte = 0;
            if (left > 0) {
                const X* from = static_cast<const X*>(f.x) + row * f.ldx + (int64_t)blk * 32;
                uint32_t v[Words<X>::kBlock];
                if (left >= 32) load_block(from, v);
                else load_block(from, (int)left, v);
                byte = scale_byte<2>(top_of(v));
                codes = nearest_codes(v, byte);
            }
            *reinterpret_cast<u32x4*>(xq + (blk * rows + row) * 16) = codes;
            xq[per_row * rows * 16 + ((blk / 8 * 2 + blk % 2) * rows + row) * 4 + (blk / 2) % 4] = (uint8_t)byte;
        }
        __syncthreads();
    }
    v16f acc = {};
    for (int g = wave; g < p.groups; g += kFewWaves) {
        const bool more = g + kFewWaves < p.groups;
        if (more) load(g + kFewWaves, next);
        if constexpr (kRaw) {
            const int row = lane % 32, half = lane / 32;
            const bool there = row < rows;
            const int r = there ? row : 0;
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const v4i v = *reinterpret_cast<const v4i*>(xq + ((g * 8 + s * 2 + half) * rows + r) * 16);
                cur.va[s] = there ? v : v4i{0, 0, 0, 0};
            }
            const int w = *reinterpret_cast<const int*>(xq + p.groups * 8 * rows * 16 + ((g * 2 + half) * rows + r) * 4);
            cur.wa = there ? w : 0;
        }
        acc = mfma4<0>(cur.vb[0], cur.va[0], acc, cur.wb, cur.wa);
        acc = mfma4<1>(cur.vb[1], cur.va[1], acc, cur.wb, cur.wa);
        acc = mfma4<2>(cur.vb[2], cur.va[2], acc, cur.wb, cur.wa);
        acc = mfma4<3>(cur.vb[3], cur.va[3], acc, cur.wb, cur.wa);
        if (more) cur = next;
    }
    // (16-byte pieces of a row in the order piece ^ row % 8: no bank conflicts)
    const int m = lane % 32, h = lane / 32, t = threadIdx.x, tm = t / 8;
    const int64_t row0 = (int64_t)blockIdx.y * 32;
    if (row0 + m < p.M) {
#pragma unroll
        for (int q = 0; q < 4; ++q)
            *reinterpret_cast<f32x4*>(sums + wave * 1024 + m * 32 + (((2 * q + h) ^ m) & 7) * 4) = f32x4{acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]};
    }
    __syncthreads();
    const int64_t row = row0 + tm, col = (int64_t)cb * 32 + (t & 7) * 4;
    if (t < 256 && row < p.M && col < p.N) {
        f32x4 v = {0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < kFewWaves; ++w) v += *reinterpret_cast<const f32x4*>(sums + w * 1024 + tm * 32 + ((t ^ tm) & 7) * 4);
        store4(p, row, col, v);
    }
}

// LDS of a workgroup; raw: with `rows` rows of `groups` groups.
size_t few_lds(int64_t rows, int groups) { return kFewWaves * 4096 + (size_t)rows * groups * (8 * 16 + 8); }
template <typename X>
daq_status launch_few(const FewArgs& f, hipStream_t st) {
    const size_t bytes = few_lds(std::is_void_v<X> ? 0 : f.d.M, f.d.groups);
    const auto kernel = k_mx4_few<X>;
    if (!allow_lds((const void*)kernel, bytes)) return DAQ_ERR_HIP;
    DAQ_LAUNCH("mx4_few", st,
               hipLaunchKernelGGL(kernel, dim3((unsigned)f.d.b_blocks, (unsigned)f.d.a_blocks), dim3(64 * kFewWaves), bytes, st, f));
    return DAQ_OK;
}

}  // namespace

// Whether the grid of a small product holds its workgroups.
static bool few_fits(int64_t a_blocks, int64_t b_blocks) { return a_blocks <= 65535 && grid_ok(b_blocks, 64 * kFewWaves); }

// Which form a product takes: the one of the least time by what was measured of each (us, launch included).
//   small products   2 + the longest of: 0.55 a group that a wave goes through; what the workgroups read at 19 TB/s (L2); B at 5 TB/s
//   128 x 128 tiles  up to a tile for each CU 3.2 + 0.55 a group; more, two to a CU: 3 + 1.17 a group for every 512
//   256 x 256 tiles  6 + 1.7 a group for every 256
// e.g. 512 x 512 x 8192: 5.3, 18, 41; 128 x 8192 x 8192: 18.6, 20, 44; 1777 x 2080 x 4096: 28, 12.4, 26; 2048 x 4096 x 4096: -, 22, 29;
// 4096 x 4096 x 4096: -, 42, 35.5; 16384 x 8192 x 8192: -, 563, 484.
// Tiles end where a descriptor does: one group more, and the last columns of a row block would read as zeros.
MatmulForm matmul_form(int64_t a_blocks, int64_t b_blocks, int64_t groups) {
    const double g = (double)groups, small = (double)(ceil_div(a_blocks, 4) * ceil_div(b_blocks, 4)), big = (double)(ceil_div(a_blocks, 8) * ceil_div(b_blocks, 8));
    const double few = !few_fits(a_blocks, b_blocks) ? 1e30 : 2.0 + std::max({0.55 * std::ceil(g / kFewWaves), (double)a_blocks * b_blocks * g * 8704 / 19e6, b_blocks * g * 4352 / 5e6});
    const bool reached = groups * kGroupSteps * 1024 <= (int64_t)kTileReach;
    const double tiles = !reached ? 1e30 : small <= 256 ? 3.2 + 0.55 * g : std::ceil(small / 512) * (3.0 + 1.17 * g);
    const double wide = !reached ? 1e30 : std::ceil(big / 256) * (6.0 + 1.7 * g);
    const double least = std::min({few, tiles, wide});
    return few == least ? MatmulForm::kFew : tiles == least ? MatmulForm::kSmall : MatmulForm::kBig;
}

// What the packed operands, the sizes and the result have to be, and the form of the product.
static daq_status matmul_check(int64_t M, int64_t N, int64_t K, const void* B, const void* D, int dtype, int64_t ldd, MatmulForm& form) {
    if (!dtype_ok(dtype)) return DAQ_ERR_INVALID_ARG;
    daq_status rc = matrix_size(M, K);
    if (rc == DAQ_OK) rc = matrix_size(N, K);
    if (rc == DAQ_OK) rc = matrix_size(M, N > 0 ? N : 1);
    if (rc != DAQ_OK) return rc;
    if (N <= 0) return DAQ_ERR_INVALID_ARG;
    if (K >= (int64_t)1 << 28) return DAQ_ERR_UNSUPPORTED;   // what is counted along k is within 32 bits
    if (M == 0) return DAQ_OK;
    if (!B || !aligned256(B) || !D || !elem_aligned(D, dtype) || ldd < N) return DAQ_ERR_INVALID_ARG;
    const int64_t a_blocks = ceil_div(M, 32), b_blocks = ceil_div(N, 32);
    form = matmul_form(a_blocks, b_blocks, ceil_div(K, kMxGroup));
    const int64_t edge = form == MatmulForm::kBig ? 8 : 4, tiles = round_up(ceil_div(a_blocks, edge) * ceil_div(b_blocks, edge), kXcd);
    if (form == MatmulForm::kFew ? !few_fits(a_blocks, b_blocks) : !grid_ok(tiles, form == MatmulForm::kBig ? 512 : 256)) return DAQ_ERR_UNSUPPORTED;
    return DAQ_OK;
}

// Whether the workgroups of the product quantize the rows themselves: nearest codes, one block a thread or two (bfloat16).  us with it and
// in two launches: 1 x 8192 x 2048 4.4 and 6.8, 4 x 8192 x 8192 9.8 and 12.3, 16 x 2048 x 2048 4.3 and 5.8, from fp32 6.7 and 6.1;
// 32 x 8192 x 2048 7.2 and 6.5.
bool raw_rows(int64_t M, int64_t K, int dtype, int mode) {
    return M <= 32 && mode == DAQ_ROUND_NEAREST && M * ceil_div(K, kMxGroup) * 8 * dtype_size(dtype) <= 2048;
}
static bool one_launch(int64_t M, int64_t N, int64_t K, int dtype, int mode) { return raw_rows(M, K, dtype, mode) && few_fits(1, ceil_div(N, 32)); }

static daq_status mx4_matmul(MatmulForm form, int64_t M, int64_t N, int64_t K, const uint8_t* A, const uint8_t* B, void* D, int dtype, int64_t ldd,
                             hipStream_t st) {
    daq_mx4_layout la, lb;
    daq_layout_mx4(M, K, &la);
    daq_layout_mx4(N, K, &lb);
    const MatmulArgs p{A, A + la.off_scales, B, B + lb.off_scales, M, N, la.row_blocks, lb.row_blocks, la.groups,
                       D, ldd, dtype == DAQ_BF16};
    switch (form) {
        case MatmulForm::kFew: return launch_few<void>(FewArgs{p, nullptr, 0, K}, st);
        case MatmulForm::kSmall: return launch_tiles<2, 2, 2, 2>(p, st);
        case MatmulForm::kBig: break;
    }
    return launch_tiles<2, 4, 4, 2>(p, st);
}

}  // namespace daq

using namespace daq;

extern "C" daq_status daq_mx4_matmul_workspace(int64_t M, int64_t N, int64_t K, size_t* bytes) {
    if (!bytes) return DAQ_ERR_INVALID_ARG;
    *bytes = 0;
    const daq_status rc = matrix_size(M, K);
    if (rc != DAQ_OK) return rc;
    return N > 0 ? matrix_size(N, K) : DAQ_ERR_INVALID_ARG;
}

extern "C" daq_status daq_mx4_matmul(int64_t M, int64_t N, int64_t K, const uint8_t* A, const uint8_t* B, void* D, daq_dtype dtype,
                                     int64_t ldd, void* workspace, size_t workspace_bytes, void* stream) {
    MatmulForm form = MatmulForm::kFew;
    const daq_status rc = matmul_check(M, N, K, B, D, dtype, ldd, form);
    if (rc != DAQ_OK) return rc;
    if (M == 0) return DAQ_OK;
    if (!A || !aligned256(A)) return DAQ_ERR_INVALID_ARG;
    return mx4_matmul(form, M, N, K, A, B, D, dtype, ldd, (hipStream_t)stream);
}

extern "C" daq_status daq_mx4_linear_workspace(int64_t M, int64_t N, int64_t K, daq_dtype x_dtype, daq_round mode, size_t* bytes) {
    if (!dtype_ok(x_dtype) || (mode != DAQ_ROUND_NEAREST && mode != DAQ_ROUND_STOCHASTIC)) return DAQ_ERR_INVALID_ARG;
    size_t product = 0;
    const daq_status rc = daq_mx4_matmul_workspace(M, N, K, &product);
    if (!bytes) return DAQ_ERR_INVALID_ARG;
    *bytes = 0;
    if (rc != DAQ_OK || one_launch(M, N, K, x_dtype, mode)) return rc;
    daq_mx4_layout L;
    daq_layout_mx4(M, K, &L);
    *bytes = (size_t)L.bytes + product;
    return DAQ_OK;
}

extern "C" daq_status daq_mx4_linear(int64_t M, int64_t N, int64_t K, const void* X, daq_dtype x_dtype, int64_t ldx, daq_round mode,
                                     uint64_t seed, const uint8_t* W, void* Y, daq_dtype y_dtype, int64_t ldy, void* workspace,
                                     size_t workspace_bytes, void* stream) {
    MatmulForm form = MatmulForm::kFew;
    daq_status rc = matmul_check(M, N, K, W, Y, y_dtype, ldy, form);
    if (rc == DAQ_OK) rc = mx4_quantize_check(X, x_dtype, M, K, ldx, mode);
    if (rc != DAQ_OK) return rc;
    if (M == 0) return DAQ_OK;
    if (one_launch(M, N, K, x_dtype, mode)) {
        daq_mx4_layout lb;
        daq_layout_mx4(N, K, &lb);
        const FewArgs f{{nullptr, nullptr, W, W + lb.off_scales, M, N, 1, lb.row_blocks, lb.groups, Y, ldy, y_dtype == DAQ_BF16}, X, ldx, K};
        return x_dtype == DAQ_BF16 ? launch_few<uint16_t>(f, (hipStream_t)stream) : launch_few<float>(f, (hipStream_t)stream);
    }
    size_t need = 0;
    rc = daq_mx4_linear_workspace(M, N, K, x_dtype, mode, &need);
    if (rc != DAQ_OK) return rc;
    if (need > 0 && (!workspace || workspace_bytes < need || !aligned256(workspace))) return DAQ_ERR_WORKSPACE;
    uint8_t* xq = static_cast<uint8_t*>(workspace);
    rc = mx4_quantize(X, x_dtype, M, K, ldx, false, mode == DAQ_ROUND_STOCHASTIC, seed, xq, (hipStream_t)stream);
    if (rc != DAQ_OK) return rc;
    return mx4_matmul(form, M, N, K, xq, W, Y, y_dtype, ldy, (hipStream_t)stream);
}
