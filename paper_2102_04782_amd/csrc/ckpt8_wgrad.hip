// Weight gradient of a linear layer from its input saved in 8 bits, dW[n][k] = sum over m of dY[m][n] * X^[m][k].
//
// A decoded code is an integer of at most seven bits times a power of two, so X^ is exact in bfloat16 and the products run on the
// bfloat16 matrix cores with fp32 sums.  An fp32 gradient is the sum of three bfloat16 values of eight bits each.
//
// Both operands have their summed axis, the tokens, outermost.  A first launch brings X^, and dY where the products do not read it as it is,
// into the order of the matrix instructions (eight tokens of a column in 16 bytes), decoding the one and splitting an fp32 dY on
// the way: each is read and written once, at 5.4 TB/s (X^ of 16384 x 4096 35 us, with a dY of 8192 columns 137).  The products then run on
// whole KiB tiles: 16384 x 8192 x 4096 884-988 us, medians of traces 939 and 943, 1.17 PFLOP/s, against 1.85 of the same instructions on registers alone, both at
// what clock the power limit leaves; torch's bfloat16 product of 8192 x 8192 x 8192 makes 1.2.
#include "tile_product.h"

namespace daq {

namespace {

constexpr int kStageM = 16 * kGroupSteps;   // tokens of a stage
constexpr int kParts = 3;                   // bfloat16 values that an fp32 value is the sum of

struct OrderArgs {
    const void* dy;
    int64_t lddy;
    const uint8_t* codes;
    const uint8_t* scales;
    int64_t pitch;
    int64_t M, N;
    uint8_t* dy_tiles;
    uint8_t* x_tiles;
    int n_blocks, k_blocks;      // row blocks of 32 of either operand
    int steps;                   // of 16 tokens, a multiple of kGroupSteps
    uint32_t dy_groups;          // workgroups of dY
};

// x = hi + mid + lo, each the leading eight bits of what is left (a value that is not finite stays whole).
__device__ __forceinline__ void split3(float x, uint32_t& hi, uint32_t& mid, uint32_t& lo) {
    const uint32_t h = __float_as_uint(x) & 0xFFFF0000u;
    hi = h >> 16;
    const bool finite = (h & 0x7F800000u) != 0x7F800000u;
    const float r = finite ? x - bits_as<float>(h) : 0.0f;
    const uint32_t m = __float_as_uint(r) & 0xFFFF0000u;
    mid = m >> 16;
    lo = __float_as_uint(r - bits_as<float>(m)) >> 16;
    if (!finite && x != x) hi |= 0x40;   // a NaN of low bits only
}

// Four columns of eight tokens a lane, as words of two neighbouring columns, to the order of the tiles, 16 bytes a column: through the
// wave's share of LDS, so that every store of the wave is half a KiB in a row.  Pieces lie there in the order piece ^ piece / 8 % 4, which
// keeps writes (every fourth piece) and reads off one another's banks.  to: the wave's 128 columns; col: the lane's first.
__device__ __forceinline__ void store_columns(uint8_t* lds, uint8_t* to, int64_t block_bytes, int blocks, const u32x2 (&v)[8]) {
    const int lane = threadIdx.x % kWave, half = lane / 32;
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            w[i] = __builtin_amdgcn_perm(v[2 * i + 1][c / 2], v[2 * i][c / 2], (c & 1) ? 0x07060302u : 0x05040100u);
        const int piece = half * 128 + (lane % 32) * 4 + c;
        *reinterpret_cast<u32x4*>(lds + (piece ^ (piece / 8 & 3)) * 16) = w;
    }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int piece = half * 128 + k * 32 + lane % 32;
        const u32x4 w = *reinterpret_cast<const u32x4*>(lds + (piece ^ (piece / 8 & 3)) * 16);
        if (k < blocks) *reinterpret_cast<u32x4*>(to + k * block_bytes + lane * 16) = w;
    }
    __builtin_amdgcn_wave_barrier();
}

// A workgroup takes 128 columns x 64 tokens of either operand, a wave 16 of the tokens, a lane four columns of eight tokens.
template <typename T>
__global__ __launch_bounds__(256) void k_ckpt8_order(OrderArgs p) {
    __shared__ __attribute__((aligned(16))) uint8_t shares[4][4096];
    uint8_t* lds = shares[threadIdx.x / kWave];
    const int lane = threadIdx.x % kWave;
    const bool of_dy = blockIdx.x < p.dy_groups;
    const uint32_t at = of_dy ? blockIdx.x : blockIdx.x - p.dy_groups;
    const int blocks = of_dy ? p.n_blocks : p.k_blocks;
    const uint32_t wide = (uint32_t)(blocks + 3) / 4, stage = at / wide;
    const int64_t step = (int64_t)stage * kGroupSteps + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int b0 = (int)(at - stage * wide) * 4, nb = min(4, blocks - b0);     // row blocks of the tiles
    const int64_t col = (int64_t)b0 * 32 + (lane % 32) * 4;
    const int64_t m0 = step * 16 + (lane / 32) * 8;
    const int64_t block_bytes = (int64_t)p.steps * 1024 * (of_dy && sizeof(T) == 4 ? kParts : 1);
    // Rows and columns behind the last ones are read from places that exist and cleared afterwards, so that a lane has all its reads
    // under way before it waits for the first.
    int64_t row[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) row[j] = min(m0 + j, p.M - 1);
    const bool cut = m0 + 8 > p.M;
    if (of_dy) {
        const T* src = static_cast<const T*>(p.dy) + col;
        constexpr int kWords = sizeof(T) == 2 ? 2 : 4;
        uint32_t q[8][kWords];
        if (p.N >= 4) {
            // (a lane at the last columns reads the last four, and moves its own to the front)
            const int64_t from = min(col, p.N - 4);
            src = static_cast<const T*>(p.dy) + from;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if constexpr (sizeof(T) == 2) {
                    const u32x2_a2 v = *reinterpret_cast<const u32x2_a2*>(src + row[j] * p.lddy);
                    q[j][0] = v[0], q[j][1] = v[1];
                } else {
                    const u32x4_a4 v = *reinterpret_cast<const u32x4_a4*>(src + row[j] * p.lddy);
#pragma unroll
                    for (int i = 0; i < 4; ++i) q[j][i] = v[i];
                }
            }
            const int64_t d = col - from;
            if (d > 0) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if constexpr (sizeof(T) == 2) {
                        const uint64_t v = d < 4 ? (((uint64_t)q[j][1] << 32) | q[j][0]) >> (16 * (d & 3)) : 0;
                        q[j][0] = (uint32_t)v, q[j][1] = (uint32_t)(v >> 32);
                    } else {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            uint32_t v = 0;
#pragma unroll
                            for (int k = 1; i + k < 4; ++k) v = d == k ? q[j][i + k] : v;
                            q[j][i] = v;
                        }
                    }
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                uint32_t e[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    e[i] = 0;
                    if (col + i < p.N) {
                        const T v = src[row[j] * p.lddy + i];
                        if constexpr (sizeof(T) == 2) e[i] = v;
                        else e[i] = __float_as_uint(v);
                    }
                }
                if constexpr (sizeof(T) == 2) {
                    q[j][0] = e[0] | (e[1] << 16), q[j][1] = e[2] | (e[3] << 16);
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) q[j][i] = e[i];
                }
            }
        }
        if (cut) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int i = 0; i < kWords; ++i) q[j][i] = m0 + j < p.M ? q[j][i] : 0u;
        }
        if constexpr (sizeof(T) == 2) {
            u32x2 v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = u32x2{q[j][0], q[j][1]};
            store_columns(lds, p.dy_tiles + b0 * block_bytes + step * 1024, block_bytes, nb, v);
        } else {
            u32x2 v[kParts][8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                uint32_t h[4][kParts];
#pragma unroll
                for (int i = 0; i < 4; ++i) split3(bits_as<float>(q[j][i]), h[i][0], h[i][1], h[i][2]);
#pragma unroll
                for (int k = 0; k < kParts; ++k) v[k][j] = u32x2{h[0][k] | (h[1][k] << 16), h[2][k] | (h[3][k] << 16)};
            }
            // the three parts of a step are tiles one after the other
#pragma unroll
            for (int k = 0; k < kParts; ++k) store_columns(lds, p.dy_tiles + b0 * block_bytes + (step * kParts + k) * 1024, block_bytes, nb, v[k]);
        }
    } else {
        const int64_t from = col < p.pitch ? col : 0;    // (columns behind the last block are not stored)
        uint32_t w[8], byte[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = *reinterpret_cast<const uint32_t*>(p.codes + row[j] * p.pitch + from);
#pragma unroll
        for (int j = 0; j < 8; ++j) byte[j] = p.scales[row[j] * (p.pitch / kMxBlock) + from / kMxBlock];
        u32x2 v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const bool in = m0 + j < p.M;
            const float s = scale_of(byte[j]);
            float e[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) e[i] = in ? (float)(int8_t)(w[j] >> (8 * i)) * s : 0.0f;
            // (exact in bfloat16: the upper halves)
            v[j] = u32x2{__builtin_amdgcn_perm(__float_as_uint(e[1]), __float_as_uint(e[0]), 0x07060302u),
                         __builtin_amdgcn_perm(__float_as_uint(e[3]), __float_as_uint(e[2]), 0x07060302u)};
        }
        store_columns(lds, p.x_tiles + b0 * block_bytes + step * 1024, block_bytes, nb, v);
    }
}

struct WgradArgs {
    TileOperand dy, x;
    int stages;
    int splits, per_split;   // parts of the stages, and stages of a part
    int tiles_n, tiles_k, per_xcd;
    int64_t N, K;
    float* dw;
    int64_t ldw;
    int accumulate;
    float* part;             // splits > 1: [split][N][pitch]
    int64_t pitch;
};

// Tiles of 32 RB WR rows x 32 CB WC columns of dW, a workgroup each, for one part of the tokens.  Order of the workgroups as in the
// 4-bit products; the parts of a tile are neighbours in it.
template <int WR, int WC, int RB, int CB, bool FLAT, int PARTS>
__global__ __launch_bounds__(64 * WR * WC, 1) void k_ckpt8_wgrad(WgradArgs p) {
    using Product = TileProduct<WR, WC, RB, CB, false, FLAT, PARTS>;
    extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
    const int64_t b = (int64_t)(blockIdx.x % kXcd) * p.per_xcd + blockIdx.x / kXcd;
    const int64_t t = b / p.splits;
    const int split = (int)(b - t * p.splits);
    if (t >= (int64_t)p.tiles_n * p.tiles_k) return;
    const int64_t band = t / (4 * p.tiles_k);
    const int rest = (int)(t - band * 4 * p.tiles_k), high = min(4, p.tiles_n - (int)band * 4);
    const int tn = (int)band * 4 + rest % high, tk = rest / high;
    constexpr int kPer = kGroupSteps / Product::kSteps;   // the plan's stages are of four steps
    Product prod;
    prod.run(p.dy, p.x, tn * WR * RB, tk * WC * CB, split * p.per_split * kPer, min(p.stages, (split + 1) * p.per_split) * kPer, lds);
    const int wave = threadIdx.x / kWave;
    const int64_t n0 = ((int64_t)tn * WR + wave / WC) * RB * 32, k0 = ((int64_t)tk * WC + wave % WC) * CB * 32;
    float* base = p.splits > 1 ? p.part + split * p.N * p.pitch : p.dw;
    const int64_t ld = p.splits > 1 ? p.pitch : p.ldw;
    const bool add = p.splits == 1 && p.accumulate;
    prod.store(false, lds, [&](int row, int col, u32x4 v) {
        const int64_t n = n0 + row, k = k0 + col;
        if (n >= p.N || k >= p.K) return;
        float* z = base + n * ld + k;
        if (k + 4 <= p.K) {
            u32x4_a4* q = reinterpret_cast<u32x4_a4*>(z);
            if (add) {
                const u32x4_a4 old = *q;
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = __float_as_uint(bits_as<float>(old[i]) + bits_as<float>(v[i]));
            }
            *q = v;
        } else {
#pragma unroll
            for (int i = 0; i < 3; ++i)
                if (k + i < p.K) z[i] = add ? z[i] + bits_as<float>(v[i]) : bits_as<float>(v[i]);
        }
    });
}

// Small products: 64 x 64 results a workgroup for one part of the tokens, its eight waves sharing these, 16 at a time, everything straight
// from memory and the next 16 tokens asked for while some are multiplied: one launch (two with several parts) and no tiles.  A lane reads
// two neighbouring columns of eight tokens of either operand, so the tiles of 32 x 32 it holds are those of even and odd columns.  Its narrow
// loads bound it, at 1.2 us a wave's step (2.0 from fp32): asking two steps ahead took 10 % longer, the scales of a step in one load the same.
struct FewGradArgs {
    const void* dy;
    int64_t lddy;
    const uint8_t* codes;
    const uint8_t* scales;
    int64_t pitch;
    int64_t M, N, K;
    int tiles_k;
    int steps, per_split;    // of 16 tokens
    float* out;              // dW, or the parts
    int64_t ld, split_stride;
    int accumulate;
};
constexpr int kFewWaves = 8, kFewGroups = 256;

template <typename T>
__global__ __launch_bounds__(64 * kFewWaves) void k_ckpt8_wgrad_few(FewGradArgs p) {
    constexpr int kOf = sizeof(T) == 4 ? kParts : 1, kWords = sizeof(T) / 2;
    extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int half = lane / 32, l32 = lane % 32;
    const uint32_t tile = blockIdx.x, tn = tile / (uint32_t)p.tiles_k, tk = tile - tn * (uint32_t)p.tiles_k;
    const int64_t n0 = (int64_t)tn * 64, k0 = (int64_t)tk * 64;
    // (a lane at the last column reads the last two and takes its own; one behind the last is not stored)
    const int64_t cn = n0 + 2 * l32, cn_from = min(cn, p.N - 2), ck = min(k0 + 2 * l32, p.pitch - 2);
    const bool second = cn == p.N - 1;
    const T* dy = static_cast<const T*>(p.dy) + cn_from;
    const uint8_t* codes = p.codes + ck;
    const uint8_t* scales = p.scales + ck / kMxBlock;
    struct Tokens {
        uint32_t y[8][kWords], c[8], s[8];
    };
    auto load = [&](int step, Tokens& o) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int64_t m = min((int64_t)step * 16 + half * 8 + j, p.M - 1);
            if constexpr (sizeof(T) == 4) {
                const u32x2_a4 q = *reinterpret_cast<const u32x2_a4*>(dy + m * p.lddy);
                o.y[j][0] = q[0], o.y[j][1] = q[1];
            } else {
                o.y[j][0] = *reinterpret_cast<const u32_a2*>(dy + m * p.lddy);
            }
            o.c[j] = *reinterpret_cast<const uint16_t*>(codes + m * p.pitch);
            o.s[j] = scales[m * (p.pitch / kMxBlock)];
        }
    };
    v16f acc[2][2], small[kOf > 1 ? 2 : 1][kOf > 1 ? 2 : 1];
#pragma unroll
    for (int a = 0; a < 2; ++a)
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            acc[a][b] = v16f{};
            if constexpr (kOf > 1) small[a][b] = v16f{};
        }
    const int s0 = blockIdx.y * p.per_split, s1 = min(p.steps, s0 + p.per_split);
    Tokens cur, next;
    if (s0 + wave < s1) load(s0 + wave, cur);
    for (int step = s0 + wave; step < s1; step += kFewWaves) {
        const bool more = step + kFewWaves < s1;
        if (more) load(step + kFewWaves, next);
        const int64_t m0 = (int64_t)step * 16 + half * 8;
        if (m0 + 8 > p.M) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const bool in = m0 + j < p.M;
#pragma unroll
                for (int w = 0; w < kWords; ++w) cur.y[j][w] = in ? cur.y[j][w] : 0u;
                cur.s[j] = in ? cur.s[j] : 1u;
                cur.c[j] = in ? cur.c[j] : 0u;
            }
        }
        v4i x[2], y[kOf][2];
        uint32_t xv[2][8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float s = scale_of(cur.s[j]);
            xv[0][j] = __float_as_uint((float)(int8_t)cur.c[j] * s);
            xv[1][j] = __float_as_uint((float)(int8_t)(cur.c[j] >> 8) * s);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
#pragma unroll
            for (int b = 0; b < 2; ++b) x[b][i] = (int)__builtin_amdgcn_perm(xv[b][2 * i + 1], xv[b][2 * i], 0x07060302u);   // (exact: upper halves)
        }
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int j = 0; j < 8; ++j) cur.y[j][0] = second ? cur.y[j][0] >> 16 : cur.y[j][0];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                y[0][0][i] = (int)__builtin_amdgcn_perm(cur.y[2 * i + 1][0], cur.y[2 * i][0], 0x05040100u);
                y[0][1][i] = (int)__builtin_amdgcn_perm(cur.y[2 * i + 1][0], cur.y[2 * i][0], 0x07060302u);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    uint32_t h[2][kParts];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const uint32_t v = b == 0 && second ? cur.y[2 * i + e][1] : cur.y[2 * i + e][b];
                        split3(bits_as<float>(v), h[e][0], h[e][1], h[e][2]);
                    }
#pragma unroll
                    for (int q = 0; q < kOf; ++q) y[q][b][i] = (int)(h[0][q] | (h[1][q] << 16));
                }
        }
#pragma unroll
        for (int a = 0; a < 2; ++a)
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                acc[a][b] = mfma16(x[a], y[0][b], acc[a][b]);
                if constexpr (kOf > 1) {
#pragma unroll
                    for (int q = kOf - 1; q > 0; --q) small[a][b] = mfma16(x[a], y[q][b], small[a][b]);
                }
            }
        if (more) cur = next;
    }
    if constexpr (kOf > 1) {
#pragma unroll
        for (int a = 0; a < 2; ++a)
#pragma unroll
            for (int b = 0; b < 2; ++b) acc[a][b] += small[a][b];
    }
    // The waves' sums meet in LDS, first those of the last four with those of the first four, then these four.  A wave's share: [n][k], 16-byte
    // pieces of a row in the order piece ^ row / 2 % 16.
    auto piece = [&](int w, int row, int at) { return reinterpret_cast<f32x4*>(lds + w * 16384 + row * 256 + ((at ^ (row >> 1)) & 15) * 16); };
    auto each = [&](auto use) {
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int e = 0; e < 2; ++e) use(b, q, e, 2 * l32 + b, q * 4 + half * 2 + e);
    };
    if (wave >= 4)
        each([&](int b, int q, int e, int row, int at) {
            *piece(wave - 4, row, at) = f32x4{acc[0][b][4 * q + 2 * e], acc[1][b][4 * q + 2 * e], acc[0][b][4 * q + 2 * e + 1], acc[1][b][4 * q + 2 * e + 1]};
        });
    __syncthreads();
    if (wave < 4)
        each([&](int b, int q, int e, int row, int at) {
            f32x4* z = piece(wave, row, at);
            *z = f32x4{acc[0][b][4 * q + 2 * e], acc[1][b][4 * q + 2 * e], acc[0][b][4 * q + 2 * e + 1], acc[1][b][4 * q + 2 * e + 1]} + *z;
        });
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int at = i * 512 + threadIdx.x, row = at / 16;
        const int64_t n = n0 + row, k = k0 + (at % 16) * 4;
        if (n >= p.N || k >= p.K) continue;
        f32x4 v = *piece(0, row, at % 16);
#pragma unroll
        for (int w = 1; w < 4; ++w) v += *piece(w, row, at % 16);
        float* z = p.out + blockIdx.y * p.split_stride + n * p.ld + k;
        if (k + 4 <= p.K) {
            u32x4_a4* q = reinterpret_cast<u32x4_a4*>(z);
            if (p.accumulate) v += __builtin_bit_cast(f32x4, (u32x4)*q);
            *q = __builtin_bit_cast(u32x4, v);
        } else {
#pragma unroll
            for (int e = 0; e < 3; ++e)
                if (k + e < p.K) z[e] = p.accumulate ? z[e] + v[e] : v[e];
        }
    }
}

// Sums of the parts, in their order; no parts: zeros.
__global__ __launch_bounds__(256) void k_ckpt8_wgrad_sum(const float* part, int splits, int64_t N, int64_t K, int64_t pitch, float* dw, int64_t ldw,
                                                         int accumulate) {
    const int64_t units = (K + 3) / 4, u = (int64_t)blockIdx.x * 256 + threadIdx.x, n = u / units, k = (u - n * units) * 4;
    if (n >= N) return;
    f32x4 sum = {0, 0, 0, 0};
    const float* from = part + n * pitch + k;
    for (int s0 = 0; s0 < splits; s0 += 8) {   // eight parts asked for at a time
        f32x4 v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = *reinterpret_cast<const f32x4*>(from + min(s0 + i, splits - 1) * N * pitch);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (s0 + i < splits) sum += v[i];
    }
    float* z = dw + n * ldw + k;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (k + i < K) z[i] = accumulate ? z[i] + sum[i] : sum[i];
}

template <int WR, int WC, int RB, int CB, bool FLAT, int PARTS>
daq_status launch_wgrad(WgradArgs p, hipStream_t st) {
    using Product = TileProduct<WR, WC, RB, CB, false, FLAT, PARTS>;
    p.tiles_n = (int)ceil_div(p.dy.blocks, WR * RB);
    p.tiles_k = (int)ceil_div(p.x.blocks, WC * CB);
    const int64_t per = ceil_div((int64_t)p.tiles_n * p.tiles_k * p.splits, kXcd);
    p.per_xcd = (int)per;
    const auto kernel = k_ckpt8_wgrad<WR, WC, RB, CB, FLAT, PARTS>;
    if (!allow_lds((const void*)kernel, Product::kLdsBytes)) return DAQ_ERR_HIP;
    DAQ_LAUNCH("ckpt8_wgrad", st, hipLaunchKernelGGL(kernel, dim3((unsigned)(per * kXcd)), dim3(64 * WR * WC), Product::kLdsBytes, st, p));
    return DAQ_OK;
}

}  // namespace

WgradPlan wgrad_plan(int64_t M, int64_t N, int64_t K, int dtype, int64_t lddy, int dy_misaligned) {
    WgradPlan w{};
    w.n_blocks = (int)ceil_div(N, 32);
    w.k_blocks = (int)ceil_div(K, 32);
    w.steps = (int)(ceil_div(M, kStageM) * kGroupSteps);
    w.parts = dtype == DAQ_BF16 ? 1 : kParts;
    w.pitch = round_up(K, 4);
    // Small products go without tiles while a workgroup to a CU leaves a wave eight steps at most; a part of the tokens has two steps a wave
    // or more, as its sum is a launch (4 us).  us without tiles and with: 64 x 64 x 64 4.5 and 7.9 (fp32 5.1 and 10.2), 1000 x 800 x 600 13.9
    // and 17.6 (20.3 and 25.9), 4096 x 256 x 256 11.7 and 16.1 (13.8 and 26.1), 16384 x 64 x 512 15.6 and 25.1 (20.6 and 30.8); past the
    // rule 1531 x 607 x 1100 30.9 and 29.0 from fp32, 2048 x 1024 x 1024 25.7 and 24.6, 100 x 4000 x 4000 56 and 21.  Two columns are read at a time.
    const int64_t few_tiles = ceil_div(N, 64) * ceil_div(K, 64), few_steps = ceil_div(M, 16);
    if (N >= 2 && few_tiles <= kFewGroups && few_tiles * few_steps <= kFewGroups * kFewWaves * 8) {
        w.few = true;
        w.per_split = (int)ceil_div(few_steps, std::max<int64_t>(1, std::min<int64_t>(kFewGroups / few_tiles, few_steps / (2 * kFewWaves))));
        w.splits = (int)ceil_div(few_steps, w.per_split);
        w.bytes = w.splits > 1 ? round_up((int64_t)w.splits * N * w.pitch * 4, 256) : 0;
        return w;
    }
    // The form and the parts of the tokens that take the least time by what was measured of them (us): a workgroup to a CU, 6 + 1.7 a
    // stage of 64 tokens for tiles of 256 x 256, 3.2 + 0.65 for tiles of 128 x 128 (1.3 with three parts of dY, which have that form
    // only); several parts of the tokens: 3 for their sum, and each part's results written and read at 4 TB/s.  E.g. 2048 x 2048 x 2048
    // 32 us on small tiles, 62 on large ones, 52 on small ones in two parts; 16384 x 8192 x 4096 918 on large ones, 1190 on small ones; 16384 x 4096 x 512
    // 346 in one part, 88 in eight; from fp32 1531 x 607 x 1100 39 in one part, 28.3 in four, 3001 x 610 x 1101 58.5, 33.4 in five.
    const int stages = w.steps / kGroupSteps;
    const double t_part = (double)N * K * 8 / 4e6;
    SplitModel small{stages, ceil_div(w.n_blocks, 4) * ceil_div(w.k_blocks, 4), stages, w.parts > 1 ? 1.3 : 0.65, 3.2, 0.0, 3.0, t_part};
    SplitModel big{stages, ceil_div(w.n_blocks, 8) * ceil_div(w.k_blocks, 8), stages, 1.7, 6.0, 0.0, 3.0, t_part};
    const int s_small = cheapest_split(small), s_big = cheapest_split(big);
    w.big = w.parts == 1 && big.cost(s_big) < small.cost(s_small);
    w.splits = w.big ? s_big : s_small;
    // A bfloat16 dY of whole 16-byte pieces can be read by the products as it is (what they reach of it at a time is within 31 bits): that
    // spares its way into tiles, and the fragments' transposing reads cost the products some, the more the more columns X has.  us with it and
    // without: 16384 x 4096 x 512 88 and 155, 16384 x 8192 x 4096 918 and 919, 4096 x 4096 x 4096 129 and 128, 16384 x 512 x 8192 211 and 213,
    // 16384 x 4096 x 8192 944 and 900; on small tiles 20000 x 704 x 704 51.5 and 59.7, 8192 x 1024 x 1024 38.1 and 41, 2048 x 2048 x 2048 33.3 and
    // 31.9, but 8192 x 512 x 2048 41.8 and 48.3.
    w.flat = dtype == DAQ_BF16 && dy_misaligned == 0 && lddy % 8 == 0 && N % 8 == 0 && lddy < ((int64_t)1 << 24) && K <= (w.big ? 8192 : 1024);
    w.per_split = (int)ceil_div(stages, w.splits);
    w.splits = (int)ceil_div(stages, w.per_split);
    w.off_x = w.flat ? 0 : (int64_t)w.n_blocks * w.steps * w.parts * 1024;
    w.off_part = w.off_x + (int64_t)w.k_blocks * w.steps * 1024;
    w.bytes = w.off_part + (w.splits > 1 ? round_up((int64_t)w.splits * N * w.pitch * 4, 256) : 0);
    return w;
}

}  // namespace daq

using namespace daq;

static daq_status wgrad_size(int64_t M, int64_t N, int64_t K) {
    if (N <= 0) return DAQ_ERR_INVALID_ARG;
    daq_status rc = matrix_size(M, K);
    if (rc == DAQ_OK) rc = matrix_size(M, N);
    if (rc == DAQ_OK) rc = matrix_size(N, K);
    // a row block's tiles are within 32 bits, with three parts of dY too
    if (rc == DAQ_OK && M >= (int64_t)1 << 24) rc = DAQ_ERR_UNSUPPORTED;
    return rc;
}

extern "C" daq_status daq_ckpt8_weight_grad_workspace(int64_t M, int64_t N, int64_t K, daq_dtype dtype, int64_t lddy, int32_t dy_misaligned,
                                                      size_t* bytes) {
    if (!bytes) return DAQ_ERR_INVALID_ARG;
    *bytes = 0;
    if (!dtype_ok(dtype) || dy_misaligned < 0) return DAQ_ERR_INVALID_ARG;
    const daq_status rc = wgrad_size(M, N, K);
    if (rc == DAQ_OK && M > 0) *bytes = (size_t)wgrad_plan(M, N, K, dtype, lddy, dy_misaligned).bytes;
    return rc;
}

extern "C" daq_status daq_ckpt8_weight_grad(int64_t M, int64_t N, int64_t K, const void* dY, daq_dtype dtype, int64_t lddy,
                                            const uint8_t* x_ckpt, float* dW, int64_t ldw, int32_t accumulate, void* workspace,
                                            size_t workspace_bytes, void* stream) {
    if (!dtype_ok(dtype)) return DAQ_ERR_INVALID_ARG;
    daq_status rc = wgrad_size(M, N, K);
    if (rc != DAQ_OK) return rc;
    if (!dW || !elem_aligned(dW, DAQ_FP32) || ldw < K) return DAQ_ERR_INVALID_ARG;
    if (M > 0 && (!dY || !elem_aligned(dY, dtype) || lddy < N || !x_ckpt || !aligned256(x_ckpt))) return DAQ_ERR_INVALID_ARG;
    hipStream_t st = (hipStream_t)stream;
    const int64_t sum_blocks = ceil_div(N * ceil_div(K, 4), 256);
    const bool sum_fits = grid_ok(sum_blocks, 256);
    if (M == 0) {   // a sum of nothing
        if (accumulate) return DAQ_OK;
        if (!sum_fits) return DAQ_ERR_UNSUPPORTED;
        DAQ_LAUNCH("ckpt8_wgrad_sum", st, hipLaunchKernelGGL(k_ckpt8_wgrad_sum, dim3((unsigned)sum_blocks), dim3(256), 0, st, nullptr, 0, N, K, 0, dW, ldw, 0));
        return DAQ_OK;
    }
    const WgradPlan w = wgrad_plan(M, N, K, dtype, lddy, (int)((uintptr_t)dY & 15u));
    if (w.bytes > 0 && (!workspace || workspace_bytes < (size_t)w.bytes || !aligned256(workspace))) return DAQ_ERR_WORKSPACE;
    daq_ckpt8_layout L;
    daq_layout_ckpt8(M, K, 1, &L);
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    if (w.few) {
        const int64_t tiles_k = ceil_div(K, 64), tiles = ceil_div(N, 64) * tiles_k;
        const bool parts = w.splits > 1;
        const FewGradArgs f{dY, lddy, x_ckpt, x_ckpt + L.off_scales, L.pitch, M, N, K, (int)tiles_k, (int)ceil_div(M, 16), w.per_split,
                            parts ? reinterpret_cast<float*>(ws) : dW, parts ? w.pitch : ldw, N * w.pitch, parts ? 0 : accumulate};
        const dim3 grid((unsigned)tiles, (unsigned)w.splits);
        constexpr int kLds = 4 * 16384;
        if (!allow_lds(dtype == DAQ_BF16 ? (const void*)k_ckpt8_wgrad_few<uint16_t> : (const void*)k_ckpt8_wgrad_few<float>, kLds)) return DAQ_ERR_HIP;
        if (dtype == DAQ_BF16) DAQ_LAUNCH("ckpt8_wgrad_few", st, hipLaunchKernelGGL(k_ckpt8_wgrad_few<uint16_t>, grid, dim3(64 * kFewWaves), kLds, st, f));
        else DAQ_LAUNCH("ckpt8_wgrad_few", st, hipLaunchKernelGGL(k_ckpt8_wgrad_few<float>, grid, dim3(64 * kFewWaves), kLds, st, f));
        if (parts)
            DAQ_LAUNCH("ckpt8_wgrad_sum", st,
                       hipLaunchKernelGGL(k_ckpt8_wgrad_sum, dim3((unsigned)sum_blocks), dim3(256), 0, st, f.out, w.splits, N, K, w.pitch, dW, ldw, accumulate));
        return DAQ_OK;
    }
    OrderArgs o{dY, lddy, x_ckpt, x_ckpt + L.off_scales, L.pitch, M, N, ws, ws + w.off_x, w.n_blocks, w.k_blocks, w.steps, 0};
    const int64_t stages = w.steps / kGroupSteps, dy_groups = w.flat ? 0 : stages * ceil_div(w.n_blocks, 4), blocks = dy_groups + stages * ceil_div(w.k_blocks, 4);
    const int64_t edge = w.big ? 8 : 4, tiles = round_up(ceil_div(w.n_blocks, edge) * ceil_div(w.k_blocks, edge) * w.splits, kXcd);
    if (!grid_ok(blocks, 256) || !grid_ok(tiles, w.big ? 512 : 256) || (w.splits > 1 && !sum_fits)) return DAQ_ERR_UNSUPPORTED;
    o.dy_groups = (uint32_t)dy_groups;
    if (dtype == DAQ_BF16) DAQ_LAUNCH("ckpt8_order", st, hipLaunchKernelGGL(k_ckpt8_order<uint16_t>, dim3((unsigned)blocks), dim3(256), 0, st, o));
    else DAQ_LAUNCH("ckpt8_order", st, hipLaunchKernelGGL(k_ckpt8_order<float>, dim3((unsigned)blocks), dim3(256), 0, st, o));
    WgradArgs p{};
    if (w.flat) p.dy = TileOperand{static_cast<const uint8_t*>(dY), nullptr, w.n_blocks, w.steps, lddy * 2, N * 2, M};
    else p.dy = TileOperand{o.dy_tiles, nullptr, w.n_blocks, w.steps * w.parts, 0, 0, 0};
    p.x = TileOperand{o.x_tiles, nullptr, w.k_blocks, w.steps, 0, 0, 0};
    p.stages = w.steps / kGroupSteps;
    p.splits = w.splits;
    p.per_split = w.per_split;
    p.N = N;
    p.K = K;
    p.dw = dW;
    p.ldw = ldw;
    p.accumulate = accumulate;
    p.part = reinterpret_cast<float*>(ws + w.off_part);
    p.pitch = w.pitch;
    if (w.parts > 1) rc = launch_wgrad<2, 2, 2, 2, false, kParts>(p, st);
    else if (w.flat) rc = w.big ? launch_wgrad<4, 2, 2, 4, true, 1>(p, st) : launch_wgrad<2, 2, 2, 2, true, 1>(p, st);
    else rc = w.big ? launch_wgrad<2, 4, 4, 2, false, 1>(p, st) : launch_wgrad<2, 2, 2, 2, false, 1>(p, st);
    if (rc != DAQ_OK || w.splits == 1) return rc;
    DAQ_LAUNCH("ckpt8_wgrad_sum", st,
               hipLaunchKernelGGL(k_ckpt8_wgrad_sum, dim3((unsigned)sum_blocks), dim3(256), 0, st, p.part, w.splits, N, K, w.pitch, dW, ldw, accumulate));
    return DAQ_OK;
}
