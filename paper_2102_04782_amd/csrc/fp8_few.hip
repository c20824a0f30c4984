// Products of 8-bit floating point matrices for few rows of A: what counts is the way of the weights.
//
// A workgroup's eight waves share the blocks of 128 of the summed axis among 1, 2, 4 or 8 of them, four blocks or more each where there are so many, and
// take 16 columns of D with each such set of waves, and up to 64 rows; what a wave needs of four blocks (three, in bfloat16) is asked for at once, and their sums meet in LDS.
// The matrix instruction is that of 16 x 16 x 128 (a block), in bfloat16 four of 16 x 16 x 32: lane l has row l % 16 and the 16-byte pieces l / 16 and
// l / 16 + 4 of a block, so that a load takes 64 bytes in a row of every row.  Where the rows are few they are quantized by every workgroup itself, into
// LDS, while its first weights are on their way: a launch less.
// Bound: memory, and at this size the wait for the first of it.  1 x 8192 x 4096 (33.8 MB) 8.4 us, 4.0 TB/s, quantized on the way, 10.1 with the weights from memory
// (in two launches 10.9 and 13.0); 21 x 2300 x 5130, fp32, 10.2 us behind 3.5 for the rows.
#include "fp8_product.h"

namespace daq {

namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
constexpr int kFewWaves = 8;

template <typename X, bool EXACT, Of OF>
__global__ __launch_bounds__(64 * kFewWaves, 4) void k_fp8_few(ProductArgs p, const X* x, int64_t ldx, int64_t K, int share) {
    constexpr bool kRaw = !std::is_void_v<X>;
    constexpr int kAhead = EXACT ? 3 : 4;                // (conversions take registers)
    extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
    __shared__ int taken[64];                            // rows of A of this tile
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), r = lane % 16, q = lane / 16;
    int64_t m0 = (int64_t)blockIdx.y * 64, m_end = p.M;
    int64_t b_first = 0;
    if constexpr (OF == Of::kExpertRows) {
        const int32_t* tiles = p.table + kTable64 * (p.experts + 1);
        if ((int)blockIdx.y >= tiles[p.experts]) return;
        const int e = expert_of_tile(tiles, p.experts, (int)blockIdx.y, lane);
        m0 = p.table[e] + ((int)blockIdx.y - tiles[e]) * 64;
        m_end = p.table[e + 1];
        b_first = (int64_t)e * p.N;
    }
    const int rows = __builtin_amdgcn_readfirstlane((int)min(m_end - m0, (int64_t)64)), tiles_m = (rows + 15) / 16;
    const int sets = kFewWaves / share, set = wave / share, turn = wave - set * share;      // of waves that share the summed axis
    const int64_t n0 = (int64_t)blockIdx.x * sets * 16, n = b_first + min(n0 + set * 16 + r, p.N - 1);      // (columns behind the last repeat it; they are not stored)
    const uint8_t* b = p.b.codes + n * p.b.pitch + q * 16;
    const uint8_t* sb = p.b.scales + n * 4;
    const int per = (p.stages + share - 1) / share, s0 = turn * per, s1 = min(s0 + per, p.stages);
    struct Block {
        v4i lo, hi;
        int scale;
    };
    auto load = [&](const uint8_t* codes, const uint8_t* scales, int64_t pitch_words, int s) {
        Block o;
        o.lo = *reinterpret_cast<const v4i*>(codes + (int64_t)s * 128);
        o.hi = *reinterpret_cast<const v4i*>(codes + (int64_t)s * 128 + 64);
        o.scale = scales[(int64_t)(s / 4) * pitch_words + s % 4];
        return o;
    };
    Block vb[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
        if (s0 + i < s1) vb[i] = load(b, sb, p.b.rows * 4, s0 + i);
    // where a row of A lies
    int64_t a_row[4];
    auto row_at = [&](int m) -> int64_t {
        const int64_t at = m0 + min(m, rows - 1);
        if constexpr (OF == Of::kExpertRows) return p.picks ? p.order[at] / p.picks : at;
        return at;
    };
    const int pitch = p.stages * 128;                    // raw: of a row in LDS, its pieces of a block in the order piece ^ row % 8
    uint8_t* const bytes = lds + rows * pitch;           // raw: scale bytes [row][stage]
    if constexpr (kRaw) {
        if ((int)threadIdx.x < rows) taken[threadIdx.x] = (int)row_at(threadIdx.x);
        __syncthreads();
        const int per_row = p.stages * 16;               // lanes of a row
        for (int i = threadIdx.x; i < rows * per_row; i += 64 * kFewWaves) {
            const int m = i / per_row, c = (i - m * per_row) * 8;
            Eight<X> v;
            const X* from = x + (int64_t)taken[m] * ldx + c;
            if (c + 8 <= K) load8(from, v);
            else load8(from, (int)max(K - c, (int64_t)0), v);
            const uint32_t byte = fp8_scale_byte(max16(top_of(v)));
            *reinterpret_cast<u32x2*>(lds + m * pitch + c / 128 * 128 + ((c / 16 % 8) ^ (m & 7)) * 16 + c % 16) = codes8(v, byte);
            if ((threadIdx.x & 15) == 0) bytes[m * p.stages + c / 128] = (uint8_t)byte;
        }
        __syncthreads();
    } else {
#pragma unroll
        for (int t = 0; t < 4; ++t) a_row[t] = row_at(t * 16 + r);
    }
    v4f acc[4] = {};
    for (int s = s0; s < s1; s += kAhead) {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            if (t >= tiles_m) break;
            Block va[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                if (s + i >= s1) break;
                if constexpr (kRaw) {
                    const int m = min(t * 16 + r, rows - 1);
                    const uint8_t* at = lds + m * pitch + (s + i) * 128;
                    va[i].lo = *reinterpret_cast<const v4i*>(at + (q ^ (m & 7)) * 16);
                    va[i].hi = *reinterpret_cast<const v4i*>(at + ((q + 4) ^ (m & 7)) * 16);
                    va[i].scale = bytes[m * p.stages + s + i];
                } else {
                    va[i] = load(p.a.codes + a_row[t] * p.a.pitch + q * 16, p.a.scales + a_row[t] * 4, p.a.rows * 4, s + i);
                }
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                if (s + i >= s1) break;
                const v8i w = __builtin_shufflevector(vb[i].lo, vb[i].hi, 0, 1, 2, 3, 4, 5, 6, 7), a = __builtin_shufflevector(va[i].lo, va[i].hi, 0, 1, 2, 3, 4, 5, 6, 7);
                if constexpr (EXACT) {
                    const float sw = scale_of((uint32_t)vb[i].scale), sa = scale_of((uint32_t)va[i].scale);
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, in_bf16(w[2 * k], w[2 * k + 1], sw)),
                                                                         __builtin_bit_cast(v8bf, in_bf16(a[2 * k], a[2 * k + 1], sa)), acc[t], 0, 0, 0);
                } else {
                    acc[t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, a, acc[t], 0, 0, 0, vb[i].scale, 0, va[i].scale);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            if (s + kAhead + i < s1) vb[i] = load(b, sb, p.b.rows * 4, s + kAhead + i);
    }
    // the waves' sums, in the waves' order
    __syncthreads();
    float* sums = reinterpret_cast<float*>(lds);         // [wave][row][16 columns]
#pragma unroll
    for (int t = 0; t < 4; ++t)
        if (t < tiles_m) *reinterpret_cast<v4f*>(sums + ((wave * tiles_m + t) * 16 + r) * 16 + q * 4) = acc[t];
    __syncthreads();
    for (int i = threadIdx.x; i < rows * sets * 4; i += 64 * kFewWaves) {
        const int m = i / (sets * 4), c = (i - m * sets * 4) * 4;
        if (n0 + c >= p.N) continue;
        v4f v = {};
        for (int w = 0; w < share; ++w) v += *reinterpret_cast<const v4f*>(sums + ((c / 16 * share + w) * tiles_m * 16 + m) * 16 + c % 16);
        const int64_t at = (m0 + m) * p.ldd + n0 + c;
        const int left = (int)min(p.N - n0 - c, (int64_t)4);
        if (p.bf16) {
            uint16_t* z = static_cast<uint16_t*>(p.d) + at;
            const u32x2_a2 o = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
            if (left == 4) *reinterpret_cast<u32x2_a2*>(z) = o;
            else
                for (int e = 0; e < left; ++e) z[e] = (uint16_t)(o[e / 2] >> (16 * (e & 1)));
        } else {
            float* z = static_cast<float*>(p.d) + at;
            if (left == 4 && !p.accumulate) *reinterpret_cast<u32x4_a4*>(z) = __builtin_bit_cast(u32x4, v);
            else
                for (int e = 0; e < left; ++e) z[e] = p.accumulate ? z[e] + v[e] : v[e];
        }
    }
}

// Waves that share the summed axis: four blocks each, but more of them where the columns do not fill the CUs.
int few_share(const ProductArgs& p, int64_t tiles) {
    int share = 8;
    while (share > 1 && p.stages <= share * 2 && ceil_div(p.N, 16 * (kFewWaves / share)) * tiles >= 512) share /= 2;
    return share;
}

template <typename X, bool EXACT, Of OF>
daq_status launch(const ProductArgs& p, int64_t tiles, int64_t most_rows, const X* x, int64_t ldx, int64_t K, hipStream_t st) {
    const size_t sums = (size_t)kFewWaves * round_up(most_rows, 16) * 64, raw = std::is_void_v<X> ? 0 : (size_t)most_rows * p.stages * 129, bytes = std::max(sums, raw);
    const auto kernel = k_fp8_few<X, EXACT, OF>;
    if (!allow_lds((const void*)kernel, bytes)) return DAQ_ERR_HIP;
    const int share = few_share(p, tiles);
    DAQ_LAUNCH("fp8_few", st, hipLaunchKernelGGL(kernel, dim3((unsigned)ceil_div(p.N, 16 * (kFewWaves / share)), (unsigned)tiles), dim3(64 * kFewWaves), bytes, st, p, x, ldx, K, share));
    return DAQ_OK;
}
template <bool EXACT, Of OF>
daq_status launch(const ProductArgs& p, int64_t tiles, int64_t most_rows, const void* x, int x_dtype, int64_t ldx, int64_t K, hipStream_t st) {
    if (!x) return launch<void, EXACT, OF>(p, tiles, most_rows, nullptr, 0, K, st);
    return x_dtype == DAQ_BF16 ? launch<uint16_t, EXACT, OF>(p, tiles, most_rows, static_cast<const uint16_t*>(x), ldx, K, st)
                               : launch<float, EXACT, OF>(p, tiles, most_rows, static_cast<const float*>(x), ldx, K, st);
}

}  // namespace

daq_status fp8_few(Of of, const ProductArgs& p, int64_t tiles, int64_t most_rows, const void* x, int x_dtype, int64_t ldx, int64_t K, hipStream_t st) {
    if (of == Of::kExpertRows)
        return p.bf16 ? launch<false, Of::kExpertRows>(p, tiles, most_rows, x, x_dtype, ldx, K, st) : launch<true, Of::kExpertRows>(p, tiles, most_rows, x, x_dtype, ldx, K, st);
    return p.bf16 ? launch<false, Of::kWhole>(p, tiles, most_rows, x, x_dtype, ldx, K, st) : launch<true, Of::kWhole>(p, tiles, most_rows, x, x_dtype, ldx, K, st);
}

}  // namespace daq
