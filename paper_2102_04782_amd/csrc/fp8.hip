// Matrices in 8-bit floating point: layout, quantization along rows, along columns and by tiles, and back.
#include <limits>
#include <type_traits>

#include "fp8_block.h"

namespace daq {

namespace {

struct Packed {
    uint8_t* codes;
    uint8_t* scales;
    int64_t rows, pitch;
};
Packed packed(uint8_t* buf, int64_t rows, int64_t cols) {
    if (!buf) return {};
    daq_fp8_layout L;
    daq_layout_fp8(rows, cols, &L);
    return {buf, buf + L.off_scales, rows, L.pitch};
}

// Blocks along the rows.  A wave takes four rows of 512 columns, the columns of a word of scale bytes, eight elements a lane: the 16 lanes of
// a block find its largest magnitude by four exchanges in registers.  Bound: memory; 16384 x 8192 bfloat16 64 us, 6.3 TB/s.
template <typename T, bool PAST>
__global__ __launch_bounds__(256) void k_fp8_rows(const T* src, int64_t ld, int64_t rows, int64_t cols, Packed to, int groups) {
    const int lane = threadIdx.x % kWave;
    const int64_t band = blockIdx.x / groups;
    const int g = (int)(blockIdx.x - band * groups);
    const int64_t r0 = band * 16 + threadIdx.x / kWave * 4, c = (int64_t)g * kFp8Group + lane * 8, left = cols - c;
    Eight<T> v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const T* from = src + (r0 + i) * ld + c;
        if (r0 + i < rows && left >= 8) load8<PAST>(from, v[i]);
        else load8(from, r0 + i < rows ? (int)max(left, (int64_t)0) : 0, v[i]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (r0 + i >= rows) break;
        uint32_t byte = fp8_scale_byte(max16(top_of(v[i])));
        if (c < to.pitch) *reinterpret_cast<u32x2*>(to.codes + (r0 + i) * to.pitch + c) = codes8(v[i], byte);
        if (c >= to.pitch) byte = 0;
        const uint32_t word = (uint32_t)__builtin_amdgcn_readlane((int)byte, 0) | (uint32_t)__builtin_amdgcn_readlane((int)byte, 16) << 8 |
                              (uint32_t)__builtin_amdgcn_readlane((int)byte, 32) << 16 | (uint32_t)__builtin_amdgcn_readlane((int)byte, 48) << 24;
        if (lane == 0) *reinterpret_cast<uint32_t*>(to.scales + ((int64_t)g * to.rows + r0 + i) * 4) = word;
    }
}

struct TileArgs {
    int64_t ld, stride;      // stride: from matrix to matrix
    int64_t rows, cols;      // of one matrix of src; experts: of the rows that the order takes from
    int col_tiles;
    int64_t row_tiles;       // of one matrix
    Packed r, c;             // by rows, by columns; codes NULL: not wanted
    // experts: tile b of the order has rows of one expert only, row p of the order is row rows[p] / picks of src, or (picks == 0) row p
    const int32_t* table;
    const int32_t* order;
    int experts, picks;
};
enum class Tiles { kBlocks, kWeights, kExperts };

// Tiles of 128 x 128 of src, which is read once: blocks along the rows and / or along the columns, or (weights) the tile as one block,
// written both ways.  A lane has eight columns of four rows, a wave 128 columns of 16 rows; codes that leave by columns are words
// of four rows each and turn in LDS, where word q of a column lies at q ^ (4 * (column / 8 % 8)), off its neighbours' banks.  Bound: memory, written in
// pieces of 128 bytes; 8192 x 8192 both ways, bfloat16 45 us, 6.0 TB/s (62 between the products of a training step), fp32 78, 5.2; as weights 44 and 82; 32 weights of 2048 x 2048
// 103, 5.2 TB/s, and 151, 5.3; 65536 x 2048 bfloat16 in the order of 32 experts 87, 6.2, taken by their tokens 65.  Neighbours in bands
// of row tiles, so that these pieces lie together by columns too, gained 7 % at 16384 x 8192 and lost 4 % at 8192 x 8192.
template <typename T, Tiles KIND, bool BYROWS, bool BYCOLS, bool PAST>
__global__ __launch_bounds__(512) void k_fp8_tiles(const T* src, TileArgs p) {
    constexpr int W = Eight<T>::kWords;
    constexpr bool kWeights = KIND == Tiles::kWeights, kExperts = KIND == Tiles::kExperts;
    __shared__ uint32_t turned[BYCOLS ? 128 * 32 : 1];
    __shared__ __attribute__((aligned(16))) uint32_t tops[8][16][W];
    __shared__ __attribute__((aligned(16))) uint8_t column_bytes[128];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, piece = lane % 16, quad = wave * 4 + lane / 16;
    const int64_t rt = blockIdx.x / p.col_tiles;
    const int64_t c0 = (int64_t)(blockIdx.x - rt * p.col_tiles) * 128, c = c0 + piece * 8;
    const int64_t mat = kWeights ? rt / p.row_tiles : 0, rb = kWeights ? rt - mat * p.row_tiles : rt;   // rb: block along the columns
    int64_t r0 = rb * 128;
    int64_t rows = p.rows;                                // rows of src, or of the order, that this tile may take, from 0 on
    bool ordered = true;
    if constexpr (kExperts) {
        const int32_t* tiles = p.table + kTable128 * (p.experts + 1);
        if (rt < tiles[p.experts]) {
            const int e = expert_of_tile(tiles, p.experts, (int)rt, lane);
            r0 = p.table[e] + (rt - tiles[e]) * 128;
            rows = p.table[e + 1];
        } else {                                          // by rows only: those behind the last of the order
            r0 = p.table[p.experts] + (rt - tiles[p.experts]) * 128;
            if (!BYROWS || r0 >= rows) return;
            ordered = false;
        }
    }
    Eight<T> v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        int64_t r = r0 + quad * 4 + i;
        const bool in = r < rows;
        if constexpr (kExperts) {
            if (p.picks) r = in ? p.order[r] / p.picks : 0;
        }
        const T* from = src + mat * p.stride + r * p.ld + c;
        const int64_t left = in ? p.cols - c : 0;
        if (left >= 8) load8<PAST>(from, v[i]);
        else load8(from, (int)max(left, (int64_t)0), v[i]);
    }
    uint32_t m[W];                                        // the largest of each column (pair of columns)
#pragma unroll
    for (int j = 0; j < W; ++j) {
        m[j] = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) m[j] = larger((const T*)nullptr, m[j], v[i].w[j]);
    }
    uint32_t whole = 0;
    if constexpr (kWeights) {
        uint32_t t = 0;
#pragma unroll
        for (int j = 0; j < W; ++j) t = max(t, top_bits((const T*)nullptr, m[j]));
        t = max16(t);
        t = max(t, (uint32_t)__shfl_xor((int)t, 16));
        t = max(t, (uint32_t)__shfl_xor((int)t, 32));
        if (lane == 0) tops[wave][0][0] = t;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < 8; ++w) whole = max(whole, tops[w][0][0]);
        whole = fp8_scale_byte(whole);
    } else if constexpr (BYCOLS) {
#pragma unroll
        for (int j = 0; j < W; ++j) {
            m[j] = larger((const T*)nullptr, m[j], (uint32_t)__shfl_xor((int)m[j], 16));
            m[j] = larger((const T*)nullptr, m[j], (uint32_t)__shfl_xor((int)m[j], 32));
            if (lane < 16) tops[wave][piece][j] = m[j];
        }
        __syncthreads();
        // a thread a column: its scale byte
        if (threadIdx.x < 128) {
            const int col = threadIdx.x;
            uint32_t t = 0;
#pragma unroll
            for (int w = 0; w < 8; ++w) t = larger((const T*)nullptr, t, tops[w][col / 8][col % 8 * W / 8]);
            const uint32_t byte = fp8_scale_byte(sizeof(T) == 4 ? t : (col & 1) ? t & 0xFFFF0000u : t << 16);
            column_bytes[col] = (uint8_t)byte;
            if (ordered && c0 + col < p.cols) {
                uint8_t* s = p.c.scales + ((rb / 4) * p.c.rows + mat * p.cols + c0 + col) * 4;
                s[rb % 4] = (uint8_t)byte;
                if (!kExperts && (rb + 1) * 128 >= p.rows)
                    for (int b = (int)(rb % 4) + 1; b < 4; ++b) s[b] = 0;
            }
        }
    }
    if constexpr (BYROWS) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t r = r0 + quad * 4 + i, at = mat * p.rows + r;
            const uint32_t byte = kWeights ? whole : fp8_scale_byte(max16(top_of(v[i])));
            if (r >= rows) continue;
            *reinterpret_cast<u32x2*>(p.r.codes + at * p.r.pitch + c) = codes8(v[i], byte);
            if (piece == 0) {
                const int64_t cb = c0 / 128;
                uint8_t* s = p.r.scales + ((cb / 4) * p.r.rows + at) * 4;
                s[cb % 4] = (uint8_t)byte;
                if (c0 + 128 >= p.cols)
                    for (int b = (int)(cb % 4) + 1; b < 4; ++b) s[b] = 0;
            }
        }
    }
    if constexpr (BYCOLS) {
        if (!ordered) return;
        u32x2 bytes = {whole * 0x01010101u, whole * 0x01010101u};      // of the lane's columns
        if constexpr (!kWeights) {
            __syncthreads();
            bytes = *reinterpret_cast<const u32x2*>(column_bytes + piece * 8);
        } else if (threadIdx.x < 128 && c0 + threadIdx.x < p.cols) {
            uint8_t* s = p.c.scales + ((rb / 4) * p.c.rows + mat * p.cols + c0 + threadIdx.x) * 4;
            s[rb % 4] = (uint8_t)whole;
            if ((rb + 1) * 128 >= p.rows)
                for (int b = (int)(rb % 4) + 1; b < 4; ++b) s[b] = 0;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
            turned[(piece * 8 + j) * 32 + (quad ^ ((piece & 7) * 4))] = codes_down(v, j, bytes[j / 4] >> (8 * (j % 4)) & 255u);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int col = threadIdx.x / 8 + i * 64, chunk = threadIdx.x % 8;
            if (c0 + col >= p.cols) break;
            const u32x4 q = *reinterpret_cast<const u32x4*>(turned + col * 32 + (chunk ^ (col / 8 % 8)) * 4);
            *reinterpret_cast<u32x4*>(p.c.codes + (mat * p.cols + c0 + col) * p.c.pitch + rb * 128 + chunk * 16) = q;
        }
    }
}

// Large sources whose rows begin with a line are read past the caches, which then hold more of the codes, for the products that follow too (all of a layer of 8192 outputs at
// 16384 x 8192 793 us instead of 825), until the codes themselves are more than the caches hold.  us without and with it, bfloat16:
//   both ways   8192 x 8192 44 and 46, 12288 x 8192 80 and 65, 16384 x 8192 115 and 88, 18432 x 8192 119 and 109, 20480 x 8192 134 and 132, 22528 x 8192 146 and 146, 24576 x 8192 158
//               and 158, 16384 x 16384 233 and 254, 65536 x 8192 428 and 445; in the order of 32 experts 65536 x 2048 114 and 86, 40960 x 4096 134 and 135, 65536 x 4096 214 and 218
//   by columns  8192 x 8192 31 and 36, 16384 x 8192 96 and 69, 16384 x 16384 196 and 145, 24576 x 16384 244 and 241, 57344 x 8192 274 and 275, 65536 x 8192 326 and 353
//   by rows     8192 x 8192 32 and 34, 16384 x 8192 69 and 64, 16384 x 16384 134 and 118, 65536 x 8192 263 and 257
// fp32 in tiles no difference, by rows 12288 x 8192 91 and 88, 65536 x 8192 493 and 490.  Where lines are shared between pieces they would be read twice (30000 x 5000: 136 and 122).
constexpr int64_t kMi = (int64_t)1 << 20, kPastFrom = 96 * kMi, kPastBoth = 160 * kMi, kPastColumns = 384 * kMi;
bool past_caches(const void* src, int64_t rows, int64_t cols, int64_t ld, int64_t size, int64_t end) {
    return rows * cols >= kPastFrom && rows * cols < end && (uintptr_t)src % 128 == 0 && ld * size % 128 == 0;
}

template <typename T, Tiles KIND, bool PAST>
daq_status launch_tiles(const T* src, const TileArgs& p, int64_t tiles, hipStream_t st) {
    const dim3 grid((unsigned)(tiles * p.col_tiles));
    auto kernel = p.r.codes ? k_fp8_tiles<T, KIND, true, true, PAST> : k_fp8_tiles<T, KIND, false, true, PAST>;
    if constexpr (KIND == Tiles::kWeights)      // (the others by rows alone: k_fp8_rows)
        if (!p.c.codes) kernel = k_fp8_tiles<T, KIND, true, false, PAST>;
    DAQ_LAUNCH("fp8_tiles", st, hipLaunchKernelGGL(kernel, grid, dim3(512), 0, st, src, p));
    return DAQ_OK;
}
template <Tiles KIND>
daq_status launch_tiles(const void* src, int dtype, const TileArgs& p, int64_t tiles, hipStream_t st) {
    if (dtype == DAQ_FP32) return launch_tiles<float, KIND, false>(static_cast<const float*>(src), p, tiles, st);
    if constexpr (KIND != Tiles::kWeights)      // (rows that several experts take are read again)
        if (p.picks == 0 && past_caches(src, p.rows, p.cols, p.ld, 2, p.r.codes ? kPastBoth : kPastColumns)) return launch_tiles<uint16_t, KIND, true>(static_cast<const uint16_t*>(src), p, tiles, st);
    return launch_tiles<uint16_t, KIND, false>(static_cast<const uint16_t*>(src), p, tiles, st);
}

// Eight columns of a row a lane.  Bound: memory; 8192 x 8192 to bfloat16 38 us, 5.3 TB/s, to fp32 63, 5.4.
template <typename T>
__global__ __launch_bounds__(256) void k_fp8_values(const uint8_t* codes, const uint8_t* scales, int64_t pitch, int64_t rows, int64_t cols, T* dst, int64_t ld) {
    const int64_t strips = (cols + 2047) / 2048, r = blockIdx.x / strips, c = (blockIdx.x - r * strips) * 2048 + threadIdx.x * 8;
    if (c >= cols) return;
    const float s = scale_of(scales[((c / kFp8Group) * rows + r) * 4 + (c / kFp8Block) % 4]);
    const u32x2 q = *reinterpret_cast<const u32x2*>(codes + r * pitch + c);
    float v[8];
#pragma unroll
    for (int d = 0; d < 2; ++d) {
        v[4 * d] = __builtin_amdgcn_cvt_f32_fp8((int)q[d], 0) * s;
        v[4 * d + 1] = __builtin_amdgcn_cvt_f32_fp8((int)q[d], 1) * s;
        v[4 * d + 2] = __builtin_amdgcn_cvt_f32_fp8((int)q[d], 2) * s;
        v[4 * d + 3] = __builtin_amdgcn_cvt_f32_fp8((int)q[d], 3) * s;
    }
    store8(dst + r * ld + c, (int)min(cols - c, (int64_t)8), v);
}

daq_status source_check(const void* src, int dtype, int64_t cols, int64_t ld) {
    return src && elem_aligned(src, dtype) && ld >= cols ? DAQ_OK : DAQ_ERR_INVALID_ARG;
}

}  // namespace

template <typename T, bool PAST>
static daq_status launch_rows(const void* src, int64_t rows, int64_t cols, int64_t ld, const Packed& to, hipStream_t st) {
    const int64_t groups = ceil_div(cols, kFp8Group);
    const dim3 grid((unsigned)(ceil_div(rows, 16) * groups));
    const auto kernel = k_fp8_rows<T, PAST>;
    DAQ_LAUNCH("fp8_rows", st, hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, static_cast<const T*>(src), ld, rows, cols, to, (int)groups));
    return DAQ_OK;
}
daq_status fp8_quantize_rows(const void* src, int dtype, int64_t rows, int64_t cols, int64_t ld, uint8_t* dst, hipStream_t st) {
    const Packed to = packed(dst, rows, cols);
    const bool past = past_caches(src, rows, cols, ld, dtype == DAQ_BF16 ? 2 : 4, std::numeric_limits<int64_t>::max());
    if (dtype == DAQ_BF16) return past ? launch_rows<uint16_t, true>(src, rows, cols, ld, to, st) : launch_rows<uint16_t, false>(src, rows, cols, ld, to, st);
    return past ? launch_rows<float, true>(src, rows, cols, ld, to, st) : launch_rows<float, false>(src, rows, cols, ld, to, st);
}

}  // namespace daq

using namespace daq;

extern "C" daq_status daq_layout_fp8(int64_t rows, int64_t cols, daq_fp8_layout* out) {
    if (!out || rows < 0 || cols < 0) return DAQ_ERR_INVALID_ARG;
    const daq_status rc = matrix_size(rows, cols > 0 ? cols : 1);
    if (rc != DAQ_OK) return rc;
    out->pitch = round_up(cols, kFp8Block);
    out->off_scales = round_up(rows * out->pitch, 256);
    out->bytes = out->off_scales + round_up(ceil_div(cols, kFp8Group) * rows * 4, 256);
    return DAQ_OK;
}

extern "C" daq_status daq_fp8_quantize(const void* src, daq_dtype dtype, int64_t rows, int64_t cols, int64_t ld, uint8_t* by_rows,
                                       uint8_t* by_columns, void* stream) {
    if (!dtype_ok(dtype)) return DAQ_ERR_INVALID_ARG;
    daq_status rc = matrix_size(rows, cols);
    if (rc == DAQ_OK && by_columns) rc = matrix_size(cols, rows > 0 ? rows : 1);
    if (rc != DAQ_OK) return rc;
    if (rows == 0) return DAQ_OK;
    if ((!by_rows && !by_columns) || !aligned256(by_rows) || !aligned256(by_columns)) return DAQ_ERR_INVALID_ARG;
    rc = source_check(src, dtype, cols, ld);
    if (rc != DAQ_OK) return rc;
    hipStream_t st = (hipStream_t)stream;
    if (!by_columns) {
        if (!fp8_rows_grid_ok(rows, cols)) return DAQ_ERR_UNSUPPORTED;
        return fp8_quantize_rows(src, dtype, rows, cols, ld, by_rows, st);
    }
    TileArgs p{ld, 0, rows, cols, (int)ceil_div(cols, 128), ceil_div(rows, 128), packed(by_rows, rows, cols), packed(by_columns, cols, rows), nullptr, nullptr, 0, 0};
    if (!grid_ok(p.row_tiles * p.col_tiles, 512)) return DAQ_ERR_UNSUPPORTED;
    return launch_tiles<Tiles::kBlocks>(src, dtype, p, p.row_tiles, st);
}

extern "C" daq_status daq_fp8_quantize_weights(const void* src, daq_dtype dtype, int64_t count, int64_t rows, int64_t cols, int64_t ld,
                                               int64_t stride, uint8_t* dst, uint8_t* dst_t, void* stream) {
    if (!dtype_ok(dtype) || count < 0 || rows <= 0) return DAQ_ERR_INVALID_ARG;
    daq_status rc = matrix_size(rows, cols);
    if (rc != DAQ_OK) return rc;
    constexpr int64_t most = ((int64_t)1 << 31) - 1;
    if (count > most / std::max(rows, cols) || (count > 0 && rows * cols > kMaxElems / count)) return DAQ_ERR_UNSUPPORTED;
    if (count == 0) return DAQ_OK;
    if ((!dst && !dst_t) || !aligned256(dst) || !aligned256(dst_t) || stride < 0) return DAQ_ERR_INVALID_ARG;
    rc = source_check(src, dtype, cols, ld);
    if (rc != DAQ_OK) return rc;
    TileArgs p{ld, stride, rows, cols, (int)ceil_div(cols, 128), ceil_div(rows, 128), packed(dst, count * rows, cols), packed(dst_t, count * cols, rows), nullptr, nullptr, 0, 0};
    if (!grid_ok(count * p.row_tiles * p.col_tiles, 512)) return DAQ_ERR_UNSUPPORTED;
    return launch_tiles<Tiles::kWeights>(src, dtype, p, count * p.row_tiles, (hipStream_t)stream);
}

extern "C" daq_status daq_fp8_dequantize(const uint8_t* src, int64_t rows, int64_t cols, void* dst, daq_dtype dtype, int64_t ld, void* stream) {
    if (!dtype_ok(dtype) || rows < 0 || cols < 0) return DAQ_ERR_INVALID_ARG;
    const daq_status rc = matrix_size(rows, cols > 0 ? cols : 1);
    if (rc != DAQ_OK) return rc;
    if (rows == 0 || cols == 0) return DAQ_OK;
    if (!src || !aligned256(src) || !dst || !elem_aligned(dst, dtype) || ld < cols) return DAQ_ERR_INVALID_ARG;
    const int64_t blocks = rows * ceil_div(cols, 2048);
    if (!grid_ok(blocks, 256)) return DAQ_ERR_UNSUPPORTED;
    const Packed q = packed(const_cast<uint8_t*>(src), rows, cols);
    if (dtype == DAQ_BF16)
        DAQ_LAUNCH("fp8_values", (hipStream_t)stream, hipLaunchKernelGGL(k_fp8_values<uint16_t>, dim3((unsigned)blocks), dim3(256), 0, (hipStream_t)stream, q.codes, q.scales, q.pitch, rows, cols, static_cast<uint16_t*>(dst), ld));
    else
        DAQ_LAUNCH("fp8_values", (hipStream_t)stream, hipLaunchKernelGGL(k_fp8_values<float>, dim3((unsigned)blocks), dim3(256), 0, (hipStream_t)stream, q.codes, q.scales, q.pitch, rows, cols, static_cast<float*>(dst), ld));
    return DAQ_OK;
}

extern "C" daq_status daq_experts_columns(int64_t tokens, int32_t picks, int32_t experts, int64_t* columns) {
    const daq_experts p{tokens, picks, experts, nullptr, nullptr, nullptr};
    if (!columns || tokens < 0 || picks <= 0 || experts <= 0) return DAQ_ERR_INVALID_ARG;
    if (experts > kMaxExperts || tokens >= kMaxSlots / picks) return DAQ_ERR_UNSUPPORTED;
    *columns = most_tiles(p, 128) * 128;
    return DAQ_OK;
}

extern "C" daq_status daq_experts_quantize(const daq_experts* plan, const void* src, daq_dtype dtype, int64_t cols, int64_t ld, int32_t sorted,
                                           uint8_t* by_rows, uint8_t* by_columns, void* stream) {
    if (!plan_ok(plan) || !dtype_ok(dtype)) return DAQ_ERR_INVALID_ARG;
    const int64_t rows = sorted ? plan_slots(*plan) : plan->tokens, columns = most_tiles(*plan, 128) * 128;
    daq_status rc = matrix_size(rows, cols);
    if (rc == DAQ_OK && by_columns) rc = matrix_size(cols, columns > 0 ? columns : 1);
    if (rc != DAQ_OK) return rc;
    if (rows == 0) return DAQ_OK;
    if ((!by_rows && !by_columns) || !aligned256(by_rows) || !aligned256(by_columns)) return DAQ_ERR_INVALID_ARG;
    rc = source_check(src, dtype, cols, ld);
    if (rc != DAQ_OK) return rc;
    const int64_t tiles = columns / 128, col_tiles = ceil_div(cols, 128);
    if ((by_rows && !fp8_rows_grid_ok(rows, cols)) || (by_columns && !grid_ok((tiles + 1) * col_tiles, 512))) return DAQ_ERR_UNSUPPORTED;
    hipStream_t st = (hipStream_t)stream;
    // rows in their order are read once for both; those that several experts take are quantized by rows on their own.  (One tile more than the order needs at
    // the most: with those that it leaves over they hold the rows behind its last.)
    const bool both = by_rows && by_columns && sorted;
    if (by_rows && !both) rc = fp8_quantize_rows(src, dtype, rows, cols, ld, by_rows, st);
    if (rc != DAQ_OK || !by_columns) return rc;
    TileArgs p{ld, 0, rows, cols, (int)col_tiles, tiles, packed(both ? by_rows : nullptr, rows, cols), packed(by_columns, cols, columns), plan->table, plan->rows, plan->experts, sorted ? 0 : plan->picks};
    return launch_tiles<Tiles::kExperts>(src, dtype, p, tiles + both, st);
}
