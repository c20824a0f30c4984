// Large products of 8-bit floating point matrices: results in bfloat16, tiles of 256 x 256, one workgroup to a CU that goes from tile to tile.
#include "fp8_product.h"

namespace daq {

namespace {

constexpr int kEdge = 256, kWaves = 4, kB = 4;              // a wave has 128 x 128 results, kB x kB tiles of 32 x 32
constexpr int kCodes = 2 * kEdge * 128, kStage = kCodes + 2 * kEdge * 4;   // bytes of a stage of 128, its scale words behind the codes
constexpr int kLds = 2 * kStage + kWaves * 4096;            // two stages, and a wave's rows of results on their way out
constexpr int kAsks = 18;                                   // requests of a wave for a stage: 128 rows of one operand, eight at a time, and their scale words
constexpr int kStores = kB * kB / 2 * 4;                    // of a wave, of a whole tile
constexpr int kPlaces = kB * kB;                            // products of a step of 64

// A stage of both operands, 128 bytes of every row, goes straight to LDS, where the 16-byte piece j of a row lies at j ^ (row / 2 % 8): eight lanes ask for
// a row's line in that order, and the fragment reads of sixteen rows share no bank.  There is one wave to a SIMD, which nothing else fills in for, so
// every place between two products is given what it can take: two reads, or a request, as the way into LDS takes 16 cycles of each of the four waves' and
// a product 64.  A stage is read out in the first half of its first step, then the stage after the next is asked for in its place, while
// the next one has until the second step to land.  Behind a tile's last stage the first two of the next tile are asked for before its results leave.
// Bound: the matrix cores at the card's power limit.  16384 x 8192 x 8192 741 us (3.0 PFLOP/s; a loop of these instructions on registers
// reaches 4.5), 8192 x 8192 x 4096 204 in a training step, 187 alone; busy 78 to 85 % of the cycles, at 1.75 to 2.2 GHz.  Where sums are short a tile's start and results count:
// 65536 x 2048 x 2048 221 us alone, and 264 as the rows of 32 experts, 256 where they lie in order (2176 tiles instead of 2048; the cores are busy 45 %), 297 in a training step.  Four waves of 128 x 128 read a third less from LDS than
// eight of 128 x 64, which reached 2.7 PFLOP/s.

// The lane, as a value that the compiler works on where it stands: places of lanes that it kept from tile to tile would cost the registers that
// the sums need.
__device__ __forceinline__ int lane_now() {
    int lane = threadIdx.x % kWave;
    asm volatile("" : "+v"(lane));
    return lane;
}

struct Source {              // what a wave asks for: 128 rows of A (waves 0 and 1) or B
    uint32_t off[16], word_off[2];
    const uint8_t* codes;
    const uint8_t* scales;
    int64_t codes_left, words_left, pitch_words;
    int s1;

    __device__ __forceinline__ void set(const ProductArgs& p, const Tile& t, bool gather, int lane) {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
        const bool of_b = wave >= kWaves / 2;
        const Fp8Operand& o = of_b ? p.b : p.a;
        const bool taken = gather && !of_b;
        const int64_t first = (of_b ? t.b0 - kEdge : t.a0) + wave * 128, end = of_b ? t.b_end : t.a_end, base = taken ? 0 : min(first, end - 1);
        auto row_of = [&](int i) {
            const int64_t r = min(first + i, end - 1);      // (rows behind the last one repeat it; they are not stored)
            return (uint32_t)(taken ? p.order[r] / p.picks : r - base);
        };
#pragma unroll
        for (int i = 0; i < 16; ++i) off[i] = row_of(i * 8 + lane / 8) * (uint32_t)o.pitch + (uint32_t)((lane % 8) ^ ((i * 4 + lane / 16) & 7)) * 16u;
#pragma unroll
        for (int i = 0; i < 2; ++i) word_off[i] = row_of(i * 64 + lane) * 4u;
        codes = o.codes + base * o.pitch;
        scales = o.scales + base * 4;
        codes_left = (o.rows - base) * o.pitch;
        words_left = (o.rows - base) * 4;
        pitch_words = o.rows * 4;
        s1 = t.s1;
    }
    // (a stage behind the last one is asked for through descriptors without an extent: LDS receives zeros)
    __device__ __forceinline__ __amdgpu_buffer_rsrc_t codes_of(int s) const { return bytes_of(codes, s < s1 ? codes_left : 0); }
    __device__ __forceinline__ __amdgpu_buffer_rsrc_t words_of(int s) const { return bytes_of(scales + (s / 4) * pitch_words, s < s1 ? words_left : 0); }
    __device__ __forceinline__ void request(int n, int wave, int s, __amdgpu_buffer_rsrc_t c, __amdgpu_buffer_rsrc_t w, uint8_t* to) const {
        if (n < 16) tile_to_lds(c, off[n], (uint32_t)s * 128u, to + (wave * 16 + n) * 1024);
        else words_to_lds(w, word_off[n - 16], 0, to + kCodes + (wave * 2 + n - 16) * 256);
    }
    __device__ __forceinline__ void ask(int wave, int s, uint8_t* to) const {
        const __amdgpu_buffer_rsrc_t c = codes_of(s), w = words_of(s);
#pragma unroll
        for (int n = 0; n < kAsks; ++n) request(n, wave, s, c, w, to);
    }
};

// The results of a wave, through its 4 KiB of LDS so that whole lines are written: 32 rows of 64 columns at a time, 16-byte pieces of a row in the order
// piece ^ row % 8.  put(row block, pair of column blocks, rows 8 k .., pieces)
template <typename Put>
__device__ __forceinline__ void results_out(const v16f (&acc)[kB][kB], uint8_t* mine, int lane, Put put) {
    const int m = lane % 32, h = lane / 32;
#pragma unroll
    for (int i = 0; i < kB; ++i)
#pragma unroll
        for (int jp = 0; jp < kB / 2; ++jp) {
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const v16f& a = acc[jp * 2 + j][i];
                    *reinterpret_cast<u32x2*>(mine + m * 128 + (((j * 4 + q) ^ m) & 7) * 16 + h * 8) = u32x2{pack_bf16(a[4 * q], a[4 * q + 1]), pack_bf16(a[4 * q + 2], a[4 * q + 3])};
                }
            __builtin_amdgcn_wave_barrier();
            u32x4 v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = *reinterpret_cast<const u32x4*>(mine + (k * 8 + lane / 8) * 128 + ((lane ^ (lane / 8)) & 7) * 16);
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int k = 0; k < 4; ++k) put(i, jp, k, v[k]);
        }
}

// lds0, lds1: the stages' places, as arguments so that the compiler knows them apart, and does not let a read of one wait for the requests into the other.
// FLUSH: rows of results are whole 16-byte pieces, and leave through one descriptor, which ends with the product's last row: every tile has the same
// number of stores, so that what is waited for is known here.
template <Of OF, bool FLUSH>
__device__ __forceinline__ void run_tiles(const ProductArgs& p, uint8_t* __restrict__ lds0, uint8_t* __restrict__ lds1, uint8_t* __restrict__ out) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int wr = wave / 2, wc = wave % 2;
    const bool gather = OF == Of::kExpertRows && p.picks != 0;
    const TileCount<kEdge, OF> count(p);
    int t = (int)(blockIdx.x / kXcd);
    Tile tile;
    if (!tile_at<kEdge, kEdge, OF>(p, count, t, 0, tile)) return;      // (an expert's last tiles: one workgroup, one tile)
    Source from;
    from.set(p, tile, gather, lane_now());
    from.ask(wave, tile.s0, lds0);
    from.ask(wave, tile.s0 + 1, lds1);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");

    v8i fr[2][kB], fc[2][kB];
    int sr[kB], sc[kB], wr_next[kB], wc_next[kB], at[2][2], at_word;     // at: of a lane in 32 rows, step and half of its 32 bytes
    auto fragment = [&](const uint8_t* p0, int block, int k) {
        const v4i lo = *reinterpret_cast<const v4i*>(p0 + block * 4096 + at[k][0]), hi = *reinterpret_cast<const v4i*>(p0 + block * 4096 + at[k][1]);
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    auto fetch = [&](const uint8_t* p0, int n, int k) {         // fragments in the order of their first use
        if (n == 1 || n > kB) fr[k][n == 1 ? 0 : n - kB] = fragment(p0, wr * kB + (n == 1 ? 0 : n - kB), k);
        else fc[k][n == 0 ? 0 : n - 1] = fragment(p0, 2 * kB + wc * kB + (n == 0 ? 0 : n - 1), k);
    };
    auto read_words = [&](const uint8_t* p0) {
#pragma unroll
        for (int i = 0; i < kB; ++i) {
            wr_next[i] = *reinterpret_cast<const int*>(p0 + kCodes + (wr * kB + i) * 128 + at_word);
            wc_next[i] = *reinterpret_cast<const int*>(p0 + kCodes + (2 * kB + wc * kB + i) * 128 + at_word);
        }
    };
    auto take_words = [&](int s) {      // the byte of stage s
#pragma unroll
        for (int i = 0; i < kB; ++i) sr[i] = wr_next[i] >> (s % 4 * 8), sc[i] = wc_next[i] >> (s % 4 * 8);
    };
    constexpr int kFree = 2 * kB + 2;                          // two products behind the last read its data have arrived
    constexpr int kDone = kPlaces - kFree;                     // requests of a stage's first step
    static_assert(2 * kB + 2 < kPlaces && kAsks <= kDone + kPlaces, "everything has its place");

    for (;;) {
        // the first stage has landed; the stores of the tile before follow the requests for the first two
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(FLUSH ? kAsks + kStores : 0) : "memory");
        __builtin_amdgcn_s_barrier();
        const int lane = lane_now();
        at_word = (lane % 32) * 4;
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int u = 0; u < 2; ++u) at[k][u] = (lane % 32) * 128 + ((k * 4 + lane / 32 * 2 + u) ^ (lane / 2 & 7)) * 16;
        v16f acc[kB][kB];
#pragma unroll
        for (int j = 0; j < kB; ++j)
#pragma unroll
            for (int i = 0; i < kB; ++i) acc[j][i] = v16f{};
        auto product = [&](int n, int k) { acc[n % kB][n / kB] = mfma8(fc[k][n % kB], fr[k][n / kB], acc[n % kB][n / kB], sc[n % kB], sr[n / kB]); };
        auto stage = [&](int s, uint8_t* here, uint8_t* next, auto stores) {
            const int later = s + 2;
            const __amdgpu_buffer_rsrc_t codes = from.codes_of(later), words = from.words_of(later);
#pragma unroll
            for (int n = 0; n < kPlaces; ++n) {
                product(n, 0);
                if (n < 2 * kB) fetch(here, n, 1);
                else if (n >= kFree) from.request(n - kFree, wave, later, codes, words, here);
                __builtin_amdgcn_sched_barrier(0);
                if (n == kFree - 1) {
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");      // this stage is read out
                    __builtin_amdgcn_s_barrier();
                }
            }
#pragma unroll
            for (int n = 0; n < kPlaces; ++n) {
                if (n == 2) {
                    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kDone + 2 + decltype(stores)::value) : "memory");      // the next stage has landed
                    __builtin_amdgcn_s_barrier();
                }
                product(n, 1);
                if (n + kDone < kAsks) from.request(n + kDone, wave, later, codes, words, here);
                if (n >= 2 && n < 2 + 2 * kB) fetch(next, n - 2, 0);
                if (n == 2 + 2 * kB) read_words(next);
                __builtin_amdgcn_sched_barrier(0);
            }
            take_words(s + 1);
        };
        read_words(lds0);
#pragma unroll
        for (int n = 0; n < 2 * kB; ++n) fetch(lds0, n, 0);
        take_words(tile.s0);
        // (an odd count has a stage of zeros behind it, a count of zero two)
        constexpr std::integral_constant<int, 0> kNone{};
        stage(tile.s0, lds0, lds1, std::integral_constant<int, FLUSH ? kStores : 0>{});
        stage(tile.s0 + 1, lds1, lds0, kNone);
#pragma nounroll
        for (int s = tile.s0 + 2; s < tile.s1; s += 2) {
            stage(s, lds0, lds1, kNone);
            stage(s + 1, lds1, lds0, kNone);
        }
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");   // the requests past the end have landed
        __builtin_amdgcn_s_barrier();
        const Tile done = tile;
        t += (int)(gridDim.x / kXcd);
        const bool more = tile_at<kEdge, kEdge, OF>(p, count, t, 0, tile);
        if (more) {
            from.set(p, tile, gather, lane_now());
            from.ask(wave, tile.s0, lds0);
            from.ask(wave, tile.s0 + 1, lds1);
        }
        uint16_t* const d = reinterpret_cast<uint16_t*>(done.d) + done.a0 * p.ldd + done.c0;
        const int rows = (int)min(done.a_end - done.a0, (int64_t)kEdge), cols = (int)min(p.N - done.c0, (int64_t)kEdge);
        const int now = lane_now(), row0 = wr * 128 + now / 8, col0 = wc * 128 + (now & 7) * 8;
        if constexpr (FLUSH) {
            const __amdgpu_buffer_rsrc_t to = bytes_of(reinterpret_cast<const uint8_t*>(d), ((rows - 1) * p.ldd + cols) * 2);
            const uint32_t off0 = (uint32_t)(row0 * (int)p.ldd + col0) * 2u;
            results_out(acc, out + wave * 4096, now, [&](int i, int jp, int k, u32x4 v) {
                const uint32_t off = off0 + (uint32_t)((i * 32 + k * 8) * (int)p.ldd + jp * 64) * 2u;
                const int where = (int)(col0 + jp * 64 < cols ? off : kTileReach);
                if (p.stream) __builtin_amdgcn_raw_buffer_store_b128(v, to, where, 0, 2);      // (non-temporal)
                else __builtin_amdgcn_raw_buffer_store_b128(v, to, where, 0, 0);
            });
            static_assert(kStores == kB * (kB / 2) * 4, "as many as results_out puts");
        } else {
            results_out(acc, out + wave * 4096, now, [&](int i, int jp, int k, u32x4 v) {
                const int m = row0 + i * 32 + k * 8, n = col0 + jp * 64;
                if (m < rows && n < cols) put8(d + m * p.ldd + n, v, cols - n);
            });
        }
        if (!more) return;
    }
}

template <Of OF, bool FLUSH>
__global__ __launch_bounds__(64 * kWaves, 1) void k_fp8_large(ProductArgs p) {
    extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
    run_tiles<OF, FLUSH>(p, lds, lds + kStage, lds + 2 * kStage);
}

template <Of OF, bool FLUSH>
daq_status launch(const ProductArgs& p, hipStream_t st) {
    // (gradients of experts take times of their own: a workgroup for each tile, which the CUs take as they get free)
    const int64_t tiles = OF == Of::kExpertWeights ? tile_groups<OF>(p) : std::min<int64_t>(tile_groups<OF>(p), 256);
    const auto kernel = k_fp8_large<OF, FLUSH>;
    if (!allow_lds((const void*)kernel, kLds)) return DAQ_ERR_HIP;
    DAQ_LAUNCH("fp8_large", st, hipLaunchKernelGGL(kernel, dim3((unsigned)tiles), dim3(64 * kWaves), kLds, st, p));
    return DAQ_OK;
}

}  // namespace

// Results of more than the caches behind L2 keep (256 MiB) pass them by: 65536 x 2048 x 2048 (256 MiB of results) 215 us instead of 251 (both of one run), 16384 x 8192 x 8192 721
// instead of 737; of half as much they stay, 8192 x 8192 x 4096 193 instead of 196.
constexpr int64_t kStreamProduct = (int64_t)192 << 20;

daq_status fp8_large(Of of, ProductArgs p, hipStream_t st) {
    p.stream = p.M * p.N * 2 * (of == Of::kExpertWeights ? p.experts : 1) >= kStreamProduct;
    const bool flush = p.N % 8 == 0 && p.ldd % 8 == 0 && p.ldd < (1 << 22) && ((uintptr_t)p.d & 15) == 0 && p.stride % 8 == 0;
    switch (of) {
        case Of::kWhole: return flush ? launch<Of::kWhole, true>(p, st) : launch<Of::kWhole, false>(p, st);
        case Of::kExpertRows: return flush ? launch<Of::kExpertRows, true>(p, st) : launch<Of::kExpertRows, false>(p, st);
        default: return flush ? launch<Of::kExpertWeights, true>(p, st) : launch<Of::kExpertWeights, false>(p, st);
    }
}

}  // namespace daq
