// A router: scores of the experts, the choice among them, the gradient of the logits, and the order of a batch's rows by expert.
#include <cmath>
#include <type_traits>

#include "fp8.h"

namespace daq {

namespace {

struct RouteArgs {
    int64_t tokens, ld;
    int experts, picks, groups, top_groups, per_group;
    int sigmoid, renormalize;
    double scale;
    const float* bias;
    float* weights;
    int32_t* chosen;
};

template <typename T> __device__ __forceinline__ float logit_at(const T* p);
template <> __device__ __forceinline__ float logit_at<float>(const float* p) { return *p; }
template <> __device__ __forceinline__ float logit_at<uint16_t>(const uint16_t* p) { return bits_as<float>((uint32_t)*p << 16); }

// The best of the wave, the lowest index of equals.
__device__ __forceinline__ void best_of_wave(double& c, int& at) {
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) {
        const double oc = __shfl_xor(c, d);
        const int oat = __shfl_xor(at, d);
        if (oc > c || (oc == c && oat < at)) {
            c = oc;
            at = oat;
        }
    }
}

// The largest of the wave, to all lanes: six exchanges in registers.
template <int CTRL, int ROWS>
__device__ __forceinline__ float max_with(float v) {
    return fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(v), __float_as_int(v), CTRL, ROWS, 0xF, false)));
}
__device__ __forceinline__ float top_of_wave(float v) {
    v = max_with<0x111, 0xF>(v);      // from 1, 2, 4 and 8 lanes before, within 16
    v = max_with<0x112, 0xF>(v);
    v = max_with<0x114, 0xF>(v);
    v = max_with<0x118, 0xF>(v);
    v = max_with<0x142, 0xA>(v);      // from the last lane of the 16, and of the 32, before
    v = max_with<0x143, 0xC>(v);
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

// The two largest of a lane and of the one that it exchanges with.
template <typename Swap>
__device__ __forceinline__ void merge_two(float& one, float& two, Swap swap) {
    const float o1 = swap(one), o2 = swap(two);
    two = fmaxf(fmaxf(two, o2), fminf(one, o1));
    one = fmaxf(one, o1);
}
template <int CTRL>
__device__ __forceinline__ float swapped(float v) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, true)); }

// Neighbouring logits, -infinity behind the last.
template <int PER>
__device__ __forceinline__ void load_logits(const float* p, int left, float (&l)[PER]) {
    if (PER >= 4 && left >= PER) {
#pragma unroll
        for (int i = 0; i < PER; i += 4) {
            const u32x4 v = *reinterpret_cast<const u32x4_a4*>(p + i);
#pragma unroll
            for (int j = 0; j < 4 && i + j < PER; ++j) l[i + j] = bits_as<float>(v[j]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < PER; ++i) l[i] = i < left ? p[i] : -__builtin_inff();
    }
}
template <int PER>
__device__ __forceinline__ void load_logits(const uint16_t* p, int left, float (&l)[PER]) {
    if (PER >= 4 && left >= PER) {
#pragma unroll
        for (int i = 0; i < PER; i += 4) {
            const u32x2 v = *reinterpret_cast<const u32x2_a2*>(p + i);
#pragma unroll
            for (int j = 0; j < 4 && i + j < PER; ++j) l[i + j] = (j & 1) ? bf16_hi(v[j / 2]) : bf16_lo(v[j / 2]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < PER; ++i) l[i] = i < left ? logit_at(p + i) : -__builtin_inff();
    }
}

// The choice in 64 bits: lane j has the expert of place j, -1 where there is none.
template <int PER>
__device__ __forceinline__ int choose_exactly(const RouteArgs& p, const float (&l)[PER], float most, const float* bias, int lane) {
    constexpr double kNone = -__builtin_inf();
    double c[PER];
    if (p.sigmoid) {
#pragma unroll
        for (int i = 0; i < PER; ++i) c[i] = 1.0 / (1.0 + exp(-(double)l[i]));
    } else {
        double sum = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            c[i] = l[i] > -__builtin_inff() ? exp((double)l[i] - (double)most) : 0.0;
            sum += c[i];
        }
#pragma unroll
        for (int d = 1; d < kWave; d *= 2) sum += __shfl_xor(sum, d);
#pragma unroll
        for (int i = 0; i < PER; ++i) c[i] = sum > 0 ? c[i] / sum : 0.0;
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int e = lane * PER + i;
        if (!(e < p.experts && l[i] > -__builtin_inff())) c[i] = kNone;
        else if (bias) c[i] += (double)bias[e];
    }
    if (p.groups > 1) {
        double total = kNone;                 // of group `lane`
        for (int g = 0; g < p.groups; ++g) {
            double one = kNone, two = kNone;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                if ((lane * PER + i) / p.per_group != g) continue;
                two = fmax(two, fmin(one, c[i]));
                one = fmax(one, c[i]);
            }
#pragma unroll
            for (int d = 1; d < kWave; d *= 2) {
                const double o1 = __shfl_xor(one, d), o2 = __shfl_xor(two, d);
                two = fmax(fmax(two, o2), fmin(one, o1));
                one = fmax(one, o1);
            }
            if (lane == g) total = two == kNone ? one : one + two;
        }
        uint64_t stay = 0;
        for (int n = 0; n < p.top_groups; ++n) {
            double best = (lane < p.groups && !(stay >> lane & 1)) ? total : kNone;
            int at = (lane < p.groups && !(stay >> lane & 1)) ? lane : kWave;
            best_of_wave(best, at);
            if (at < kWave) stay |= (uint64_t)1 << at;
        }
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int g = (lane * PER + i) / p.per_group;
            if (g >= p.groups || !(stay >> g & 1)) c[i] = kNone;
        }
    }
    int expert = -1;
    for (int j = 0; j < p.picks; ++j) {
        double best = kNone;
        int at = 0x7FFFFFFF;
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (c[i] > best) {
                best = c[i];
                at = lane * PER + i;
            }
        best_of_wave(best, at);
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (lane * PER + i == at) c[i] = kNone;
        if (lane == j && best > kNone) expert = at;
    }
    return expert;
}

// A wave a token; lane l has the experts l * PER .. of it.  The choice is made in 32 bits, by the logits themselves where no bias counts (the scores rise with
// them), otherwise by scores that are off by less than 2^-19 (of 1, or of the largest c).  Wherever two c that decide are nearer to one another than that, or logits
// than 64 bits keep their scores apart, the wave chooses again in 64 bits.  What bounds it are vector instructions, some 25 for a place.
template <typename T, int PER>
__global__ __launch_bounds__(256) void k_route(const T* logits, RouteArgs p) {
    constexpr float kNone = -__builtin_inff();
    const int lane = threadIdx.x % kWave;
    const int64_t t = (int64_t)blockIdx.x * 4 + threadIdx.x / kWave;
    if (t >= p.tokens) return;
    const T* row = logits + t * p.ld;
    const int first = lane * PER;
    float l[PER], c[PER];
    load_logits<PER>(row + first, p.experts - first, l);
    bool bad = false;
    float most = kNone;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        bad |= l[i] != l[i] || (!p.sigmoid && l[i] == __builtin_inff());
        most = fmaxf(most, l[i]);
    }
    most = top_of_wave(most);
    const bool by_score = p.bias || p.groups > 1;
    if (by_score) {
        if (p.sigmoid) {
#pragma unroll
            for (int i = 0; i < PER; ++i) c[i] = __builtin_amdgcn_rcpf(1.f + __expf(-l[i]));
        } else {
            float sum = 0;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                c[i] = l[i] > kNone ? __expf(l[i] - most) : 0.f;
                sum += c[i];
            }
#pragma unroll
            for (int d = 1; d < kWave; d *= 2) sum += __shfl_xor(sum, d);
            const float over = sum > 0 ? __builtin_amdgcn_rcpf(sum) : 0.f;
#pragma unroll
            for (int i = 0; i < PER; ++i) c[i] *= over;
        }
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        if (p.bias && first + i < p.experts) c[i] += p.bias[first + i];
        bad |= by_score && first + i < p.experts && l[i] > kNone && c[i] != c[i];
        if (!by_score || !(l[i] > kNone)) c[i] = l[i] > kNone ? l[i] : kNone;
    }
    bad = __any(bad);
    // what c may be off by, and whether the wave has to choose again
    float top = kNone;
#pragma unroll
    for (int i = 0; i < PER; ++i) top = fmaxf(top, fabsf(c[i]) < __builtin_inff() ? fabsf(c[i]) : 0.f);
    const float off = by_score ? fmaxf(1.f, top_of_wave(top)) * 0x1p-19f : 0.f;
    bool again = false;
    if (p.groups > 1) {
        float one = kNone, two = kNone, total;
        const int lanes = p.per_group / PER;
        uint64_t mine = ~(uint64_t)0;         // lanes of this lane's group
        if (lanes * PER == p.per_group && (lanes & (lanes - 1)) == 0) {
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                two = fmaxf(two, fminf(one, c[i]));
                one = fmaxf(one, c[i]);
            }
            if (lanes >= 2) merge_two(one, two, swapped<0xB1>);
            if (lanes >= 4) merge_two(one, two, swapped<0x4E>);
            if (lanes >= 8) merge_two(one, two, swapped<0x141>);
            if (lanes >= 16) merge_two(one, two, swapped<0x140>);
            if (lanes >= 32) merge_two(one, two, [](float v) { return __shfl_xor(v, 16); });
            total = two == kNone ? one : one + two;
            float before = __builtin_inff();
            uint64_t stay = 0;
            for (int n = 0; n <= p.top_groups && n < p.groups; ++n) {
                const bool left = first < p.experts && !(stay >> lane & 1);
                const float best = top_of_wave(left ? total : kNone);
                const uint64_t at = __ballot(left && total == best);
                if (n == p.top_groups) {
                    again |= best > kNone && !(before - best > 4 * off);
                    break;
                }
                if (at) stay |= (lanes == kWave ? ~(uint64_t)0 : ((uint64_t)1 << lanes) - 1) << (__builtin_ctzll(at) / lanes * lanes);
                before = best;
            }
            if (!(stay >> lane & 1)) mine = 0;
        } else {
            again = true;                     // groups that do not lie in whole lanes
        }
        if (!mine) {
#pragma unroll
            for (int i = 0; i < PER; ++i) c[i] = kNone;
        }
        if (!p.bias) {                        // the logits of those that stay
#pragma unroll
            for (int i = 0; i < PER; ++i) c[i] = c[i] > kNone ? l[i] : kNone;
        }
    }
    int expert = -1;
    float before = __builtin_inff();
    for (int j = 0; j <= p.picks && !again; ++j) {
        float m = kNone;
#pragma unroll
        for (int i = 0; i < PER; ++i) m = fmaxf(m, c[i]);
        const float best = top_of_wave(m);
        if (best == kNone) break;
        if (p.bias) again = !(before - best > 2 * off);
        else again = (before > best && before - best < 0x1p-36f) || best < (p.sigmoid ? -600.f : most - 600.f) || (p.sigmoid && best > 10.f);
        before = best;
        if (j == p.picks) break;
        const int owner = __builtin_ctzll(__ballot(m == best));
        int at = 0;
#pragma unroll
        for (int i = PER - 1; i >= 0; --i) at = c[i] == best ? i : at;
        at = __builtin_amdgcn_readlane(at, owner);
#pragma unroll
        for (int i = 0; i < PER; ++i) c[i] = lane == owner && i == at ? kNone : c[i];
        expert = lane == j ? owner * PER + at : expert;
    }
    if (again && !bad) expert = choose_exactly<PER>(p, l, most, p.bias, lane);
    // the weights of the places in 64 bits
    const bool there = expert >= 0;
    const double x = there ? (double)logit_at(row + expert) : 0.0;
    double s = 0, total = 1;
    if (p.sigmoid) {
        s = 1.0 / (1.0 + exp(-x));
    } else {
        s = exp(x - (there ? (double)most : 0.0));
        if (!p.renormalize) {
            total = 0;
#pragma unroll
            for (int i = 0; i < PER; ++i) total += l[i] > kNone ? exp((double)l[i] - (double)most) : 0.0;
#pragma unroll
            for (int d = 1; d < kWave; d *= 2) total += __shfl_xor(total, d);
        }
    }
    if (!there) s = 0;
    if (p.renormalize) {                      // (places are lanes 0 .. 31)
        total = s;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) total += __shfl_xor(total, d);
    }
    if (lane < p.picks) {
        p.weights[t * p.picks + lane] = bad ? __builtin_nanf("") : (float)(total > 0 ? s / total * p.scale : 0.0);
        p.chosen[t * p.picks + lane] = bad ? -1 : expert;
    }
}

struct RouteBackArgs {
    int64_t tokens, ld, ldd;
    int experts, picks;
    int sigmoid, renormalize;
    float scale;
    const float* dweights;
    const int32_t* chosen;
};

template <typename F>
__device__ __forceinline__ F wave_sum(F v) {
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) v += __shfl_xor(v, d);
    return v;
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) v = fmaxf(v, __shfl_xor(v, d));
    return v;
}

// A wave a token: the chosen ones' part in lane j for place j, then the row, zero or (softmax that is not renormalised) the others' part.
template <typename T>
__global__ __launch_bounds__(256) void k_route_back(const T* logits, T* dlogits, RouteBackArgs p) {
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int64_t t = (int64_t)blockIdx.x * 4 + wave;
    __shared__ float row[4][kMaxExperts];
    if (t >= p.tokens) return;
    const T* from = logits + t * p.ld;
    T* to = dlogits + t * p.ldd;
    const int e = lane < p.picks ? p.chosen[t * p.picks + lane] : -1;
    const bool there = e >= 0 && e < p.experts;
    const float g = there ? p.dweights[t * p.picks + lane] : 0.f, l = there ? logit_at(from + e) : 0.f;
    float* mine = row[wave];
    for (int i = lane; i < p.experts; i += kWave) mine[i] = 0.f;
    float d = 0.f;                             // of the chosen one's logit
    float most = 0.f, sum = 1.f, back = 0.f;
    if (p.sigmoid || p.renormalize) {
        // s and, where it is renormalised, its share of the chosen ones', which may all be tiny: in 64 bits, as in the forward pass
        double s, rest = 1.0;
        if (p.sigmoid) {
            const double ex = exp(-fabs((double)l)), one = 1.0 / (1.0 + ex);
            s = l >= 0 ? one : ex * one;
            rest = l >= 0 ? ex * one : one;
        } else {
            most = wave_max(there ? l : -__builtin_inff());
            s = exp((double)l - (double)most);
        }
        if (!there) s = 0;
        double v = g;
        if (p.renormalize) {
            const double total = wave_sum(s);
            s = total > 0 ? s / total : 0.0;
            v -= wave_sum(g * s);
        }
        d = (float)(p.scale * v * s * rest);
    } else {
        float m = -__builtin_inff();
        for (int i = lane; i < p.experts; i += kWave) m = fmaxf(m, logit_at(from + i));
        most = wave_max(m);
        float total = 0.f;
        for (int i = lane; i < p.experts; i += kWave) total += expf(logit_at(from + i) - most);
        sum = wave_sum(total);
        const float s = there ? expf(l - most) / sum : 0.f;
        back = wave_sum(p.scale * g * s);
        d = p.scale * g;
    }
    const bool any = __any(there);
    for (int j = 0; j < p.picks; ++j) {        // one after the other: an expert that a token names twice has both parts
        if (lane == j && there) mine[e] += d;
        __builtin_amdgcn_wave_barrier();
    }
    for (int i = lane; i < p.experts; i += kWave) {
        float v = mine[i];
        if (!p.sigmoid && !p.renormalize) v = any ? expf(logit_at(from + i) - most) / sum * (v - back) : 0.f;
        if constexpr (sizeof(T) == 4) to[i] = v;
        else to[i] = (T)(pack_bf16(v, 0.f) & 0xFFFFu);
    }
}

// ---- the order of the rows --------------------------------------------------------------------
// A workgroup takes a run of slots, 1024 at a time.  counts[block][expert] by a first launch; the second adds up what stands before its own
// run and places it.  Within a wave a slot's rank among those of its expert comes from ten votes, one a bit of the expert's number.
constexpr int kPlanThreads = 1024, kPlanWaves = kPlanThreads / kWave;

struct PlanArgs {
    const int32_t* chosen;
    int64_t slots;
    int experts, blocks, rounds;
    int32_t* per_block;       // [blocks][experts]
    int32_t *counts, *table, *rows, *place;
};

// The lanes whose slots have the same expert (-1: none) as this lane's.
__device__ __forceinline__ uint64_t same_expert(int e) {
    uint64_t same = __ballot(e >= 0);
#pragma unroll
    for (int b = 0; b < 10; ++b) {
        const uint64_t has = __ballot(e >> b & 1);
        same &= (e >> b & 1) ? has : ~has;
    }
    return same;
}
__device__ __forceinline__ int slot_expert(const PlanArgs& p, int64_t slot) {
    const int e = slot < p.slots ? p.chosen[slot] : -1;
    return e >= 0 && e < p.experts ? e : -1;
}

__global__ __launch_bounds__(kPlanThreads) void k_plan_count(PlanArgs p) {
    __shared__ int n[kMaxExperts];
    for (int e = threadIdx.x; e < p.experts; e += kPlanThreads) n[e] = 0;
    __syncthreads();
    const int lane = threadIdx.x % kWave;
    for (int r = 0; r < p.rounds; ++r) {
        const int e = slot_expert(p, ((int64_t)blockIdx.x * p.rounds + r) * kPlanThreads + threadIdx.x);
        const uint64_t same = same_expert(e);
        if (e >= 0 && __builtin_ctzll(same) == lane) atomicAdd(n + e, __popcll(same));      // (whole numbers: any order)
    }
    __syncthreads();
    for (int e = threadIdx.x; e < p.experts; e += kPlanThreads) p.per_block[(int64_t)blockIdx.x * p.experts + e] = n[e];
}

// Sums over 1024 threads of what stands before each of them; the total to all.
__device__ __forceinline__ int before_me(int v, int* per_wave, int& total) {
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    int sum = v;
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) {
        const int o = __shfl_up(sum, d);
        if (lane >= d) sum += o;
    }
    if (lane == kWave - 1) per_wave[wave] = sum;
    __syncthreads();
    int first = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kPlanWaves; ++w) {
        const int n = per_wave[w];
        first += w < wave ? n : 0;
        total += n;
    }
    __syncthreads();
    return first + sum - v;
}

__global__ __launch_bounds__(kPlanThreads) void k_plan_place(PlanArgs p) {
    __shared__ int next[kMaxExperts];                       // the row of an expert's next slot
    __shared__ uint16_t ranks[kPlanWaves][kMaxExperts];     // slots of an expert in a wave of this round
    __shared__ int per_wave[kPlanWaves];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, e0 = threadIdx.x;
    int before = 0, all = 0;                                // slots of expert e0 in the runs before this one, and in all
    if (p.blocks == 1) {
        next[e0] = 0;
        __syncthreads();
        for (int r = 0; r < p.rounds; ++r) {
            const int e = slot_expert(p, (int64_t)r * kPlanThreads + threadIdx.x);
            const uint64_t same = same_expert(e);
            if (e >= 0 && __builtin_ctzll(same) == lane) atomicAdd(next + e, __popcll(same));
        }
        __syncthreads();
        all = next[e0];
    } else if (e0 < p.experts) {
        for (int b = 0; b < p.blocks; ++b) {
            const int n = p.per_block[(int64_t)b * p.experts + e0];
            all += n;
            before += b < (int)blockIdx.x ? n : 0;
        }
    }
    int total;
    const int first = before_me(all, per_wave, total);
    if (e0 < p.experts) next[e0] = first + before;
    if (blockIdx.x == 0) {
        int t256, t128, t64;
        const int b256 = before_me((all + 255) / 256, per_wave, t256), b128 = before_me((all + 127) / 128, per_wave, t128),
                  b64 = before_me((all + 63) / 64, per_wave, t64);
        const int pitch = p.experts + 1;
        if (e0 < p.experts) {
            p.counts[e0] = all;
            p.table[kTableRows * pitch + e0] = first;
            p.table[kTable256 * pitch + e0] = b256;
            p.table[kTable128 * pitch + e0] = b128;
            p.table[kTable64 * pitch + e0] = b64;
        }
        if (e0 == 0) {
            p.table[kTableRows * pitch + p.experts] = total;
            p.table[kTable256 * pitch + p.experts] = t256;
            p.table[kTable128 * pitch + p.experts] = t128;
            p.table[kTable64 * pitch + p.experts] = t64;
        }
    }
    for (int r = 0; r < p.rounds; ++r) {
        for (int i = threadIdx.x; i < kPlanWaves * p.experts; i += kPlanThreads) ranks[i / p.experts][i % p.experts] = 0;
        __syncthreads();
        const int64_t slot = ((int64_t)blockIdx.x * p.rounds + r) * kPlanThreads + threadIdx.x;
        const int e = slot_expert(p, slot);
        const uint64_t same = same_expert(e);
        const int rank = __popcll(same & (((uint64_t)1 << lane) - 1));
        if (e >= 0 && rank == 0) ranks[wave][e] = (uint16_t)__popcll(same);
        __syncthreads();
        int moved = 0;
        if (e0 < p.experts) {                               // where each wave's slots of expert e0 begin
#pragma unroll
            for (int w = 0; w < kPlanWaves; ++w) {
                const int n = ranks[w][e0];
                ranks[w][e0] = (uint16_t)moved;
                moved += n;
            }
        }
        __syncthreads();
        if (slot < p.slots) {
            const int row = e >= 0 ? next[e] + ranks[wave][e] + rank : -1;
            p.place[slot] = row;
            if (row >= 0) p.rows[row] = (int)slot;
            if (slot >= total) p.rows[slot] = -1;
        }
        __syncthreads();
        if (e0 < p.experts) next[e0] += moved;
    }
}

struct PlanShape {
    int blocks, rounds;
};
PlanShape plan_shape(int64_t slots) {
    if (slots <= 4 * kPlanThreads) return {1, (int)std::max<int64_t>(1, ceil_div(slots, kPlanThreads))};
    const int64_t rounds = ceil_div(slots, 256 * kPlanThreads);
    return {(int)ceil_div(slots, rounds * kPlanThreads), (int)rounds};
}

daq_status route_check(int64_t tokens, int32_t experts, const void* logits, int dtype, int64_t ld, const daq_route_opts* o) {
    if (!o || tokens < 0 || experts <= 0 || !dtype_ok(dtype) || (o->scores != DAQ_SCORES_SOFTMAX && o->scores != DAQ_SCORES_SIGMOID)) return DAQ_ERR_INVALID_ARG;
    if (o->groups <= 0 || experts % o->groups || o->top_groups <= 0 || o->top_groups > o->groups || o->picks <= 0 ||
        o->picks > experts / o->groups * o->top_groups || !(std::fabs(o->scale) < INFINITY))
        return DAQ_ERR_INVALID_ARG;
    if (experts > kMaxExperts || o->picks > 32 || o->groups > 64 || tokens >= kMaxSlots) return DAQ_ERR_UNSUPPORTED;
    if (tokens == 0) return DAQ_OK;
    return logits && elem_aligned(logits, dtype) && ld >= experts ? DAQ_OK : DAQ_ERR_INVALID_ARG;
}
bool a4(const void* p) { return ((uintptr_t)p & 3u) == 0; }

template <typename T>
daq_status launch_route(const T* logits, const RouteArgs& p, hipStream_t st) {
    const auto kernel = p.experts <= 64 ? k_route<T, 1> : p.experts <= 128 ? k_route<T, 2> : p.experts <= 256 ? k_route<T, 4> : p.experts <= 512 ? k_route<T, 8> : k_route<T, 16>;
    DAQ_LAUNCH("route", st, hipLaunchKernelGGL(kernel, dim3((unsigned)ceil_div(p.tokens, 4)), dim3(256), 0, st, logits, p));
    return DAQ_OK;
}
template <typename T>
daq_status launch_back(const T* logits, T* dlogits, const RouteBackArgs& p, hipStream_t st) {
    DAQ_LAUNCH("route_back", st, hipLaunchKernelGGL(k_route_back<T>, dim3((unsigned)ceil_div(p.tokens, 4)), dim3(256), 0, st, logits, dlogits, p));
    return DAQ_OK;
}

}  // namespace

}  // namespace daq

using namespace daq;

extern "C" daq_status daq_route(int64_t tokens, int32_t experts, const void* logits, daq_dtype dtype, int64_t ld, const float* bias,
                                const daq_route_opts* opts, float* weights, int32_t* chosen, void* stream) {
    const daq_status rc = route_check(tokens, experts, logits, dtype, ld, opts);
    if (rc != DAQ_OK || tokens == 0) return rc;
    if (!a4(bias) || !weights || !a4(weights) || !chosen || !a4(chosen)) return DAQ_ERR_INVALID_ARG;
    const RouteArgs p{tokens, ld, experts, opts->picks, opts->groups, opts->top_groups, experts / opts->groups, opts->scores == DAQ_SCORES_SIGMOID,
                      opts->renormalize != 0, (double)opts->scale, bias, weights, chosen};
    return dtype == DAQ_BF16 ? launch_route(static_cast<const uint16_t*>(logits), p, (hipStream_t)stream)
                             : launch_route(static_cast<const float*>(logits), p, (hipStream_t)stream);
}

extern "C" daq_status daq_route_backward(int64_t tokens, int32_t experts, const float* dweights, const void* logits, daq_dtype dtype, int64_t ld,
                                         const int32_t* chosen, const daq_route_opts* opts, void* dlogits, int64_t ldd, void* stream) {
    const daq_status rc = route_check(tokens, experts, logits, dtype, ld, opts);
    if (rc != DAQ_OK || tokens == 0) return rc;
    if (!dweights || !a4(dweights) || !chosen || !a4(chosen) || !dlogits || !elem_aligned(dlogits, dtype) || ldd < experts) return DAQ_ERR_INVALID_ARG;
    const RouteBackArgs p{tokens, ld, ldd, experts, opts->picks, opts->scores == DAQ_SCORES_SIGMOID, opts->renormalize != 0, opts->scale, dweights, chosen};
    return dtype == DAQ_BF16 ? launch_back(static_cast<const uint16_t*>(logits), static_cast<uint16_t*>(dlogits), p, (hipStream_t)stream)
                             : launch_back(static_cast<const float*>(logits), static_cast<float*>(dlogits), p, (hipStream_t)stream);
}

extern "C" daq_status daq_experts_plan_workspace(int64_t tokens, int32_t picks, int32_t experts, size_t* bytes) {
    if (!bytes) return DAQ_ERR_INVALID_ARG;
    *bytes = 0;
    if (tokens < 0 || picks <= 0 || experts <= 0) return DAQ_ERR_INVALID_ARG;
    if (experts > kMaxExperts || tokens >= kMaxSlots / picks) return DAQ_ERR_UNSUPPORTED;
    const PlanShape s = plan_shape(tokens * picks);
    if (s.blocks > 1) *bytes = (size_t)round_up((int64_t)s.blocks * experts * 4, 256);
    return DAQ_OK;
}

extern "C" daq_status daq_experts_plan(int64_t tokens, int32_t picks, int32_t experts, const int32_t* chosen, int32_t* counts, int32_t* table,
                                       int32_t* rows, int32_t* place, void* workspace, size_t workspace_bytes, void* stream) {
    size_t need = 0;
    const daq_status rc = daq_experts_plan_workspace(tokens, picks, experts, &need);
    if (rc != DAQ_OK) return rc;
    if (!counts || !a4(counts) || !table || !a4(table)) return DAQ_ERR_INVALID_ARG;
    if (tokens > 0 && (!chosen || !a4(chosen) || !rows || !a4(rows) || !place || !a4(place))) return DAQ_ERR_INVALID_ARG;
    if (need > 0 && (!workspace || workspace_bytes < need || !aligned256(workspace))) return DAQ_ERR_WORKSPACE;
    const PlanShape s = plan_shape(tokens * picks);
    const PlanArgs p{chosen, tokens * picks, experts, s.blocks, s.rounds, static_cast<int32_t*>(workspace), counts, table, rows, place};
    hipStream_t st = (hipStream_t)stream;
    if (s.blocks > 1) DAQ_LAUNCH("plan_count", st, hipLaunchKernelGGL(k_plan_count, dim3((unsigned)s.blocks), dim3(kPlanThreads), 0, st, p));
    DAQ_LAUNCH("plan_place", st, hipLaunchKernelGGL(k_plan_place, dim3((unsigned)s.blocks), dim3(kPlanThreads), 0, st, p));
    return DAQ_OK;
}
