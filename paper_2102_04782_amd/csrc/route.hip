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

// A wave a token; lane l has the experts l, l + 64, ..
template <typename T, int PER>
__global__ __launch_bounds__(256) void k_route(const T* logits, RouteArgs p) {
    constexpr double kNone = -__builtin_inf();
    const int lane = threadIdx.x % kWave;
    const int64_t t = (int64_t)blockIdx.x * 4 + threadIdx.x / kWave;
    if (t >= p.tokens) return;
    double s[PER], c[PER];
    float l[PER];
    bool bad = false;
    float most = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int e = i * kWave + lane;
        l[i] = e < p.experts ? logit_at(logits + t * p.ld + e) : -__builtin_inff();
        bad |= l[i] != l[i] || (!p.sigmoid && l[i] == __builtin_inff());
        most = fmaxf(most, l[i]);
    }
    if (p.sigmoid) {
#pragma unroll
        for (int i = 0; i < PER; ++i) s[i] = 1.0 / (1.0 + exp(-(double)l[i]));
    } else {
#pragma unroll
        for (int d = 1; d < kWave; d *= 2) most = fmaxf(most, __shfl_xor(most, d));
        double sum = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            s[i] = l[i] > -__builtin_inff() ? exp((double)l[i] - (double)most) : 0.0;
            sum += s[i];
        }
#pragma unroll
        for (int d = 1; d < kWave; d *= 2) sum += __shfl_xor(sum, d);
#pragma unroll
        for (int i = 0; i < PER; ++i) s[i] = sum > 0 ? s[i] / sum : 0.0;
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int e = i * kWave + lane;
        c[i] = kNone;
        if (e < p.experts && l[i] > -__builtin_inff()) c[i] = p.bias ? s[i] + (double)p.bias[e] : s[i];
        if (c[i] != c[i]) bad = true;
    }
    bad = __any(bad);
    if (p.groups > 1 && !bad) {
        double total = kNone;                 // of group `lane`
        for (int g = 0; g < p.groups; ++g) {
            double one = kNone, two = kNone;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int e = i * kWave + lane;
                if (e / p.per_group != g) continue;
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
            const int g = (i * kWave + lane) / p.per_group;
            if (g >= p.groups || !(stay >> g & 1)) c[i] = kNone;
        }
    }
    double mine = 0;                          // lane j: the score of place j
    int expert = -1;
    for (int j = 0; j < p.picks; ++j) {
        double best = kNone;
        int at = 0x7FFFFFFF;
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (c[i] > best) {
                best = c[i];
                at = i * kWave + lane;
            }
        best_of_wave(best, at);
        double score = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (i * kWave + lane == at) {
                score = s[i];
                c[i] = kNone;
            }
        const bool any = best > kNone;
        score = __shfl(score, at % kWave);
        if (lane == j && any) {
            mine = score;
            expert = at;
        }
    }
    double sum = mine;
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) sum += __shfl_xor(sum, d);
    if (lane < p.picks) {
        double w = mine * p.scale;
        if (p.renormalize) w = sum > 0 ? mine / sum * p.scale : 0.0;
        p.weights[t * p.picks + lane] = bad ? __builtin_nanf("") : (float)w;
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
