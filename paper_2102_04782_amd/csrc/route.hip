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

// A sigmoid in 64 bits, by the smaller exponential: e^-l they do not hold where l < -709, the sigmoid down to -745.
__device__ __forceinline__ double sigmoid_of(double l) {
    const double ex = exp(-fabs(l));
    return (l >= 0 ? 1.0 : ex) / (1.0 + ex);
}

// Values as whole numbers of the same order, for one instruction a comparison; kNoKey is below all of them (it is a NaN's).
constexpr int kNoKey = (int)0x80000000;
__device__ __forceinline__ int key_of(float v) {
    const int b = __float_as_int(v);
    return b ^ ((b >> 31) & 0x7FFFFFFF);
}
__device__ __forceinline__ float of_key(int k) { return __int_as_float(k ^ ((k >> 31) & 0x7FFFFFFF)); }

// The largest of the wave, to all lanes: six exchanges in registers.
template <int CTRL, int ROWS>
__device__ __forceinline__ int max_with(int v) {
    return max(v, __builtin_amdgcn_update_dpp(kNoKey, v, CTRL, ROWS, 0xF, false));
}
__device__ __forceinline__ int top_of_wave(int v) {
    v = max_with<0x111, 0xF>(v);      // from 1, 2, 4 and 8 lanes before, within 16
    v = max_with<0x112, 0xF>(v);
    v = max_with<0x114, 0xF>(v);
    v = max_with<0x118, 0xF>(v);
    v = max_with<0x142, 0xA>(v);      // from the last lane of the 16, and of the 32, before
    v = max_with<0x143, 0xC>(v);
    return __builtin_amdgcn_readlane(v, 63);
}

// The two largest of a lane and of the one that it exchanges with.
template <typename Swap>
__device__ __forceinline__ void merge_two(int& one, int& two, Swap swap) {
    const int o1 = swap(one), o2 = swap(two);
    two = max(max(two, o2), min(one, o1));
    one = max(one, o1);
}
template <int CTRL>
__device__ __forceinline__ int swapped(int v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, 0xF, 0xF, true); }

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
        for (int i = 0; i < PER; ++i) c[i] = sigmoid_of((double)l[i]);
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
// than 64 bits keep their scores apart, the wave chooses again in 64 bits.  16384 x 256 fp32, sigmoid, bias, 4 of 8 groups, 8 places 34.5 us, where its bytes take 4.  Bound: some 730 vector
// instructions a token, 25 of them for a place: 20 us at one every four cycles of a SIMD, and those in 64 bits take longer; its waves wait a third of their cycles, one
// exchange behind the other.  Four tokens a wave took 40 us (registers).
template <typename T, int PER>
__global__ __launch_bounds__(256) void k_route(const T* logits, RouteArgs p) {
    constexpr float kNone = -__builtin_inff();
    const int lane = threadIdx.x % kWave;
    const int64_t t = (int64_t)blockIdx.x * 4 + threadIdx.x / kWave;
    if (t >= p.tokens) return;
    const T* row = logits + t * p.ld;
    const int first = lane * PER;
    float l[PER];
    load_logits<PER>(row + first, p.experts - first, l);
    bool bad = false;
    float most = kNone;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        l[i] += 0.f;                          // (-0 to 0: they are equals, their keys are not)
        bad |= l[i] != l[i] || (!p.sigmoid && l[i] == __builtin_inff());
        most = fmaxf(most, l[i]);
    }
    most = of_key(top_of_wave(key_of(most)));
    const bool by_score = p.bias || p.groups > 1;
    int c[PER];                               // as keys
    float off = 0.f;                          // what a c may be off by
    if (by_score) {
        float v[PER], top = 1.f;
        if (p.sigmoid) {
#pragma unroll
            for (int i = 0; i < PER; ++i) v[i] = __builtin_amdgcn_rcpf(1.f + __expf(-l[i]));
        } else {
            float sum = 0;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                v[i] = l[i] > kNone ? __expf(l[i] - most) : 0.f;
                sum += v[i];
            }
#pragma unroll
            for (int d = 1; d < kWave; d *= 2) sum += __shfl_xor(sum, d);
            const float over = sum > 0 ? __builtin_amdgcn_rcpf(sum) : 0.f;
#pragma unroll
            for (int i = 0; i < PER; ++i) v[i] *= over;
        }
        if (p.bias) {
            float b[PER];
            load_logits<PER>(p.bias + first, p.experts - first, b);
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                v[i] += b[i];
                top = fmaxf(top, fabsf(v[i]) < __builtin_inff() ? fabsf(v[i]) : 0.f);
                bad |= l[i] > kNone && v[i] != v[i];
            }
            top = of_key(top_of_wave(key_of(top)));
        }
        off = top * 0x1p-19f;
#pragma unroll
        for (int i = 0; i < PER; ++i) c[i] = l[i] > kNone && v[i] > kNone ? key_of(v[i]) : kNoKey;
    } else {
#pragma unroll
        for (int i = 0; i < PER; ++i) c[i] = l[i] > kNone ? key_of(l[i]) : kNoKey;
    }
    bad = __any(bad);
    bool again = false;                       // whether the wave has to choose again
    if (p.groups > 1) {
        const int lanes = p.per_group / PER;
        if (lanes * PER == p.per_group && (lanes & (lanes - 1)) == 0) {
            int one = kNoKey, two = kNoKey;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                two = max(two, min(one, c[i]));
                one = max(one, c[i]);
            }
            if (lanes >= 2) merge_two(one, two, swapped<0xB1>);
            if (lanes >= 4) merge_two(one, two, swapped<0x4E>);
            if (lanes >= 8) merge_two(one, two, swapped<0x141>);
            if (lanes >= 16) merge_two(one, two, swapped<0x140>);
            if (lanes >= 32) merge_two(one, two, [](int v) { return __shfl_xor(v, 16); });
            int total = two == kNoKey ? one : key_of(of_key(one) + of_key(two));
            float before = __builtin_inff();
            uint64_t stay = 0;
            for (int n = 0; n <= p.top_groups && n < p.groups; ++n) {
                const int best = top_of_wave(total);
                if (n == p.top_groups) {
                    again |= best != kNoKey && !(before - of_key(best) > 4 * off);
                    break;
                }
                const uint64_t at = __ballot(total == best);
                if (best != kNoKey) {
                    const uint64_t these = (lanes == kWave ? ~(uint64_t)0 : ((uint64_t)1 << lanes) - 1) << (__builtin_ctzll(at) / lanes * lanes);
                    stay |= these;
                    if (these >> lane & 1) total = kNoKey;
                    before = of_key(best);
                }
            }
            const bool in = stay >> lane & 1;
#pragma unroll
            for (int i = 0; i < PER; ++i) c[i] = in ? (p.bias || c[i] == kNoKey) ? c[i] : key_of(l[i]) : kNoKey;      // (no bias: the logits of those that stay)
        } else {
            again = true;                     // groups that do not lie in whole lanes
        }
    }
    int expert = -1;
    if (!again) {
        // a lane's own in descending order, equals in the order of their indices, which are four bits each of `at`
        constexpr bool kSorted = PER <= 4;
        uint32_t at = 0x3210u;
        if constexpr (kSorted) {
            int ix[PER];
#pragma unroll
            for (int i = 0; i < PER; ++i) ix[i] = i;
#pragma unroll
            for (int n = 0; n < PER - 1; ++n)
#pragma unroll
                for (int i = 0; i < PER - 1 - n; ++i) {
                    const bool swap = c[i] < c[i + 1];
                    const int ci = c[i], xi = ix[i];
                    c[i] = swap ? c[i + 1] : ci;
                    ix[i] = swap ? ix[i + 1] : xi;
                    c[i + 1] = swap ? ci : c[i + 1];
                    ix[i + 1] = swap ? xi : ix[i + 1];
                }
            at = 0;
#pragma unroll
            for (int i = 0; i < PER; ++i) at |= (uint32_t)ix[i] << (4 * i);
        }
        float before = __builtin_inff();
        for (int j = 0; j <= p.picks; ++j) {
            int m = c[0];
            if constexpr (!kSorted) {
#pragma unroll
                for (int i = 1; i < PER; ++i) m = max(m, c[i]);
            }
            const int key = top_of_wave(m);
            if (key == kNoKey) break;
            const float best = of_key(key);
            if (p.bias) again |= !(before - best > 2 * off);
            else again |= (before > best && before - best < 0x1p-36f) || best < (p.sigmoid ? -600.f : most - 600.f) || (p.sigmoid && best > 10.f);
            before = best;
            if (j == p.picks) break;
            const int owner = __builtin_ctzll(__ballot(m == key));
            const bool mine = lane == owner;
            int which;
            if constexpr (kSorted) {
                which = __builtin_amdgcn_readlane((int)at, owner) & 15;
#pragma unroll
                for (int i = 0; i < PER; ++i) c[i] = mine ? (i + 1 < PER ? c[i + 1 < PER ? i + 1 : i] : kNoKey) : c[i];
                at = mine ? at >> 4 : at;
            } else {
                int first_of = 0;
#pragma unroll
                for (int i = PER - 1; i >= 0; --i) first_of = c[i] == key ? i : first_of;
                which = __builtin_amdgcn_readlane(first_of, owner);
#pragma unroll
                for (int i = 0; i < PER; ++i) c[i] = mine && i == which ? kNoKey : c[i];
            }
            expert = lane == j ? owner * PER + which : expert;
        }
    }
    if (again && !bad) expert = choose_exactly<PER>(p, l, most, p.bias, lane);
    // the weights of the places in 64 bits
    const bool there = expert >= 0;
    const double x = there ? (double)logit_at(row + expert) : 0.0;
    double s = 0, total = 1;
    if (p.sigmoid) {
        s = sigmoid_of(x);
    } else {
        // renormalised, they are the chosen ones' own softmax, also where 64 bits hold none of their scores
        if (p.renormalize) most = of_key(top_of_wave(key_of(there ? (float)x : kNone)));
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
    int each, slot;           // tokens of a wave; log2 of the lanes for a token's places
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

__device__ __forceinline__ void store_logits(float* p, const float* v, int left) {
    if (left >= 4) *reinterpret_cast<u32x4_a4*>(p) = __builtin_bit_cast(u32x4, f32x4{v[0], v[1], v[2], v[3]});
    else
        for (int i = 0; i < left; ++i) p[i] = v[i];
}
__device__ __forceinline__ void store_logits(uint16_t* p, const float* v, int left) {
    if (left >= 4) *reinterpret_cast<u32x2_a2*>(p) = u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
    else
        for (int i = 0; i < left; ++i) p[i] = (uint16_t)(pack_bf16(v[i], 0.f) & 0xFFFFu);
}

// What the wave's lanes wrote to LDS before is there for what they read behind (LDS serves a wave in order; the compiler is told to).
__device__ __forceinline__ void lds_in_order() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
}

// Lane n << slot + j has place j of the wave's token n.  The chosen ones' part goes to its place of the row by way of LDS; the others' is zero or, where the softmax is not
// renormalised, needs the row.  Bound: memory and the 64-bit exponentials; 16384 x 256 fp32, 8 places, 7.6 us (17 MB written; the
// logits' lines of the chosen ones are most of them read), softmax without renormalisation 11.7, bfloat16 10.8 (rows read and written, 34 and 17 MB; exponentials in 32 bits).
template <typename T, int PARTS>
__global__ __launch_bounds__(256) void k_route_back(const T* logits, T* dlogits, RouteBackArgs p) {
    __shared__ __attribute__((aligned(16))) float rows[4][PARTS * 256];
    const int lane = threadIdx.x % kWave;
    const int64_t t0 = ((int64_t)blockIdx.x * 4 + threadIdx.x / kWave) * p.each;
    if (t0 >= p.tokens) return;
    float* const row = rows[threadIdx.x / kWave];
    const int tok = lane >> p.slot, j = lane & ((1 << p.slot) - 1);
    const int64_t t = t0 + tok;
    const bool held = tok < p.each && t < p.tokens && j < p.picks;
    const int e = held ? p.chosen[t * p.picks + j] : -1;
    const bool there = e >= 0 && e < p.experts;
    const float g = there ? p.dweights[t * p.picks + j] : 0.f, l = there ? logit_at(logits + t * p.ld + e) : 0.f;
    const bool dense = !p.sigmoid && !p.renormalize;
    float d = 0.f;                             // of the chosen one's logit
    if (!dense) {
        // s and, where it is renormalised, its share of the chosen ones', which may all be tiny: in 64 bits, as in the forward pass
        double s, rest = 1.0;
        if (p.sigmoid) {
            const double ex = exp(-fabs((double)l)), one = 1.0 / (1.0 + ex);
            s = l >= 0 ? one : ex * one;
            rest = l >= 0 ? ex * one : one;
        } else {
            float most = there ? l : -__builtin_inff();
            for (int k = 1; k < 1 << p.slot; k *= 2) most = fmaxf(most, __shfl_xor(most, k));
            s = exp((double)l - (double)most);
        }
        if (!there) s = 0;
        double v = g;
        if (p.renormalize) {
            double total = s, mean = g * s;
            for (int k = 1; k < 1 << p.slot; k *= 2) {
                total += __shfl_xor(total, k);
                mean += __shfl_xor(mean, k);
            }
            if (!(total > 0)) total = 1.0;      // (all scores are zero)
            s /= total;                         // (1 over a sum of sigmoids may be beyond 64 bits)
            v -= mean / total;
        }
        d = (float)(p.scale * v * s * rest);
    }
    // an expert that a token names twice: its places one after the other
    bool twice = false;
    for (int k = 1; k < p.picks; ++k) {
        const int other = __shfl(e, lane - k);      // (of all lanes: a lane that does not take part has nothing to give)
        twice |= there && j >= k && other == e;
    }
    const bool any_twice = __any(twice);
    for (int n = 0; n < p.each && t0 + n < p.tokens; ++n) {
        const bool mine = there && tok == n;
        const bool any = __any(mine);
        float x[PARTS][4], sum = 1.f, back = 0.f;          // dense: the row's exponentials
        if (dense) {
            float m = -__builtin_inff();
#pragma unroll
            for (int i = 0; i < PARTS; ++i) {
                load_logits<4>(logits + (t0 + n) * p.ld + i * 256 + lane * 4, p.experts - i * 256 - lane * 4, x[i]);
#pragma unroll
                for (int k = 0; k < 4; ++k) m = fmaxf(m, x[i][k]);
            }
            m = wave_max(m);
            float total = 0.f;
#pragma unroll
            for (int i = 0; i < PARTS; ++i)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    x[i][k] = expf(x[i][k] - m);
                    total += x[i][k];
                }
            sum = wave_sum(total);
            back = wave_sum(mine ? p.scale * g * (expf(l - m) / sum) : 0.f);
            if (mine) d = p.scale * g;
        }
#pragma unroll
        for (int i = 0; i < PARTS; ++i) *reinterpret_cast<f32x4*>(row + i * 256 + lane * 4) = f32x4{0, 0, 0, 0};
        lds_in_order();
        if (!any_twice) {
            if (mine) row[e] = d;
        } else {
            for (int k = 0; k < p.picks; ++k) {
                if (mine && j == k) row[e] += d;
                lds_in_order();
            }
        }
        lds_in_order();
#pragma unroll
        for (int i = 0; i < PARTS; ++i) {
            f32x4 z = *reinterpret_cast<const f32x4*>(row + i * 256 + lane * 4);
            if (dense) {
#pragma unroll
                for (int k = 0; k < 4; ++k) z[k] = any ? x[i][k] / sum * (z[k] - back) : 0.f;
            }
            const float v[4] = {z[0], z[1], z[2], z[3]};
            store_logits(dlogits + (t0 + n) * p.ldd + i * 256 + lane * 4, v, p.experts - i * 256 - lane * 4);
        }
        lds_in_order();
    }
}

// ---- the order of the rows --------------------------------------------------------------------
// A workgroup takes a run of slots, 1024 at a time.  counts[block][expert] by a first launch; the second adds up what stands before its own
// run and places it.  Within a wave a slot's rank among those of its expert comes from ten votes, one a bit of the expert's number; no atomics decide an order.
// Bound: launches and the waits of a dozen steps one behind the other; 131072 slots, 256 experts 4.2 + 12 us, up to 4096 slots one launch of 5.
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

// Of four values of each of 1024 threads: the sums of what stands before each thread, and the totals, to all.
__device__ __forceinline__ void before_me(const int (&v)[4], int (*per_wave)[kPlanWaves], int (&first)[4], int (&total)[4]) {
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    int sum[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        sum[k] = v[k];
#pragma unroll
        for (int d = 1; d < kWave; d *= 2) {
            const int o = __shfl_up(sum[k], d);
            if (lane >= d) sum[k] += o;
        }
        if (lane == kWave - 1) per_wave[k][wave] = sum[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        first[k] = sum[k] - v[k];
        total[k] = 0;
#pragma unroll
        for (int w = 0; w < kPlanWaves; ++w) {
            const int n = per_wave[k][w];
            first[k] += w < wave ? n : 0;
            total[k] += n;
        }
    }
}

__global__ __launch_bounds__(kPlanThreads) void k_plan_place(PlanArgs p) {
    __shared__ int next[kMaxExperts];                       // the row of an expert's next slot
    __shared__ __attribute__((aligned(16))) uint16_t ranks[kPlanWaves][kMaxExperts];     // slots of an expert in a wave of this round
    __shared__ int per_wave[4][kPlanWaves];
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
    } else {
        // the runs shared among as many threads of an expert as there are, sixteen asked for at a time
        int* sums = reinterpret_cast<int*>(&ranks[0][0]);   // [part][all, before][expert]
        const int wide = (p.experts + kWave - 1) / kWave * kWave, parts = kPlanThreads / wide, part = threadIdx.x / wide, e = threadIdx.x - part * wide;
        if (part < parts && e < p.experts) {
            int a = 0, f = 0;
            for (int b0 = part; b0 < p.blocks; b0 += 16 * parts) {
                int n[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) n[i] = b0 + i * parts < p.blocks ? p.per_block[(int64_t)(b0 + i * parts) * p.experts + e] : 0;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    a += n[i];
                    f += b0 + i * parts < (int)blockIdx.x ? n[i] : 0;
                }
            }
            sums[(part * 2) * wide + e] = a;
            sums[(part * 2 + 1) * wide + e] = f;
        }
        __syncthreads();
        if (e0 < p.experts) {
            for (int i = 0; i < parts; ++i) {
                all += sums[(i * 2) * wide + e0];
                before += sums[(i * 2 + 1) * wide + e0];
            }
        }
        __syncthreads();
    }
    int first[4], totals[4];
    before_me({all, (all + 255) / 256, (all + 127) / 128, (all + 63) / 64}, per_wave, first, totals);
    static_assert(kTableRows == 0 && kTable256 == 1 && kTable128 == 2 && kTable64 == 3, "in this order");
    const int total = totals[0];
    if (e0 < p.experts) next[e0] = first[0] + before;
    if (blockIdx.x == 0) {
        if (e0 < p.experts) p.counts[e0] = all;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (e0 < p.experts) p.table[k * (p.experts + 1) + e0] = first[k];
            if (e0 == 0) p.table[k * (p.experts + 1) + p.experts] = totals[k];
        }
    }
    for (int r = 0; r < p.rounds; ++r) {
        for (int w = threadIdx.x / 128; w < kPlanWaves; w += kPlanThreads / 128)          // 16 bytes a thread
            if (threadIdx.x % 128 * 8 < (unsigned)p.experts) *reinterpret_cast<u32x4*>(&ranks[w][threadIdx.x % 128 * 8]) = u32x4{0, 0, 0, 0};
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
    const auto kernel = p.experts <= 256 ? k_route_back<T, 1> : p.experts <= 512 ? k_route_back<T, 2> : k_route_back<T, 4>;
    DAQ_LAUNCH("route_back", st, hipLaunchKernelGGL(kernel, dim3((unsigned)ceil_div(p.tokens, 4 * p.each)), dim3(256), 0, st, logits, dlogits, p));
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
    if (!grid_ok(ceil_div(tokens, 4), 256)) return DAQ_ERR_UNSUPPORTED;
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
    // what is computed in 64 bits takes a wave as long for one token's places as for several's: four tokens a wave, once there are enough of them (16384 x 256,
    // 8 places, 7.6 us instead of 12)
    const int slot = opts->picks <= 8 ? 3 : opts->picks <= 16 ? 4 : 5, each = tokens >= 8192 ? std::min(4, kWave >> slot) : 1;
    if (!grid_ok(ceil_div(tokens, 4 * each), 256)) return DAQ_ERR_UNSUPPORTED;
    const RouteBackArgs p{tokens, ld, ldd, experts, opts->picks, opts->scores == DAQ_SCORES_SIGMOID, opts->renormalize != 0, each, slot, opts->scale, dweights, chosen};
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
