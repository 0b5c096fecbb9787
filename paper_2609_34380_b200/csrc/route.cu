// Routing: the experts of each token and their weights, from the router's logits.
//
//   s = softmax(x) or sigmoid(x);  c = s + bias;  groups by the sum of their two largest c;  top-k of c;  w = s / sum * scale
//
// One warp per token.  A choice is a whole number, and two of the values that it compares may be nearer than 32 bits tell apart, so it is made as in 64 bits.
// 64-bit arithmetic throughout is bound by its exponentials and butterflies (16384 tokens, 256 experts in 8 groups: 129 us).  So a
// row is first done in 32 bits, with the gaps between the values that the choice rests on held against a bound on their errors; only a row with a
// smaller gap, or with anything out of the ordinary (infinities, scores that vanish), is done again in 64 bits -- well below one row in a
// hundred.  Without bias and groups the scores rise with the logits, and the logits themselves are compared, exactly.
//   * Lane i holds neighbouring experts (16 of them at most come by two loads), so that a group is a stretch of lanes, and of equal
//     values the lower lane's is the lower index.
//   * top-k: the lanes' best as whole numbers in the floats' order, one warp-wide maximum and one ballot a choice.
//   * The weights need one accurate exponential a lane: lane j has choice j.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "dps_internal.h"
#include "sm100.cuh"
#include "step_ops.h"

namespace dps {

namespace {

constexpr int kThreads = 128;
constexpr int kWarps = kThreads / 32;
constexpr unsigned kAll = 0xFFFFFFFFu;

struct RouteParams {
    const void* logits;
    int64_t stride, tokens;
    const float* bias;
    int32_t* token_of_row;
    int32_t* expert_of_row;
    float* weights;
    int* status;
    int experts, groups, top_groups, top_k;
    int per_lane, group_lanes;     // experts of a lane; lanes of a group, a power of two (0: groups that are no stretches of so many lanes)
    float scale;
    bool sigmoid, renormalise;
};

__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(__half v) { return __half2float(v); }
__device__ __forceinline__ float widen(__nv_bfloat16 v) { return __bfloat162float(v); }

// The larger value, of equal ones the lower index, of the whole warp; index INT_MAX where there is none.
__device__ __forceinline__ void warp_best(double& value, int& index) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const double v = __shfl_xor_sync(kAll, value, o);
        const int i = __shfl_xor_sync(kAll, index, o);
        if (i != INT32_MAX && (index == INT32_MAX || v > value || (v == value && i < index))) {
            value = v;
            index = i;
        }
    }
}

// One row in 64 bits, whatever it holds; lane i has experts i, i + 32, ..
template <typename T, int PER>
__device__ __noinline__ void route_in_64_bits(const RouteParams& p, int64_t token) {
    const int lane = threadIdx.x & 31;
    const T* row = static_cast<const T*>(p.logits) + token * p.stride;

    double score[PER], choice[PER];
    double top = -INFINITY;
    bool bad = false;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int e = i * 32 + lane;
        score[i] = e < p.experts ? (double)widen(row[e]) : -INFINITY;
        bad |= score[i] != score[i];
        top = fmax(top, score[i]);
    }
    if (p.sigmoid) {
#pragma unroll
        for (int i = 0; i < PER; ++i) score[i] = 1.0 / (1.0 + exp(-score[i]));
    } else {
        for (int o = 16; o > 0; o >>= 1) top = fmax(top, __shfl_xor_sync(kAll, top, o));
        double sum = 0.0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            score[i] = i * 32 + lane < p.experts ? exp(score[i] - top) : 0.0;
            sum += score[i];
        }
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(kAll, sum, o);
#pragma unroll
        for (int i = 0; i < PER; ++i) score[i] /= sum;
    }
    unsigned open = 0;                                      // this lane's experts that may be taken
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int e = i * 32 + lane;
        choice[i] = score[i];
        if (e < p.experts) {
            if (p.bias != nullptr) choice[i] += (double)p.bias[e];
            bad |= choice[i] != choice[i];
            open |= 1u << i;
        }
    }
    const auto give_up = [&] {
        if (lane == 0) atomicExch(p.status, (int)DPS_ERR_DATA);
        if (lane < p.top_k) {
            const int64_t at = token * p.top_k + lane;
            p.expert_of_row[at] = -1;
            p.weights[at] = 0.f;
            if (p.token_of_row != nullptr) p.token_of_row[at] = (int32_t)token;
        }
    };
    if (__any_sync(kAll, bad)) return give_up();
    if (p.top_groups < p.groups) {
        const int size = p.experts / p.groups;
        double worth = -INFINITY;                           // of group `lane`
        for (int g = 0; g < p.groups; ++g) {
            double one = -INFINITY, two = -INFINITY;        // the two largest of it
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int e = i * 32 + lane;
                if (e < p.experts && e / size == g) {
                    two = fmax(two, fmin(one, choice[i]));
                    one = fmax(one, choice[i]);
                }
            }
            for (int o = 16; o > 0; o >>= 1) {
                const double a = __shfl_xor_sync(kAll, one, o), b = __shfl_xor_sync(kAll, two, o);
                two = fmax(fmax(two, b), fmin(one, a));
                one = fmax(one, a);
            }
            if (lane == g) worth = size > 1 ? one + two : one;
        }
        if (__any_sync(kAll, worth != worth)) return give_up();     // +Inf and -Inf among the choices
        unsigned kept = 0;
        for (int j = 0; j < p.top_groups; ++j) {
            double v = worth;
            int g = lane < p.groups && !((kept >> lane) & 1u) ? lane : INT32_MAX;
            warp_best(v, g);
            kept |= 1u << g;
        }
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int e = i * 32 + lane;
            if (e < p.experts && !((kept >> (e / size)) & 1u)) open &= ~(1u << i);
        }
    }
    double sum = 0.0, mine = 0.0;                           // lane j keeps choice j
    int taken = -1;
    for (int j = 0; j < p.top_k; ++j) {
        double v = 0.0, s = 0.0;
        int at = INT32_MAX;
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (((open >> i) & 1u) && (at == INT32_MAX || choice[i] > v)) {
                v = choice[i];
                s = score[i];
                at = i * 32 + lane;
            }
        int e = at;
        warp_best(v, e);
        const int owner = e & 31;
        s = __shfl_sync(kAll, s, owner);
        if (lane == owner) open &= ~(1u << (e >> 5));
        if (lane == j) {
            taken = e;
            mine = s;
        }
        sum += s;
    }
    if (lane < p.top_k) {
        const int64_t at = token * p.top_k + lane;
        double w = mine;
        if (p.renormalise) w = sum > 0.0 ? w / sum : 0.0;
        p.expert_of_row[at] = taken;
        p.weights[at] = (float)(w * p.scale);
        if (p.token_of_row != nullptr) p.token_of_row[at] = (int32_t)token;
    }
}

// Floats as whole numbers in their order; 0 is below all of them.
__device__ __forceinline__ unsigned ordered(float v) {
    const unsigned u = __float_as_uint(v);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float from_ordered(unsigned u) { return __uint_as_float(u & 0x80000000u ? u & 0x7FFFFFFFu : ~u); }
__device__ __forceinline__ float exp_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x * 1.4426950408889634f));
    return y;
}

// PER neighbouring logits, by the widest loads that the row's address allows.
template <typename T, int PER>
__device__ __forceinline__ void load_logits(const T* at, int count, float (&x)[PER]) {
    constexpr int kBytes = PER * (int)sizeof(T), kWide = kBytes < 16 ? kBytes : 16;
    if (count == PER && (reinterpret_cast<uintptr_t>(at) & (kWide - 1)) == 0) {
        union {
            T values[PER];
            uint4 v16[kBytes < 16 ? 1 : kBytes / 16];
            uint2 v8;
            uint32_t v4;
        } u;
        if (kBytes >= 16) {
#pragma unroll
            for (int i = 0; i < kBytes / 16; ++i) u.v16[i] = reinterpret_cast<const uint4*>(at)[i];
        } else if (kBytes == 8) u.v8 = *reinterpret_cast<const uint2*>(at);
        else if (kBytes == 4) u.v4 = *reinterpret_cast<const uint32_t*>(at);
        else u.values[0] = at[0];
#pragma unroll
        for (int i = 0; i < PER; ++i) x[i] = widen(u.values[i]);
    } else {
#pragma unroll
        for (int i = 0; i < PER; ++i) x[i] = i < count ? widen(at[i]) : 0.f;
    }
}

template <typename T, int PER>
__global__ void __launch_bounds__(kThreads) route_experts_kernel(const RouteParams p) {
    sm100::grid_launch_dependents();
    sm100::grid_dependency_wait();
    const int lane = threadIdx.x & 31;
    const int first = min(lane * p.per_lane, p.experts), count = min(p.per_lane, p.experts - first);
    float bias[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) bias[i] = p.bias != nullptr && i < count ? p.bias[first + i] : 0.f;
    const bool by_groups = p.top_groups < p.groups, direct = p.bias == nullptr && !by_groups;
    const int group = p.group_lanes > 0 ? lane / p.group_lanes : 0;

    for (int64_t token = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5); token < p.tokens; token += (int64_t)gridDim.x * kWarps) {
        float x[PER];
        load_logits<T, PER>(static_cast<const T*>(p.logits) + token * p.stride + first, count, x);
        bool odd = by_groups && p.group_lanes == 0;         // this row is none for 32 bits
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (i < count) {
                odd |= !(fabsf(x[i]) < INFINITY) || !(fabsf(bias[i]) < INFINITY);
                top = fmaxf(top, x[i]);
            }
        if (__any_sync(kAll, odd)) {
            route_in_64_bits<T, PER>(p, token);
            continue;
        }
        top = from_ordered(__reduce_max_sync(kAll, ordered(top)));
        float scale = 1.f, bound = 4e-6f;                   // softmax: 1 / sum;  on the error of a choice value, besides its own rounding
        unsigned key[PER];
        if (direct && (p.sigmoid || p.renormalise)) {
#pragma unroll
            for (int i = 0; i < PER; ++i) key[i] = i < count ? ordered(x[i]) : 0u;
        } else {
            float score[PER], sum = 0.f;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                score[i] = p.sigmoid ? __fdividef(1.f, 1.f + exp_approx(-x[i])) : i < count ? exp_approx(x[i] - top) : 0.f;
                sum += score[i];
            }
            if (!p.sigmoid) {
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(kAll, sum, o);
                scale = 1.f / sum;
                bound *= scale;                             // (the largest score)
            }
#pragma unroll
            for (int i = 0; i < PER; ++i) key[i] = i < count ? ordered(direct ? x[i] : score[i] * scale + bias[i]) : 0u;
        }
        bool close = false;
        if (by_groups) {
            float one = -INFINITY, two = -INFINITY;         // the two largest of the lane, then of its group
#pragma unroll
            for (int i = 0; i < PER; ++i)
                if (i < count) {
                    const float c = from_ordered(key[i]);
                    two = fmaxf(two, fminf(one, c));
                    one = fmaxf(one, c);
                }
            for (int o = 1; o < p.group_lanes; o <<= 1) {
                const float a = __shfl_xor_sync(kAll, one, o), b = __shfl_xor_sync(kAll, two, o);
                two = fmaxf(fmaxf(two, b), fminf(one, a));
                one = fmaxf(one, a);
            }
            const float worth = two == -INFINITY ? one : one + two;
            int better = 0;                                 // groups in front of this one
            for (int g = 0; g < p.groups; ++g) {
                const float other = __shfl_sync(kAll, worth, g * p.group_lanes);
                if (g != group) {
                    better += other > worth;
                    close |= fabsf(other - worth) <= 2.f * bound + 1e-6f * (fabsf(one) + fabsf(two == -INFINITY ? 0.f : two));
                }
            }
            if (better >= p.top_groups) {
#pragma unroll
                for (int i = 0; i < PER; ++i) key[i] = 0u;
            }
            close = __any_sync(kAll, close && group < p.groups);
        }
        unsigned mine = 0u;                                 // the lane's best
#pragma unroll
        for (int i = 0; i < PER; ++i) mine = max(mine, key[i]);
        int taken = -1;                                     // lane j keeps choice j
        float logit = 0.f, last = 0.f;
        for (int j = 0; j <= p.top_k; ++j) {
            const unsigned best = __reduce_max_sync(kAll, mine);
            if (best == 0u) break;                          // (behind the last choice: no other expert is left)
            const float value = from_ordered(best), gap = last - value;
            if (j > 0) close |= direct ? gap > 0.f && gap < 1e-9f : gap <= 2.f * bound + 2e-7f * (fabsf(value) + fabsf(last));
            last = value;
            if (j == p.top_k) break;
            const int owner = __ffs(__ballot_sync(kAll, mine == best)) - 1;
            int at = 0;
            float v = 0.f;
            if (lane == owner) {
                mine = 0u;
#pragma unroll
                for (int i = PER - 1; i >= 0; --i)
                    if (key[i] == best) {                   // the first of equal ones
                        at = i;
                        v = x[i];
                    }
#pragma unroll
                for (int i = 0; i < PER; ++i) {
                    if (i == at) key[i] = 0u;
                    mine = max(mine, key[i]);
                }
            }
            at = __shfl_sync(kAll, at, owner);
            v = __shfl_sync(kAll, v, owner);
            if (lane == j) {
                taken = owner * p.per_lane + at;
                logit = v;
            }
        }
        // the weights: of the choices alone if they are divided by their sum
        const bool chosen = lane < p.top_k;
        const float low = from_ordered(__reduce_min_sync(kAll, chosen ? ordered(logit) : 0xFFFFFFFFu)),
                    high = from_ordered(__reduce_max_sync(kAll, chosen ? ordered(logit) : 0u));
        // scores that 64 bits cannot tell apart (1 - e^-x beyond 16), or that vanish
        if (p.sigmoid) close |= (direct && high >= 16.f) || low <= -60.f;
        else close |= low - top <= -60.f;
        if (close) {
            route_in_64_bits<T, PER>(p, token);
            continue;
        }
        float w = 0.f;
        if (chosen) w = p.sigmoid ? 1.f / (1.f + expf(-logit)) : p.renormalise ? expf(logit - high) : expf(logit - top) * scale;
        if (p.renormalise) {
            float sum = w;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(kAll, sum, o);
            w /= sum;
        }
        if (chosen) {
            const int64_t at = token * p.top_k + lane;
            p.expert_of_row[at] = taken;
            p.weights[at] = w * p.scale;
            if (p.token_of_row != nullptr) p.token_of_row[at] = (int32_t)token;
        }
    }
}

template <typename T>
cudaError_t launch(const RouteParams& p, cudaStream_t stream) {
    cudaLaunchConfig_t cfg = {};
    const int64_t ctas = (p.tokens + kWarps - 1) / kWarps, resident = (int64_t)sm_count() * 12;
    cfg.gridDim = dim3((unsigned)(ctas < resident ? ctas : resident));
    cfg.blockDim = dim3(kThreads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const int per = p.per_lane;
    const cudaError_t e = per <= 1    ? cudaLaunchKernelEx(&cfg, route_experts_kernel<T, 1>, p)
                          : per <= 2  ? cudaLaunchKernelEx(&cfg, route_experts_kernel<T, 2>, p)
                          : per <= 4  ? cudaLaunchKernelEx(&cfg, route_experts_kernel<T, 4>, p)
                          : per <= 8  ? cudaLaunchKernelEx(&cfg, route_experts_kernel<T, 8>, p)
                          : per <= 16 ? cudaLaunchKernelEx(&cfg, route_experts_kernel<T, 16>, p)
                                      : cudaLaunchKernelEx(&cfg, route_experts_kernel<T, 32>, p);
    if (e == cudaSuccess) count_launch();
    return e;
}

}  // namespace

cudaError_t launch_route_experts(const void* logits, int64_t logits_stride, int32_t type, int64_t tokens, int32_t experts, const float* bias,
                                 int32_t scoring, int32_t groups, int32_t top_groups, int32_t top_k, bool renormalise, float scale,
                                 int32_t* token_of_row, int32_t* expert_of_row, float* weights, int* status, cudaStream_t stream) {
    RouteParams p;
    p.logits = logits;
    p.stride = logits_stride;
    p.tokens = tokens;
    p.bias = bias;
    p.token_of_row = token_of_row;
    p.expert_of_row = expert_of_row;
    p.weights = weights;
    p.status = status;
    p.experts = experts;
    p.groups = groups;
    p.top_groups = top_groups;
    p.top_k = top_k;
    p.per_lane = (experts + 31) / 32;
    const int size = experts / groups, lanes = size / p.per_lane;
    p.group_lanes = size % p.per_lane == 0 && (lanes & (lanes - 1)) == 0 ? lanes : 0;
    p.scale = scale;
    p.sigmoid = scoring == DPS_SCORE_SIGMOID;
    p.renormalise = renormalise;
    return type == DPS_TYPE_FP16 ? launch<__half>(p, stream) : type == DPS_TYPE_BF16 ? launch<__nv_bfloat16>(p, stream) : launch<float>(p, stream);
}

}  // namespace dps
