// Routing: the experts of each token and their weights, from the router's logits.
//
//   s = softmax(x) or sigmoid(x);  c = s + bias;  groups by the sum of their two largest c;  top-k of c;  w = s / sum * scale
//
// One warp per token.  A choice is a whole number, and two of the values that it compares may be nearer than 32 bits tell apart, so it is made as in 64 bits.
// 64-bit arithmetic throughout is bound by its exponentials and butterflies (16384 tokens, 256 experts in 8 groups: 129 us).  So a
// row is first done in 32 bits, with the gaps between the values that the choice rests on held against a bound on their errors; only a row with a
// smaller gap, or with anything out of the ordinary (infinities, scores that vanish or saturate), is done again in 64 bits -- well below one row in a
// hundred of ordinary logits.  Without bias and groups the scores rise with the logits, and the 32-bit rows compare the logits themselves, which is exact; scores
// that are equal in 64 bits (sigmoids of 38 and 45) are left to the 64-bit rows, where they tie.  Groups that are no power of two of lanes at ceil(experts / 32)
// experts a lane (72 in 8, 100 in 10), or that have an infinite bias, have every row done in 64 bits.
//   * Lane i holds neighbouring experts (16 of them at most come by two loads), so that a group is a stretch of lanes, and of equal
//     values the lower lane's is the lower index.
//   * top-k: the lanes' best as whole numbers in the floats' order, one warp-wide maximum and one ballot a choice.
//   * The weights need one accurate exponential a lane: lane j has choice j.
// 16384 tokens, 256 experts in 8 groups, sigmoid and bias: 26 us, 900 warp instructions a row with the issue slots 64 % busy (10 MB, 1.5 us of HBM; so bound
// by instructions).  Maxima over all of a lane's values for each choice instead of sorted lists took 58 us, gaps looked over choice by choice (and slower rows in 64 bits) 44; blocks of 32 or 64
// threads, or one per four tokens, 25.7 to 28.2.  8 tokens of 8 experts: 2.0 us, a launch.  16384 tokens without groups or bias, softmax: 12.1 us for 128 experts, 10.6 for
// 64.  With groups that have every row done in 64 bits: 72 experts in 8 84 us, 120 in 8 91, 100 in 10 105.
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

// Numbers as whole numbers in their order; 0 is below all of them.  (v + 0 makes one of the two zeros.)
__device__ __forceinline__ uint64_t ordered(double v) {
    const uint64_t u = (uint64_t)__double_as_longlong(v + 0.0);
    return u >> 63 ? ~u : u | 0x8000000000000000ull;
}
__device__ __forceinline__ uint64_t warp_max(uint64_t v) {
    const unsigned high = __reduce_max_sync(kAll, (unsigned)(v >> 32));
    const unsigned low = __reduce_max_sync(kAll, (unsigned)(v >> 32) == high ? (unsigned)v : 0u);
    return (uint64_t)high << 32 | low;
}

// One row in 64 bits, whatever it holds.  Lane i has p.per_lane neighbouring experts, as below, so that of equal values the lower lane's is the lower index.
template <typename T, int PER>
__device__ __noinline__ void route_in_64_bits(const RouteParams& p, int64_t token) {
    const int lane = threadIdx.x & 31;
    const int first = min(lane * p.per_lane, p.experts), count = min(p.per_lane, p.experts - first);
    const T* row = static_cast<const T*>(p.logits) + token * p.stride;

    double score[PER], top = -INFINITY;
    bool bad = false;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        score[i] = i < count ? (double)widen(row[first + i]) : -INFINITY;
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
            score[i] = i < count ? exp(score[i] - top) : 0.0;
            sum += score[i];
        }
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(kAll, sum, o);
#pragma unroll
        for (int i = 0; i < PER; ++i) score[i] /= sum;
    }
    uint64_t key[PER];                                      // 0: none, or not to be taken any more
    double one = -INFINITY, two = -INFINITY;                // the lane's two largest choice values
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        key[i] = 0;
        if (i < count) {
            const double c = p.bias != nullptr ? score[i] + (double)p.bias[first + i] : score[i];
            bad |= c != c;
            key[i] = ordered(c);
            two = fmax(two, fmin(one, c));
            one = fmax(one, c);
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
        if (p.group_lanes > 0) {
            for (int o = 1; o < p.group_lanes; o <<= 1) {
                const double a = __shfl_xor_sync(kAll, one, o), b = __shfl_xor_sync(kAll, two, o);
                two = fmax(fmax(two, b), fmin(one, a));
                one = fmax(one, a);
            }
            worth = __shfl_sync(kAll, size > 1 ? one + two : one, lane * p.group_lanes & 31);
        } else {
            for (int g = 0; g < p.groups; ++g) {
                one = two = -INFINITY;
#pragma unroll
                for (int i = 0; i < PER; ++i)
                    if (i < count && first + i >= g * size && first + i < (g + 1) * size) {
                        const double c = p.bias != nullptr ? score[i] + (double)p.bias[first + i] : score[i];
                        two = fmax(two, fmin(one, c));
                        one = fmax(one, c);
                    }
                for (int o = 16; o > 0; o >>= 1) {
                    const double a = __shfl_xor_sync(kAll, one, o), b = __shfl_xor_sync(kAll, two, o);
                    two = fmax(fmax(two, b), fmin(one, a));
                    one = fmax(one, a);
                }
                if (lane == g) worth = size > 1 ? one + two : one;
            }
        }
        if (__any_sync(kAll, lane < p.groups && worth != worth)) return give_up();       // +Inf and -Inf among the choices
        uint64_t value = lane < p.groups ? ordered(worth) : 0;
        unsigned kept = 0;
        for (int j = 0; j < p.top_groups; ++j) {
            const uint64_t best = warp_max(value);
            const int g = __ffs(__ballot_sync(kAll, value == best)) - 1;
            kept |= 1u << g;
            if (lane == g) value = 0;
        }
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (i < count && !((kept >> ((first + i) / size)) & 1u)) key[i] = 0;
    }
    double sum = 0.0, mine = 0.0;                           // lane j keeps choice j
    int taken = -1;
    for (int j = 0; j < p.top_k; ++j) {
        uint64_t local = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) local = max(local, key[i]);
        const uint64_t best = warp_max(local);
        const int owner = __ffs(__ballot_sync(kAll, local == best)) - 1;
        int at = 0;
        double s = 0.0;
#pragma unroll
        for (int i = PER - 1; i >= 0; --i)
            if (key[i] == best) {                           // the first of equal ones
                at = i;
                s = score[i];
            }
        if (lane == owner) {
#pragma unroll
            for (int i = 0; i < PER; ++i)
                if (i == at) key[i] = 0;
        }
        at = __shfl_sync(kAll, at, owner);
        s = __shfl_sync(kAll, s, owner);
        if (lane == j) {
            taken = owner * p.per_lane + at;
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

// Descending, by exchanges in pairs (a bitonic network).
template <int PER>
__device__ __forceinline__ void sort_down(unsigned (&key)[PER]) {
#pragma unroll
    for (int size = 2; size <= PER; size *= 2)
#pragma unroll
        for (int step = size / 2; step > 0; step /= 2)
#pragma unroll
            for (int i = 0; i < PER; ++i)
                if ((i & step) == 0) {
                    const unsigned x = key[i], y = key[i + step];
                    key[i] = (i & size) == 0 ? max(x, y) : min(x, y);
                    key[i + step] = (i & size) == 0 ? min(x, y) : max(x, y);
                }
}

// A lane's values are sorted once, with the expert's number in the lane (the lower the larger) in their lowest bits: a choice then costs a
// maximum, a ballot and a step in one lane's list.  The bits are no loss to FP16 and BF16 logits, whose 32-bit forms end in zeros.
template <typename T, int PER>
__global__ void __launch_bounds__(kThreads, PER <= 8 ? 8 : 4) route_experts_kernel(const RouteParams p) {
    sm100::grid_launch_dependents();
    sm100::grid_dependency_wait();
    constexpr unsigned kIndex = PER - 1;                    // PER is a power of two
    constexpr float kCut = PER * 1.2e-7f;                   // what the lowest bits may take from a value, relative to it
    const int lane = threadIdx.x & 31;
    const int first = min(lane * p.per_lane, p.experts), count = min(p.per_lane, p.experts - first);
    const bool by_groups = p.top_groups < p.groups, direct = p.bias == nullptr && !by_groups;
    const int group = p.group_lanes > 0 ? lane / p.group_lanes : 0;
    float bias[PER], odd_bias = 0.f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        bias[i] = p.bias != nullptr && i < count ? p.bias[first + i] : 0.f;
        odd_bias += bias[i] * 0.f;                          // NaN from one that is not finite
    }
    const bool never = (by_groups && p.group_lanes == 0) || odd_bias != 0.f;         // (NaN differs from 0)

    for (int64_t token = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5); token < p.tokens; token += (int64_t)gridDim.x * kWarps) {
        const T* const row = static_cast<const T*>(p.logits) + token * p.stride;
        float x[PER], odd = 0.f;
        load_logits<T, PER>(row + first, count, x);
#pragma unroll
        for (int i = 0; i < PER; ++i) odd += x[i] * 0.f;
        if (__any_sync(kAll, never || odd != 0.f)) {
            route_in_64_bits<T, PER>(p, token);
            continue;
        }
        float top = 0.f, scale = 1.f, bound = 5e-7f;        // softmax: the largest logit, 1 / sum;  on the error of a score
        unsigned key[PER];
        if (!p.sigmoid) {
            top = -INFINITY;
#pragma unroll
            for (int i = 0; i < PER; ++i)
                if (i < count) top = fmaxf(top, x[i]);
            top = from_ordered(__reduce_max_sync(kAll, ordered(top)));
        }
        if (direct && (p.sigmoid || p.renormalise)) {
#pragma unroll
            for (int i = 0; i < PER; ++i) key[i] = ordered(x[i] + 0.f);      // (one of the two zeros)
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
                bound = 2e-6f * scale;                      // (the largest score is scale; the smaller ones are off by less)
            }
#pragma unroll
            for (int i = 0; i < PER; ++i) key[i] = ordered(direct ? x[i] + 0.f : score[i] * scale + bias[i]);
        }
#pragma unroll
        for (int i = 0; i < PER; ++i) key[i] = i < count ? (key[i] & ~kIndex) | (kIndex - i) : 0u;
        sort_down<PER>(key);
        bool close = false;
        if (by_groups) {
            float one = key[0] != 0u ? from_ordered(key[0]) : -INFINITY, two = PER > 1 && key[PER > 1] != 0u ? from_ordered(key[PER > 1]) : -INFINITY;
            for (int o = 1; o < p.group_lanes; o <<= 1) {
                const float a = __shfl_xor_sync(kAll, one, o), b = __shfl_xor_sync(kAll, two, o);
                two = fmaxf(fmaxf(two, b), fminf(one, a));
                one = fmaxf(one, a);
            }
            const bool single = two == -INFINITY;
            const float worth = single ? one : one + two, size = fabsf(one) + (single ? 0.f : fabsf(two));
            int better = 0;                                 // groups in front of this one
#pragma unroll 4
            for (int g = 0; g < p.groups; ++g) better += __shfl_sync(kAll, worth, g * p.group_lanes) > worth;
            const bool live = group < p.groups, kept = live && better < p.top_groups;
            // the border between the groups that stay and those that go: too near, or the place of several equal ones
            const float in = from_ordered(__reduce_min_sync(kAll, kept ? ordered(worth) : 0xFFFFFFFFu)),
                        out = from_ordered(__reduce_max_sync(kAll, live && !kept ? ordered(worth) : 0u)),
                        most = from_ordered(__reduce_max_sync(kAll, live ? ordered(size) : 0u));
            close = in - out <= 4.f * bound + (2.f * kCut + 1e-6f) * most || __popc(__ballot_sync(kAll, kept)) != p.top_groups * p.group_lanes;
            if (!kept) {
#pragma unroll
                for (int i = 0; i < PER; ++i) key[i] = 0u;
            }
        }
        unsigned won = 0u;                                  // lane j keeps choice j: its key, and the lane that it comes from
        int from = 0;
        for (int j = 0; j < p.top_k; ++j) {
            const unsigned best = __reduce_max_sync(kAll, key[0] & ~kIndex);
            const int owner = __ffs(__ballot_sync(kAll, (key[0] & ~kIndex) == best)) - 1;
            const unsigned got = __shfl_sync(kAll, key[0], owner);
            if (lane == j) {
                won = got;
                from = owner;
            }
            if (lane == owner) {
#pragma unroll
                for (int i = 0; i + 1 < PER; ++i) key[i] = key[i + 1];
                key[PER - 1] = 0u;
            }
        }
        const int taken = from * p.per_lane + (int)(kIndex - (won & kIndex));
        {                                                   // every choice against the one behind it, the last one against the best that is left (0: none)
            const unsigned rest = __reduce_max_sync(kAll, key[0] & ~kIndex), after = __shfl_down_sync(kAll, won, 1);
            const unsigned below = (lane == p.top_k - 1 ? rest : after) & ~kIndex;
            const float value = from_ordered(won & ~kIndex), other = from_ordered(below), gap = value - other, error = kCut * (fabsf(value) + fabsf(other));
            close |= lane < p.top_k && below != 0u &&
                     (direct ? (gap > 0.f && gap < 1e-9f) || (sizeof(T) == 4 && gap <= error) : gap <= 2.f * bound + error + 2e-7f * fabsf(value));
        }
        // the weights: of the choices alone if they are divided by their sum
        const bool chosen = lane < p.top_k;
        const float logit = chosen ? widen(row[taken]) : 0.f;
        const float low = from_ordered(__reduce_min_sync(kAll, chosen ? ordered(logit) : 0xFFFFFFFFu)),
                    high = from_ordered(__reduce_max_sync(kAll, chosen ? ordered(logit) : 0u));
        // scores that 64 bits cannot tell apart (1 - e^-x beyond 16), or that vanish
        if (p.sigmoid) close |= (direct && high >= 16.f) || low <= -60.f;
        else close |= low - top <= -60.f;
        if (__any_sync(kAll, close)) {
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
    const int64_t ctas = (p.tokens + kWarps - 1) / kWarps, resident = (int64_t)sm_count() * 8;
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
