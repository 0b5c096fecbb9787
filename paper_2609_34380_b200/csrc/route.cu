// Routing: the experts of each token and their weights, from the router's logits.
//
//   s = softmax(x) or sigmoid(x);  c = s + bias;  groups by the sum of their two largest c;  top-k of c;  w = s / sum * scale
//
// One warp per token; lane i holds experts i, i + 32, ...  Two of the values that the choice compares may be nearer than 32 bits tell
// apart, and a choice is a whole number: it is made on 64-bit values.
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

template <typename T, int PER>
__global__ void __launch_bounds__(kThreads) route_experts_kernel(const RouteParams p) {
    sm100::grid_launch_dependents();
    sm100::grid_dependency_wait();
    const int lane = threadIdx.x & 31;
    const int64_t token = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
    if (token >= p.tokens) return;
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

template <typename T>
cudaError_t launch(const RouteParams& p, cudaStream_t stream) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((p.tokens + kWarps - 1) / kWarps));
    cfg.blockDim = dim3(kThreads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const int per = (p.experts + 31) / 32;
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
    p.scale = scale;
    p.sigmoid = scoring == DPS_SCORE_SIGMOID;
    p.renormalise = renormalise;
    return type == DPS_TYPE_FP16 ? launch<__half>(p, stream) : type == DPS_TYPE_BF16 ? launch<__nv_bfloat16>(p, stream) : launch<float>(p, stream);
}

}  // namespace dps
