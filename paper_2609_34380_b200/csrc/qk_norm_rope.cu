// Norms of queries and keys for each head, position rotation and the write into the paged cache, in one pass over the QKV linear's
// output.
//
//   y = x / sqrt(mean(x^2) + eps) * w;  pairs (a, b) -> (a cos - b sin, b cos + a sin);  keys and values to their slot
//
// A stream: every element is read once and written once, bound by HBM for prompts and by latency for a few tokens.  A head is
// a group of LANES lanes (8, 16 or 32: the power of two that covers head_dim / 8), each lane holding 8 neighbouring elements in one
// 16-byte load; the mean is a butterfly over the group, and the other half of a rotated pair is 8 elements of another lane, which
// come by shuffle as they were loaded (four words; the norm's factor is the same, the weight is that lane's and loaded once).  A warp
// serves up to kHeads heads per group of one token: their loads are in flight together, and the token's row of the table and the
// weights are read once for all of them.  All arithmetic in 32 bits, one rounding at the store.
#include "dps_internal.h"
#include "sm100.cuh"
#include "step_ops.h"
#include "warp_mma.cuh"

namespace dps {

namespace {

using warp::Half2;

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kHeads = 4;

struct QkParams {
    const unsigned char* qkv;
    int64_t qkv_stride;
    const int64_t* slots;
    const int32_t* positions;
    const float* cos_sin;
    const unsigned char* q_weight;
    const unsigned char* k_weight;
    unsigned char* q_out;
    int64_t q_out_stride;
    unsigned char* k;
    unsigned char* v;
    int64_t block_stride, token_stride, head_stride, cache_slots, max_position, tokens;
    int* status;
    int page, dim, q_heads, kv_heads, rotated, tasks;
    float eps;
};

__device__ __forceinline__ uint4 load16(const void* p) { return *reinterpret_cast<const uint4*>(p); }

template <typename T>
__device__ __forceinline__ void widen(const uint4& v, float (&x)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = Half2<T>::unpack(w[i]);
        x[2 * i] = f.x;
        x[2 * i + 1] = f.y;
    }
}

template <typename T, int LANES, bool INTERLEAVED>
__global__ void __launch_bounds__(kThreads) qk_norm_rope_kernel(const QkParams p) {
    sm100::grid_launch_dependents();
    sm100::grid_dependency_wait();
    constexpr int kGroups = 32 / LANES;                     // heads side by side in a warp
    const int lane = threadIdx.x & 31, chunk = lane % LANES, group = lane / LANES;
    const int64_t task = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
    const int64_t token = task / p.tasks;
    if (token >= p.tokens) return;
    const int first = (int)(task - token * p.tasks) * (kHeads * kGroups) + group;
    const int heads = p.q_heads + 2 * p.kv_heads;
    const int64_t slot = p.slots[token];
    if (slot < 0) return;                                   // padding
    const int position = p.rotated > 0 ? p.positions[token] : 0;
    if (slot >= p.cache_slots || (p.rotated > 0 && (position < 0 || position >= p.max_position))) {
        if (lane == 0) atomicExch(p.status, (int)DPS_ERR_DATA);
        return;
    }
    const bool there = chunk * 8 < p.dim;

    uint4 raw[kHeads];
#pragma unroll
    for (int i = 0; i < kHeads; ++i) {
        const int head = first + i * kGroups;
        raw[i] = there && head < heads ? load16(p.qkv + (token * p.qkv_stride + (int64_t)head * p.dim + chunk * 8) * 2)
                                       : make_uint4(0, 0, 0, 0);
    }
    // the rotation of this lane's elements, and the lane that holds their partners
    const int half = p.rotated / 2;                         // a multiple of 8
    const bool turns = chunk * 8 < p.rotated;
    const bool upper = !INTERLEAVED && chunk * 8 >= half;
    const int partner = INTERLEAVED || !turns ? lane : upper ? lane - half / 8 : lane + half / 8;
    constexpr int kAngles = INTERLEAVED ? 4 : 8;
    float cosine[kAngles], sine[kAngles];
    if (turns) {
        const float* row = p.cos_sin + (int64_t)position * p.rotated + (INTERLEAVED ? chunk * 4 : chunk * 8 - (upper ? half : 0));
#pragma unroll
        for (int i = 0; i < kAngles; i += 4) {
            const float4 c = *reinterpret_cast<const float4*>(row + i), s = *reinterpret_cast<const float4*>(row + half + i);
            cosine[i] = c.x, cosine[i + 1] = c.y, cosine[i + 2] = c.z, cosine[i + 3] = c.w;
            sine[i] = s.x, sine[i + 1] = s.y, sine[i + 2] = s.z, sine[i + 3] = s.w;
        }
    }
    const int64_t to = (slot / p.page) * p.block_stride + (slot % p.page) * p.token_stride + chunk * 8;

#pragma unroll
    for (int i = 0; i < kHeads; ++i) {
        const int head = first + i * kGroups;               // the same branch for a group, not for a warp: shuffles stay outside
        const bool is_q = head < p.q_heads, is_v = head >= p.q_heads + p.kv_heads;
        uint4 other;
        other.x = __shfl_sync(0xFFFFFFFFu, raw[i].x, partner);
        other.y = __shfl_sync(0xFFFFFFFFu, raw[i].y, partner);
        other.z = __shfl_sync(0xFFFFFFFFu, raw[i].z, partner);
        other.w = __shfl_sync(0xFFFFFFFFu, raw[i].w, partner);
        float x[8], y[8];
        widen<T>(raw[i], x);
        widen<T>(other, y);
        if (p.q_weight != nullptr) {
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) sum += x[e] * x[e];
#pragma unroll
            for (int o = 1; o < LANES; o <<= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
            const float scale = 1.f / sqrtf(sum / p.dim + p.eps);
            if (there) {
                const unsigned char* w = is_q ? p.q_weight : p.k_weight;
                float wx[8], wy[8];
                widen<T>(load16(w + chunk * 16), wx);
                widen<T>(load16(w + (chunk + partner - lane) * 16), wy);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    x[e] = x[e] * scale * wx[e];
                    y[e] = y[e] * scale * wy[e];
                }
            }
        }
        if (turns) {
            if (INTERLEAVED) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float a = x[2 * e], b = x[2 * e + 1];
                    x[2 * e] = a * cosine[e % kAngles] - b * sine[e % kAngles];
                    x[2 * e + 1] = b * cosine[e % kAngles] + a * sine[e % kAngles];
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float s = sine[e % kAngles];
                    x[e] = x[e] * cosine[e % kAngles] + y[e] * (upper ? s : -s);
                }
            }
        }
        if (there && head < heads) {
            uint4 packed = raw[i];
            if (!is_v) {
                packed.x = Half2<T>::pack(x[0], x[1]);
                packed.y = Half2<T>::pack(x[2], x[3]);
                packed.z = Half2<T>::pack(x[4], x[5]);
                packed.w = Half2<T>::pack(x[6], x[7]);
            }
            unsigned char* at = is_q   ? p.q_out + (token * p.q_out_stride + (int64_t)head * p.dim + chunk * 8) * 2
                                : is_v ? p.v + (to + (head - p.q_heads - p.kv_heads) * p.head_stride) * 2
                                       : p.k + (to + (head - p.q_heads) * p.head_stride) * 2;
            *reinterpret_cast<uint4*>(at) = packed;
        }
    }
}

template <typename T, int LANES>
cudaError_t launch(QkParams p, bool interleaved, cudaStream_t stream) {
    constexpr int kPerTask = kHeads * (32 / LANES);
    p.tasks = (p.q_heads + 2 * p.kv_heads + kPerTask - 1) / kPerTask;
    const int64_t ctas = (p.tokens * p.tasks + kWarps - 1) / kWarps;
    if (ctas > INT32_MAX) return cudaErrorInvalidConfiguration;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3(kThreads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = interleaved ? cudaLaunchKernelEx(&cfg, qk_norm_rope_kernel<T, LANES, true>, p)
                                      : cudaLaunchKernelEx(&cfg, qk_norm_rope_kernel<T, LANES, false>, p);
    if (e == cudaSuccess) count_launch();
    return e;
}

template <typename T>
cudaError_t launch_typed(const QkParams& p, bool interleaved, cudaStream_t stream) {
    return p.dim <= 64 ? launch<T, 8>(p, interleaved, stream) : p.dim <= 128 ? launch<T, 16>(p, interleaved, stream)
                                                                              : launch<T, 32>(p, interleaved, stream);
}

}  // namespace

cudaError_t launch_qk_norm_rope(const void* qkv, int64_t qkv_stride, int64_t tokens, int32_t q_heads, const dps_kv_cache& cache,
                                const int64_t* slots, const int32_t* positions, const float* cos_sin, int64_t max_position,
                                int32_t rotated, bool interleaved, const void* q_weight, const void* k_weight, float eps, void* q_out,
                                int64_t q_out_stride, int* status, cudaStream_t stream) {
    QkParams p;
    p.qkv = static_cast<const unsigned char*>(qkv);
    p.qkv_stride = qkv_stride;
    p.slots = slots;
    p.positions = positions;
    p.cos_sin = cos_sin;
    p.q_weight = static_cast<const unsigned char*>(q_weight);
    p.k_weight = static_cast<const unsigned char*>(k_weight);
    p.q_out = static_cast<unsigned char*>(q_out);
    p.q_out_stride = q_out_stride;
    p.k = static_cast<unsigned char*>(cache.k);
    p.v = static_cast<unsigned char*>(cache.v);
    p.block_stride = cache.block_stride;
    p.token_stride = cache.token_stride;
    p.head_stride = cache.head_stride;
    p.cache_slots = cache.blocks * cache.page_tokens;
    p.max_position = max_position;
    p.tokens = tokens;
    p.status = status;
    p.page = cache.page_tokens;
    p.dim = cache.head_dim;
    p.q_heads = q_heads;
    p.kv_heads = cache.heads;
    p.rotated = rotated;
    p.tasks = 0;
    p.eps = eps;
    return cache.type == DPS_TYPE_FP16 ? launch_typed<__half>(p, interleaved, stream) : launch_typed<__nv_bfloat16>(p, interleaved, stream);
}

}  // namespace dps
