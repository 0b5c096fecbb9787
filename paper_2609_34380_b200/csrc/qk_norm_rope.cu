// Norms of queries and keys for each head, position rotation and the write into the paged cache, in one pass over the QKV linear's
// output.
//
//   y = x / sqrt(mean(x^2) + eps) * w;  pairs (a, b) -> (a cos - b sin, b cos + a sin);  keys and values to their slot
//
// A stream: every element is read once and written once, bound by HBM for prompts and by latency for a few tokens.  A head is
// a group of LANES lanes (8, 16 or 32: the power of two that covers head_dim / 8), each lane holding 8 of its elements in two pieces of
// four: where the head is rotated by halves, four of the lower half and their partners of the upper half, else neighbours.  So a
// rotated pair is always within a lane, and only the mean needs a butterfly over the group.  With the weights and the rotation a lane's
// elements are u = (P A + Q B) f and v = (Q C + P D) f, f = 1 / sqrt(mean + eps): A .. D are formed once for all the heads that a warp
// serves, kHeads per group, all queries or all keys of one token, whose loads are in flight together.  All arithmetic in 32 bits, one
// rounding at the store.
//
// 8192 tokens of 64 + 8 + 8 heads of 128, FP16: 340 MB in 59.7 to 65 us with the GPU, 5.2 to 5.7 TB/s, 79 to 87 % of what a copy reaches; 999 tokens of 24 + 6 + 6 heads of 96
// 4.4 us, one token 2.4 us.  Few heads leave lanes idle: 8192 tokens of 12 + 1 + 1 heads of 96 22.1 us (47 MB, 7.2 us), of 4 + 4 + 4 heads of 80 17.2 (34 MB, 5.2).  What did not hold: 16-byte pieces of one half, partners by shuffle and weights widened for each head 115 us, bound by the number of
// instructions; loads in the order of their use and arithmetic by single values 79 us; blocks of 256 threads, whose places wait for the slowest of
// eight warps, 66 us (64 threads 59.6, but 5.1 us for the 999 tokens); three heads a group 70.8 us, five 63.6; several tasks a warp, one after another, 75.
#include "dps_internal.h"
#include "sm100.cuh"
#include "step_ops.h"
#include "warp_mma.cuh"

namespace dps {

namespace {

using warp::Half2;

constexpr int kThreads = 128;
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
    int page, dim, q_heads, kv_heads, rotated, q_tasks, kv_tasks;        // warps per token: q_tasks + 2 kv_tasks
    float eps;
};

// Two 32-bit values that one instruction works on.
struct Two {
    unsigned long long v;
    Two() = default;
    __device__ __forceinline__ Two(float a, float b) { asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b)); }
    __device__ __forceinline__ float2 both() const {
        float2 f;
        asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(v));
        return f;
    }
};
__device__ __forceinline__ Two operator*(Two a, Two b) {
    Two r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ Two fma2(Two a, Two b, Two c) {
    Two r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}

// A lane's eight elements of a head, in two pieces of four.
struct Pieces {
    uint2 a, b;
};
__device__ __forceinline__ Pieces load_pieces(const unsigned char* head, int a, int b) {
    return Pieces{*reinterpret_cast<const uint2*>(head + a * 2), *reinterpret_cast<const uint2*>(head + b * 2)};
}
// ... as the members P and Q of four pairs: the pieces, or, interleaved, even and odd elements.
template <typename T, bool INTERLEAVED>
__device__ __forceinline__ void widen(const Pieces& v, float (&p)[4], float (&q)[4]) {
    const float2 w[4] = {Half2<T>::unpack(v.a.x), Half2<T>::unpack(v.a.y), Half2<T>::unpack(v.b.x), Half2<T>::unpack(v.b.y)};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        p[i] = INTERLEAVED ? w[i].x : i % 2 ? w[i / 2].y : w[i / 2].x;
        q[i] = INTERLEAVED ? w[i].y : i % 2 ? w[2 + i / 2].y : w[2 + i / 2].x;
    }
}
template <typename T, bool INTERLEAVED>
__device__ __forceinline__ Pieces narrow(const float (&p)[4], const float (&q)[4]) {
    Pieces v;
    v.a.x = INTERLEAVED ? Half2<T>::pack(p[0], q[0]) : Half2<T>::pack(p[0], p[1]);
    v.a.y = INTERLEAVED ? Half2<T>::pack(p[1], q[1]) : Half2<T>::pack(p[2], p[3]);
    v.b.x = INTERLEAVED ? Half2<T>::pack(p[2], q[2]) : Half2<T>::pack(q[0], q[1]);
    v.b.y = INTERLEAVED ? Half2<T>::pack(p[3], q[3]) : Half2<T>::pack(q[2], q[3]);
    return v;
}

template <typename T, int LANES, bool INTERLEAVED>
__global__ void __launch_bounds__(kThreads) qk_norm_rope_kernel(const QkParams p) {
    sm100::grid_launch_dependents();
    sm100::grid_dependency_wait();
    constexpr int kGroups = 32 / LANES;                     // heads side by side in a warp
    const int lane = threadIdx.x & 31, chunk = lane % LANES, group = lane / LANES;
    const int tasks = p.q_tasks + 2 * p.kv_tasks;
    const unsigned id = blockIdx.x * kWarps + (threadIdx.x >> 5);       // (below 2^31: checked on the host)
    const int64_t token = id / tasks;
    if (token >= p.tokens) return;
    int task = (int)(id % tasks), kind = 0;                 // queries, keys or values
    if (task >= p.q_tasks) {
        task -= p.q_tasks;
        kind = task < p.kv_tasks ? 1 : 2;
        if (kind == 2) task -= p.kv_tasks;
    }
    // All that does not hang on anything else is asked for at once: a warp's life is the latency of two loads, its row and then the rotation's.
    const int64_t slot = p.slots[token];
    const bool rotates = p.rotated > 0;
    const int position = rotates ? p.positions[token] : 0;
    const bool there = chunk * 8 < p.dim, turns = chunk * 8 < p.rotated;
    const bool halves = !INTERLEAVED && turns;
    const int first = halves ? chunk * 4 : chunk * 8, second = halves ? p.rotated / 2 + chunk * 4 : chunk * 8 + 4;
    const int heads = kind == 0 ? p.q_heads : p.kv_heads, head0 = task * (kHeads * kGroups) + group;
    const unsigned char* from = p.qkv + (token * p.qkv_stride + (int64_t)((kind == 0 ? 0 : kind == 1 ? p.q_heads : p.q_heads + p.kv_heads) + head0) * p.dim) * 2;
    const int live = there ? (heads - head0 + kGroups - 1) / kGroups : 0;        // this lane's heads, up to kHeads of them
    Pieces raw[kHeads];
#pragma unroll
    for (int i = 0; i < kHeads; ++i) {
        raw[i] = i < live ? load_pieces(from, first, second) : Pieces{make_uint2(0, 0), make_uint2(0, 0)};
        from += kGroups * p.dim * 2;
    }
    float wp[4] = {1.f, 1.f, 1.f, 1.f}, wq[4] = {1.f, 1.f, 1.f, 1.f};
    if (p.q_weight != nullptr && there && kind < 2) widen<T, INTERLEAVED>(load_pieces(kind == 0 ? p.q_weight : p.k_weight, first, second), wp, wq);
    if (slot < 0) return;                                   // padding
    if (slot >= p.cache_slots || (rotates && (position < 0 || position >= p.max_position))) {
        if (lane == 0) atomicExch(p.status, (int)DPS_ERR_DATA);
        return;
    }
    unsigned char* to;                                      // of this token's heads, and how far apart they are
    int64_t step = p.dim;
    if (kind == 0) to = p.q_out + token * p.q_out_stride * 2;
    else {
        const bool narrow_slot = slot <= UINT32_MAX;
        const int64_t block = narrow_slot ? (unsigned)slot / (unsigned)p.page : slot / p.page, within = slot - block * p.page;
        to = (kind == 1 ? p.k : p.v) + (block * p.block_stride + within * p.token_stride) * 2;
        step = p.head_stride;
    }
    to += (head0 * step + first) * 2;
    step *= kGroups * 2;
    const int apart = (second - first) * 2;
    if (kind == 2) {
#pragma unroll
        for (int i = 0; i < kHeads; ++i) {
            if (i < live) {
                *reinterpret_cast<uint2*>(to) = raw[i].a;
                *reinterpret_cast<uint2*>(to + apart) = raw[i].b;
            }
            to += step;
        }
        return;
    }
    Two a[2], b[2], c[2], d[2];                             // u = (P a + Q b) f, v = (Q c + P d) f
    {
        float cosine[4] = {1.f, 1.f, 1.f, 1.f}, sine[4] = {0.f, 0.f, 0.f, 0.f};
        if (turns) {
            const float* const row = p.cos_sin + (int64_t)position * p.rotated + chunk * 4;
            const float4 x = *reinterpret_cast<const float4*>(row), y = *reinterpret_cast<const float4*>(row + p.rotated / 2);
            cosine[0] = x.x, cosine[1] = x.y, cosine[2] = x.z, cosine[3] = x.w;
            sine[0] = y.x, sine[1] = y.y, sine[2] = y.z, sine[3] = y.w;
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const Two w(wp[2 * e], wp[2 * e + 1]), z(wq[2 * e], wq[2 * e + 1]), cs(cosine[2 * e], cosine[2 * e + 1]), sn(sine[2 * e], sine[2 * e + 1]);
            a[e] = w * cs;
            b[e] = z * sn * Two(-1.f, -1.f);
            c[e] = z * cs;
            d[e] = w * sn;
        }
    }
    const float per_element = 1.f / p.dim;
#pragma unroll
    for (int i = 0; i < kHeads; ++i) {
        float x[4], y[4], factor = 1.f;
        widen<T, INTERLEAVED>(raw[i], x, y);
        const Two px[2] = {Two(x[0], x[1]), Two(x[2], x[3])}, py[2] = {Two(y[0], y[1]), Two(y[2], y[3])};
        if (p.q_weight != nullptr) {
            const Two squares = fma2(px[0], px[0], fma2(px[1], px[1], fma2(py[0], py[0], py[1] * py[1])));
            const float2 halves_of = squares.both();
            float sum = halves_of.x + halves_of.y;
#pragma unroll
            for (int o = 1; o < LANES; o <<= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
            factor = rsqrtf(sum * per_element + p.eps);
        }
        float u[4], v[4];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            Two s = px[e] * a[e], t = py[e] * c[e];
            if (turns) {                                    // (an infinite element meets no zero elsewhere)
                s = fma2(py[e], b[e], s);
                t = fma2(px[e], d[e], t);
            }
            const float2 f = (s * Two(factor, factor)).both(), g = (t * Two(factor, factor)).both();
            u[2 * e] = f.x, u[2 * e + 1] = f.y, v[2 * e] = g.x, v[2 * e + 1] = g.y;
        }
        if (i < live) {
            const Pieces out = narrow<T, INTERLEAVED>(u, v);
            *reinterpret_cast<uint2*>(to) = out.a;
            *reinterpret_cast<uint2*>(to + apart) = out.b;
        }
        to += step;
    }
}

template <typename T, int LANES>
cudaError_t launch(QkParams p, bool interleaved, cudaStream_t stream) {
    constexpr int kPerTask = kHeads * (32 / LANES);
    p.q_tasks = (p.q_heads + kPerTask - 1) / kPerTask;
    p.kv_tasks = (p.kv_heads + kPerTask - 1) / kPerTask;
    const int64_t ctas = (p.tokens * (p.q_tasks + 2 * p.kv_tasks) + kWarps - 1) / kWarps;
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
    p.q_tasks = p.kv_tasks = 0;                             // the launch knows how many heads a warp serves
    p.eps = eps;
    return cache.type == DPS_TYPE_FP16 ? launch_typed<__half>(p, interleaved, stream) : launch_typed<__nv_bfloat16>(p, interleaved, stream);
}

}  // namespace dps
