// Attention of one new token per request over a paged key-value cache.
//
//   out[b][h] = sum_t p_t V[t],  p = softmax_t(scale q[b][h] . K[t])
//
// Every key and value is read once and takes part in 4 * (heads that share it) operations per element: a stream bound by HBM.
// The kernel is built around that stream:
//   * The work is a flat list of tiles, 64 tokens of one (request, key-value head) each, in that order.  A resident grid cuts it into
//     equal runs, one per CTA, whatever the lengths are: each CTA sums the lengths itself (they are on the device) and finds its
//     run's start.  So one long request is spread over the GPU, and a ragged batch leaves no SM behind.
//   * A warp owns 16 tokens of each tile and a ring of asynchronous 16-byte copies of its own: no barrier inside a run, and the
//     copies run on across the borders of requests and heads.  The ids of the blocks are fetched one tile ahead of the copies.
//   * Keys times queries: S^T (16 tokens x 8 heads) = K (16 x dim) Q^T by m16n8k16 products, the tokens being the rows of the
//     matrix product: up to eight heads that share the keys cost one column block, one head alone does too.  The scores' maximum and sum run along (in 32
//     bits, by powers of two).  Values: O^T (dim x 8 heads) += V^T P^T, where P is handed over as the sum of two 16-bit values, so
//     that the weights keep 16 to 22 bits of precision and the result differs from 64-bit sums by its own rounding only.
//   * At the end of a (request, head) the CTA's four warps are joined through shared memory.  If the run covers only a part of it, the
//     part goes to the workspace, and the CTA that comes last (a counter per split) joins the parts in their order.
#include "dps_internal.h"
#include "sm100.cuh"
#include "step_ops.h"
#include "warp_mma.cuh"

namespace dps {

namespace {

using warp::Half2;

constexpr int kThreads = 128;
constexpr int kWarps = 4;
constexpr int kTile = 64;             // tokens of a tile
constexpr int kWarpTokens = 16;       // ... of them a warp's
constexpr int kMaxCtas = 1024;        // counters in the workspace

// Workspace: header, a counter per CTA, two parts per CTA.
constexpr uint64_t kReady = 0x647073417474316Full;
constexpr size_t kHeaderBytes = 256, kCounterBytes = kMaxCtas * sizeof(unsigned);

struct AttentionParams {
    const void* q;
    int64_t q_row, q_head;
    const void* k;
    const void* v;
    int64_t blocks, block_stride, token_stride, head_stride;
    const int32_t* table;
    int64_t table_stride;
    const int32_t* lengths;
    void* out;
    unsigned char* workspace;
    int* status;
    int64_t longest;      // tokens that a row of the table can name
    int page, kv_heads, dim, group, chunks, requests;
    float scale_log2;
};

__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ int clamped_length(const AttentionParams& p, int b) {
    const int n = p.lengths[b];
    return n <= 0 ? 0 : (int64_t)n > p.longest ? (int)p.longest : n;
}
__device__ __forceinline__ int tiles_of(int length) { return (int)(((unsigned)length + kTile - 1) / kTile); }

// A place in the list of tiles.
struct Place {
    int b, h, j, tiles, length;    // request, key-value head (and chunk of its queries), tile of them; the request's tiles and tokens
    __device__ __forceinline__ void next(const AttentionParams& p, int heads) {
        if (++j < tiles) return;
        j = 0;
        if (++h < heads) return;
        h = 0;
        do length = clamped_length(p, ++b);
        while (length == 0 && b + 1 < p.requests);
        tiles = tiles_of(length);
    }
};

template <int DP, int NB>
struct Shape {
    static constexpr int kStageBytes = kWarpTokens * DP * 2 * 2;            // a warp's keys and values
    static constexpr int kStages = DP == 64 ? 6 : 3;
    static constexpr int kCtas = DP == 256 ? 1 : 2;                         // per SM
    static constexpr int kPitch = DP + 4;                                   // floats of a head's row while warps are joined
    static constexpr int kJoinBytes = kWarps * 8 * kPitch * 4;
    static constexpr int kBytes = kWarps * kStages * kStageBytes + kJoinBytes;
    static constexpr int kPartFloats = 8 * NB * (DP + 2);                   // a part: sums, then maximum and total of each head
};

// Joins `count` running sums of one head and one group of four elements.
struct Joined {
    float m = -INFINITY, l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    __device__ __forceinline__ void rescale(float top) {
        if (top > m) {
            const float w = exp2_approx(m - top);
            l *= w;
            o.x *= w;
            o.y *= w;
            o.z *= w;
            o.w *= w;
            m = top;
        }
    }
    __device__ __forceinline__ void add(float part_m, float part_l, const float4& part) {
        rescale(part_m);
        const float w = part_m == -INFINITY ? 0.f : exp2_approx(part_m - m);      // (a NaN in the sums stays one)
        l += w * part_l;
        o.x += w * part.x;
        o.y += w * part.y;
        o.z += w * part.z;
        o.w += w * part.w;
    }
};

template <typename T, int DP, int NB>
__global__ void __launch_bounds__(kThreads, (Shape<DP, NB>::kCtas))
paged_attention_kernel(const AttentionParams p) {
    using S = Shape<DP, NB>;
    constexpr int kRowChunks = DP / 8;                                      // 16-byte chunks of a token's keys
    constexpr int kCopies = kWarpTokens * kRowChunks / 32;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ int64_t s_scan[kWarps];
    __shared__ unsigned s_mask[kWarps][S::kStages];
    __shared__ float2 s_stat[kWarps][8];
    __shared__ Place s_first;
    __shared__ int s_flag;

    sm100::grid_launch_dependents();
    sm100::grid_dependency_wait();

    const int tid = threadIdx.x, lane = tid & 31, warp_id = tid >> 5;
    const int heads = p.kv_heads * p.chunks;
    const int ctas = gridDim.x, cta = blockIdx.x;

    // ---- the list's length, and where this CTA's run starts
    if (tid == 0) s_flag = *reinterpret_cast<const uint64_t*>(p.workspace) == kReady;
    const int per = (p.requests + kThreads - 1) / kThreads;
    const int first_request = min(tid * per, p.requests), last_request = min(first_request + per, p.requests);
    int64_t mine = 0;
    for (int b = first_request; b < last_request; ++b) mine += tiles_of(clamped_length(p, b));
    int64_t upto = mine;
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t u = __shfl_up_sync(0xFFFFFFFFu, upto, o);
        if (lane >= o) upto += u;
    }
    if (lane == 31) s_scan[warp_id] = upto;
    __syncthreads();
    if (!s_flag) {                                                          // a workspace that was not prepared
        if (cta == 0 && tid == 0) atomicExch(p.status, (int)DPS_ERR_WORKSPACE);
        return;
    }
    int64_t total = 0, before = upto - mine;
    for (int w = 0; w < kWarps; ++w) {
        if (w < warp_id) before += s_scan[w];
        total += s_scan[w];
    }
    const int64_t all = total * heads, each = all / ctas;
    const int more = (int)(all - each * ctas);                              // the first CTAs have one tile more
    const int64_t start = cta * each + min(cta, more);
    const int64_t count = each + (cta < more ? 1 : 0);
    if (count > 0) {
        const int64_t at = start / heads;                                   // in tiles of requests
        if (at >= before && at < before + mine) {
            int b = first_request;
            int64_t from = before;
            int length = clamped_length(p, b), tiles = tiles_of(length);
            while (at >= from + tiles && b + 1 < last_request) {
                from += tiles;
                length = clamped_length(p, ++b);
                tiles = tiles_of(length);
            }
            const int64_t inside = start - from * heads;
            const int h = (int)(inside / tiles);
            s_first = Place{b, h, (int)(inside - (int64_t)h * tiles), tiles, length};
        }
    }
    // requests without tokens: zeros; a length that is none
    for (int b = cta; b < p.requests; b += ctas) {
        const int n = p.lengths[b];
        if (tid == 0 && (n < 0 || (int64_t)n > p.longest)) atomicExch(p.status, (int)DPS_ERR_DATA);
        if (n <= 0 || p.longest == 0) {
            const int64_t row = (int64_t)p.kv_heads * p.group * p.dim / 8;
            uint4* to = reinterpret_cast<uint4*>(p.out) + b * row;
            for (int64_t i = tid; i < row; i += kThreads) to[i] = make_uint4(0, 0, 0, 0);
        }
    }
    if (count == 0) return;
    __syncthreads();

    // ---- copies into the ring
    const uint32_t ring = sm100::smem_u32(smem) + warp_id * S::kStages * S::kStageBytes;
    const unsigned char* const k_base = static_cast<const unsigned char*>(p.k);
    const unsigned char* const v_base = static_cast<const unsigned char*>(p.v);
    Place ahead = s_first;
    int64_t left = count;                                                   // tiles not yet asked for
    auto block_of = [&](const Place& at) {                                  // of this lane's row
        const int64_t token = (int64_t)at.j * kTile + warp_id * kWarpTokens + (lane & 15);
        return token < at.length ? p.table[at.b * p.table_stride + (int)token / p.page] : 0;
    };
    int block = block_of(ahead);
    auto ask = [&](int stage) {
        if (left > 0) {
            const int64_t token = (int64_t)ahead.j * kTile + warp_id * kWarpTokens + (lane & 15);
            const bool inside = token < ahead.length, known = (unsigned)block < (uint64_t)p.blocks;
            if (inside && !known) atomicExch(p.status, (int)DPS_ERR_DATA);
            const unsigned mask = __ballot_sync(0xFFFFFFFFu, inside && known) & 0xFFFFu;
            if (lane == 0) s_mask[warp_id][stage] = mask;
            const int64_t off = inside && known ? (block * p.block_stride + ((int)token % p.page) * p.token_stride +
                                                   (ahead.h / p.chunks) * p.head_stride) * 2 : 0;
            if (mask != 0) {
                const uint32_t to = ring + stage * S::kStageBytes;
#pragma unroll
                for (int i = 0; i < kCopies; ++i) {
                    const int at = i * 32 + lane, row = at / kRowChunks, c = at % kRowChunks;
                    const int64_t from = __shfl_sync(0xFFFFFFFFu, off, row) + c * 16;
                    const bool wanted = ((mask >> row) & 1u) && c * 8 < p.dim;
                    const uint32_t dst = to + row * (DP * 2) + ((c ^ (row & 7)) << 4);
                    warp::copy16(dst, k_base + (wanted ? from : 0), wanted ? 16 : 0);
                    warp::copy16(dst + kWarpTokens * DP * 2, v_base + (wanted ? from : 0), wanted ? 16 : 0);
                }
            }
            if (--left > 0) {
                ahead.next(p, heads);
                block = block_of(ahead);
            }
        }
        warp::copy_commit();
    };
#pragma unroll
    for (int s = 0; s < S::kStages - 1; ++s) ask(s);

    // ---- the run
    uint32_t qf[NB][DP / 16][2];
    float o[NB][DP / 16][4], m[NB][2], l[NB][2];
    const int column = lane & 3, row = lane >> 2;                           // of a fragment: heads 2 column, 2 column + 1; token row
    Place at = s_first;
    bool fresh = true;                                                      // a (request, head) starts here
    const bool from_start = at.j == 0;                                      // the run's first one starts with it
    bool first_unit = true;
    int stage = 0;
    const uint32_t k_lane = (lane & 15) * (DP * 2);                         // ldmatrix row of the keys: tokens 0-15, chunk 0 or 1
    const uint32_t v_row = (lane & 7) + ((lane >> 4) << 3);                 // of the values: tokens 0-7 / 8-15, chunk by bit 3

    for (int64_t done = 0; done < count; ++done) {
        if (fresh) {
            fresh = false;
            const int kv = at.h / p.chunks, chunk = at.h % p.chunks;
            const unsigned char* q_base = static_cast<const unsigned char*>(p.q) +
                                          (at.b * p.q_row + ((int64_t)kv * p.group + chunk * 8 * NB) * p.q_head) * 2;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                const int head = nb * 8 + row;
                const bool there = chunk * 8 * NB + head < p.group;
                const unsigned char* q_row = q_base + (there ? head * p.q_head : 0) * 2;
#pragma unroll
                for (int i = 0; i < DP / 16; ++i)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int d = i * 16 + e * 8 + column * 2;
                        qf[nb][i][e] = there && d < p.dim ? *reinterpret_cast<const uint32_t*>(q_row + d * 2) : 0u;
                    }
                m[nb][0] = m[nb][1] = -INFINITY;
                l[nb][0] = l[nb][1] = 0.f;
#pragma unroll
                for (int i = 0; i < DP / 16; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[nb][i][e] = 0.f;
            }
        }
        warp::copy_wait<S::kStages - 2>();
        __syncwarp();
        ask(stage == 0 ? S::kStages - 1 : stage - 1);                       // the stage that the step before has read
        const unsigned mask = s_mask[warp_id][stage];
        if (mask != 0) {
            const uint32_t keys = ring + stage * S::kStageBytes, values = keys + kWarpTokens * DP * 2;
            float s[NB][2][4];
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[nb][0][e] = s[nb][1][e] = 0.f;
#pragma unroll
            for (int i = 0; i < DP / 16; ++i) {
                uint32_t a[4];
                warp::ldmatrix_x4(a, keys + k_lane + (((i * 2 + (lane >> 4)) ^ (lane & 7)) << 4));
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) Half2<T>::mma(s[nb][i & 1], a, qf[nb][i][0], qf[nb][i][1]);
            }
            const bool low = (mask >> row) & 1u, high = (mask >> (row + 8)) & 1u;
            uint32_t ph[NB][2], pl[NB][2];
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                float x[4], top[2], scale[2];
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = (e < 2 ? low : high) ? (s[nb][0][e] + s[nb][1][e]) * p.scale_log2 : -INFINITY;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float t = fmaxf(x[e], x[e + 2]);
                    t = fmaxf(t, __shfl_xor_sync(0xFFFFFFFFu, t, 4));
                    t = fmaxf(t, __shfl_xor_sync(0xFFFFFFFFu, t, 8));
                    t = fmaxf(t, __shfl_xor_sync(0xFFFFFFFFu, t, 16));
                    t = fmaxf(t, m[nb][e]);
                    top[e] = t == -INFINITY ? 0.f : t;
                    scale[e] = exp2_approx(m[nb][e] - top[e]);
                    m[nb][e] = t;
                }
                float pr[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) pr[e] = exp2_approx(x[e] - top[e & 1]);
#pragma unroll
                for (int e = 0; e < 2; ++e) l[nb][e] = l[nb][e] * scale[e] + (pr[e] + pr[e + 2]);
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint32_t h2 = Half2<T>::pack(pr[2 * e], pr[2 * e + 1]);
                    const float2 back = Half2<T>::unpack(h2);
                    ph[nb][e] = warp::transpose8x8(h2);
                    pl[nb][e] = warp::transpose8x8(Half2<T>::pack(pr[2 * e] - back.x, pr[2 * e + 1] - back.y));
                }
                if (__any_sync(0xFFFFFFFFu, scale[0] != 1.f || scale[1] != 1.f)) {
#pragma unroll
                    for (int i = 0; i < DP / 16; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[nb][i][e] *= scale[e & 1];
                }
            }
#pragma unroll
            for (int i = 0; i < DP / 16; ++i) {
                uint32_t a[4];
                warp::ldmatrix_x4_trans(a, values + v_row * (DP * 2) + (((i * 2 + ((lane >> 3) & 1)) ^ (lane & 7)) << 4));
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    Half2<T>::mma(o[nb][i], a, ph[nb][0], ph[nb][1]);
                    Half2<T>::mma(o[nb][i], a, pl[nb][0], pl[nb][1]);
                }
            }
        }
        if (++stage == S::kStages) stage = 0;

        // ---- the end of a (request, head), or of the run
        const bool ends = at.j == at.tiles - 1;
        if (ends || done + 1 == count) {
            const bool starts_here = !first_unit || from_start;
            const bool whole = ends && starts_here;
            // of the split: its first tile in the list, its first and last CTA
            const int64_t unit = start + done - at.j, unit_last = unit + at.tiles - 1;
            const int64_t big = (int64_t)more * (each + 1);
            const int cta0 = (int)(unit < big ? unit / (each + 1) : more + (unit - big) / each);
            const int cta1 = (int)(unit_last < big ? unit_last / (each + 1) : more + (unit_last - big) / each);
            unsigned* const counters = reinterpret_cast<unsigned*>(p.workspace + kHeaderBytes);
            float* const parts = reinterpret_cast<float*>(p.workspace + kHeaderBytes + kCounterBytes);
            float* const part = parts + (int64_t)(2 * cta + (starts_here ? 1 : 0)) * S::kPartFloats;
            const int kv = at.h / p.chunks, chunk = at.h % p.chunks;
            const int used = min(p.group - chunk * 8 * NB, 8 * NB);         // heads
            T* const out = static_cast<T*>(p.out) + ((int64_t)at.b * p.kv_heads * p.group + (int64_t)kv * p.group + chunk * 8 * NB) * p.dim;
            constexpr int kQuads = DP / 4, kHeadsAtOnce = kThreads / kQuads;
            const int quad = tid % kQuads, sub = tid / kQuads;
            float* const join = reinterpret_cast<float*>(smem + kWarps * S::kStages * S::kStageBytes);
            auto store = [&](int head, const Joined& r) {
                if (head < used && quad * 4 < p.dim) {
                    const float inv = 1.f / r.l;
                    uint2 packed;
                    packed.x = Half2<T>::pack(r.o.x * inv, r.o.y * inv);
                    packed.y = Half2<T>::pack(r.o.z * inv, r.o.w * inv);
                    *reinterpret_cast<uint2*>(out + (int64_t)head * p.dim + quad * 4) = packed;
                }
            };
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int x = 4; x < 32; x <<= 1) l[nb][e] += __shfl_xor_sync(0xFFFFFFFFu, l[nb][e], x);
                if (row == 0) {
                    s_stat[warp_id][2 * column] = make_float2(m[nb][0], l[nb][0]);
                    s_stat[warp_id][2 * column + 1] = make_float2(m[nb][1], l[nb][1]);
                }
#pragma unroll
                for (int i = 0; i < DP / 16; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        join[(warp_id * 8 + 2 * column + (e & 1)) * S::kPitch + i * 16 + row + (e >> 1) * 8] = o[nb][i][e];
                __syncthreads();
#pragma unroll
                for (int head = sub; head < 8; head += kHeadsAtOnce) {
                    Joined r;
#pragma unroll
                    for (int w = 0; w < kWarps; ++w) {
                        const float2 st = s_stat[w][head];
                        r.add(st.x, st.y, *reinterpret_cast<const float4*>(&join[(w * 8 + head) * S::kPitch + quad * 4]));
                    }
                    if (whole) store(nb * 8 + head, r);
                    else {
                        *reinterpret_cast<float4*>(part + (nb * 8 + head) * DP + quad * 4) = r.o;
                        if (quad == 0) *reinterpret_cast<float2*>(part + 8 * NB * DP + (nb * 8 + head) * 2) = make_float2(r.m, r.l);
                    }
                }
                __syncthreads();
            }
            if (!whole) {
                __threadfence();
                __syncthreads();
                if (tid == 0) s_flag = atomicAdd(&counters[cta0], 1u) == (unsigned)(cta1 - cta0);
                __syncthreads();
                if (s_flag) {                                               // all parts are there: join them
                    __threadfence();
                    for (int head = sub; head < used; head += kHeadsAtOnce) {
                        Joined r;
                        constexpr int kBatch = 8;
                        for (int c = cta0; c <= cta1; c += kBatch) {
                            float2 st[kBatch];
                            float4 v[kBatch];
#pragma unroll
                            for (int i = 0; i < kBatch; ++i)
                                if (c + i <= cta1) {
                                    const float* from = parts + (int64_t)(2 * (c + i) + (c + i == cta0 ? 1 : 0)) * S::kPartFloats;
                                    st[i] = __ldcg(reinterpret_cast<const float2*>(from + 8 * NB * DP + head * 2));
                                    v[i] = __ldcg(reinterpret_cast<const float4*>(from + head * DP + quad * 4));
                                }
#pragma unroll
                            for (int i = 0; i < kBatch; ++i)
                                if (c + i <= cta1) r.add(st[i].x, st[i].y, v[i]);
                        }
                        store(head, r);
                    }
                    if (tid == 0) counters[cta0] = 0;
                }
            }
            fresh = true;
            first_unit = false;
        }
        if (done + 1 < count) at.next(p, heads);
    }
}

__global__ void workspace_init_kernel(unsigned char* workspace) {
    for (int i = threadIdx.x; i < kMaxCtas; i += blockDim.x) reinterpret_cast<unsigned*>(workspace + kHeaderBytes)[i] = 0;
    if (threadIdx.x == 0) *reinterpret_cast<uint64_t*>(workspace) = kReady;
}

// What a shape takes: the head size's and the sharing heads' kernel.
int padded_dim(int dim) { return dim <= 64 ? 64 : dim <= 128 ? 128 : 256; }
// More than eight queries per key: two column blocks in one pass, as far as the registers hold them.
int column_blocks(int group, int dim) { return group > 8 && dim <= 128 ? 2 : 1; }

template <typename T, int DP, int NB>
cudaError_t launch(const AttentionParams& p, int64_t most_tiles, cudaStream_t stream) {
    using S = Shape<DP, NB>;
    static PerDeviceOnce once;
    const auto kernel = paged_attention_kernel<T, DP, NB>;
    cudaError_t e = once.run([&] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kBytes); });
    if (e != cudaSuccess) return e;
    int64_t ctas = (int64_t)sm_count() * S::kCtas;
    if (ctas > kMaxCtas) ctas = kMaxCtas;
    if (ctas > most_tiles) ctas = most_tiles;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = S::kBytes;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, kernel, p);
    if (e == cudaSuccess) count_launch();
    return e;
}

template <typename T>
cudaError_t launch_typed(const AttentionParams& p, int64_t most_tiles, cudaStream_t stream) {
    const bool two = column_blocks(p.group, p.dim) == 2;
    switch (padded_dim(p.dim)) {
        case 64: return two ? launch<T, 64, 2>(p, most_tiles, stream) : launch<T, 64, 1>(p, most_tiles, stream);
        case 128: return two ? launch<T, 128, 2>(p, most_tiles, stream) : launch<T, 128, 1>(p, most_tiles, stream);
        default: return launch<T, 256, 1>(p, most_tiles, stream);
    }
}

}  // namespace

size_t attention_workspace_bytes(int32_t q_heads, int32_t kv_heads, int32_t head_dim) {
    const int blocks = column_blocks(q_heads / kv_heads, head_dim), dim = padded_dim(head_dim);
    const int64_t ctas = (int64_t)sm_count() * (dim == 256 ? 1 : 2);
    return kHeaderBytes + kCounterBytes + (size_t)(ctas < kMaxCtas ? ctas : kMaxCtas) * 2 * 8 * blocks * (dim + 2) * sizeof(float);
}

cudaError_t launch_attention_workspace_init(void* workspace, cudaStream_t stream) {
    workspace_init_kernel<<<1, 256, 0, stream>>>(static_cast<unsigned char*>(workspace));
    const cudaError_t e = cudaGetLastError();
    if (e == cudaSuccess) count_launch();
    return e;
}

cudaError_t launch_paged_attention(const void* q, int64_t q_row, int64_t q_head, int64_t requests, int32_t q_heads,
                                   const dps_kv_cache& cache, const int32_t* table, int64_t table_stride, int64_t table_width,
                                   const int32_t* lengths, float scale, void* out, void* workspace, int* status, cudaStream_t stream) {
    AttentionParams p;
    p.q = q;
    p.q_row = q_row;
    p.q_head = q_head;
    p.k = cache.k;
    p.v = cache.v;
    p.blocks = cache.blocks;
    p.block_stride = cache.block_stride;
    p.token_stride = cache.token_stride;
    p.head_stride = cache.head_stride;
    p.table = table;
    p.table_stride = table_stride;
    p.lengths = lengths;
    p.out = out;
    p.workspace = static_cast<unsigned char*>(workspace);
    p.status = status;
    const int64_t longest = table_width * cache.page_tokens;                // (both below 2^31)
    p.longest = longest < INT32_MAX ? longest : INT32_MAX;
    p.page = cache.page_tokens;
    p.kv_heads = cache.heads;
    p.dim = cache.head_dim;
    p.group = q_heads / cache.heads;
    p.chunks = (p.group + 8 * column_blocks(p.group, p.dim) - 1) / (8 * column_blocks(p.group, p.dim));
    p.requests = (int)requests;
    p.scale_log2 = scale * 1.4426950408889634f;
    int64_t most = (p.longest + kTile - 1) / kTile * p.kv_heads * p.chunks;
    most = most > kMaxCtas ? kMaxCtas : most;
    most = most * requests < 1 ? 1 : most * requests;
    return cache.type == DPS_TYPE_FP16 ? launch_typed<__half>(p, most, stream) : launch_typed<__nv_bfloat16>(p, most, stream);
}

}  // namespace dps
