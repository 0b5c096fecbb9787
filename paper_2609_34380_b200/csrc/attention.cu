// Attention of one new token per request over a paged key-value cache.
//
//   out[b][h] = sum_t p_t V[t],  p = softmax_t(scale q[b][h] . K[t])
//
// Every key and value is read once for up to eight queries that share it (sixteen up to a head size of 128; each further eight or sixteen read it again) and takes
// part in 4 operations per element and query: a stream bound by HBM.
// The kernel is built around that stream:
//   * The work is a flat list of tiles, 64 tokens of one (request, key-value head) each, in that order.  A resident grid cuts it into
//     equal runs, one per CTA, whatever the lengths are: each CTA sums the lengths itself (they are on the device) and finds its
//     run's start.  So one long request is spread over the GPU, and a ragged batch leaves no SM behind.
//   * Warps that copy feed warps that compute, each of the latter with 16 tokens of every tile and a ring of stages of its own: no
//     barrier among them inside a (request, head), and the copies run on across the borders of requests and heads.  The tokens' blocks are looked
//     up one tile ahead, so a page may end anywhere.
//   * Keys times queries: S^T (16 tokens x 8 heads) = K (16 x dim) Q^T by m16n8k16 products, the tokens being the rows of the
//     matrix product: up to eight heads that share the keys cost one column block, one head alone does too.  The scores' maximum and sum run along (in 32
//     bits, by powers of two).  Values: O^T (dim x 8 heads) += V^T P^T, where P is handed over as the sum of two 16-bit values: a weight
//     keeps 16 bits of precision as BF16, 22 as FP16, there down to 2^-39 of the largest weight so far (kLift).  The sums are 32 bits wide.
//   * At the end of a (request, head) the CTA's four warps are joined through shared memory.  If the run covers only a part of it, the
//     part goes to the workspace, and the CTA that comes last (a counter per split) joins the parts in their order.
//
// Measured in graphs, three sets of inputs in turn, against the floor of the bytes at a copy's 6.58 TB/s: one request of 131071 tokens, 64 / 8 heads of 128, 88 to
// 96 us on different GPUs (81.6; the same access pattern without arithmetic takes 80.5); 112 requests up to 8190, 60 / 10 heads of 96, 321 to 360 (262); 8 requests up to 4096,
// 64 / 8 heads, 22.1 (12.9: the start and the joins take 4.5); 32 requests of 1 to 3001 tokens, 32 / 32 heads, 33.7 (19.5: half of the 992 units have less than
// 20 tokens, and each unit costs its CTA 1.7 to 2.8 us); one short request 4.7.  Other shapes, 16 requests up to 8192: 32 / 8 heads of 64 29.5 (16.6), 64 / 4 of 128 33.9 (16.7),
// 96 / 4 of 128, read twice, 54.5 (16.7), 16 / 4 of 256 45.5 (33.2), 64 / 4 of 256, read twice, 85.6 (33.3).  Warps that copy for themselves took 101 us for the
// 131071 tokens, a bulk copy per row 134 to 161, registers without shared memory 140.
#include "dps_internal.h"
#include "sm100.cuh"
#include "step_ops.h"
#include "warp_mma.cuh"

namespace dps {

namespace {

using warp::Half2;

constexpr int kWarps = 4;             // that compute; further ones copy
constexpr int kThreads = kWarps * 32;
constexpr int kTile = 64;             // tokens of a tile
constexpr int kWarpTokens = 16;       // ... of them a warp's
constexpr int kUnitCost = 1;          // what the end of a (request, head) costs, in tiles (short units that count for less: 34 -> 46 us for 32 mixed requests)
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
    unsigned page_magic, page_shift;      // token / page = token * page_magic >> page_shift, for tokens below 2^31
    float scale_log2;
};

__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// Adds one; the counter's value before.  What this thread has seen is seen by whoever counts after it.
__device__ __forceinline__ unsigned count_in(unsigned* counter) {
    unsigned before;
    asm volatile("atom.add.acq_rel.gpu.global.u32 %0, [%1], 1;" : "=r"(before) : "l"(counter) : "memory");
    return before;
}
__device__ __forceinline__ int clamped_length(const AttentionParams& p, int b) {
    const int n = p.lengths[b];
    return n <= 0 ? 0 : (int64_t)n > p.longest ? (int)p.longest : n;
}
__device__ __forceinline__ int tiles_of(int length) { return (int)(((unsigned)length + kTile - 1) / kTile); }
// Places that a (request, head) takes in the list: its tiles, and those that stand for its end.
__device__ __forceinline__ int places_of(int tiles) { return tiles > 0 ? tiles + kUnitCost : 0; }

// FP16 ends at 2^-24, and what a long tail of weights below that adds up to is not nothing beside one large weight whose value is small (3000 tokens, 19
// below the largest score: 13 % of the result were lost).  So all weights are 2^15 times their value, the largest 2^15; the factor goes out with the division by their total.
template <typename T> constexpr float kLift = 32768.f;
template <> constexpr float kLift<__nv_bfloat16> = 1.f;

// A place in the list of tiles.
struct Place {
    int b, h, j, tiles, length;    // request, key-value head (and chunk of its queries), tile of them; the request's tiles and tokens
    int rel;                       // how far into the run
    __device__ __forceinline__ void next_unit(const AttentionParams& p, int heads) {
        rel += places_of(tiles) - j;
        j = 0;
        if (++h < heads) return;
        h = 0;
        do length = clamped_length(p, ++b);
        while (length == 0 && b + 1 < p.requests);
        tiles = tiles_of(length);
    }
    __device__ __forceinline__ void next(const AttentionParams& p, int heads) {
        if (j + 1 == tiles) next_unit(p, heads);
        else {
            ++j;
            ++rel;
        }
    }
    // whether next() stays below `length` places
    __device__ __forceinline__ bool goes_on(int length) const { return rel + 1 + (j + 1 == tiles ? kUnitCost : 0) < length;
    }
};

template <int DP, int NB>
struct Shape {
    static constexpr int kRowBytes = DP * 2;
    static constexpr int kValues = kWarpTokens * kRowBytes;                 // where the values start in a stage
    static constexpr int kStageBytes = 2 * kValues;
    static constexpr int kStages = DP == 64 ? 6 : 3;
    static constexpr int kCtas = DP == 256 ? 1 : 2;                         // per SM
    // warps that copy: as many as leave the others the registers they need
    static constexpr int kProducers = DP == 256 ? 4 : 2;
    static constexpr bool kQueriesAhead = NB * DP < 256;                    // the next queries wait in registers
    static constexpr int kAllThreads = kThreads + 32 * kProducers;
    static_assert(8 * DP * 4 <= kValues, "a warp's sums take the place of the values it has read last");
    static constexpr int kBytes = kWarps * kStages * kStageBytes;
    static constexpr int kPartFloats = 8 * NB * (DP + 2);                   // a part: sums, then maximum and total of each head
};

// Infinite values.  A sum that has met one is NaN where the formula's is infinite: the value is multiplied by the 16-bit remainder of its weight too (zero or
// negative, for half of all weights), by a weight that 32 bits do not hold, by a rescaling of the sum.  Every weight being positive, the formula's answer hangs
// on the values alone: the infinity that is there, NaN if both are, or a NaN.  So a thread that has stored a NaN although the weights' total is a number
// (in the output kOdd stands for it) reads that column once more over its CTA's run, when all tiles of the run are done and before the parts are joined; the
// factors of the joining are never zero, so that a part's infinity stays one.  In a function of its own this costs finite values 0 to 0.7 % (32 mixed requests 33.97
// -> 34.10 us; sixteen queries per key 33.8 -> 34.4, 2 %); at the place of the store it was 0.5 to 6 %.  One infinity among 131071 tokens: 0.28 ms instead of 0.09.
constexpr unsigned kOdd = 0x7FFEu;                                          // a rounded NaN is 0x7FFF in both types
constexpr float kLeast = 1.17549435e-38f;                                   // 2^-126
// Ones in the lowest bits of those of a pair that have this magnitude.
__device__ __forceinline__ unsigned which(unsigned pair, unsigned magnitude) { return __vcmpeq2(pair & 0x7FFF7FFFu, magnitude * 0x10001u) & 0x00010001u; }
// Of four elements, those that `asked` names (a bit each): the infinity among tokens [from, to) of a request's values, or NaN.
template <typename T>
__device__ __forceinline__ void infinities_of(const AttentionParams& p, int b, int kv, int d, int from, int to, unsigned asked, float (&out)[4]) {
    unsigned up = 0, down = 0;                                              // a NaN counts as both
    int64_t index = from / p.page, at = from;
    for (; at < to && (up & down & asked) != asked; ++index) {
        const int64_t ends = (index + 1) * p.page, stop = ends < to ? ends : to;
        const int id = p.table[b * p.table_stride + index];
        if ((unsigned)id < (uint64_t)p.blocks) {
            const T* v = static_cast<const T*>(p.v) + id * p.block_stride + (at - index * p.page) * p.token_stride + kv * p.head_stride + d;
#pragma unroll 8
            for (int n = (int)(stop - at); n > 0; --n, v += p.token_stride) {
                const uint2 raw = *reinterpret_cast<const uint2*>(v);
                const float2 x = Half2<T>::unpack(raw.x), y = Half2<T>::unpack(raw.y);
                const float e[4] = {x.x, x.y, y.x, y.y};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    up |= (unsigned)!(e[i] < INFINITY) << i;
                    down |= (unsigned)!(e[i] > -INFINITY) << i;
                }
            }
        }
        at = stop;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (asked >> i & 1u) out[i] = (up ^ down) >> i & 1u ? (up >> i & 1u ? INFINITY : -INFINITY) : NAN;
}

// Joins `count` running sums of one head and one group of four elements.
struct Joined {
    float m = -INFINITY, l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    __device__ __forceinline__ void rescale(float top) {
        if (top > m) {
            const float w = fmaxf(exp2_approx(m - top), kLeast);
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

// A (request, head) that several CTAs hold parts of: the CTAs.
struct Split {
    int first = 0, last = -1;      // none
    int b = 0, h = 0;
};

// Of a (key-value head and chunk of its queries): the head, how many queries, where four elements of one of them go.
__device__ __forceinline__ int kv_of(const AttentionParams& p, int h) { return p.chunks == 1 ? h : h / p.chunks; }
template <int NB>
__device__ __forceinline__ int heads_in(const AttentionParams& p, int h) { return p.chunks == 1 ? p.group : min(p.group - h % p.chunks * 8 * NB, 8 * NB); }
template <typename T, int NB>
__device__ __forceinline__ uint2* place_of(const AttentionParams& p, int b, int h, int head, int quad) {
    const int kv = kv_of(p, h);
    return reinterpret_cast<uint2*>(static_cast<T*>(p.out) + (((int64_t)b * p.kv_heads + kv) * p.group + (h - kv * p.chunks) * 8 * NB + head) * p.dim + quad * 4);
}

// What one thread has stored of its CTA's run, starting at `at`, with NaN for infinities: elements of the output where the (request, head) is whole, of a part where not.
template <typename T, int DP, int NB>
__device__ __noinline__ void settle_infinities(const AttentionParams& p, Place at, int count, float* parts) {
    constexpr int kQuads = DP / 4, kHeadsAtOnce = kThreads / kQuads;
    const int quad = threadIdx.x % kQuads, sub = threadIdx.x / kQuads;
    for (;;) {
        const int tiles = min(at.tiles - at.j, count - at.rel), from = at.j * kTile;        // of it in this run
        const int to = (int)min((int64_t)from + (int64_t)tiles * kTile, (int64_t)at.length), kv = kv_of(p, at.h);
        const bool whole = tiles == at.tiles;
        float* const part = parts + (int64_t)(2 * blockIdx.x + (at.j == 0 ? 1 : 0)) * Shape<DP, NB>::kPartFloats;
        for (int head = sub; head < heads_in<NB>(p, at.h) && quad * 4 < p.dim; head += kHeadsAtOnce) {
            unsigned asked = 0;
            float value[4];
            uint2* const place = place_of<T, NB>(p, at.b, at.h, head, quad);
            float* const sums = part + head * DP + quad * 4;
            if (whole) {
                const uint2 packed = *place;
                const unsigned x = which(packed.x, kOdd), y = which(packed.y, kOdd);
                asked = (x & 1u) | (x >> 16) << 1 | (y & 1u) << 2 | (y >> 16) << 3;
                const float2 v = Half2<T>::unpack(packed.x), w = Half2<T>::unpack(packed.y);
                value[0] = v.x, value[1] = v.y, value[2] = w.x, value[3] = w.y;
            } else {
                const float l = part[8 * NB * DP + head * 2 + 1];
                for (int i = 0; i < 4; ++i) {
                    value[i] = sums[i];
                    asked |= (unsigned)(value[i] != value[i] && l < INFINITY) << i;
                }
            }
            if (asked == 0) continue;
            infinities_of<T>(p, at.b, kv, quad * 4, from, to, asked, value);
            if (whole) *place = make_uint2(Half2<T>::pack(value[0], value[1]), Half2<T>::pack(value[2], value[3]));
            else
                for (int i = 0; i < 4; ++i) sums[i] = value[i];
        }
        if (at.rel + places_of(at.tiles) - at.j >= count) return;
        at.next_unit(p, p.kv_heads * p.chunks);
    }
}

template <typename T, int DP, int NB>
__global__ void __launch_bounds__((Shape<DP, NB>::kAllThreads), (Shape<DP, NB>::kCtas))
paged_attention_kernel(const __grid_constant__ AttentionParams p) {
    using S = Shape<DP, NB>;
    extern __shared__ __align__(1024) unsigned char smem[];                 // the rows are aligned to their size
    __shared__ __align__(8) uint64_t s_full[kWarps][S::kStages], s_empty[kWarps][S::kStages];
    __shared__ int64_t s_scan[kWarps];
    __shared__ unsigned s_mask[kWarps][S::kStages];
    __shared__ float2 s_stat[kWarps][8];
    __shared__ Place s_first;
    __shared__ int s_flag[2];
    __shared__ bool s_odd[kThreads];                                        // whether the thread has stored a NaN that may be an infinity

    sm100::grid_launch_dependents();
    const int tid = threadIdx.x, lane = tid & 31, warp_id = tid >> 5;
    if (lane == 0 && warp_id < kWarps) {
        for (int i = 0; i < S::kStages; ++i) {
            sm100::mbar_init(sm100::smem_u32(&s_full[warp_id][i]), 33);     // 32 lanes' copies and the mask
            sm100::mbar_init(sm100::smem_u32(&s_empty[warp_id][i]), 1);
        }
        sm100::fence_barrier_init();
    }
    __syncwarp();
    sm100::grid_dependency_wait();

    const int heads = p.kv_heads * p.chunks;
    const int ctas = gridDim.x, cta = blockIdx.x;

    // ---- the list's length, and where this CTA's run starts
    if (tid == 0) s_flag[0] = *reinterpret_cast<const uint64_t*>(p.workspace) == kReady;
    const int per = (p.requests + kThreads - 1) / kThreads;
    const int first_request = min(tid * per, p.requests), last_request = warp_id < kWarps ? min(first_request + per, p.requests) : first_request;
    int64_t mine = 0;
    for (int b = first_request; b < last_request; ++b) mine += places_of(tiles_of(clamped_length(p, b)));
    int64_t upto = mine;
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t u = __shfl_up_sync(0xFFFFFFFFu, upto, o);
        if (lane >= o) upto += u;
    }
    if (lane == 31 && warp_id < kWarps) s_scan[warp_id] = upto;
    __syncthreads();
    if (!s_flag[0]) {                                                       // a workspace that was not prepared
        if (cta == 0 && tid == 0) atomicExch(p.status, (int)DPS_ERR_WORKSPACE);
        return;
    }
    int64_t total = 0, before = upto - mine;
    for (int w = 0; w < kWarps; ++w) {
        if (w < warp_id) before += s_scan[w];
        total += s_scan[w];
    }
    const int64_t all = total * heads;
    const bool narrow = all <= INT32_MAX;                                   // (64-bit divisions take 100 ns each)
    const int64_t each = narrow ? (int)all / ctas : all / ctas;
    const int more = (int)(all - each * ctas);                              // the first CTAs have one tile more
    const int64_t start = cta * each + min(cta, more);
    const int count = (int)each + (cta < more ? 1 : 0);                     // (below 2^31: checked on the host)
    if (count > 0) {
        const int64_t at = narrow ? (int)start / heads : start / heads;     // in tiles of requests
        if (at >= before && at < before + mine) {
            int b = first_request;
            int64_t from = before;
            int length = clamped_length(p, b), tiles = tiles_of(length);
            while (at >= from + places_of(tiles) && b + 1 < last_request) {
                from += places_of(tiles);
                length = clamped_length(p, ++b);
                tiles = tiles_of(length);
            }
            const int64_t inside = start - from * heads;
            const int places = places_of(tiles), h = narrow ? (int)inside / places : (int)(inside / places);
            Place first{b, h, (int)(inside - (int64_t)h * places), tiles, length, 0};
            if (first.j >= tiles) {                                         // behind the last tile: the next one's first
                if (places - first.j < count) first.next_unit(p, heads);
                else first.rel = count;
            }
            s_first = first;
        }
    }
    // requests without tokens: zeros; a length that is none
    const auto look_for_empty = [&](int thread, int threads) {
        for (int b = cta; b < p.requests; b += ctas) {
            const int n = p.lengths[b];
            if (thread == 0 && (n < 0 || (int64_t)n > p.longest)) atomicExch(p.status, (int)DPS_ERR_DATA);
            if (n <= 0 || p.longest == 0) {
                const int64_t row = (int64_t)p.kv_heads * p.group * p.dim / 8;
                uint4* to = reinterpret_cast<uint4*>(p.out) + b * row;
                for (int64_t i = thread; i < row; i += threads) to[i] = make_uint4(0, 0, 0, 0);
            }
        }
    };
    __syncthreads();
    if (count == 0 || s_first.rel >= count) {                               // no tile
        look_for_empty(tid, S::kAllThreads);
        return;
    }

    // ---- the warps that copy: each serves kServed of the others, 16 tokens of every tile for each
    if (warp_id >= kWarps) {
        constexpr int kServed = kWarps / S::kProducers, kLooks = (kServed * kWarpTokens + 31) / 32;
        constexpr int kRowChunks = DP / 8, kRowsAtOnce = 32 / kRowChunks;   // 16-byte chunks of a row, rows of one copy instruction
        // A lane copies chunk c of rows lane_row, lane_row + kRowsAtOnce, ...  Chunk c of row t lies at t * kRowBytes + (c ^ (t & 7)) * 16, so
        // that the eight rows of a matrix fragment fall on different banks; an exclusive or of the whole address does it, the rows being aligned.
        const int served = (warp_id - kWarps) * kServed;                    // the first one
        const int lane_row = lane / kRowChunks, lane_chunk = lane % kRowChunks;
        const uint32_t lane_dst = sm100::smem_u32(smem) + served * S::kStages * S::kStageBytes + lane_row * S::kRowBytes + ((lane_chunk ^ lane_row) << 4);
        const unsigned char* const lane_src = static_cast<const unsigned char*>(p.k) + lane_chunk * 16;
        const int64_t to_values = static_cast<const unsigned char*>(p.v) - static_cast<const unsigned char*>(p.k);
        const int64_t row_step = p.token_stride * 2;
        const bool chunk_there = lane_chunk * 8 < p.dim;
        const bool eights = p.page % 8 == 0;                                // eight rows in a row lie in one block, a token stride apart
        Place at = s_first;
        int id[kLooks], within[kLooks];                                     // of this lane's tokens: the block and the place in it
        int64_t head_off = 0;
        auto token_of = [&](int l) { return at.j * kTile + served * kWarpTokens + l * 32 + lane; };   // (a last tile's last token is below 2^31)
        auto mine_of = [&](int l) { return token_of(l) < at.length && l * 32 + lane < kServed * kWarpTokens; };
        auto look_up = [&](bool first) {
            if (first || at.j == 0) head_off = (int64_t)(p.chunks == 1 ? at.h : at.h / p.chunks) * p.head_stride;
#pragma unroll
            for (int l = 0; l < kLooks; ++l)
                if (mine_of(l)) {
                    const int index = (int)(((uint64_t)(unsigned)token_of(l) * p.page_magic) >> p.page_shift);
                    within[l] = token_of(l) - index * p.page;
                    id[l] = p.table[at.b * p.table_stride + index];
                }
        };
        look_up(true);
        int stage = 0;
        uint32_t parity = 1;                                                // the first round of the ring waits for nobody
        bool late = false;                                                  // a stage did not come back in time: no more waits, the lanes stay together
        for (bool more_tiles = true; more_tiles;) {
            int64_t off[kLooks];
            unsigned wanted[kLooks];
#pragma unroll
            for (int l = 0; l < kLooks; ++l) {
                const bool inside = mine_of(l), known = inside && (unsigned)id[l] < (uint64_t)p.blocks;
                if (inside && !known) atomicExch(p.status, (int)DPS_ERR_DATA);
                off[l] = known ? (id[l] * p.block_stride + within[l] * p.token_stride + head_off) * 2 : 0;
                wanted[l] = __ballot_sync(0xFFFFFFFFu, known);
            }
            more_tiles = at.goes_on(count);
            if (more_tiles) {
                at.next(p, heads);
                look_up(false);
            }
#pragma unroll
            for (int c = 0; c < kServed; ++c) {
                const uint32_t full = sm100::smem_u32(&s_full[served + c][stage]);
                const uint32_t empty = sm100::smem_u32(&s_empty[served + c][stage]);
                if (!sm100::mbar_try_wait(empty, parity)) {
                    if (!late && !sm100::mbar_wait(empty, parity)) late = true;
                }
                const int64_t c_off = off[c * kWarpTokens / 32];
                const unsigned mask = (wanted[c * kWarpTokens / 32] >> (c * kWarpTokens % 32)) & 0xFFFFu;
                if (mask != 0) {
                    const uint32_t dst = lane_dst + (c * S::kStages + stage) * S::kStageBytes;
                    const unsigned lane_mask = chunk_there ? mask >> lane_row : 0u;
                    const unsigned char* row = lane_src;
#pragma unroll
                    for (int first = 0; first < kWarpTokens; first += kRowsAtOnce) {
                        if (!eights) row = lane_src + __shfl_sync(0xFFFFFFFFu, c_off, c * kWarpTokens % 32 + first + lane_row);
                        else if (first % 8 == 0) row = lane_src + __shfl_sync(0xFFFFFFFFu, c_off, c * kWarpTokens % 32 + first) + lane_row * row_step;
                        else row += kRowsAtOnce * row_step;
                        const bool there = (lane_mask >> first) & 1u;
                        const unsigned char* from = there ? row : static_cast<const unsigned char*>(p.k);
                        const uint32_t to = (dst ^ ((first & 7) << 4)) + first * S::kRowBytes;
                        warp::copy16(to, from, there ? 16 : 0);
                        warp::copy16(to + S::kValues, from + to_values, there ? 16 : 0);
                    }
                }
                if (lane == 0) {
                    s_mask[served + c][stage] = mask;
                    sm100::mbar_arrive(full);
                }
                warp::copies_arrive(full);
            }
            if (++stage == S::kStages) {
                stage = 0;
                parity ^= 1;
            }
        }
        look_for_empty(tid - kThreads, S::kAllThreads - kThreads);          // (while the others are still computing)
        if (late) atomicExch(p.status, (int)DPS_ERR_CUDA);
        warp::copies_wait();
        return;
    }

    // ---- the warps that compute
    const int column = lane & 3, row = lane >> 2;                           // of a fragment: heads 2 column, 2 column + 1; token row
    // queries of a (request, head): fragments of Q^T; where registers allow, the next one's are fetched while this one's tokens are read
    uint32_t qf[NB][DP / 16][2], q_next[NB][DP / 16][2];
    auto fetch_queries = [&](const Place& of, uint32_t (&to)[NB][DP / 16][2]) {
        const int kv = p.chunks == 1 ? of.h : of.h / p.chunks, chunk = of.h - kv * p.chunks;
        const unsigned char* base = static_cast<const unsigned char*>(p.q) + (of.b * p.q_row + ((int64_t)kv * p.group + chunk * 8 * NB) * p.q_head) * 2;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            const int head = nb * 8 + row;
            const bool there = chunk * 8 * NB + head < p.group;
            const unsigned char* q_row = base + (there ? head * p.q_head : 0) * 2;
#pragma unroll
            for (int i = 0; i < DP / 16; ++i)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int d = i * 16 + e * 8 + column * 2;
                    to[nb][i][e] = there && d < p.dim ? *reinterpret_cast<const uint32_t*>(q_row + d * 2) : 0u;
                }
        }
    };
    float o[NB][DP / 16][4], m[NB][2], l[NB][2];
    Place at = s_first;
    if (S::kQueriesAhead) fetch_queries(at, q_next);
    bool fresh = true;                                                      // a (request, head) starts here
    const bool from_start = at.j == 0;                                      // the run's first one starts with it
    bool first_unit = true, lost = false;                                   // lost: a copy did not arrive in time
    Split head_split, tail_split;                                           // of the run's first and last (request, head)
    // ldmatrix rows: of the keys tokens 0-15 of chunk 0, then of chunk 1; of the values tokens 0-7 of chunk 0 and of 1, then 8-15
    const uint32_t ring = sm100::smem_u32(smem) + warp_id * S::kStages * S::kStageBytes;
    const uint32_t k_frag = ring + (lane & 15) * S::kRowBytes + (((lane >> 4) ^ (lane & 7)) << 4);
    const uint32_t v_frag = ring + S::kValues + ((lane & 7) + ((lane >> 4) << 3)) * S::kRowBytes + ((((lane >> 3) & 1) ^ (lane & 7)) << 4);
    unsigned* const counters = reinterpret_cast<unsigned*>(p.workspace + kHeaderBytes);
    float* const parts = reinterpret_cast<float*>(p.workspace + kHeaderBytes + kCounterBytes);
    constexpr int kQuads = DP / 4, kHeadsAtOnce = kThreads / kQuads;
    const int quad = tid % kQuads, sub = tid / kQuads;
    auto heads_of = [&](int h) { return heads_in<NB>(p, h); };
    auto store = [&](int b, int h, int head, const float4& v, float factor) {
        if (quad * 4 < p.dim) {
            uint2 packed;
            packed.x = Half2<T>::pack(v.x * factor, v.y * factor);
            packed.y = Half2<T>::pack(v.z * factor, v.w * factor);
            const uint2 odd = make_uint2(which(packed.x, 0x7FFFu), which(packed.y, 0x7FFFu));
            if ((odd.x | odd.y) != 0u && factor > 0.f && factor < INFINITY) {
                packed = make_uint2(packed.x ^ odd.x, packed.y ^ odd.y);
                s_odd[tid] = true;
            }
            *place_of<T, NB>(p, b, h, head, quad) = packed;
        }
    };
    s_odd[tid] = false;
    auto meet = [] {                                                        // of the computing warps
        __syncwarp();
        sm100::named_barrier_sync(1, kThreads);
    };

    int stage = 0;
    uint32_t parity = 0;
    for (bool more_tiles = true; more_tiles;) {
        more_tiles = at.goes_on(count);
        if (fresh) {
            fresh = false;
            if (!S::kQueriesAhead) fetch_queries(at, qf);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
                for (int i = 0; i < DP / 16; ++i) {
                    if (S::kQueriesAhead) {
                        qf[nb][i][0] = q_next[nb][i][0];
                        qf[nb][i][1] = q_next[nb][i][1];
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[nb][i][e] = 0.f;
                }
                m[nb][0] = m[nb][1] = -INFINITY;
                l[nb][0] = l[nb][1] = 0.f;
            }
            if (S::kQueriesAhead && at.rel + places_of(at.tiles) - at.j < count) {
                Place soon = at;
                soon.next_unit(p, heads);
                fetch_queries(soon, q_next);
            }
        }
        if (!lost && !sm100::mbar_wait(sm100::smem_u32(&s_full[warp_id][stage]), parity)) lost = true;
        __syncwarp();
        const unsigned mask = s_mask[warp_id][stage];
        if (mask != 0) {
            const uint32_t keys = k_frag + stage * S::kStageBytes, values = v_frag + stage * S::kStageBytes;
            float s[NB][2][4];
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[nb][0][e] = s[nb][1][e] = 0.f;
#pragma unroll
            for (int i = 0; i < DP / 16; ++i) {
                uint32_t a[4];
                warp::ldmatrix_x4(a, keys ^ (i << 5));
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
                for (int e = 0; e < 4; ++e) pr[e] = exp2_approx(x[e] - top[e & 1]) * kLift<T>;
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
                warp::ldmatrix_x4_trans(a, values ^ (i << 5));
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    Half2<T>::mma(o[nb][i], a, ph[nb][0], ph[nb][1]);
                    Half2<T>::mma(o[nb][i], a, pl[nb][0], pl[nb][1]);
                }
            }
        }

        // ---- the end of a (request, head), or of the run
        const bool ends = at.j == at.tiles - 1;
        if (ends || !more_tiles) {
            const bool starts_here = !first_unit || from_start;
            const bool whole = ends && starts_here;
            // the stage just read is this warp's until it hands it back: its sums for the others, element d of a head at d ^ (head / 2 % 4 * 8),
            // which spreads the fragments over the banks
            auto sum_of = [&](int w, int head, int d) {
                return reinterpret_cast<float*>(smem + (w * S::kStages + stage) * S::kStageBytes + S::kValues) + head * DP + (d ^ ((head >> 1 & 3) * 8));
            };
            float* const part = parts + (int64_t)(2 * cta + (starts_here ? 1 : 0)) * S::kPartFloats;
            if (!whole) {                                                   // its first and last tile in the list, and their CTAs
                const int64_t unit = start + at.rel - at.j, unit_last = unit + at.tiles - 1, big = (int64_t)more * (each + 1);
                Split of;
                of.first = (int)(unit < big ? unit / (each + 1) : more + (unit - big) / each);
                of.last = (int)(unit_last < big ? unit_last / (each + 1) : more + (unit_last - big) / each);
                of.b = at.b;
                of.h = at.h;
                if (starts_here) tail_split = of;
                else head_split = of;
            }
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                __syncwarp();
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
                        *sum_of(warp_id, 2 * column + (e & 1), i * 16 + row + (e >> 1) * 8) = o[nb][i][e];
                meet();
#pragma unroll
                for (int head = sub; head < 8; head += kHeadsAtOnce) {
                    if (nb * 8 + head >= heads_of(at.h)) break;
                    Joined r;
#pragma unroll
                    for (int w = 0; w < kWarps; ++w) {
                        const float2 st = s_stat[w][head];
                        r.add(st.x, st.y, *reinterpret_cast<const float4*>(sum_of(w, head, quad * 4)));
                    }
                    if (whole) store(at.b, at.h, nb * 8 + head, r.o, 1.f / r.l);
                    else {
                        if (r.o.x != r.o.x || r.o.y != r.o.y || r.o.z != r.o.z || r.o.w != r.o.w) s_odd[tid] = true;
                        *reinterpret_cast<float4*>(part + (nb * 8 + head) * DP + quad * 4) = r.o;
                        if (quad == 0) *reinterpret_cast<float2*>(part + 8 * NB * DP + (nb * 8 + head) * 2) = make_float2(r.m, r.l);
                    }
                }
                meet();
            }
            fresh = true;
            first_unit = false;
        }
        __syncwarp();
        if (lane == 0) sm100::mbar_arrive(sm100::smem_u32(&s_empty[warp_id][stage]));
        if (++stage == S::kStages) {
            stage = 0;
            parity ^= 1;
        }
        if (more_tiles) at.next(p, heads);
    }
    if (lost) atomicExch(p.status, (int)DPS_ERR_CUDA);
    if (s_odd[tid]) settle_infinities<T, DP, NB>(p, s_first, count, parts);

    // ---- the splits that this CTA holds a part of: whoever comes last joins the parts, in their order
    if (head_split.last < 0 && tail_split.last < 0) return;
    meet();
    if (tid < 2) {
        const Split of = tid == 0 ? head_split : tail_split;
        // (the CTA's part, which the barrier has put in front of this, goes with it for all of the GPU)
        s_flag[tid] = of.last >= 0 && count_in(&counters[of.first]) == (unsigned)(of.last - of.first);
    }
    meet();
#pragma unroll 1
    for (int i = 0; i < 2; ++i) {
        if (!s_flag[i]) continue;
        const Split of = i == 0 ? head_split : tail_split;
        const int n = of.last - of.first + 1, used = heads_of(of.h);
        // kAtOnce parts at a time, their maxima and totals and their sums asked for together.  (One part after another, the 37 parts of a long request took
        // 14 us; as bulk copies into shared memory, which want a fence between the two kinds of access, 6.)
        constexpr int kMine = 8 * NB / kHeadsAtOnce, kAtOnce = kMine <= 2 ? 16 : DP == 256 ? 8 : 4;   // heads of a thread
        constexpr int kTeam = kQuads < 32 ? kQuads : 32;                    // neighbouring lanes that serve the same head: lane c of them weighs part c
        const auto part_of = [&](int c) { return parts + (int64_t)(2 * (of.first + c) + (c == 0 ? 1 : 0)) * S::kPartFloats; };
        Joined r[kMine];
#pragma unroll 1
        for (int c0 = 0; c0 < n; c0 += kAtOnce) {
            const int member = lane % kTeam, left = n - c0;
            float2 st[kMine];
            float4 v[kAtOnce][kMine];
#pragma unroll
            for (int x = 0; x < kMine; ++x)
                st[x] = __ldcg(reinterpret_cast<const float2*>(part_of(c0 + min(member, left - 1)) + 8 * NB * DP + (sub + x * kHeadsAtOnce) * 2));
#pragma unroll
            for (int c = 0; c < kAtOnce; ++c) {
                const float* const from = part_of(c0 + min(c, left - 1)) + sub * DP + quad * 4;
#pragma unroll
                for (int x = 0; x < kMine; ++x) v[c][x] = __ldcg(reinterpret_cast<const float4*>(from + x * kHeadsAtOnce * DP));
            }
#pragma unroll
            for (int x = 0; x < kMine; ++x) {
                if (member >= min(left, kAtOnce)) st[x] = make_float2(-INFINITY, 0.f);
                float top = st[x].x;
#pragma unroll
                for (int e = 1; e < kTeam; e <<= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, e));
                r[x].rescale(top);
                const float w = fmaxf(exp2_approx(st[x].x - r[x].m), kLeast);
                float total_of = w * st[x].y;
#pragma unroll
                for (int e = 1; e < kTeam; e <<= 1) total_of += __shfl_xor_sync(0xFFFFFFFFu, total_of, e);
                r[x].l += total_of;
#pragma unroll
                for (int c = 0; c < kAtOnce; ++c) {
                    const float f = __shfl_sync(0xFFFFFFFFu, w, lane / kTeam * kTeam + c);
                    if (c < left) {
                        r[x].o.x += f * v[c][x].x;
                        r[x].o.y += f * v[c][x].y;
                        r[x].o.z += f * v[c][x].z;
                        r[x].o.w += f * v[c][x].w;
                    }
                }
            }
        }
#pragma unroll
        for (int x = 0; x < kMine; ++x)
            if (sub + x * kHeadsAtOnce < used) store(of.b, of.h, sub + x * kHeadsAtOnce, r[x].o, r[x].l > 0.f ? 1.f / r[x].l : NAN);
        if (tid == 0) counters[of.first] = 0;                               // ready for the next call
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
    cfg.blockDim = dim3(S::kAllThreads);
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
    page_division(p.page, p.page_magic, p.page_shift);
    p.kv_heads = cache.heads;
    p.dim = cache.head_dim;
    p.group = q_heads / cache.heads;
    p.chunks = (p.group + 8 * column_blocks(p.group, p.dim) - 1) / (8 * column_blocks(p.group, p.dim));
    p.requests = (int)requests;
    p.scale_log2 = scale * 1.4426950408889634f;
    // a CTA counts its tiles in 32 bits, and the grid has at least as many CTAs as the smallest list that needs them
    int64_t most = (p.longest + kTile - 1) / kTile * p.kv_heads * p.chunks;
    most = most > kMaxCtas ? kMaxCtas : most;
    most = most * requests < 1 ? 1 : most * requests;
    return cache.type == DPS_TYPE_FP16 ? launch_typed<__half>(p, most, stream) : launch_typed<__nv_bfloat16>(p, most, stream);
}

}  // namespace dps
