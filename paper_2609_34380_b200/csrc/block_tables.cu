// The block tables, positions and cache slots of a step, from the request lengths: one launch.
//
// Everything follows from two running sums over the requests: of their new tokens (where a request's rows start in the flat batch)
// and of the blocks that they take (where its share of the granted ids starts).  Bound by latency: a decode step is a few hundred
// bytes, the largest steps a megabyte.  So nothing is exchanged between CTAs: each sums all requests itself (out of L2), keeps the
// sums of the requests' runs -- one run per thread -- in shared memory, and then serves its share of the three lists (requests, granted
// blocks, rows), finding the request of an item by bisection of those sums and a walk through one run.
// 1500 requests, 65536 rows: 7.2 us in a graph (pages by division 8.3; 512 threads a block 7.5, 256 8.5), 9.0 in a stream; 13 requests, one token each: 3.5.
#include "dps_internal.h"
#include "sm100.cuh"
#include "step_ops.h"

namespace dps {

namespace {

struct TableParams {
    const int32_t* lengths;
    const int32_t* new_tokens;
    const int32_t* granted;
    int32_t* table;
    int64_t table_stride, table_width, blocks, tokens, granted_count;
    int32_t* lengths_out;
    int32_t* token_starts;
    int32_t* positions;
    int64_t* slots;
    int32_t* granted_used;
    int* status;
    int requests, page;
    unsigned page_magic, page_shift;        // n / page = n * page_magic >> page_shift, for n below 2^31
    __device__ __forceinline__ int pages(int n) const { return (int)(((uint64_t)(unsigned)n * page_magic) >> page_shift); }
    __device__ __forceinline__ int pages_up(int n) const { return n > 0 ? pages(n - 1) + 1 : 0; }
};

// One request: what it has, what it adds, where its shares start.
struct Request {
    int64_t row, share;          // first row of the batch, first granted block
    int length, added;           // added: rows that it occupies
    int have, fresh;             // blocks in the table, blocks to take
    bool valid;
    // row and share are set; reads the rest
    __device__ __forceinline__ void read(const TableParams& p, int b) {
        length = p.lengths[b];
        const int m = p.new_tokens[b];
        added = m < 0 ? 0 : m;
        const int64_t after = (int64_t)length + m;
        valid = length >= 0 && m >= 0 && after <= INT32_MAX && (added == 0 || row + added <= p.tokens);
        const int need = valid ? p.pages_up((int)after) : 0;
        valid &= need <= p.table_width;
        have = valid ? p.pages_up(length) : 0;
        fresh = valid ? need - have : 0;
    }
    __device__ __forceinline__ bool served(const TableParams& p) const { return valid && (fresh == 0 || share + fresh <= p.granted_count); }
    __device__ __forceinline__ void pass() {
        row += added;
        share += fresh;
    }
};

// Exclusive running sums of two numbers over the block's threads, and their totals: one barrier.
struct Pair {
    int64_t rows, share;
};
template <int THREADS>
__device__ __forceinline__ Pair block_scan(Pair v, Pair* s_warp, Pair* total) {
    constexpr int kWarps = THREADS / 32;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const auto warp_scan = [&](Pair x) {                     // inclusive
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t r = __shfl_up_sync(0xFFFFFFFFu, x.rows, o), t = __shfl_up_sync(0xFFFFFFFFu, x.share, o);
            if (lane >= o) {
                x.rows += r;
                x.share += t;
            }
        }
        return x;
    };
    const Pair upto = warp_scan(v);
    if (lane == 31) s_warp[warp] = upto;
    __syncthreads();
    const Pair warps = warp_scan(lane < kWarps ? s_warp[lane] : Pair{0, 0});
    *total = Pair{__shfl_sync(0xFFFFFFFFu, warps.rows, 31), __shfl_sync(0xFFFFFFFFu, warps.share, 31)};
    const int64_t rows = __shfl_sync(0xFFFFFFFFu, warps.rows, (warp + 31) & 31), share = __shfl_sync(0xFFFFFFFFu, warps.share, (warp + 31) & 31);
    return Pair{(warp > 0 ? rows : 0) + upto.rows - v.rows, (warp > 0 ? share : 0) + upto.share - v.share};
}

// The last of the runs that starts at or before x (their starts never fall).
template <int THREADS>
__device__ __forceinline__ int run_of(const int* starts, int x) {
    int at = 0;
#pragma unroll
    for (int step = THREADS / 2; step > 0; step >>= 1)
        if (starts[at + step] <= x) at += step;
    return at;
}

// (256 threads for as many requests: 13 requests, one token each, took 5.6 us with 1024 threads and two sums after one another.)
template <int THREADS>
__global__ void __launch_bounds__(THREADS) extend_block_tables_kernel(const TableParams p) {
    __shared__ int s_row[THREADS], s_share[THREADS];         // where the runs' rows and granted blocks start, cut off at the ends of the lists
    __shared__ Pair s_warp[2][THREADS / 32];
    __shared__ int64_t s_used[THREADS / 32];
    sm100::grid_launch_dependents();
    sm100::grid_dependency_wait();
    const int tid = threadIdx.x;
    const int per = (p.requests + THREADS - 1) / THREADS;
    const int first = min(tid * per, p.requests), last = min(first + per, p.requests);
    Request r;
    Pair all;
    const auto sums = [&](int64_t row, bool bounded) {       // of this thread's run: its rows, its share with the rows' end respected or not
        Pair v{0, 0};
        for (int b = first; b < last; ++b) {
            r.row = bounded ? row + v.rows : INT64_MIN / 2;  // (rows that never reach the end)
            r.read(p, b);
            v.rows += r.added;
            v.share += r.fresh;
        }
        return v;
    };
    Pair at = block_scan<THREADS>(sums(0, false), s_warp[0], &all);
    if (all.rows > p.tokens) {                               // some rows pass the end: their requests take no blocks
        const int64_t row = at.rows;
        at = block_scan<THREADS>(sums(row, true), s_warp[1], &all);
    }
    const int64_t row0 = at.rows, share0 = at.share, all_rows = all.rows, all_taken = all.share;
    s_row[tid] = (int)min(row0, p.tokens);
    s_share[tid] = (int)min(share0, p.granted_count);
    __syncthreads();
    bool bad = false;

    // the requests, by the first CTA
    if (blockIdx.x == 0) {
        int64_t used = 0;
        r.row = row0;
        r.share = share0;
        for (int b = first; b < last; ++b) {
            r.read(p, b);
            const bool served = r.served(p);
            p.lengths_out[b] = served ? r.length + r.added : r.length;
            p.token_starts[b] = (int)min(r.row, (int64_t)INT32_MAX);
            bad |= !served;
            if (served && r.fresh > 0) used = r.share + r.fresh;
            r.pass();
        }
        if (tid == 0) p.token_starts[p.requests] = (int)min(all_rows, (int64_t)INT32_MAX);
        if (all_taken <= p.granted_count) {
            if (tid == 0) p.granted_used[0] = (int)all_taken;
        } else {                                             // the largest end of a request that was served
            for (int o = 16; o > 0; o >>= 1) used = max(used, __shfl_xor_sync(0xFFFFFFFFu, used, o));
            if ((tid & 31) == 0) s_used[tid >> 5] = used;
            __syncthreads();
            if (tid == 0) {
                for (int w = 0; w < THREADS / 32; ++w) used = max(used, s_used[w]);
                p.granted_used[0] = (int)used;
            }
        }
    }

    const int64_t stride = (int64_t)gridDim.x * THREADS, mine = (int64_t)blockIdx.x * THREADS + tid;
    // the granted blocks: into the table
    for (int64_t g = mine; g < p.granted_count && g < all_taken; g += stride) {
        const int run = run_of<THREADS>(s_share, (int)g);
        int b = run * per;
        const int end = min(b + per, p.requests);
        r.row = s_row[run];
        r.share = s_share[run];
        for (; b < end; ++b) {
            r.read(p, b);
            if (g < r.share + r.fresh) break;
            r.pass();
        }
        if (b == end || !r.served(p)) continue;
        int block = p.granted[g];
        if ((uint32_t)block >= (uint64_t)p.blocks) {
            block = -1;
            bad = true;
        }
        p.table[b * p.table_stride + r.have + (g - r.share)] = block;
    }
    // the rows
    for (int64_t t = mine; t < p.tokens; t += stride) {
        int position = 0;
        int64_t slot = -1;
        if (t < all_rows) {
            const int run = run_of<THREADS>(s_row, (int)t);
            int b = run * per;
            const int end = min(b + per, p.requests);
            r.row = s_row[run];
            r.share = s_share[run];
            for (; b < end; ++b) {
                r.read(p, b);
                if (t < r.row + r.added) break;
                r.pass();
            }
            if (b < end && r.served(p)) {
                position = r.length + (int)(t - r.row);
                const int index = p.pages(position);
                // the entries behind `have` may be written by another CTA just now: they are read where they come from
                const int block = index < r.have ? p.table[b * p.table_stride + index] : p.granted[r.share + index - r.have];
                if ((uint32_t)block < (uint64_t)p.blocks) slot = (int64_t)block * p.page + (position - index * p.page);
                else bad = true;
            }
        }
        p.positions[t] = position;
        p.slots[t] = slot;
    }
    if (bad) atomicExch(p.status, (int)DPS_ERR_DATA);
}

}  // namespace

cudaError_t launch_extend_block_tables(const int32_t* lengths, const int32_t* new_tokens, int64_t requests, const int32_t* granted,
                                       int64_t granted_count, int32_t* table, int64_t table_stride, int64_t table_width, int32_t page,
                                       int64_t blocks, int32_t* lengths_out, int32_t* token_starts, int32_t* positions, int64_t* slots,
                                       int64_t tokens, int32_t* granted_used, int* status, cudaStream_t stream) {
    TableParams p;
    p.lengths = lengths;
    p.new_tokens = new_tokens;
    p.granted = granted;
    p.table = table;
    p.table_stride = table_stride;
    p.table_width = table_width;
    p.blocks = blocks;
    p.tokens = tokens;
    p.granted_count = granted_count;
    p.lengths_out = lengths_out;
    p.token_starts = token_starts;
    p.positions = positions;
    p.slots = slots;
    p.granted_used = granted_used;
    p.status = status;
    p.requests = (int)requests;
    p.page = page;
    page_division(page, p.page_magic, p.page_shift);
    const int64_t items = tokens > granted_count ? tokens : granted_count;
    const int threads = requests <= 256 ? 256 : 1024;
    int64_t ctas = (items + threads - 1) / threads;
    if (ctas > sm_count()) ctas = sm_count();
    if (ctas < 1) ctas = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3(threads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = threads == 256 ? cudaLaunchKernelEx(&cfg, extend_block_tables_kernel<256>, p) : cudaLaunchKernelEx(&cfg, extend_block_tables_kernel<1024>, p);
    if (e == cudaSuccess) count_launch();
    return e;
}

}  // namespace dps
