// The C ABI of the operators of a decoder step between its linear layers: argument validation, then the launchers.
// Nothing here allocates, synchronises or enqueues anything before every argument has been looked at.
#include "dps_internal.h"
#include "step_ops.h"

using namespace dps;

namespace {

constexpr int64_t kLimit = (int64_t)1 << 31;

inline bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
inline bool overlap(const void* a, size_t a_bytes, const void* b, size_t b_bytes) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y + b_bytes && y < x + a_bytes;
}

// Whether `bytes` bytes at `out` lie over one of n rows of `width` bytes, `stride` apart.  (Room between the rows is no row, if they follow one another.)
bool over_rows(const void* out, size_t bytes, const void* rows, int64_t n, int64_t stride, int64_t width) {
    if (bytes == 0 || n == 0 || width <= 0 || !overlap(out, bytes, rows, (size_t)((n > 1 ? (n - 1) * stride : 0) + width))) return false;
    if (n == 1 || stride < width) return true;
    const int64_t apart = (int64_t)(reinterpret_cast<uintptr_t>(out) - reinterpret_cast<uintptr_t>(rows)) % stride, column = apart < 0 ? apart + stride : apart;
    return column < width || column + (int64_t)bytes > stride;
}

dps_status check_cache(const dps_kv_cache* c) {
    if (c == nullptr) return DPS_ERR_NULL;
    if (c->type != DPS_TYPE_FP16 && c->type != DPS_TYPE_BF16) return DPS_ERR_UNSUPPORTED;
    if (c->head_dim <= 0 || c->head_dim > 256 || c->head_dim % 8 != 0) return DPS_ERR_SHAPE;
    if (c->heads <= 0 || c->heads > 65535 || c->page_tokens <= 0 || c->blocks < 0 || c->blocks >= kLimit) return DPS_ERR_SHAPE;
    if (c->block_stride < 0 || c->token_stride < 0 || c->head_stride < 0) return DPS_ERR_SHAPE;
    const auto even = [](int64_t n, int64_t stride) { return n <= 1 || stride % 8 == 0; };      // (a stride that is never taken may be any)
    if (!even(c->blocks, c->block_stride) || !even(c->page_tokens, c->token_stride) || !even(c->heads, c->head_stride)) return DPS_ERR_ALIGN;
    // the largest offset in bytes fits 63 bits
    const int64_t most = (int64_t)1 << 60;
    const auto reach = [&](int64_t n, int64_t stride) { return n <= 1 || stride <= most / n; };
    if (!reach(c->blocks, c->block_stride) || !reach(c->page_tokens, c->token_stride) || !reach(c->heads, c->head_stride)) return DPS_ERR_SHAPE;
    if (c->blocks > 0 && (!c->k || !c->v)) return DPS_ERR_NULL;
    if (!aligned(c->k, 16) || !aligned(c->v, 16)) return DPS_ERR_ALIGN;
    return DPS_OK;
}

dps_status of(cudaError_t e) { return e == cudaSuccess ? DPS_OK : DPS_ERR_CUDA; }

}  // namespace

extern "C" {

dps_status dps_extend_block_tables(const int32_t* lengths, const int32_t* new_tokens, int64_t B, const int32_t* granted, int64_t G,
                                   int32_t* block_table, int64_t table_stride, int64_t table_width, int32_t page_tokens,
                                   int64_t blocks, int32_t* lengths_out, int32_t* token_starts, int32_t* positions, int64_t* slots,
                                   int64_t T, int32_t* granted_used, void* cuda_stream) {
    if (B < 0 || B > ((int64_t)1 << 20) || G < 0 || G >= kLimit || T < 0 || T >= kLimit || page_tokens <= 0) return DPS_ERR_SHAPE;
    if (table_width < 0 || table_width >= kLimit || blocks < 0 || blocks >= kLimit) return DPS_ERR_SHAPE;
    if (B > 1 && (table_stride < table_width || table_stride > INT64_MAX / 8 / B)) return DPS_ERR_SHAPE;
    if (!token_starts || !granted_used) return DPS_ERR_NULL;
    if (B > 0 && (!lengths || !new_tokens || !lengths_out || (table_width > 0 && !block_table))) return DPS_ERR_NULL;
    if ((G > 0 && !granted) || (T > 0 && (!positions || !slots))) return DPS_ERR_NULL;
    for (const void* p : {(const void*)lengths, (const void*)new_tokens, (const void*)granted, (const void*)block_table,
                          (const void*)lengths_out, (const void*)token_starts, (const void*)positions, (const void*)granted_used})
        if (!aligned(p, 4)) return DPS_ERR_ALIGN;
    if (!aligned(slots, 8)) return DPS_ERR_ALIGN;
    // the inputs are read by every block of the launch while others write the outputs
    struct Array {
        const void* at;
        size_t bytes;
    };
    const size_t n = (size_t)B * 4;
    const Array inputs[] = {{lengths, n}, {new_tokens, n}, {granted, (size_t)G * 4}};
    const Array outputs[] = {{lengths_out, n}, {token_starts, n + 4}, {positions, (size_t)T * 4}, {slots, (size_t)T * 8}, {granted_used, 4}};
    const auto meet = [](const Array& a, const Array& b) { return a.bytes > 0 && b.bytes > 0 && overlap(a.at, a.bytes, b.at, b.bytes); };
    for (const Array& out : outputs) {
        for (const Array& in : inputs)
            if (meet(out, in)) return DPS_ERR_DATA;
        for (const Array& other : outputs)
            if (&other != &out && meet(out, other)) return DPS_ERR_DATA;
    }
    int* status;
    const dps_status st = device_status_word(&status);
    if (st != DPS_OK) return st;
    return of(launch_extend_block_tables(lengths, new_tokens, B, granted, G, block_table, table_stride, table_width, page_tokens, blocks,
                                         lengths_out, token_starts, positions, slots, T, granted_used, status,
                                         static_cast<cudaStream_t>(cuda_stream)));
}

dps_status dps_qk_norm_rope(const void* qkv, int64_t qkv_stride, int64_t T, int32_t q_heads, const dps_kv_cache* cache,
                            const int64_t* slots, const int32_t* positions, const float* cos_sin, int64_t max_position,
                            int32_t rotated, int32_t interleaved, const void* q_weight, const void* k_weight, float eps, void* q_out,
                            int64_t q_out_stride, void* cuda_stream) {
    const dps_status ok = check_cache(cache);
    if (ok != DPS_OK) return ok;
    if (T < 0 || T >= kLimit || q_heads < 0 || q_heads > 65535) return DPS_ERR_SHAPE;
    if (rotated < 0 || rotated > cache->head_dim || rotated % 16 != 0 || max_position < 0 || max_position >= kLimit) return DPS_ERR_SHAPE;
    if (!(eps >= 0.f)) return DPS_ERR_SHAPE;
    const int64_t row = ((int64_t)q_heads + 2 * cache->heads) * cache->head_dim, q_row = (int64_t)q_heads * cache->head_dim;
    if (T > 1 && (qkv_stride < row || q_out_stride < q_row)) return DPS_ERR_SHAPE;
    if (T > 1 && (qkv_stride > INT64_MAX / 4 / T || q_out_stride > INT64_MAX / 4 / T)) return DPS_ERR_SHAPE;
    if (T > 1 && (qkv_stride % 8 != 0 || q_out_stride % 8 != 0)) return DPS_ERR_ALIGN;
    // warps are numbered in 31 bits; one serves at least four query, key or value heads of a token
    if (T * (((int64_t)q_heads + 3) / 4 + 2 * (((int64_t)cache->heads + 3) / 4)) >= kLimit - 64) return DPS_ERR_SHAPE;
    if (T == 0) return DPS_OK;
    if (!qkv || !slots || (q_heads > 0 && !q_out)) return DPS_ERR_NULL;
    if (rotated > 0 && (!positions || !cos_sin)) return DPS_ERR_NULL;
    if ((q_weight == nullptr) != (k_weight == nullptr)) return DPS_ERR_NULL;
    if (!aligned(qkv, 16) || !aligned(q_out, 16) || !aligned(cos_sin, 16) || !aligned(q_weight, 16) || !aligned(k_weight, 16)) return DPS_ERR_ALIGN;
    if (!aligned(slots, 8) || !aligned(positions, 4)) return DPS_ERR_ALIGN;
    // in place each warp writes what it has read itself; with other strides, or over other columns, it would write another one's.  (Rows of one stride may
    // lie between each other: columns of one wide buffer.)
    if (q_heads > 0 && (q_out != qkv || (T > 1 && q_out_stride != qkv_stride))) {
        const auto span = [&](int64_t stride, int64_t width) { return (size_t)(((T - 1) * (T > 1 ? stride : 0) + width) * 2); };
        if (overlap(qkv, span(qkv_stride, row), q_out, span(q_out_stride, q_row))) {
            if (T == 1 || q_out_stride != qkv_stride) return DPS_ERR_DATA;
            const int64_t apart = (int64_t)(reinterpret_cast<uintptr_t>(q_out) - reinterpret_cast<uintptr_t>(qkv)) / 2 % qkv_stride;
            const int64_t column = apart < 0 ? apart + qkv_stride : apart;      // of the queries in qkv's rows
            if (column < row || column + q_row > qkv_stride) return DPS_ERR_DATA;
        }
    }
    int* status;
    const dps_status st = device_status_word(&status);
    if (st != DPS_OK) return st;
    return of(launch_qk_norm_rope(qkv, qkv_stride, T, q_heads, *cache, slots, positions, cos_sin, max_position, rotated, interleaved != 0,
                                  q_weight, k_weight, eps, q_out, q_out_stride, status, static_cast<cudaStream_t>(cuda_stream)));
}

dps_status dps_paged_attention(const void* q, int64_t q_row_stride, int64_t q_head_stride, int64_t B, int32_t q_heads,
                               const dps_kv_cache* cache, const int32_t* block_table, int64_t table_stride, int64_t table_width,
                               const int32_t* lengths, float scale, void* out, void* workspace, size_t workspace_bytes,
                               void* cuda_stream) {
    const dps_status ok = check_cache(cache);
    if (ok != DPS_OK) return ok;
    if (B < 0 || B > ((int64_t)1 << 20) || q_heads <= 0 || q_heads > 65535 || q_heads % cache->heads != 0) return DPS_ERR_SHAPE;
    if (table_width < 0 || table_width >= kLimit || (B > 1 && (table_stride < table_width || table_stride > INT64_MAX / 8 / B)))
        return DPS_ERR_SHAPE;
    if (q_row_stride < 0 || q_head_stride < 0 || (B > 1 && q_row_stride > INT64_MAX / 4 / B) || q_head_stride > INT64_MAX / 4 / q_heads)
        return DPS_ERR_SHAPE;
    if ((B > 1 && q_row_stride % 8 != 0) || (q_heads > 1 && q_head_stride % 8 != 0)) return DPS_ERR_ALIGN;
    if (!(scale - scale == 0.f)) return DPS_ERR_SHAPE;      // Inf, NaN
    // tiles of 64 tokens: a block counts its share of them in 32 bits
    const int64_t longest = table_width * cache->page_tokens < kLimit ? table_width * cache->page_tokens : kLimit;
    if ((longest / 64 + 2) * q_heads >= ((int64_t)1 << 38) / (B > 0 ? B : 1)) return DPS_ERR_SHAPE;
    if (B == 0) return DPS_OK;
    if (!q || !lengths || !out || (table_width > 0 && !block_table)) return DPS_ERR_NULL;
    if (!aligned(q, 16) || !aligned(out, 16) || !aligned(block_table, 4) || !aligned(lengths, 4)) return DPS_ERR_ALIGN;
    if (!workspace || !aligned(workspace, 16)) return DPS_ERR_WORKSPACE;
    if (workspace_bytes < attention_workspace_bytes(q_heads, cache->heads, cache->head_dim)) return DPS_ERR_WORKSPACE;
    // in place the queries that a result replaces are its own, which all its parts have read; in another layout they would be others'
    const int64_t dense = (int64_t)q_heads * cache->head_dim;
    const bool in_place = out == q && (B == 1 || q_row_stride == dense) && (q_heads == 1 || q_head_stride == cache->head_dim);
    if (!in_place && over_rows(out, (size_t)(B * dense * 2), q, B, q_row_stride * 2, ((q_heads - 1) * q_head_stride + cache->head_dim) * 2)) return DPS_ERR_DATA;
    int* status;
    const dps_status st = device_status_word(&status);
    if (st != DPS_OK) return st;
    return of(launch_paged_attention(q, q_row_stride, q_head_stride, B, q_heads, *cache, block_table, table_stride, table_width, lengths,
                                     scale, out, workspace, status, static_cast<cudaStream_t>(cuda_stream)));
}

size_t dps_paged_attention_workspace_bytes(int32_t q_heads, int32_t kv_heads, int32_t head_dim) {
    if (kv_heads <= 0 || q_heads <= 0 || q_heads > 65535 || q_heads % kv_heads != 0 || head_dim <= 0 || head_dim > 256 || head_dim % 8 != 0)
        return 0;
    return attention_workspace_bytes(q_heads, kv_heads, head_dim);
}

dps_status dps_paged_attention_workspace_init(void* workspace, size_t workspace_bytes, void* cuda_stream) {
    if (!workspace || !aligned(workspace, 16) || workspace_bytes < attention_workspace_bytes(1, 1, 64)) return DPS_ERR_WORKSPACE;
    int* status;
    const dps_status st = device_status_word(&status);
    if (st != DPS_OK) return st;
    return of(launch_attention_workspace_init(workspace, static_cast<cudaStream_t>(cuda_stream)));
}

dps_status dps_route_experts(const void* logits, int64_t logits_stride, int32_t type, int64_t T, int32_t E, const float* bias,
                             int32_t scoring, int32_t groups, int32_t top_groups, int32_t top_k, int32_t renormalise, float scale,
                             int32_t* token_of_row, int32_t* expert_of_row, float* weights, void* cuda_stream) {
    if (type != DPS_TYPE_FP16 && type != DPS_TYPE_BF16 && type != DPS_TYPE_FP32) return DPS_ERR_UNSUPPORTED;
    if (scoring != DPS_SCORE_SOFTMAX && scoring != DPS_SCORE_SIGMOID) return DPS_ERR_MODE;
    if (T < 0 || E <= 0 || E > kRouteMaxExperts || groups <= 0 || groups > kRouteMaxGroups || E % groups != 0) return DPS_ERR_SHAPE;
    if (top_groups <= 0 || top_groups > groups || top_k <= 0 || top_k > kRouteMaxTop || top_k > top_groups * (E / groups)) return DPS_ERR_SHAPE;
    if (T > ((int64_t)1 << 30) || T * top_k >= kLimit || (T > 1 && (logits_stride < E || logits_stride > INT64_MAX / 8 / T))) return DPS_ERR_SHAPE;
    if (T == 0) return DPS_OK;
    if (!logits || !expert_of_row || !weights) return DPS_ERR_NULL;
    if (!aligned(logits, type == DPS_TYPE_FP32 ? 4 : 2) || !aligned(bias, 4) || !aligned(token_of_row, 4) || !aligned(expert_of_row, 4) ||
        !aligned(weights, 4))
        return DPS_ERR_ALIGN;
    // a warp writes its token's choices while others have yet to read their logits
    const int64_t size = type == DPS_TYPE_FP32 ? 4 : 2;
    const size_t choices = (size_t)(T * top_k) * 4;
    for (const void* out : {(const void*)token_of_row, (const void*)expert_of_row, (const void*)weights})
        if (out != nullptr && (over_rows(out, choices, logits, T, logits_stride * size, E * size) || (bias != nullptr && overlap(out, choices, bias, (size_t)E * 4))))
            return DPS_ERR_DATA;
    int* status;
    const dps_status st = device_status_word(&status);
    if (st != DPS_OK) return st;
    return of(launch_route_experts(logits, logits_stride, type, T, E, bias, scoring, groups, top_groups, top_k, renormalise != 0, scale,
                                   token_of_row, expert_of_row, weights, status, static_cast<cudaStream_t>(cuda_stream)));
}

}  // extern "C"
