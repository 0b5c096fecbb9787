// The operators of a decoder step between its linear layers: launchers (host side, not part of the ABI).  Arguments as in
// include/dps.h, checked by step_api.cu; `status` is the current device's status word.
#pragma once
#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/dps.h"

namespace dps {

// n / page = n * magic >> shift for every n below 2^31: with 2^(s - 1) < page <= 2^s, magic = ceil(2^(31 + s) / page) fits 32 bits.
inline void page_division(int32_t page, unsigned& magic, unsigned& shift) {
    int log = 0;
    while (((int64_t)1 << log) < page) ++log;
    shift = 31 + log;
    magic = (unsigned)((((uint64_t)1 << shift) + page - 1) / page);
}

cudaError_t launch_extend_block_tables(const int32_t* lengths, const int32_t* new_tokens, int64_t requests, const int32_t* granted,
                                       int64_t granted_count, int32_t* table, int64_t table_stride, int64_t table_width, int32_t page,
                                       int64_t blocks, int32_t* lengths_out, int32_t* token_starts, int32_t* positions, int64_t* slots,
                                       int64_t tokens, int32_t* granted_used, int* status, cudaStream_t stream);

cudaError_t launch_qk_norm_rope(const void* qkv, int64_t qkv_stride, int64_t tokens, int32_t q_heads, const dps_kv_cache& cache,
                                const int64_t* slots, const int32_t* positions, const float* cos_sin, int64_t max_position,
                                int32_t rotated, bool interleaved, const void* q_weight, const void* k_weight, float eps, void* q_out,
                                int64_t q_out_stride, int* status, cudaStream_t stream);

cudaError_t launch_paged_attention(const void* q, int64_t q_row, int64_t q_head, int64_t requests, int32_t q_heads,
                                   const dps_kv_cache& cache, const int32_t* table, int64_t table_stride, int64_t table_width,
                                   const int32_t* lengths, float scale, void* out, void* workspace, int* status, cudaStream_t stream);
size_t attention_workspace_bytes(int32_t q_heads, int32_t kv_heads, int32_t head_dim);
cudaError_t launch_attention_workspace_init(void* workspace, cudaStream_t stream);

constexpr int kRouteMaxExperts = 1024, kRouteMaxGroups = 32, kRouteMaxTop = 32;
cudaError_t launch_route_experts(const void* logits, int64_t logits_stride, int32_t type, int64_t tokens, int32_t experts, const float* bias,
                                 int32_t scoring, int32_t groups, int32_t top_groups, int32_t top_k, bool renormalise, float scale,
                                 int32_t* token_of_row, int32_t* expert_of_row, float* weights, int* status, cudaStream_t stream);

}  // namespace dps
