// attention_launch.hpp — interface between the C-ABI host code (forward.cpp) and
// the attention kernels (attention.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace mezo {

constexpr uint32_t kMaxHeadDim = 128;

struct AttentionArgs {
    uint64_t q, k, v, out;
    uint64_t lse;      // fp32 [q_tokens, heads], or 0
    uint64_t table;    // int64 [docs, 5]: q_first, q_len, k_first, k_len, prefix
    uint64_t partial;  // of split documents
    const float* slopes;
    // bytes from one token and from one head to the next
    uint64_t q_token, q_head, k_token, k_head, v_token, v_head, o_token, o_head;
    uint64_t q_tokens, k_tokens;  // rows of q and out, of k and v
    uint32_t docs, heads, kv_heads, group, dim, max_q, max_k, splits;
    uint32_t chunk;    // keys of a split, a multiple of 64
    uint32_t causal, dtype;
    float scale, softcap;
};

// How a call is cut: the most workgroups that share a document's keys, the keys of
// each, and the bytes of `partial`.
struct AttentionPlan {
    uint32_t splits, chunk;
    uint64_t workspace;
};
AttentionPlan plan_attention(uint32_t docs, uint32_t heads, uint32_t kv_heads, uint32_t dim, uint32_t max_q,
                             uint32_t max_k);

hipError_t launch_attention(const AttentionArgs& args, hipStream_t stream);

}  // namespace mezo
