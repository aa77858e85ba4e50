// attention_launch.hpp — interface between the C-ABI host code (forward.cpp) and
// the attention kernels (attention.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "plans.hpp"

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

hipError_t launch_attention(const AttentionArgs& args, hipStream_t stream);

}  // namespace mezo
