// cache_append_launch.hpp — interface between the C-ABI host code (generation.cpp)
// and the kernels that append to a paged cache (cache_append.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace mezo {

// Strides in bytes.
struct AppendArgs {
    uint64_t q, k, v, q_out;  // q and q_out: 0 where there are no queries
    uint64_t k_cache, v_cache;
    uint64_t table;      // int64 [docs, 5]: q_first, q_len, first entry, k_len, (prefix)
    uint64_t pages;      // uint32 [entries]
    uint64_t freqs;      // fp32 [rot / 2]
    uint64_t positions;  // int64 [tokens], or 0
    uint64_t q_token, q_head, k_token, k_head, v_token, v_head, o_token, o_head;
    uint64_t kc_page, kc_row, kc_head, vc_page, vc_row, vc_head;
    uint64_t tokens, entries;
    uint32_t docs, heads, kv_heads, dim, rot, interleaved, dtype;
    uint32_t n_pages, page_shift, max_q;
    uint32_t tile, parts;  // tokens of a workgroup; workgroups that share a tile's heads
};

hipError_t launch_cache_append(const AppendArgs& args, hipStream_t stream);

}  // namespace mezo
