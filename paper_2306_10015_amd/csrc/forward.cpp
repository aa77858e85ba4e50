// forward.cpp — the C ABI of the forward pass's operators (include/mezo.h):
// argument checks and launches on the caller's stream. Nothing here allocates;
// scratch memory is the caller's.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "../../include/mezo.h"
#include "attention_launch.hpp"
#include "checks.hpp"
#include "f8_launch.hpp"
#include "host.hpp"
#include "token_loss_launch.hpp"

namespace {

using namespace mezo;

// ---- 8-bit storage -----------------------------------------------------------

// Sizes of an 8-bit matrix.
bool f8_sizes(uint64_t rows, uint64_t cols)
{
    return rows >= 1 && cols >= 1 && rows <= MEZO_F8_MAX_ROWS && cols <= MEZO_F8_MAX_COLS &&
           rows <= MEZO_MAX_NUMEL / mezo::f8_code_stride(cols);
}

Range f8_codes(const void* codes, uint64_t rows, uint64_t cols)
{
    return {address(codes), rows * mezo::f8_code_stride(cols)};
}

Range f8_scales(const void* scales, uint64_t rows, uint64_t cols)
{
    return {address(scales), rows * mezo::f8_scale_stride(cols)};
}

// The checks of a quantization, and its kernel's arguments.
int check_quantize(const void* src, uint32_t dtype, uint64_t rows, uint64_t cols, uint64_t ld, void* codes,
                   void* scales, mezo::F8QuantArgs& a)
{
    if (!dense(dtype)) return MEZO_EDTYPE;
    if (!src || !codes || !scales || !f8_sizes(rows, cols) || (rows > 1 && ld < cols)) return MEZO_EINVAL;
    if (!aligned(src, element_bytes(dtype)) || !aligned(codes, 16) || !aligned(scales, 4)) return MEZO_EINVAL;
    uint64_t bytes;
    if (!matrix_bytes(rows, cols, ld, element_bytes(dtype), bytes)) return MEZO_EINVAL;
    const Range in = {address(src), bytes}, c = f8_codes(codes, rows, cols), s = f8_scales(scales, rows, cols);
    const Range read[2] = {in, c};
    if (!whole(in) || !whole(c) || !whole(s)) return MEZO_EINVAL;
    if (clashes(c, &in, 1) || clashes(s, read, 2)) return MEZO_EOVERLAP;
    a.values = in.at;
    a.ld = ld;
    a.codes = c.at;
    a.scales = s.at;
    a.rows = static_cast<uint32_t>(rows);
    a.cols = static_cast<uint32_t>(cols);
    a.dtype = dtype;
    return MEZO_OK;
}

// The checks of a product, and its kernel's arguments.
int check_matmul(const void* x_codes, const void* x_scales, const void* w_codes, const void* w_scales, uint64_t m,
                 uint64_t n, uint64_t k, void* c, uint32_t c_dtype, uint64_t ldc, void* workspace,
                 uint64_t workspace_bytes, mezo::F8MatmulArgs& a)
{
    if (!dense(c_dtype)) return MEZO_EDTYPE;
    if (!x_codes || !x_scales || !w_codes || !w_scales || !c || !f8_sizes(m, k) || !f8_sizes(n, k) ||
        m > MEZO_MAX_NUMEL / n || (m > 1 && ldc < n))
        return MEZO_EINVAL;
    if (!aligned(x_codes, 16) || !aligned(w_codes, 16) || !aligned(x_scales, 4) || !aligned(w_scales, 4) ||
        !aligned(c, element_bytes(c_dtype)))
        return MEZO_EINVAL;
    const uint64_t need = mezo::f8_matmul_workspace(m, n, k, c_dtype == MEZO_F32);
    if (need && (!workspace || workspace_bytes < need || !aligned(workspace, 16))) return MEZO_EINVAL;
    uint64_t bytes;
    if (!matrix_bytes(m, n, ldc, element_bytes(c_dtype), bytes)) return MEZO_EINVAL;
    const Range out = {address(c), bytes}, scratch = {address(workspace), need};
    const Range read[5] = {f8_codes(x_codes, m, k), f8_scales(x_scales, m, k), f8_codes(w_codes, n, k),
                           f8_scales(w_scales, n, k), out};
    for (const Range& r : read)
        if (!whole(r)) return MEZO_EINVAL;
    if (need && !whole(scratch)) return MEZO_EINVAL;
    if (clashes(out, read, 4) || (need && clashes(scratch, read, 5))) return MEZO_EOVERLAP;
    a.x = read[0].at;
    a.xs = read[1].at;
    a.w = read[2].at;
    a.ws = read[3].at;
    a.c = out.at;
    a.ldc = ldc;
    a.partial = scratch.at;
    a.m = static_cast<uint32_t>(m);
    a.n = static_cast<uint32_t>(n);
    a.k = static_cast<uint32_t>(k);
    a.out_dtype = c_dtype;
    return MEZO_OK;
}

// The layout of a linear call's workspace: x's codes, its scales, the product's.
struct LinearSpace {
    uint64_t scales, product, bytes;
};

LinearSpace linear_space(uint64_t m, uint64_t n, uint64_t k, uint32_t c_dtype)
{
    LinearSpace s;
    s.scales = m * mezo::f8_code_stride(k);
    s.product = s.scales + (m * mezo::f8_scale_stride(k) + 15) / 16 * 16;
    s.bytes = s.product + mezo::f8_matmul_workspace(m, n, k, c_dtype == MEZO_F32);
    return s;
}

int f8_linear(const void* x, uint32_t x_dtype, uint64_t ldx, const void* w_codes, const uint8_t* w_scales, uint64_t m,
              uint64_t n, uint64_t k, void* c, uint32_t c_dtype, uint64_t ldc, void* workspace,
              uint64_t workspace_bytes, void* stream)
{
    if (!dense(x_dtype) || !dense(c_dtype)) return MEZO_EDTYPE;
    if (!workspace || !aligned(workspace, 16) || !f8_sizes(m, k) || !f8_sizes(n, k)) return MEZO_EINVAL;
    const LinearSpace s = linear_space(m, n, k, c_dtype);
    if (workspace_bytes < s.bytes || !whole({address(workspace), s.bytes})) return MEZO_EINVAL;
    char* const codes = static_cast<char*>(workspace);
    mezo::F8QuantArgs q;
    mezo::F8MatmulArgs a;
    int rc = check_quantize(x, x_dtype, m, k, ldx, codes, codes + s.scales, q);
    if (rc == MEZO_OK)
        rc = check_matmul(codes, codes + s.scales, w_codes, w_scales, m, n, k, c, c_dtype, ldc, codes + s.product,
                          workspace_bytes - s.product, a);
    if (rc != MEZO_OK) return rc;
    uint64_t in = 0, out = 0;  // (both checked to fit)
    matrix_bytes(m, k, ldx, element_bytes(x_dtype), in);
    matrix_bytes(m, n, ldc, element_bytes(c_dtype), out);
    const Range scratch = {address(workspace), s.bytes};
    const Range others[4] = {{address(x), in}, {address(c), out}, f8_codes(w_codes, n, k), f8_scales(w_scales, n, k)};
    if (overlap(others[0], others[1]) || clashes(scratch, others, 4)) return MEZO_EOVERLAP;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    MEZO_HIP(mezo::launch_f8_quantize(q, st));
    MEZO_HIP(mezo::launch_f8_matmul(a, st));
    return MEZO_OK;
}

// ---- attention -------------------------------------------------------------------

// The sizes of an attention call that do not depend on its pointers.
bool attention_sizes(const mezo_attention_t& a)
{
    return a.heads >= 1 && a.kv_heads >= 1 && a.heads <= MEZO_ATTENTION_MAX_HEADS && a.heads % a.kv_heads == 0 &&
           a.dim >= 8 && a.dim <= mezo::kMaxHeadDim && a.dim % 8 == 0 && a.q_tokens <= MEZO_MAX_NUMEL &&
           a.k_tokens <= MEZO_MAX_NUMEL;
}

// Rows of work: what of max_q and max_k can be.
uint64_t most_q(const mezo_attention_t& a) { return a.max_q < a.q_tokens ? a.max_q : a.q_tokens; }
uint64_t most_k(const mezo_attention_t& a) { return a.max_k < a.k_tokens ? a.max_k : a.k_tokens; }

bool attention_empty(const mezo_attention_t& a) { return a.n_docs == 0 || most_q(a) == 0; }

// Whether the launch's grid holds the call.
bool attention_fits(const mezo_attention_t& a)
{
    const uint64_t q = most_q(a), k = most_k(a);
    return uint64_t(a.n_docs) * a.kv_heads < (1u << 24) && q * (a.heads / a.kv_heads) <= 65535ull * 128 &&
           k < (1ull << 31) - 256 && uint64_t(a.n_docs) * q * a.heads < (1ull << 40);
}

mezo::AttentionPlan attention_plan(const mezo_attention_t& a)
{
    return mezo::plan_attention(a.n_docs, a.heads, a.kv_heads, a.dim, static_cast<uint32_t>(most_q(a)),
                                static_cast<uint32_t>(most_k(a)));
}

int attention(const mezo_attention_t* p, void* workspace, uint64_t workspace_bytes, void* stream)
{
    if (!p) return MEZO_EINVAL;
    const mezo_attention_t& a = *p;
    if (!dense(a.dtype)) return MEZO_EDTYPE;
    if (!attention_sizes(a)) return MEZO_EINVAL;
    if (!std::isfinite(a.scale) || !std::isfinite(a.softcap) || a.softcap < 0.0f) return MEZO_ERANGE;
    if (attention_empty(a)) return MEZO_OK;
    if (!a.q || !a.out || !a.docs || (a.k_tokens && (!a.k || !a.v)) || !attention_fits(a)) return MEZO_EINVAL;
    const uint64_t e = element_bytes(a.dtype), align = 16 / e;
    if (!aligned(a.q, 16) || !aligned(a.k, 16) || !aligned(a.v, 16) || !aligned(a.out, 16) || !aligned(a.docs, 8) ||
        !aligned(a.lse, 4) || !aligned(a.slopes, 4))
        return MEZO_EINVAL;
    const uint64_t strides[8] = {a.q_token, a.q_head, a.k_token, a.k_head, a.v_token, a.v_head, a.o_token, a.o_head};
    for (uint64_t s : strides)
        if (s % align) return MEZO_EINVAL;
    if (a.k_token * e >= MEZO_ATTENTION_MAX_STRIDE || a.v_token * e >= MEZO_ATTENTION_MAX_STRIDE) return MEZO_EINVAL;
    // the bytes of each array; out's elements must not share memory with each other
    Range r[4];
    for (int i = 0; i < 4; ++i) {
        const uint64_t tokens = i == 1 || i == 2 ? a.k_tokens : a.q_tokens, heads = i == 1 || i == 2 ? a.kv_heads : a.heads;
        const void* const at[4] = {a.q, a.k, a.v, a.out};
        uint64_t n = 0, m = 0;
        if (tokens && (__builtin_mul_overflow(tokens - 1, strides[2 * i], &n) ||
                       __builtin_mul_overflow(heads - 1, strides[2 * i + 1], &m) || __builtin_add_overflow(n, m, &n) ||
                       __builtin_add_overflow(n, a.dim, &n) || __builtin_mul_overflow(n, e, &n)))
            return MEZO_EINVAL;
        r[i] = {address(at[i]), n};
        if (!whole(r[i])) return MEZO_EINVAL;
    }
    using wide = unsigned __int128;
    const wide oh = a.o_head, ot = a.o_token, h1 = a.heads - 1, t1 = a.q_tokens - 1;
    const bool by_token = (h1 == 0 || oh >= a.dim) && (t1 == 0 || ot >= h1 * oh + a.dim);  // [tokens, heads, dim]
    const bool by_head = (t1 == 0 || ot >= a.dim) && (h1 == 0 || oh >= t1 * ot + a.dim);   // [heads, tokens, dim]
    if (!by_token && !by_head) return MEZO_EOVERLAP;
    const mezo::AttentionPlan plan = attention_plan(a);
    if (plan.workspace && (!workspace || workspace_bytes < plan.workspace || !aligned(workspace, 16))) return MEZO_EINVAL;
    const Range lse = {address(a.lse), a.lse ? a.q_tokens * a.heads * 4 : 0},
                scratch = {address(workspace), plan.workspace};
    const Range read[7] = {r[0], r[1], r[2], {address(a.docs), a.n_docs * 40ull},
                           {address(a.slopes), a.slopes ? a.heads * 4ull : 0}, r[3], lse};
    if (!whole(read[3]) || !whole(read[4]) || !whole(lse) || !whole(scratch)) return MEZO_EINVAL;
    if (clashes(r[3], read, 5) || (a.lse && clashes(lse, read, 6)) || (plan.workspace && clashes(scratch, read, 7)))
        return MEZO_EOVERLAP;
    mezo::AttentionArgs g;
    g.q = r[0].at;
    g.k = r[1].at;
    g.v = r[2].at;
    g.out = r[3].at;
    g.lse = lse.at;
    g.table = address(a.docs);
    g.partial = scratch.at;
    g.slopes = a.slopes;
    g.q_token = a.q_token * e;
    g.q_head = a.q_head * e;
    g.k_token = a.k_token * e;
    g.k_head = a.k_head * e;
    g.v_token = a.v_token * e;
    g.v_head = a.v_head * e;
    g.o_token = a.o_token * e;
    g.o_head = a.o_head * e;
    g.q_tokens = a.q_tokens;
    g.k_tokens = a.k_tokens;
    g.docs = a.n_docs;
    g.heads = a.heads;
    g.kv_heads = a.kv_heads;
    g.group = a.heads / a.kv_heads;
    g.dim = a.dim;
    g.max_q = static_cast<uint32_t>(most_q(a));
    g.max_k = static_cast<uint32_t>(most_k(a));
    g.splits = plan.splits;
    g.chunk = plan.chunk;
    g.causal = a.causal ? 1u : 0u;
    g.dtype = a.dtype;
    g.scale = a.scale;
    g.softcap = a.softcap;
    MEZO_HIP(mezo::launch_attention(g, static_cast<hipStream_t>(stream)));
    return MEZO_OK;
}

// ---- the token loss ------------------------------------------------------------

uint64_t loss_workspace(uint64_t rows, uint64_t vocab)
{
    if (rows == 0 || vocab == 0) return 0;
    const uint64_t parts = mezo::loss_parts(rows, vocab);
    return parts > 1 ? rows * parts * sizeof(float2) : 0;
}

int token_loss(const void* logits, uint32_t dtype, uint64_t rows, uint64_t vocab, uint64_t ld, const int64_t* targets,
               float* losses, float* mean, void* workspace, uint64_t workspace_bytes, void* stream)
{
    if (!dense(dtype)) return MEZO_EDTYPE;
    if (rows == 0) return MEZO_EINVAL;
    if (!logits || !targets || !losses || vocab == 0 || rows > MEZO_LOSS_MAX_ROWS || (rows > 1 && ld < vocab))
        return MEZO_EINVAL;
    if (!aligned(logits, element_bytes(dtype)) || !aligned(targets, 8) || !aligned(losses, 4) || !aligned(mean, 4))
        return MEZO_EINVAL;
    uint64_t bytes;
    if (!matrix_bytes(rows, vocab, ld, element_bytes(dtype), bytes)) return MEZO_EINVAL;
    const uint64_t need = loss_workspace(rows, vocab);
    if (need && (!workspace || workspace_bytes < need || !aligned(workspace, 16))) return MEZO_EINVAL;
    const Range read[5] = {{address(logits), bytes}, {address(targets), rows * 8}, {address(losses), rows * 4},
                           {address(mean), mean ? 4u : 0u}, {address(workspace), need}};
    for (const Range& r : read)
        if (!whole(r)) return MEZO_EINVAL;
    if (clashes(read[2], read, 2) || (mean && clashes(read[3], read, 3)) || (need && clashes(read[4], read, 4)))
        return MEZO_EOVERLAP;
    mezo::LossArgs a;
    a.logits = read[0].at;
    a.ld = ld;
    a.vocab = vocab;
    a.targets = targets;
    a.losses = losses;
    a.mean = mean;
    a.rows = static_cast<uint32_t>(rows);
    a.parts = mezo::loss_parts(rows, vocab);
    a.partial = need ? static_cast<float2*>(workspace) : nullptr;
    a.dtype = dtype;
    MEZO_HIP(mezo::launch_token_loss(a, static_cast<hipStream_t>(stream)));
    return MEZO_OK;
}

}  // namespace

extern "C" {

int mezo_f8_quantize(const void* src, uint32_t src_dtype, uint64_t rows, uint64_t cols, uint64_t ld, void* codes,
                     uint8_t* scales, void* stream)
{
    return guarded("mezo_f8_quantize", [&]() -> int {
        mezo::F8QuantArgs a;
        const int rc = check_quantize(src, src_dtype, rows, cols, ld, codes, scales, a);
        if (rc != MEZO_OK) return rc;
        MEZO_HIP(mezo::launch_f8_quantize(a, static_cast<hipStream_t>(stream)));
        return MEZO_OK;
    });
}

uint64_t mezo_f8_matmul_workspace(uint64_t m, uint64_t n, uint64_t k, uint32_t c_dtype)
{
    return dense(c_dtype) && f8_sizes(m, k) && f8_sizes(n, k) ? mezo::f8_matmul_workspace(m, n, k, c_dtype == MEZO_F32) : 0;
}

int mezo_f8_matmul(const void* x_codes, const uint8_t* x_scales, const void* w_codes, const uint8_t* w_scales,
                   uint64_t m, uint64_t n, uint64_t k, void* c, uint32_t c_dtype, uint64_t ldc, void* workspace,
                   uint64_t workspace_bytes, void* stream)
{
    return guarded("mezo_f8_matmul", [&]() -> int {
        mezo::F8MatmulArgs a;
        const int rc = check_matmul(x_codes, x_scales, w_codes, w_scales, m, n, k, c, c_dtype, ldc, workspace,
                                    workspace_bytes, a);
        if (rc != MEZO_OK) return rc;
        MEZO_HIP(mezo::launch_f8_matmul(a, static_cast<hipStream_t>(stream)));
        return MEZO_OK;
    });
}

uint64_t mezo_f8_linear_workspace(uint64_t m, uint64_t n, uint64_t k, uint32_t c_dtype)
{
    return dense(c_dtype) && f8_sizes(m, k) && f8_sizes(n, k) ? linear_space(m, n, k, c_dtype).bytes : 0;
}

int mezo_f8_linear(const void* x, uint32_t x_dtype, uint64_t ldx, const void* w_codes, const uint8_t* w_scales,
                   uint64_t m, uint64_t n, uint64_t k, void* c, uint32_t c_dtype, uint64_t ldc, void* workspace,
                   uint64_t workspace_bytes, void* stream)
{
    return guarded("mezo_f8_linear", [&] {
        return f8_linear(x, x_dtype, ldx, w_codes, w_scales, m, n, k, c, c_dtype, ldc, workspace, workspace_bytes,
                         stream);
    });
}

uint64_t mezo_attention_workspace(const mezo_attention_t* a)
{
    if (!a || !dense(a->dtype) || !attention_sizes(*a) || attention_empty(*a) || !attention_fits(*a)) return 0;
    return attention_plan(*a).workspace;
}

int mezo_attention(const mezo_attention_t* a, void* workspace, uint64_t workspace_bytes, void* stream)
{
    return guarded("mezo_attention", [&] { return attention(a, workspace, workspace_bytes, stream); });
}

uint64_t mezo_token_loss_workspace(uint64_t rows, uint64_t vocab) { return loss_workspace(rows, vocab); }

int mezo_token_loss(const void* logits, uint32_t dtype, uint64_t rows, uint64_t vocab, uint64_t ld,
                    const int64_t* targets, float* losses, float* mean, void* workspace, uint64_t workspace_bytes,
                    void* stream)
{
    return guarded("mezo_token_loss", [&] {
        return token_loss(logits, dtype, rows, vocab, ld, targets, losses, mean, workspace, workspace_bytes, stream);
    });
}

}  // extern "C"
