// generation.cpp — the C ABI of the operators of generation over a paged cache
// (include/mezo.h): argument checks and launches on the caller's stream. Nothing here
// allocates; scratch memory is the caller's.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "../../include/mezo.h"
#include "attention_launch.hpp"
#include "cache_append_launch.hpp"
#include "checks.hpp"
#include "host.hpp"
#include "nf4_linear_launch.hpp"

namespace {

using namespace mezo;

// An array of `count` parts of `extent` bytes, `stride` bytes apart (its outermost dimension).
struct Strided {
    uint64_t at, stride, count, extent;
};

// Its whole stretch (false: it does not end within the address space).
bool stretch(const Strided& s, Range& r)
{
    uint64_t n = 0;
    if (s.count && s.extent &&
        (__builtin_mul_overflow(s.count - 1, s.stride, &n) || __builtin_add_overflow(n, s.extent, &n)))
        return false;
    r = {s.at, n};
    return whole(r);
}

// Whether two arrays share no memory: their stretches do not meet, or one's parts lie in the
// gaps of the other (as the queries and keys of one projection's output do).
bool apart(const Strided& a, const Strided& b)
{
    Range ra, rb;
    if (!stretch(a, ra) || !stretch(b, rb)) return false;
    if (!overlap(ra, rb)) return true;
    if (a.stride != b.stride || a.stride == 0) return false;
    const uint64_t d = (b.at >= a.at ? b.at - a.at : a.stride - (a.at - b.at) % a.stride) % a.stride;
    return a.extent <= d && d + b.extent <= a.stride;
}

// (outer, inner) dimensions of n and m vectors of dim elements of e bytes, strides in
// elements, as parts of the dimension with the larger stride. false: past 64 bits.
bool parts_of(const void* at, uint64_t n, uint64_t n_stride, uint64_t m, uint64_t m_stride, uint64_t dim, uint64_t e,
              Strided& s)
{
    const bool outer = m <= 1 || (n > 1 && n_stride >= m_stride);
    const uint64_t count = outer ? n : m, stride = outer ? n_stride : m_stride;
    const uint64_t within = outer ? m : n, step = outer ? m_stride : n_stride;
    uint64_t extent = 0, bytes = 0;
    if (n == 0 || m == 0) {
        s = {address(at), 0, 0, 0};
        return true;
    }
    if (__builtin_mul_overflow(within - 1, step, &extent) || __builtin_add_overflow(extent, dim, &extent) ||
        __builtin_mul_overflow(extent, e, &extent) || __builtin_mul_overflow(stride, e, &bytes))
        return false;
    s = {address(at), bytes, count, extent};
    Range r;
    return stretch(s, r);
}

// Whether no two of an array's vectors share memory.
bool distinct(uint64_t n, uint64_t n_stride, uint64_t m, uint64_t m_stride, uint64_t dim)
{
    using wide = unsigned __int128;
    const wide a = n_stride, b = m_stride, n1 = n ? n - 1 : 0, m1 = m ? m - 1 : 0;
    return ((m1 == 0 || b >= dim) && (n1 == 0 || a >= m1 * b + dim)) ||
           ((n1 == 0 || a >= dim) && (m1 == 0 || b >= n1 * a + dim));
}

// The rows of a page: a power of two from MEZO_PAGE_MIN_ROWS to MEZO_PAGE_MAX_ROWS.
bool page_rows(uint32_t rows)
{
    return rows >= MEZO_PAGE_MIN_ROWS && rows <= MEZO_PAGE_MAX_ROWS && (rows & (rows - 1)) == 0;
}

// The pages of a cache as parts of one page each (false: past 64 bits).
bool cache_parts(const void* at, uint64_t n_pages, uint64_t page, uint32_t rows, uint64_t row, uint64_t heads,
                 uint64_t head, uint64_t dim, uint64_t e, Strided& s)
{
    Strided inner;
    Range r;
    if (!parts_of(at, rows, row, heads, head, dim, e, inner) || !stretch(inner, r)) return false;
    uint64_t bytes = 0;
    if (__builtin_mul_overflow(page, e, &bytes)) return false;
    s = {address(at), bytes, n_pages, r.bytes};
    return stretch(s, r);
}

// Whether the rows of the keys' pages lie in the gaps of the values' rows, or the other way round
// (as where each row of an array holds a token's keys and then its values): rows of all heads
// together, the same distance apart, also from page to page.
bool rows_apart(uint64_t k, uint64_t v, uint64_t n_pages, uint64_t k_page, uint64_t v_page, uint64_t k_row, uint64_t v_row,
                uint64_t heads, uint64_t k_head, uint64_t v_head, uint64_t dim, uint64_t e)
{
    if (k_row != v_row || k_row == 0 || (n_pages > 1 && (k_page % k_row || v_page % k_row))) return false;
    const uint64_t stride = k_row * e, k_bytes = ((heads - 1) * k_head + dim) * e, v_bytes = ((heads - 1) * v_head + dim) * e;
    const uint64_t d = (v >= k ? v - k : stride - (k - v) % stride) % stride;
    return k_bytes <= d && d + v_bytes <= stride;
}

// ---- appending to a paged cache ----------------------------------------------------

int cache_append(const mezo_append_t* p, void* stream)
{
    if (!p) return MEZO_EINVAL;
    const mezo_append_t& a = *p;
    if (!dense(a.dtype)) return MEZO_EDTYPE;
    const uint32_t heads = a.q ? a.heads : 0;
    if (a.kv_heads == 0 || a.kv_heads > MEZO_ATTENTION_MAX_HEADS || heads > MEZO_ATTENTION_MAX_HEADS || (a.q && !heads) ||
        a.dim < 8 || a.dim > kMaxHeadDim || a.dim % 8 || a.rot > a.dim || a.rot % 2 || !page_rows(a.page_rows) ||
        a.tokens > MEZO_MAX_NUMEL || a.n_entries > MEZO_MAX_NUMEL || a.n_pages >= (1ull << 32))
        return MEZO_EINVAL;
    const uint64_t most = a.max_q < a.tokens ? a.max_q : a.tokens;
    if (a.n_docs == 0 || most == 0) return MEZO_OK;
    if (!a.k || !a.v || !a.docs || (a.n_pages && (!a.k_cache || !a.v_cache)) || (a.n_entries && !a.pages) ||
        (a.q && !a.q_out) || (a.rot && !a.freqs) || most > (1ull << 28) / a.n_docs)
        return MEZO_EINVAL;
    if (!aligned(a.q, 16) || !aligned(a.k, 16) || !aligned(a.v, 16) || !aligned(a.q_out, 16) || !aligned(a.k_cache, 16) ||
        !aligned(a.v_cache, 16) || !aligned(a.docs, 8) || !aligned(a.positions, 8) || !aligned(a.pages, 4) ||
        !aligned(a.freqs, 4))
        return MEZO_EINVAL;
    const uint64_t e = element_bytes(a.dtype), align = 16 / e;
    const uint64_t strides[14] = {a.q_token, a.q_head, a.k_token, a.k_head, a.v_token, a.v_head, a.o_token,
                                  a.o_head, a.kc_page, a.kc_row, a.kc_head, a.vc_page, a.vc_row, a.vc_head};
    for (uint64_t s : strides)
        if (s % align) return MEZO_EINVAL;
    Strided q = {0, 0, 0, 0}, out = q, k, v, kc, vc;
    if (a.q && (!parts_of(a.q, a.tokens, a.q_token, heads, a.q_head, a.dim, e, q) ||
                !parts_of(a.q_out, a.tokens, a.o_token, heads, a.o_head, a.dim, e, out)))
        return MEZO_EINVAL;
    if (!parts_of(a.k, a.tokens, a.k_token, a.kv_heads, a.k_head, a.dim, e, k) ||
        !parts_of(a.v, a.tokens, a.v_token, a.kv_heads, a.v_head, a.dim, e, v) ||
        !cache_parts(a.k_cache, a.n_pages, a.kc_page, a.page_rows, a.kc_row, a.kv_heads, a.kc_head, a.dim, e, kc) ||
        !cache_parts(a.v_cache, a.n_pages, a.vc_page, a.page_rows, a.vc_row, a.kv_heads, a.vc_head, a.dim, e, vc))
        return MEZO_EINVAL;
    const Strided read[4] = {{address(a.docs), 0, 1, a.n_docs * 40ull},
                             {address(a.pages), 0, 1, a.n_entries * 4},
                             {address(a.freqs), 0, 1, a.rot / 2 * 4ull},
                             {address(a.positions), 0, 1, a.positions ? a.tokens * 8 : 0}};
    for (const Strided& r : read) {
        Range s;
        if (!stretch(r, s)) return MEZO_EINVAL;
    }
    // what is written shares memory with nothing, itself neither; but the queries may be turned
    // where they are
    if (!distinct(a.page_rows, a.kc_row, a.kv_heads, a.kc_head, a.dim) || (a.n_pages > 1 && kc.stride < kc.extent) ||
        !distinct(a.page_rows, a.vc_row, a.kv_heads, a.vc_head, a.dim) || (a.n_pages > 1 && vc.stride < vc.extent) ||
        (!apart(kc, vc) && !rows_apart(kc.at, vc.at, a.n_pages, a.kc_page, a.vc_page, a.kc_row, a.vc_row, a.kv_heads,
                                       a.kc_head, a.vc_head, a.dim, e)) ||
        (a.q && !distinct(a.tokens, a.o_token, heads, a.o_head, a.dim)))
        return MEZO_EOVERLAP;
    const Strided in[3] = {q, k, v};
    const bool in_place = a.q && a.q == a.q_out && a.q_token == a.o_token && a.q_head == a.o_head;
    for (int i = 0; i < 3; ++i)
        if (!apart(kc, in[i]) || !apart(vc, in[i]) || (!(in_place && i == 0) && !apart(out, in[i]))) return MEZO_EOVERLAP;
    for (const Strided& r : read)
        if (!apart(kc, r) || !apart(vc, r) || !apart(out, r)) return MEZO_EOVERLAP;
    if (!apart(out, kc) || !apart(out, vc)) return MEZO_EOVERLAP;
    AppendArgs g;
    g.q = address(a.q);
    g.k = address(a.k);
    g.v = address(a.v);
    g.q_out = a.q ? address(a.q_out) : 0;
    g.k_cache = address(a.k_cache);
    g.v_cache = address(a.v_cache);
    g.table = address(a.docs);
    g.pages = address(a.pages);
    g.freqs = address(a.freqs);
    g.positions = address(a.positions);
    uint64_t* const to[14] = {&g.q_token, &g.q_head, &g.k_token, &g.k_head, &g.v_token, &g.v_head, &g.o_token,
                              &g.o_head, &g.kc_page, &g.kc_row, &g.kc_head, &g.vc_page, &g.vc_row, &g.vc_head};
    for (int i = 0; i < 14; ++i) *to[i] = strides[i] * e;
    g.tokens = a.tokens;
    g.entries = a.n_entries;
    g.docs = a.n_docs;
    g.heads = heads;
    g.kv_heads = a.kv_heads;
    g.dim = a.dim;
    g.rot = a.rot;
    g.interleaved = a.interleaved ? 1u : 0u;
    g.dtype = a.dtype;
    g.n_pages = static_cast<uint32_t>(a.n_pages);
    g.page_shift = static_cast<uint32_t>(__builtin_ctz(a.page_rows));
    g.max_q = static_cast<uint32_t>(most);
    g.tile = g.parts = 1;  // (the launch's)
    MEZO_HIP(launch_cache_append(g, static_cast<hipStream_t>(stream)));
    return MEZO_OK;
}

// ---- attention over a paged cache -----------------------------------------------------

// The sizes of a call that do not depend on its pointers.
bool paged_sizes(const mezo_attention_t& a, const mezo_pages_t& c)
{
    return a.heads >= 1 && a.kv_heads >= 1 && a.heads <= MEZO_ATTENTION_MAX_HEADS && a.heads % a.kv_heads == 0 &&
           a.dim >= 8 && a.dim <= kMaxHeadDim && a.dim % 8 == 0 && a.q_tokens <= MEZO_MAX_NUMEL && page_rows(c.rows) &&
           c.n_entries <= MEZO_MAX_NUMEL && c.n_pages < (1ull << 32) && c.tree_words <= MEZO_TREE_MAX_WORDS &&
           (!c.tree || c.tree_words);
}

uint64_t paged_q(const mezo_attention_t& a) { return a.max_q < a.q_tokens ? a.max_q : a.q_tokens; }
uint64_t paged_k(const mezo_attention_t& a, const mezo_pages_t& c)
{
    const uint64_t all = c.n_pages ? c.n_entries * c.rows : 0;
    return a.max_k < all ? a.max_k : all;
}

bool paged_empty(const mezo_attention_t& a) { return a.n_docs == 0 || paged_q(a) == 0; }

// Whether the launch's grid holds the call.
bool paged_fits(const mezo_attention_t& a, const mezo_pages_t& c)
{
    const uint64_t q = paged_q(a), k = paged_k(a, c);
    return uint64_t(a.n_docs) * a.kv_heads < (1u << 24) && q * (a.heads / a.kv_heads) <= 65535ull * 128 &&
           k < (1ull << 31) - 256 && uint64_t(a.n_docs) * q * a.heads < (1ull << 40);
}

AttentionPlan paged_plan(const mezo_attention_t& a, const mezo_pages_t& c)
{
    return plan_attention(a.n_docs, a.heads, a.kv_heads, a.dim, static_cast<uint32_t>(paged_q(a)),
                          static_cast<uint32_t>(paged_k(a, c)));
}

int paged_attention(const mezo_attention_t* pa, const mezo_pages_t* pc, void* workspace, uint64_t workspace_bytes,
                    void* stream)
{
    if (!pa || !pc) return MEZO_EINVAL;
    const mezo_attention_t& a = *pa;
    const mezo_pages_t& c = *pc;
    if (!dense(a.dtype)) return MEZO_EDTYPE;
    // (a tree's tokens have no distance by their places in the cache, and no order but the tree's)
    if (!paged_sizes(a, c) || (c.tree && (a.slopes || !a.causal))) return MEZO_EINVAL;
    if (!std::isfinite(a.scale) || !std::isfinite(a.softcap) || a.softcap < 0.0f) return MEZO_ERANGE;
    if (paged_empty(a)) return MEZO_OK;
    if (!a.q || !a.out || !a.docs || (c.n_pages && (!a.k || !a.v)) || (c.n_entries && !c.list) || !paged_fits(a, c))
        return MEZO_EINVAL;
    if (!aligned(a.q, 16) || !aligned(a.k, 16) || !aligned(a.v, 16) || !aligned(a.out, 16) || !aligned(a.docs, 8) ||
        !aligned(a.lse, 4) || !aligned(a.slopes, 4) || !aligned(c.list, 4) || !aligned(c.tree, 8))
        return MEZO_EINVAL;
    const uint64_t e = element_bytes(a.dtype), align = 16 / e;
    const uint64_t strides[10] = {a.q_token, a.q_head, a.k_token, a.k_head, a.v_token, a.v_head, a.o_token, a.o_head,
                                  c.k_page, c.v_page};
    for (uint64_t s : strides)
        if (s % align) return MEZO_EINVAL;
    if (a.k_token * e >= MEZO_ATTENTION_MAX_STRIDE || a.v_token * e >= MEZO_ATTENTION_MAX_STRIDE ||
        a.k_token >= MEZO_ATTENTION_MAX_STRIDE || a.v_token >= MEZO_ATTENTION_MAX_STRIDE)
        return MEZO_EINVAL;
    // a page's rows, and the next page, by 32 bits
    constexpr uint64_t kMost = 1ull << 32;
    if (c.k_page >= kMost / e || c.v_page >= kMost / e || a.k_token * c.rows >= kMost / e || a.v_token * c.rows >= kMost / e)
        return MEZO_EINVAL;
    Strided s[4];
    if (!parts_of(a.q, a.q_tokens, a.q_token, a.heads, a.q_head, a.dim, e, s[0]) ||
        !parts_of(a.out, a.q_tokens, a.o_token, a.heads, a.o_head, a.dim, e, s[3]) ||
        !cache_parts(a.k, c.n_pages, c.k_page, c.rows, a.k_token, a.kv_heads, a.k_head, a.dim, e, s[1]) ||
        !cache_parts(a.v, c.n_pages, c.v_page, c.rows, a.v_token, a.kv_heads, a.v_head, a.dim, e, s[2]))
        return MEZO_EINVAL;
    Range r[4];
    for (int i = 0; i < 4; ++i)
        if (!stretch(s[i], r[i])) return MEZO_EINVAL;
    if (!distinct(a.q_tokens, a.o_token, a.heads, a.o_head, a.dim)) return MEZO_EOVERLAP;
    const AttentionPlan plan = paged_plan(a, c);
    if (plan.workspace && (!workspace || workspace_bytes < plan.workspace || !aligned(workspace, 16))) return MEZO_EINVAL;
    const Range lse = {address(a.lse), a.lse ? a.q_tokens * a.heads * 4 : 0},
                scratch = {address(workspace), plan.workspace};
    const Range read[9] = {r[0], r[1], r[2], {address(a.docs), a.n_docs * 40ull},
                           {address(a.slopes), a.slopes ? a.heads * 4ull : 0}, {address(c.list), c.n_entries * 4},
                           {address(c.tree), c.tree ? a.q_tokens * c.tree_words * 8 : 0}, r[3], lse};
    for (int i = 3; i < 9; ++i)
        if (!whole(read[i])) return MEZO_EINVAL;
    if (!whole(scratch)) return MEZO_EINVAL;
    if (clashes(r[3], read, 7) || (a.lse && clashes(lse, read, 8)) || (plan.workspace && clashes(scratch, read, 9)))
        return MEZO_EOVERLAP;
    PagedArgs g;
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
    g.k_page = static_cast<uint32_t>(c.k_page * e);
    g.v_page = static_cast<uint32_t>(c.v_page * e);
    g.q_tokens = a.q_tokens;
    g.k_tokens = 0;  // (the pages say what there is)
    g.pages = address(c.list);
    g.entries = c.n_pages ? c.n_entries : 0;
    g.tree = address(c.tree);
    g.tree_words = c.tree ? c.tree_words : 0;
    g.n_pages = static_cast<uint32_t>(c.n_pages);
    g.page_shift = static_cast<uint32_t>(__builtin_ctz(c.rows));
    g.docs = a.n_docs;
    g.heads = a.heads;
    g.kv_heads = a.kv_heads;
    g.group = a.heads / a.kv_heads;
    g.dim = a.dim;
    g.max_q = static_cast<uint32_t>(paged_q(a));
    g.max_k = static_cast<uint32_t>(paged_k(a, c));
    g.splits = plan.splits;
    g.chunk = plan.chunk;
    g.causal = a.causal ? 1u : 0u;
    g.dtype = a.dtype;
    g.scale = a.scale;
    g.softcap = a.softcap;
    MEZO_HIP(launch_paged_attention(g, static_cast<hipStream_t>(stream)));
    return MEZO_OK;
}

// ---- products with 4-bit weights ---------------------------------------------------

bool nf4_sizes(uint64_t m, uint64_t n, uint64_t k)
{
    // (rows as they are laid out, so that no launch is larger than a grid)
    const uint64_t columns = k <= MEZO_F8_MAX_COLS ? nf4_columns(k) : 0;
    return m >= 1 && n >= 1 && k >= 1 && columns && n <= MEZO_MAX_NUMEL / columns && m <= MEZO_MAX_NUMEL / columns &&
           m <= MEZO_MAX_NUMEL / n;
}

int nf4_linear(const void* x, uint32_t x_dtype, uint64_t ldx, const void* codes, const float* absmax, uint64_t m,
               uint64_t n, uint64_t k, void* c, uint32_t c_dtype, uint64_t ldc, void* workspace, uint64_t workspace_bytes,
               void* stream)
{
    if (!dense(x_dtype) || !dense(c_dtype)) return MEZO_EDTYPE;
    if (!x || !codes || !absmax || !c || !nf4_sizes(m, n, k) || (m > 1 && (ldx < k || ldc < n))) return MEZO_EINVAL;
    if (!aligned(x, element_bytes(x_dtype)) || !aligned(c, element_bytes(c_dtype)) || !aligned(codes, 16) ||
        !aligned(absmax, 16))
        return MEZO_EINVAL;
    const uint64_t need = nf4_space(m, n, k, x_dtype == MEZO_F32).bytes;
    if (need && (!workspace || workspace_bytes < need || !aligned(workspace, 16))) return MEZO_EINVAL;
    uint64_t in = 0, out = 0;
    if (!matrix_bytes(m, k, ldx, element_bytes(x_dtype), in) || !matrix_bytes(m, n, ldc, element_bytes(c_dtype), out))
        return MEZO_EINVAL;
    const Range all[5] = {{address(x), in}, {address(codes), (n * k + 1) / 2}, {address(absmax), (n * k + 63) / 64 * 4},
                          {address(c), out}, {address(workspace), need}};
    for (const Range& r : all)
        if (!whole(r)) return MEZO_EINVAL;
    if (clashes(all[3], all, 3) || (need && clashes(all[4], all, 4))) return MEZO_EOVERLAP;
    NF4LinearArgs g;
    g.x = address(x);
    g.ldx = m > 1 ? ldx : k;
    g.codes = address(codes);
    g.absmax = address(absmax);
    g.c = address(c);
    g.ldc = m > 1 ? ldc : n;
    g.workspace = address(workspace);
    g.m = m;
    g.n = n;
    g.k = k;
    g.x_dtype = x_dtype;
    g.c_dtype = c_dtype;
    MEZO_HIP(launch_nf4_linear(g, static_cast<hipStream_t>(stream)));
    return MEZO_OK;
}

}  // namespace

extern "C" {

uint64_t mezo_nf4_linear_workspace(uint64_t m, uint64_t n, uint64_t k, uint32_t x_dtype, uint32_t c_dtype)
{
    return dense(x_dtype) && dense(c_dtype) && nf4_sizes(m, n, k) ? nf4_space(m, n, k, x_dtype == MEZO_F32).bytes : 0;
}

int mezo_nf4_linear(const void* x, uint32_t x_dtype, uint64_t ldx, const void* codes, const float* absmax, uint64_t m,
                    uint64_t n, uint64_t k, void* c, uint32_t c_dtype, uint64_t ldc, void* workspace,
                    uint64_t workspace_bytes, void* stream)
{
    return guarded("mezo_nf4_linear", [&] {
        return nf4_linear(x, x_dtype, ldx, codes, absmax, m, n, k, c, c_dtype, ldc, workspace, workspace_bytes, stream);
    });
}

int mezo_cache_append(const mezo_append_t* a, void* stream)
{
    return guarded("mezo_cache_append", [&] { return cache_append(a, stream); });
}

uint64_t mezo_paged_attention_workspace(const mezo_attention_t* a, const mezo_pages_t* pages)
{
    if (!a || !pages || !dense(a->dtype) || !paged_sizes(*a, *pages) || paged_empty(*a) || !paged_fits(*a, *pages)) return 0;
    return paged_plan(*a, *pages).workspace;
}

int mezo_paged_attention(const mezo_attention_t* a, const mezo_pages_t* pages, void* workspace, uint64_t workspace_bytes,
                         void* stream)
{
    return guarded("mezo_paged_attention",
                   [&] { return paged_attention(a, pages, workspace, workspace_bytes, stream); });
}

}  // extern "C"
