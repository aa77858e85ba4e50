// generation_host_check.cpp — TEST INFRASTRUCTURE ONLY: drives the host code of the
// C entry points of generation (generation.cpp, built with AddressSanitizer and
// UndefinedBehaviorSanitizer) on a machine without a GPU. The launches are replaced
// by functions that check what they are handed: whatever a call passes on must be
// what include/mezo.h allows, computed here in 128 bits and apart from
// generation.cpp; small arrays vector by vector.
//
// Every argument is taken through its ordinary values and the ends of its type, one
// and two at a time. Exit status 0 when every check passed.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdio>
#include <cstring>
#include <vector>

#include "attention_launch.hpp"
#include "cache_append_launch.hpp"
#include "mezo.h"
#include "nf4_linear_launch.hpp"

using u128 = unsigned __int128;

static int g_checks, g_failed;
static unsigned long g_launches;

#define CHECK(cond)                                                                     \
    do {                                                                                \
        ++g_checks;                                                                     \
        if (!(cond) && ++g_failed <= 20)                                                \
            std::fprintf(stderr, "%s:%d: check failed: %s\n", __FILE__, __LINE__, #cond); \
    } while (0)

// A stretch of memory, its end in 128 bits.
struct Span {
    u128 from, to;
};

static Span span(uint64_t at, u128 bytes) { return {at, u128(at) + bytes}; }
static bool apart(Span a, Span b) { return a.from == a.to || b.from == b.to || a.to <= b.from || b.to <= a.from; }
static bool in_memory(Span a) { return a.to <= (u128(1) << 64); }
static u128 matrix(u128 rows, u128 cols, u128 ld, u128 element) { return ((rows - 1) * ld + cols) * element; }

static Span g_workspace;

extern "C" const char* hipGetErrorString(hipError_t) { return "stand-in"; }

// An array of vectors of `bytes`, by up to three dimensions.
struct Array {
    uint64_t at;
    u128 n[3], stride[3], bytes;

    u128 count() const { return n[0] * n[1] * n[2]; }
    Span all() const
    {
        if (!count()) return span(at, 0);
        return span(at, (n[0] - 1) * stride[0] + (n[1] - 1) * stride[1] + (n[2] - 1) * stride[2] + bytes);
    }
    void vectors(std::vector<Span>& out) const
    {
        for (u128 i = 0; i < n[0]; ++i)
            for (u128 j = 0; j < n[1]; ++j)
                for (u128 k = 0; k < n[2]; ++k) {
                    const u128 from = at + i * stride[0] + j * stride[1] + k * stride[2];
                    out.push_back({from, from + bytes});
                }
    }
};

// Whether no two of some arrays' vectors meet (those that are too many to list: not decided).
static bool disjoint(const std::vector<Array>& arrays)
{
    u128 total = 0;
    for (const Array& a : arrays) total += a.count();
    if (total > 4096) return true;
    std::vector<Span> v;
    for (const Array& a : arrays) a.vectors(v);
    std::sort(v.begin(), v.end(), [](const Span& a, const Span& b) { return a.from < b.from; });
    for (size_t i = 1; i < v.size(); ++i)
        if (v[i].from < v[i - 1].to) return false;
    return true;
}

static Array plain(uint64_t at, u128 bytes) { return {at, {bytes ? u128(1) : u128(0), 1, 1}, {0, 0, 0}, bytes}; }

namespace mezo {

hipError_t launch_cache_append(const AppendArgs& a, hipStream_t)
{
    ++g_launches;
    const u128 e = a.dtype == MEZO_F32 ? 4 : 2, dim = a.dim * e;
    CHECK(a.dtype <= MEZO_BF16 && a.docs >= 1 && a.kv_heads >= 1 && (a.q == 0) == (a.heads == 0));
    CHECK(a.dim >= 8 && a.dim <= 128 && a.dim % 8 == 0 && a.rot % 2 == 0 && a.rot <= a.dim && (!a.rot || a.freqs));
    CHECK(a.max_q >= 1 && a.max_q <= a.tokens && u128(a.docs) * a.max_q <= (1u << 28));
    CHECK(a.page_shift >= 3 && a.page_shift <= 16 && a.k && a.v && a.table && (!a.entries || a.pages));
    CHECK((a.q | a.k | a.v | a.q_out | a.k_cache | a.v_cache) % 16 == 0);
    CHECK((a.table | a.positions) % 8 == 0 && (a.pages | a.freqs) % 4 == 0 && (!a.n_pages || (a.k_cache && a.v_cache)));
    const uint64_t strides[] = {a.q_token, a.q_head, a.k_token, a.k_head, a.v_token, a.v_head, a.o_token,
                                a.o_head, a.kc_page, a.kc_row, a.kc_head, a.vc_page, a.vc_row, a.vc_head};
    for (uint64_t s : strides) CHECK(s % 16 == 0);
    const u128 rows = u128(1) << a.page_shift;
    const Array q = {a.q, {a.tokens, a.heads, 1}, {a.q_token, a.q_head, 0}, dim},
                out = {a.q_out, {a.tokens, a.heads, 1}, {a.o_token, a.o_head, 0}, dim},
                k = {a.k, {a.tokens, a.kv_heads, 1}, {a.k_token, a.k_head, 0}, dim},
                v = {a.v, {a.tokens, a.kv_heads, 1}, {a.v_token, a.v_head, 0}, dim},
                kc = {a.k_cache, {a.n_pages, rows, a.kv_heads}, {a.kc_page, a.kc_row, a.kc_head}, dim},
                vc = {a.v_cache, {a.n_pages, rows, a.kv_heads}, {a.vc_page, a.vc_row, a.vc_head}, dim},
                table = plain(a.table, u128(a.docs) * 40), pages = plain(a.pages, u128(a.entries) * 4),
                freqs = plain(a.freqs, a.rot / 2 * 4), positions = plain(a.positions, a.positions ? u128(a.tokens) * 8 : 0);
    for (const Array& x : {q, out, k, v, kc, vc, table, pages, freqs, positions}) CHECK(in_memory(x.all()));
    const bool in_place = a.q && a.q == a.q_out && a.q_token == a.o_token && a.q_head == a.o_head;
    CHECK(disjoint({out, kc, vc}));  // (each of itself, too)
    for (const Array& written : {out, kc, vc})
        for (const Array& read : {k, v, table, pages, freqs, positions}) {
            // (what is read may meet itself)
            std::vector<Span> one, other;
            if (written.count() + read.count() > 2000) continue;
            written.vectors(one);
            read.vectors(other);
            for (const Span& x : one)
                for (const Span& y : other) CHECK(apart(x, y));
        }
    for (const Array& written : {out, kc, vc}) {
        if ((&written == &out && in_place) || written.count() + q.count() > 2000) continue;
        if (written.at == out.at && in_place) continue;
        std::vector<Span> one, other;
        written.vectors(one);
        q.vectors(other);
        for (const Span& x : one)
            for (const Span& y : other) CHECK(apart(x, y));
    }
    return hipSuccess;
}

hipError_t launch_paged_attention(const PagedArgs& a, hipStream_t)
{
    ++g_launches;
    const u128 e = a.dtype == MEZO_F32 ? 4 : 2, dim = a.dim * e;
    CHECK(a.dtype <= MEZO_BF16 && a.docs >= 1 && a.heads >= 1 && a.kv_heads >= 1 && a.group * a.kv_heads == a.heads);
    CHECK(a.dim >= 8 && a.dim <= 128 && a.dim % 8 == 0 && a.max_q >= 1 && a.max_q <= a.q_tokens);
    CHECK(a.page_shift >= 3 && a.page_shift <= 16 && (!a.entries || (a.pages && a.n_pages && a.k && a.v)));
    CHECK(a.q && a.out && a.table && (a.q | a.k | a.v | a.out) % 16 == 0 && a.table % 8 == 0 && (a.lse | a.pages) % 4 == 0);
    CHECK((a.q_token | a.q_head | a.k_token | a.k_head | a.v_token | a.v_head | a.o_token | a.o_head | a.k_page | a.v_page) %
              16 == 0);
    const u128 rows = u128(1) << a.page_shift;
    CHECK(a.k_token < MEZO_ATTENTION_MAX_STRIDE && a.v_token < MEZO_ATTENTION_MAX_STRIDE);
    CHECK(rows * a.k_token < (u128(1) << 32) && rows * a.v_token < (u128(1) << 32));
    CHECK(std::isfinite(a.scale) && std::isfinite(a.softcap) && a.softcap >= 0);
    CHECK(!a.tree || (a.tree % 8 == 0 && a.tree_words >= 1 && a.tree_words <= 1024 && !a.slopes && a.causal));
    // the grid, and the keys' 32-bit arithmetic
    CHECK(u128(a.docs) * a.kv_heads < (1u << 24) && (u128(a.max_q) * a.group + 127) / 128 <= 65535);
    CHECK(a.max_k < (1ull << 31) - 256 && u128(a.max_k) <= a.entries * rows && a.splits >= 1 && a.splits <= 64);
    const Array q = {a.q, {a.q_tokens, a.heads, 1}, {a.q_token, a.q_head, 0}, dim},
                out = {a.out, {a.q_tokens, a.heads, 1}, {a.o_token, a.o_head, 0}, dim},
                k = {a.k, {a.n_pages, rows, a.kv_heads}, {a.k_page, a.k_token, a.k_head}, dim},
                v = {a.v, {a.n_pages, rows, a.kv_heads}, {a.v_page, a.v_token, a.v_head}, dim};
    const Span read[] = {q.all(), k.all(), v.all(), span(a.table, u128(a.docs) * 40), span(a.pages, u128(a.entries) * 4),
                         span(a.tree, a.tree ? u128(a.q_tokens) * a.tree_words * 8 : 0),
                         span(reinterpret_cast<uint64_t>(a.slopes), a.slopes ? u128(a.heads) * 4 : 0)};
    const u128 kept = u128(a.splits) * a.docs * a.max_q * a.heads;
    const Span lse = span(a.lse, a.lse ? u128(a.q_tokens) * a.heads * 4 : 0),
               partial = span(a.partial, a.splits > 1 ? (kept + 1) / 2 * 16 + kept * a.dim * 4 : 0);
    for (const Span& r : read) {
        CHECK(in_memory(r));
        CHECK(apart(r, out.all()) && apart(r, lse) && apart(r, partial));
    }
    CHECK(in_memory(out.all()) && in_memory(lse) && apart(out.all(), lse) && apart(out.all(), partial) && apart(lse, partial));
    CHECK(disjoint({out}));
    if (a.splits > 1) CHECK(a.partial % 16 == 0 && partial.from >= g_workspace.from && partial.to <= g_workspace.to);
    return hipSuccess;
}

hipError_t launch_nf4_linear(const NF4LinearArgs& a, hipStream_t)
{
    ++g_launches;
    const u128 xe = a.x_dtype == MEZO_F32 ? 4 : 2, ce = a.c_dtype == MEZO_F32 ? 4 : 2, m = a.m, n = a.n, k = a.k;
    CHECK(a.x_dtype <= MEZO_BF16 && a.c_dtype <= MEZO_BF16 && m >= 1 && n >= 1 && k >= 1);
    CHECK(m <= (1u << 30) && n <= (1u << 30) && k <= (1u << 23) && m * k <= MEZO_MAX_NUMEL && n * k <= MEZO_MAX_NUMEL &&
          m * n <= MEZO_MAX_NUMEL);
    CHECK(a.x && a.codes && a.absmax && a.c && a.x % xe == 0 && a.c % ce == 0 && (a.codes | a.absmax) % 16 == 0);
    CHECK(a.ldx >= a.k && a.ldc >= a.n);
    const Span c = span(a.c, matrix(m, n, a.ldc, ce)),
               read[] = {span(a.x, matrix(m, k, a.ldx, xe)), span(a.codes, (n * k + 1) / 2), span(a.absmax, (n * k + 63) / 64 * 4)};
    CHECK(in_memory(c));
    for (const Span& r : read) CHECK(in_memory(r) && apart(r, c) && apart(r, g_workspace));
    CHECK(apart(c, g_workspace));
    // what the launch lays out in the workspace: activations, a slab of weights, a split's sums
    const bool wide = a.x_dtype == MEZO_F32;
    const NF4Cut cut = cut_nf4(a.m, a.n, a.k, wide);
    const NF4Space s = nf4_space(a.m, a.n, a.k, wide);
    const u128 columns = (k + 63) / 64 * 64, planes = wide ? 3 : 1;
    CHECK(cut.splits >= 1 && cut.splits <= 16 && s.weights % 16 == 0 && s.partial % 16 == 0);
    if (cut.tile == kThin) {
        CHECK(cut.thin_rows == 0 || cut.thin_rows == 16 || cut.thin_rows == 64 || cut.thin_rows == 128);
        if (cut.thin_rows) CHECK(k % 64 == 0 && u128(s.weights) >= m * k * xe);
        if (!cut.thin_rows) CHECK(u128(s.weights) >= m * columns * 2 * planes);
        CHECK(cut.thin_rows != 16 || m <= 4);
        if (cut.splits > 1) CHECK(u128(s.bytes) >= s.partial + cut.splits * m * ((n + 3) / 4) * 16);
    } else {
        CHECK(cut.slab >= 1 && u128(s.weights) >= m * columns * 2 * planes);
        CHECK(u128(s.partial) >= s.weights + cut.slab * columns * 2 * planes);
        if (cut.splits > 1) CHECK(u128(s.bytes) >= s.partial + cut.splits * m * ((u128(cut.slab) + 3) / 4) * 16);
        // offsets within a tile by 32 bits, and the grids
        CHECK(255 * columns * 2 + 128 < (u128(1) << 32));
        CHECK((m * (columns / 8) + 255) / 256 < (u128(1) << 31) && (u128(cut.slab) * (columns / 8) + 255) / 256 < (u128(1) << 31));
        CHECK(((m + 63) / 64) * ((u128(cut.slab) + 63) / 64) < (u128(1) << 31));
    }
    // lanes of a launch's first dimension, 32 bits
    const u128 most = u128(1) << 32, lanes = m * (columns / 8) + 255;
    CHECK(lanes < most);
    if (cut.tile == kThin) {
        const u128 rows = cut.thin_rows ? cut.thin_rows : 16;
        CHECK((n + rows - 1) / rows * (cut.thin_rows ? 1024 : 512) < most && (m + 3) / 4 <= 65535);
    } else {
        const u128 size = cut.tile == k256x256 ? 256 : (cut.tile == k128x128 ? 128 : 64);
        CHECK((m + size - 1) / size * ((u128(cut.slab) + size - 1) / size) * (size == 256 ? 512 : 256) < most);
    }
    if (cut.splits > 1) CHECK(m * (cut.tile == kThin ? n : u128(cut.slab)) + 255 < most);
    CHECK(u128(s.bytes) <= g_workspace.to - g_workspace.from);
    return hipSuccess;
}

}  // namespace mezo

// ---- the calls -----------------------------------------------------------------------

static void* P(uint64_t at) { return reinterpret_cast<void*>(at); }

// Addresses of buffers that lie 2^32 bytes apart; none is read.
static uint64_t buffer(int i) { return 0x7F0000000000ull + uint64_t(i) * 0x100000000ull; }

static bool documented(int rc)
{
    return rc == MEZO_OK || rc == MEZO_EINVAL || rc == MEZO_EDTYPE || rc == MEZO_EOVERLAP || rc == MEZO_ERANGE;
}

template <class Call>
static int made(uint64_t workspace, uint64_t bytes, Call&& call)
{
    g_workspace = span(workspace, bytes);
    const unsigned long before = g_launches;
    const int rc = call();
    CHECK(documented(rc));
    if (rc != MEZO_OK) CHECK(g_launches == before);  // a refused call enqueues nothing
    return rc;
}

// The values an argument is taken through beside its ordinary one.
static const uint64_t kSizes[] = {0, 1, 2, 3, 8, 63, 64, 127, 128, 1000, 4097, 65536, 1ull << 20, (1ull << 23) + 1, 1ull << 24,
                                  (1ull << 30) + 1, 1ull << 31, (1ull << 32) - 1, 1ull << 32, 1ull << 36, 1ull << 48,
                                  1ull << 61, 1ull << 62, 1ull << 63, ~0ull - 127, ~0ull};
static const uint64_t kAddresses[] = {0, 1, 4, 8, 0x7F0000000008ull, 0x7F0000000010ull, 0x7F0000000080ull, 0x7F0000000400ull,
                                      0x7F0100000040ull, 0x7F0200000100ull, 0x7F0300000010ull, 0x7F0400000040ull,
                                      0x7F0500000100ull, ~0ull - 15, ~0ull - 255, 1ull << 63};
static const uint64_t kTypes[] = {0, 1, 2, 3, 0xFFFFFFFFu};

struct Argument {
    uint64_t value;
    const uint64_t* others;
    size_t count;
};
template <size_t N>
static Argument from(uint64_t value, const uint64_t (&others)[N])
{
    return {value, others, N};
}

// Every call with one or two of its arguments changed.
template <class Call>
static void sweep(const std::vector<Argument>& args, Call&& call)
{
    std::vector<uint64_t> v;
    for (const Argument& a : args) v.push_back(a.value);
    call(v);
    for (size_t i = 0; i < args.size(); ++i)
        for (size_t x = 0; x < args[i].count; ++x) {
            v[i] = args[i].others[x];
            call(v);
            for (size_t j = i + 1; j < args.size(); ++j) {
                for (size_t y = 0; y < args[j].count; ++y) {
                    v[j] = args[j].others[y];
                    call(v);
                }
                v[j] = args[j].value;
            }
            v[i] = args[i].value;
        }
}

static int append(const std::vector<uint64_t>& v)
{
    mezo_append_t a = {};
    a.q = P(v[0]);
    a.k = P(v[1]);
    a.v = P(v[2]);
    a.q_out = P(v[3]);
    a.k_cache = P(v[4]);
    a.v_cache = P(v[5]);
    a.docs = static_cast<const int64_t*>(P(v[6]));
    a.pages = static_cast<const int32_t*>(P(v[7]));
    a.freqs = static_cast<const float*>(P(v[8]));
    a.positions = static_cast<const int64_t*>(P(v[9]));
    uint64_t* const wide[] = {&a.tokens, &a.n_pages, &a.n_entries, &a.max_q,  &a.q_token, &a.q_head,
                              &a.k_token, &a.k_head, &a.v_token,   &a.v_head, &a.o_token, &a.o_head,
                              &a.kc_page, &a.kc_row, &a.kc_head,   &a.vc_page, &a.vc_row, &a.vc_head};
    for (int i = 0; i < 18; ++i) *wide[i] = v[10 + i];
    uint32_t* const narrow[] = {&a.n_docs, &a.heads, &a.kv_heads, &a.dim, &a.page_rows, &a.rot, &a.interleaved, &a.dtype};
    for (int i = 0; i < 8; ++i) *narrow[i] = uint32_t(v[28 + i]);
    return made(0, 0, [&] { return mezo_cache_append(&a, nullptr); });
}

static void appends()
{
    CHECK(mezo_cache_append(nullptr, nullptr) == MEZO_EINVAL);
    // arrays of their own; and queries, keys and values of one projection, keys and values of one cache
    const uint64_t one = buffer(0);
    const uint64_t at[2][6] = {{buffer(0), buffer(1), buffer(2), buffer(3), buffer(4), buffer(5)},
                               {one, one + 256, one + 384, one, buffer(4), buffer(4) + 2048}};
    for (int form = 0; form < 2; ++form) {
        const uint64_t token = form ? 256 : 128, key = form ? 256 : 64, page = form ? 2048 : 1024;
        std::vector<Argument> args;
        for (uint64_t x : at[form]) args.push_back(from(x, kAddresses));
        for (int i = 6; i < 10; ++i) args.push_back(from(buffer(i + 2), kAddresses));
        const uint64_t sizes[] = {5, 3, 2, 5, token, 64, key, 64, key, 64, token, 64, page, 64, 64, page, 64, 64, 2, 2, 1, 64, 16, 64};
        for (uint64_t x : sizes) args.push_back(from(x, kSizes));
        args.push_back(from(0, kTypes));
        args.push_back(from(MEZO_BF16, kTypes));
        sweep(args, append);
    }
}

static void attention()
{
    CHECK(mezo_paged_attention(nullptr, nullptr, nullptr, 0, nullptr) == MEZO_EINVAL);
    const uint32_t floats[] = {0, 0x3F800000u, 0xBF800000u, 0x7F800000u, 0x7FC00000u, 0x7F7FFFFFu, 1u};
    std::vector<uint64_t> bits(floats, floats + 7);
    const Argument number = {0x3E000000u, bits.data(), bits.size()}, cap = {0, bits.data(), bits.size()};
    for (uint64_t keys : {20ull, 5000ull}) {
        const uint64_t entries = keys / 16 + 1;
        sweep({from(buffer(0), kAddresses), from(buffer(1), kAddresses), from(buffer(2), kAddresses), from(buffer(3), kAddresses),
               from(buffer(4), kAddresses), from(buffer(5), kAddresses), from(0, kAddresses), from(buffer(7), kAddresses),
               from(0, kAddresses), from(10, kSizes), from(128, kSizes), from(64, kSizes), from(64, kSizes), from(64, kSizes),
               from(64, kSizes), from(64, kSizes), from(128, kSizes), from(64, kSizes), from(10, kSizes), from(keys, kSizes),
               from(entries, kSizes), from(entries + 2, kSizes), from(1024, kSizes), from(1024, kSizes), from(1, kSizes),
               from(2, kSizes), from(1, kSizes), from(64, kSizes), from(MEZO_F32, kTypes), from(1, kTypes), from(16, kSizes),
               from(1, kSizes), number, cap, from(buffer(6), kAddresses)},
              [](const std::vector<uint64_t>& v) {
                  mezo_attention_t a = {};
                  mezo_pages_t c = {};
                  a.q = P(v[0]);
                  a.k = P(v[1]);
                  a.v = P(v[2]);
                  a.out = P(v[3]);
                  a.lse = static_cast<float*>(P(v[4]));
                  a.docs = static_cast<const int64_t*>(P(v[5]));
                  a.slopes = static_cast<const float*>(P(v[6]));
                  c.list = static_cast<const int32_t*>(P(v[7]));
                  c.tree = static_cast<const uint64_t*>(P(v[8]));
                  uint64_t* const wide[] = {&a.q_tokens, &a.q_token, &a.q_head, &a.k_token, &a.k_head, &a.v_token, &a.v_head,
                                            &a.o_token, &a.o_head, &a.max_q, &a.max_k, &c.n_entries, &c.n_pages, &c.k_page, &c.v_page};
                  for (int i = 0; i < 15; ++i) *wide[i] = v[9 + i];
                  uint32_t* const narrow[] = {&a.n_docs, &a.heads, &a.kv_heads, &a.dim, &a.dtype, &a.causal, &c.rows, &c.tree_words};
                  for (int i = 0; i < 8; ++i) *narrow[i] = uint32_t(v[24 + i]);
                  const uint32_t f[2] = {uint32_t(v[32]), uint32_t(v[33])};
                  std::memcpy(&a.scale, &f[0], 4);
                  std::memcpy(&a.softcap, &f[1], 4);
                  const uint64_t need = mezo_paged_attention_workspace(&a, &c);
                  for (uint64_t bytes : {need, need ? need - 1 : need}) {
                      const unsigned long before = g_launches;
                      made(v[34], bytes, [&] { return mezo_paged_attention(&a, &c, P(v[34]), bytes, nullptr); });
                      if (bytes < need) CHECK(g_launches == before);
                  }
              });
    }
}

static void products()
{
    const uint64_t cases[][3] = {{5, 60, 256}, {1, 3000, 4096}, {300, 500, 1000}, {70, 50, 33}};
    for (const auto& s : cases)
        for (uint32_t type : {MEZO_F32, MEZO_BF16})
            sweep({from(buffer(0), kAddresses), from(type, kTypes), from(s[2], kSizes), from(buffer(1), kAddresses),
                   from(buffer(2), kAddresses), from(s[0], kSizes), from(s[1], kSizes), from(s[2], kSizes),
                   from(buffer(3), kAddresses), from(MEZO_BF16, kTypes), from(s[1], kSizes), from(buffer(9), kAddresses)},
                  [](const std::vector<uint64_t>& v) {
                      const uint64_t need = mezo_nf4_linear_workspace(v[5], v[6], v[7], uint32_t(v[1]), uint32_t(v[9]));
                      for (uint64_t bytes : {need, need ? need - 1 : need}) {
                          const int rc = made(v[11], bytes, [&] {
                              return mezo_nf4_linear(P(v[0]), uint32_t(v[1]), v[2], P(v[3]), static_cast<float*>(P(v[4])), v[5],
                                                     v[6], v[7], P(v[8]), uint32_t(v[9]), v[10], P(v[11]), bytes, nullptr);
                          });
                          if (bytes < need) CHECK(rc != MEZO_OK);
                      }
                  });
}

int main()
{
    appends();
    const unsigned long a = g_launches;
    attention();
    const unsigned long b = g_launches;
    products();
    CHECK(a > 100 && b - a > 100 && g_launches - b > 100);  // the sweeps reach the launches
    std::printf("%d checks, %lu launches, %d failed\n", g_checks, g_launches, g_failed);
    return g_failed != 0;
}
