// forward_host_check.cpp — TEST INFRASTRUCTURE ONLY: drives the host code of the
// forward pass's C entry points (forward.cpp, built with AddressSanitizer and
// UndefinedBehaviorSanitizer) on a machine without a GPU. The launches are replaced
// by functions that check what they are handed: whatever a call passes on must be
// what include/mezo.h allows, computed here in 128 bits and apart from forward.cpp.
//
// Every argument is taken through its ordinary values and the ends of its type, one
// and two at a time. Exit status 0 when every check passed.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdio>
#include <cstring>
#include <vector>

#include "attention_launch.hpp"
#include "f8_launch.hpp"
#include "mezo.h"
#include "token_loss_launch.hpp"

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
static u128 blocks(u128 cols) { return (cols + 127) / 128; }

// What was written to and read from by the launches of one call.
static std::vector<Span> g_read, g_written;

static void writes(Span s)
{
    CHECK(in_memory(s));
    for (const Span& r : g_read) CHECK(apart(s, r));
    for (const Span& w : g_written) CHECK(apart(s, w));
    g_written.push_back(s);
}

static void reads(Span s)
{
    CHECK(in_memory(s));
    g_read.push_back(s);
}

// The workspace of the call that is being made.
static Span g_workspace;

extern "C" const char* hipGetErrorString(hipError_t) { return "stand-in"; }

namespace mezo {

hipError_t launch_f8_quantize(const F8QuantArgs& a, hipStream_t)
{
    ++g_launches;
    const u128 element = a.dtype == MEZO_F32 ? 4 : 2;
    CHECK(a.dtype <= MEZO_BF16 && a.rows >= 1 && a.cols >= 1 && (a.rows == 1 || a.ld >= a.cols));
    CHECK(a.values && a.codes && a.scales && a.values % element == 0 && a.codes % 16 == 0 && a.scales % 4 == 0);
    CHECK(u128(a.rows) * blocks(a.cols) * 128 <= MEZO_MAX_NUMEL);
    reads(span(a.values, matrix(a.rows, a.cols, a.ld, element)));
    writes(span(a.codes, u128(a.rows) * blocks(a.cols) * 128));
    writes(span(a.scales, u128(a.rows) * ((blocks(a.cols) + 3) / 4 * 4)));
    return hipSuccess;
}

hipError_t launch_f8_matmul(const F8MatmulArgs& a, hipStream_t)
{
    ++g_launches;
    const u128 element = a.out_dtype == MEZO_F32 ? 4 : 2;
    CHECK(a.out_dtype <= MEZO_BF16 && a.m >= 1 && a.n >= 1 && a.k >= 1 && (a.m == 1 || a.ldc >= a.n));
    CHECK(a.x && a.xs && a.w && a.ws && a.c && a.c % element == 0);
    CHECK(a.x % 16 == 0 && a.w % 16 == 0 && a.xs % 4 == 0 && a.ws % 4 == 0);
    const u128 codes = blocks(a.k) * 128, scales = (blocks(a.k) + 3) / 4 * 4;
    std::vector<Span> operands = {span(a.x, a.m * codes), span(a.xs, a.m * scales), span(a.w, a.n * codes),
                                  span(a.ws, a.n * scales)};
    // (a linear call's own codes and scales, written just before, are among these)
    const Span c = span(a.c, matrix(a.m, a.n, a.ldc, element));
    CHECK(in_memory(c));
    for (const Span& o : operands) CHECK(in_memory(o) && apart(c, o));
    for (const Span& r : g_read) CHECK(apart(c, r));
    for (const Span& w : g_written) CHECK(apart(c, w));
    const F8Cut cut = cut_product(a.m, a.n, a.k, a.out_dtype == MEZO_F32);
    if (cut.splits > 1) {
        const Span p = span(a.partial, u128(cut.splits) * a.m * ((a.n + 3) / 4) * 16);
        CHECK(a.partial % 16 == 0 && p.from >= g_workspace.from && p.to <= g_workspace.to && apart(p, c));
        for (const Span& o : operands) CHECK(apart(p, o));
    }
    return hipSuccess;
}

hipError_t launch_attention(const AttentionArgs& a, hipStream_t)
{
    ++g_launches;
    const u128 e = a.dtype == MEZO_F32 ? 4 : 2;
    CHECK(a.dtype <= MEZO_BF16 && a.docs >= 1 && a.heads >= 1 && a.kv_heads >= 1 && a.group * a.kv_heads == a.heads);
    CHECK(a.dim >= 8 && a.dim <= 128 && a.dim % 8 == 0 && a.max_q >= 1 && a.max_q <= a.q_tokens && a.max_k <= a.k_tokens);
    CHECK(a.q && a.out && a.table && (!a.k_tokens || (a.k && a.v)));
    CHECK((a.q | a.k | a.v | a.out) % 16 == 0 && a.table % 8 == 0 && a.lse % 4 == 0);
    CHECK((a.q_token | a.q_head | a.k_token | a.k_head | a.v_token | a.v_head | a.o_token | a.o_head) % 16 == 0);
    CHECK(a.k_token < MEZO_ATTENTION_MAX_STRIDE && a.v_token < MEZO_ATTENTION_MAX_STRIDE);
    CHECK(std::isfinite(a.scale) && std::isfinite(a.softcap) && a.softcap >= 0);
    // the grid, and the keys' 32-bit arithmetic
    CHECK(u128(a.docs) * a.kv_heads < (1u << 24) && (u128(a.max_q) * a.group + 127) / 128 <= 65535);
    CHECK(a.max_k < (1ull << 31) - 256 && a.splits >= 1 && a.splits <= 64);
    auto array = [&](uint64_t at, u128 tokens, u128 heads, u128 token, u128 head) {
        return span(at, tokens ? (tokens - 1) * token + (heads - 1) * head + a.dim * e : 0);
    };
    reads(array(a.q, a.q_tokens, a.heads, a.q_token, a.q_head));
    reads(array(a.k, a.k_tokens, a.kv_heads, a.k_token, a.k_head));
    reads(array(a.v, a.k_tokens, a.kv_heads, a.v_token, a.v_head));
    reads(span(a.table, u128(a.docs) * 40));
    if (a.slopes) reads(span(reinterpret_cast<uint64_t>(a.slopes), u128(a.heads) * 4));
    writes(array(a.out, a.q_tokens, a.heads, a.o_token, a.o_head));
    if (a.lse) writes(span(a.lse, u128(a.q_tokens) * a.heads * 4));
    // no two elements of out share memory
    const u128 dim = a.dim * e, ot = a.o_token, oh = a.o_head, t1 = a.q_tokens - 1, h1 = a.heads - 1;
    CHECK(((!h1 || oh >= dim) && (!t1 || ot >= h1 * oh + dim)) || ((!t1 || ot >= dim) && (!h1 || oh >= t1 * ot + dim)));
    if (a.splits > 1) {
        const u128 kept = u128(a.splits) * a.docs * a.max_q * a.heads;
        const Span p = span(a.partial, (kept + 1) / 2 * 16 + kept * a.dim * 4);
        CHECK(a.partial % 16 == 0 && p.from >= g_workspace.from && p.to <= g_workspace.to);
        writes(p);
    }
    return hipSuccess;
}

hipError_t launch_token_loss(const LossArgs& a, hipStream_t)
{
    ++g_launches;
    const u128 element = a.dtype == MEZO_F32 ? 4 : 2;
    CHECK(a.dtype <= MEZO_BF16 && a.rows >= 1 && a.rows <= MEZO_LOSS_MAX_ROWS && a.vocab >= 1);
    CHECK(a.logits && a.logits % element == 0 && a.targets && a.losses && (a.rows == 1 || a.ld >= a.vocab));
    const uint64_t targets = reinterpret_cast<uint64_t>(a.targets), losses = reinterpret_cast<uint64_t>(a.losses),
                   mean = reinterpret_cast<uint64_t>(a.mean), partial = reinterpret_cast<uint64_t>(a.partial);
    CHECK(targets % 8 == 0 && losses % 4 == 0 && mean % 4 == 0 && a.parts == loss_parts(a.rows, a.vocab));
    reads(span(a.logits, matrix(a.rows, a.vocab, a.ld, element)));
    reads(span(targets, u128(a.rows) * 8));
    writes(span(losses, u128(a.rows) * 4));
    if (mean) writes(span(mean, 4));
    CHECK((a.parts > 1) == (partial != 0));
    if (partial) {
        const Span p = span(partial, u128(a.rows) * a.parts * 8);
        CHECK(partial % 16 == 0 && p.from >= g_workspace.from && p.to <= g_workspace.to);
        writes(p);
    }
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
    g_read.clear();
    g_written.clear();
    g_workspace = span(workspace, bytes);
    const unsigned long before = g_launches;
    const int rc = call();
    CHECK(documented(rc));
    if (rc != MEZO_OK) CHECK(g_launches == before);  // a refused call enqueues nothing
    return rc;
}

// The values an argument is taken through beside its ordinary one.
static const uint64_t kSizes[] = {0, 1, 2, 3, 63, 64, 127, 129, 1000, 4097, 65536, 1ull << 20, (1ull << 23) + 1, 1ull << 24,
                                  (1ull << 30) + 1, (1ull << 31) - 256, 1ull << 31, (1ull << 32) - 1, 1ull << 32, 1ull << 36,
                                  1ull << 48, 1ull << 61, 1ull << 62, 1ull << 63, ~0ull - 127, ~0ull};
static const uint64_t kAddresses[] = {0, 1, 4, 8, 0x7F0000000008ull, 0x7F0000000010ull, 0x7F0000000400ull, 0x7F0100000040ull,
                                      0x7F0200000100ull, 0x7F0300000010ull, 0x7F0400000040ull, ~0ull - 15, ~0ull - 255,
                                      (1ull << 63)};
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

static void quantize()
{
    sweep({from(buffer(0), kAddresses), from(MEZO_F32, kTypes), from(4, kSizes), from(256, kSizes), from(256, kSizes),
           from(buffer(1), kAddresses), from(buffer(2), kAddresses)},
          [](const std::vector<uint64_t>& v) {
              made(0, 0, [&] {
                  return mezo_f8_quantize(P(v[0]), uint32_t(v[1]), v[2], v[3], v[4], P(v[5]), static_cast<uint8_t*>(P(v[6])),
                                          nullptr);
              });
          });
}

static void products()
{
    for (uint64_t k : {256ull, 40000ull})
        sweep({from(buffer(0), kAddresses), from(buffer(1), kAddresses), from(buffer(2), kAddresses), from(buffer(3), kAddresses),
               from(5, kSizes), from(60, kSizes), from(k, kSizes), from(buffer(4), kAddresses), from(MEZO_BF16, kTypes),
               from(64, kSizes), from(buffer(5), kAddresses)},
              [](const std::vector<uint64_t>& v) {
                  const uint64_t need = mezo_f8_matmul_workspace(v[4], v[5], v[6], uint32_t(v[8]));
                  for (uint64_t bytes : {need, need ? need - 1 : need}) {
                      const int rc = made(v[10], bytes, [&] {
                          return mezo_f8_matmul(P(v[0]), static_cast<uint8_t*>(P(v[1])), P(v[2]), static_cast<uint8_t*>(P(v[3])),
                                                v[4], v[5], v[6], P(v[7]), uint32_t(v[8]), v[9], P(v[10]), bytes, nullptr);
                      });
                      if (bytes < need) CHECK(rc != MEZO_OK);
                  }
              });
    sweep({from(buffer(0), kAddresses), from(MEZO_F32, kTypes), from(256, kSizes), from(buffer(2), kAddresses),
           from(buffer(3), kAddresses), from(5, kSizes), from(60, kSizes), from(256, kSizes), from(buffer(4), kAddresses),
           from(MEZO_BF16, kTypes), from(64, kSizes), from(buffer(5), kAddresses)},
          [](const std::vector<uint64_t>& v) {
              const uint64_t need = mezo_f8_linear_workspace(v[5], v[6], v[7], uint32_t(v[9]));
              for (uint64_t bytes : {need, need ? need - 1 : need}) {
                  const int rc = made(v[11], bytes, [&] {
                      return mezo_f8_linear(P(v[0]), uint32_t(v[1]), v[2], P(v[3]), static_cast<uint8_t*>(P(v[4])), v[5], v[6],
                                            v[7], P(v[8]), uint32_t(v[9]), v[10], P(v[11]), bytes, nullptr);
                  });
                  if (bytes < need) CHECK(rc != MEZO_OK);
              }
          });
}

static void attention()
{
    CHECK(mezo_attention(nullptr, nullptr, 0, nullptr) == MEZO_EINVAL);
    CHECK(mezo_attention_workspace(nullptr) == 0);
    const uint32_t floats[] = {0, 0x3F800000u, 0xBF800000u, 0x7F800000u, 0xFF800000u, 0x7FC00000u, 0x7F7FFFFFu, 1u};
    std::vector<uint64_t> bits(floats, floats + 8);
    const Argument number = {0x3E000000u, bits.data(), bits.size()}, cap = {0, bits.data(), bits.size()};
    for (uint64_t keys : {20ull, 5000ull})
        sweep({from(buffer(0), kAddresses), from(buffer(1), kAddresses), from(buffer(2), kAddresses), from(buffer(3), kAddresses),
               from(buffer(4), kAddresses), from(buffer(5), kAddresses), from(0, kAddresses), from(10, kSizes), from(keys, kSizes),
               from(128, kSizes), from(64, kSizes), from(64, kSizes), from(64, kSizes), from(64, kSizes), from(64, kSizes),
               from(128, kSizes), from(64, kSizes), from(10, kSizes), from(keys, kSizes), from(1, kSizes), from(2, kSizes),
               from(1, kSizes), from(64, kSizes), from(MEZO_F32, kTypes), from(1, kTypes), number, cap, from(buffer(6), kAddresses)},
              [](const std::vector<uint64_t>& v) {
                  mezo_attention_t a;
                  a.q = P(v[0]);
                  a.k = P(v[1]);
                  a.v = P(v[2]);
                  a.out = P(v[3]);
                  a.lse = static_cast<float*>(P(v[4]));
                  a.docs = static_cast<const int64_t*>(P(v[5]));
                  a.slopes = static_cast<const float*>(P(v[6]));
                  uint64_t* const wide[] = {&a.q_tokens, &a.k_tokens, &a.q_token, &a.q_head, &a.k_token, &a.k_head, &a.v_token,
                                            &a.v_head,   &a.o_token,  &a.o_head,  &a.max_q,  &a.max_k};
                  for (int i = 0; i < 12; ++i) *wide[i] = v[7 + i];
                  uint32_t* const narrow[] = {&a.n_docs, &a.heads, &a.kv_heads, &a.dim, &a.dtype, &a.causal};
                  for (int i = 0; i < 6; ++i) *narrow[i] = uint32_t(v[19 + i]);
                  const uint32_t f[2] = {uint32_t(v[25]), uint32_t(v[26])};
                  std::memcpy(&a.scale, &f[0], 4);
                  std::memcpy(&a.softcap, &f[1], 4);
                  const uint64_t need = mezo_attention_workspace(&a);
                  for (uint64_t bytes : {need, need ? need - 1 : need}) {
                      const unsigned long before = g_launches;
                      made(v[27], bytes, [&] { return mezo_attention(&a, P(v[27]), bytes, nullptr); });
                      if (bytes < need) CHECK(g_launches == before);
                  }
              });
}

// An array of no elements shares memory with nothing, wherever its pointer points.
static void empty_arrays()
{
    mezo_attention_t a = {};
    a.q = P(buffer(0));
    a.out = P(buffer(1));
    a.k = a.v = P(buffer(1) + 64);
    a.docs = static_cast<const int64_t*>(P(buffer(2)));
    a.q_tokens = a.max_q = 4;
    a.q_token = a.o_token = a.q_head = a.o_head = a.k_token = a.k_head = a.v_token = a.v_head = 64;
    a.n_docs = a.heads = a.kv_heads = 1;
    a.dim = 64;
    a.scale = 1.0f;
    CHECK(made(0, 0, [&] { return mezo_attention(&a, nullptr, 0, nullptr); }) == MEZO_OK);
    a.k_tokens = a.max_k = 1;
    CHECK(made(0, 0, [&] { return mezo_attention(&a, nullptr, 0, nullptr); }) == MEZO_EOVERLAP);
}

static void loss()
{
    for (uint64_t vocab : {100ull, 50272ull})
        sweep({from(buffer(0), kAddresses), from(MEZO_F32, kTypes), from(5, kSizes), from(vocab, kSizes), from(vocab, kSizes),
               from(buffer(1), kAddresses), from(buffer(2), kAddresses), from(buffer(3), kAddresses), from(buffer(4), kAddresses)},
              [](const std::vector<uint64_t>& v) {
                  const uint64_t need = mezo_token_loss_workspace(v[2], v[3]);
                  for (uint64_t bytes : {need, need ? need - 1 : need})
                      made(v[8], bytes, [&] {
                          return mezo_token_loss(P(v[0]), uint32_t(v[1]), v[2], v[3], v[4], static_cast<int64_t*>(P(v[5])),
                                                 static_cast<float*>(P(v[6])), static_cast<float*>(P(v[7])), P(v[8]), bytes,
                                                 nullptr);
                      });
              });
}

int main()
{
    quantize();
    const unsigned long a = g_launches;
    products();
    const unsigned long b = g_launches;
    attention();
    empty_arrays();
    const unsigned long c = g_launches;
    loss();
    CHECK(a > 100 && b - a > 100 && c - b > 100 && g_launches - c > 100);  // the sweeps reach the launches
    std::printf("%d checks, %lu launches, %d failed\n", g_checks, g_launches, g_failed);
    return g_failed != 0;
}
