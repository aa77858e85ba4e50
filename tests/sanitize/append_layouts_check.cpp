// append_layouts_check.cpp — TEST INFRASTRUCTURE ONLY: which layouts of a cache the append
// takes, on a machine without a GPU. generation.cpp is built with AddressSanitizer and
// UndefinedBehaviorSanitizer, its launches are replaced, and small layouts of keys and
// values are compared vector by vector: whatever is accepted shares no memory, and the
// layouts that are documented to be accepted are. Exit status 0 when every check passed.
#include <hip/hip_runtime.h>

#include <cstdio>
#include <random>
#include <vector>

#include "attention_launch.hpp"
#include "cache_append_launch.hpp"
#include "mezo.h"
#include "nf4_linear_launch.hpp"

extern "C" const char* hipGetErrorString(hipError_t) { return "stand-in"; }

namespace mezo {
hipError_t launch_cache_append(const AppendArgs&, hipStream_t) { return hipSuccess; }
hipError_t launch_paged_attention(const PagedArgs&, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_nf4_linear(const NF4LinearArgs&, hipStream_t) { return hipErrorInvalidValue; }
}  // namespace mezo

static int g_checks, g_failed;

#define CHECK(cond)                                                                           \
    do {                                                                                      \
        ++g_checks;                                                                           \
        if (!(cond) && ++g_failed <= 20)                                                      \
            std::fprintf(stderr, "%s:%d: check failed: %s\n", __FILE__, __LINE__, #cond);     \
    } while (0)

// Elements from one page, row and head to the next, of bf16 heads of kDim.
struct Layout {
    uint64_t at, page, row, head;
};
constexpr uint64_t kDim = 8, kRows = 8, kBase = 0x7F0000000000ull;

static int append(const Layout& k, const Layout& v, uint64_t pages, uint32_t heads)
{
    mezo_append_t a = {};
    a.k = reinterpret_cast<void*>(kBase + (1ull << 32));
    a.v = reinterpret_cast<void*>(kBase + (2ull << 32));
    a.docs = reinterpret_cast<int64_t*>(kBase + (3ull << 32));
    a.pages = reinterpret_cast<int32_t*>(kBase + (4ull << 32));
    a.k_cache = reinterpret_cast<void*>(k.at);
    a.v_cache = reinterpret_cast<void*>(v.at);
    a.tokens = a.max_q = a.n_entries = a.n_docs = 1;
    a.n_pages = pages;
    a.k_token = a.v_token = heads * kDim;
    a.k_head = a.v_head = kDim;
    a.kc_page = k.page, a.kc_row = k.row, a.kc_head = k.head;
    a.vc_page = v.page, a.vc_row = v.row, a.vc_head = v.head;
    a.kv_heads = heads;
    a.dim = kDim;
    a.page_rows = kRows;
    a.dtype = MEZO_BF16;
    return mezo_cache_append(&a, nullptr);
}

// Whether no two vectors of the two arrays meet.
static bool disjoint(const Layout& k, const Layout& v, uint64_t pages, uint32_t heads)
{
    // (all offsets are whole vectors' or half ones': a map of bytes in steps of 16)
    std::vector<uint8_t> used;
    const uint64_t first = k.at < v.at ? k.at : v.at;
    for (const Layout* l : {&k, &v})
        for (uint64_t p = 0; p < pages; ++p)
            for (uint64_t r = 0; r < kRows; ++r)
                for (uint64_t h = 0; h < heads; ++h) {
                    const uint64_t at = (l->at - first + (p * l->page + r * l->row + h * l->head) * 2) / 16;
                    if (used.size() <= at) used.resize(at + 1);
                    if (used[at]++) return false;
                }
    return true;
}

int main()
{
    const uint64_t w = kDim, b = 2;  // a vector, and its bytes an element
    // [pages, rows, 2, heads, dim], either one first, with room in each row or behind each page
    for (uint32_t heads : {1u, 2u, 5u})
        for (uint64_t pages : {1ull, 4ull})
            for (uint64_t room : {0ull, 1ull, 3ull})
                for (uint64_t behind : {0ull, 1ull, 2ull}) {
                    const uint64_t row = (2 * heads + room) * w, page = (kRows + behind) * row;
                    const Layout one = {kBase, page, row, w}, other = {kBase + heads * w * b, page, row, w};
                    CHECK(disjoint(one, other, pages, heads));
                    CHECK(append(one, other, pages, heads) == MEZO_OK && append(other, one, pages, heads) == MEZO_OK);
                    // [pages, 2, rows, heads, dim], [2, pages, ...]
                    const Layout half = {kBase + kRows * row * b, 2 * page, row, w}, whole = {kBase, 2 * page, row, w};
                    CHECK(append(whole, half, pages, heads) == MEZO_OK && append(half, whole, pages, heads) == MEZO_OK);
                    const Layout far = {kBase + pages * page * b, page, row, w};
                    CHECK(append(one, far, pages, heads) == MEZO_OK && append(far, one, pages, heads) == MEZO_OK);
                    // a row that ends in the other's
                    if (heads > 1) {
                        const Layout into = {kBase + (heads - 1) * w * b, page, row, w};
                        CHECK(append(one, into, pages, heads) == MEZO_EOVERLAP && append(into, one, pages, heads) == MEZO_EOVERLAP);
                    }
                }
    // anything else: what is accepted is apart
    std::mt19937 random(1);
    auto pick = [&](uint64_t most) { return random() % (most + 1); };
    int accepted = 0, meeting = 0;
    for (int i = 0; i < 400000; ++i) {
        const uint32_t heads = uint32_t(1 + pick(3));
        const uint64_t pages = pick(3);
        Layout l[2];
        l[0] = {kBase + 16 * pick(40), w * pick(60), w * pick(8), w * pick(8)};
        l[1] = pick(1) ? l[0] : Layout{0, w * pick(60), w * pick(8), w * pick(8)};
        if (!pick(2)) l[1].row = l[0].row;
        if (!pick(2)) l[1].page = l[0].page;
        l[1].at = kBase + 16 * pick(40);
        const bool apart = disjoint(l[0], l[1], pages, heads);
        const int rc = append(l[0], l[1], pages, heads);
        CHECK(rc == MEZO_OK || rc == MEZO_EOVERLAP);
        accepted += rc == MEZO_OK && pages;
        meeting += !apart;
        if (rc == MEZO_OK) CHECK(apart);
    }
    CHECK(accepted > 1000 && meeting > 1000);
    std::printf("%d checks, %d accepted, %d failed\n", g_checks, accepted, g_failed);
    return g_failed != 0;
}
