// nf4_linear_launch.hpp — how a product with 4-bit weights is cut, and the interface
// between the C-ABI host code (generation.cpp) and its kernels (nf4_linear.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "plans.hpp"

namespace mezo {

// Rows of expanded weights and of activations laid out for the matrix instructions: whole
// stages of 64 columns, zeros after the last.
constexpr uint64_t nf4_columns(uint64_t k) { return (k + 63) / 64 * 64; }

// fp32 activations (and the weights beside them) are three bf16 each.
constexpr uint64_t nf4_planes(bool wide_x) { return wide_x ? 3 : 1; }

// A product's cut: its tile, the workgroups that share out k, and the weights' rows that are
// expanded at a time.
struct NF4Cut {
    F8Tile tile;  // kThin: weights read as they are, thin_rows rows of them a workgroup (0: in any order)
    uint32_t splits;
    uint64_t slab;
    uint32_t thin_rows;
};

// Bytes of expanded weights at a time: what the last-level cache holds.
constexpr uint64_t kNF4SlabBytes = 1ull << 28;

// The most activations for which weights whose rows do not end with a block are decoded where they
// are used (64 x 16384 x 4100 bf16 53 us, expanded 72; past 64 they would be decoded twice).
constexpr uint64_t kNF4Ragged = 64;

inline NF4Cut cut_nf4(uint64_t m, uint64_t n, uint64_t k, bool wide_x)
{
    const uint64_t row = nf4_columns(k) * 2 * nf4_planes(wide_x);
    uint64_t slab = kNF4SlabBytes / row / 256 * 256;
    if (slab < 256) slab = 256;
    if (slab > n) slab = n;
    // Up to so many rows the expanding does not pay: 256 x 16384 x 4096 bf16 75 us both ways, 128 41
    // and 64; fp32, where a slice of 16 rows takes as long as its products, 1024 x 4096 x 4096 275
    // and 278, 256 78 and 129.
    if (m <= (wide_x ? 1024 : 256) && k % 64 == 0) {
        // A workgroup a CU. One to four activations and few weights: 16 rows each and all of k
        // (4096 x 4096 8.4 us, 64 rows and k in four 10). Many rows: 128 each where that saves
        // rounds over the CUs; one takes 1.6 times as long as with 64 (1 x 50272 x 4096 36.6 us
        // in two rounds of 128, 43.7 in four of 64; 1 x 16384 x 4096 18.1 and 12.6 in one).
        const uint64_t rounds64 = ((n + 63) / 64 + 255) / 256, rounds128 = ((n + 127) / 128 + 255) / 256;
        // (and past 2^27 rows, of which 64 a workgroup are more lanes than a grid holds)
        const bool wide_group = (wide_x ? m > 16 : m <= 32 && 8 * rounds128 < 5 * rounds64) || n > 1ull << 27;
        const uint64_t rows = m <= 4 && n <= 4096 ? 16 : (wide_group ? 128 : 64);
        // k split where the rows leave CUs without work, in parts of 16 blocks at least
        const uint64_t groups = (n + rows - 1) / rows * (wide_x ? (m + 15) / 16 : (m + 63) / 64);
        const uint64_t want = groups >= 160 ? 1 : 256 / groups, most = k / 64 / 16;
        const uint64_t splits = want < most ? want : most;
        return {kThin, uint32_t(splits < 1 ? 1 : (splits > 16 ? 16 : splits)), 0, uint32_t(rows)};
    }
    // Rows that do not end with a block: 16 or 32 of them a workgroup, k split as above.
    if (m <= kNF4Ragged && k % 64 && n <= 1ull << 26) {
        const uint64_t groups = (n + 15) / 16 * ((m + 63) / 64), want = groups >= 160 ? 1 : 256 / groups,
                       most = nf4_columns(k) / 64 / 16, splits = want < most ? want : most;
        return {kThin, uint32_t(splits < 1 ? 1 : (splits > 16 ? 16 : splits)), 0, 0};
    }
    // The tile and the split of k that take the least time by what was measured: a stage of 64
    // columns takes a round of workgroups over the CUs 1640 ns with one tile of 256 x 256 a CU,
    // 900 with two of 128 x 128, 750 with four of 64 x 64; a
    // split's sums go out and back at 4 TB/s, and their join is a launch of 4 us.
    struct Kind {
        F8Tile tile;
        uint64_t size, slots, stage;
    };
    constexpr Kind kinds[3] = {{k256x256, 256, 256, 1640}, {k128x128, 128, 512, 900}, {k64x64, 64, 1024, 750}};
    const uint64_t stages = nf4_columns(k) / 64 * (wide_x ? 6 : 1);
    NF4Cut best = {k64x64, 1, slab, 0};
    uint64_t least = ~0ull;
    for (const Kind& t : kinds)
        for (uint64_t splits = 1; splits <= 16 && (splits == 1 || stages / splits >= 8); ++splits) {
            const uint64_t rounds = (tiles_of(m, slab, t.size, t.size) * splits + t.slots - 1) / t.slots;
            const uint64_t join = splits == 1 ? 0 : 4000 + splits * m * slab / 500;
            const uint64_t time = rounds * ((stages + splits - 1) / splits) * t.stage + join;
            if (time < least) {
                least = time;
                best.tile = t.tile;
                best.splits = uint32_t(splits);
            }
        }
    return best;
}

// The parts of a call's workspace, from its start: activations laid out, weights expanded,
// partial sums; all multiples of 16 bytes.
struct NF4Space {
    uint64_t weights, partial, bytes;
};

inline NF4Space nf4_space(uint64_t m, uint64_t n, uint64_t k, bool wide_x)
{
    const NF4Cut c = cut_nf4(m, n, k, wide_x);
    const uint64_t row = nf4_columns(k) * 2 * nf4_planes(wide_x);
    NF4Space s;
    // (few rows are laid out in their own type where they do not lie on 16 bytes)
    s.weights = c.tile == kThin && c.thin_rows ? m * k * (wide_x ? 4 : 2) : m * row;
    s.partial = s.weights + c.slab * row;
    s.bytes = s.partial + (c.splits > 1 ? c.splits * m * (((c.tile == kThin ? n : c.slab) + 3) / 4 * 16) : 0);
    return s;
}

struct NF4LinearArgs {
    uint64_t x, ldx;    // activations [m, k], elements from one row to the next
    uint64_t codes, absmax;
    uint64_t c, ldc;    // [m, n]
    uint64_t workspace;
    uint64_t m, n, k;
    uint32_t x_dtype, c_dtype;
};

hipError_t launch_nf4_linear(const NF4LinearArgs& args, hipStream_t stream);

}  // namespace mezo
