// plans.hpp — the layout of 8-bit storage, and how the forward pass's operators are
// cut into workgroups: arithmetic of the host alone, which the launches, the argument
// checks and host tests share.
#pragma once

#include <stdint.h>

namespace mezo {

// ---- 8-bit storage and its product ---------------------------------------------

// Elements of a row that share a scale, and the bytes of a stored row.
constexpr uint64_t kF8Block = 128;
constexpr uint64_t f8_blocks(uint64_t cols) { return (cols + kF8Block - 1) / kF8Block; }
constexpr uint64_t f8_code_stride(uint64_t cols) { return f8_blocks(cols) * kF8Block; }
constexpr uint64_t f8_scale_stride(uint64_t cols) { return (f8_blocks(cols) + 3) / 4 * 4; }

// The kernels, and how a product is cut into them: its tile, and the workgroups that
// share out k.
enum F8Tile { kThin, k64x64, k128x128, k256x256 };
constexpr uint32_t kThinRows = 64;  // weights' rows of a workgroup of kThin

struct F8Cut {
    F8Tile tile;
    uint32_t splits;
};

constexpr uint64_t tiles_of(uint64_t m, uint64_t n, uint64_t bm, uint64_t bn)
{
    return ((m + bm - 1) / bm) * ((n + bn - 1) / bn);
}

inline F8Cut cut_product(uint64_t m, uint64_t n, uint64_t k, bool wide)
{
    if (m <= 64) {
        // Split where that brings two workgroups to a CU that would have none or one, each with
        // 8 blocks at least: the join costs a launch (one token: 4096 x 16384 weights 20.7 us
        // in 256 workgroups, 18.5 in 512; 12345 x 5000 in 193 14.2, in 386 16.8).
        const uint64_t tiles = tiles_of(m, n, 64, kThinRows);
        const uint64_t want = tiles >= 160 ? 1 : 512 / tiles, most = f8_blocks(k) / 8;
        const uint64_t splits = want < most ? want : most;
        return {kThin, uint32_t(splits < 1 ? 1 : (splits > 16 ? 16 : splits))};
    }
    // Rounds of workgroups over the 256 CUs, one of 256 x 256 or two of 128 x 128 each: a
    // round of the former takes 1.8 times one of the latter (60 and 33 us at k = 4096), for
    // twice the work. 3000 x 5000 x 4096: 56 us in 240 large tiles, 61 in 960 small ones;
    // 300 x 50272 x 768: 36 in 394 large ones, 27 in 1179.
    const uint64_t t128 = tiles_of(m, n, 128, 128);
    const uint64_t rounds128 = (t128 + 511) / 512, rounds256 = (tiles_of(m, n, 256, 256) + 255) / 256;
    if (!wide && 9 * rounds256 <= 5 * rounds128) return {k256x256, 1};
    if (t128 >= 200) return {k128x128, 1};
    // Too few of those for the CUs: smaller tiles, and k split where it is long, in parts of
    // 16 blocks at least (128 x 4096 x 16384 to bf16: 79 us in 32 tiles of 128, 60 in 128 of
    // 64, 24 with k in four; 1024 x 768 x 3000: 18, 9, 13 with k in two).
    const uint64_t want = 512 / tiles_of(m, n, 64, 64), most = f8_blocks(k) / 16;
    const uint64_t splits = want < most ? want : most;
    return {k64x64, uint32_t(splits < 1 ? 1 : (splits > 16 ? 16 : splits))};
}

// Bytes of a split product's partial sums (0: not split); wide: to fp32.
inline uint64_t f8_matmul_workspace(uint64_t m, uint64_t n, uint64_t k, bool wide)
{
    const F8Cut c = cut_product(m, n, k, wide);
    return c.splits > 1 ? c.splits * m * ((n + 3) / 4 * 16) : 0;
}

// ---- attention -------------------------------------------------------------------

// How a call is cut: the most workgroups that share a document's keys, the keys of
// each, and the bytes of `partial`.
struct AttentionPlan {
    uint32_t splits, chunk;
    uint64_t workspace;
};
// Few rows: the waves of a workgroup share out the keys.
inline bool by_keys(uint64_t rows) { return rows <= 32; }

inline AttentionPlan plan_attention(uint32_t docs, uint32_t heads, uint32_t kv_heads, uint32_t dim, uint32_t max_q,
                                    uint32_t max_k)
{
    const uint64_t rows = uint64_t(max_q) * (heads / kv_heads);
    const uint64_t tiles = by_keys(rows) ? 1 : (rows + 127) / 128;
    const uint64_t groups = uint64_t(docs) * kv_heads * tiles;
    // Split where the groups alone leave CUs idle, into chunks of keys rather than parts
    // of a document: documents of any length then give equal work. A few rows leave little
    // behind for the join, and eight workgroups a CU keep the memory busy. Of many rows the
    // join costs as much as 256 keys do, so they are split where there are fewer groups
    // than CUs, to two a CU. Against the rule of few rows for both, bf16: 8 documents of 512
    // tokens, 16 heads of 64, 52 -> 16 us; 2048 tokens, 32 heads of 128, 102 -> 62; 64 tokens
    // over 16000 keys, 32 heads of 128, 91 -> 57. fp32: the same three 90 -> 49, 339 -> 260,
    // 292 -> 244, 4 documents of 1000 tokens, 16 heads of 128, 220 -> 147; single documents
    // of few heads lose (2048 tokens, 12 heads of 64, 92 -> 102; 3000, 4 heads, 67 -> 78).
    AttentionPlan p = {1, 64, 0};
    const uint64_t wanted = by_keys(rows) ? 2048 : 512;
    if (groups >= wanted / 2 || max_k <= 256) return p;
    uint64_t chunk = (max_k * groups / wanted + 63) / 64 * 64;
    chunk = chunk < 256 ? 256 : chunk;
    while ((max_k + chunk - 1) / chunk > 64) chunk += 64;
    const uint64_t splits = (max_k + chunk - 1) / chunk, kept = splits * docs * max_q * heads;
    if (splits == 1) return p;
    p.splits = uint32_t(splits);
    p.chunk = uint32_t(chunk);
    p.workspace = (kept + 1) / 2 * 16 + kept * dim * 4;
    return p;
}

// ---- the token loss ----------------------------------------------------------------

// One or two rows of together so many logits at most: one workgroup. A row of 50272 fp32
// logits takes 6.8 us in it, 7.5 in 12 workgroups and a second launch, which costs the
// host 4 us more.
constexpr uint64_t kOneGroup = 65536;
constexpr bool one_group(uint64_t rows, uint64_t vocab) { return rows <= 2 && vocab <= kOneGroup / rows; }

// Rows shorter than this take a wave each.
constexpr uint64_t kWaveRow = 2048;

// How many workgroups share a row (1: the row's own workgroup writes its loss).
inline uint32_t loss_parts(uint64_t rows, uint64_t vocab)
{
    if (one_group(rows, vocab)) return 1;
    // enough workgroups that the last round over the CUs is a small part of all, each with a
    // few KB at least
    const uint64_t want = (2048 + rows - 1) / rows, most = vocab / 4096;
    const uint64_t parts = want < most ? want : most;
    return vocab < kWaveRow || parts < 1 ? 1u : uint32_t(parts < 16 ? parts : 16);
}

}  // namespace mezo
