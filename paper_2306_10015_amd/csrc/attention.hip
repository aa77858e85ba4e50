// attention.hip — attention of a packed batch of documents, the middle of a
// decoder layer's forward pass. For query i of a document with nq queries and nk
// keys (its queries are the last of its tokens, pos = i + nk - nq), per head:
//   s_j = scale q_i . k_j,  s_j = cap tanh(s_j / cap) if capped,
//   s_j = s_j - slope |pos - j| if biased,
//   out = sum_j softmax_j(s) v_j over the visible keys j < limit,
// limit = nk, or max(pos + 1, prefix) if causal: every mask this serves (documents,
// causal, a prefix seen both ways, their mixtures) is "the first so many keys of the
// own document", one number a row. A row that sees nothing gives 0 and lse -inf.
//
// One pass over the keys with a running reference m and l = sum 2^(s - m) (scores
// in units of log 2). m need not be the maximum, any reference cancels: it moves
// only when a row's maximum has passed it by kSlack, so that the accumulator is
// seldom rescaled; a term is then at most 2^kSlack.
//
// Scores are computed transposed, keys x queries: a lane's 16 results of a 32x32
// tile are then 16 keys of one query, the row's statistics are a lane's own (and
// its partner's, 32 lanes away), and the probabilities are already where the second
// product wants its operand, with the keys in an order that its other operand, the
// values, follows: no exchange between lanes. The values' operand needs the columns
// of the tile: ds_read_b64_tr_b16 transposes 4 keys x 16 columns at a time (bf16);
// fp32 reads them one by one.
// All sums are fp32, on v_mfma_f32_32x32x16_bf16. bf16: probabilities are rounded to
// bf16 for the product with the values (as large an error as the output's own
// rounding), l sums them unrounded. fp32: every operand is split into three bf16, and
// six of the nine products are summed, all above 2^-24 of the whole: 192 cycles for 16
// columns where v_mfma_f32_32x32x2_f32 takes 512. The split is exact down to 2^-110; of what
// is smaller it loses up to 2^-134 (bf16's numbers end at 2^-133). In a key that is 2^-24 of
// a score where the query is of 2^110; in the values it shows in a result below kSmallest,
// see below. A number so large that its first part is infinite gives NaN, see below.
//
// The rows of a tile are (query, head) pairs of the heads that share a key/value
// head, so these read it once. Two shapes of workgroup:
//   rows: each wave has 32 rows of its own and all share stages of 64 keys (fp32: 32);
//   keys: at most 32 rows (single tokens): all waves have the same rows, each takes
//         every kWaves-th stage of 32 keys through LDS of its own, without barriers,
//         and they join at the end. One buffer for K and one for V: K of the next
//         stage loads under the softmax and the product with V, V under the scores,
//         and eight waves a CU keep the memory busy.
// Where that gives too few workgroups for the GPU, a document's keys are split over
// several, which leave (m, l, accumulator) and a second kernel joins them.
//
// A masked key takes no part whatever its value: its probability is 0, but 0 times
// an infinite or NaN value is not. So a row whose result is not finite is computed
// once more, from its visible keys alone (careful_row). Finite inputs get there only
// where their scores or a sum of theirs leave fp32's range, or where a result in fp32
// is so small (but not 0) that the values' split may show in it: multiplying each value
// by 2^16 before the split would do as well, for 2 to 4% of the time of all calls.
#include <type_traits>

#include "attention_launch.hpp"
#include "lds_dma.hpp"
#include "records.hpp"
#include "stream_io.hpp"

namespace mezo {

typedef float v16f_t __attribute__((ext_vector_type(16)));
typedef float v4f_t __attribute__((ext_vector_type(4)));
typedef __bf16 v8bf_t __attribute__((ext_vector_type(8)));
typedef __bf16 v4bf_t __attribute__((ext_vector_type(4)));
typedef short v4s_t __attribute__((ext_vector_type(4)));
typedef float v2f_t __attribute__((ext_vector_type(2)));

constexpr float kLog2e = 1.44269504088896341f;
constexpr float kLn2 = 0.693147180559945309f;
constexpr float kLowest = -3.0e38f;  // a reference below every score that counts
constexpr float kSlack = 8.0f;
constexpr float kSmallest = 0x1p-110f;  // of fp32 results
constexpr uint64_t kMostTokens = (1u << 31) - 256;  // of a document

struct Document {
    uint64_t q_first, k_first;
    int nq, nk, prefix;
};

// A value that is the same for all lanes, in scalar registers.
__device__ __forceinline__ int64_t uniform(int64_t x)
{
    const uint32_t lo = __builtin_amdgcn_readfirstlane(uint32_t(uint64_t(x)));
    const uint32_t hi = __builtin_amdgcn_readfirstlane(uint32_t(uint64_t(x) >> 32));
    return int64_t(uint64_t(hi) << 32 | lo);
}

// A document's row of the table, cut to the arrays it points into: no table makes
// a kernel leave them.
__device__ __forceinline__ Document read_document(const AttentionArgs& a, uint32_t d)
{
    const MEZO_GLOBAL int64_t* t = reinterpret_cast<const MEZO_GLOBAL int64_t*>(a.table) + uint64_t(d) * 5;
    auto within = [&](int64_t y, uint64_t top) {
        const int64_t x = uniform(y);
        return x < 0 ? 0 : (uint64_t(x) > top ? top : uint64_t(x));
    };
    auto count = [](uint64_t left) { return left < kMostTokens ? left : kMostTokens; };
    Document r;
    r.q_first = within(t[0], a.q_tokens);
    r.nq = int(within(t[1], count(a.q_tokens - r.q_first)));
    r.k_first = within(t[2], a.k_tokens);
    r.nk = int(within(t[3], count(a.k_tokens - r.k_first)));
    r.prefix = int(within(t[4], uint64_t(r.nk)));
    return r;
}

// How many of its document's keys query i sees.
__device__ __forceinline__ int visible(const AttentionArgs& a, const Document& d, int i)
{
    const int pos = d.nk - d.nq + i;
    if (!a.causal) return d.nk;
    return pos + 1 > d.prefix ? pos + 1 : d.prefix;  // pos < nk, prefix >= 0
}

// The score function's constants, for scores in units of log 2.
struct Score {
    float c;      // scale log2 e
    float k, w;   // capped: x = w - 2 w / (1 + 2^(k s)), k = 2 scale log2 e / cap, w = cap log2 e
    float cap, scale, share;  // share = scale / cap
    bool capped;
};

__device__ __forceinline__ Score score_of(const AttentionArgs& a)
{
    Score s;
    s.scale = a.scale;
    s.cap = a.softcap;
    s.capped = a.softcap > 0.0f;
    s.c = a.scale * kLog2e;
    // (finite, so that a score of 0 stays 0 under the smallest caps)
    constexpr float kLargest = 1e38f;
    s.share = s.capped ? fminf(fmaxf(a.scale / a.softcap, -kLargest), kLargest) : 0.0f;
    s.k = 2.0f * kLog2e * s.share;
    s.w = a.softcap * kLog2e;
    return s;
}

// The cap by two transcendentals: a capped score before the bias is w - 2 w r. Its error is
// 2^-23 cap, since 1 + 2^(k x) keeps no more of x.
__device__ __forceinline__ float cap_share(const Score& s, float x)
{
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x * s.k));
}

// A capped score before the bias, in units of log 2. bf16 takes the short form as long as its
// error does not show in a result of bf16, fp32 the library's tanh as long as neither w nor
// x scale / cap can leave the range in which they keep their digits.
template <bool kF>
constexpr float kMostCap = kF ? 0x1p64f : 256.0f;

template <bool kF>
__device__ __forceinline__ float capped(const Score& s, float x)
{
    if constexpr (kF) return s.w * tanhf(x * s.scale / s.cap);
    return __builtin_fmaf(cap_share(s, x), -2.0f * s.w, s.w);
}

// The same in its own units, of any cap, to 2^-21 of the score itself: tanh y by its series
// below a quarter, (1 - t) / (1 + t) with t = exp(-2 |y|) above.
__device__ __forceinline__ float capped_any(const Score& s, float x)
{
    const float y = x * s.share, y2 = y * y, t = __builtin_amdgcn_exp2f(fabsf(y) * (-2.0f * kLog2e));
    float series = __builtin_fmaf(y2, 62.0f / 2835, -17.0f / 315);
    series = __builtin_fmaf(y2, series, 2.0f / 15);
    series = __builtin_fmaf(y2, series, -1.0f / 3);
    series = __builtin_fmaf(y2, series, 1.0f);
    const float above = copysignf((1.0f - t) * __builtin_amdgcn_rcpf(1.0f + t), y);
    return fabsf(y) < 0.25f ? x * s.scale * series : s.cap * above;
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// The larger of this lane's and its partner's value, 32 lanes away, and their sum.
__device__ __forceinline__ float max_halves(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

__device__ __forceinline__ float sum_halves(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

template <bool kF>
__device__ __forceinline__ float load_element(uint64_t addr, uint32_t i)
{
    if constexpr (kF) return reinterpret_cast<const gfloat_t*>(addr)[i];
    return __uint_as_float(uint32_t(reinterpret_cast<const gu16_t*>(addr)[i]) << 16);
}

template <bool kF>
__device__ __forceinline__ void store_element(uint64_t addr, uint32_t i, float x)
{
    if constexpr (kF)
        reinterpret_cast<gfloat_t*>(addr)[i] = x;
    else
        reinterpret_cast<MEZO_GLOBAL __bf16*>(addr)[i] = static_cast<__bf16>(x);
}

// Where row (i, h) of a document keeps what a split of its keys found: (m, l), m in the
// scores' own units and -inf where no key was seen, and the accumulator, dim floats; with
// -l in the place of l, the accumulator is divided by l.
struct PartialRow {
    uint64_t stats, acc;
};
__device__ __forceinline__ PartialRow partial_row(const AttentionArgs& a, uint32_t split, uint32_t doc, int i,
                                                  uint32_t h)
{
    const uint64_t rows = uint64_t(a.docs) * a.max_q * a.heads;
    const uint64_t row = (uint64_t(doc) * a.max_q + uint64_t(i)) * a.heads + h;
    const uint64_t at = split * rows + row;
    return {a.partial + at * 8, a.partial + (a.splits * rows + 1) / 2 * 16 + at * a.dim * 4};
}

// lse = m + ln l (-inf where l is 0)
__device__ __forceinline__ void store_lse(const AttentionArgs& a, uint64_t token, uint32_t h, float m, float ln_l)
{
    if (a.lse) reinterpret_cast<gfloat_t*>(a.lse)[token * a.heads + h] = ln_l == -__builtin_inff() ? ln_l : m + ln_l;
}

// A row by its visible keys alone, k0 <= j < k1, 64 at a time; the whole wave works on it.
// A lane has a key's score, then columns l and l + 64 of the accumulator. Where the other
// kernels' arithmetic leaves fp32's range this one's does not: scores are in their own units
// (in those of log 2 the largest floats are too large), and the accumulator is the mean of
// the values so far, never more than the largest of them. A key that is NaN to the row ends
// it: nothing that follows changes its result.
template <bool kF>
__device__ __forceinline__ void careful_row(const AttentionArgs& a, const Document& d, uint32_t doc, uint32_t kvh,
                                         uint32_t split, int i, uint32_t h, int k0, int k1)
{
    constexpr uint32_t kPer = kF ? 4 : 8;  // elements of 16 bytes
    const Score sc = score_of(a);
    const uint32_t l = threadIdx.x & 63u;
    const uint64_t q = a.q + (d.q_first + uint64_t(i)) * a.q_token + h * a.q_head;
    const float slope = a.slopes ? a.slopes[h] : 0.0f;
    float q2[2], acc[2] = {0.0f, 0.0f}, m = -__builtin_inff(), sum = 0.0f;
    for (uint32_t c = 0; c < 2; ++c) q2[c] = l + 64 * c < a.dim ? load_element<kF>(q, l + 64 * c) : 0.0f;
    for (int j0 = k0; j0 < k1; j0 += 64) {
        const int n = k1 - j0 < 64 ? k1 - j0 : 64, j = j0 + (int(l) < n ? int(l) : n - 1);
        const uint64_t k = a.k + (d.k_first + uint64_t(j)) * a.k_token + kvh * a.k_head;
        float s = 0.0f;
        for (uint32_t c0 = 0; c0 < a.dim; c0 += 4 * kPer) {
            u32x4_t w[4];
#pragma unroll
            for (uint32_t u = 0; u < 4; ++u) {
                const uint32_t c = c0 + u * kPer;
                w[u] = u32x4_t{0, 0, 0, 0};
                if (c < a.dim) w[u] = *reinterpret_cast<const gu32x4_t*>(k + c * (16 / kPer));
            }
            const uint32_t part = __float_as_uint(c0 < 64 ? q2[0] : q2[1]);
#pragma unroll
            for (uint32_t e = 0; e < 4 * kPer; ++e) {
                const u32x4_t x = w[e / kPer];
                const uint32_t bits = kF ? x[e % 4] : (e & 1 ? x[e % 8 / 2] & 0xFFFF0000u : x[e % 8 / 2] << 16);
                s = __builtin_fmaf(__uint_as_float(__builtin_amdgcn_readlane(part, (c0 + e) & 63u)),
                                   __uint_as_float(bits), s);
            }
        }
        if (sc.capped)
            s = sc.cap <= kMostCap<true> ? sc.cap * tanhf(s * sc.scale / sc.cap) : capped_any(sc, s);
        else
            s *= sc.scale;
        if (a.slopes) s -= slope * fabsf(float(d.nk - d.nq + i - j));
        if (int(l) >= n) s = -__builtin_inff();
        float top = s;
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off));
        top = fmaxf(m, top);
        const float ref = top == -__builtin_inff() ? 0.0f : top;  // (all scores so far are -inf)
        float old = exp2_fast((m - ref) * kLog2e), p = exp2_fast((s - ref) * kLog2e);
        float all = p;
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) all += __shfl_xor(all, off);
        m = top;
        old *= sum;
        sum = old + all;
        if (__any(sum != sum)) {  // (of all lanes)
            acc[0] = acc[1] = __builtin_nanf("");
            break;
        }
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
        p *= inv;
        for (uint32_t c = 0; c < 2; ++c) acc[c] *= old * inv;
        const uint64_t v = a.v + (d.k_first + uint64_t(j0)) * a.v_token + kvh * a.v_head;
        constexpr int kAhead = 8;  // loads in flight
        for (int g = 0; g < n; g += kAhead) {
            float x[kAhead][2];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const uint64_t at = v + uint64_t(g + u < n ? g + u : n - 1) * a.v_token;
#pragma unroll
                for (uint32_t c = 0; c < 2; ++c)
                    x[u][c] = l + 64 * c < a.dim ? load_element<kF>(at, l + 64 * c) : 0.0f;
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                if (g + u >= n) break;
                const float pj = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(p), g + u));
#pragma unroll
                for (uint32_t c = 0; c < 2; ++c) acc[c] = __builtin_fmaf(pj, x[u][c], acc[c]);
            }
        }
    }
    const uint64_t token = d.q_first + uint64_t(i);
    if (a.splits > 1) {
        const PartialRow p = partial_row(a, split, doc, i, h);
        if (l == 0) *reinterpret_cast<MEZO_GLOBAL v2f_t*>(p.stats) = v2f_t{m, -sum};
        for (uint32_t c = 0; c < 2; ++c)
            if (l + 64 * c < a.dim) reinterpret_cast<gfloat_t*>(p.acc)[l + 64 * c] = acc[c];
        return;
    }
    for (uint32_t c = 0; c < 2; ++c)
        if (l + 64 * c < a.dim) store_element<kF>(a.out + token * a.o_token + h * a.o_head, l + 64 * c, acc[c]);
    if (l == 0) store_lse(a, token, h, m, logf(sum));
}

// A float as the sum of three bf16: its 24 bits in 8 and 8 and 8.
struct Split {
    v8bf_t h, m, l;
};

__device__ __forceinline__ Split split(const float (&x)[8])
{
    Split s;
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) {
        s.h[i] = static_cast<__bf16>(x[i]);
        const float r = x[i] - static_cast<float>(s.h[i]);
        s.m[i] = static_cast<__bf16>(r);
        s.l[i] = static_cast<__bf16>(r - static_cast<float>(s.m[i]));
    }
    return s;
}

// c + a b of split operands, but for the terms below 2^-24 of the largest.
__device__ __forceinline__ v16f_t product(const Split& a, const Split& b, v16f_t c)
{
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.m, b.m, c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.l, b.h, c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.h, b.l, c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.m, b.h, c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.h, b.m, c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.h, b.h, c, 0, 0, 0);
}

// The tile of one type and padded head size: how it lies in LDS and what the
// matrix instructions take from it.
template <bool kF, uint32_t kD>
struct Tile {
    static constexpr uint32_t kElement = kF ? 4 : 2;
    static constexpr uint32_t kRow = kD * kElement;     // bytes of a key's row
    static constexpr uint32_t kChunks = kRow / 16;
    static constexpr uint32_t kLoadRows = 1024 / kRow;  // rows of one load of a wave
    static constexpr uint32_t kQ = kD / 16;             // operands of a row: 16 columns each
    using Operand = std::conditional_t<kF, Split, v8bf_t>;

    // The order of a row's chunks in LDS, such that the lanes that read together read
    // different banks (64 of 4 bytes): of K 16 rows at one chunk, of V (bf16) 4 rows at 64
    // bytes. Both patterns return every kPeriod rows (for fp32, which reads less in the time
    // of its matrix instructions, as often as a wave's loads do).
    static constexpr uint32_t kPeriod = kF ? 8 : 16;
    static __device__ __forceinline__ uint32_t k_swizzle(uint32_t row)
    {
        return kChunks >= 16 ? row & (kPeriod - 1) : (row >> 1) & 7u;
    }
    static __device__ __forceinline__ uint32_t v_swizzle(uint32_t row)
    {
        if constexpr (kF) return 0;
        return kChunks >= 16 ? (row & 3u) << 2 : (row & 2u) << 1;
    }

    // Columns 16 c + 8 (l / 32) .. + 7 of the query at `at` that exist (dim of them).
    static __device__ __forceinline__ Operand query(uint64_t at, uint32_t c, uint32_t dim, uint32_t l)
    {
        u32x4_t w[kElement / 2];
#pragma unroll
        for (uint32_t e = 0; e < kElement / 2; ++e) {
            const uint32_t byte = (c * 16 + (l >> 5) * 8) * kElement + e * 16;
            w[e] = u32x4_t{0, 0, 0, 0};
            if (byte < dim * kElement) w[e] = *reinterpret_cast<const gu32x4_t*>(at + byte);
        }
        if constexpr (kF) {
            float x[8];
#pragma unroll
            for (uint32_t e = 0; e < 8; ++e) x[e] = __uint_as_float(w[e / 4][e % 4]);
            return split(x);
        } else {
            return __builtin_bit_cast(v8bf_t, w[0]);
        }
    }

    // s + 32 keys (from row of K's stage) x 32 queries
    static __device__ __forceinline__ v16f_t scores(const uint8_t* k, uint32_t row, const Operand (&q)[kQ], uint32_t l,
                                                    v16f_t s)
    {
        const uint32_t r = row + (l & 31u);
        auto chunk = [&](uint32_t i) { return *reinterpret_cast<const u32x4_t*>(k + r * kRow + ((i ^ k_swizzle(r)) * 16)); };
#pragma unroll
        for (uint32_t c = 0; c < kQ; ++c) {
            if constexpr (kF) {
                const u32x4_t lo = chunk(4 * c + 2 * (l >> 5)), hi = chunk(4 * c + 2 * (l >> 5) + 1);
                float x[8];
#pragma unroll
                for (uint32_t e = 0; e < 4; ++e) {
                    x[e] = __uint_as_float(lo[e]);
                    x[e + 4] = __uint_as_float(hi[e]);
                }
                s = product(split(x), q[c], s);
            } else {
                s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf_t, chunk(2 * c + (l >> 5))), q[c], s,
                                                            0, 0, 0);
            }
        }
        return s;
    }

    // acc += values x probabilities of 32 keys (from row of V's stage)
    static __device__ __forceinline__ void values(const uint8_t* v, uint32_t row, const v16f_t& p, v16f_t (&acc)[kD / 32],
                                                  uint32_t l)
    {
        if constexpr (kF) {
#pragma unroll
            for (uint32_t u = 0; u < 2; ++u) {  // 16 keys an instruction, in the order below
                float pv[8];
#pragma unroll
                for (uint32_t j = 0; j < 8; ++j) pv[j] = p[8 * u + j];
                const Split ps = split(pv);
                const uint32_t r = row + 16 * u + 4 * (l >> 5);
#pragma unroll
                for (uint32_t t = 0; t < kD / 32; ++t) {
                    float x[8];
#pragma unroll
                    for (uint32_t j = 0; j < 8; ++j)
                        x[j] = *reinterpret_cast<const float*>(v + (r + 8 * (j >> 2) + (j & 3)) * kRow +
                                                               (t * 32 + (l & 31u)) * 4);
                    acc[t] = product(split(x), ps, acc[t]);
                }
            }
        } else {
#pragma unroll
            for (uint32_t u = 0; u < 2; ++u) {  // 16 keys an instruction
                v8bf_t pb;
#pragma unroll
                for (uint32_t j = 0; j < 8; ++j) pb[j] = static_cast<__bf16>(p[8 * u + j]);
#pragma unroll
                for (uint32_t t = 0; t < kD / 32; ++t) {
                    // columns t * 32 + l % 32; keys 4 h .. + 3 and 8 + 4 h .. + 3 of the 16, h = l / 32
                    const uint32_t r = row + 16 * u + 4 * (l >> 5) + ((l & 15u) >> 2);
                    const uint32_t chunk = t * 4 + ((l >> 4) & 1u) * 2 + ((l & 3u) >> 1);
                    const uint32_t at = r * kRow + ((chunk ^ v_swizzle(r)) * 16) + (l & 1u) * 8;
                    const uint32_t at8 = (r + 8) * kRow + ((chunk ^ v_swizzle(r + 8)) * 16) + (l & 1u) * 8;
                    typedef __attribute__((address_space(3))) v4s_t lv4s_t;
                    const v4s_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lv4s_t*)(v + at));
                    const v4s_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lv4s_t*)(v + at8));
                    const v8bf_t w = __builtin_bit_cast(
                        v8bf_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
                    acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w, pb, acc[t], 0, 0, 0);
                }
            }
        }
    }
};

// The score functions that have a loop of their own in the bf16 kernels by rows, which
// the vector instructions of the softmax bound (the others use kGeneral: fp32 is bound by
// splitting its operands, calls by keys by memory; but the code of tanh, even where it is not
// run, costs fp32 3%, so uncapped scores have kUncapped there: 16 documents of 50 to 2048
// tokens, 16 heads of 128, 1242 -> 1202 us). Vector instructions a score that counts, over
// calls of 8192 causal tokens: plain 6.0 (heads of 64) to 6.9 (128), biased 9.6, capped 9.8,
// of which two transcendentals take two slots each; kGeneral 15.8 with a cap and a bias, 17.3
// with a cap past the short form.
//  kPlain:  no cap, no bias, scale > 0: the maximum is taken of the products themselves,
//           and one fma scales a product and subtracts the reference.
//  kBiased: no cap, scale > 0. Away from the diagonal the bias is linear in the key: a
//           constant of each of a lane's 16 results, which the products are added to
//           instead of to zero, and one term a stage, which joins the reference.
//  kCapped: no bias, and a cap up to 66 (under larger ones most rows would be followed to
//           their end). No score can pass the cap, so the maximum is taken only until a row's reference is within kHeadroom of it (for nearly all
//           rows that is the first stage), and the cap's last fma subtracts the reference.
//           Terms are then at most 2^kHeadroom; a row whose sums overflow all the same
//           (values above 2^34 after a rise of that much) is one for careful_row.
enum Mode { kGeneral, kPlain, kBiased, kCapped, kUncapped };
constexpr float kHeadroom = 80.0f;

// The waves a SIMD that the registers are kept down for: what LDS allows, and as far as
// nothing spills.
template <bool kF, uint32_t kD, bool kKeys>
constexpr uint32_t waves_per_simd()
{
    if (kF) return kD > 64 ? 1 : 2;
    return kD > 64 || kKeys ? 2 : 3;
}

// kKeys: the workgroup's waves share out the keys; else the rows.
template <bool kF, uint32_t kD, uint32_t kWaves, bool kKeys, Mode kMode>
__global__ void __launch_bounds__(kWaves * 64, (waves_per_simd<kF, kD, kKeys>())) attention_kernel(AttentionArgs a)
{
    using T = Tile<kF, kD>;
    constexpr uint32_t kStage = kKeys || kF ? 32 : 64;  // keys of a stage
    constexpr uint32_t kBytes = kStage * T::kRow;
    constexpr uint32_t kSets = kKeys ? kWaves : 1;
    constexpr uint32_t kBuffers = kKeys ? 1 : 2;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[kSets][kBuffers][2][kBytes];  // [..][0] K, [1] V

    const uint32_t l = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // Workgroups go round the 8 XCDs. By rows, all tiles of a key/value head want one
    // XCD's L2; by keys nothing is read twice, and an XCD that reads one head alone, a few
    // hundred bytes of every token, keeps to a part of its memory channels: the heads
    // turn with the document and the split (170 -> 162 us on 24 tokens over 16384 keys).
    const uint32_t doc = blockIdx.x / a.kv_heads;
    const uint32_t kvh = (blockIdx.x + (kKeys ? doc + blockIdx.z : 0)) % a.kv_heads;
    const Document d = read_document(a, doc);
    const uint32_t rows = (uint32_t(d.nq) < a.max_q ? uint32_t(d.nq) : a.max_q) * a.group;
    // the last tiles see the most keys: first
    constexpr uint32_t kTileRows = kKeys ? 32 : 32 * kWaves;
    const uint32_t tile0 = (gridDim.y - 1 - blockIdx.y) * kTileRows;
    if (tile0 >= rows) return;
    const uint32_t tile1 = tile0 + kTileRows < rows ? tile0 + kTileRows : rows;

    // this lane's row: a (query, head) pair; past the end the last one's again
    const uint32_t first = tile0 + (kKeys ? 0 : wave * 32), row = first + (l & 31u);
    auto query = [&](uint32_t r) { return int((r < tile1 ? r : tile1 - 1) / a.group); };
    const int i = query(row);
    const uint32_t h = kvh * a.group + (row < tile1 ? row : tile1 - 1) % a.group;
    const bool valid = row < tile1;
    const int limit = visible(a, d, i) > 0 ? visible(a, d, i) : 0;
    // the wave's rows see all keys below low and none from high
    auto seen = [&](uint32_t r) {
        const int n = int(__builtin_amdgcn_readfirstlane(uint32_t(visible(a, d, query(r)))));
        return n > 0 ? n : 0;
    };
    // (a wave without a row has nothing to do but to load its part of the stages)
    const int low = seen(first), high = first < tile1 ? seen(first + 31) : 0, last = seen(tile1 - 1);

    // the stages of this split of the workgroup's keys (the last one takes those past max_k)
    const uint32_t stages = (uint32_t(last) + kStage - 1) / kStage, per = a.chunk / kStage;
    const uint32_t s0 = blockIdx.z * per, s1 = blockIdx.z + 1 == a.splits || s0 + per > stages ? stages : s0 + per;
    if (a.splits > 1 && s0 >= stages) return;  // the join does not look for these

    typename T::Operand q[T::kQ];
    {
        const uint64_t at = a.q + (d.q_first + uint64_t(i)) * a.q_token + h * a.q_head;
#pragma unroll
        for (uint32_t c = 0; c < T::kQ; ++c) q[c] = T::query(at, c, a.dim, l);
    }
    const uint64_t kbase = a.k + d.k_first * a.k_token + kvh * a.k_head;
    const uint64_t vbase = a.v + d.k_first * a.v_token + kvh * a.v_head;
    const uint32_t lds0 = lds_offset(&lds[kKeys ? wave : 0][0][0][0]);
    // K or V of stage s into buffer b. A lane's chunk of a row follows the swizzle; columns past a narrower head's end are loaded from its
    // first chunk: for K the query is 0 there, of V they are not stored. Keys past the
    // document's end: the last one again.
    constexpr uint32_t kLoads = kBytes / 1024 / (kKeys ? 1 : kWaves);  // a wave's
    constexpr uint32_t kPatterns = T::kPeriod / T::kLoadRows;
    static_assert(kLoads % kPatterns == 0, "a wave's first load has the first pattern");
    auto column = [&](bool isv, uint32_t r) {
        const uint32_t chunk = (l % T::kChunks) ^ (isv ? T::v_swizzle(r) : T::k_swizzle(r));
        return chunk * 16 < a.dim * T::kElement ? chunk * 16 : 0;
    };
    uint32_t koff[kPatterns], voff[kPatterns];
#pragma unroll
    for (uint32_t n = 0; n < kPatterns; ++n) {
        const uint32_t r = l / T::kChunks;
        koff[n] = r * uint32_t(a.k_token) + column(false, n * T::kLoadRows + r);
        voff[n] = r * uint32_t(a.v_token) + column(true, n * T::kLoadRows + r);
    }
    auto load = [&](auto isv, uint32_t s, uint32_t b) {
        constexpr bool kV = decltype(isv)::value;
        const uint64_t token = kV ? a.v_token : a.k_token;
        const uint64_t base = (kV ? vbase : kbase) + uint64_t(s) * kStage * token;
        const uint32_t to = lds0 + (2 * b + (kV ? 1 : 0)) * kBytes, at0 = kKeys ? 0 : wave * kLoads;
        if ((s + 1) * kStage <= uint32_t(d.nk)) {
            uint64_t at = base + at0 * T::kLoadRows * token;
#pragma unroll
            for (uint32_t n = 0; n < kLoads; ++n, at += T::kLoadRows * token)
                dma_to_lds(at, (kV ? voff : koff)[n % kPatterns], to + (at0 + n) * 1024);
        } else {
            const uint32_t left = uint32_t(d.nk) - s * kStage - 1;
#pragma unroll
            for (uint32_t n = 0; n < kLoads; ++n) {
                const uint32_t r = (at0 + n) * T::kLoadRows + l / T::kChunks;
                dma_to_lds(base, (r < left ? r : left) * uint32_t(token) + column(kV, r), to + (at0 + n) * 1024);
            }
        }
    };
    constexpr std::integral_constant<bool, false> kOfK{};
    constexpr std::integral_constant<bool, true> kOfV{};

    const Score sc = score_of(a);
    const float slope = a.slopes ? a.slopes[h] * kLog2e : 0.0f;
    const int pos = d.nk - d.nq + i;
    v16f_t acc[kD / 32] = {};
    float m = kLowest, sum = 0.0f;
    [[maybe_unused]] bool watch = true;  // (of the wave) the maximum is still taken
    // the positions of the wave's first and last query
    [[maybe_unused]] const int pos0 = d.nk - d.nq + int(__builtin_amdgcn_readfirstlane(uint32_t(query(first))));
    [[maybe_unused]] const int pos1 = d.nk - d.nq + int(__builtin_amdgcn_readfirstlane(uint32_t(query(first + 31))));
    // the bias of a lane's results before the diagonal, but for a term a stage, as a product
    v16f_t bias = {};
    const float per_key = kMode == kBiased ? slope / sc.c : 0.0f;
    if constexpr (kMode == kBiased) {
#pragma unroll
        for (uint32_t e = 0; e < 16; ++e) bias[e] = per_key * float(8 * (e >> 2) + (e & 3));
    }

    const uint32_t step = kKeys ? kWaves : 1, begin = s0 + (kKeys ? wave : 0);
    if (begin < s1) {
        load(kOfK, begin, 0);
        load(kOfV, begin, 0);
    }
    uint32_t b = 0;
    for (uint32_t s = begin; s < s1; s += step, b ^= kBuffers - 1) {
        const bool more = s + step < s1;
        if constexpr (kKeys) {
            dma_wait<kLoads>();  // K of this stage; its V may still come
        } else {
            dma_wait();
            lds_barrier();  // everyone's part of this stage is there, and the other buffer is read
            if (more) {
                load(kOfK, s + step, b ^ 1);
                load(kOfV, s + step, b ^ 1);
            }
        }
        const int k0 = int(s * kStage);
        if constexpr (!kKeys)
            if (k0 >= high) continue;  // (of the wave)
        const uint8_t* kt = lds[kKeys ? wave : 0][b][0];
        const uint8_t* vt = lds[kKeys ? wave : 0][b][1];
        const bool edge = k0 + int(kStage) > low;  // some query of the wave does not see them all
        {
            constexpr uint32_t kT = kStage / 32;
            v16f_t x[kT];
            float off[kT];  // what is still to be added to x[t]
            float top = kLowest;
#pragma unroll
            for (uint32_t t = 0; t < kT; ++t) {
                x[t] = T::scores(kt, t * 32, q, l, bias);
                if constexpr (kKeys) {
                    lds_wait();  // K's buffer is read: the next stage's loads under the rest of this one
                    if (more) load(kOfK, s + step, 0);
                }
            }
#pragma unroll
            for (uint32_t t = 0; t < kT; ++t) {
                // this lane's keys: key, and 8 (e / 4) + e % 4 more
                const int key = k0 + int(t * 32 + 4 * (l >> 5));
                const float from = float(pos - key);
                off[t] = 0.0f;
                if constexpr (kMode == kCapped) {
#pragma unroll
                    for (uint32_t e = 0; e < 16; ++e) x[t][e] = cap_share(sc, x[t][e]);
                }
                if constexpr (kMode == kBiased) {
                    off[t] = -slope * from;
                    if (k0 > pos1) {  // all keys past all queries
                        off[t] = slope * from;
#pragma unroll
                        for (uint32_t e = 0; e < 16; ++e) x[t][e] = __builtin_fmaf(-2.0f, bias[e], x[t][e]);
                    } else if (k0 + int(kStage) > pos0 + 1) {  // some past some
                        off[t] = 0.0f;
#pragma unroll
                        for (uint32_t e = 0; e < 16; ++e)
                            x[t][e] = __builtin_fmaf(-per_key, fabsf(from - float(8 * (e >> 2) + (e & 3))),
                                                     x[t][e] - bias[e]);
                    }
                }
                if constexpr (kMode == kGeneral || kMode == kUncapped) {
                    if (kMode == kGeneral && sc.capped) {
                        if (sc.cap <= kMostCap<kF>) {  // (uniform)
#pragma unroll
                            for (uint32_t e = 0; e < 16; ++e) x[t][e] = capped<kF>(sc, x[t][e]);
                        } else {
#pragma unroll
                            for (uint32_t e = 0; e < 16; ++e) x[t][e] = capped_any(sc, x[t][e]) * kLog2e;
                        }
                    } else {
#pragma unroll
                        for (uint32_t e = 0; e < 16; ++e) x[t][e] *= sc.c;
                    }
                    if (a.slopes) {
#pragma unroll
                        for (uint32_t e = 0; e < 16; ++e)
                            x[t][e] = __builtin_fmaf(-slope, fabsf(from - float(8 * (e >> 2) + (e & 3))), x[t][e]);
                    }
                }
                if (edge) {
                    const int left = limit - key;
#pragma unroll
                    for (uint32_t e = 0; e < 16; ++e)
                        if (int(8 * (e >> 2) + (e & 3)) >= left)
                            x[t][e] = kMode == kCapped ? __builtin_inff() : -__builtin_inff();
                }
                if constexpr (kMode == kCapped) {
                    if (watch) {
                        float least = x[t][0];
#pragma unroll
                        for (uint32_t e = 1; e < 16; ++e) least = fminf(least, x[t][e]);
                        top = fmaxf(top, __builtin_fmaf(least, -2.0f * sc.w, sc.w));
                    }
                } else {
                    float most = x[t][0];
#pragma unroll
                    for (uint32_t e = 1; e < 16; ++e) most = fmaxf(most, x[t][e]);
                    top = fmaxf(top, kMode == kGeneral || kMode == kUncapped ? most : most * sc.c + off[t]);
                }
            }
            if (kMode != kCapped || watch) {
                top = max_halves(top);
                if (__any(top > m + kSlack)) {
                    const float now = fmaxf(m, top), old = exp2_fast(m - now);
                    m = now;
                    sum *= old;
#pragma unroll
                    for (uint32_t t = 0; t < kD / 32; ++t)
#pragma unroll
                        for (uint32_t e = 0; e < 16; ++e) acc[t][e] *= old;
                }
                if constexpr (kMode == kCapped) watch = __any(sc.w - m > kHeadroom);
            }
            [[maybe_unused]] float factor = sc.c;
            if constexpr (kMode == kPlain || kMode == kBiased) {
                // The short form below rounds differently from what the reference was
                // taken of, by 2^-24 of it: not where that is more than 2^-8.
                if (__any(fabsf(m) > 65536.0f || fabsf(off[0]) > 65536.0f)) {
#pragma unroll
                    for (uint32_t t = 0; t < kT; ++t) {
#pragma unroll
                        for (uint32_t e = 0; e < 16; ++e) {
                            x[t][e] = x[t][e] * sc.c + off[t] - m;
                        }
                        off[t] = m;
                    }
                    factor = 1.0f;
                }
            }
#pragma unroll
            for (uint32_t t = 0; t < kT; ++t) {
                const float ref = m - off[t];
                [[maybe_unused]] const float room = sc.w - m;
#pragma unroll
                for (uint32_t e = 0; e < 16; ++e) {
                    if constexpr (kMode == kPlain || kMode == kBiased)
                        x[t][e] = exp2_fast(__builtin_fmaf(x[t][e], factor, -ref));
                    else if constexpr (kMode == kCapped)
                        x[t][e] = exp2_fast(__builtin_fmaf(x[t][e], -2.0f * sc.w, room));
                    else
                        x[t][e] = exp2_fast(x[t][e] - ref);
                    sum += x[t][e];
                }
                if constexpr (kKeys) {
                    if (more)
                        dma_wait<kLoads>();
                    else
                        dma_wait();
                }
                T::values(vt, t * 32, x[t], acc, l);
                if constexpr (kKeys) {
                    lds_wait();
                    if (more) load(kOfV, s + step, 0);
                }
            }
        }
    }
    sum = sum_halves(sum);

    // the tiles of 32 columns that this wave stores: all, or its part of those that the
    // waves' sums over their keys join in, in the order of the waves
    constexpr uint32_t kTiles = kD / 32, kMine = !kKeys ? kTiles : (kTiles > kWaves ? kTiles / kWaves : 1);
    const uint32_t t0 = kKeys ? wave * kMine : 0;
    v16f_t mine[kMine];
    __shared__ uint32_t bad_rows;
    if constexpr (kKeys) {
        __shared__ float stats[kWaves][2][32];
        float* room = reinterpret_cast<float*>(&lds[0][0][0][0]);  // [kWaves][kTiles][16][64]
        static_assert(kWaves * kTiles * 16 * 64 * 4 <= sizeof(lds), "the joined tiles fit");
        if (l < 32) {
            stats[wave][0][l] = m;
            stats[wave][1][l] = sum;
        }
        if (threadIdx.x == 0) bad_rows = 0;
        __syncthreads();
        float now = stats[0][0][l & 31u];
#pragma unroll
        for (uint32_t w = 1; w < kWaves; ++w) now = fmaxf(now, stats[w][0][l & 31u]);
        const float old = exp2_fast(m - now);
#pragma unroll
        for (uint32_t t = 0; t < kTiles; ++t)
#pragma unroll
            for (uint32_t e = 0; e < 16; ++e) room[((wave * kTiles + t) * 16 + e) * 64 + l] = acc[t][e] * old;
        m = now;
        sum = 0.0f;
#pragma unroll
        for (uint32_t w = 0; w < kWaves; ++w) sum += stats[w][1][l & 31u] * exp2_fast(stats[w][0][l & 31u] - now);
        __syncthreads();
#pragma unroll
        for (uint32_t t = 0; t < kMine; ++t)
#pragma unroll
            for (uint32_t e = 0; e < 16; ++e) {
                float x = 0.0f;
                if (t0 + t < kTiles)
#pragma unroll
                    for (uint32_t w = 0; w < kWaves; ++w) x += room[((w * kTiles + t0 + t) * 16 + e) * 64 + l];
                mine[t][e] = x;
            }
    } else {
#pragma unroll
        for (uint32_t t = 0; t < kTiles; ++t) mine[t] = acc[t];
    }

    const bool split = a.splits > 1;
    const float inv = split ? 1.0f : (sum == 0.0f ? 0.0f : 1.0f / sum);
    float zero = 0.0f;  // NaN once a result is not finite
    [[maybe_unused]] float least = __builtin_inff();  // the smallest that is not 0
#pragma unroll
    for (uint32_t t = 0; t < kMine; ++t)
#pragma unroll
        for (uint32_t e = 0; e < 16; ++e) {
            mine[t][e] *= inv;
            const float size = fabsf(mine[t][e]);
            zero = __builtin_fmaf(size, 0.0f, zero);
            if constexpr (kF) least = fminf(least, size == 0.0f ? __builtin_inff() : size);
        }
    // a sum of 0: no key seen, or only scores below the first reference
    bool good = zero == 0.0f && sum < __builtin_inff() && (sum > 0.0f || limit <= int(s0 * kStage));
    if constexpr (kF) good = good && least >= (split ? kSmallest * sum : kSmallest);  // (a split's are not divided yet)
    // rows that are not good in some column
    uint64_t bad = __ballot(valid && !good);
    uint32_t again = uint32_t(bad | (bad >> 32));
    if constexpr (kKeys) {
        if (again && l == 0) atomicOr(&bad_rows, again);
        __syncthreads();
        again = bad_rows;
    }
    again = __builtin_amdgcn_readfirstlane(again);
    if (valid && !(again >> (l & 31u) & 1u)) {
        const uint64_t token = d.q_first + uint64_t(i);
        const PartialRow p = partial_row(a, blockIdx.z, doc, i, h);
        if (l < 32 && t0 == 0) {
            if (split)
                *reinterpret_cast<MEZO_GLOBAL v2f_t*>(p.stats) = v2f_t{sum == 0.0f ? -__builtin_inff() : m * kLn2, sum};
            else
                store_lse(a, token, h, m * kLn2, __builtin_amdgcn_logf(sum) * kLn2);
        }
        const uint64_t o = a.out + token * a.o_token + h * a.o_head;
#pragma unroll
        for (uint32_t t = 0; t < kMine; ++t)
#pragma unroll
            for (uint32_t e = 0; e < 16; e += 4) {
                const uint32_t c = (t0 + t) * 32 + 8 * (e >> 2) + 4 * (l >> 5);
                if (c >= a.dim) continue;
                const v4f_t w = {mine[t][e], mine[t][e + 1], mine[t][e + 2], mine[t][e + 3]};
                if (split)
                    *reinterpret_cast<MEZO_GLOBAL v4f_t*>(p.acc + c * 4) = w;
                else if constexpr (kF)
                    *reinterpret_cast<MEZO_GLOBAL v4f_t*>(o + c * 4) = w;
                else
                    *reinterpret_cast<MEZO_GLOBAL v4bf_t*>(o + c * 2) = __builtin_convertvector(w, v4bf_t);
            }
    }
    // (by keys all waves have the same rows: each takes its share of these)
    if constexpr (kKeys) again &= (0xFFFFFFFFu / ((1u << kWaves) - 1)) << wave;
    while (__builtin_expect(again != 0, 0)) {
        const uint32_t lane = uint32_t(__builtin_ctz(again));
        again &= again - 1;
        const int ri = query(first + lane);
        const uint32_t rh = kvh * a.group + (first + lane) % a.group;
        const int rlimit = visible(a, d, ri), end = int(s1 * kStage);
        careful_row<kF>(a, d, doc, kvh, blockIdx.z, ri, rh, int(s0 * kStage), end < rlimit ? end : rlimit);
    }
}

// The splits of a row, joined in their order: a wave a row, a lane a split for the
// statistics and two columns of the accumulator a lane. splits <= 64.
template <bool kF>
__global__ void __launch_bounds__(256) attention_join_kernel(AttentionArgs a)
{
    const uint32_t l = threadIdx.x & 63u;
    const uint64_t row = uint64_t(blockIdx.x) * 4 + (threadIdx.x >> 6);
    if (row >= uint64_t(a.docs) * a.max_q * a.heads) return;
    const uint32_t h = uint32_t(row % a.heads);
    const int i = int(row / a.heads % a.max_q);
    const uint32_t doc = uint32_t(row / a.heads / a.max_q);
    const Document d = read_document(a, doc);
    if (i >= d.nq) return;
    const int limit0 = visible(a, d, i);
    const uint32_t limit = limit0 > 0 ? uint32_t(limit0) : 0;
    const uint32_t most = (limit + a.chunk - 1) / a.chunk, splits = most < a.splits ? most : a.splits;
    float m = -__builtin_inff(), sum = 0.0f;
    if (l < splits) {
        const v2f_t s = *reinterpret_cast<const MEZO_GLOBAL v2f_t*>(partial_row(a, l, doc, i, h).stats);
        m = s.x;
        sum = s.y;
    }
    float top = m;
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off));
    // (a split without a key of this row has the sum 0 and the accumulator 0)
    float weight = exp2_fast((m - (top == -__builtin_inff() ? 0.0f : top)) * kLog2e);
    const float part_sum = sum;
    sum = fabsf(sum) * weight;
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off);
    // (at most 1 in all: the accumulator does not overflow)
    weight *= (sum == 0.0f ? 0.0f : 1.0f / sum) * (part_sum < 0.0f ? -part_sum : 1.0f);
    float acc[2] = {0.0f, 0.0f};
    constexpr uint32_t kAhead = 8;  // loads in flight
    for (uint32_t s0 = 0; s0 < splits; s0 += kAhead) {
        float part[kAhead][2];
#pragma unroll
        for (uint32_t s = 0; s < kAhead; ++s) {
            const uint64_t at = partial_row(a, s0 + s < splits ? s0 + s : splits - 1, doc, i, h).acc;
#pragma unroll
            for (uint32_t c = 0; c < 2; ++c)
                part[s][c] = l + 64 * c < a.dim ? reinterpret_cast<const gfloat_t*>(at)[l + 64 * c] : 0.0f;
        }
#pragma unroll
        for (uint32_t s = 0; s < kAhead; ++s) {
            if (s0 + s >= splits) break;
            const float w = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(weight), s0 + s));
#pragma unroll
            for (uint32_t c = 0; c < 2; ++c) acc[c] += part[s][c] * w;
        }
    }
    const uint64_t token = d.q_first + uint64_t(i);
    for (uint32_t c = 0; c < 2; ++c)
        if (l + 64 * c < a.dim) store_element<kF>(a.out + token * a.o_token + h * a.o_head, l + 64 * c, acc[c]);
    if (l == 0) store_lse(a, token, h, top, logf(sum));
}

template <bool kF, uint32_t kD>
hipError_t launch(AttentionArgs a, hipStream_t stream)
{
    constexpr uint32_t kKeyWaves = kF && kD > 64 ? 2 : 4;
    void* params[] = {&a};
    const uint64_t rows = uint64_t(a.max_q) * a.group;
    const bool keys = by_keys(rows);
    const dim3 grid(a.docs * a.kv_heads, uint32_t(keys ? 1 : (rows + 127) / 128), a.splits);
    const void* f = reinterpret_cast<const void*>(attention_kernel<kF, kD, 4, false, kGeneral>);
    if (keys) {
        f = reinterpret_cast<const void*>(attention_kernel<kF, kD, kKeyWaves, true, kGeneral>);
    } else if constexpr (!kF) {
        if (a.softcap == 0.0f && !a.slopes && a.scale > 0.0f)
            f = reinterpret_cast<const void*>(attention_kernel<kF, kD, 4, false, kPlain>);
        else if (a.softcap == 0.0f && a.scale > 0.0f)
            f = reinterpret_cast<const void*>(attention_kernel<kF, kD, 4, false, kBiased>);
        else if (a.softcap > 0.0f && a.softcap <= 66.0f && !a.slopes)
            f = reinterpret_cast<const void*>(attention_kernel<kF, kD, 4, false, kCapped>);
    } else if (a.softcap == 0.0f) {
        f = reinterpret_cast<const void*>(attention_kernel<kF, kD, 4, false, kUncapped>);
    }
    const hipError_t e = hipLaunchKernel(f, grid, dim3(keys ? kKeyWaves * 64 : 256), params, 0, stream);
    if (e != hipSuccess || a.splits == 1) return e;
    const uint64_t all = uint64_t(a.docs) * a.max_q * a.heads;
    return hipLaunchKernel(reinterpret_cast<const void*>(attention_join_kernel<kF>), dim3(uint32_t((all + 3) / 4)),
                           dim3(256), params, 0, stream);
}

hipError_t launch_attention(const AttentionArgs& args, hipStream_t stream)
{
    if (args.dtype == kF32) return args.dim <= 64 ? launch<true, 64>(args, stream) : launch<true, 128>(args, stream);
    return args.dim <= 64 ? launch<false, 64>(args, stream) : launch<false, 128>(args, stream);
}

}  // namespace mezo
