// nf4_linear.hip — c = x w^T with weights in 4-bit storage, which are not written out in full:
// w_e = v[code_e] absmax[e / 64] of the flattened matrix [n, k], as mezo_nf4_dequantize gives
// it in the type of x (fp32, or that rounded to bf16). Products are summed in fp32 and the sum
// is rounded once.
//
// bf16: the products of bf16 are exact in v_mfma_f32_16x16x32_bf16. fp32: each operand is
// three bf16, its 24 bits in 8 and 8 and 8, and six of the nine products are summed: all but the
// second part by the third and the third by itself. Parts are rounded to nearest where operands are
// laid out, and what is left out is at most 2^-24 of the product; the kernels of few rows cut those of
// one operand, where they use it (rounding there costs 6%: 1 x 16384 x 4096 23.0 -> 24.5 us), and
// leave out up to 3 2^-24. With both operands cut it would be 2^-21, and always towards 0. The parts of a value
// below 2^-110 end at bf16's last bit, 2^-133; one that is infinite or NaN makes its row NaN.
//
// Few rows: codes go to LDS as they are and are looked up in a table of all pairs there, in
// front of the matrix instructions that use them (nf4_thin_kernel, below). The lookups bound
// it, and the loads of the codes under them: one row by 16384 x 4096 weights 11 us (37 MB, 3.4
// TB/s), 24 rows by 4096 x 16384 17, 64 rows by 16384 x 4096 20.
// Few rows where k is no multiple of 64: codes go straight into registers (nf4_ragged_kernel).
// Many rows: a slab of the weights is expanded into the workspace (2 bytes an element, 6 for
// fp32), and a tiled product reads it. Expanding costs 2.5 bytes an element once, the product
// 2 m operations: from a few hundred rows on it does not show (8192 x 16384 x 4096: 31 us of
// 860, 1.3 PFLOP/s bf16).
#include <type_traits>

#include "lds_dma.hpp"
#include "nf4.hpp"
#include "nf4_linear_launch.hpp"
#include "records.hpp"
#include "stream_io.hpp"

namespace mezo {

typedef float v4f_t __attribute__((ext_vector_type(4)));
typedef __bf16 v4bf_t __attribute__((ext_vector_type(4)));
typedef __bf16 v8bf_t __attribute__((ext_vector_type(8)));
typedef MEZO_GLOBAL uint8_t gu8_t;
typedef MEZO_GLOBAL uint32_t gu32_t;

// ---- laying out ------------------------------------------------------------------

// The upper 16 bits of two floats.
__device__ __forceinline__ uint32_t upper_halves(float lo, float hi)
{
    return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
}

// Floats as three bf16 each, eight at a time, their parts cut or rounded to nearest. Cutting
// keeps the largest floats finite by itself; where rounding would not, the first part is the
// largest bf16. A part of what is not finite is not finite.
struct Planes {
    v8bf_t p[3];
};

template <bool kCut>
__device__ __forceinline__ Planes planes_of(const float (&x)[8])
{
    constexpr float kLargest = 0x1.FEp127f;
    Planes o;
    float r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = x[i];
#pragma unroll
    for (int p = 0; p < 3; ++p) {
        if constexpr (kCut) {
            uint32_t u[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) u[i] = upper_halves(r[2 * i], r[2 * i + 1]);
            o.p[p] = __builtin_bit_cast(v8bf_t, u32x4_t{u[0], u[1], u[2], u[3]});
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                o.p[p][i] = static_cast<__bf16>(p ? r[i] : __builtin_amdgcn_fmed3f(r[i], -kLargest, kLargest));
        }
        if (p < 2)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                r[i] -= kCut ? __uint_as_float(__float_as_uint(r[i]) & 0xFFFF0000u) : static_cast<float>(o.p[p][i]);
    }
    return o;
}

// Eight values as one or three planes of bf16, 16 bytes each.
template <bool kWide>
__device__ __forceinline__ void store_planes(uint64_t at, uint64_t plane, const float (&x)[8])
{
    if constexpr (kWide) {
        const Planes o = planes_of<false>(x);
#pragma unroll
        for (int p = 0; p < 3; ++p) *reinterpret_cast<gu32x4_t*>(at + p * plane) = __builtin_bit_cast(u32x4_t, o.p[p]);
    } else {
        v8bf_t b;
#pragma unroll
        for (int i = 0; i < 8; ++i) b[i] = static_cast<__bf16>(x[i]);
        *reinterpret_cast<gu32x4_t*>(at) = __builtin_bit_cast(u32x4_t, b);
    }
}

struct LayArgs {
    uint64_t from, absmax;  // values and nothing, or codes and scales
    uint64_t ld;            // values: elements from one row to the next
    uint64_t to, plane;     // rows of `columns` bf16; bytes from one plane to the next
    uint64_t first, last;   // codes: the first row's first element, and the end of all
    uint64_t rows, k, columns;
};

// A unit of 8 columns by its number: its row and first column (32 bits where they hold the
// number: a division in 64 takes as long as the rest).
struct Unit {
    uint64_t row, col;
};
__device__ __forceinline__ Unit unit_of(const LayArgs& a, uint64_t i)
{
    const uint64_t per_row = a.columns / 8;
    if (a.rows * per_row <= 0xFFFFFFFFu) {  // (uniform)
        const uint32_t row = uint32_t(i) / uint32_t(per_row);
        return {row, (i - uint64_t(row) * per_row) * 8};
    }
    const uint64_t row = i / per_row;
    return {row, (i - row * per_row) * 8};
}

// Rows of values into planes: a lane 8 columns.
template <bool kF>
__global__ void __launch_bounds__(256) nf4_lay_values_kernel(LayArgs a)
{
    const uint64_t i = uint64_t(blockIdx.x) * 256 + threadIdx.x;
    if (i >= a.rows * (a.columns / 8)) return;
    const Unit at = unit_of(a, i);
    const uint64_t row = at.row, c = at.col;
    float x[8];
#pragma unroll
    for (uint32_t j = 0; j < 8; ++j) {
        x[j] = 0.0f;
        if (c + j < a.k) {
            const uint64_t e = row * a.ld + c + j;
            if constexpr (kF)
                x[j] = reinterpret_cast<const gfloat_t*>(a.from)[e];
            else
                x[j] = __uint_as_float(uint32_t(reinterpret_cast<const gu16_t*>(a.from)[e]) << 16);
        }
    }
    store_planes<kF>(a.to + i * 16, a.plane, x);
}

// Rows of whole blocks of values, copied next to each other: a lane 8 columns.
template <bool kF>
__global__ void __launch_bounds__(256) nf4_copy_rows_kernel(LayArgs a)
{
    using element_t = std::conditional_t<kF, gu32_t, gu16_t>;
    const uint64_t i = uint64_t(blockIdx.x) * 256 + threadIdx.x;
    if (i >= a.rows * (a.columns / 8)) return;
    const Unit at = unit_of(a, i);
    const element_t* from = reinterpret_cast<const element_t*>(a.from) + at.row * a.ld + at.col;
    element_t* to = reinterpret_cast<element_t*>(a.to) + i * 8;
#pragma unroll
    for (uint32_t j = 0; j < 8; ++j) to[j] = from[j];
}

// The codes of elements e .. e + 7, of `last` in all.
__device__ __forceinline__ uint32_t eight_codes(uint64_t codes, uint64_t e, uint64_t last)
{
    auto word = [&](uint64_t i) {
        const uint64_t bytes = (last + 1) / 2;
        if (4 * i + 4 <= bytes) return reinterpret_cast<const gu32_t*>(codes)[i];
        uint32_t w = 0;
        for (uint64_t b = 4 * i; b < bytes; ++b) w |= uint32_t(reinterpret_cast<const gu8_t*>(codes)[b]) << (8 * (b - 4 * i));
        return w;
    };
    const uint32_t shift = uint32_t(e & 7u) * 4;
    const uint32_t lo = word(e >> 3);
    if (shift == 0) return lo;
    return uint32_t((uint64_t(word((e >> 3) + 1)) << 32 | lo) >> shift);
}

constexpr uint32_t kExpandUnits = 4;
typedef float v2f_t __attribute__((ext_vector_type(2)));

// Rows of weights into planes: a lane 8 columns at a time, kExpandUnits of them, whose loads
// are all under way before the first is used. A code's value comes from the lane that holds it.
// kWhole: k is a multiple of 8, so a unit is a whole word of codes under one scale.
template <bool kWide, bool kWhole>
__global__ void __launch_bounds__(256) nf4_expand_kernel(LayArgs a)
{
    uint32_t table = 0;
#pragma unroll
    for (uint32_t i = 0; i < kNF4Codes; ++i)
        table = (threadIdx.x & 15u) == i ? __builtin_bit_cast(uint32_t, kNF4Values[i]) : table;
    const uint64_t i0 = uint64_t(blockIdx.x) * (256 * kExpandUnits) + threadIdx.x, all = a.rows * (a.columns / 8);
    [[maybe_unused]] const uint64_t top = (a.last - 1) / kNF4Block;
    uint32_t codes[kExpandUnits], valid[kExpandUnits];
    float s0[kExpandUnits];
    [[maybe_unused]] uint32_t left[kExpandUnits];
    [[maybe_unused]] float s1[kExpandUnits];
#pragma unroll
    for (uint32_t u = 0; u < kExpandUnits; ++u) {
        const uint64_t i = i0 + u * 256;
        const Unit at = unit_of(a, i < all ? i : all - 1);
        valid[u] = at.col >= a.k ? 0u : (a.k - at.col < 8 ? uint32_t(a.k - at.col) : 8u);
        const uint64_t e = a.first + at.row * a.k + (valid[u] ? at.col : 0), b = e / kNF4Block;
        s0[u] = reinterpret_cast<const gfloat_t*>(a.absmax)[b];
        if constexpr (kWhole) {
            codes[u] = __builtin_nontemporal_load(reinterpret_cast<const gu32_t*>(a.from) + e / 8);
        } else {
            codes[u] = eight_codes(a.from, e, a.last);
            left[u] = kNF4Block - uint32_t(e % kNF4Block);
            s1[u] = left[u] >= 8 ? s0[u] : reinterpret_cast<const gfloat_t*>(a.absmax)[b < top ? b + 1 : top];
        }
    }
#pragma unroll
    for (uint32_t u = 0; u < kExpandUnits; ++u) {
        const uint64_t i = i0 + u * 256;
        float x[8];
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j)  // (by all lanes: any of them may be asked)
            x[j] = __uint_as_float(uint32_t(__builtin_amdgcn_ds_bpermute(int((codes[u] >> (4 * j) & 15u) << 2), int(table))));
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j) {
            if constexpr (kWhole)
                x[j] = valid[u] ? x[j] * s0[u] : 0.0f;
            else
                x[j] = j < valid[u] ? x[j] * (j < left[u] ? s0[u] : s1[u]) : 0.0f;
        }
        if (i < all) store_planes<kWide>(a.to + i * 16, a.plane, x);
    }
}

// ---- the product of what was laid out ------------------------------------------------

struct NF4MatmulArgs {
    uint64_t x, w;              // first planes
    uint64_t x_plane, w_plane;  // bytes from one plane to the next
    uint64_t c, ldc;
    uint64_t partial;           // fp32 [splits, m, n rounded up to 4] of a split product
    uint32_t m, n, stages;      // 64 columns each
    uint32_t x_row, w_row;      // bytes
    uint32_t splits;
};

template <bool kWideOut>
__device__ __forceinline__ void store4(const NF4MatmulArgs& a, bool whole, uint32_t row, uint32_t col, v4f_t v)
{
    using Out = std::conditional_t<kWideOut, float, __bf16>;
    typedef Out out4_t __attribute__((ext_vector_type(4)));
    const out4_t b = __builtin_convertvector(v, out4_t);
    MEZO_GLOBAL Out* p = reinterpret_cast<MEZO_GLOBAL Out*>(a.c) + row * a.ldc + col;
    if (whole && col + 4 <= a.n) {
        *reinterpret_cast<MEZO_GLOBAL out4_t*>(p) = b;
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i)
            if (col + i < a.n) p[i] = b[i];
    }
}

template <bool kWideOut>
__device__ __forceinline__ bool whole_groups(const NF4MatmulArgs& a)
{
    constexpr uint64_t kBytes = kWideOut ? 4 : 2;
    return ((a.c | (a.ldc * kBytes)) & (4 * kBytes - 1)) == 0;
}

__device__ __forceinline__ uint64_t partial_at(const NF4MatmulArgs& a, uint32_t split, uint32_t row, uint32_t col)
{
    return a.partial + ((uint64_t(split) * a.m + row) * ((a.n + 3) / 4) + col / 4) * 16;
}

// The pairs of planes of an fp32 product, the smallest first: (x's, w's).
__device__ __forceinline__ uint32_t plane_of_x(uint32_t pair) { return 0x001021u >> (4 * pair) & 15u; }
__device__ __forceinline__ uint32_t plane_of_w(uint32_t pair) { return 0x010201u >> (4 * pair) & 15u; }

// Tiles of kBM activations x kBN weights, kWM x kWN waves. Weights are the matrix
// instruction's rows and activations its columns, so that a lane's four results lie next to
// each other in a row of c. A stage is 64 columns (128 bytes) of every row of the tile, loaded
// straight into LDS, two stages, one computed on while the other loads. A row's eight 16-byte
// chunks are stored at chunk ^ ((row / 2) & 7): the 16 rows of a fragment then spread over all
// 64 banks. fp32: the loop goes over the pairs of planes one after another.
template <uint32_t kBM, uint32_t kBN, uint32_t kWM, uint32_t kWN, bool kWide, bool kWideOut>
__global__ void __launch_bounds__(kWM* kWN * 64) nf4_matmul_kernel(NF4MatmulArgs a)
{
    constexpr uint32_t kWaves = kWM * kWN, kRows = kBM + kBN;
    constexpr uint32_t kFM = kBM / kWM / 16, kFN = kBN / kWN / 16;  // fragments of a wave
    constexpr uint32_t kLoads = kRows / 8 / kWaves;                 // 8 rows a load
    static_assert(kRows % (8 * kWaves) == 0 && kBM % 64 == 0 && kBN % 64 == 0);
    __shared__ __attribute__((aligned(1024))) uint8_t lds[2][kRows * 128];

    const uint32_t l = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // workgroups go round the 8 XCDs: each XCD gets a compact part of c (its L2 then holds the
    // rows its workgroups share), in groups of 8 tile rows
    const uint32_t tm = (a.m + kBM - 1) / kBM, tn = (a.n + kBN - 1) / kBN, tiles = tm * tn;
    const uint32_t xcd = blockIdx.x % 8, each = tiles / 8, rest = tiles % 8;
    const uint32_t id = blockIdx.x / 8 + xcd * each + (xcd < rest ? xcd : rest);
    const uint32_t band = id / (8 * tn), height = tm - band * 8 < 8 ? tm - band * 8 : 8;
    const uint32_t in = id - band * 8 * tn;
    const uint32_t m0 = (band * 8 + in % height) * kBM, n0 = in / height * kBN;

    const uint32_t all = (kWide ? 6 : 1) * a.stages;
    const uint32_t begin = uint32_t(uint64_t(all) * blockIdx.y / a.splits),
                   end = uint32_t(uint64_t(all) * (blockIdx.y + 1) / a.splits);
    // a load is 8 rows of x or of w; rows past the end: the last one's again
    const uint64_t x0 = a.x + uint64_t(m0) * a.x_row, w0 = a.w + uint64_t(n0) * a.w_row;
    const uint32_t xlast = a.m - m0 - 1, wlast = a.n - n0 - 1;
    uint32_t src[kLoads];  // this lane's 16 bytes of each of its rows
#pragma unroll
    for (uint32_t i = 0; i < kLoads; ++i) {
        const uint32_t first = (wave * kLoads + i) * 8;
        const bool ofx = first < kBM;
        const uint32_t r = first + (l >> 3) - (ofx ? 0 : kBM), last = ofx ? xlast : wlast;
        const uint32_t swizzle = (first / 2 + (l >> 4)) & 7u;  // (row / 2) & 7
        src[i] = (r < last ? r : last) * (ofx ? a.x_row : a.w_row) + ((l & 7u) ^ swizzle) * 16;
    }
    const uint32_t lds0 = lds_offset(&lds[0][0]) + wave * kLoads * 1024;
    auto stage = [&](uint32_t s, uint32_t buffer) {
        uint64_t xs = x0, ws = w0;
        uint32_t kb = s;
        if constexpr (kWide) {
            const uint32_t pair = s / a.stages;
            kb = s - pair * a.stages;
            xs += plane_of_x(pair) * a.x_plane;
            ws += plane_of_w(pair) * a.w_plane;
        }
#pragma unroll
        for (uint32_t i = 0; i < kLoads; ++i)
            dma_to_lds(((wave * kLoads + i) * 8 < kBM ? xs : ws) + uint64_t(kb) * 128, src[i],
                       lds0 + buffer * kRows * 128 + i * 1024);
    };

    const uint32_t fr = l & 15u, fg = l >> 4;
    const uint32_t wm = (wave / kWN) * kFM * 16, wn = (wave % kWN) * kFN * 16;
    v4f_t acc[kFM][kFN] = {};
    stage(begin, 0);
    for (uint32_t s = begin; s < end; ++s) {
        const uint32_t buffer = (s - begin) & 1u;
        dma_wait();
        lds_barrier();  // stage s is there, and nobody reads the other one any more
        if (s + 1 < end) stage(s + 1, buffer ^ 1u);
        const uint8_t* t = lds[buffer];
        struct Fragment {
            v8bf_t v[2];
        };
        auto fragment = [&](uint32_t row) {
            const uint32_t r = row + fr;
            Fragment f;
            f.v[0] = *reinterpret_cast<const v8bf_t*>(t + r * 128 + ((fg ^ (fr >> 1)) * 16));
            f.v[1] = *reinterpret_cast<const v8bf_t*>(t + r * 128 + (((fg + 4) ^ (fr >> 1)) * 16));
            return f;
        };
        Fragment w[kFN], next = fragment(wm);
#pragma unroll
        for (uint32_t j = 0; j < kFN; ++j) w[j] = fragment(kBM + wn + j * 16);
#pragma unroll
        for (uint32_t i = 0; i < kFM; ++i) {
            const Fragment x = next;
            if (i + 1 < kFM) next = fragment(wm + (i + 1) * 16);
#pragma unroll
            for (uint32_t j = 0; j < kFN; ++j)
#pragma unroll
                for (uint32_t h = 0; h < 2; ++h)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[j].v[h], x.v[h], acc[i][j], 0, 0, 0);
        }
    }
    const bool whole = whole_groups<kWideOut>(a);
    if (whole || a.splits > 1) {
#pragma unroll
        for (uint32_t i = 0; i < kFM; ++i) {
            const uint32_t row = m0 + wm + i * 16 + fr;
            if (row >= a.m) continue;
#pragma unroll
            for (uint32_t j = 0; j < kFN; ++j) {
                const uint32_t col = n0 + wn + j * 16 + fg * 4;
                if (a.splits == 1)
                    store4<kWideOut>(a, whole, row, col, acc[i][j]);
                else if (col < a.n)
                    *reinterpret_cast<MEZO_GLOBAL v4f_t*>(partial_at(a, blockIdx.y, row, col)) = acc[i][j];
            }
        }
        return;
    }
    // Where rows of c do not lie on the alignment of four columns, a wave's part of the tile goes
    // through LDS, 16 rows at a time, and out with neighbouring lanes on neighbouring columns (lanes
    // would store one by one, 4 columns apart).
    using Out = std::conditional_t<kWideOut, float, __bf16>;
    constexpr uint32_t kCols = kFN * 16;
    static_assert(kWaves * 16 * (kCols + 4) * 4 <= sizeof(lds), "the rows fit");
    lds_barrier();  // the last stage is read
    float* room = reinterpret_cast<float*>(&lds[0][0]) + wave * 16 * (kCols + 4);
    const uint32_t col = l % kCols, n = n0 + wn + col;
    MEZO_GLOBAL Out* c = reinterpret_cast<MEZO_GLOBAL Out*>(a.c) + n;
#pragma unroll
    for (uint32_t i = 0; i < kFM; ++i) {
#pragma unroll
        for (uint32_t j = 0; j < kFN; ++j)
            *reinterpret_cast<v4f_t*>(room + fr * (kCols + 4) + j * 16 + fg * 4) = acc[i][j];
        lds_wait();  // (the wave's own room)
        for (uint32_t r = l / kCols; r < 16; r += 64 / kCols) {
            const uint32_t row = m0 + wm + i * 16 + r;
            if (row < a.m && n < a.n) c[row * a.ldc] = static_cast<Out>(room[r * (kCols + 4) + col]);
        }
        lds_wait();
    }
}

// The sums of a product whose k was split, joined in the order of the splits.
template <bool kWideOut>
__global__ void __launch_bounds__(256) nf4_join_kernel(NF4MatmulArgs a)
{
    const uint32_t groups = (a.n + 3) / 4;
    const uint64_t i = uint64_t(blockIdx.x) * 256 + threadIdx.x;
    if (i >= uint64_t(a.m) * groups) return;
    const uint32_t row = uint32_t(i / groups), col = uint32_t(i % groups) * 4;
    v4f_t sum = {};
    for (uint32_t s = 0; s < a.splits; ++s)
        sum += *reinterpret_cast<const MEZO_GLOBAL v4f_t*>(partial_at(a, s, row, col));
    store4<kWideOut>(a, true, row, col, sum);
}

// The same where rows of c do not lie on the alignment of four columns: a lane a column.
template <bool kWideOut>
__global__ void __launch_bounds__(256) nf4_join_columns_kernel(NF4MatmulArgs a)
{
    using Out = std::conditional_t<kWideOut, float, __bf16>;
    const uint64_t i = uint64_t(blockIdx.x) * 256 + threadIdx.x;
    if (i >= uint64_t(a.m) * a.n) return;
    const uint32_t row = uint32_t(i / a.n), col = uint32_t(i - uint64_t(row) * a.n);
    float sum = 0.0f;
    for (uint32_t s = 0; s < a.splits; ++s)
        sum += reinterpret_cast<const gfloat_t*>(partial_at(a, s, row, col))[col & 3u];
    (reinterpret_cast<MEZO_GLOBAL Out*>(a.c) + row * a.ldc)[col] = static_cast<Out>(sum);
}

// ---- few rows -----------------------------------------------------------------------

// A product of few activations reads each weight once and is bound by that as long as decoding
// stays cheap. A byte of codes is looked up whole: a table holds the two values of each byte,
// 32 times over, a copy for each lane of a half wave, so that a lane's lookups never meet
// another's bank (17 to 32 activations and the first two parts of fp32 have 16 copies, a
// copy for two lanes); the address is the byte in bits 8 .. 15 and the lane below, one v_perm_b32.
// Then a multiplication by the block's scale each and one conversion: 2 vector instructions a
// weight in bf16 (selecting by v_perm_b32 out of registers takes 4).
//
// A workgroup takes kRowWaves * kRG * 16 of the weights' rows and a share of k; its waves are
// kRowWaves x kKWaves: a stage is a block of 64 for each of the kKWaves, of all the rows, with
// their scales and the activations beside them, loaded straight into LDS kDepth - 1 stages
// ahead. The order of k within a block does not matter as long as both operands agree: a lane
// takes 16 weights next to each other. The waves' sums join in LDS, in their order.
//
// What bounds it is LDS: 8 bytes a lookup of two weights, and the activations, which each
// group of kRG * 16 rows reads again (1 x 16384 x 4096: 13.2 us in groups of 16, 12.6 in 32;
// the loads alone take 9.7, the rest alone 12.1). With 16 copies of the table instead of 32
// lookups meet, and the room is another stage's: 32 activations 16.8 -> 16.1 us, one 12.6 ->
// 14.2. Issuing a stage's lookups under the products of the one before, 8 waves instead of 16,
// and two workgroups a CU with half a table each lost.
struct NF4ThinArgs {
    uint64_t x, codes, absmax, c, ldc, partial;
    uint32_t m, n, blocks;  // blocks of 64 of a row
    uint32_t x_row;         // bytes
    uint32_t splits;
};

typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));

// c + w x of split operands, the smallest products first.
__device__ __forceinline__ v4f_t product(const Planes& w, const Planes& x, v4f_t c)
{
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w.p[1], x.p[1], c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w.p[0], x.p[2], c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w.p[2], x.p[0], c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w.p[0], x.p[1], c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w.p[1], x.p[0], c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(w.p[0], x.p[0], c, 0, 0, 0);
}

constexpr uint32_t kThinWaves = 16;

// fp32: the table holds the three parts of each value, and a block's sum is scaled as a whole.
// The values are kept 2^-7 of themselves, so that no sum of 64 products of finite activations
// overflows where its scaled value does not.
constexpr float kThinScale = 0x1p-7f;

template <bool kF, uint32_t kRowWaves, uint32_t kRG, uint32_t kXRows, uint32_t kDepth, uint32_t kCopies, bool kWideOut>
__global__ void __launch_bounds__(kThinWaves * 64) nf4_thin_kernel(NF4ThinArgs a)
{
    constexpr uint32_t kKWaves = kThinWaves / kRowWaves, kRows = kRowWaves * kRG * 16;
    constexpr uint32_t kFM = kXRows < 16 ? 1 : kXRows / 16;
    constexpr uint32_t kElement = kF ? 4 : 2;
    // a stage in LDS: codes [kRows][kCodeChunks], activations [kXRows][kXChunks] of 16 bytes,
    // scales [kRows][kKWaves] of 4
    constexpr uint32_t kCodeChunks = kKWaves * 2, kXChunks = kKWaves * 4 * kElement;
    constexpr uint32_t kCodeLoads = kRows * kCodeChunks / 64, kXLoads = kXRows * kXChunks / 64,
                       kScaleLoads = kRows * kKWaves / 64;
    constexpr uint32_t kXAt = kCodeLoads * 1024, kScaleAt = kXAt + kXLoads * 1024,
                       kStage = kScaleAt + kScaleLoads * 256;
    static_assert(kRows * kCodeChunks % 64 == 0 && kXRows * kXChunks % 64 == 0 && kRows * kKWaves % 64 == 0);
    constexpr uint32_t kLoads = kCodeLoads + kXLoads + kScaleLoads, kPerWave = (kLoads + kThinWaves - 1) / kThinWaves;
    // (one object, the table first: its addresses then need no base)
    constexpr uint32_t kTable = kF ? kNF4Pairs * 256 : kNF4Pairs * kCopies * sizeof(v2f_t);
    __shared__ __attribute__((aligned(1024))) uint8_t memory[kTable + kDepth * kStage];
    uint8_t* const lds = memory + kTable;
    static_assert(kKWaves * kRows * kFM * 16 * 4 <= sizeof(memory), "the waves' sums fit");

    const uint32_t l = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t n0 = blockIdx.x * kRows, m0 = blockIdx.z * kXRows;
    const uint32_t stages = (a.blocks + kKWaves - 1) / kKWaves;
    const uint32_t s0 = uint32_t(uint64_t(stages) * blockIdx.y / a.splits),
                   s1 = uint32_t(uint64_t(stages) * (blockIdx.y + 1) / a.splits);

    // The order of a row's chunks in LDS, such that the 16 rows that are read together lie on
    // different banks.
    auto code_swizzle = [](uint32_t r) { return kCodeChunks >= 16 ? r & 15u : (r >> 1) & 7u; };
    auto x_swizzle = [](uint32_t r) { return r & 15u; };

    // This wave's loads of a stage (those left over: the last one again). A lane's row never
    // changes and its column moves on by `step` bytes a stage, to the row's end.
    uint64_t base[kPerWave];
    uint32_t row_at[kPerWave], col[kPerWave], step[kPerWave], end[kPerWave], to[kPerWave];
    bool words[kPerWave];
#pragma unroll
    for (uint32_t j = 0; j < kPerWave; ++j) {
        const uint32_t i0 = wave + j * kThinWaves, i = i0 < kLoads ? i0 : kLoads - 1;
        words[j] = false;
        if (i < kCodeLoads) {
            const uint32_t g = i * 64 + l, r = g / kCodeChunks, last = a.n - n0 - 1;
            base[j] = a.codes + uint64_t(n0) * a.blocks * 32;
            row_at[j] = (r < last ? r : last) * (a.blocks * 32);
            col[j] = ((g % kCodeChunks) ^ code_swizzle(r)) * 16;
            step[j] = kCodeChunks * 16;
            end[j] = a.blocks * 32 - 16;
            to[j] = i * 1024;
        } else if (i < kCodeLoads + kXLoads) {
            const uint32_t g = (i - kCodeLoads) * 64 + l, r = g / kXChunks, last = a.m - m0 - 1;
            base[j] = a.x + uint64_t(m0) * a.x_row;
            row_at[j] = (r < last ? r : last) * a.x_row;
            col[j] = ((g % kXChunks) ^ x_swizzle(r)) * 16;
            step[j] = kXChunks * 16;
            end[j] = a.blocks * 64 * kElement - 16;
            to[j] = kXAt + (i - kCodeLoads) * 1024;
        } else {
            const uint32_t g = (i - kCodeLoads - kXLoads) * 64 + l, r = g / kKWaves, last = a.n - n0 - 1;
            base[j] = a.absmax + uint64_t(n0) * a.blocks * 4;
            row_at[j] = (r < last ? r : last) * (a.blocks * 4);
            col[j] = g % kKWaves * 4;
            step[j] = kKWaves * 4;
            end[j] = a.blocks * 4 - 4;
            to[j] = kScaleAt + (i - kCodeLoads - kXLoads) * 256;
            words[j] = true;
        }
    }
    const uint32_t lds0 = lds_offset(lds);
    auto load = [&](uint32_t s, uint32_t buffer) {
#pragma unroll
        for (uint32_t j = 0; j < kPerWave; ++j) {
            const uint32_t at = col[j] + s * step[j], off = row_at[j] + (at < end[j] ? at : end[j]);
            if (words[j])
                dma_word_to_lds(base[j], off, lds0 + buffer * kStage + to[j]);
            else
                dma_to_lds(base[j], off, lds0 + buffer * kStage + to[j]);
        }
    };
    uint32_t ahead = s0;
    for (uint32_t d = 0; d + 1 < kDepth && ahead < s1; ++d, ++ahead) load(ahead, (ahead - s0) % kDepth);
    {
        // (a lane writes its part of a byte's copies)
        constexpr uint32_t kEach = kThinWaves * 64 / kNF4Pairs;
        const uint32_t byte = threadIdx.x / kEach;
        v2f_t v = {0.0f, 0.0f};
#pragma unroll
        for (uint32_t i = 0; i < kNF4Codes; ++i) {
            v.x = (byte & 15u) == i ? kNF4Values[i] : v.x;
            v.y = (byte >> 4) == i ? kNF4Values[i] : v.y;
        }
        if constexpr (kF) {
            // a row of 256 bytes: the pair's first and second parts 16 times, its third 32 times
            const float lo[8] = {v.x * kThinScale, v.y * kThinScale, 0, 0, 0, 0, 0, 0};
            const Planes p = planes_of<false>(lo);
            const u32x4_t a0 = __builtin_bit_cast(u32x4_t, p.p[0]), a1 = __builtin_bit_cast(u32x4_t, p.p[1]),
                          a2 = __builtin_bit_cast(u32x4_t, p.p[2]);
            const u32x4_t w = threadIdx.x % 4 < 2 ? u32x4_t{a0[0], a1[0], a0[0], a1[0]} : u32x4_t{a2[0], a2[0], a2[0], a2[0]};
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i)
                *reinterpret_cast<u32x4_t*>(memory + byte * 256 + threadIdx.x % 4 * 64 + i * 16) = w;
        } else {
            const v4f_t twice = {v.x, v.y, v.x, v.y};
#pragma unroll
            for (uint32_t i = 0; i < kCopies / 2 / kEach; ++i)
                *reinterpret_cast<v4f_t*>(memory + (byte * (kCopies / 2) + i * kEach + threadIdx.x % kEach) * 16) = twice;
        }
    }

    const uint32_t fr = l & 15u, fg = l >> 4;
    const uint32_t rw = wave / kKWaves, q = wave % kKWaves;
    const uint32_t mine = kF ? (l & 15u) * 8 : (l % kCopies) * 8;  // this lane's copy
    [[maybe_unused]] const uint32_t third = 128 + (l & 31u) * 4;   // and of third parts
    // where this lane reads in a stage: of each of its groups of 16 rows, and of the activations
    const uint32_t xr = kXRows < 16 ? fr % kXRows : fr;
    uint32_t code_at[kRG], scale_at[kRG], x_at[2];
#pragma unroll
    for (uint32_t g = 0; g < kRG; ++g) {
        const uint32_t r = (rw * kRG + g) * 16 + fr;
        code_at[g] = (r * kCodeChunks + ((2 * q + (fg >> 1)) ^ code_swizzle(r))) * 16 + (fg & 1u) * 8;
        scale_at[g] = kScaleAt + ((kF ? (rw * kRG + g) * 16 + fg * 4 : r) * kKWaves + q) * 4;
    }
#pragma unroll
    for (uint32_t h = 0; h < 2; ++h)
        x_at[h] = kXAt + (xr * kXChunks + (((q * 8 + fg * 2 + h) * (kElement / 2)) ^ x_swizzle(xr))) * 16;
    v4f_t acc[kRG][kFM] = {};
    for (uint32_t s = s0; s < s1; ++s) {
        // stage s is there (all that is in flight after it: whole stages), and the one before it
        // is read by all
        if (ahead - s == kDepth - 1)
            dma_wait<(kDepth - 2) * kPerWave>();
        else
            dma_wait();
        lds_barrier();
        if (ahead < s1) {
            load(ahead, (ahead - s0) % kDepth);
            ++ahead;
        }
        if (s * kKWaves + q >= a.blocks) continue;  // (of the wave)
        const uint8_t* t = lds + (s - s0) % kDepth * kStage;
        // 16 weights of a row for each group, all lookups under way before the first is used
        u32x2_t code[kRG];
#pragma unroll
        for (uint32_t g = 0; g < kRG; ++g) code[g] = *reinterpret_cast<const u32x2_t*>(t + code_at[g]);
        if constexpr (kF) {
            u32x2_t w[kRG][2][4];
            uint32_t w3[kRG][2][4];
#pragma unroll
            for (uint32_t g = 0; g < kRG; ++g)
#pragma unroll
                for (uint32_t h = 0; h < 2; ++h)
#pragma unroll
                    for (uint32_t i = 0; i < 4; ++i) {
                        const uint32_t byte = 0x0C0C0000u | (4 + i) << 8;
                        w[g][h][i] = *reinterpret_cast<const u32x2_t*>(memory + __builtin_amdgcn_perm(code[g][h], mine, byte));
                        w3[g][h][i] = *reinterpret_cast<const uint32_t*>(memory + __builtin_amdgcn_perm(code[g][h], third, byte));
                    }
            __builtin_amdgcn_sched_barrier(0);
            v4f_t sum[kRG][kFM] = {};  // of this block, unscaled
#pragma unroll
            for (uint32_t h = 0; h < 2; ++h) {
                Planes p[kRG];
#pragma unroll
                for (uint32_t g = 0; g < kRG; ++g) {
                    p[g].p[0] = __builtin_bit_cast(v8bf_t, u32x4_t{w[g][h][0].x, w[g][h][1].x, w[g][h][2].x, w[g][h][3].x});
                    p[g].p[1] = __builtin_bit_cast(v8bf_t, u32x4_t{w[g][h][0].y, w[g][h][1].y, w[g][h][2].y, w[g][h][3].y});
                    p[g].p[2] = __builtin_bit_cast(v8bf_t, u32x4_t{w3[g][h][0], w3[g][h][1], w3[g][h][2], w3[g][h][3]});
                }
#pragma unroll
                for (uint32_t f = 0; f < kFM; ++f) {
                    const u32x4_t lo = *reinterpret_cast<const u32x4_t*>(t + x_at[h] + f * 16 * kXChunks * 16);
                    const u32x4_t hi = *reinterpret_cast<const u32x4_t*>(t + (x_at[h] ^ 16u) + f * 16 * kXChunks * 16);
                    float v[8];
#pragma unroll
                    for (uint32_t i = 0; i < 4; ++i) {
                        v[i] = __uint_as_float(lo[i]);
                        v[i + 4] = __uint_as_float(hi[i]);
                    }
                    const Planes x = planes_of<true>(v);
#pragma unroll
                    for (uint32_t g = 0; g < kRG; ++g) sum[g][f] = product(p[g], x, sum[g][f]);
                }
            }
#pragma unroll
            for (uint32_t g = 0; g < kRG; ++g)
#pragma unroll
                for (uint32_t i = 0; i < 4; ++i) {  // a lane's results are rows 4 fg .. + 3
                    const float scale = *reinterpret_cast<const float*>(t + scale_at[g] + i * kKWaves * 4);
#pragma unroll
                    for (uint32_t f = 0; f < kFM; ++f) acc[g][f][i] = __builtin_fmaf(sum[g][f][i], scale, acc[g][f][i]);
                }
        } else {
            float scale[kRG];
            v2f_t w[kRG][2][4];
#pragma unroll
            for (uint32_t g = 0; g < kRG; ++g) scale[g] = *reinterpret_cast<const float*>(t + scale_at[g]);
#pragma unroll
            for (uint32_t g = 0; g < kRG; ++g)
#pragma unroll
                for (uint32_t h = 0; h < 2; ++h)
#pragma unroll
                    for (uint32_t i = 0; i < 4; ++i) {
                        const uint32_t at = kCopies == 32 ? __builtin_amdgcn_perm(code[g][h], mine, 0x0C0C0000u | (4 + i) << 8)
                                                          : (code[g][h] >> (8 * i) & 255u) * (kCopies * 8) | mine;
                        w[g][h][i] = *reinterpret_cast<const v2f_t*>(memory + at);
                    }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (uint32_t h = 0; h < 2; ++h) {  // 32 of the block's 64 columns: 8 of each lane
                v8bf_t x[kFM];
#pragma unroll
                for (uint32_t f = 0; f < kFM; ++f)
                    x[f] = *reinterpret_cast<const v8bf_t*>(t + x_at[h] + f * 16 * kXChunks * 16);
#pragma unroll
                for (uint32_t g = 0; g < kRG; ++g) {
                    v8bf_t b;
#pragma unroll
                    for (uint32_t i = 0; i < 4; ++i) {
                        b[2 * i] = static_cast<__bf16>(w[g][h][i].x * scale[g]);
                        b[2 * i + 1] = static_cast<__bf16>(w[g][h][i].y * scale[g]);
                    }
#pragma unroll
                    for (uint32_t f = 0; f < kFM; ++f)
                        acc[g][f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, x[f], acc[g][f], 0, 0, 0);
                }
            }
        }
    }

    // the waves' sums, joined in the order of their blocks
    lds_barrier();  // the last stage is read
    constexpr uint32_t kTiles = kRowWaves * kRG * kFM;
    v4f_t* room = reinterpret_cast<v4f_t*>(memory);  // [kKWaves][kTiles][64]
#pragma unroll
    for (uint32_t g = 0; g < kRG; ++g)
#pragma unroll
        for (uint32_t f = 0; f < kFM; ++f) room[(q * kTiles + (rw * kRG + g) * kFM + f) * 64 + l] = acc[g][f];
    lds_barrier();
    NF4MatmulArgs o;
    o.c = a.c;
    o.ldc = a.ldc;
    o.partial = a.partial;
    o.m = a.m;
    o.n = a.n;
    const bool whole = whole_groups<kWideOut>(o);
    for (uint32_t t = wave; t < kTiles; t += kThinWaves) {
        v4f_t sum = room[t * 64 + l];
#pragma unroll
        for (uint32_t w = 1; w < kKWaves; ++w) sum += room[(w * kTiles + t) * 64 + l];
        if constexpr (kF) sum *= 1.0f / kThinScale;
        const uint32_t row = m0 + t % kFM * 16 + fr, column = n0 + t / kFM * 16 + fg * 4;
        if ((kXRows < 16 && fr >= kXRows) || row >= a.m || column >= a.n) continue;
        if (a.splits == 1)
            store4<kWideOut>(o, whole, row, column, sum);
        else
            *reinterpret_cast<MEZO_GLOBAL v4f_t*>(partial_at(o, blockIdx.y, row, column)) = sum;
    }
}

// ---- few rows, and blocks that run over the ends of the weights' -------------------------

// Where k is no multiple of 64 a row begins anywhere in a block, or within a byte. A workgroup
// takes kRG groups of 16 rows of weights, its waves every kRaggedWaves-th 64 columns of them. A lane
// has 16 weights next to each other, as above: of its row's three words of codes it shifts out two,
// by the same shift in every stage, since 64 columns are whole words; the weights before and behind
// the end of a block are the same ones in every stage too, so that it takes two scales and selects.
// A code's value comes from the lane that holds it. Codes and scales are read a stage ahead, straight
// into registers: rows lie on no alignment. (Loads into LDS would go from the 16 bytes that a row
// begins in, a chunk more a row, and the shift would be one of LDS reads; not built.)
// What bounds it is the number of those loads, each of 16 rows, and of the activations' (1 x 16384
// x 4100 bf16 26 us, 16 rows 31, 64 rows 53, in fp32 33, 45 and 130; expanded and through tiles 69,
// 69, 72 and 220, 221, 250). So both scales are one load; with a load each it took 31, 36 and 58 us,
// and then values by pairs out of LDS took as long, 64 weights a lane 28, 37 and 89, groups of 16
// rows alone 33, 41 and 83.
constexpr uint32_t kRaggedWaves = 8;

struct NF4RaggedArgs {
    uint64_t x, x_plane, x_row;  // laid out in planes, zeros behind column k
    uint64_t codes, absmax, c, ldc, partial;
    uint64_t k;
    uint32_t m, n, splits;
};

template <bool kF, uint32_t kRG, uint32_t kFM, bool kWideOut>
__global__ void __launch_bounds__(kRaggedWaves * 64) nf4_ragged_kernel(NF4RaggedArgs a)
{
    __shared__ v4f_t room[kRaggedWaves][kRG * kFM][64];
    const uint32_t l = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t fr = l & 15u, fg = l >> 4, n0 = blockIdx.x * kRG * 16, m0 = blockIdx.z * kFM * 16;
    uint32_t table = 0;
#pragma unroll
    for (uint32_t i = 0; i < kNF4Codes; ++i) table = fr == i ? __builtin_bit_cast(uint32_t, kNF4Values[i]) : table;
    const uint32_t stages = uint32_t((a.k + 63) / 64);
    const uint32_t s0 = uint32_t(uint64_t(stages) * blockIdx.y / a.splits),
                   s1 = uint32_t(uint64_t(stages) * (blockIdx.y + 1) / a.splits);

    // this lane's first weights of stage 0, rows past the end: the last one's
    const uint64_t all = a.n * a.k, words = (all + 1) / 2 / 4, top = (all - 1) / kNF4Block;
    // (bytes from the workgroup's first row: 32 rows of up to 2^23 weights)
    const uint64_t first = n0 * a.k, code0 = a.codes + first / 8 * 4, scale0 = a.absmax + first / kNF4Block * 4;
    uint64_t e0[kRG];
    uint32_t shift[kRG], left[kRG], code_at[kRG], scale_at[kRG];
#pragma unroll
    for (uint32_t g = 0; g < kRG; ++g) {
        const uint32_t row = n0 + g * 16 + fr;
        e0[g] = (row < a.n ? row : a.n - 1) * a.k + 16 * fg;
        shift[g] = uint32_t(e0[g] & 7u) * 4;
        left[g] = kNF4Block - uint32_t(e0[g] % kNF4Block);
        code_at[g] = uint32_t(e0[g] / 8 - first / 8) * 4;
        scale_at[g] = uint32_t(e0[g] / kNF4Block - first / kNF4Block) * 4;
    }
    // the stages whose three words are whole words of the codes and whose blocks have a next one,
    // by all lanes
    const uint32_t last_row = n0 + kRG * 16 - 1 < a.n ? n0 + kRG * 16 - 1 : a.n - 1;
    const uint64_t furthest = last_row * a.k + 48, word = furthest / 8 + 3, block = furthest / kNF4Block + 1;
    uint64_t most = words < word || top < block ? 0 : (words - word) / 8 + 1;
    if (most > top - block + 1) most = top - block + 1;
    const uint32_t safe = most < stages ? uint32_t(most) : stages;

    struct Codes {
        uint32_t w[3];
        float scale[2];
    };
    auto fetch = [&](uint32_t g, uint32_t s) {
        Codes c;
        const uint64_t from = code0 + uint64_t(s) * 32, scales = scale0 + uint64_t(s) * 4;
#pragma unroll
        for (uint32_t i = 0; i < 3; ++i) c.w[i] = *reinterpret_cast<const gu32_t*>(from + code_at[g] + 4 * i);
#pragma unroll
        for (uint32_t i = 0; i < 2; ++i) c.scale[i] = reinterpret_cast<const gfloat_t*>(scales + scale_at[g])[i];
        return c;
    };
    auto fetch_last = [&](uint32_t g, uint32_t s) {
        Codes c;
        const uint64_t e = e0[g] + uint64_t(s) * 64, b = e / kNF4Block, at = e & ~uint64_t(7);
        c.w[0] = eight_codes(a.codes, at, all);
        c.w[1] = eight_codes(a.codes, at + 8, all);
        c.w[2] = eight_codes(a.codes, at + 16, all);
        const gfloat_t* scales = reinterpret_cast<const gfloat_t*>(a.absmax);
        c.scale[0] = scales[b < top ? b : top];
        c.scale[1] = scales[left[g] >= 16 || b >= top ? (b < top ? b : top) : b + 1];
        return c;
    };

    uint32_t x_at[kFM];  // (up to 64 rows of 2^24 bytes)
#pragma unroll
    for (uint32_t f = 0; f < kFM; ++f) {
        const uint32_t r = m0 + f * 16 + fr;
        x_at[f] = (r < a.m ? r : a.m - 1) * uint32_t(a.x_row) + fg * 32;
    }
    constexpr uint32_t kPlanes = kF ? 3 : 1;
    v4f_t acc[kRG][kFM] = {};
    struct Activations {
        v8bf_t x[kFM][2][kPlanes];
    };
    auto activations = [&](uint32_t s) {
        Activations o;
#pragma unroll
        for (uint32_t f = 0; f < kFM; ++f)
#pragma unroll
            for (uint32_t h = 0; h < 2; ++h)
#pragma unroll
                for (uint32_t p = 0; p < kPlanes; ++p)
                    o.x[f][h][p] = *reinterpret_cast<const MEZO_GLOBAL v8bf_t*>(a.x + p * a.x_plane + uint64_t(s) * 128 + x_at[f] + h * 16);
        return o;
    };
    auto step = [&](uint32_t s, const Codes (&now)[kRG], const Activations& in) {
        const auto& x = in.x;
        const uint64_t column = uint64_t(s) * 64 + 16 * fg;
        const uint32_t valid = column >= a.k ? 0u : (a.k - column < 16 ? uint32_t(a.k - column) : 16u);
#pragma unroll
        for (uint32_t g = 0; g < kRG; ++g) {
            const uint32_t codes[2] = {__builtin_amdgcn_alignbit(now[g].w[1], now[g].w[0], shift[g]),
                                       __builtin_amdgcn_alignbit(now[g].w[2], now[g].w[1], shift[g])};
            float w[16];
#pragma unroll
            for (uint32_t i = 0; i < 16; ++i)
                // (the lane by bits 2 to 7: of four lanes that hold a value any will do)
                w[i] = __uint_as_float(uint32_t(__builtin_amdgcn_ds_bpermute(
                    int(i % 8 ? codes[i / 8] >> (4 * (i % 8) - 2) : codes[i / 8] << 2), int(table))));
#pragma unroll
            for (uint32_t i = 0; i < 16; ++i) w[i] *= i < left[g] ? now[g].scale[0] : now[g].scale[1];
            if (s + 1 == stages) {  // (what follows the row is not its own, and may not be finite)
#pragma unroll
                for (uint32_t i = 0; i < 16; ++i) w[i] = i < valid ? w[i] : 0.0f;
            }
#pragma unroll
            for (uint32_t h = 0; h < 2; ++h) {
                if constexpr (kF) {
                    const float v[8] = {w[8 * h], w[8 * h + 1], w[8 * h + 2], w[8 * h + 3], w[8 * h + 4], w[8 * h + 5],
                                        w[8 * h + 6], w[8 * h + 7]};
                    const Planes p = planes_of<true>(v);
#pragma unroll
                    for (uint32_t f = 0; f < kFM; ++f)
                        acc[g][f] = product(p, Planes{{x[f][h][0], x[f][h][1], x[f][h][2]}}, acc[g][f]);
                } else {
                    v8bf_t b;
#pragma unroll
                    for (uint32_t i = 0; i < 8; ++i) b[i] = static_cast<__bf16>(w[8 * h + i]);
#pragma unroll
                    for (uint32_t f = 0; f < kFM; ++f)
                        acc[g][f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, x[f][h][0], acc[g][f], 0, 0, 0);
                }
            }
        }
    };
    // The stages whose words are all there, then the others, by code of their own: where the two
    // ways to read meet, the compiler waits for the loads.
    Codes now[kRG], next[kRG] = {};
    const uint32_t end = s1 < safe ? s1 : safe;
    uint32_t s = s0 + wave;
    if (s < end)
#pragma unroll
        for (uint32_t g = 0; g < kRG; ++g) next[g] = fetch(g, s);
    for (; s < end; s += kRaggedWaves) {
#pragma unroll
        for (uint32_t g = 0; g < kRG; ++g) now[g] = next[g];
        const Activations x = activations(s);
        if (s + kRaggedWaves < end)
#pragma unroll
            for (uint32_t g = 0; g < kRG; ++g) next[g] = fetch(g, s + kRaggedWaves);
        step(s, now, x);
    }
    for (; s < s1; s += kRaggedWaves) {
#pragma unroll
        for (uint32_t g = 0; g < kRG; ++g) now[g] = fetch_last(g, s);
        step(s, now, activations(s));
    }

    // the waves' sums, joined in their order
#pragma unroll
    for (uint32_t t = 0; t < kRG * kFM; ++t) room[wave][t][l] = acc[t / kFM][t % kFM];
    __syncthreads();
    NF4MatmulArgs o;
    o.c = a.c;
    o.ldc = a.ldc;
    o.partial = a.partial;
    o.m = a.m;
    o.n = a.n;
    const bool whole = whole_groups<kWideOut>(o);
    for (uint32_t t = wave; t < kRG * kFM; t += kRaggedWaves) {
        v4f_t sum = room[0][t][l];
#pragma unroll
        for (uint32_t w = 1; w < kRaggedWaves; ++w) sum += room[w][t][l];
        const uint32_t out = m0 + t % kFM * 16 + fr, column = n0 + t / kFM * 16 + fg * 4;
        if (out >= a.m || column >= a.n) continue;
        if (a.splits == 1)
            store4<kWideOut>(o, whole, out, column, sum);
        else
            *reinterpret_cast<MEZO_GLOBAL v4f_t*>(partial_at(o, blockIdx.y, out, column)) = sum;
    }
}

// ---- launches ---------------------------------------------------------------------

template <class Args>
hipError_t run(const void* f, dim3 grid, uint32_t lanes, Args& a, hipStream_t stream)
{
    void* params[] = {&a};
    return hipLaunchKernel(f, grid, dim3(lanes), params, 0, stream);
}

template <bool kWideOut>
hipError_t join(NF4MatmulArgs& a, hipStream_t stream)
{
    constexpr uint64_t kBytes = kWideOut ? 4 : 2;
    const bool whole = ((a.c | (a.ldc * kBytes)) & (4 * kBytes - 1)) == 0;
    const uint64_t lanes = a.m * uint64_t(whole ? (a.n + 3) / 4 : a.n);
    return run(whole ? reinterpret_cast<const void*>(nf4_join_kernel<kWideOut>)
                     : reinterpret_cast<const void*>(nf4_join_columns_kernel<kWideOut>),
               dim3(uint32_t((lanes + 255) / 256)), 256, a, stream);
}

template <bool kWide, bool kWideOut>
hipError_t launch_tiled(const NF4LinearArgs& a, const NF4Cut& cut, hipStream_t stream)
{
    const uint64_t columns = nf4_columns(a.k), row = columns * 2;
    const NF4Space space = nf4_space(a.m, a.n, a.k, kWide);
    // bf16 activations that lie as the loads want them are read where they are
    const bool direct = !kWide && columns == a.k && ((a.x | (a.ldx * 2)) & 15u) == 0 && a.ldx * 2 <= (1u << 24);
    LayArgs lay = {};
    lay.k = a.k;
    lay.columns = columns;
    if (!direct) {
        lay.from = a.x;
        lay.ld = a.ldx;
        lay.to = a.workspace;
        lay.plane = a.m * row;
        lay.rows = a.m;
        const hipError_t e = run(reinterpret_cast<const void*>(nf4_lay_values_kernel<kWide>),
                                 dim3(uint32_t((a.m * (columns / 8) + 255) / 256)), 256, lay, stream);
        if (e != hipSuccess) return e;
    }
    NF4MatmulArgs g = {};
    g.x = direct ? a.x : a.workspace;
    g.x_row = uint32_t(direct ? a.ldx * 2 : row);
    g.x_plane = a.m * row;
    g.w = a.workspace + space.weights;
    g.w_row = uint32_t(row);
    g.w_plane = cut.slab * row;
    g.ldc = a.ldc;
    g.partial = a.workspace + space.partial;
    g.m = uint32_t(a.m);
    g.stages = uint32_t(columns / 64);
    g.splits = cut.splits;
    lay.from = a.codes;
    lay.absmax = a.absmax;
    lay.to = g.w;
    lay.plane = g.w_plane;
    lay.last = a.n * a.k;
    for (uint64_t n0 = 0; n0 < a.n; n0 += cut.slab) {
        lay.rows = a.n - n0 < cut.slab ? a.n - n0 : cut.slab;
        lay.first = n0 * a.k;
        hipError_t e = run(a.k % 8 ? reinterpret_cast<const void*>(nf4_expand_kernel<kWide, false>)
                                   : reinterpret_cast<const void*>(nf4_expand_kernel<kWide, true>),
                           dim3(uint32_t((lay.rows * (columns / 8) + 256 * kExpandUnits - 1) / (256 * kExpandUnits))), 256, lay, stream);
        if (e != hipSuccess) return e;
        g.n = uint32_t(lay.rows);
        g.c = a.c + n0 * (kWideOut ? 4 : 2);
        auto go = [&](auto* f, uint64_t bm, uint64_t bn, uint32_t lanes) {
            return run(reinterpret_cast<const void*>(f), dim3(uint32_t(tiles_of(a.m, lay.rows, bm, bn)), cut.splits), lanes,
                       g, stream);
        };
        switch (cut.tile) {
        case k256x256: e = go(nf4_matmul_kernel<256, 256, 2, 4, kWide, kWideOut>, 256, 256, 512); break;
        case k128x128: e = go(nf4_matmul_kernel<128, 128, 2, 2, kWide, kWideOut>, 128, 128, 256); break;
        default: e = go(nf4_matmul_kernel<64, 64, 2, 2, kWide, kWideOut>, 64, 64, 256);
        }
        if (e != hipSuccess) return e;
        if (cut.splits > 1) {
            e = join<kWideOut>(g, stream);
            if (e != hipSuccess) return e;
        }
    }
    return hipSuccess;
}

template <bool kWide, bool kWideOut>
hipError_t launch_thin(const NF4LinearArgs& a, const NF4Cut& cut, hipStream_t stream)
{
    constexpr uint64_t kElement = kWide ? 4 : 2;
    const NF4Space space = nf4_space(a.m, a.n, a.k, kWide);
    NF4ThinArgs g = {};
    g.x = a.x;
    g.x_row = uint32_t(a.ldx * kElement);
    if (((a.x | (a.ldx * kElement)) & 15u) || a.ldx * kElement > (1u << 24)) {  // the loads want whole 16 bytes
        LayArgs lay = {};
        lay.from = a.x;
        lay.ld = a.ldx;
        lay.to = a.workspace;
        lay.rows = a.m;
        lay.k = lay.columns = a.k;
        const hipError_t e = run(reinterpret_cast<const void*>(nf4_copy_rows_kernel<kWide>),
                                 dim3(uint32_t((a.m * (a.k / 8) + 255) / 256)), 256, lay, stream);
        if (e != hipSuccess) return e;
        g.x = a.workspace;
        g.x_row = uint32_t(a.k * kElement);
    }
    g.codes = a.codes;
    g.absmax = a.absmax;
    g.c = a.c;
    g.ldc = a.ldc;
    g.partial = a.workspace + space.partial;
    g.m = uint32_t(a.m);
    g.n = uint32_t(a.n);
    g.blocks = uint32_t(a.k / kNF4Block);
    g.splits = cut.splits;
    auto go = [&](auto* f, uint64_t rows, uint64_t x_rows) {
        return run(reinterpret_cast<const void*>(f),
                   dim3(uint32_t((a.n + rows - 1) / rows), cut.splits, uint32_t((a.m + x_rows - 1) / x_rows)),
                   kThinWaves * 64, g, stream);
    };
    hipError_t e = hipErrorInvalidValue;
    switch (cut.thin_rows) {
    case 16: e = go(nf4_thin_kernel<kWide, 1, 1, 4, kWide ? 3 : 4, 32, kWideOut>, 16, 4); break;
    case 128:
        if constexpr (kWide) {
            e = go(nf4_thin_kernel<true, 4, 2, 16, 2, 32, kWideOut>, 128, 16);
        } else {
            if (a.m <= 4)
                e = go(nf4_thin_kernel<false, 2, 4, 4, 2, 32, kWideOut>, 128, 4);
            else
                e = go(nf4_thin_kernel<false, 4, 2, 32, 2, 32, kWideOut>, 128, 32);
        }
        break;
    default:
        if (a.m <= 4)
            e = go(nf4_thin_kernel<kWide, 2, 2, 4, 3, 32, kWideOut>, 64, 4);
        else if (a.m <= 16 || kWide)
            e = go(nf4_thin_kernel<kWide, 4, 1, 16, kWide ? 3 : 4, 32, kWideOut>, 64, 16);
        else if constexpr (!kWide) {
            if (a.m <= 32)
                e = go(nf4_thin_kernel<false, 2, 2, 32, 2, 16, kWideOut>, 64, 32);
            else
                e = go(nf4_thin_kernel<false, 4, 1, 64, 2, 32, kWideOut>, 64, 64);
        }
    }
    if (e != hipSuccess || cut.splits == 1) return e;
    NF4MatmulArgs j = {};
    j.c = a.c;
    j.ldc = a.ldc;
    j.partial = g.partial;
    j.m = g.m;
    j.n = g.n;
    j.splits = cut.splits;
    return join<kWideOut>(j, stream);
}

template <bool kWide, bool kWideOut>
hipError_t launch_ragged(const NF4LinearArgs& a, const NF4Cut& cut, hipStream_t stream)
{
    const uint64_t columns = nf4_columns(a.k), row = columns * 2;
    LayArgs lay = {};
    lay.k = a.k;
    lay.columns = columns;
    lay.from = a.x;
    lay.ld = a.ldx;
    lay.to = a.workspace;
    lay.plane = a.m * row;
    lay.rows = a.m;
    hipError_t e = run(reinterpret_cast<const void*>(nf4_lay_values_kernel<kWide>),
                       dim3(uint32_t((a.m * (columns / 8) + 255) / 256)), 256, lay, stream);
    if (e != hipSuccess) return e;
    NF4RaggedArgs g = {};
    g.x = a.workspace;
    g.x_plane = a.m * row;
    g.x_row = row;
    g.codes = a.codes;
    g.absmax = a.absmax;
    g.c = a.c;
    g.ldc = a.ldc;
    g.partial = a.workspace + nf4_space(a.m, a.n, a.k, kWide).partial;
    g.k = a.k;
    g.m = uint32_t(a.m);
    g.n = uint32_t(a.n);
    g.splits = cut.splits;
    auto go = [&](auto* f, uint64_t rows, uint64_t x_rows) {
        return run(reinterpret_cast<const void*>(f),
                   dim3(uint32_t((a.n + rows - 1) / rows), cut.splits, uint32_t((a.m + x_rows - 1) / x_rows)), kRaggedWaves * 64, g,
                   stream);
    };
    auto by_groups = [&](auto groups) {
        constexpr uint32_t kRG = decltype(groups)::value;
        if (a.m <= 16) return go(nf4_ragged_kernel<kWide, kRG, 1, kWideOut>, 16 * kRG, 16);
        if constexpr (!kWide)
            if (a.m > 32) return go(nf4_ragged_kernel<kWide, kRG, 4, kWideOut>, 16 * kRG, 64);
        return go(nf4_ragged_kernel<kWide, kRG, 2, kWideOut>, 16 * kRG, 32);
    };
    // (32 rows share the activations' reads where that leaves a workgroup for every two CUs)
    e = a.n <= 4096 ? by_groups(std::integral_constant<uint32_t, 1>{}) : by_groups(std::integral_constant<uint32_t, 2>{});
    if (e != hipSuccess || cut.splits == 1) return e;
    NF4MatmulArgs j = {};
    j.c = a.c;
    j.ldc = a.ldc;
    j.partial = g.partial;
    j.m = g.m;
    j.n = g.n;
    j.splits = cut.splits;
    return join<kWideOut>(j, stream);
}

template <bool kWide, bool kWideOut>
hipError_t launch_any(const NF4LinearArgs& a, hipStream_t stream)
{
    const NF4Cut cut = cut_nf4(a.m, a.n, a.k, kWide);
    if (cut.tile == kThin && !cut.thin_rows) return launch_ragged<kWide, kWideOut>(a, cut, stream);
    return cut.tile == kThin ? launch_thin<kWide, kWideOut>(a, cut, stream) : launch_tiled<kWide, kWideOut>(a, cut, stream);
}

hipError_t launch_nf4_linear(const NF4LinearArgs& a, hipStream_t stream)
{
    if (a.x_dtype == kF32)
        return a.c_dtype == kF32 ? launch_any<true, true>(a, stream) : launch_any<true, false>(a, stream);
    return a.c_dtype == kF32 ? launch_any<false, true>(a, stream) : launch_any<false, false>(a, stream);
}

}  // namespace mezo
