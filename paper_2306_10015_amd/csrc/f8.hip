// f8.hip — 8-bit floating point storage and its product: what a forward pass
// over weights that were perturbed just before computes with.
//
// A row is stored in blocks of 128 elements, each e4m3 codes and one scale 2^e:
// the least power of two with max|w| <= 448 * 2^e. A power of two scales exactly,
// so a code is w rounded once, and it is what the matrix instructions take as a
// block's scale, so the product needs no multiply of its own for it:
//   c_mn = sum_b 2^(ex_mb + ew_nb) sum_{k in b} x_mk w_nk.
//
// Two arithmetics, chosen by the output's type:
//  bf16: v_mfma_scale_f32_16x16x128_f8f6f4. One instruction covers a block. Its
//        inner sum of 128 products keeps about 16 bits (2-norm error of a product
//        of normal rows 1.5e-5, with a few loud channels 5e-5, the same from 1 to
//        128 blocks; measured), far below bf16's own rounding of 1.7e-3.
//  fp32: the codes are widened to bf16 in registers, their scales applied, and
//        v_mfma_f32_16x16x32_bf16 sums the exact products in fp32 (error 1e-8 to
//        2e-7, as a chain of fp32 additions), at half the rate. Widening is exact
//        down to bf16's last bit, 2^-133: of blocks with scales below 2^-124, whose
//        largest value is below 2^-115, it rounds what lies under that.
#include <type_traits>

#include "f8_launch.hpp"
#include "lds_dma.hpp"
#include "records.hpp"
#include "stream_io.hpp"

namespace mezo {

typedef int v8i_t __attribute__((ext_vector_type(8)));
typedef float v4f_t __attribute__((ext_vector_type(4)));
typedef __bf16 v2bf_t __attribute__((ext_vector_type(2)));
typedef __bf16 v8bf_t __attribute__((ext_vector_type(8)));
typedef MEZO_GLOBAL uint8_t gu8_t;
typedef MEZO_GLOBAL uint32_t gu32_t;
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef MEZO_GLOBAL u32x2_t gu32x2_t;

// ---- quantization --------------------------------------------------------------
//
// Bound by memory (fp32: 5 bytes an element, bf16: 3) as long as its instructions are
// few: two bf16 matrices of 8192 x 16384 and 4096 x 16384 took 103 us at 14.6 vector
// instructions an element (94% of the cycles) and take 95 us, 6.3 TB/s, at 8.9 (61%). A
// lane takes 16 bytes of a row, so that loads and stores are whole lines; a block is 16
// (bf16) or 32 (fp32) lanes, which find its maximum by DPP, on the bits without the sign
// (which order as the values do), two bf16 at a time. The codes come from the
// instructions that divide by a block's scale as they convert. A lane starts kQuantLoads
// loads before it uses any.
constexpr uint32_t kQuantThreads = 256;
constexpr uint32_t kQuantLoads = 2;

typedef uint16_t u16x2_t __attribute__((ext_vector_type(2)));
typedef int16_t i16x2_t __attribute__((ext_vector_type(2)));

template <int kCtrl>
__device__ __forceinline__ uint32_t dpp_max(uint32_t x)
{
    const uint32_t y = uint32_t(__builtin_amdgcn_update_dpp(0, int(x), kCtrl, 0xF, 0xF, false));
    return x > y ? x : y;
}

// The maximum over the kLanes lanes of a block (16 or 32).
template <uint32_t kLanes>
__device__ __forceinline__ uint32_t max_block(uint32_t x)
{
    x = dpp_max<0xB1>(x);   // lanes 1 apart
    x = dpp_max<0x4E>(x);   // 2 apart
    x = dpp_max<0x141>(x);  // half a row mirrored
    x = dpp_max<0x140>(x);
    if constexpr (kLanes == 32) {
        const uint32_t y = uint32_t(__shfl_xor(int(x), 16));
        x = x > y ? x : y;
    }
    return x;
}

// 16 bytes of a row: its values, and the largest magnitude's bits (as of a float).
template <uint32_t kDtype>
struct Sixteen {
    static constexpr uint32_t kPer = kDtype == kF32 ? 4 : 8;
    uint32_t p[4];

    __device__ __forceinline__ float value(uint32_t j) const
    {
        if constexpr (kDtype == kF32) return __uint_as_float(p[j]);
        return __uint_as_float(j & 1 ? p[j / 2] & 0xFFFF0000u : p[j / 2] << 16);
    }
    __device__ __forceinline__ uint32_t largest() const
    {
        if constexpr (kDtype == kF32) {
            uint32_t m = 0;
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) m = m > (p[j] & 0x7FFFFFFFu) ? m : p[j] & 0x7FFFFFFFu;
            return m;
        } else {
            u16x2_t m = {0, 0};
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j)
                m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2_t, p[j] & 0x7FFF7FFFu));
            return uint32_t(m.x > m.y ? m.x : m.y) << 16;
        }
    }
    // The same of the finite values alone.
    __device__ __forceinline__ uint32_t largest_finite() const
    {
        uint32_t m = 0;
#pragma unroll
        for (uint32_t j = 0; j < kPer; ++j) {
            const uint32_t u = __float_as_uint(value(j)) & 0x7FFFFFFFu;
            if (u < 0x7F800000u && u > m) m = u;
        }
        return m;
    }
    // Codes of the values over 2^e.
    __device__ __forceinline__ void codes(int e, uint32_t (&code)[kPer / 4]) const
    {
        const float scale = __uint_as_float(uint32_t(e + 127) << 23);
#pragma unroll
        for (uint32_t j = 0; j < kPer / 4; ++j) {
            i16x2_t c = {0, 0};
            if constexpr (kDtype == kF32) {
                c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, value(4 * j), value(4 * j + 1), scale, false);
                c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, value(4 * j + 2), value(4 * j + 3), scale, true);
            } else {
                c = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c, __builtin_bit_cast(v2bf_t, p[2 * j]), scale, false);
                c = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c, __builtin_bit_cast(v2bf_t, p[2 * j + 1]), scale, true);
            }
            code[j] = __builtin_bit_cast(uint32_t, c);
        }
    }
    // The same step by step, for values that are not finite (coded NaN) and for e = -127,
    // which no float's exponent holds.
    __device__ __forceinline__ void codes_of_any(int e, uint32_t (&code)[kPer / 4]) const
    {
        const float inv = __uint_as_float(uint32_t(127 - e) << 23);
#pragma unroll
        for (uint32_t j = 0; j < kPer / 4; ++j) {
            int c = __builtin_amdgcn_cvt_pk_fp8_f32(value(4 * j) * inv, value(4 * j + 1) * inv, 0, false);
            c = __builtin_amdgcn_cvt_pk_fp8_f32(value(4 * j + 2) * inv, value(4 * j + 3) * inv, c, true);
            code[j] = uint32_t(c);
        }
    }
};

template <uint32_t kDtype, bool kAligned>
__global__ void __launch_bounds__(kQuantThreads) f8_quantize_kernel(F8QuantArgs a)
{
    using Values = Sixteen<kDtype>;
    constexpr uint32_t kBytes = kDtype == kF32 ? 4 : 2;
    constexpr uint32_t kPer = Values::kPer;       // elements of a lane
    constexpr uint32_t kLanes = kF8Block / kPer;  // lanes of a block
    constexpr uint32_t kUnits = kQuantThreads * kQuantLoads;
    const uint32_t blocks = uint32_t(f8_blocks(a.cols)), per_row = blocks * kLanes;
    // the workgroup's first unit (rows * blocks <= 2^27: 32 bits hold every unit)
    const uint32_t first = blockIdx.x * kUnits, row0 = first / per_row, rest = first - row0 * per_row;
    uint32_t row[kQuantLoads], col[kQuantLoads];  // col: the lane's first element
    Values w[kQuantLoads];
#pragma unroll
    for (uint32_t i = 0; i < kQuantLoads; ++i) {
        const uint32_t u = rest + i * kQuantThreads + threadIdx.x;
        if (per_row >= kUnits) {  // (uniform) the next row at most
            const bool next = u >= per_row;
            row[i] = row0 + (next ? 1 : 0);
            col[i] = (u - (next ? per_row : 0)) * kPer;
        } else {
            row[i] = row0 + u / per_row;
            col[i] = u % per_row * kPer;
        }
        if (row[i] >= a.rows) col[i] = a.cols + kPer;  // nothing to read
        const uint64_t at = a.values + (row[i] * a.ld + col[i]) * kBytes;
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) w[i].p[j] = 0;
        if (kAligned && col[i] + kPer <= a.cols) {
            const uint4 v = load_stream(at);
            w[i].p[0] = v.x;
            w[i].p[1] = v.y;
            w[i].p[2] = v.z;
            w[i].p[3] = v.w;
        } else {
#pragma unroll
            for (uint32_t j = 0; j < kPer; ++j)
                if (col[i] + j < a.cols) {
                    if constexpr (kDtype == kF32)
                        w[i].p[j] = reinterpret_cast<const gu32_t*>(at)[j];
                    else
                        w[i].p[j / 2] |= uint32_t(reinterpret_cast<const gu16_t*>(at)[j]) << (16 * (j & 1));
                }
        }
    }
#pragma unroll
    for (uint32_t i = 0; i < kQuantLoads; ++i) {
        uint32_t top = max_block<kLanes>(w[i].largest());
        const bool finite = !__any(top >= 0x7F800000u);  // of the wave
        if (!finite) top = max_block<kLanes>(w[i].largest_finite());
        // top = (1 + f) 2^x: e = x - 8, one more where 1 + f > 1.75 = 448 / 2^8
        int e = int(top >> 23) - 127 - 8 + ((top & 0x7FFFFFu) > 0x600000u ? 1 : 0);
        e = top == 0 ? 0 : (e < -127 ? -127 : e);
        uint32_t code[kPer / 4];
        if (finite && !__any(e == -127))
            w[i].codes(e, code);
        else
            w[i].codes_of_any(e, code);
        if (row[i] >= a.rows) continue;
        const uint32_t block = col[i] / kF8Block;
        const uint64_t at = a.codes + uint64_t(row[i]) * blocks * kF8Block + col[i];
        if constexpr (kPer == 8)
            *reinterpret_cast<gu32x2_t*>(at) = u32x2_t{code[0], code[1]};
        else
            *reinterpret_cast<gu32_t*>(at) = code[0];
        // the block's scale, and after the last one's the row's padding
        const uint32_t lane = col[i] % kF8Block / kPer;
        if (lane < 4) {
            const uint32_t stride = uint32_t(f8_scale_stride(a.cols));
            gu8_t* s = reinterpret_cast<gu8_t*>(a.scales) + uint64_t(row[i]) * stride;
            if (lane == 0) s[block] = uint8_t(e + 127);
            if (block == blocks - 1 && lane > 0 && block + lane < stride) s[block + lane] = 0;
        }
    }
}

hipError_t launch_f8_quantize(const F8QuantArgs& args, hipStream_t stream)
{
    const uint32_t bytes = args.dtype == kF32 ? 4 : 2;
    const bool aligned = ((args.values | (args.ld * bytes)) & 15u) == 0;
    const uint64_t units = uint64_t(args.rows) * f8_blocks(args.cols) * (kF8Block * bytes / 16);
    const uint64_t per = kQuantThreads * kQuantLoads;
    F8QuantArgs a = args;
    void* params[] = {&a};
    const void* f;
    if (args.dtype == kF32)
        f = aligned ? reinterpret_cast<const void*>(f8_quantize_kernel<kF32, true>)
                    : reinterpret_cast<const void*>(f8_quantize_kernel<kF32, false>);
    else
        f = aligned ? reinterpret_cast<const void*>(f8_quantize_kernel<kBF16, true>)
                    : reinterpret_cast<const void*>(f8_quantize_kernel<kBF16, false>);
    return hipLaunchKernel(f, dim3(uint32_t((units + per - 1) / per)), dim3(kQuantThreads), params, 0, stream);
}

// ---- the product ----------------------------------------------------------------

// A lane's 32 codes of a row's block, ready for the matrix instructions. Which 32
// of the 128 a lane holds does not matter as long as both operands agree: a block
// has one scale and the sum over it has no order.
template <bool kWide>
struct Operand;

template <>
struct Operand<false> {
    v8i_t v;
    int scale;  // the biased exponent in the low byte
    __device__ __forceinline__ void set(uint4 lo, uint4 hi, uint32_t s)
    {
        v = v8i_t{int(lo.x), int(lo.y), int(lo.z), int(lo.w), int(hi.x), int(hi.y), int(hi.z), int(hi.w)};
        scale = int(s);
    }
};

template <>
struct Operand<true> {
    v8bf_t v[4];
    __device__ __forceinline__ void set(uint4 lo, uint4 hi, uint32_t s)
    {
        const float scale = __uint_as_float((s & 0xFFu) << 23);  // (the exponent is all the conversion reads)
        const uint32_t d[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const v2bf_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(d[2 * q + h], scale, false);
                const v2bf_t b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(d[2 * q + h], scale, true);
                v[q][4 * h] = a.x;
                v[q][4 * h + 1] = a.y;
                v[q][4 * h + 2] = b.x;
                v[q][4 * h + 3] = b.y;
            }
        }
    }
};

__device__ __forceinline__ v4f_t mma(const Operand<false>& a, const Operand<false>& b, v4f_t c)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a.v, b.v, c, 0, 0, 0, a.scale, 0, b.scale);
}

__device__ __forceinline__ v4f_t mma(const Operand<true>& a, const Operand<true>& b, v4f_t c)
{
#pragma unroll
    for (int q = 0; q < 4; ++q) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v[q], b.v[q], c, 0, 0, 0);
    return c;
}

typedef __bf16 v4bf_t __attribute__((ext_vector_type(4)));

// A lane's four results, columns col .. col + 3 of a row of c: fp32 if kWide, else
// bf16. `whole`: every group of four columns lies on 4 elements' alignment.
template <bool kWide>
__device__ __forceinline__ void store4(const F8MatmulArgs& a, bool whole, uint32_t row, uint32_t col, v4f_t v)
{
    const uint64_t e = row * a.ldc + col;
    if constexpr (kWide) {
        gfloat_t* p = reinterpret_cast<gfloat_t*>(a.c) + e;
        if (whole && col + 4 <= a.n) {
            *reinterpret_cast<MEZO_GLOBAL v4f_t*>(p) = v;
        } else {
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i)
                if (col + i < a.n) p[i] = v[i];
        }
    } else {
        const v4bf_t b = __builtin_convertvector(v, v4bf_t);
        MEZO_GLOBAL __bf16* p = reinterpret_cast<MEZO_GLOBAL __bf16*>(a.c) + e;
        if (whole && col + 4 <= a.n) {
            *reinterpret_cast<MEZO_GLOBAL v4bf_t*>(p) = b;
        } else {
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i)
                if (col + i < a.n) p[i] = b[i];
        }
    }
}

template <bool kWide>
__device__ __forceinline__ bool whole_groups(const F8MatmulArgs& a)
{
    constexpr uint64_t kBytes = kWide ? 4 : 2;
    return ((a.c | (a.ldc * kBytes)) & (4 * kBytes - 1)) == 0;
}

// Where a split of k leaves its sums: rows of whole groups of four columns.
__device__ __forceinline__ uint64_t partial_at(const F8MatmulArgs& a, uint32_t split, uint32_t row, uint32_t col)
{
    return a.partial + ((uint64_t(split) * a.m + row) * ((a.n + 3) / 4) + col / 4) * 16;
}

// A lane's four results of a tile: into c, or of a split product into its partials.
template <bool kWide>
__device__ __forceinline__ void store_result(const F8MatmulArgs& a, bool whole, uint32_t split, uint32_t row,
                                             uint32_t col, v4f_t v)
{
    if (a.splits == 1)
        store4<kWide>(a, whole, row, col, v);
    else if (col < a.n)
        *reinterpret_cast<MEZO_GLOBAL v4f_t*>(partial_at(a, split, row, col)) = v;
}

// Tiles of kBM activations x kBN weights, kWM x kWN waves. Weights are the matrix
// instruction's rows and activations its columns, so that a lane's four results
// lie next to each other in a row of c.
//
// A stage is one block of 128 of every row of the tile, loaded straight into LDS;
// two stages, one computed on while the other loads. A row's eight 16-byte chunks
// are stored at chunk ^ ((row / 2) & 7): the 16 rows of a fragment then spread over
// all 64 banks. The scales of four blocks are a word of a row; they come the same way,
// every fourth stage.
template <uint32_t kBM, uint32_t kBN, uint32_t kWM, uint32_t kWN, bool kWide>
__global__ void __launch_bounds__(kWM* kWN * 64) f8_matmul_kernel(F8MatmulArgs a)
{
    constexpr uint32_t kWaves = kWM * kWN, kRows = kBM + kBN;
    constexpr uint32_t kFM = kBM / kWM / 16, kFN = kBN / kWN / 16;  // fragments of a wave
    constexpr uint32_t kLoads = kRows / 8 / kWaves;                 // 8 rows a load
    static_assert(kRows % (8 * kWaves) == 0 && kRows <= kWaves * 64 && kBM % 64 == 0 && kBN % 64 == 0);
    __shared__ __attribute__((aligned(1024))) uint8_t lds[2][kRows * 128];
    __shared__ __attribute__((aligned(256))) uint32_t scales[2][kRows];

    const uint32_t l = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // workgroups go round the 8 XCDs: give each XCD a compact part of c (its L2 then
    // holds the rows its workgroups share), in groups of 8 tile rows
    const uint32_t tm = (a.m + kBM - 1) / kBM, tn = (a.n + kBN - 1) / kBN, tiles = tm * tn;
    const uint32_t xcd = blockIdx.x % 8, each = tiles / 8, rest = tiles % 8;
    const uint32_t id = blockIdx.x / 8 + xcd * each + (xcd < rest ? xcd : rest);
    const uint32_t band = id / (8 * tn), height = tm - band * 8 < 8 ? tm - band * 8 : 8;
    const uint32_t in = id - band * 8 * tn;
    const uint32_t m0 = (band * 8 + in % height) * kBM, n0 = in / height * kBN;

    // this workgroup's blocks of k: whole words of scales
    const uint32_t all = uint32_t(f8_blocks(a.k)), words4 = (all + 3) / 4;
    const uint32_t begin = words4 * blockIdx.y / a.splits * 4, end4 = words4 * (blockIdx.y + 1) / a.splits * 4;
    const uint32_t blocks = end4 < all ? end4 : all;
    const uint32_t stride = uint32_t(f8_code_stride(a.k)), sstride = uint32_t(f8_scale_stride(a.k));
    // a load is 8 rows of x or of w; rows past the end: the last one's again
    const uint64_t x0 = a.x + uint64_t(m0) * stride, w0 = a.w + uint64_t(n0) * stride;
    const uint32_t xlast = a.m - m0 - 1, wlast = a.n - n0 - 1;
    uint32_t src[kLoads];  // this lane's 16 bytes of each of its rows
#pragma unroll
    for (uint32_t i = 0; i < kLoads; ++i) {
        const uint32_t first = (wave * kLoads + i) * 8;
        const uint32_t r = first + (l >> 3) - (first < kBM ? 0 : kBM), last = first < kBM ? xlast : wlast;
        // (row / 2) & 7 of row first + l / 8 of the tile
        const uint32_t swizzle = (first / 2 + (l >> 4)) & 7u;
        src[i] = (r < last ? r : last) * stride + ((l & 7u) ^ swizzle) * 16;
    }
    // a word of scales a lane, 64 rows a wave (waves left over: the first rows' again)
    const uint32_t srow = wave * 64 % kRows;
    const uint64_t words = srow < kBM ? a.xs + uint64_t(m0) * sstride : a.ws + uint64_t(n0) * sstride;
    uint32_t word;
    {
        const uint32_t r = srow + l - (srow < kBM ? 0 : kBM), last = srow < kBM ? xlast : wlast;
        word = (r < last ? r : last) * sstride;
    }
    const uint32_t lds0 = lds_offset(&lds[0][0]) + wave * kLoads * 1024;
    const uint32_t sc0 = lds_offset(&scales[0][0]) + srow * 4;
    auto stage = [&](uint32_t kb) {
#pragma unroll
        for (uint32_t i = 0; i < kLoads; ++i)
            dma_to_lds(((wave * kLoads + i) * 8 < kBM ? x0 : w0) + uint64_t(kb) * 128, src[i],
                       lds0 + (kb & 1) * kRows * 128 + i * 1024);
    };
    auto scale_words = [&](uint32_t group) {
        dma_word_to_lds(words + uint64_t(group) * 4, word, sc0 + (group & 1) * kRows * 4);
    };

    const uint32_t fr = l & 15u, fg = l >> 4;
    const uint32_t wm = (wave / kWN) * kFM * 16, wn = (wave % kWN) * kFN * 16;
    v4f_t acc[kFM][kFN] = {};
    uint32_t sx[kFM], sw[kFN];  // the scales of four blocks
    struct Fragment {
        uint4 lo, hi;
    };
    scale_words(begin >> 2);
    stage(begin);
    for (uint32_t kb = begin; kb < blocks; ++kb) {
        dma_wait();
        lds_barrier();  // stage kb is there, and nobody reads the other one any more
        if (kb + 1 < blocks) stage(kb + 1);
        if ((kb & 3u) == 0) {
            const uint32_t* s = scales[(kb >> 2) & 1];
#pragma unroll
            for (uint32_t i = 0; i < kFM; ++i) sx[i] = s[wm + i * 16 + fr];
#pragma unroll
            for (uint32_t i = 0; i < kFN; ++i) sw[i] = s[kBM + wn + i * 16 + fr];
            if (kb + 4 < blocks) scale_words((kb >> 2) + 1);
        }
        const uint8_t* t = lds[kb & 1];
        const uint32_t shift = (kb & 3u) * 8;
        auto fragment = [&](uint32_t row) {
            const uint32_t r = row + fr;
            Fragment f;
            f.lo = *reinterpret_cast<const uint4*>(t + r * 128 + ((fg ^ (fr >> 1)) * 16));
            f.hi = *reinterpret_cast<const uint4*>(t + r * 128 + (((fg + 4) ^ (fr >> 1)) * 16));
            return f;
        };
        Operand<kWide> w[kFN];
        Fragment next = fragment(wm);
#pragma unroll
        for (uint32_t j = 0; j < kFN; ++j) {
            const Fragment f = fragment(kBM + wn + j * 16);
            w[j].set(f.lo, f.hi, sw[j] >> shift);
        }
#pragma unroll
        for (uint32_t i = 0; i < kFM; ++i) {
            const Fragment f = next;
            if (i + 1 < kFM) next = fragment(wm + (i + 1) * 16);
            Operand<kWide> x;
            x.set(f.lo, f.hi, sx[i] >> shift);
#pragma unroll
            for (uint32_t j = 0; j < kFN; ++j) acc[i][j] = mma(w[j], x, acc[i][j]);
        }
    }
    // Where rows of c do not lie on the alignment of four columns, a lane's results would go
    // out one by one, neighbouring lanes 4 columns apart: such a tile goes through LDS, each
    // wave's part through room of its own, and out with neighbouring lanes on neighbouring
    // columns (1237 x 8191 x 2050 to fp32: 70 -> 56 us).
    const bool whole = whole_groups<kWide>(a);
    if (whole || a.splits > 1) {
#pragma unroll
        for (uint32_t i = 0; i < kFM; ++i) {
            const uint32_t row = m0 + wm + i * 16 + fr;
            if (row < a.m) {
#pragma unroll
                for (uint32_t j = 0; j < kFN; ++j)
                    store_result<kWide>(a, whole, blockIdx.y, row, n0 + wn + j * 16 + fg * 4, acc[i][j]);
            }
        }
        return;
    }
    using Out = std::conditional_t<kWide, float, __bf16>;
    constexpr uint32_t kCols = kFN * 16, kPerChunk = 16 / sizeof(Out), kChunks = kCols / kPerChunk;
    static_assert(kWaves * kFM * 16 * kCols * sizeof(Out) <= sizeof(lds), "the tile fits");
    lds_barrier();  // the last stage is read
    Out* room = reinterpret_cast<Out*>(&lds[0][0]) + wave * kFM * 16 * kCols;
    // a row's 16-byte chunks at chunk ^ row, against bank conflicts
    auto at = [&](uint32_t row, uint32_t col) {
        return row * kCols + ((col / kPerChunk) ^ (row % kChunks)) * kPerChunk + col % kPerChunk;
    };
#pragma unroll
    for (uint32_t i = 0; i < kFM; ++i)
#pragma unroll
        for (uint32_t j = 0; j < kFN; ++j) {
            Out* p = room + at(i * 16 + fr, j * 16 + fg * 4);
            if constexpr (kWide)
                *reinterpret_cast<v4f_t*>(p) = acc[i][j];
            else
                *reinterpret_cast<v4bf_t*>(p) = __builtin_convertvector(acc[i][j], v4bf_t);
        }
    lds_wait();
    constexpr uint32_t kRowsOut = 64 / kCols;  // rows a wave stores at once
    const uint32_t col = l % kCols, n = n0 + wn + col;
    if (n >= a.n) return;
    MEZO_GLOBAL Out* c = reinterpret_cast<MEZO_GLOBAL Out*>(a.c) + n;
#pragma unroll 4
    for (uint32_t r = l / kCols; r < kFM * 16; r += kRowsOut) {
        const uint32_t row = m0 + wm + r;
        if (row < a.m) c[row * a.ldc] = room[at(r, col)];
    }
}

// A product of few activations, m <= 16 kFM: bound by the weights' bytes. A
// workgroup takes 64 weights' rows, a wave 16 of them, and a share of k. A stage is
// two blocks of every row (256 bytes, and the word that holds their scales), loaded
// straight into LDS, two stages ahead (one for m > 32), two workgroups a CU. Fragments loaded from global memory straight
// into registers would need neither LDS nor barriers, but there neighbouring lanes
// read different rows, and the address units take such a load apart line by line:
// 25 us for 24 activations and 16384 x 4096 weights, as slow with all weights in L2.
constexpr uint32_t kThinBlocks = 2, kThinBytes = kThinBlocks * 128;

template <uint32_t kFM, bool kWide>
__global__ void __launch_bounds__(256) f8_thin_kernel(F8MatmulArgs a)
{
    constexpr uint32_t kX = kFM * 16, kRows = kThinRows + kX, kStage = kRows * kThinBytes;
    constexpr uint32_t kDepth = kFM == 4 ? 2 : 3;
    constexpr uint32_t kLoadRows = 1024 / kThinBytes, kChunks = kThinBytes / 16;
    constexpr uint32_t kWLoads = kThinRows / kLoadRows / 4, kXLoads = kX / kLoadRows / 4;  // a wave's
    constexpr uint32_t kPerStage = kWLoads + kXLoads + 1;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[kDepth][kStage];
    __shared__ __attribute__((aligned(256))) uint32_t scales[kDepth][kThinRows + 64];

    const uint32_t l = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t n0 = blockIdx.x * kThinRows;
    const uint32_t blocks = uint32_t(f8_blocks(a.k)), stages = (blocks + kThinBlocks - 1) / kThinBlocks;
    const uint32_t s0 = stages * blockIdx.y / a.splits, s1 = stages * (blockIdx.y + 1) / a.splits;
    const uint32_t stride = uint32_t(f8_code_stride(a.k)), sstride = uint32_t(f8_scale_stride(a.k));
    const uint64_t w0 = a.w + uint64_t(n0) * stride, ws0 = a.ws + uint64_t(n0) * sstride;
    const uint32_t wend = a.n - n0 - 1, xend = a.m - 1;
    // wave 0 loads x's scales, the others w's (three times the same)
    const uint64_t words = wave == 0 ? a.xs : ws0;
    const uint32_t word = (l < (wave == 0 ? xend : wend) ? l : (wave == 0 ? xend : wend)) * sstride;
    const uint32_t lds0 = lds_offset(&lds[0][0]);
    const uint32_t sc0 = lds_offset(&scales[0][0]) + (wave == 0 ? kThinRows * 4 : 0);
    auto load = [&](uint32_t s, uint32_t buffer) {
        // past the row's end (its blocks are no multiple of four): its last bytes again
        const uint32_t col0 = s * kThinBytes + l % kChunks * 16, last = stride - 16;
#pragma unroll
        for (uint32_t i = 0; i < kWLoads + kXLoads; ++i) {
            const bool ofw = i < kWLoads;
            const uint32_t at = ofw ? wave * kWLoads + i : wave * kXLoads + i - kWLoads;
            const uint32_t r = at * kLoadRows + l / kChunks;
            const uint32_t end = ofw ? wend : xend, col = col0 ^ ((r & 15u) * 16);
            dma_to_lds(ofw ? w0 : a.x, (r < end ? r : end) * stride + (col < last ? col : last),
                       lds0 + buffer * kStage + ((ofw ? 0 : kThinRows / kLoadRows) + at) * 1024);
        }
        dma_word_to_lds(words + uint64_t(s * kThinBlocks / 4) * 4, word, sc0 + buffer * (kThinRows + 64) * 4);
    };
    const uint32_t fr = l & 15u, fg = l >> 4;
    v4f_t acc[kFM] = {};
    uint32_t ahead = s0;
    for (uint32_t d = 0; d + 1 < kDepth && ahead < s1; ++d, ++ahead) load(ahead, (ahead - s0) % kDepth);
    for (uint32_t s = s0; s < s1; ++s) {
        // stage s is there (all that is in flight after it: whole stages), and the one
        // before it is read by all
        if (ahead - s == kDepth - 1)
            dma_wait<(kDepth - 2) * kPerStage>();
        else
            dma_wait();
        lds_barrier();
        if (ahead < s1) {
            load(ahead, (ahead - s0) % kDepth);
            ++ahead;
        }
        const uint32_t buffer = (s - s0) % kDepth;
        const uint8_t* t = lds[buffer];
        const uint32_t sw = scales[buffer][wave * 16 + fr];
        uint32_t sx[kFM];
#pragma unroll
        for (uint32_t i = 0; i < kFM; ++i) sx[i] = scales[buffer][kThinRows + i * 16 + fr];
        const uint32_t n = blocks - s * kThinBlocks;
#pragma unroll
        for (uint32_t d = 0; d < kThinBlocks; ++d) {
            if (d >= n) break;
            auto fragment = [&](uint32_t row, uint32_t scale) {
                const uint8_t* p = t + (row + fr) * kThinBytes;  // chunks at chunk ^ (row & 15)
                Operand<kWide> o;
                o.set(*reinterpret_cast<const uint4*>(p + (((8 * d + fg) ^ fr) * 16)),
                      *reinterpret_cast<const uint4*>(p + (((8 * d + fg + 4) ^ fr) * 16)),
                      scale >> (8 * ((s * kThinBlocks + d) & 3u)));
                return o;
            };
            const Operand<kWide> w = fragment(wave * 16, sw);
#pragma unroll
            for (uint32_t i = 0; i < kFM; ++i)
                acc[i] = mma(w, fragment(kThinRows + i * 16, sx[i]), acc[i]);
        }
    }
    const bool whole = whole_groups<kWide>(a);
#pragma unroll
    for (uint32_t i = 0; i < kFM; ++i) {
        const uint32_t row = i * 16 + fr, col = n0 + wave * 16 + fg * 4;
        if (row < a.m) store_result<kWide>(a, whole, blockIdx.y, row, col, acc[i]);
    }
}

// The sums of a product whose k was split, joined in the order of the splits.
template <bool kWide>
__global__ void __launch_bounds__(256) f8_join_kernel(F8MatmulArgs a)
{
    const uint32_t groups = (a.n + 3) / 4;
    const uint64_t i = uint64_t(blockIdx.x) * 256 + threadIdx.x;
    if (i >= uint64_t(a.m) * groups) return;
    const uint32_t row = uint32_t(i / groups), col = uint32_t(i % groups) * 4;
    v4f_t sum = {};
    for (uint32_t s = 0; s < a.splits; ++s)
        sum += *reinterpret_cast<const MEZO_GLOBAL v4f_t*>(partial_at(a, s, row, col));
    store4<kWide>(a, whole_groups<kWide>(a), row, col, sum);
}

template <bool kWide>
hipError_t launch_product(F8MatmulArgs a, hipStream_t stream)
{
    const F8Cut cut = cut_product(a.m, a.n, a.k, kWide);
    a.splits = cut.splits;
    void* params[] = {&a};
    auto go = [&](auto* f, uint64_t bm, uint64_t bn, uint32_t lanes) {
        const dim3 groups(uint32_t(tiles_of(a.m, a.n, bm, bn)), a.splits);
        return hipLaunchKernel(reinterpret_cast<const void*>(f), groups, dim3(lanes), params, 0, stream);
    };
    hipError_t e = hipErrorInvalidValue;
    switch (cut.tile) {
    case kThin:
        if (a.m <= 16)
            e = go(f8_thin_kernel<1, kWide>, 64, kThinRows, 256);
        else if (a.m <= 32)
            e = go(f8_thin_kernel<2, kWide>, 64, kThinRows, 256);
        else
            e = go(f8_thin_kernel<4, kWide>, 64, kThinRows, 256);
        break;
    case k64x64: e = go(f8_matmul_kernel<64, 64, 2, 2, kWide>, 64, 64, 256); break;
    case k128x128: e = go(f8_matmul_kernel<128, 128, 2, 2, kWide>, 128, 128, 256); break;
    case k256x256:
        if constexpr (!kWide) e = go(f8_matmul_kernel<256, 256, 2, 4, false>, 256, 256, 512);
        break;
    }
    if (e != hipSuccess || a.splits == 1) return e;
    const uint64_t groups = uint64_t(a.m) * ((a.n + 3) / 4);
    return hipLaunchKernel(reinterpret_cast<const void*>(f8_join_kernel<kWide>), dim3(uint32_t((groups + 255) / 256)),
                           dim3(256), params, 0, stream);
}

hipError_t launch_f8_matmul(const F8MatmulArgs& args, hipStream_t stream)
{
    return args.out_dtype == kF32 ? launch_product<true>(args, stream) : launch_product<false>(args, stream);
}

}  // namespace mezo
