// cache_append.hip — the keys and values of new tokens into the pages of a cache, turned by
// their positions on the way; the same tokens' queries turned with them. Token i of a
// document with nq new ones of nk stands at place r = nk - nq + i, which is row r % R of the
// page that entry r / R of its list names, and its position is r unless positions are given:
//   (x_a, x_b) -> (x_a cos t - x_b sin t, x_a sin t + x_b cos t),  t = position * freqs[j],
// for pair j of a head's first `rot` columns: (j, j + rot / 2), or (2j, 2j + 1) where
// interleaved. The other columns and the values are copied.
//
// The angle is a product of up to 2^31 and a float: in fp32 it would be off by 2^-24 of
// itself, 1e-3 after 16384 radians. It is formed in fp64, brought to half a turn there, and
// sine and cosine are taken of that in fp32, once a token and pair: all heads read them from
// LDS. Turned values are computed in fp32 and rounded once.
//
// Bound by memory: each value is read and written once. A lane moves vectors of kW elements
// (16 bytes where half of `rot` is a multiple of them, which the usual sizes are; else the
// largest power of two that divides it): a vector of a pair's first columns and the one of
// their partners, or a vector of whole pairs. Neighbouring lanes take neighbouring vectors of
// a head, then heads, then tokens.
#include "cache_append_launch.hpp"
#include "records.hpp"
#include "stream_io.hpp"

namespace mezo {

constexpr uint32_t kAppendThreads = 256;
constexpr uint32_t kMostAngles = 4096;  // of a workgroup, in LDS
constexpr uint32_t kMostTile = 64;      // tokens of a workgroup

template <uint32_t kBytes>
struct Bits;
template <>
struct Bits<2> {
    typedef uint16_t type;
};
template <>
struct Bits<4> {
    typedef uint32_t type;
};

// kW elements of fp32 or bf16.
template <bool kF, uint32_t kW>
struct Vector {
    typedef typename Bits<kF ? 4 : 2>::type element_t;
    typedef element_t type __attribute__((ext_vector_type(kW)));
    type v;

    __device__ __forceinline__ void load(uint64_t at) { v = *reinterpret_cast<const MEZO_GLOBAL type*>(at); }
    __device__ __forceinline__ void store(uint64_t at) const { *reinterpret_cast<MEZO_GLOBAL type*>(at) = v; }
    __device__ __forceinline__ float get(uint32_t i) const
    {
        if constexpr (kF) return __uint_as_float(v[i]);
        return __uint_as_float(uint32_t(v[i]) << 16);
    }
    __device__ __forceinline__ void set(uint32_t i, float x)
    {
        if constexpr (kF)
            v[i] = __float_as_uint(x);
        else
            v[i] = __builtin_bit_cast(uint16_t, static_cast<__bf16>(x));
    }
};

template <bool kF>
struct Vector<kF, 1> {
    typedef typename Bits<kF ? 4 : 2>::type type;
    type v;
    __device__ __forceinline__ void load(uint64_t at) { v = *reinterpret_cast<const MEZO_GLOBAL type*>(at); }
    __device__ __forceinline__ void store(uint64_t at) const { *reinterpret_cast<MEZO_GLOBAL type*>(at) = v; }
    __device__ __forceinline__ float get(uint32_t) const
    {
        if constexpr (kF) return __uint_as_float(v);
        return __uint_as_float(uint32_t(v) << 16);
    }
    __device__ __forceinline__ void set(uint32_t, float x)
    {
        if constexpr (kF)
            v = __float_as_uint(x);
        else
            v = __builtin_bit_cast(uint16_t, static_cast<__bf16>(x));
    }
};

// Where the tokens of a workgroup's tile go.
struct Slot {
    uint64_t k, v;  // their rows of the cache; 0: nowhere
};

// Lanes over (token, head, vector) of `count` vectors a head, in this order from the last:
// each lane keeps its vector and steps through the heads.
template <class F>
__device__ __forceinline__ void over_heads(uint32_t tokens, uint32_t heads, uint32_t count, F&& body)
{
    const uint32_t step = kAppendThreads / count, lane_head = threadIdx.x / count, c = threadIdx.x - lane_head * count;
    if (lane_head >= step) return;
    uint32_t h = lane_head, t = 0;
    while (h >= heads) {
        h -= heads;
        ++t;
    }
    while (t < tokens) {
        body(t, h, c);
        h += step;
        while (h >= heads) {
            h -= heads;
            ++t;
        }
    }
}

template <bool kF, uint32_t kW, bool kPairs>
__global__ void __launch_bounds__(kAppendThreads) cache_append_kernel(AppendArgs a)
{
    constexpr uint32_t kElement = kF ? 4 : 2;
    __shared__ float2 turn[kMostAngles];  // (cos, sin) of [token, pair]
    __shared__ Slot slots[kMostTile];

    const uint32_t tiles = (a.max_q + a.tile - 1) / a.tile, work = blockIdx.x / a.parts, part = blockIdx.x % a.parts;
    const uint32_t doc = work / tiles, first = (work % tiles) * a.tile;
    // the document's row of the table, cut to the arrays: no table makes the kernel leave them
    const MEZO_GLOBAL int64_t* row = reinterpret_cast<const MEZO_GLOBAL int64_t*>(a.table) + uint64_t(doc) * 5;
    auto within = [](int64_t x, uint64_t top) { return x < 0 ? 0 : (uint64_t(x) > top ? top : uint64_t(x)); };
    const uint64_t q_first = within(row[0], a.tokens), nq = within(row[1], a.tokens - q_first);
    const uint64_t entry = within(row[2], a.entries), nk = within(row[3], (a.entries - entry) << a.page_shift);
    const uint64_t some = nq < a.max_q ? nq : a.max_q;
    if (first >= some) return;
    const uint32_t tokens = some - first < a.tile ? uint32_t(some - first) : a.tile;
    const uint64_t token0 = q_first + first;
    const int64_t place0 = int64_t(nk) - int64_t(nq) + first;

    const uint32_t pairs = a.rot / 2;
    for (uint32_t i = threadIdx.x; i < tokens * pairs; i += kAppendThreads) {
        const uint32_t t = i / pairs, j = i - t * pairs;
        const int64_t position = a.positions ? reinterpret_cast<const MEZO_GLOBAL int64_t*>(a.positions)[token0 + t]
                                             : place0 + t;
        const double turns = double(position) * double(reinterpret_cast<const gfloat_t*>(a.freqs)[j]) *
                             0.15915494309189533577;  // 1 / (2 pi)
        float s, c;
        sincospif(float(2.0 * (turns - rint(turns))), &s, &c);
        turn[i] = make_float2(c, s);
    }
    if (threadIdx.x < tokens) {
        Slot s = {0, 0};
        const int64_t place = place0 + threadIdx.x;
        if (place >= 0) {
            const uint32_t page = reinterpret_cast<const MEZO_GLOBAL uint32_t*>(a.pages)[entry + (uint64_t(place) >> a.page_shift)];
            const uint64_t at = uint64_t(place) & ((1u << a.page_shift) - 1);
            if (page < a.n_pages) s = {a.k_cache + page * a.kc_page + at * a.kc_row, a.v_cache + page * a.vc_page + at * a.vc_row};
        }
        slots[threadIdx.x] = s;
    }
    __syncthreads();

    using V = Vector<kF, kW>;
    constexpr uint32_t kVector = kW * kElement;
    // this workgroup's heads
    const uint32_t h0 = a.heads * part / a.parts, heads = a.heads * (part + 1) / a.parts - h0;
    const uint32_t g0 = a.kv_heads * part / a.parts, kv_heads = a.kv_heads * (part + 1) / a.parts - g0;

    // one vector of a head that is turned, and the one of its partners, from `in` to `out`
    auto turned = [&](uint64_t in, uint64_t out, uint32_t t, uint32_t c) {
        const float2* cs = turn + t * pairs;
        if constexpr (kPairs) {
            V x;
            x.load(in + c * kVector);
            V y = x;
#pragma unroll
            for (uint32_t i = 0; i + 1 < kW; i += 2) {
                const float2 u = cs[(c * kW + i) / 2];
                const float p = x.get(i), q = x.get(i + 1);
                y.set(i, __builtin_fmaf(p, u.x, -(q * u.y)));
                y.set(i + 1, __builtin_fmaf(p, u.y, q * u.x));
            }
            y.store(out + c * kVector);
        } else {
            const uint32_t half = pairs * kElement;
            V x, y;
            x.load(in + c * kVector);
            y.load(in + half + c * kVector);
            V u = x, w = y;
#pragma unroll
            for (uint32_t i = 0; i < kW; ++i) {
                const float2 z = cs[c * kW + i];
                const float p = x.get(i), q = y.get(i);
                u.set(i, __builtin_fmaf(p, z.x, -(q * z.y)));
                w.set(i, __builtin_fmaf(p, z.y, q * z.x));
            }
            u.store(out + c * kVector);
            w.store(out + half + c * kVector);
        }
    };
    auto copied = [&](uint64_t in, uint64_t out) {
        V x;
        x.load(in);
        x.store(out);
    };
    const uint32_t turning = kPairs ? a.rot / kW : pairs / kW, rest = (a.dim - a.rot) / kW;
    if (a.q && heads) {
        const uint64_t in0 = a.q + token0 * a.q_token + h0 * a.q_head, out0 = a.q_out + token0 * a.o_token + h0 * a.o_head;
        if (turning)
            over_heads(tokens, heads, turning, [&](uint32_t t, uint32_t h, uint32_t c) {
                turned(in0 + t * a.q_token + h * a.q_head, out0 + t * a.o_token + h * a.o_head, t, c);
            });
        if (rest)
            over_heads(tokens, heads, rest, [&](uint32_t t, uint32_t h, uint32_t c) {
                const uint32_t at = a.rot * kElement + c * kVector;
                copied(in0 + t * a.q_token + h * a.q_head + at, out0 + t * a.o_token + h * a.o_head + at);
            });
    }
    if (!kv_heads) return;
    const uint64_t k0 = a.k + token0 * a.k_token + g0 * a.k_head, v0 = a.v + token0 * a.v_token + g0 * a.v_head;
    if (turning)
        over_heads(tokens, kv_heads, turning, [&](uint32_t t, uint32_t h, uint32_t c) {
            if (slots[t].k) turned(k0 + t * a.k_token + h * a.k_head, slots[t].k + (g0 + h) * a.kc_head, t, c);
        });
    if (rest)
        over_heads(tokens, kv_heads, rest, [&](uint32_t t, uint32_t h, uint32_t c) {
            const uint32_t at = a.rot * kElement + c * kVector;
            if (slots[t].k) copied(k0 + t * a.k_token + h * a.k_head + at, slots[t].k + (g0 + h) * a.kc_head + at);
        });
    over_heads(tokens, kv_heads, a.dim * kElement / 16, [&](uint32_t t, uint32_t h, uint32_t c) {
        if (!slots[t].v) return;
        Vector<kF, 16 / kElement> x;
        x.load(v0 + t * a.v_token + h * a.v_head + c * 16);
        x.store(slots[t].v + (g0 + h) * a.vc_head + c * 16);
    });
}

template <bool kF, uint32_t kW>
hipError_t launch(AppendArgs& a, hipStream_t stream)
{
    constexpr uint32_t kFull = kF ? 4 : 8;
    // the longest vectors that divide what is turned
    const uint32_t divides = a.interleaved ? a.rot : a.rot / 2;
    if constexpr (kW > 1)
        if (divides % kW != 0) return launch<kF, kW / 2>(a, stream);
    static_assert(kW <= kFull);
    const uint32_t pairs = a.rot / 2;
    // Tokens of a workgroup: about 32 KB of what is read, so that the angles' latency is a
    // small part, as long as that leaves work for all CUs; few tokens: their heads are shared out.
    const uint32_t bytes = (a.heads + 2 * a.kv_heads) * a.dim * (kF ? 4 : 2);
    uint32_t tile = bytes >= 32768 ? 1 : 32768 / bytes;
    tile = tile > kMostTile ? kMostTile : tile;
    if (pairs && tile > kMostAngles / pairs) tile = kMostAngles / pairs;
    const uint64_t tokens = uint64_t(a.docs) * a.max_q;
    while (tile > 1 && tokens / tile < 512) tile /= 2;
    a.tile = tile;
    const uint64_t groups = uint64_t(a.docs) * ((a.max_q + tile - 1) / tile);
    a.parts = groups >= 256 ? 1 : (groups >= 64 ? 2 : 4);
    if (a.parts > a.kv_heads) a.parts = a.kv_heads;
    void* params[] = {&a};
    const void* f;
    if constexpr (kW == 1)  // (pairs next to each other are even in number)
        f = reinterpret_cast<const void*>(cache_append_kernel<kF, 1, false>);
    else
        f = a.interleaved ? reinterpret_cast<const void*>(cache_append_kernel<kF, kW, true>)
                          : reinterpret_cast<const void*>(cache_append_kernel<kF, kW, false>);
    return hipLaunchKernel(f, dim3(uint32_t(groups * a.parts)), dim3(kAppendThreads), params, 0, stream);
}

hipError_t launch_cache_append(const AppendArgs& args, hipStream_t stream)
{
    AppendArgs a = args;
    return a.dtype == kF32 ? launch<true, 4>(a, stream) : launch<false, 8>(a, stream);
}

}  // namespace mezo
