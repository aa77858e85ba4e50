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
// a head, then heads, then tokens. Packed prompts on the 6.7B shapes, 842 MB read and written:
// 151 us, 5.6 TB/s (a copy of 1 GiB 5.2); 24 tokens of 32 heads on 8 of 128 take 8 us, one 5:
// the chain from the table to the list to the page's row.
#include <type_traits>

#include "cache_append_launch.hpp"
#include "records.hpp"
#include "stream_io.hpp"

namespace mezo {

constexpr uint32_t kAppendThreads = 256;
constexpr uint32_t kMostAngles = 1024;  // of a workgroup, in LDS (8 KB: eight workgroups a CU)
constexpr uint32_t kTileBytes = 32768;
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

    __device__ __forceinline__ void load(uint64_t at) { v = __builtin_nontemporal_load(reinterpret_cast<const MEZO_GLOBAL type*>(at)); }
    template <bool kStream>
    __device__ __forceinline__ void store(uint64_t at) const
    {
        if constexpr (kStream)
            __builtin_nontemporal_store(v, reinterpret_cast<MEZO_GLOBAL type*>(at));
        else
            *reinterpret_cast<MEZO_GLOBAL type*>(at) = v;
    }
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
    __device__ __forceinline__ void load(uint64_t at) { v = __builtin_nontemporal_load(reinterpret_cast<const MEZO_GLOBAL type*>(at)); }
    template <bool kStream>
    __device__ __forceinline__ void store(uint64_t at) const
    {
        if constexpr (kStream)
            __builtin_nontemporal_store(v, reinterpret_cast<MEZO_GLOBAL type*>(at));
        else
            *reinterpret_cast<MEZO_GLOBAL type*>(at) = v;
    }
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

// Lanes over (token, head, vector) of `count` vectors a head: each keeps its vector and steps
// through the heads, kAhead of them at a time, whose loads are all under way before the first
// is used.
constexpr uint32_t kAhead = 2;

template <class S, class L, class F>
__device__ __forceinline__ void over_heads(uint32_t tokens, uint32_t heads, uint32_t count, L&& load, F&& finish)
{
    const uint32_t step = kAppendThreads / count, lane_head = threadIdx.x / count, c = threadIdx.x - lane_head * count;
    if (lane_head >= step) return;
    uint32_t h = lane_head, t = 0;
    auto wrap = [&] {
        while (h >= heads) {
            h -= heads;
            ++t;
        }
    };
    wrap();
    while (t < tokens) {
        S s[kAhead];
        uint32_t st[kAhead], sh[kAhead];
#pragma unroll
        for (uint32_t u = 0; u < kAhead; ++u) {
            st[u] = t;
            sh[u] = h;
            if (t < tokens) load(s[u], t, h, c);
            h += step;
            wrap();
        }
#pragma unroll
        for (uint32_t u = 0; u < kAhead; ++u)
            if (st[u] < tokens) finish(s[u], st[u], sh[u], c);
    }
}

template <bool kF, uint32_t kW, bool kPairs, bool kStream>
__global__ void __launch_bounds__(kAppendThreads) cache_append_kernel(AppendArgs a)
{
    constexpr uint32_t kElement = kF ? 4 : 2;
    __shared__ float2 turn[kMostAngles];  // (cos, sin) of [token, pair]
    __shared__ Slot slots[kMostTile];

    const uint32_t id = blockIdx.y * gridDim.x + blockIdx.x, work = id / a.parts, part = id % a.parts;
    const uint32_t tiles = (a.max_q + a.tile - 1) / a.tile, doc = work / tiles, first = (work % tiles) * a.tile;
    if (doc >= a.docs) return;
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

    // a vector of a head that is turned, and the one of its partners
    struct Both {
        V x, y;
    };
    const uint32_t half = pairs * kElement;
    auto load = [&](Both& s, uint64_t in, uint32_t c) {
        s.x.load(in + c * kVector);
        if constexpr (!kPairs) s.y.load(in + half + c * kVector);
    };
    auto turned = [&](const Both& s, uint64_t out, uint32_t t, uint32_t c) {
        const float2* cs = turn + t * pairs;
        Both o = s;
        if constexpr (kPairs) {
#pragma unroll
            for (uint32_t i = 0; i + 1 < kW; i += 2) {
                const float2 u = cs[(c * kW + i) / 2];
                const float p = s.x.get(i), q = s.x.get(i + 1);
                o.x.set(i, __builtin_fmaf(p, u.x, -(q * u.y)));
                o.x.set(i + 1, __builtin_fmaf(p, u.y, q * u.x));
            }
            o.x.template store<kStream>(out + c * kVector);
        } else {
#pragma unroll
            for (uint32_t i = 0; i < kW; ++i) {
                const float2 z = cs[c * kW + i];
                const float p = s.x.get(i), q = s.y.get(i);
                o.x.set(i, __builtin_fmaf(p, z.x, -(q * z.y)));
                o.y.set(i, __builtin_fmaf(p, z.y, q * z.x));
            }
            o.x.template store<kStream>(out + c * kVector);
            o.y.template store<kStream>(out + half + c * kVector);
        }
    };
    const uint32_t turning = kPairs ? a.rot / kW : pairs / kW, rest = (a.dim - a.rot) / kW, rot = a.rot * kElement;
    if (a.q && heads) {
        const uint64_t in0 = a.q + token0 * a.q_token + h0 * a.q_head, out0 = a.q_out + token0 * a.o_token + h0 * a.o_head;
        if (turning)
            over_heads<Both>(
                tokens, heads, turning,
                [&](Both& s, uint32_t t, uint32_t h, uint32_t c) { load(s, in0 + t * a.q_token + h * a.q_head, c); },
                [&](const Both& s, uint32_t t, uint32_t h, uint32_t c) {
                    turned(s, out0 + t * a.o_token + h * a.o_head, t, c);
                });
        if (rest)
            over_heads<V>(
                tokens, heads, rest,
                [&](V& s, uint32_t t, uint32_t h, uint32_t c) { s.load(in0 + t * a.q_token + h * a.q_head + rot + c * kVector); },
                [&](const V& s, uint32_t t, uint32_t h, uint32_t c) {
                    s.template store<kStream>(out0 + t * a.o_token + h * a.o_head + rot + c * kVector);
                });
    }
    if (!kv_heads) return;
    const uint64_t k0 = a.k + token0 * a.k_token + g0 * a.k_head, v0 = a.v + token0 * a.v_token + g0 * a.v_head;
    if (turning)
        over_heads<Both>(
            tokens, kv_heads, turning,
            [&](Both& s, uint32_t t, uint32_t h, uint32_t c) { load(s, k0 + t * a.k_token + h * a.k_head, c); },
            [&](const Both& s, uint32_t t, uint32_t h, uint32_t c) {
                if (slots[t].k) turned(s, slots[t].k + (g0 + h) * a.kc_head, t, c);
            });
    if (rest)
        over_heads<V>(
            tokens, kv_heads, rest,
            [&](V& s, uint32_t t, uint32_t h, uint32_t c) { s.load(k0 + t * a.k_token + h * a.k_head + rot + c * kVector); },
            [&](const V& s, uint32_t t, uint32_t h, uint32_t c) {
                if (slots[t].k) s.template store<kStream>(slots[t].k + (g0 + h) * a.kc_head + rot + c * kVector);
            });
    using Whole = Vector<kF, 16 / kElement>;
    over_heads<Whole>(
        tokens, kv_heads, a.dim * kElement / 16,
        [&](Whole& s, uint32_t t, uint32_t h, uint32_t c) { s.load(v0 + t * a.v_token + h * a.v_head + c * 16); },
        [&](const Whole& s, uint32_t t, uint32_t h, uint32_t c) {
            if (slots[t].v) s.template store<kStream>(slots[t].v + (g0 + h) * a.vc_head + c * 16);
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
    uint32_t tile = bytes >= kTileBytes ? 1 : kTileBytes / bytes;
    tile = tile > kMostTile ? kMostTile : tile;
    if (pairs && tile > kMostAngles / pairs) tile = kMostAngles / pairs;
    const uint64_t tokens = uint64_t(a.docs) * a.max_q;
    while (tile > 1 && tokens / tile < 512) tile /= 2;
    a.tile = tile;
    const uint64_t groups = uint64_t(a.docs) * ((a.max_q + tile - 1) / tile);
    a.parts = groups >= 256 ? 1 : (groups >= 64 ? 2 : 4);
    if (a.parts > a.kv_heads) a.parts = a.kv_heads;
    void* params[] = {&a};
    // Calls larger than the caches write around them.
    const bool stream_out = tokens * bytes > (64u << 20);
    auto pick = [&](auto streams) {
        constexpr bool kStream = decltype(streams)::value;
        if constexpr (kW > 1)  // (pairs next to each other are even in number)
            if (a.interleaved) return reinterpret_cast<const void*>(cache_append_kernel<kF, kW, true, kStream>);
        return reinterpret_cast<const void*>(cache_append_kernel<kF, kW, false, kStream>);
    };
    const void* f = stream_out ? pick(std::integral_constant<bool, true>{}) : pick(std::integral_constant<bool, false>{});
    // (a dimension of the grid holds less than 2^32 lanes)
    constexpr uint64_t kMostGroups = 1u << 22;
    const uint64_t all = groups * a.parts, across = all < kMostGroups ? all : kMostGroups;
    return hipLaunchKernel(f, dim3(uint32_t(across), uint32_t((all + across - 1) / across)), dim3(kAppendThreads), params, 0,
                           stream);
}

hipError_t launch_cache_append(const AppendArgs& args, hipStream_t stream)
{
    AppendArgs a = args;
    return a.dtype == kF32 ? launch<true, 4>(a, stream) : launch<false, 8>(a, stream);
}

}  // namespace mezo
