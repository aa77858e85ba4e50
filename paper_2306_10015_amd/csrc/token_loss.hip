// token_loss.hip — the loss of Algorithm 1's two forward passes: for every
// token t with a target y >= 0
//   loss_t = ln sum_v exp(x_tv) - x_ty,
// and the mean over those tokens, from logits x of fp32 or bf16 storage.
//
// One pass over the logits: every lane keeps the running maximum m of what it
// has read and s = sum exp(x - m), rescaled when m grows; the lanes' pairs join
// as s = s1 exp(m1 - m) + s2 exp(m2 - m). All of it in fp32, exp as
// exp2((x - m) log2 e) with the difference formed first, so that its error does
// not grow with |m|: the loss of a pass enters the projected gradient as a
// difference of two nearly equal numbers. The mean is summed in fp64 in a fixed
// order, so equal logits give equal losses, bit for bit.
#include "records.hpp"
#include "stream_io.hpp"
#include "token_loss_launch.hpp"

namespace mezo {

constexpr uint32_t kLossThreads = 256;
constexpr uint32_t kFinishThreads = 1024;
// 16-byte loads a lane issues before it uses any.
constexpr uint32_t kLossLoads = 4;
constexpr float kLog2e = 1.44269504088896341f;

struct MaxSum {
    float m, s;
};

// What to subtract: the maximum, or 0 while nothing (or only -inf) was read.
__device__ __forceinline__ float finite_ref(float m) { return m == -__builtin_inff() ? 0.0f : m; }

__device__ __forceinline__ MaxSum join(MaxSum a, MaxSum b)
{
    const float m = fmaxf(a.m, b.m), r = finite_ref(m);
    return {m, a.s * __builtin_amdgcn_exp2f((a.m - r) * kLog2e) + b.s * __builtin_amdgcn_exp2f((b.m - r) * kLog2e)};
}

template <uint32_t N>
__device__ __forceinline__ void take(MaxSum& a, const float (&x)[N])
{
    float m = a.m;
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) m = fmaxf(m, x[i]);
    const float r = finite_ref(m);
    float s = a.s * __builtin_amdgcn_exp2f((a.m - r) * kLog2e);
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) s += __builtin_amdgcn_exp2f((x[i] - r) * kLog2e);
    a = {m, s};
}

template <uint32_t kDtype>
struct Row {
    static constexpr uint32_t kBytes = kDtype == kF32 ? 4 : 2;
    static constexpr uint32_t kPer16 = 16 / kBytes;
    uint64_t addr;

    __device__ __forceinline__ float at(uint64_t i) const
    {
        if constexpr (kDtype == kF32) return reinterpret_cast<const gfloat_t*>(addr)[i];
        return __uint_as_float(uint32_t(reinterpret_cast<const gu16_t*>(addr)[i]) << 16);
    }
    // The values of 16 bytes.
    __device__ static __forceinline__ void unpack(uint4 v, float* x)
    {
        const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {
            if constexpr (kDtype == kF32) {
                x[i] = __uint_as_float(u[i]);
            } else {
                x[2 * i] = __uint_as_float(u[i] << 16);
                x[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
            }
        }
    }
};

// A lane's (maximum, sum) over its share of part `part` of `parts` of a row;
// lane l of kLanes. Rows may start at any element: the elements up to the first
// 16-byte boundary and past the last go one to a lane.
template <uint32_t kDtype, uint32_t kLanes>
__device__ __forceinline__ MaxSum read_row(Row<kDtype> row, uint64_t vocab, uint32_t part, uint32_t parts, uint32_t l)
{
    constexpr uint32_t kPer = Row<kDtype>::kPer16;
    const uint64_t head0 = ((16u - (row.addr & 15u)) & 15u) / Row<kDtype>::kBytes;
    const uint64_t head = head0 < vocab ? head0 : vocab;
    const uint64_t vecs = (vocab - head) / kPer;
    const uint64_t tail = head + vecs * kPer;  // its first element
    const uint64_t v0 = vecs * part / parts, v1 = vecs * (part + 1) / parts;
    const uint64_t base = row.addr + head * Row<kDtype>::kBytes;
    MaxSum a = {-__builtin_inff(), 0.0f};
    uint64_t v = v0 + l;
    for (; v + (kLossLoads - 1) * kLanes < v1; v += kLossLoads * kLanes) {
        uint4 w[kLossLoads];
#pragma unroll
        for (uint32_t i = 0; i < kLossLoads; ++i) w[i] = load_stream(base + (v + i * kLanes) * 16);
        float x[kLossLoads * kPer];
#pragma unroll
        for (uint32_t i = 0; i < kLossLoads; ++i) Row<kDtype>::unpack(w[i], x + i * kPer);
        take(a, x);
    }
    for (; v < v1; v += kLanes) {
        float x[kPer];
        Row<kDtype>::unpack(load_stream(base + v * 16), x);
        take(a, x);
    }
    if (part == 0 && l < head) {
        const float x[1] = {row.at(l)};
        take(a, x);
    }
    if (part == parts - 1 && tail + l < vocab) {
        const float x[1] = {row.at(tail + l)};
        take(a, x);
    }
    return a;
}

__device__ __forceinline__ MaxSum join_wave(MaxSum a)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) a = join(a, {__shfl_xor(a.m, off), __shfl_xor(a.s, off)});
    return a;
}

// A target past the vocabulary has no logit: its loss is NaN.
template <uint32_t kDtype>
__device__ __forceinline__ float loss_of(MaxSum a, Row<kDtype> row, uint64_t vocab, int64_t target)
{
    if (uint64_t(target) >= vocab) return __builtin_nanf("");
    return (a.m - row.at(uint64_t(target))) + logf(a.s);
}

// kLanes = 64: a row to a wave, for short rows; kLossThreads: a row (or a part
// of one) to a workgroup.
template <uint32_t kDtype, uint32_t kLanes>
__global__ void __launch_bounds__(kLossThreads) loss_rows_kernel(LossArgs a)
{
    const uint32_t l = threadIdx.x % kLanes;
    const uint64_t t = uint64_t(blockIdx.x) * (kLossThreads / kLanes) + threadIdx.x / kLanes;
    if (t >= a.rows) return;  // whole waves; whole workgroups where they share a row
    const int64_t target = a.targets[t];
    const Row<kDtype> row = {a.logits + t * a.ld * Row<kDtype>::kBytes};
    if (target < 0) {  // not counted: nothing of the row is read
        if (l == 0 && a.parts == 1) a.losses[t] = 0.0f;
        return;
    }
    MaxSum s = join_wave(read_row<kDtype, kLanes>(row, a.vocab, blockIdx.y, a.parts, l));
    if constexpr (kLanes > 64) {
        __shared__ MaxSum part[kLanes / 64];
        if ((l & 63u) == 0) part[l >> 6] = s;
        __syncthreads();
        s = part[0];
#pragma unroll
        for (uint32_t i = 1; i < kLanes / 64; ++i) s = join(s, part[i]);
    }
    if (l != 0) return;
    if (a.parts > 1)
        a.partial[t * a.parts + blockIdx.y] = make_float2(s.m, s.s);
    else
        a.losses[t] = loss_of(s, row, a.vocab, target);
}

// One workgroup: the losses of rows in parts, and the mean.
template <uint32_t kDtype>
__global__ void __launch_bounds__(kFinishThreads) loss_finish_kernel(LossArgs a)
{
    // a lane's rows in batches, whose loads are all under way before the first is used (16384
    // rows: 9.4 -> 6.6 us)
    constexpr uint32_t kBatch = 8;
    double sum = 0.0;
    uint32_t count = 0;
    for (uint64_t t0 = threadIdx.x; t0 < a.rows; t0 += kBatch * kFinishThreads) {
        int64_t target[kBatch];
        float loss[kBatch];
#pragma unroll
        for (uint32_t j = 0; j < kBatch; ++j) {
            const uint64_t t = t0 + j * kFinishThreads;
            target[j] = t < a.rows ? a.targets[t] : -1;
            loss[j] = t < a.rows && a.parts == 1 ? a.losses[t] : 0.0f;
        }
#pragma unroll
        for (uint32_t j = 0; j < kBatch; ++j) {
            const uint64_t t = t0 + j * kFinishThreads;
            if (a.parts > 1 && t < a.rows) {
                if (target[j] >= 0) {
                    const float2* p = a.partial + t * a.parts;
                    MaxSum s = {p[0].x, p[0].y};
                    for (uint32_t i = 1; i < a.parts; ++i) s = join(s, {p[i].x, p[i].y});
                    loss[j] = loss_of(s, Row<kDtype>{a.logits + t * a.ld * Row<kDtype>::kBytes}, a.vocab, target[j]);
                }
                a.losses[t] = loss[j];
            }
            if (target[j] >= 0) {
                sum += double(loss[j]);
                ++count;
            }
        }
    }
    if (!a.mean) return;
    __shared__ double sums[kFinishThreads / 64];
    __shared__ uint32_t counts[kFinishThreads / 64];
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
        sum += __shfl_xor(sum, off);
        count += __shfl_xor(count, off);
    }
    if ((threadIdx.x & 63u) == 0) {
        sums[threadIdx.x >> 6] = sum;
        counts[threadIdx.x >> 6] = count;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        for (uint32_t i = 1; i < kFinishThreads / 64; ++i) {
            sum += sums[i];
            count += counts[i];
        }
        *a.mean = count ? float(sum / double(count)) : 0.0f;
    }
}

// A few short rows: one workgroup reads them all, one after another, and takes the mean.
template <uint32_t kDtype>
__global__ void __launch_bounds__(kFinishThreads) loss_all_kernel(LossArgs a)
{
    __shared__ MaxSum part[kFinishThreads / 64];
    double sum = 0.0;
    uint32_t count = 0;
    for (uint32_t t = 0; t < a.rows; ++t) {
        const int64_t target = a.targets[t];
        float loss = 0.0f;
        if (target >= 0) {  // (uniform)
            const Row<kDtype> row = {a.logits + t * a.ld * Row<kDtype>::kBytes};
            const MaxSum s = join_wave(read_row<kDtype, kFinishThreads>(row, a.vocab, 0, 1, threadIdx.x));
            if ((threadIdx.x & 63u) == 0) part[threadIdx.x >> 6] = s;
            __syncthreads();
            // every wave joins the 16 parts: the same values in the same order
            const uint32_t l = threadIdx.x & 63u;
            MaxSum all = l < kFinishThreads / 64 ? part[l] : MaxSum{-__builtin_inff(), 0.0f};
            all = join_wave(all);
            loss = loss_of(all, row, a.vocab, target);
            sum += double(loss);
            ++count;
            __syncthreads();  // the parts are read
        }
        if (threadIdx.x == 0) a.losses[t] = loss;
    }
    if (threadIdx.x == 0 && a.mean) *a.mean = count ? float(sum / double(count)) : 0.0f;
}

template <uint32_t kDtype>
hipError_t launch(LossArgs a, hipStream_t stream)
{
    void* params[] = {&a};
    if (one_group(a.rows, a.vocab))
        return hipLaunchKernel(reinterpret_cast<const void*>(loss_all_kernel<kDtype>), dim3(1), dim3(kFinishThreads),
                               params, 0, stream);
    const bool wave = a.vocab < kWaveRow;
    const void* f = wave ? reinterpret_cast<const void*>(loss_rows_kernel<kDtype, 64>)
                         : reinterpret_cast<const void*>(loss_rows_kernel<kDtype, kLossThreads>);
    const uint32_t per = wave ? kLossThreads / 64 : 1;
    const hipError_t e = hipLaunchKernel(f, dim3((a.rows + per - 1) / per, a.parts), dim3(kLossThreads), params, 0, stream);
    if (e != hipSuccess || (a.parts == 1 && !a.mean)) return e;
    return hipLaunchKernel(reinterpret_cast<const void*>(loss_finish_kernel<kDtype>), dim3(1), dim3(kFinishThreads),
                           params, 0, stream);
}

hipError_t launch_token_loss(const LossArgs& args, hipStream_t stream)
{
    return args.dtype == kF32 ? launch<kF32>(args, stream) : launch<kBF16>(args, stream);
}

}  // namespace mezo
