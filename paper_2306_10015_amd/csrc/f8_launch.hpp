// f8_launch.hpp — interface between the C-ABI host code (forward.cpp) and the
// 8-bit storage kernels (f8.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "plans.hpp"

namespace mezo {

struct F8QuantArgs {
    uint64_t values;  // device address, fp32 or bf16
    uint64_t ld;      // elements from one row to the next
    uint64_t codes;
    uint64_t scales;
    uint32_t rows;
    uint32_t cols;
    uint32_t dtype;
};

struct F8MatmulArgs {
    uint64_t x, xs;  // codes and scales of the m activations' rows
    uint64_t w, ws;  // and of the n weights' rows
    uint64_t c;      // [m, n] of out_dtype
    uint64_t ldc;    // elements from one row of c to the next
    uint64_t partial;  // fp32 [splits, m, n rounded up to 4] of a split product
    uint32_t m, n, k;
    uint32_t out_dtype;
    uint32_t splits;  // workgroups that share out k (set by the launch)
};

hipError_t launch_f8_quantize(const F8QuantArgs& args, hipStream_t stream);

hipError_t launch_f8_matmul(const F8MatmulArgs& args, hipStream_t stream);

}  // namespace mezo
