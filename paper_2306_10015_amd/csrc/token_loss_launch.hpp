// token_loss_launch.hpp — interface between the C-ABI host code (forward.cpp)
// and the token loss kernels (token_loss.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "plans.hpp"

namespace mezo {

struct LossArgs {
    uint64_t logits;  // device address of row 0, fp32 or bf16
    uint64_t ld;      // elements from one row to the next
    uint64_t vocab;
    const int64_t* targets;
    float* losses;
    float* mean;      // or null
    float2* partial;  // (maximum, sum) of every part of every row; null if parts == 1
    uint32_t rows;
    uint32_t parts;   // of a row, each a workgroup
    uint32_t dtype;
};

hipError_t launch_token_loss(const LossArgs& args, hipStream_t stream);

}  // namespace mezo
