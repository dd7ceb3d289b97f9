// What the host side and the kernels of the calls between a block's linears share.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>
#include "lqer.h"

namespace lqer {

struct NormArgs {
    const void* x;
    const void* residual;          // null: h = x, nothing is stored
    void* h;
    const void* weight;
    int x_type, res_type, weight_type;
    int64_t rows, cols, ldx, ldr, ldh, ldv;
    float eps;
    int bits;
    int8_t* codes;
    uint8_t* exps;
    uint16_t* values;              // may be null
};
hipError_t launch_rmsnorm_mx(const NormArgs& a, hipStream_t s);

}  // namespace lqer
