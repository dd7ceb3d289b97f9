// C entry points of the calls between a block's linears: what the host can see of their arguments is checked here.
#include "serve.h"

using namespace lqer;

namespace {

bool type_ok(int t) { return t == LQER_F32 || t == LQER_BF16; }
// a row stride in elements whose rows start on 16 bytes
bool stride_ok(int64_t ld, int64_t least, int type) { return ld >= least && (ld & (type == LQER_F32 ? 3 : 7)) == 0; }
bool aligned(const void* p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
constexpr int64_t kMaxGrid = 0x7FFFFFFF;

}  // namespace

extern "C" {

int lqer_rmsnorm_mx(const void* x_dev, int x_type, int64_t rows, int64_t cols, int64_t ldx, const void* residual_dev, int64_t ldr,
                    void* h_dev, int64_t ldh, int res_type, const void* weight_dev, int weight_type, float eps, int elem_bits,
                    int8_t* codes_dev, uint8_t* exps_dev, uint16_t* values_dev, int64_t ldv, void* hip_stream) {
    if (!type_ok(x_type) || !type_ok(weight_type) || (elem_bits != 8 && elem_bits != 6)) return LQER_ERR_UNSUPPORTED;
    const bool res = residual_dev || h_dev;
    if (res && !type_ok(res_type)) return LQER_ERR_UNSUPPORTED;
    if (rows < 0 || rows > kMaxGrid || cols < 0 || (cols & 15) != 0 || !(eps >= 0.f)) return LQER_ERR_SHAPE;
    if (rows == 0 || cols == 0) return LQER_OK;
    if (!x_dev || !weight_dev || !codes_dev || !exps_dev || (res && (!residual_dev || !h_dev))) return LQER_ERR_NULL;
    if (!stride_ok(ldx, cols, x_type) || !aligned(x_dev, 16) || !aligned(weight_dev, 16) || !aligned(codes_dev, 16)) return LQER_ERR_SHAPE;
    if (res && (!stride_ok(ldr, cols, res_type) || !stride_ok(ldh, cols, res_type) || !aligned(residual_dev, 16) || !aligned(h_dev, 16)))
        return LQER_ERR_SHAPE;
    if (values_dev && (!stride_ok(ldv, cols, LQER_BF16) || !aligned(values_dev, 16))) return LQER_ERR_SHAPE;
    const NormArgs a{x_dev, residual_dev, h_dev, weight_dev, x_type, res_type, weight_type, rows, cols, ldx, ldr, ldh, ldv, eps, elem_bits,
                     codes_dev, exps_dev, values_dev};
    return launch_rmsnorm_mx(a, (hipStream_t)hip_stream) == hipSuccess ? LQER_OK : LQER_ERR_HIP;
}

}  // extern "C"
