// C entry points of the calls between a block's linears: what the host can see of their arguments is checked here.
#include "serve.h"

using namespace lqer;

namespace {

bool type_ok(int t) { return t == LQER_F32 || t == LQER_BF16; }
// a row stride in elements whose rows start on 16 bytes
bool stride_ok(int64_t ld, int64_t least, int type) { return ld >= least && (ld & (type == LQER_F32 ? 3 : 7)) == 0; }
bool aligned(const void* p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
constexpr int64_t kMaxGrid = 0x7FFFFFFF;

// The sizes of a call with adapters; false where it does not take them.  (N: the second axis of a grid counts 64 columns.)
bool adapter_sizes(AdapterArgs& a, int64_t M, int64_t K, int64_t N, int R, int n) {
    if (M < 0 || M > kMaxGrid / 2 || K <= 0 || (K & 7) != 0 || N < 0 || N > 65535 * 64ll || R <= 0 || R > kMaxAdapterRank || (R & 7) != 0 || n <= 0 ||
        n > kMaxAdapters)
        return false;
    a.M = M; a.K = K; a.N = N; a.R = R; a.n = n;
    return true;
}

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

size_t lqer_adapters_workspace_bytes(int64_t M, int64_t K, int64_t N, int R, int n_adapters) {
    AdapterArgs a{};
    if (!adapter_sizes(a, M, K, N, R, n_adapters) || M == 0 || N == 0) return 0;
    return plan_adapters(a, nullptr);
}

int lqer_adapters_forward(const uint16_t* X_dev, int64_t M, int64_t K, int64_t ldx, const int32_t* ids_dev, const uint16_t* A_dev,
                          const uint16_t* B_dev, int n_adapters, int R, const int32_t* ranks_dev, const float* scales_dev,
                          const float* Y_in_dev, int64_t ldyi, float* Y_out_dev, int64_t N, int64_t ldyo, void* workspace_dev,
                          size_t workspace_bytes, void* hip_stream) {
    AdapterArgs a{};
    if (n_adapters > kMaxAdapters || R > kMaxAdapterRank) return LQER_ERR_UNSUPPORTED;
    if (!adapter_sizes(a, M, K, N, R, n_adapters)) return LQER_ERR_SHAPE;
    if (M == 0 || N == 0) return LQER_OK;
    if (!X_dev || !ids_dev || !A_dev || !B_dev || !Y_in_dev || !Y_out_dev) return LQER_ERR_NULL;
    if (!stride_ok(ldx, K, LQER_BF16) || !aligned(X_dev, 16) || !aligned(A_dev, 16) || !aligned(B_dev, 16)) return LQER_ERR_SHAPE;
    if (!stride_ok(ldyi, N, LQER_F32) || !stride_ok(ldyo, N, LQER_F32) || !aligned(Y_in_dev, 16) || !aligned(Y_out_dev, 16)) return LQER_ERR_SHAPE;
    if (!aligned(ids_dev, 4) || !aligned(ranks_dev, 4) || !aligned(scales_dev, 4)) return LQER_ERR_SHAPE;
    if (Y_in_dev == Y_out_dev && ldyi != ldyo) return LQER_ERR_SHAPE;
    if (!workspace_dev || !aligned(workspace_dev, 256) || plan_adapters(a, workspace_dev) > workspace_bytes) return LQER_ERR_WORKSPACE;
    a.X = X_dev; a.ldx = ldx; a.ids = ids_dev; a.A = A_dev; a.B = B_dev; a.ranks = ranks_dev; a.scales = scales_dev;
    a.Y_in = Y_in_dev; a.ldyi = ldyi; a.Y_out = Y_out_dev; a.ldyo = ldyo;
    return launch_adapters(a, (hipStream_t)hip_stream) == hipSuccess ? LQER_OK : LQER_ERR_HIP;
}

}  // extern "C"
