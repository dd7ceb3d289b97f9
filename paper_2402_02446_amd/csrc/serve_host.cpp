// C entry points of the calls between a block's linears: what the host can see of their arguments is checked here.
#include "serve.h"

using namespace lqer;

namespace {

bool type_ok(int t) { return t == LQER_F32 || t == LQER_BF16; }
// a row stride in elements whose rows start on 16 bytes
bool stride_ok(int64_t ld, int64_t least, int type) { return ld >= least && (ld & (type == LQER_F32 ? 3 : 7)) == 0; }
bool aligned(const void* p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
constexpr int64_t kMaxGrid = 0x7FFFFFFF;

// (a launch counts its threads in 32 bits: 256 to a tile of 64 tokens)
constexpr int64_t kMaxAdapterTokens = 1 << 29;

// The sizes of a call with adapters; false where it does not take them.  (N: the documented limit; blocks of 64 columns and workgroups for them are
// counted in 32 bits, far from their end.)
bool adapter_sizes(AdapterArgs& a, int64_t M, int64_t K, int64_t N, int R, int n) {
    if (M < 0 || M > kMaxAdapterTokens || K <= 0 || (K & 7) != 0 || N < 0 || N > 65535 * 64ll || R <= 0 || R > kMaxAdapterRank || (R & 7) != 0 || n <= 0 ||
        n > kMaxAdapters)
        return false;
    a.M = M; a.K = K; a.N = N; a.R = R; a.n = n;
    return true;
}

bool kv4_format_ok(int P, int D) { return P >= 16 && P <= 1024 && (P & (P - 1)) == 0 && (D == 64 || D == 128 || D == 256); }
// (slots, and sums of two token counts, are 32 bits wide on the device)
constexpr int64_t kMaxTokens = 1 << 30;
bool kv4_pool_ok(int64_t pages, int P, int heads) { return pages > 0 && heads > 0 && heads <= 1024 && pages <= kMaxTokens / P; }

int kv4_shape_status(const lqer_kv4_shape& s) {
    if (!kv4_format_ok(s.page_tokens, s.head_dim) || !type_ok(s.out_type)) return LQER_ERR_UNSUPPORTED;
    if (!kv4_pool_ok(s.pages, s.page_tokens, s.kv_heads) || s.q_heads <= 0 || s.q_heads > 65536 || s.q_heads % s.kv_heads != 0) return LQER_ERR_SHAPE;
    if (s.n_requests < 0 || s.n_requests > 65535 || s.table_ld <= 0 || s.table_ld > kMaxTokens / s.page_tokens || s.Tq < 0 || s.Tq > kMaxGrid / 2 / s.q_heads)
        return LQER_ERR_SHAPE;
    const int64_t row = (int64_t)s.q_heads * s.head_dim;
    if (!stride_ok(s.ldq, row, LQER_BF16) || !stride_ok(s.ldo, row, LQER_BF16)) return LQER_ERR_SHAPE;
    if (s.max_q < 0 || s.max_kv < 0 || (s.causal != 0 && s.causal != 1) || s.window < 0 || !(s.scale == s.scale)) return LQER_ERR_SHAPE;
    return LQER_OK;
}

}  // namespace

extern "C" {

int lqer_rmsnorm_mx(const void* x_dev, int x_type, int64_t rows, int64_t cols, int64_t ldx, const void* residual_dev, int64_t ldr,
                    void* h_dev, int64_t ldh, int res_type, const void* weight_dev, int weight_type, float eps, int elem_bits,
                    int8_t* codes_dev, uint8_t* exps_dev, uint16_t* values_dev, int64_t ldv, void* hip_stream) {
    if (!type_ok(x_type) || !type_ok(weight_type) || (elem_bits != 8 && elem_bits != 6)) return LQER_ERR_UNSUPPORTED;
    const bool res = residual_dev || h_dev;
    if (res && !type_ok(res_type)) return LQER_ERR_UNSUPPORTED;
    if (rows < 0 || rows > kMaxGrid || cols < 0 || (cols & 15) != 0 || !(eps >= 0.f && eps <= 3.402823466e38f)) return LQER_ERR_SHAPE;
    if (rows == 0 || cols == 0) return LQER_OK;
    if (!x_dev || !weight_dev || !codes_dev || !exps_dev || (res && (!residual_dev || !h_dev))) return LQER_ERR_NULL;
    if (!stride_ok(ldx, cols, x_type) || !aligned(x_dev, 16) || !aligned(weight_dev, 16) || !aligned(codes_dev, 16)) return LQER_ERR_SHAPE;
    if (res && (!stride_ok(ldr, cols, res_type) || !stride_ok(ldh, cols, res_type) || !aligned(residual_dev, 16) || !aligned(h_dev, 16)))
        return LQER_ERR_SHAPE;
    if (res && residual_dev == h_dev && ldr != ldh) return LQER_ERR_SHAPE;
    if (values_dev && (!stride_ok(ldv, cols, LQER_BF16) || !aligned(values_dev, 16))) return LQER_ERR_SHAPE;
    const NormArgs a{x_dev, residual_dev, h_dev, weight_dev, x_type, res_type, weight_type, rows, cols, ldx, ldr, ldh, ldv, eps, elem_bits,
                     codes_dev, exps_dev, values_dev, 0};
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

size_t lqer_kv4_page_bytes(int page_tokens, int head_dim) {
    return kv4_format_ok(page_tokens, head_dim) ? (size_t)page_tokens * head_dim * 9 / 8 : 0;
}

int lqer_kv4_append(uint8_t* pool_dev, int64_t pages, int page_tokens, int kv_heads, int head_dim, const void* k_dev, int64_t ldk,
                    const void* v_dev, int64_t ldv, int kv_type, int64_t T, const int32_t* slots_dev, void* hip_stream) {
    if (!kv4_format_ok(page_tokens, head_dim) || !type_ok(kv_type)) return LQER_ERR_UNSUPPORTED;
    if (!kv4_pool_ok(pages, page_tokens, kv_heads) || T < 0) return LQER_ERR_SHAPE;
    if (T == 0) return LQER_OK;
    if (!pool_dev || !k_dev || !v_dev || !slots_dev) return LQER_ERR_NULL;
    const int64_t row = (int64_t)kv_heads * head_dim;
    if (!stride_ok(ldk, row, kv_type) || !stride_ok(ldv, row, kv_type) || !aligned(k_dev, 16) || !aligned(v_dev, 16) || !aligned(pool_dev, 16) ||
        !aligned(slots_dev, 4))
        return LQER_ERR_SHAPE;
    const Kv4AppendArgs a{pool_dev, pages, __builtin_ctz((unsigned)page_tokens), kv_heads, head_dim, k_dev, v_dev, ldk, ldv, kv_type, T, slots_dev};
    return launch_kv4_append(a, (hipStream_t)hip_stream) == hipSuccess ? LQER_OK : LQER_ERR_HIP;
}

size_t lqer_kv4_attention_workspace_bytes(const lqer_kv4_shape* shape) {
    if (!shape || kv4_shape_status(*shape) != LQER_OK || shape->Tq == 0 || shape->n_requests == 0) return 0;
    Kv4Args a{};
    a.sh = *shape;
    return plan_kv4(a, nullptr);
}

int lqer_kv4_attention(const lqer_kv4_shape* shape, const uint8_t* pool_dev, const uint16_t* q_dev, const int32_t* cu_q_dev,
                       const int32_t* kv_len_dev, const int32_t* table_dev, void* out_dev, void* workspace_dev, size_t workspace_bytes,
                       void* hip_stream) {
    if (!shape) return LQER_ERR_NULL;
    if (const int st = kv4_shape_status(*shape); st != LQER_OK) return st;
    if (shape->Tq == 0 || shape->n_requests == 0) return LQER_OK;
    if (!pool_dev || !q_dev || !cu_q_dev || !kv_len_dev || !table_dev || !out_dev) return LQER_ERR_NULL;
    if (!aligned(pool_dev, 16) || !aligned(q_dev, 16) || !aligned(out_dev, 16) || !aligned(cu_q_dev, 4) || !aligned(kv_len_dev, 4) || !aligned(table_dev, 4))
        return LQER_ERR_SHAPE;
    Kv4Args a{};
    a.sh = *shape;
    a.pool = pool_dev; a.q = q_dev; a.cu_q = cu_q_dev; a.kv_len = kv_len_dev; a.table = table_dev; a.out = out_dev;
    const size_t need = plan_kv4(a, workspace_dev);
    if (need && (!workspace_dev || !aligned(workspace_dev, 256) || need > workspace_bytes)) return LQER_ERR_WORKSPACE;
    return launch_kv4_attention(a, (hipStream_t)hip_stream) == hipSuccess ? LQER_OK : LQER_ERR_HIP;
}

}  // extern "C"
