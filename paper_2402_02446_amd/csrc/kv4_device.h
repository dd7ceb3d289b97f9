// Device helpers of the MXINT4 cache: where a page's parts lie, and its code words as operands of the bf16 matrix instructions.
#pragma once
#include "serve.h"
#include "mx_device.h"

namespace lqer {

// Byte offsets inside the record of one page and head, of token `off` (values: group `off / 4`).
template <int D>
struct Kv4Record {
    int P_bits;
    __device__ __forceinline__ int64_t bytes() const { return ((int64_t)(D * 9 / 8)) << P_bits; }
    __device__ __forceinline__ int key(int off) const { return off * (D / 2); }
    __device__ __forceinline__ int value(int off4) const { return ((D / 2) << P_bits) + off4 * (D * 2); }
    __device__ __forceinline__ int key_exp(int off) const { return (D << P_bits) + off * (D / 16); }
    __device__ __forceinline__ int value_exp(int off4) const { return ((D + D / 16) << P_bits) + off4 * (D / 4); }
};

// What the queries of one tile of rows of a request see of its cache.  Rows are (query, head of the group) pairs, query by query.
struct Kv4Rows {
    int first, n, len;     // first row of q, queries, cached tokens
    int row0, rows;        // this tile's first row, and how many it has
    int lo, hi;            // cached tokens that any of them may see: [lo, hi)

    __device__ __forceinline__ int position(int i) const { return len - n + i; }
};

// Request b.  Numbers on the device are taken into the ranges of the arrays that were handed over.
__device__ __forceinline__ Kv4Rows kv4_request(const Kv4Args& a, int b) {
    Kv4Rows r;
    const int64_t c0 = a.cu_q[b], c1 = a.cu_q[b + 1];
    const int64_t q0 = min(max(c0, (int64_t)0), a.sh.Tq), q1 = min(max(c1, q0), a.sh.Tq);
    r.first = (int)q0;
    r.n = (int)(q1 - q0);
    r.len = (int)min((int64_t)max(a.kv_len[b], 0), (int64_t)a.sh.table_ld << a.P_bits);
    r.row0 = r.rows = r.lo = r.hi = 0;
    return r;
}

__device__ __forceinline__ int kv4_row_end(const Kv4Args& a, const Kv4Rows& r, int i) {
    return a.sh.causal ? min(max(r.position(i) + 1, 0), r.len) : r.len;
}
__device__ __forceinline__ int kv4_row_begin(const Kv4Args& a, const Kv4Rows& r, int i) {
    return a.sh.window > 0 ? (int)min(max((int64_t)r.position(i) - a.sh.window + 1, (int64_t)0), (int64_t)r.len) : 0;
}

__device__ __forceinline__ void kv4_tile(const Kv4Args& a, Kv4Rows& r, int row0, int most) {
    r.row0 = row0;
    r.rows = min(r.n * a.group - row0, most);
    const int i0 = row0 / a.group, i1 = (row0 + r.rows - 1) / a.group;
    r.lo = kv4_row_begin(a, r, i0);
    r.hi = kv4_row_end(a, r, i1);
    if (r.hi < r.lo) r.hi = r.lo;
}

// Whether this request is the business of the kernel for many rows (MANY) or of the other one.
template <bool MANY>
__device__ __forceinline__ bool kv4_mine(const Kv4Args& a, const Kv4Rows& r) {
    if (MANY) return !a.few.run || (int64_t)r.n * a.group > a.few_rows;
    return !a.many.run || (int64_t)r.n * a.group <= a.few_rows;
}

// The parts that a tile's tokens are cut into: their length and number.  Parts begin at multiples of 32 tokens.
template <bool MANY>
__device__ __forceinline__ int kv4_parts(const Kv4Args& a, const Kv4Rows& r, int& chunk) {
    const Kv4Plan& plan = MANY ? a.many : a.few;
    const int lo = r.lo & ~31, all = r.hi > r.lo ? r.hi - lo : 0;
    if (!MANY && r.row0 + r.rows > plan.cap) {         // rows beyond the estimate: no room for their parts
        chunk = (all + 31) & ~31;
        return all > 0 ? 1 : 0;
    }
    chunk = plan.chunk;
    const int least = (all + plan.splits - 1) / plan.splits;
    if (least > chunk) chunk = (least + 31) & ~31;
    return (all + chunk - 1) / chunk;
}

// Where the parts of a row (query row orow, query head h; row of request b and cached head) lie.
template <bool MANY>
__device__ __forceinline__ int64_t kv4_part(const Kv4Args& a, int b, int head, int row, int64_t orow, int h) {
    if (MANY) return (orow * a.sh.q_heads + h) * a.many.splits;
    return (((int64_t)b * a.sh.kv_heads + head) * a.few.cap + row) * a.few.splits;
}

// fp32 scale 2^(eb - 127 - 2 + 9) of a block of the cache (w_scale of the weights): the byte is at most 247.
__device__ __forceinline__ float kv4_scale(uint32_t eb) { return f32_from_bits((eb + 7u) << 23); }

// the maximum and the sum over the lanes that share lane % 16
__device__ __forceinline__ float quad_rows_max(float v) {
    const auto a = __builtin_amdgcn_permlane16_swap(f32_bits(v), f32_bits(v), false, false);
    v = __builtin_fmaxf(f32_from_bits(a[0]), f32_from_bits(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(f32_bits(v), f32_bits(v), false, false);
    return __builtin_fmaxf(f32_from_bits(b[0]), f32_from_bits(b[1]));
}
__device__ __forceinline__ float quad_rows_sum(float v) {
    const auto a = __builtin_amdgcn_permlane16_swap(f32_bits(v), f32_bits(v), false, false);
    v = f32_from_bits(a[0]) + f32_from_bits(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(f32_bits(v), f32_bits(v), false, false);
    return f32_from_bits(b[0]) + f32_from_bits(b[1]);
}

__device__ __forceinline__ float exp2_fast(float v) { return __builtin_amdgcn_exp2f(v); }

__device__ __forceinline__ uint32_t pack_bf16_near(float a, float b) {         // rounded to nearest even
    const bf16x2 p = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, p);
}

}  // namespace lqer
