// Root-mean-square norm with the residual's addition and an MXINT result: h = x + r, v = h * rsqrt(mean(h^2) + eps) * w,
// codes and exponent bytes of v, and on request the values of the codes in bf16.
//
// Bound by memory: per value 4 or 2 B of x and of r, as much of h, 1 + 1/16 B of codes, 2 B of values.  One pass: a row's h
// stays in the registers of the wavefronts that share the row between the sum of its squares and its codes; only rows
// too long for that are read twice.  A lane owns 8 neighbouring values (16 B loads of bf16, 8 B stores of codes, 16 B
// of values), so a block of 16 is a pair of lanes, which agree on its exponent with one lane permutation.
//
// The mean and v are computed in 64 bits, which run at fp32's rate here and hide behind the memory: what decides a code is
// then h alone, not the order in which a row was summed.  v * 2^(fraction bits - e) is rounded to an integer by the addition of 1.5 * 2^52
// in the same fused multiply-add: the low word of the sum is the code.
//
// Measured: 8192 rows of 8192 (fp32 x, bf16 residual, values) 128 to 132 us, 5.7 TB/s of what has to move (a large copy: 5.05); 203 of 4112 5.2 us;
// one of 4096 3.4 us.
#include "serve.h"
#include "mx_device.h"

namespace lqer {

namespace {

constexpr int kLane = 8;                       // values a lane owns per step

struct Eight { float v[8]; };

template <int TYPE>
__device__ __forceinline__ Eight load8(const void* base, int64_t at) {
    Eight r;
    if (TYPE == LQER_F32) {
        const f32x4* p = reinterpret_cast<const f32x4*>((const float*)base + at);
        const f32x4 a = p[0], b = p[1];
#pragma unroll
        for (int i = 0; i < 4; ++i) { r.v[i] = a[i]; r.v[4 + i] = b[i]; }
    } else {
        const u32x4 w = *reinterpret_cast<const u32x4*>((const uint16_t*)base + at);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            r.v[2 * i] = f32_from_bits(w[i] << 16);
            r.v[2 * i + 1] = f32_from_bits(w[i] & 0xFFFF0000u);
        }
    }
    return r;
}

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {             // rounded to nearest even
    const bf16x2 p = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, p);
}

template <int TYPE>
__device__ __forceinline__ void store8(void* base, int64_t at, const Eight& r) {
    if (TYPE == LQER_F32) {
        f32x4* p = reinterpret_cast<f32x4*>((float*)base + at);
        p[0] = f32x4{r.v[0], r.v[1], r.v[2], r.v[3]};
        p[1] = f32x4{r.v[4], r.v[5], r.v[6], r.v[7]};
    } else {
        *reinterpret_cast<u32x4*>((uint16_t*)base + at) = u32x4{pack_bf16(r.v[0], r.v[1]), pack_bf16(r.v[2], r.v[3]),
                                                               pack_bf16(r.v[4], r.v[5]), pack_bf16(r.v[6], r.v[7])};
    }
}

// 1 / sqrt(v) from the hardware's estimate and two Newton steps; 0 for v = 0
__device__ __forceinline__ double rsqrt64(double v) {
    if (!(v > 0.0)) return v == 0.0 ? 0.0 : v;                               // (NaN goes on)
    double y = __builtin_amdgcn_rsq(v);
    y = y * __builtin_fma(-0.5 * v * y, y, 1.5);
    return y * __builtin_fma(-0.5 * v * y, y, 1.5);
}

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) v += __shfl_xor(v, m);
    return v;
}

// 8 values of v of a block (the pair's other lane has the other 8): codes as two words, the block's exponent byte, and the values
template <int BITS>
__device__ __forceinline__ uint32_t code8(const double (&t)[8], u32x2& w, u32x4& values) {
    constexpr int F = BITS - 2, TOP = (1 << (BITS - 1)) - 1;
    int hi = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) hi = max(hi, (int)(__builtin_bit_cast(uint64_t, t[i]) >> 32) & 0x7FFFFFFF);
    hi = max(hi, __builtin_amdgcn_mov_dpp(hi, 0xB1, 0xF, 0xF, true));        // quad_perm [1,0,3,2]
    const int eb = min(max((hi >> 20) - 1023 + 127, 0), 254);
    const double up = __builtin_bit_cast(double, (uint64_t)(1023 + F + 127 - eb) << 52);
    const float down = x_scale((uint32_t)eb, F);
    int c[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const double s = __builtin_fma(t[i], up, 6755399441055744.0);        // 1.5 * 2^52: |t * up| < 2^F * 2
        c[i] = min(max((int)(uint32_t)__builtin_bit_cast(uint64_t, s), -TOP), TOP);
    }
#pragma unroll
    for (int j = 0; j < 2; ++j)
        w[j] = (uint32_t)(c[4 * j] & 0xFF) | ((uint32_t)(c[4 * j + 1] & 0xFF) << 8) | ((uint32_t)(c[4 * j + 2] & 0xFF) << 16) |
               ((uint32_t)c[4 * j + 3] << 24);
#pragma unroll
    for (int j = 0; j < 4; ++j) values[j] = pack_bf16_exact((float)c[2 * j] * down, (float)c[2 * j + 1] * down);
    return (uint32_t)eb;
}

template <int XT, int RT, int BITS>
struct Row {
    const NormArgs& a;
    int64_t row;
    __device__ __forceinline__ Eight h(int64_t c) const {
        Eight v = load8<XT>(a.x, row * a.ldx + c);
        if (RT >= 0) {
            const Eight r = load8<RT>(a.residual, row * a.ldr + c);
#pragma unroll
            for (int i = 0; i < 8; ++i) v.v[i] += r.v[i];
        }
        return v;
    }
    __device__ __forceinline__ void put(int64_t c, const Eight& h, double inv, bool on) const {
        Eight w;
#pragma unroll
        for (int i = 0; i < 8; ++i) w.v[i] = 0.f;
        if (on) w = a.weight_type == LQER_F32 ? load8<LQER_F32>(a.weight, c) : load8<LQER_BF16>(a.weight, c);
        double t[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = (double)h.v[i] * ((double)w.v[i] * inv);
        u32x2 codes;
        u32x4 values;
        const uint32_t eb = code8<BITS>(t, codes, values);
        if (!on) return;
        if (RT >= 0) store8<(RT >= 0 ? RT : 0)>(a.h, row * a.ldh + c, h);
        *reinterpret_cast<u32x2*>(a.codes + row * a.cols + c) = codes;
        if (a.values) *reinterpret_cast<u32x4*>(a.values + row * a.ldv + c) = values;
        if ((c & 8) == 0) a.exps[row * (a.cols / 16) + c / 16] = (uint8_t)eb;
    }
};

// blockDim = (threads of a row, rows of the workgroup).  STEPS: steps of 8 values a lane keeps in registers; 0: any number, the
// row is read twice.
template <int XT, int RT, int BITS, int STEPS>
__global__ __launch_bounds__(1024) void rmsnorm_mx_kernel(NormArgs a) {
    __shared__ double part[16];
    const int64_t row = a.first + (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
    const bool live = row < a.rows;
    const Row<XT, RT, BITS> r{a, row};
    const int64_t stride = (int64_t)blockDim.x * kLane;
    const int64_t c0 = (int64_t)threadIdx.x * kLane;
    Eight keep[STEPS > 0 ? STEPS : 1];
    double sum = 0.0;
    if (STEPS > 0) {
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
#pragma unroll
            for (int i = 0; i < 8; ++i) keep[s].v[i] = 0.f;
            if (live && c0 + s * stride < a.cols) keep[s] = r.h(c0 + s * stride);
        }
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = __builtin_fma((double)keep[s].v[i], (double)keep[s].v[i], sum);
    } else if (live) {
        for (int64_t c = c0; c < a.cols; c += stride) {
            const Eight h = r.h(c);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = __builtin_fma((double)h.v[i], (double)h.v[i], sum);
        }
    }
    sum = wave_sum(sum);
    if (blockDim.x > 64) {                      // (then one row to a workgroup)
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
        __syncthreads();
        sum = 0.0;
        for (int w = 0; w < (int)blockDim.x / 64; ++w) sum += part[w];
    }
    const double inv = rsqrt64(sum / (double)a.cols + (double)a.eps);
    if (STEPS > 0) {
#pragma unroll
        for (int s = 0; s < STEPS; ++s) r.put(c0 + s * stride, keep[s], inv, live && c0 + s * stride < a.cols);
    } else {
        for (int64_t c = c0; c - c0 < a.cols; c += stride) {                  // (all lanes of a wavefront, as many times)
            const bool on = live && c < a.cols;
            Eight h;
#pragma unroll
            for (int i = 0; i < 8; ++i) h.v[i] = 0.f;
            if (on) h = r.h(c);
            r.put(c, h, inv, on);
        }
    }
}

// A launch counts its threads in 32 bits: so many rows have at most 2^31.
constexpr int64_t kRowsAtOnce = 1 << 21;

template <int XT, int RT, int BITS>
hipError_t launch(NormArgs a, hipStream_t s) {
    const int64_t units = a.cols / kLane;
    int tx, ty = 1, steps;
    if (units <= 128) { tx = 64; ty = 4; }
    else if (units <= 512) { tx = 256; }
    else if (units <= 2048) { tx = 512; }
    else { tx = 1024; }
    steps = (int)((units + tx - 1) / tx);
    const dim3 block(tx, ty);
    for (; a.first < a.rows; a.first += kRowsAtOnce) {
        const int64_t rows = a.rows - a.first < kRowsAtOnce ? a.rows - a.first : kRowsAtOnce;
        const dim3 grid((unsigned)((rows + ty - 1) / ty));
        if (steps <= 1) hipLaunchKernelGGL((rmsnorm_mx_kernel<XT, RT, BITS, 1>), grid, block, 0, s, a);
        else if (steps <= 2) hipLaunchKernelGGL((rmsnorm_mx_kernel<XT, RT, BITS, 2>), grid, block, 0, s, a);
        else if (steps <= 4) hipLaunchKernelGGL((rmsnorm_mx_kernel<XT, RT, BITS, 4>), grid, block, 0, s, a);
        else hipLaunchKernelGGL((rmsnorm_mx_kernel<XT, RT, BITS, 0>), grid, block, 0, s, a);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <int XT, int RT>
hipError_t launch_bits(const NormArgs& a, hipStream_t s) {
    return a.bits == 8 ? launch<XT, RT, 8>(a, s) : launch<XT, RT, 6>(a, s);
}

}  // namespace

hipError_t launch_rmsnorm_mx(const NormArgs& a, hipStream_t s) {
    if (a.x_type == LQER_F32) {
        if (!a.residual) return launch_bits<LQER_F32, -1>(a, s);
        return a.res_type == LQER_F32 ? launch_bits<LQER_F32, LQER_F32>(a, s) : launch_bits<LQER_F32, LQER_BF16>(a, s);
    }
    if (!a.residual) return launch_bits<LQER_BF16, -1>(a, s);
    return a.res_type == LQER_F32 ? launch_bits<LQER_BF16, LQER_F32>(a, s) : launch_bits<LQER_BF16, LQER_BF16>(a, s);
}

}  // namespace lqer
