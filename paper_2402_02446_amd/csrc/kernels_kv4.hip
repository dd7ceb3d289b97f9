// The MXINT4 cache of keys and values: appending to it, and attention of few query rows over it.
//
// Appending is bound by its launch (2.3 to 3.5 us up to 200 tokens of 8 heads of 128, 2781 7.5); a lane turns 8 values into one word, its
// neighbour has the block's other 8.
//
// Attention of few rows (query, head of the group), 16 to a workgroup, is bound by the cache's bytes, 4.5 bits a value: every word is
// read once by each tile of rows, and turned into bf16 operands in registers.  A wavefront takes 32 cached tokens a step:
//   S^T = K Q^T   tokens as rows of the 16 x 16 x 32 matrix instruction, query rows as columns: lane (t, g) reads 16 contiguous
//                 bytes of token t's key at D = 128, whole blocks, so that no block's scale crosses lanes
//   softmax       running maximum and sum per column; lane (q, g) holds the scores of the tokens 4 g .. 4 g + 3 of either 16
//   O^T += V^T P^T  the scores' registers are the operand as they are: the contraction runs over the tokens in the order in which the lanes
//                 hold them.  The values of four tokens lie side by side in the cache for that: 16 bytes are the lane's 4 tokens
//                 by 8 dimensions; pairs of tokens are formed by two byte permutations.  The weights go in as
//                 two bf16 terms: the matrix instructions are idle most of the time here.
// A part of the axis goes to a workgroup, whose four wavefronts take every fourth step and join in LDS; parts are joined
// by a second kernel, in order.  Masks are applied where a step reaches a row's limits only.  Tokens beyond the lengths may hold anything:
// their scores are replaced, and the exponents of their values cleared, so that a weight of 0 meets a finite number.
//
// Measured (64 / 8 heads of 128, parts + joining): 4 requests of 100003 tokens 99 + 5 us, the words at 4.6 TB/s (345 vector and 24 matrix
// instructions a step, 58 % of the cycles the former); 16 of up to 4096 17.5 + 4; 517 tokens of 32 heads in one part 10.
#include <algorithm>

#include "kv4_device.h"

namespace lqer {

namespace {

constexpr float kLog2e = 1.44269504088896340736f;

// ---- appending ------------------------------------------------------------------------------------------------------------
template <int TYPE>
__global__ __launch_bounds__(256) void kv4_append_kernel(Kv4AppendArgs a) {
    const int words = a.D / 8, per = a.heads * words;                  // words of a token's keys; as many of its values
    for (int64_t t = (int64_t)blockIdx.y * blockDim.y + threadIdx.y; t < a.T; t += (int64_t)gridDim.y * blockDim.y) {
        const int64_t slot = a.slots[t];
        if (slot < 0 || slot >= (a.pages << a.P_bits)) continue;       // (the same for both lanes of a block)
        const int off = (int)(slot & ((1 << a.P_bits) - 1));
        for (int e = blockIdx.x * blockDim.x + threadIdx.x; e < 2 * per; e += gridDim.x * blockDim.x) {
            const bool is_v = e >= per;
            const int x = is_v ? e - per : e, head = x / words, w = x - head * words;
            float v[8];
            const int64_t at = t * (is_v ? a.ldv : a.ldk) + (int64_t)8 * x;
            const void* src = is_v ? a.v : a.k;
            if (TYPE == LQER_F32) {
                const f32x4* p = reinterpret_cast<const f32x4*>((const float*)src + at);
                const f32x4 lo = p[0], hi = p[1];
#pragma unroll
                for (int i = 0; i < 4; ++i) { v[i] = lo[i]; v[4 + i] = hi[i]; }
            } else {
                const u32x4 b = *reinterpret_cast<const u32x4*>((const uint16_t*)src + at);
#pragma unroll
                for (int i = 0; i < 4; ++i) { v[2 * i] = f32_from_bits(b[i] << 16); v[2 * i + 1] = f32_from_bits(b[i] & 0xFFFF0000u); }
            }
            float m = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) m = __builtin_fmaxf(m, __builtin_fabsf(v[i]));
            m = __builtin_fmaxf(m, dpp_move<0xB1>(m));                 // quad_perm [1,0,3,2]: the block's other half
            const uint32_t eb = min((f32_bits(m) >> 23) & 0xFFu, 247u);
            uint32_t word = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float r = __builtin_rintf(__builtin_amdgcn_ldexpf(v[i], 2 + 127 - (int)eb));
                const uint32_t mag = (uint32_t)__builtin_fminf(__builtin_fabsf(r), 7.0f);
                const uint32_t neg = mag != 0 && r < 0.f ? 1u : 0u;
                if (i < 4) word |= (mag | neg << 7) << (8 * i);
                else word |= mag << (8 * (i - 4) + 4) | neg << (8 * ((i - 3) & 3) + 3);
            }
            const int64_t D = a.D;
            uint8_t* rec = a.pool + ((slot >> a.P_bits) * a.heads + head) * ((D * 9 / 8) << a.P_bits);
            if (is_v) {
                *reinterpret_cast<uint32_t*>(rec + ((D / 2) << a.P_bits) + ((int64_t)(off >> 2) * words + w) * 16 + (off & 3) * 4) = word;
                if ((w & 1) == 0) rec[((D + D / 16) << a.P_bits) + ((int64_t)(off >> 2) * (words / 2) + w / 2) * 4 + (off & 3)] = (uint8_t)eb;
            } else {
                *reinterpret_cast<uint32_t*>(rec + ((int64_t)off * words + w) * 4) = word;
                if ((w & 1) == 0) rec[(D << a.P_bits) + (int64_t)off * (words / 2) + w / 2] = (uint8_t)eb;
            }
        }
    }
}

// ---- attention of few rows --------------------------------------------------------------------------------------------------
template <int D>
struct Step {                                     // what a lane reads of 16 cached tokens
    static constexpr int KW = D / 32;             // words of a key, and their exponents
    static constexpr int VW = D >= 128 ? D / 128 : 1;
    u32x4 k[KW > 4 ? 2 : 1];
    u32x4 v[VW];
    uint32_t ke;
    uint32_t ve[VW];

    // rec, off: uniform; the lane's own offsets are small and the same for every step
    __device__ __forceinline__ void load(const uint8_t* rec, Kv4Record<D> R, int off, int i, int g) {
        const uint8_t* const kp = rec + R.key(off);
        const uint8_t* const ep = rec + R.key_exp(off);
        const uint32_t ko = (uint32_t)(i * (D / 2) + g * (D / 8)), eo = (uint32_t)(i * (D / 16) + g * (D / 64));
        if (D == 64) {
            const u32x2 w = *reinterpret_cast<const u32x2*>(kp + ko);
            k[0] = u32x4{w[0], w[1], 0, 0};
            ke = *(ep + eo);
        } else if (D == 128) {
            k[0] = *reinterpret_cast<const u32x4*>(kp + ko);
            ke = *reinterpret_cast<const uint16_t*>(ep + eo);
        } else {
            k[0] = *reinterpret_cast<const u32x4*>(kp + ko);
            k[KW > 4 ? 1 : 0] = *reinterpret_cast<const u32x4*>(kp + ko + 16);
            ke = *reinterpret_cast<const uint32_t*>(ep + eo);
        }
        const uint8_t* const vp = rec + R.value(off / 4);
        const uint8_t* const xp = rec + R.value_exp(off / 4);
#pragma unroll
        for (int h = 0; h < VW; ++h) {
            const uint32_t word = (uint32_t)(D == 64 ? i / 2 : 16 * h + i);
            v[h] = *reinterpret_cast<const u32x4*>(vp + (uint32_t)(g * (2 * D)) + word * 16);
            ve[h] = *reinterpret_cast<const uint32_t*>(xp + (uint32_t)(g * (D / 4)) + word / 2 * 4);
        }
    }
};

// Four tokens' words -> the halves (two tokens each) of the operands of `dims` output dimensions: half[x][p] = (token 2 p, token 2 p + 1) at
// dimension x of the lane's.
template <int D>
__device__ __forceinline__ void values_of_four(u32x4 w, uint32_t exps, int lane_i, uint32_t (&half)[D == 64 ? 4 : 8][2]) {
    constexpr int PAIRS = D == 64 ? 2 : 4;
    uint32_t t[4][PAIRS];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float s = kv4_scale((exps >> (8 * j)) & 0xFFu);
        const uint32_t r0 = (D == 64 && (lane_i & 1) ? __builtin_amdgcn_alignbit(w[j], w[j], 4) : w[j]) & 0x87878787u;
        t[j][0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(r0, s, false));
        t[j][1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(r0, s, true));
        if (D != 64) {
            const uint32_t r1 = __builtin_amdgcn_alignbit(w[j], w[j], 4) & 0x87878787u;
            t[j][PAIRS - 2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(r1, s, false));
            t[j][PAIRS - 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(r1, s, true));
        }
    }
#pragma unroll
    for (int x = 0; x < PAIRS; ++x)
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            half[2 * x][p] = __builtin_amdgcn_perm(t[2 * p + 1][x], t[2 * p][x], 0x05040100u);
            half[2 * x + 1][p] = __builtin_amdgcn_perm(t[2 * p + 1][x], t[2 * p][x], 0x07060302u);
        }
}

template <int D>
__global__ __launch_bounds__(256, D == 64 ? 4 : D == 128 ? 3 : 2) void kv4_few_kernel(Kv4Args a) {
    constexpr int KW = D / 32, NO = D / 16, WAVES = 4;
    __shared__ float join_o[WAVES][16][D + 4];
    __shared__ float join_m[WAVES][16], join_l[WAVES][16];
    // (the wavefront's number as a scalar: its steps, pages and their addresses are then computed once, not by every lane)
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 15, g = lane >> 4;
    const int head = blockIdx.x % a.sh.kv_heads, b = blockIdx.y, split = blockIdx.z;
    Kv4Rows r = kv4_request(a, b);
    if (!kv4_mine<false>(a, r)) return;
    const Kv4Record<D> R{a.P_bits};
    const int32_t* const table = a.table + (int64_t)b * a.sh.table_ld;
    // scores stay as the product gives them, the factor to units of log 2 goes into the exponential's multiply-add: a negative one turns the
    // queries' signs instead, so that the largest score is the largest weight
    // (0 as the smallest normal number: a masked score is minus infinity)
    const float to_log2 = __builtin_fmaxf(__builtin_fabsf(a.sh.scale) * kLog2e, 0x1p-126f);
    const uint32_t turn = a.sh.scale < 0.f ? 0x80008000u : 0u;
    for (int row0 = blockIdx.x / a.sh.kv_heads * 16; row0 < r.n * a.group; row0 += a.few.row_tiles * 16) {
        kv4_tile(a, r, row0, 16);
        int chunk;
        const int parts = kv4_parts<false>(a, r, chunk);
        if (split >= parts && split > 0) continue;
        // this lane's column
        const int row = r.row0 + min(i, r.rows - 1), query = row / a.group;
        const int64_t out_row = r.first + query;
        const int q_head = head * a.group + row - query * a.group;
        const int begin = kv4_row_begin(a, r, query), end = kv4_row_end(a, r, query);
        // what every row of the tile sees: from its last row's beginning to its first row's end
        const int all_begin = kv4_row_begin(a, r, (r.row0 + r.rows - 1) / a.group), all_end = kv4_row_end(a, r, r.row0 / a.group);
        const int lo = (r.lo & ~31) + split * chunk, hi = min(r.hi, lo + chunk);
        Frag q[KW];
        {
            const uint16_t* p = a.q + out_row * a.sh.ldq + (int64_t)q_head * D + g * (D / 4);
#pragma unroll
            for (int c = 0; c < KW; ++c) q[c].u = *reinterpret_cast<const u32x4*>(p + 8 * c) ^ turn;
        }
        f32x4 o[NO];
#pragma unroll
        for (int x = 0; x < NO; ++x) o[x] = f32x4{0.f, 0.f, 0.f, 0.f};
        float m = -__builtin_inff(), l = 0.f;

        int page_base = -(1 << 30), page_of_lane = -1;                 // 64 entries of the request's table, one to a lane
        const auto fetch = [&](int t0, Step<D> (&step)[2], bool (&there)[2]) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int t = t0 + 16 * h, index = t >> a.P_bits;
                if (index - page_base >= 64 || index < page_base) {
                    page_base = index;
                    page_of_lane = index + lane < a.sh.table_ld ? table[index + lane] : -1;
                }
                const int page = __builtin_amdgcn_readlane(page_of_lane, index - page_base);
                there[h] = page >= 0 && page < a.sh.pages;
                const uint8_t* rec = a.pool + ((int64_t)(there[h] ? page : 0) * a.sh.kv_heads + head) * R.bytes();
                step[h].load(rec, R, t & ((1 << a.P_bits) - 1), i, g);
            }
        };
        Step<D> next[2];
        bool next_there[2];
        if (lo + 32 * wave < hi) fetch(lo + 32 * wave, next, next_there);
        for (int t0 = lo + 32 * wave; t0 < hi; t0 += 32 * WAVES) {
            Step<D> step[2] = {next[0], next[1]};
            const bool there[2] = {next_there[0], next_there[1]};
            if (t0 + 32 * WAVES < hi) fetch(t0 + 32 * WAVES, next, next_there);    // while this step is computed
            f32x4 s[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                s[h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < KW; ++c)
                    s[h] = mfma16(unpack_w8(step[h].k[c / 4][c % 4], kv4_scale((step[h].ke >> (8 * (c / 2))) & 0xFFu)), q[c].v, s[h]);
            }
            if (!there[0] || !there[1] || t0 + 32 > all_end || t0 < all_begin) {
                // a step that reaches some row's limits: the values' exponents of tokens that no row sees, the scores that a row does not see
                int at = t0;
                asm volatile("" : "+s"(at));       // (a branch: left alone, the comparisons are done in every step and one of two results taken)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int t = at + 16 * h + 4 * g + j;
                        if (!there[h] || t >= r.hi || t < r.lo) {
#pragma unroll
                            for (int x = 0; x < Step<D>::VW; ++x) step[h].ve[x] &= ~(0xFFu << (8 * j));
                        }
                        if (!there[h] || t >= end || t < begin) s[h][j] = -__builtin_inff();
                    }
            }
            float top = m;
#pragma unroll
            for (int j = 0; j < 4; ++j) top = __builtin_fmaxf(top, __builtin_fmaxf(s[0][j], s[1][j]));
            top = quad_rows_max(top);
            if (__ballot(top != m)) {
                const float down = m == -__builtin_inff() ? 0.f : exp2_fast((m - top) * to_log2);
                l *= down;
#pragma unroll
                for (int x = 0; x < NO; ++x) o[x] *= down;
                m = top;
            }
            const float base = m == -__builtin_inff() ? 0.f : m * to_log2;
            Frag p, p2;                            // the weights in two bf16 terms
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int j = 0; j < 4; j += 2) {
                    const float e0 = exp2_fast(__builtin_fmaf(s[h][j], to_log2, -base));
                    const float e1 = exp2_fast(__builtin_fmaf(s[h][j + 1], to_log2, -base));
                    l += e0;
                    l += e1;
                    const uint32_t w = pack_bf16_near(e0, e1);
                    p.u[2 * h + j / 2] = w;
                    p2.u[2 * h + j / 2] = pack_bf16_near(e0 - f32_from_bits(w << 16), e1 - f32_from_bits(w & 0xFFFF0000u));
                }
#pragma unroll
            for (int x = 0; x < Step<D>::VW; ++x) {
                uint32_t va[D == 64 ? 4 : 8][2], vb[D == 64 ? 4 : 8][2];
                values_of_four<D>(step[0].v[x], step[0].ve[x], i, va);
                values_of_four<D>(step[1].v[x], step[1].ve[x], i, vb);
#pragma unroll
                for (int d = 0; d < (D == 64 ? 4 : 8); ++d) {
                    Frag f;
                    f.u = u32x4{va[d][0], va[d][1], vb[d][0], vb[d][1]};
                    o[8 * x + d] = mfma16(f.v, p2.v, o[8 * x + d]);
                    o[8 * x + d] = mfma16(f.v, p.v, o[8 * x + d]);
                }
            }
        }
        l = quad_rows_sum(l);
        // the wavefronts' parts, joined
        if (g == 0) {
            join_m[wave][i] = m == -__builtin_inff() ? m : m * to_log2;
            join_l[wave][i] = l;
        }
#pragma unroll
        for (int x = 0; x < NO; x += 4)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int d = D == 64 ? 16 * g + 4 * j : 128 * (x / 8) + 32 * g + 8 * j + x % 8;
                *reinterpret_cast<f32x4*>(&join_o[wave][i][d]) = f32x4{o[x][j], o[x + 1][j], o[x + 2][j], o[x + 3][j]};
            }
        __syncthreads();
        for (int e = threadIdx.x; e < r.rows * (D / 4); e += 256) {
            const int c = e / (D / 4), d = e % (D / 4) * 4;
            float top = join_m[0][c];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) top = __builtin_fmaxf(top, join_m[w][c]);
            f32x4 sum = {0.f, 0.f, 0.f, 0.f};
            float weights = 0.f;
            // (nothing seen: sums of 0; scores of NaN alone leave no maximum either, and sums of NaN)
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const float f = top > -__builtin_inff() ? exp2_fast(join_m[w][c] - top) : 1.0f;
                weights += f * join_l[w][c];
                sum += f * *reinterpret_cast<const f32x4*>(&join_o[w][c][d]);
            }
            const int rr = r.row0 + c, qu = rr / a.group;
            const int64_t orow = r.first + qu;
            const int h = head * a.group + rr - qu * a.group;
            if (parts > 1) {
                const int64_t at = kv4_part<false>(a, b, head, rr, orow, h) + split;
                *reinterpret_cast<f32x4*>(a.few.part_o + at * D + d) = sum;
                if (d == 0) a.few.part_ml[at] = float2{top, weights};
            } else {
                sum *= weights > 0.f ? 1.0f / weights : 0.f;
                const int64_t at = orow * a.sh.ldo + (int64_t)h * D + d;
                if (a.sh.out_type == LQER_F32) *reinterpret_cast<f32x4*>((float*)a.out + at) = sum;
                else *reinterpret_cast<u32x2*>((uint16_t*)a.out + at) = u32x2{pack_bf16_near(sum[0], sum[1]), pack_bf16_near(sum[2], sum[3])};
            }
        }
        __syncthreads();
    }
}

// The parts of every row, joined in order: WAVES wavefronts to a row.  A wavefront's lanes hold 4 dimensions of one part or of
// several neighbouring ones, the factors of up to 64 parts at a time lie in its lanes.
template <int D, int WAVES, bool MANY>
__global__ __launch_bounds__(256) void kv4_join_kernel(Kv4Args a) {
    constexpr int ROWS = MANY ? kManyRows : 16;
    const Kv4Plan& plan = MANY ? a.many : a.few;
    constexpr int LANES = D / 4, AT_ONCE = 64 / LANES;                 // lanes of a part, parts of a wavefront's load
    __shared__ f32x4 join[4][LANES];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), d = lane % LANES, sub = lane / LANES;
    const int head = blockIdx.x % a.sh.kv_heads, b = blockIdx.z;
    Kv4Rows r = kv4_request(a, b);
    if (!kv4_mine<MANY>(a, r)) return;
    for (int row0 = blockIdx.x / a.sh.kv_heads * ROWS; row0 < r.n * a.group; row0 += plan.row_tiles * ROWS) {
        kv4_tile(a, r, row0, ROWS);
        int chunk;
        const int parts = kv4_parts<MANY>(a, r, chunk);
        const int c = blockIdx.y * (4 / WAVES) + wave / WAVES;         // this wavefront's row of the tile
        if (parts <= 1) continue;                                      // (uniform over the workgroup: so is every barrier below)
        const bool on = c < r.rows;
        const int row = r.row0 + min(c, r.rows - 1), query = row / a.group;
        const int64_t orow = r.first + query;
        const int h = head * a.group + row - query * a.group;
        const int64_t at = kv4_part<MANY>(a, b, head, row, orow, h);
        const f32x4* const po = reinterpret_cast<const f32x4*>(plan.part_o + at * D) + d;
        float top = -__builtin_inff();
        for (int s = lane; s < parts; s += 64) top = __builtin_fmaxf(top, plan.part_ml[at + s].x);
        top = wave_max(top);
        f32x4 sum = {0.f, 0.f, 0.f, 0.f};
        float weights = 0.f;
        for (int s0 = 0; s0 < parts; s0 += 64) {
            float f = 0.f;
            if (s0 + lane < parts) {
                const float2 ml = plan.part_ml[at + s0 + lane];
                f = ml.x > -__builtin_inff() ? exp2_fast(ml.x - top) : 0.f;
                weights += f * ml.y;
            }
            const int here = min(64, parts - s0);
            for (int s = AT_ONCE * (wave % WAVES); s < here; s += 4 * AT_ONCE * WAVES) {
                f32x4 v[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int p = min(s + u * AT_ONCE * WAVES + sub, here - 1);
                    v[u] = po[(int64_t)(s0 + p) * LANES];
                }
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int p = s + u * AT_ONCE * WAVES + sub;
                    const float w = __shfl(f, p & 63);
                    if (p < here) sum += w * v[u];
                }
            }
        }
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) weights += __shfl_xor(weights, m);
#pragma unroll
        for (int m = LANES; m < 64; m <<= 1)
#pragma unroll
            for (int j = 0; j < 4; ++j) sum[j] += __shfl_xor(sum[j], m);
        if (WAVES > 1) {
            if (sub == 0) join[wave][d] = sum;
            __syncthreads();
            sum = join[0][d];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) sum += join[w][d];
            __syncthreads();
        }
        if (!on || sub != 0 || wave % WAVES != 0) continue;
        sum *= weights > 0.f ? 1.0f / weights : 0.f;
        const int64_t o = orow * a.sh.ldo + (int64_t)h * D + 4 * d;
        if (a.sh.out_type == LQER_F32) *reinterpret_cast<f32x4*>((float*)a.out + o) = sum;
        else *reinterpret_cast<u32x2*>((uint16_t*)a.out + o) = u32x2{pack_bf16_near(sum[0], sum[1]), pack_bf16_near(sum[2], sum[3])};
    }
}

// a workgroup to a row where it may have many parts, a wavefront otherwise
template <int D, bool MANY>
hipError_t join(const Kv4Args& a, hipStream_t s) {
    const Kv4Plan& plan = MANY ? a.many : a.few;
    const unsigned rows = MANY ? kManyRows : 16;
    const dim3 grid((unsigned)(plan.row_tiles * a.sh.kv_heads), plan.splits > 8 ? rows : rows / 4, (unsigned)a.sh.n_requests);
    if (plan.splits > 8) hipLaunchKernelGGL((kv4_join_kernel<D, 4, MANY>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((kv4_join_kernel<D, 1, MANY>), grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

template <int D>
hipError_t launch_d(const Kv4Args& a, hipStream_t s) {
    if (a.many.run) {
        hipError_t e = launch_kv4_many(a, s);
        if (e == hipSuccess && a.many.splits > 1) e = join<D, true>(a, s);
        if (e != hipSuccess) return e;
    }
    if (!a.few.run) return hipSuccess;
    // (parts outermost: those that only the longest requests have come last, and what is at work is spread evenly)
    const dim3 grid((unsigned)(a.few.row_tiles * a.sh.kv_heads), (unsigned)a.sh.n_requests, (unsigned)a.few.splits);
    hipLaunchKernelGGL((kv4_few_kernel<D>), grid, dim3(256), 0, s, a);
    if (hipError_t e = hipGetLastError(); e != hipSuccess || a.few.splits == 1) return e;
    return join<D, false>(a, s);
}

// Up to so many cached tokens a workgroup of the kernel for few rows takes all of them, five steps a wavefront, ten where the launch has 128 workgroups
// and more: about as long as parts of one step and the launch that joins them, and one launch less for the host (us in a graph, whole / parts: 517 tokens
// of 32 heads 12 / 12; 37 requests of up to 1036 tokens 18 / 18; one of 1200 with a single cached head 17 / 12).
constexpr int64_t kWholeTokens = 640;

// The cached tokens of `lots` tiles cut into parts: `least` tokens at least, and no more than give `wanted` workgroups, all at work at once.
void cut(Kv4Plan& p, int64_t seen, int64_t lots, int64_t least, int64_t wanted) {
    int64_t chunk = std::max(least, (seen * lots / wanted + 127) / 128 * 128);
    if (chunk > (1 << 30)) chunk = 1 << 30;
    p.chunk = (int)chunk;
    p.splits = (int)std::min<int64_t>((seen + chunk - 1) / chunk, 65535);
}

}  // namespace

hipError_t launch_kv4_append(const Kv4AppendArgs& a, hipStream_t s) {
    const int items = 2 * a.heads * (a.D / 8);
    const int x = items >= 256 ? 256 : items > 64 ? 128 : items > 32 ? 64 : 32, y = 256 / x;
    int64_t gy = (a.T + y - 1) / y;
    if (gy > 65535) gy = 65535;
    const dim3 grid((unsigned)((items + x - 1) / x), (unsigned)gy), block((unsigned)x, (unsigned)y);
    if (a.type == LQER_F32) hipLaunchKernelGGL((kv4_append_kernel<LQER_F32>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((kv4_append_kernel<LQER_BF16>), grid, block, 0, s, a);
    return hipGetLastError();
}

size_t plan_kv4(Kv4Args& a, void* workspace) {
    const lqer_kv4_shape& sh = a.sh;
    a.group = sh.q_heads / sh.kv_heads;
    a.P_bits = __builtin_ctz((unsigned)sh.page_tokens);
    a.few_rows = kFewRows;
    const int64_t rows = (int64_t)sh.max_q * a.group, most_tiles = 65535 / sh.kv_heads;
    const auto tiles = [&](int64_t n, int64_t of) { return (int)std::max<int64_t>(1, std::min<int64_t>((n + of - 1) / of, most_tiles)); };
    a.many = Kv4Plan{};
    a.few = Kv4Plan{};
    a.many.run = rows > kFewRows;
    // Beside the kernel for many rows the one for few runs whenever some request may have few: the lengths are on the device, Tq counts rows that no request
    // has, and max_q is an estimate.  (A single request is taken to be as long as max_q says, unless q has not so many rows.)
    a.few.run = !a.many.run || sh.n_requests > 1 || sh.Tq < sh.max_q;
    a.many.row_tiles = tiles(rows, kManyRows);
    a.few.cap = (int)std::max<int64_t>(1, std::min<int64_t>(rows, kFewRows));
    a.few.row_tiles = tiles(a.few.cap, 16);
    int64_t seen = std::max(sh.max_kv, 1);
    if (sh.window > 0) seen = std::min<int64_t>(seen, (int64_t)sh.window + sh.max_q + 31);
    const int64_t heads = (int64_t)sh.n_requests * sh.kv_heads;
    // 128 tokens are a step of 32 for each wavefront of a workgroup, 512 are eight tiles of a workgroup for many rows: those keep two
    // workgroups to a compute unit, the others three: 768.  Short parts of few rows (up to nine steps a wavefront) are cut a little finer: where the
    // requests' lengths differ many of the 768 have nothing to do (us, 1024 / 768: 16 requests of up to 4096 tokens 24 / 28, all of 4096 30 / 30, 8 of up to
    // 12538 32 / 36; long ones not: 4 of 100003 110 / 103), but not below two steps, which the joining would outweigh (one of 16000 17 / 14).
    const int64_t lots = heads * a.few.row_tiles;
    if (seen <= (lots >= 128 ? 2 * kWholeTokens : kWholeTokens)) cut(a.few, seen, lots, seen, 768);
    else if (cut(a.few, seen, lots, 128, 768); a.few.chunk <= 1152) cut(a.few, seen, lots, 256, 1024);
    cut(a.many, seen, heads * a.many.row_tiles, 512, 512);
    size_t at = 0;
    const auto place = [&](Kv4Plan& p, int64_t n) {
        if (!p.run) return;
        // (what the parts write and the join reads is bounded: the parts' sums are fp32)
        while (p.splits > 1 && p.splits * n * sh.head_dim * 4 > ((int64_t)256 << 20)) p.splits = (p.splits + 1) / 2;
        if (p.splits == 1) return;
        n *= p.splits;
        p.part_o = (float*)((uint8_t*)workspace + at);
        p.part_ml = (float2*)((uint8_t*)workspace + at + n * sh.head_dim * 4);
        at += (size_t)(n * (sh.head_dim * 4 + 8) + 255) / 256 * 256;
    };
    place(a.few, heads * a.few.cap);
    place(a.many, sh.Tq * sh.q_heads);
    return at;
}

hipError_t launch_kv4_attention(const Kv4Args& a, hipStream_t s) {
    if (a.sh.head_dim == 64) return launch_d<64>(a, s);
    return a.sh.head_dim == 128 ? launch_d<128>(a, s) : launch_d<256>(a, s);
}

}  // namespace lqer
