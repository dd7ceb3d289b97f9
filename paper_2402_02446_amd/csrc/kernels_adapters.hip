// Low-rank adapters of many requests beside one layer: Y[m] += s_a (X[m] A_a^T) B_a^T with a = ids[m].
//
// Two products with a group of tokens of one adapter each: the projection T = X A^T (K long, R wide), split along K so that few groups fill the
// chip too, its partial sums in the workspace; and Y + T B^T, which adds the partial sums of its group's T up, in order.  What
// bounds them: with few tokens the bytes of the A and B of the adapters in the batch, each read by one group; with many the
// bytes of X and of Y in and out.
//
// Groups.  Up to 64 tokens a wavefront of every workgroup finds the groups that there are by itself, through a table in LDS; the workgroups are shared out
// among the groups.  Beyond, one workgroup sorts the tokens by adapter first
// and lists tiles of up to 16 or 64 of them.  Tokens without an adapter are a group of rank 0: their rows are copied.
//
// Matrix instructions: 16 x 16 x 32 bf16.  Projection: ranks as rows and tokens as columns, so that a lane holds four neighbouring ranks
// of one token.  Second product: tokens as rows and as columns every NT-th output column, so that a lane holds NT neighbouring columns
// and 16 lanes a run of them: Y is read and written in whole cache lines.  The K axis is permuted in chunks of 64, where a lane group owns 32
// contiguous bytes of a row.  T goes into the second product as three bf16 terms (24 bits): X, A and B are bf16, so every product is
// exact and the sums are fp32.
//
// Measured (projection + second product, us): 16 tokens of 4096 x 4096 rank 16 3.8 + 5.1; 64 of 8192 x 28672 with 48 adapters of up to 64 ranks
// 7.6 + 24, B's lines at 5.3 TB/s; 203 of 4112 x 11000 5.2 + 7.3, sorting 3.6; 4096 of 8192 x 28672 rank 32 26 + 192, Y at 4.9 TB/s, sorting 8.
#include "serve.h"
#include "mx_device.h"

namespace lqer {

namespace {

constexpr int64_t kNarrowTokens = 1024;  // most tokens that are sorted into tiles of 16
constexpr int kWide = 64;              // most tokens of a tile; and the calls whose tokens need no sorting

struct Group {
    int adapter;                       // -1: none
    int count;                         // tokens
    int part, parts;                   // this workgroup's share of the group's work; part >= parts: nothing to do
};

__device__ __forceinline__ int adapter_of(const AdapterArgs& a, int64_t m) {
    const int id = a.ids[m];
    return id >= 0 && id < a.n ? id : -1;
}

// What the lanes of a wavefront stored in LDS before is there for all of them.
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// What this workgroup works on, and its group's tokens in rows[] (LDS).  Uniform over the workgroup; holds barriers.
// Without sorting, parts = 0: all workgroups are shared out evenly among the groups that there are; otherwise `parts` to each group or tile.
template <bool SORTED>
__device__ __forceinline__ Group find_group(const AdapterArgs& a, int parts, int* rows) {
    __shared__ Group found;
    if (!SORTED) {
        __shared__ uint8_t seen[kMaxAdapters + 1];
        __shared__ int lowest[kWide];
        if (threadIdx.x < 64) {
            const int lane = threadIdx.x;
            const bool in = lane < a.M;
            const int id = in ? adapter_of(a, lane) : -2, at = id < 0 ? a.n : id;
            // The tokens of an adapter find one and the same of them in the table, whichever that is; the lowest of those that found it leads the group, so that the
            // groups have the same order in every workgroup.
            lowest[lane] = kWide;
            if (in) __hip_atomic_store(&seen[at], (uint8_t)lane, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
            wave_sync();
            const int met = in ? __hip_atomic_load(&seen[at], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP) : 0;
            if (in) atomicMin(&lowest[met], lane);
            wave_sync();
            const uint64_t firsts = __ballot(in && lowest[met] == lane);
            const int groups = (int)__popcll(firsts);
            const bool mine = ((firsts >> lane) & 1) && (int)__popcll(firsts & ((1ull << lane) - 1)) == (int)(blockIdx.x % groups);
            const int adapter = __builtin_amdgcn_readlane(id, (int)__builtin_ctzll(__ballot(mine)));
            const uint64_t same = __ballot(id == adapter);
            if (id == adapter) rows[__popcll(same & ((1ull << lane) - 1))] = lane;
            if (lane == 0) found = Group{adapter, (int)__popcll(same), (int)(blockIdx.x / groups), parts > 0 ? parts : (int)(gridDim.x / groups)};
        }
    } else {
        const int tile = (int)(blockIdx.x / parts);
        if (tile >= a.list[0]) return {-1, 0, 0, 0};
        const AdapterTile t = a.tiles[tile];
        if ((int)threadIdx.x < t.count) rows[threadIdx.x] = a.order[t.start + threadIdx.x];
        if (threadIdx.x == 0) found = Group{t.adapter, t.count, (int)(blockIdx.x % parts), parts};
    }
    __syncthreads();
    return found;
}

__device__ __forceinline__ int rank_of(const AdapterArgs& a, int adapter) {
    if (adapter < 0) return 0;
    return a.ranks ? min(max(a.ranks[adapter], 0), a.R) : a.R;
}

// T[split][token][rank]: RT tiles of 16 ranks, up to 16 tokens at a time; the four wavefronts share the chunks of K.
template <int RT, bool SORTED>
__global__ __launch_bounds__(256) void adapter_project_kernel(AdapterArgs a) {
    __shared__ int rows[kWide];
    __shared__ f32x4 part[4 * RT * 64];
    const Group gr = find_group<SORTED>(a, a.splits, rows);
    const int rank = rank_of(a, gr.adapter);
    if (gr.part >= gr.parts || rank == 0) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, g = lane >> 4;
    const int64_t per = a.k_split, k_lo = gr.part * per, k_hi = min(a.K, k_lo + per);
    const uint16_t* const A = a.A + (int64_t)gr.adapter * a.R * a.K;
    float* const T = a.T + (int64_t)gr.part * a.M * a.Rp;
    for (int t0 = 0; t0 < gr.count; t0 += 16) {
        const int64_t row = rows[min(t0 + i, gr.count - 1)];
        const uint16_t* const x = a.X + row * a.ldx;
        f32x4 acc[RT];
#pragma unroll
        for (int r = 0; r < RT; ++r) acc[r] = f32x4{0.f, 0.f, 0.f, 0.f};
        // AHEAD chunks' loads are issued before the first one's products
        constexpr int AHEAD = RT <= 2 ? 4 : RT == 4 ? 2 : 1;
        for (int64_t k0 = k_lo + 64 * wave; k0 < k_hi; k0 += AHEAD * 256) {
            Frag xf[AHEAD][2], af[AHEAD][2][RT];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int64_t k = k0 + u * 256 + 16 * g + 8 * h;
                    const bool in = k < k_hi;
                    xf[u][h].u = u32x4{0, 0, 0, 0};
                    if (in) xf[u][h].u = *reinterpret_cast<const u32x4*>(x + k);
#pragma unroll
                    for (int r = 0; r < RT; ++r) {
                        af[u][h][r].u = u32x4{0, 0, 0, 0};
                        if (in && 16 * r + i < rank) af[u][h][r].u = *reinterpret_cast<const u32x4*>(A + (int64_t)(16 * r + i) * a.K + k);
                    }
                }
#pragma unroll
            for (int u = 0; u < AHEAD; ++u)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int r = 0; r < RT; ++r) acc[r] = mfma16(af[u][h][r].v, xf[u][h].v, acc[r]);
        }
        // the wavefronts' sums, in order
#pragma unroll
        for (int r = 0; r < RT; ++r) part[(wave * RT + r) * 64 + lane] = acc[r];
        __syncthreads();
        for (int r = wave; r < RT; r += 4) {
            f32x4 s = part[r * 64 + lane];
#pragma unroll
            for (int w = 1; w < 4; ++w) s += part[(w * RT + r) * 64 + lane];
            if (t0 + i < gr.count && 16 * r + 4 * g < a.Rp) *reinterpret_cast<f32x4*>(T + row * a.Rp + 16 * r + 4 * g) = s;
        }
        __syncthreads();
    }
}

// The same for tiles of 64 tokens, 16 to a wavefront.  Stages of CK values of K go through LDS: neighbouring lanes load neighbouring 16 bytes of a row
// (the operands' own order, one row a lane, would be the address unit's worst case: 38 us for 4096 tokens of 8192 values and rank 32), and A is
// read once for all four wavefronts.  The 16-byte cells of row r change places by the low bits of r, off the same banks.
template <int RT>
__global__ __launch_bounds__(256) void adapter_project_wide_kernel(AdapterArgs a) {
    constexpr int CK = RT == 8 ? 64 : 128, C = CK / 8;             // cells of a row
    constexpr int XN = kWide * C / 256, AN = (16 * RT * C + 255) / 256;
    __shared__ int rows[kWide];
    __shared__ u32x4 stage[2][(kWide + 16 * RT) * C];
    const Group gr = find_group<true>(a, a.splits, rows);
    const int rank = rank_of(a, gr.adapter);
    if (gr.part >= gr.parts || rank == 0) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, i = lane & 15, g = lane >> 4;
    const int64_t k_lo = gr.part * a.k_split, k_hi = min(a.K, k_lo + a.k_split);
    const int c = tid % C, r0 = tid / C;                           // this thread's cell of the rows r0, r0 + 256 / C ..
    const uint16_t* const A = a.A + (int64_t)gr.adapter * a.R * a.K + 8 * c;
    const uint16_t* x[XN];
#pragma unroll
    for (int n = 0; n < XN; ++n) x[n] = a.X + rows[min(r0 + n * (256 / C), gr.count - 1)] * a.ldx + 8 * c;
    u32x4 xv[XN], av[AN];
    const auto load = [&](int64_t k) {
        const bool in = k + 8 * c < k_hi;
#pragma unroll
        for (int n = 0; n < XN; ++n) {
            xv[n] = u32x4{0, 0, 0, 0};
            if (in) xv[n] = *reinterpret_cast<const u32x4*>(x[n] + k);
        }
#pragma unroll
        for (int n = 0; n < AN; ++n) {
            const int r = r0 + n * (256 / C);
            av[n] = u32x4{0, 0, 0, 0};
            if (in && r < rank) av[n] = *reinterpret_cast<const u32x4*>(A + (int64_t)r * a.K + k);
        }
    };
    f32x4 acc[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) acc[r] = f32x4{0.f, 0.f, 0.f, 0.f};
    load(k_lo);
    int buf = 0;
    for (int64_t k0 = k_lo; k0 < k_hi; k0 += CK, buf ^= 1) {
        u32x4* const xs = stage[buf];
        u32x4* const as = stage[buf] + kWide * C;
#pragma unroll
        for (int n = 0; n < XN; ++n) {
            const int r = r0 + n * (256 / C);
            xs[r * C + (c ^ (r & 7))] = xv[n];
        }
#pragma unroll
        for (int n = 0; n < AN; ++n) {
            const int r = r0 + n * (256 / C);
            if (r < 16 * RT) as[r * C + (c ^ (r & 7))] = av[n];
        }
        if (k0 + CK < k_hi) load(k0 + CK);
        __syncthreads();                   // (the other buffer was last read before the barrier of the stage before)
        if (16 * wave >= gr.count) continue;
#pragma unroll
        for (int s = 0; s < CK / 32; ++s) {
            const int cell = (4 * s + g) ^ (i & 7);
            Frag xf, af[RT];
            xf.u = xs[(16 * wave + i) * C + cell];
#pragma unroll
            for (int r = 0; r < RT; ++r) af[r].u = as[(16 * r + i) * C + cell];
#pragma unroll
            for (int r = 0; r < RT; ++r) acc[r] = mfma16(af[r].v, xf.v, acc[r]);
        }
    }
    if (16 * wave + i >= gr.count) return;
    float* const T = a.T + ((int64_t)gr.part * a.M + rows[16 * wave + i]) * a.Rp + 4 * g;
#pragma unroll
    for (int r = 0; r < RT; ++r)
        if (16 * r + 4 * g < a.Rp) *reinterpret_cast<f32x4*>(T + 16 * r) = acc[r];
}

// Y_out = Y_in + T B^T of one group and several blocks of 64 NT output columns; KK steps of 32 ranks.
template <int KK, int NT>
struct Columns {                                           // a wavefront's B: NT tiles of 16 columns, every NT-th one from the t-th on
    Frag b[NT][KK];
    __device__ __forceinline__ void load(const AdapterArgs& a, const uint16_t* B, int64_t n0, int rank, int i, int g) {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int k = 0; k < KK; ++k) {
                const int64_t n = n0 + NT * i + t;
                const int r = 32 * k + 8 * g;
                b[t][k].u = u32x4{0, 0, 0, 0};
                if (n < a.N && r < rank) b[t][k].u = *reinterpret_cast<const u32x4*>(B + n * a.R + r);
            }
    }
    // what lies beyond the rank in its last eight may be anything
    __device__ __forceinline__ void cut(int rank, int g) {
        if ((rank & 7) == 0) return;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int k = 0; k < KK; ++k) {
                const int left = rank - 32 * k - 8 * g;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (2 * j + 1 >= left) b[t][k].u[j] &= 2 * j >= left ? 0u : 0xFFFFu;
            }
    }
};

// A lane's NT neighbouring columns of the four rows 4 g .. 4 g + 3 of a step's 16 tokens: 16 lanes are NT cache lines of a row.
template <int NT>
struct FourRows {
    float y[4][NT];
    typedef float vec __attribute__((ext_vector_type(NT)));

    // rows: the step's tokens, `count` of them
    template <bool STORE, typename P>
    __device__ __forceinline__ void move(P* base, int64_t ld, const int* rows, int count, int64_t n, int64_t N, int g) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (4 * g + j >= count) continue;
            P* p = base + rows[4 * g + j] * ld + n;
            if (n + NT <= N) {
                if constexpr (STORE) {
                    vec v;
#pragma unroll
                    for (int t = 0; t < NT; ++t) v[t] = y[j][t];
                    *reinterpret_cast<vec*>(p) = v;
                } else {
                    const vec v = *reinterpret_cast<const vec*>(p);
#pragma unroll
                    for (int t = 0; t < NT; ++t) y[j][t] = v[t];
                }
            } else {
#pragma unroll
                for (int t = 0; t < NT; ++t)
                    if (n + t < N) {
                        if constexpr (STORE) p[t] = y[j][t];
                        else y[j][t] = p[t];
                    }
            }
        }
    }
};

template <int KK, int NT, bool SORTED, bool WIDE>
__global__ __launch_bounds__(256) void adapter_expand_kernel(AdapterArgs a) {
    constexpr int TROWS = WIDE ? kWide : 16;
    constexpr int LD = 32 * KK + 8;                        // (a row's length in LDS: 16 bytes more than its ranks, off the same banks)
    __shared__ int rows[kWide];
    __shared__ __align__(16) uint16_t terms[3][TROWS][LD];
    const Group gr = find_group<SORTED>(a, SORTED ? a.parts : 0, rows);
    const int blocks = (int)((a.N + 64 * NT - 1) / (64 * NT));
    const int columns = gr.parts > 0 ? (blocks + gr.parts - 1) / gr.parts : 0;
    if (gr.part >= gr.parts || (int64_t)gr.part * columns >= blocks) return;
    const int rank = rank_of(a, gr.adapter);
    if (rank == 0 && a.Y_in == a.Y_out) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, g = lane >> 4;
    const int64_t first = ((int64_t)gr.part * columns * 4 + wave) * 16 * NT;
    const uint16_t* const B = a.B + (int64_t)(gr.adapter < 0 ? 0 : gr.adapter) * a.N * a.R;
    Columns<KK, NT> next;                                  // what comes from far away first
    next.load(a, B, first, rank, i, g);
    const float scale = rank > 0 && a.scales ? a.scales[gr.adapter] : 1.0f;
    FourRows<NT> y_next;
    y_next.template move<false>(a.Y_in, a.ldyi, rows, min(gr.count, 16), first + NT * i, a.N, g);
    for (int t0 = 0; t0 < gr.count; t0 += TROWS) {
        const int here = min(gr.count - t0, TROWS);
        if (rank > 0) {
            // T: the parts' sums, in order, eight loads at a time; its three bf16 terms
            for (int e = threadIdx.x; e < here * 8 * KK; e += 256) {
                const int t = e / (8 * KK), r = e % (8 * KK) * 4;
                f32x4 v = {0.f, 0.f, 0.f, 0.f};
                if (r < rank) {
                    const float* p = a.T + (int64_t)rows[t0 + t] * a.Rp + r;
                    for (int s0 = 0; s0 < a.splits; s0 += 8) {
                        f32x4 x[8];
#pragma unroll
                        for (int s = 0; s < 8; ++s) x[s] = *reinterpret_cast<const f32x4*>(p + (int64_t)min(s0 + s, a.splits - 1) * a.M * a.Rp);
#pragma unroll
                        for (int s = 0; s < 8; ++s)
                            if (s0 + s < a.splits) v += x[s];
                    }
                }
                uint32_t w[3][2];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float f = r + j < rank ? v[j] * scale : 0.f;
                    // cut off after 8 bits each, which is as exact as rounding and never rounds to infinity; an infinity has no rest
                    const float t1 = f32_from_bits(f32_bits(f) & 0xFFFF0000u);
                    const float f2 = __builtin_fabsf(f) < __builtin_inff() ? f - t1 : 0.f;
                    const float t2 = f32_from_bits(f32_bits(f2) & 0xFFFF0000u);
                    const uint32_t u[3] = {f32_bits(t1) >> 16, f32_bits(t2) >> 16, f32_bits(f2 - t2) >> 16};
#pragma unroll
                    for (int q = 0; q < 3; ++q) w[q][j >> 1] = j & 1 ? w[q][j >> 1] | u[q] << 16 : u[q];
                }
#pragma unroll
                for (int q = 0; q < 3; ++q) *reinterpret_cast<u32x2*>(&terms[q][t][r]) = u32x2{w[q][0], w[q][1]};
            }
            __syncthreads();
        }
        // steps of 16 tokens by this wavefront's columns, block by block; a step's Y is loaded during the one before, a block's B during
        // the whole block before
        if (t0 > 0) y_next.template move<false>(a.Y_in, a.ldyi, rows + t0, min(here, 16), first + NT * i, a.N, g);
        Columns<KK, NT> now = next;
        for (int c = 0, tt = 0; c < columns;) {
            const int64_t n0 = first + (int64_t)c * 64 * NT;
            if (n0 >= a.N) break;                          // (of this wavefront alone: no barrier below)
            if (tt == 0) {
                now = next;
                now.cut(rank, g);
                const bool more = c + 1 < columns && n0 + 64 * NT < a.N;       // (the last workgroups' share may end before)
                if (more || t0 + TROWS < gr.count) next.load(a, B, more ? n0 + 64 * NT : first, rank, i, g);
            }
            FourRows<NT> y = y_next;
            const int tile = tt;
            tt += 16;
            if (tt >= here) { tt = 0; ++c; }
            if (c < columns)
                y_next.template move<false>(a.Y_in, a.ldyi, rows + t0 + tt, min(here - tt, 16), first + (int64_t)c * 64 * NT + NT * i, a.N, g);
            if (rank > 0) {
                f32x4 acc[NT];
#pragma unroll
                for (int t = 0; t < NT; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int q = 2; q >= 0; --q)
#pragma unroll
                    for (int k = 0; k < KK; ++k) {
                        Frag f;
                        f.u = *reinterpret_cast<const u32x4*>(&terms[q][tile + i][32 * k + 8 * g]);
#pragma unroll
                        for (int t = 0; t < NT; ++t) acc[t] = mfma16(f.v, now.b[t][k].v, acc[t]);
                    }
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int j = 0; j < 4; ++j) y.y[j][t] += acc[t][j];
            }
            y.template move<true>(a.Y_out, a.ldyo, rows + t0 + tile, min(here - tile, 16), n0 + NT * i, a.N, g);
        }
        __syncthreads();
    }
}

// A place in the count of a lane's adapter (id; -2: no token).  Lanes that all have the same one, as in prompts, take theirs with one
// atomic: 64 on one address wait for each other.
__device__ __forceinline__ int take_place(int* count, int n, int id) {
    const int lane = threadIdx.x & 63;
    const uint64_t in = __ballot(id != -2);
    if (in == 0) return 0;
    const int lead = (int)__builtin_ctzll(in), first = __builtin_amdgcn_readlane(id, lead);
    if (__ballot(id == first) == in) {
        int base = 0;
        if (lane == lead) base = atomicAdd(&count[first < 0 ? n : first], (int)__popcll(in));
        return __builtin_amdgcn_readlane(base, lead) + (int)__popcll(in & ((1ull << lane) - 1));
    }
    return id != -2 ? atomicAdd(&count[id < 0 ? n : id], 1) : 0;
}

// Tokens in the order of their adapters (those without one last) and the tiles of up to 64 of them: one workgroup.  The order
// within an adapter is that of the atomics' arrival; a token's result does not depend on its place.  Up to 8192 tokens each has its place
// in its adapter's count from the counting itself; beyond, they are read and counted again once the counts' sums are known.
__global__ __launch_bounds__(1024) void adapter_sort_kernel(AdapterArgs a) {
    extern __shared__ int count[];                         // [n + 1], then where each adapter's next token goes
    __shared__ int sums[2][16];
    constexpr int EACH = 8;                                // tokens of a thread at a time: their loads go out together
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6, bins = a.n + 1;
    for (int b = t; b < bins; b += 1024) count[b] = 0;
    int bin[EACH], place[EACH];
    __syncthreads();
    for (int64_t m0 = 0; m0 < a.M; m0 += 1024 * EACH) {
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int64_t m = m0 + 1024 * e + t;
            bin[e] = m < a.M ? adapter_of(a, m) : -2;
        }
#pragma unroll
        for (int e = 0; e < EACH; ++e) place[e] = take_place(count, a.n, bin[e]);
    }
    __syncthreads();
    const int each = (bins + 1023) / 1024, b0 = min(t * each, bins), b1 = min(b0 + each, bins);
    int tokens = 0, tiles = 0;
    for (int b = b0; b < b1; ++b) {
        tokens += count[b];
        tiles += (count[b] + a.tile - 1) / a.tile;
    }
    int before_tokens = tokens, before_tiles = tiles;      // sums over the threads before this one
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int x = __shfl_up(before_tokens, d), y = __shfl_up(before_tiles, d);
        if (lane >= d) { before_tokens += x; before_tiles += y; }
    }
    if (lane == 63) { sums[0][wave] = before_tokens; sums[1][wave] = before_tiles; }
    before_tokens -= tokens;
    before_tiles -= tiles;
    __syncthreads();
    int all = 0;
    for (int w = 0; w < 16; ++w) {
        if (w < wave) { before_tokens += sums[0][w]; before_tiles += sums[1][w]; }
        all += sums[1][w];
    }
    if (t == 0) a.list[0] = all;
    for (int b = b0; b < b1; ++b) {
        const int c = count[b];
        count[b] = before_tokens;
        for (int s = 0; s < c; s += a.tile)
            a.tiles[before_tiles++] = AdapterTile{b < a.n ? b : -1, before_tokens + s, min(c - s, a.tile), 0};
        before_tokens += c;
    }
    __syncthreads();
    if (a.M <= 1024 * EACH) {
#pragma unroll
        for (int e = 0; e < EACH; ++e)
            if (bin[e] != -2) a.order[count[bin[e] < 0 ? a.n : bin[e]] + place[e]] = 1024 * e + t;
        return;
    }
    for (int64_t m0 = 0; m0 < a.M; m0 += 1024 * EACH) {
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int64_t m = m0 + 1024 * e + t;
            bin[e] = m < a.M ? adapter_of(a, m) : -2;
        }
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int at = take_place(count, a.n, bin[e]);
            if (bin[e] != -2) a.order[at] = (int)(m0 + 1024 * e + t);
        }
    }
}

// the most groups (few tokens) or tiles that there can be
int64_t most_groups(const AdapterArgs& a) { return a.tile == 0 ? a.M : a.M / a.tile + (a.M < a.n + 1 ? a.M : a.n + 1); }

template <int RT>
hipError_t project(const AdapterArgs& a, hipStream_t s) {
    const dim3 grid((unsigned)(most_groups(a) * a.splits));
    if (a.tile == 0) hipLaunchKernelGGL((adapter_project_kernel<RT, false>), grid, dim3(256), 0, s, a);
    else if (a.tile < kWide) hipLaunchKernelGGL((adapter_project_kernel<RT, true>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((adapter_project_wide_kernel<RT>), grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

// A workgroup takes several blocks of columns one after another, T summed up once for all, where about eight workgroups
// to a compute unit are left (few tokens: four, which share the groups that there are out evenly).
template <int KK, int NT, bool SORTED, bool WIDE>
hipError_t expand(AdapterArgs a, hipStream_t s) {
    const int64_t blocks = (a.N + 64 * NT - 1) / (64 * NT), groups = most_groups(a);
    int64_t grid = groups * blocks;
    if (!SORTED) {
        if (grid > 1024) grid = 1024;              // (more than groups: M <= 64)
    } else {
        int64_t columns = grid / 2048;
        columns = columns < 1 ? 1 : columns > blocks ? blocks : columns;
        a.parts = (int)((blocks + columns - 1) / columns);
        grid = groups * a.parts;
    }
    hipLaunchKernelGGL((adapter_expand_kernel<KK, NT, SORTED, WIDE>), dim3((unsigned)grid), dim3(256), 0, s, a);
    return hipGetLastError();
}

template <int KK>
hipError_t expand(const AdapterArgs& a, hipStream_t s) {
    // (ranks above 64: fewer columns, or their B leaves one wavefront a SIMD)
    if (a.tile == kWide) return expand<KK, KK == 4 ? 2 : 4, true, true>(a, s);
    if (a.tile > 0) return expand<KK, KK == 4 ? 2 : 4, true, false>(a, s);
    return a.M * ((a.N + 127) / 128) >= 1024 ? expand<KK, 2, false, false>(a, s) : expand<KK, 1, false, false>(a, s);
}

}  // namespace

size_t plan_adapters(AdapterArgs& a, void* workspace) {
    a.Rp = (a.R + 15) / 16 * 16;
    // Up to 64 tokens need no sorting.  Tiles of 16 tokens, whose four wavefronts share K, as long as they are not many; of 64, which read A and B a quarter
    // as often, beyond (us, 16 / 64: 300 tokens of 4096 x 4096 rank 16 14 / 17, 630 of 5696 x 2208 rank 64 23 / 31, 1000 of 672 x 532 rank 128
    // 18 / 30 and of 4096 x 4096 rank 16 21 / 22; 1000 of 4096 x 11008 rank 64 with 24 adapters 48 / 39, 1500 of 4096 x 4096 rank 32 27 / 25, 3000 of 2048 x 2048
    // rank 128 56 / 44).  By tokens alone the rule is wrong next to its limit for wide layers with many ranks, whose B counts: the 48 / 39.
    a.tile = a.M <= kWide ? 0 : a.M <= kNarrowTokens ? 16 : kWide;
    // Parts of K: at least 512 values each, at most 8 parts (that many loads sum T up at once), and with many tokens no more than give two
    // workgroups to a compute unit
    int64_t parts = (a.K + 511) / 512;
    if (parts > 8) parts = 8;
    if (a.tile > 0) {
        const int64_t tiles = (a.M + a.tile - 1) / a.tile, want = (512 + tiles - 1) / tiles;
        if (parts > want) parts = want;
    }
    a.k_split = ((a.K + parts - 1) / parts + 63) / 64 * 64;
    a.splits = (int)((a.K + a.k_split - 1) / a.k_split);
    const auto up = [](int64_t v) { return (v + 255) / 256 * 256; };
    uint8_t* const base = (uint8_t*)workspace;
    int64_t at = up((int64_t)a.splits * a.M * a.Rp * 4);
    a.T = (float*)base;
    a.list = nullptr;
    a.tiles = nullptr;
    a.order = nullptr;
    if (a.tile > 0) {
        a.list = (int*)(base + at);
        at += 256;
        a.tiles = (AdapterTile*)(base + at);
        at += up(most_groups(a) * (int64_t)sizeof(AdapterTile));
        a.order = (int*)(base + at);
        at += up(a.M * 4);
    }
    return (size_t)at;
}

hipError_t launch_adapters(const AdapterArgs& a, hipStream_t s) {
    if (a.tile > 0) {
        hipLaunchKernelGGL(adapter_sort_kernel, dim3(1), dim3(1024), (size_t)(a.n + 1) * 4, s, a);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    hipError_t e;
    if (a.R <= 16) e = project<1>(a, s);
    else if (a.R <= 32) e = project<2>(a, s);
    else if (a.R <= 64) e = project<4>(a, s);
    else e = project<8>(a, s);
    if (e != hipSuccess) return e;
    if (a.R <= 32) return expand<1>(a, s);
    if (a.R <= 64) return expand<2>(a, s);
    return expand<4>(a, s);
}

}  // namespace lqer
