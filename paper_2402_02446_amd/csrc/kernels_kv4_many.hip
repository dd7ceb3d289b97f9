// Attention of many query rows over the MXINT4 cache: prompts, and chunks of them.
//
// Bound by the matrix instructions and the exponentials beside them.  A workgroup has 128 rows (query, head of the group) of one cached head,
// 32 to each of its four wavefronts, and takes the cached tokens in tiles of 64 (32 at D = 256).  All four turn a tile's words into bf16
// once, a lane 16 bytes of a key and a cell of four tokens by eight dimensions of values, a wavefront 16 tokens, and store them in LDS as the operands of the
// 32 x 32 x 16 matrix instruction in the order in which the wavefronts read them, 64 lanes x 16 bytes; two tiles' room, so that
// one barrier a tile is enough, and the next tile's words are loaded meanwhile.
//   S^T = K Q^T      tokens as rows, query rows as columns: a lane holds half of the tokens of one row, the lane 32 further the others
//   O^T += V^T P^T   the scores' registers are the operand as they are (tokens in the order in which the lanes hold them)
// The running maximum is moved only when a score passes it by more than 2^8: until then the weights, relative to the older
// maximum, are at most 2^8, which costs no precision, and the accumulators need no rescaling.  The weights enter the product as one bf16
// term (relative 2^-8 at most), their sum in fp32: bf16 outputs are then 2.3e-3 from the exact ones (relative Frobenius; their own rounding is
// 1.7e-3 of that).  Two terms take longer: 2 x 2048 queries on 6144 tokens, 64 / 8 heads, 718 us and with two terms 947, one prompt of 2048 92 and 114, 2 x 2048
// queries on 6144 at D = 64 527 and 660, on 3008 at D = 256 262 and 294.
//
// Measured: 2 x 2048 queries on up to 6144 tokens, 64 / 8 heads of 128 (374 GFLOP) 0.93 M cycles, which are 450 to 510 us in the first calls after a
// pause and 400 after some sixty back to back, as the card's clock has it; the matrix instructions are busy 39 % of the cycles, vector instructions 51 %, LDS 35 %: with two wavefronts to a SIMD they come one after another.  Not faster: reads
// of LDS scheduled ahead, exponentials pinned among the matrix instructions, wavefront priorities, tiles of 32 tokens with three workgroups
// to a compute unit (13 % slower), 64 rows to a wavefront (35 % slower: 508 registers, one wavefront to a SIMD).
#include "kv4_device.h"

namespace lqer {

namespace {

constexpr float kLog2e = 1.44269504088896340736f;

template <int D>
struct Tile {
    static constexpr int TOKENS = D == 256 ? 32 : 64;
    static constexpr int KEYS = TOKENS * D * 2;                    // bytes of a tile's keys in LDS; as many of its values
    static constexpr int E = 256 / D;                              // dimensions of a word that share a tile of 32 output dimensions
};

// A lane's words of a tile, on their way: 32 dimensions of a key, and a cell of values.  A wavefront's are those of the same 16 tokens, which
// lie in one page: its number is a scalar.  At D = 64 the first 32 lanes have the keys and the others the values.
struct Words {
    u32x4 k, v;
    uint32_t ke, ve;
};
template <int D>
struct Part {
    int sub;               // which 16 tokens of the tile
    int t, c;              // key: token of the 16, which 32 dimensions
    int four, word;        // values: which four tokens of the 16, word of eight dimensions
    bool k, v;
    __device__ __forceinline__ Part(int wave, int lane) {
        sub = D == 256 ? wave >> 1 : wave;
        t = lane & 15;
        c = D == 64 ? (lane >> 4) & 1 : D == 128 ? lane >> 4 : (lane >> 4) + 4 * (wave & 1);
        const int cell = D == 64 ? lane & 31 : lane;
        four = D == 256 ? cell >> 4 : cell / (D / 8);
        word = D == 256 ? (cell & 15) + 16 * (wave & 1) : cell % (D / 8);
        k = D != 64 || lane < 32;
        v = D != 64 || lane >= 32;
    }
};

// page: of the wavefront's 16 tokens, one of the pool's.  (No branch here, and no use of what is loaded: the words are waited for when the
// tile before them is done.)
template <int D>
__device__ __forceinline__ void load_words(const Kv4Args& a, const Kv4Record<D> R, const Part<D>& part, int page, int head, int t0, Words& w) {
    const int off = (t0 + 16 * part.sub) & ((1 << a.P_bits) - 1);
    const uint8_t* const rec = a.pool + ((int64_t)page * a.sh.kv_heads + head) * R.bytes();
    if (part.k) {
        w.k = *reinterpret_cast<const u32x4*>(rec + R.key(off) + (uint32_t)(part.t * (D / 2) + 16 * part.c));
        w.ke = *reinterpret_cast<const uint16_t*>(rec + R.key_exp(off) + (uint32_t)(part.t * (D / 16) + 2 * part.c));
    }
    if (part.v) {
        w.v = *reinterpret_cast<const u32x4*>(rec + R.value(off / 4) + (uint32_t)(part.four * (2 * D) + part.word * 16));
        w.ve = *reinterpret_cast<const uint32_t*>(rec + R.value_exp(off / 4) + (uint32_t)(part.four * (D / 4) + part.word / 2 * 4));
    }
}

// The values' exponents of tokens outside [from, end) cleared: they may hold anything, their weights are 0 and meet a finite number.
template <int D>
__device__ __forceinline__ void clear_unseen(const Part<D>& part, int t0, int from, int end, Words& w) {
    const int t = t0 + 16 * part.sub + 4 * part.four, before = from - t, n = end - t;
    if (before > 0) w.ve = before < 4 ? w.ve >> (8 * before) << (8 * before) : 0u;
    if (n < 4) w.ve = n > 0 ? w.ve & ((1u << (8 * n)) - 1u) : 0u;
}

// ... and into LDS as operands.  Keys: [32 tokens][step of 16 dimensions][64 lanes][16 B]; values: [tile of 32 output dimensions][step of 16
// tokens][64 lanes][16 B], output dimension 8 w + e being row E w + e % E of tile e / E.
template <int D>
__device__ __forceinline__ void store_words(const Words& w, const Part<D>& part, uint8_t* keys, uint8_t* values) {
    using T = Tile<D>;
    if (part.k) {
        uint8_t* const at = keys + (part.sub / 2) * (32 * D * 2) + (4 * part.c * 32 + (part.sub & 1) * 16 + part.t) * 16;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            Frag f;
            f.v = unpack_w8(w.k[j], kv4_scale((w.ke >> (8 * (j / 2))) & 0xFFu));
            *reinterpret_cast<u32x4*>(at + j * 32 * 16) = f.u;
        }
    }
    if (part.v) {
        uint32_t t[4][4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            Frag f;
            f.v = unpack_w8(w.v[j], kv4_scale((w.ve >> (8 * j)) & 0xFFu));
#pragma unroll
            for (int x = 0; x < 4; ++x) t[j][x] = f.u[x];
        }
        u32x2 half[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t sel = e & 1 ? 0x07060302u : 0x05040100u;
            half[e] = u32x2{__builtin_amdgcn_perm(t[1][e / 2], t[0][e / 2], sel), __builtin_amdgcn_perm(t[3][e / 2], t[2][e / 2], sel)};
        }
        // tokens 4 hh .. and 8 + 4 hh .. of the 16: the two halves of lane half hh
        constexpr int BLOCK = T::TOKENS / 16 * 64;                 // cells of a tile of output dimensions
        uint8_t* const at = values + (part.sub * 64 + (part.four & 1) * 32 + T::E * part.word) * 16;
        if (D == 64) {
#pragma unroll
            for (int e = 0; e < 8; ++e) *reinterpret_cast<u32x2*>(at + ((e / T::E) * BLOCK + e % T::E) * 16 + (part.four >> 1) * 8) = half[e];
        } else {
            // the other half of a cell is 32 lanes away: the lower lanes take both of the dimensions 0 to 3, the upper ones of 4 to 7, and write
            // whole cells of 16 bytes (halves of 8 would meet in the same banks four at a time)
            uint8_t* const mine = at + (part.four >> 1) * (4 / T::E) * BLOCK * 16;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const auto x = __builtin_amdgcn_permlane32_swap(half[e][0], half[e + 4][0], false, false);
                const auto y = __builtin_amdgcn_permlane32_swap(half[e][1], half[e + 4][1], false, false);
                *reinterpret_cast<u32x4*>(mine + ((e / T::E) * BLOCK + e % T::E) * 16) = u32x4{x[0], y[0], x[1], y[1]};
            }
        }
    }
}

__device__ __forceinline__ float halves_max(float v) {
    const auto b = __builtin_amdgcn_permlane32_swap(f32_bits(v), f32_bits(v), false, false);
    return __builtin_fmaxf(f32_from_bits(b[0]), f32_from_bits(b[1]));
}

template <int D>
__global__ __launch_bounds__(256, D == 256 ? 1 : 2) void kv4_many_kernel(Kv4Args a) {
    using T = Tile<D>;
    constexpr int QS = D / 16, NO = D / 32, U = T::TOKENS / 32;
    __shared__ __align__(16) uint8_t keys[2][T::KEYS];
    __shared__ __align__(16) uint8_t values[2][T::KEYS];
    __shared__ __align__(16) uint32_t absent[2][4];              // whether a tile's 16 tokens have a page that is none of the pool's
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 31, hh = lane >> 5;
    const int head = blockIdx.y % a.sh.kv_heads, b = blockIdx.z, split = blockIdx.x;
    Kv4Rows r = kv4_request(a, b);
    if (!kv4_mine<true>(a, r)) return;
    const Kv4Record<D> R{a.P_bits};
    const Part<D> part(wave, lane);
    const int32_t* const table = a.table + (int64_t)b * a.sh.table_ld;
    const float to_log2 = __builtin_fmaxf(__builtin_fabsf(a.sh.scale) * kLog2e, 0x1p-126f);      // as for few rows
    const uint32_t turn = a.sh.scale < 0.f ? 0x80008000u : 0u;
    const int all_rows = r.n * a.group, tiles = (all_rows + kManyRows - 1) / kManyRows;
    // (the last rows see the most tokens of a causal prompt: they start first)
    for (int tile = tiles - 1 - (int)(blockIdx.y / a.sh.kv_heads); tile >= 0; tile -= a.many.row_tiles) {
        kv4_tile(a, r, tile * kManyRows, kManyRows);
        int chunk;
        const int parts = kv4_parts<true>(a, r, chunk);
        if (split >= parts && split > 0) continue;
        const int lo = (r.lo & ~31) + split * chunk, hi = min(r.hi, lo + chunk);
        // this wavefront's rows, this lane's
        const int w_first = min(r.row0 + 32 * wave, r.row0 + r.rows - 1), w_last = min(w_first + 31, r.row0 + r.rows - 1);
        const bool idle = 32 * wave >= r.rows;
        const int row = min(r.row0 + 32 * wave + i, r.row0 + r.rows - 1), query = row / a.group;
        const int64_t orow = r.first + query;
        const int h = head * a.group + row - query * a.group;
        const int begin = kv4_row_begin(a, r, query), end = kv4_row_end(a, r, query);
        const int w_begin = kv4_row_begin(a, r, w_first / a.group), w_end = idle ? 0 : kv4_row_end(a, r, w_last / a.group);
        const int all_begin = kv4_row_begin(a, r, w_last / a.group), all_end = kv4_row_end(a, r, w_first / a.group);
        Frag q[QS];
        {
            const uint16_t* p = a.q + orow * a.sh.ldq + (int64_t)h * D + 8 * hh;
#pragma unroll
            for (int s = 0; s < QS; ++s) q[s].u = *reinterpret_cast<const u32x4*>(p + 16 * s) ^ turn;
        }
        f32x16 o[NO];
#pragma unroll
        for (int x = 0; x < NO; ++x)
#pragma unroll
            for (int j = 0; j < 16; ++j) o[x][j] = 0.f;
        float m = -__builtin_inff(), l = 0.f;
        int page_base = 0, page_of_lane = 0, page = 0;         // 64 entries of the request's table, one to a lane; the next words' page
        bool fresh = true;
        const auto fetch = [&](int t0, Words& w) {
            const int index = (t0 + 16 * part.sub) >> a.P_bits;
            if (fresh || index - page_base >= 64) {
                page_base = index;
                page_of_lane = index + lane < a.sh.table_ld ? table[index + lane] : -1;
                fresh = false;
            }
            page = __builtin_amdgcn_readlane(page_of_lane, index - page_base);
            if (page >= a.sh.pages) page = -1;
            load_words<D>(a, R, part, page < 0 ? 0 : page, head, t0, w);
        };
        Words words;
        if (lo < hi) fetch(lo, words);
        int buf = 0;
        for (int t0 = lo; t0 < hi; t0 += T::TOKENS, buf ^= 1) {
            if (page < 0 || t0 < r.lo || t0 + T::TOKENS > hi) clear_unseen<D>(part, t0, page < 0 ? hi : r.lo, hi, words);
            store_words<D>(words, part, keys[buf], values[buf]);
            absent[buf][part.sub] = page < 0 ? 1u : 0u;
            if (t0 + T::TOKENS < hi) fetch(t0 + T::TOKENS, words);
            __syncthreads();
            if (t0 >= w_end || t0 + T::TOKENS <= w_begin) continue;      // nothing that this wavefront's rows see
            const u32x4 gone = *reinterpret_cast<const u32x4*>(absent[buf]);
            f32x16 s[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int j = 0; j < 16; ++j) s[u][j] = 0.f;
#pragma unroll
            for (int x = 0; x < QS; ++x)
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    Frag f;
                    f.u = *reinterpret_cast<const u32x4*>(keys[buf] + u * (32 * D * 2) + (x * 64 + lane) * 16);
                    s[u] = mfma32(f.v, q[x].v, s[u]);
                }
            const uint32_t none = U > 1 ? gone[0] | gone[1] | gone[2] | gone[3] : gone[0] | gone[1];
            if (t0 < all_begin || t0 + T::TOKENS > all_end || t0 + T::TOKENS > hi || __builtin_amdgcn_readfirstlane(none) != 0) {
                int at = t0;
                asm volatile("" : "+s"(at));       // (a branch: left alone, the comparisons are done for every tile)
                const int stop = min(end, hi);
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        const int k = 8 * (j >> 2) + 4 * hh + (j & 3), t = at + 32 * u + k;
                        if (t >= stop || t < begin || gone[2 * u + (j >> 3)] != 0) s[u][j] = -__builtin_inff();
                    }
            }
            float top = s[0][0];
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int j = 0; j < 16; ++j) top = __builtin_fmaxf(top, s[u][j]);
            top = halves_max(top) * to_log2;
            if (__ballot(top > m + 8.0f)) {        // (also the first score: m is minus infinity)
                const float next = __builtin_fmaxf(m, top), down = m == -__builtin_inff() ? 0.f : exp2_fast(m - next);
                l *= down;
#pragma unroll
                for (int x = 0; x < NO; ++x) o[x] *= down;
                m = next;
            }
            const float base = m == -__builtin_inff() ? 0.f : m;
            Frag p[2 * U];
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int j = 0; j < 16; j += 2) {
                    const float e0 = exp2_fast(__builtin_fmaf(s[u][j], to_log2, -base));
                    const float e1 = exp2_fast(__builtin_fmaf(s[u][j + 1], to_log2, -base));
                    l += e0;
                    l += e1;
                    p[2 * u + (j >> 3)].u[(j >> 1) & 3] = pack_bf16_near(e0, e1);
                }
#pragma unroll
            for (int k = 0; k < 2 * U; ++k)
#pragma unroll
                for (int x = 0; x < NO; ++x) {
                    Frag f;
                    f.u = *reinterpret_cast<const u32x4*>(values[buf] + ((x * (2 * U) + k) * 64 + lane) * 16);
                    o[x] = mfma32(f.v, p[k].v, o[x]);
                }
        }
        __syncthreads();                           // (the next tile of rows stores into LDS from its beginning)
        {
            const auto both = __builtin_amdgcn_permlane32_swap(f32_bits(l), f32_bits(l), false, false);
            l = f32_from_bits(both[0]) + f32_from_bits(both[1]);
        }
        if (32 * wave + i >= r.rows) continue;
        const float by = parts > 1 ? 1.0f : l > 0.f ? 1.0f / l : 0.f;
        const int64_t at = parts > 1 ? kv4_part<true>(a, b, head, row, orow, h) + split : 0;
        if (parts > 1 && hh == 0) a.many.part_ml[at] = float2{m, l};
        // rows of the output tiles: register j of lane half hh is row 8 (j / 4) + 4 hh + j % 4; eight neighbouring dimensions lie in E
        // registers of every tile
#pragma unroll
        for (int j = 0; j < 16; j += T::E) {
            const int row_of = 8 * (j >> 2) + 4 * hh + (j & 3), word = row_of / T::E;
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = o[e / T::E][j + e % T::E] * by;
            if (parts > 1) {
                f32x4* p = reinterpret_cast<f32x4*>(a.many.part_o + at * D + 8 * word);
                p[0] = f32x4{v[0], v[1], v[2], v[3]};
                p[1] = f32x4{v[4], v[5], v[6], v[7]};
            } else if (a.sh.out_type == LQER_F32) {
                f32x4* p = reinterpret_cast<f32x4*>((float*)a.out + orow * a.sh.ldo + (int64_t)h * D + 8 * word);
                p[0] = f32x4{v[0], v[1], v[2], v[3]};
                p[1] = f32x4{v[4], v[5], v[6], v[7]};
            } else {
                *reinterpret_cast<u32x4*>((uint16_t*)a.out + orow * a.sh.ldo + (int64_t)h * D + 8 * word) =
                    u32x4{pack_bf16_near(v[0], v[1]), pack_bf16_near(v[2], v[3]), pack_bf16_near(v[4], v[5]), pack_bf16_near(v[6], v[7])};
            }
        }
    }
}

template <int D>
hipError_t launch_d(const Kv4Args& a, hipStream_t s) {
    const dim3 grid((unsigned)a.many.splits, (unsigned)(a.many.row_tiles * a.sh.kv_heads), (unsigned)a.sh.n_requests);
    hipLaunchKernelGGL((kv4_many_kernel<D>), grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_kv4_many(const Kv4Args& a, hipStream_t s) {
    if (a.sh.head_dim == 64) return launch_d<64>(a, s);
    return a.sh.head_dim == 128 ? launch_d<128>(a, s) : launch_d<256>(a, s);
}

}  // namespace lqer
