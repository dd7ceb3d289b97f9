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
    int64_t first;                 // set by launch_rmsnorm_mx: the launch's first row
};
hipError_t launch_rmsnorm_mx(const NormArgs& a, hipStream_t s);

constexpr int kMaxAdapters = 8192;     // their counts lie in LDS while tokens are sorted
constexpr int kMaxAdapterRank = 128;
struct AdapterTile { int adapter, start, count, unused; };       // adapter -1: tokens without one
struct AdapterArgs {
    const uint16_t* X;
    int64_t M, K, ldx;
    const int32_t* ids;
    const uint16_t* A;
    const uint16_t* B;
    int n, R;
    const int32_t* ranks;
    const float* scales;
    const float* Y_in;
    int64_t ldyi;
    float* Y_out;
    int64_t N, ldyo;
    // set by plan_adapters
    int Rp;                // R in whole tiles of 16: T's row length
    int tile;              // tokens of a tile; 0: few tokens, unsorted
    int splits;            // parts of K, of k_split values each
    int64_t k_split;
    float* T;              // [splits][M][Rp]
    int* list;             // more than 64 tokens: number of tiles,
    AdapterTile* tiles;    // the tiles,
    int* order;            // and the tokens in their order
    // set by launch_adapters
    int parts;             // workgroups of the second product to a tile
};
// Lays the call's scratch out and returns its bytes.
size_t plan_adapters(AdapterArgs& a, void* workspace);
hipError_t launch_adapters(const AdapterArgs& a, hipStream_t s);

// ---- the cache of keys and values in MXINT4 (formats in lqer.h) ------------------------------------------------------------
struct Kv4AppendArgs {
    uint8_t* pool;
    int64_t pages;
    int P_bits;            // log2 of a page's tokens
    int heads, D;
    const void* k;
    const void* v;
    int64_t ldk, ldv;
    int type;
    int64_t T;
    const int32_t* slots;
};
hipError_t launch_kv4_append(const Kv4AppendArgs& a, hipStream_t s);

constexpr int kFewRows = 64;           // query rows (query, head of the group) that the kernel for few rows takes, in tiles of 16
constexpr int kManyRows = 128;         // rows of a workgroup of the kernel for many

// How one of the two kernels is laid out: tiles of query rows (query, head of the group) and parts of the cached tokens.
struct Kv4Plan {
    bool run;
    int row_tiles;         // tiles of rows of a request that have workgroups of their own
    int chunk;             // cached tokens of a part, at least
    int splits;            // most parts
    int cap;               // few rows: the rows of a request and cached head that have room for their parts
    float* part_o;         // [..][splits][D]: a part's sum of weighted values,
    float2* part_ml;       // [..][splits]: its maximum (in units of log 2) and sum of weights; [n_requests][kv_heads][cap] or [Tq][q_heads]
};
struct Kv4Args {
    lqer_kv4_shape sh;
    const uint8_t* pool;
    const uint16_t* q;
    const int32_t* cu_q;
    const int32_t* kv_len;
    const int32_t* table;
    void* out;
    // set by plan_kv4
    int group;             // query heads of a cached head
    int P_bits;
    int few_rows;          // requests of up to so many rows go to the kernel for few, where both run
    Kv4Plan few, many;
};
size_t plan_kv4(Kv4Args& a, void* workspace);
hipError_t launch_kv4_attention(const Kv4Args& a, hipStream_t s);
hipError_t launch_kv4_many(const Kv4Args& a, hipStream_t s);          // kernels_kv4_many.hip

}  // namespace lqer
