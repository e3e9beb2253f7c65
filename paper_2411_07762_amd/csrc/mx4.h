// Microscaled 4 bits: what the quantizer and the products share.
#pragma once
#include "aser_internal.h"

static const int64_t kMxWord = 128;         // channels of a scale word: four blocks of 32, 64 bytes of codes

static inline int64_t mx4_words(int64_t n) { return ceil_div64(n, kMxWord); }
// Place of word 0 of a row, in units of 64 bytes of codes or 4 of scales; the next word is kMxNext further.  Matrix e begins at e * mx4_size.
static const int kMxNext = 16;
__host__ __device__ static inline int64_t mx4_at(int64_t row, int64_t words) { return (row >> 4) * words * 16 + (row & 15); }
__host__ __device__ static inline int64_t mx4_size(int64_t rows, int64_t words) { return ((rows + 15) >> 4) * words * 16; }
// Checks of structs that have been given; `who` names the entry point.  Which arrays of a plan a call needs is its own matter.
int aser_plan_check(aser_ctx* ctx, const char* who, const aser_expert_plan* p);
int aser_mx4_check(aser_ctx* ctx, const char* who, const aser_mx4* t, bool may_be_empty);

// Rows in groups that have a matrix each: the positions offsets[e] .. offsets[e + 1] - 1 are those of matrix e.
struct MxGroups {
    const int32_t* offsets;      // null: one group of all positions
    const int32_t* order;        // not null: position p reads row order[p] / top_k
    int count, top_k;
    int64_t positions;
    int64_t most_tiles(int64_t bm) const {                   // no more tiles of bm positions than this, however the positions fall
        return offsets ? positions / bm + (count < positions ? count : positions) : ceil_div64(positions, bm);
    }
};

// Tiles of bm positions that there are.
__device__ __forceinline__ int64_t mx4_tiles(const MxGroups& g, int bm) {
    if (!g.offsets) return (g.positions + bm - 1) / bm;
    const int lane = threadIdx.x & 63;
    const int32_t most = (int32_t)g.positions;
    int32_t sum = 0;
    for (int e = lane; e < g.count; e += 64) {
        const int32_t a = g.offsets[e], b = g.offsets[e + 1];
        const int32_t s = a < 0 ? 0 : a > most ? most : a, t = b > most ? most : b;
        sum += t > s ? (t - s + bm - 1) / bm : 0;
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
    return __builtin_amdgcn_readfirstlane(sum);
}
// Workgroup `tile`'s matrix, first position and number of positions.  False: there is no such tile.  Every wavefront looks for itself: a
// lane has a group, and the running sum of the groups' tiles says whose the tile is.
__device__ __forceinline__ bool mx4_find_tile(const MxGroups& g, int64_t tile, int bm, int* e, int64_t* p0, int* rows) {
    if (!g.offsets) {
        const int64_t left = g.positions - tile * bm;
        *e = 0;
        *p0 = tile * bm;
        *rows = (int)(left < bm ? left : bm);
        return left > 0;
    }
    const int lane = threadIdx.x & 63;
    const int32_t most = (int32_t)g.positions;
    int32_t before = 0;
    for (int e0 = 0; e0 < g.count; e0 += 64) {
        int32_t s = 0, n = 0;
        if (e0 + lane < g.count) {
            const int32_t a = g.offsets[e0 + lane], b = g.offsets[e0 + lane + 1];
            s = a < 0 ? 0 : a > most ? most : a;
            const int32_t t = b > most ? most : b;
            n = t > s ? t - s : 0;
        }
        const int32_t mine = (n + bm - 1) / bm;
        int32_t upto = mine;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int32_t v = __shfl_up(upto, d);
            if (lane >= d) upto += v;
        }
        const uint64_t over = __ballot(before + upto > tile);
        if (over) {
            const int at = __builtin_ctzll(over);
            const int32_t i = (int32_t)tile - before - __builtin_amdgcn_readlane(upto - mine, at), first = __builtin_amdgcn_readlane(s, at);
            const int32_t left = __builtin_amdgcn_readlane(n, at) - i * bm;
            *e = e0 + at;
            *p0 = first + (int64_t)i * bm;
            *rows = left < bm ? left : bm;
            return true;
        }
        before += __builtin_amdgcn_readlane(upto, 63);
    }
    return false;
}
__device__ __forceinline__ int64_t mx4_row(const MxGroups& g, int64_t p) {
    if (!g.order) return p;
    const int32_t pair = g.order[p];
    const int32_t most = (int32_t)g.positions - 1;
    return (pair < 0 ? 0 : pair > most ? most : pair) / g.top_k;
}
