// Microscaled 4 bits: what the quantizer and the products share.
#pragma once
#include "aser_internal.h"

static const int64_t kMxWord = 128;         // channels of a scale word: four blocks of 32, 64 bytes of codes

// A dimension of a launch has fewer than 2^32 threads.  Where more are wanted, workgroups are numbered over two dimensions, kMxAcross of them in the first.
static const int64_t kMxAcross = (int64_t)1 << 23;
static inline bool mx4_fits(int64_t workgroups, int64_t threads) { return workgroups <= (int64_t)UINT32_MAX / threads; }

static inline int64_t mx4_words(int64_t n) { return ceil_div64(n, kMxWord); }
// Rows are in panels of 16: the word of scales of a row is at mx4_at, in words, the following one kMxNext further; the 16 bytes of codes of block q are at
// 16 mx4_code + 256 q bytes, those of the following word 64 kMxNext bytes further.  Matrix e begins e mx4_size words and 64 times as many bytes behind the first.
static const int kMxNext = 16;
__host__ __device__ static inline int64_t mx4_at(int64_t row, int64_t words) { return (row >> 4) * words * 16 + (row & 15); }
__host__ __device__ static inline int64_t mx4_code(int64_t row, int64_t words) { return (row >> 4) * words * 64 + (row & 15); }
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

// Between a wavefront's writes to LDS and other lanes' reads of them, and back: LDS serves a wavefront's accesses in order, so that the compiler has to keep it is all that is wanted.
__device__ __forceinline__ void mx4_lanes_meet() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// The sum over the lanes up to this one, by moves within rows of 16 lanes and from the last of a row to the following rows.  Every workgroup begins with this: with shuffles through
// LDS 48 rows on 64 experts, 1408 x 2048, take 33.1 us instead of 32.0.
__device__ __forceinline__ uint32_t mx4_sums_upto(uint32_t v) {
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xF, 0xF, false);       // row_shr by 1, 2, 4, 8
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xF, 0xF, false);
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xF, 0xF, false);
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xF, 0xF, false);
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xA, 0xF, false);       // row_bcast of lane 15 to rows 1 and 3, of lane 31 to rows 2 and 3
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xC, 0xF, false);
    return v;
}

// Tiles of bm positions that there are.
__device__ __forceinline__ uint32_t mx4_tiles(const MxGroups& g, int bm) {
    if (!g.offsets) return (uint32_t)((g.positions + bm - 1) / bm);
    const int lane = threadIdx.x & 63;
    const int32_t most = (int32_t)g.positions;
    int32_t sum = 0;
    for (int e = lane; e < g.count; e += 64) {
        const int32_t a = g.offsets[e], b = g.offsets[e + 1];
        const int32_t s = a < 0 ? 0 : a > most ? most : a, t = b > most ? most : b;
        sum += t > s ? (t - s + bm - 1) / bm : 0;
    }
    return (uint32_t)__builtin_amdgcn_readlane((int)mx4_sums_upto((uint32_t)sum), 63);
}
// Tiles of bm positions, `across` of them beside each other for other outputs, numbered matrix by matrix: the matrix that number id belongs to, its first position, the
// number of its positions, and id's place among its tiles.  False: there is no such tile.  Every wavefront looks for itself: a lane has a matrix, and the
// running sum of their tiles says whose the number is.
__device__ __forceinline__ bool mx4_find(const MxGroups& g, uint64_t id, int bm, uint32_t across, int* e, int64_t* first, int* count, uint32_t* place) {
    if (!g.offsets) {
        *e = 0;
        *first = 0;
        *count = (int)g.positions;
        *place = (uint32_t)id;
        return (int64_t)((uint32_t)id / across) * bm < g.positions;
    }
    const int lane = threadIdx.x & 63;
    const int32_t most = (int32_t)g.positions;
    uint32_t before = 0;
    for (int e0 = 0; e0 < g.count; e0 += 64) {
        int32_t s = 0, n = 0;
        if (e0 + lane < g.count) {
            const int32_t a = g.offsets[e0 + lane], b = g.offsets[e0 + lane + 1];
            s = a < 0 ? 0 : a > most ? most : a;
            const int32_t t = b > most ? most : b;
            n = t > s ? t - s : 0;
        }
        const uint32_t mine = (uint32_t)((n + bm - 1) / bm);
        const uint32_t upto = mx4_sums_upto(mine);
        const uint64_t over = __ballot((uint64_t)(before + upto) * across > id);      // offsets that make no sense can name more tiles than 32 bits count
        if (over) {
            const int at = __builtin_ctzll(over);
            *e = e0 + at;
            *first = __builtin_amdgcn_readlane(s, at);
            *count = __builtin_amdgcn_readlane(n, at);
            *place = (uint32_t)(id - (uint64_t)(before + (uint32_t)__builtin_amdgcn_readlane((int)(upto - mine), at)) * across);
            return true;
        }
        before += (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
    }
    return false;
}
// The same for one tile across: the tile's matrix, first position and number of positions.
__device__ __forceinline__ bool mx4_find_tile(const MxGroups& g, uint32_t tile, int bm, int* e, int64_t* p0, int* rows) {
    int count;
    uint32_t place;
    int64_t first;
    if (!mx4_find(g, tile, bm, 1, e, &first, &count, &place)) return false;
    const int left = count - (int)place * bm;
    *p0 = first + (int64_t)place * bm;
    *rows = left < bm ? left : bm;
    return true;
}
__device__ __forceinline__ int64_t mx4_row(const MxGroups& g, int64_t p) {
    if (!g.order) return p;
    const int32_t pair = g.order[p];
    const int32_t most = (int32_t)g.positions - 1;
    return (pair < 0 ? 0 : pair > most ? most : pair) / g.top_k;
}
