// What the attention kernels for few rows and for prompts share.
#pragma once
#include "bf16_pair.h"
#include "paged_kv.h"

typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

constexpr float kNone = -3.402823466e38f;         // running maximum before any key: the lowest finite value, so that every logit above it counts

// n / d for 0 <= n < 2^31 as (n m) >> (31 + s): with 2^s >= d and m = floor(2^(31 + s) / d) + 1 the product is above n 2^(31 + s) / d by less than
// 2^(31 + s) / d.  A division by a number that is not known to the compiler takes some 150 cycles.
struct Divider {
    uint32_t m; int s;
    __host__ static Divider by(uint32_t d) {
        Divider x{0u, 31};
        while (((uint64_t)1 << (x.s - 31)) < d) ++x.s;
        x.m = (uint32_t)(((uint64_t)1 << x.s) / d + 1);
        return x;
    }
    __device__ __forceinline__ int operator()(int n) const { return (int)((uint64_t)(uint32_t)n * m >> s); }
};

struct AttnArgs {
    PagedArgs p;
    Divider by_group, by_kv, by_tiles, by_split;  // divisions by p.group, p.n_kv, row_tiles and tiles_per_split
    const uint16_t* q; int64_t ldq;
    uint16_t* out; int64_t ldo;
    float c;                                      // scale * log2(e)
    int window, sinks;                            // window 0: none
    int few_rows;                                 // requests of up to so many rows (tokens * group) take the kernel for few rows, -1: none does
    int splits, tiles_per_split, row_tiles;       // the kernel for few rows: parts of the key axis, their steps, most row tiles of a request
    float* part_o; float2* part_ml;               // results of splits: [row tile and head][split][row][D], [..][split][row] (maximum, sum)
    // the kernel for prompts: the same of its own, and its grid: tiles times heads, times splits, then the few rows' (by_pairs: times splits again)
    int prompt_splits, prompt_blocks, prompt_all, prompt_joins;
    Divider by_blocks, by_pairs;
    float* prompt_o; float2* prompt_ml;
};

// Tiles of TILE keys that some row of positions [p_lo, p_hi] may see: [0, sink_tiles) and [main0, main0 + main_tiles).
template <int TILE>
struct KeyTiles {
    int sink_tiles, main0, total;
    __device__ __forceinline__ KeyTiles(int p_lo, int p_hi, int window, int sinks) {
        main0 = 0;
        sink_tiles = 0;
        if (window > 0) {
            const int low = p_lo - window + 1;
            main0 = low > 0 ? low / TILE : 0;
            const int s = (min(sinks, p_hi + 1) + TILE - 1) / TILE;
            sink_tiles = min(s, main0);
        }
        total = p_hi < 0 ? 0 : sink_tiles + p_hi / TILE - main0 + 1;
    }
    // Tiles, counted from the first, that begin at or before key `p`.
    __device__ __forceinline__ int count_up_to(int p) const {
        const int t = p < 0 ? 0 : p / TILE + 1;
        return t <= main0 ? min(t, sink_tiles) : sink_tiles + t - main0;
    }
    __device__ __forceinline__ int first_key(int i) const { return (i < sink_tiles ? i : main0 + i - sink_tiles) * TILE; }
};

// Request and row tile of the tile-th pair of them in the kernels for few rows.  A request's first row tile is often the only one with rows, and
// workgroups go to the XCDs and their shader engines in turn: at every row_tiles-th place those with work would meet on a part of the device (31 tokens over 8192
// keys each beside a request of 16 new tokens: 373 us, in this order 202).  So the order of a request's row tiles turns from request to request.
struct FewTile {
    int seq, row_tile;
    __device__ __forceinline__ FewTile(const AttnArgs& g, int tile) {
        seq = g.by_tiles(tile);
        const int turn = seq + g.by_tiles(seq), x = tile - seq * g.row_tiles - (turn - g.by_tiles(turn) * g.row_tiles);
        row_tile = x < 0 ? x + g.row_tiles : x;
    }
};

// Words that no kernel of this call writes, through the scalar cache: beside copies into LDS the compiler takes vector loads for them, and
// waits for those together with every copy in flight.
typedef const __attribute__((address_space(4))) int32_t* ScalarInts;
__device__ __forceinline__ ScalarInts scalar_ints(const int32_t* p) { return (ScalarInts)(uintptr_t)p; }

// Two codes of 8 bits, sign-extended, as two bf16 values in a word.
template <int B>
__device__ __forceinline__ uint32_t codes_pair(uint32_t w) {
    return upper_halves((float)(int8_t)(w >> (8 * B)), (float)(int8_t)(w >> (8 * B + 8)));
}

// prompt_attention.hip: a call where some request may have more than few_rows rows; keys: the most that a row sees.  Its workspace begins at
// byte ws_at of ctx's, behind that of the requests of few rows.
size_t aser_attention_prompt_workspace(int64_t tokens, int64_t n_seq, int64_t n_kv, int64_t group, int head_dim, int64_t keys);
int aser_attention_prompt(aser_ctx* ctx, AttnArgs g, int head_dim, int64_t keys, size_t ws_at);
