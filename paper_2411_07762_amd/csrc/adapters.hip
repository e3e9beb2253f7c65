// Low-rank adapters of many requests beside a projection that they share:
//     Y[t] = Y0[t] + s_a (x_t A_a^T) B_a^T,   a the adapter of row t.
// Rows with the same adapter are taken 16 or 32 at a time, so that an adapter is read once for so many of its rows, wherever they
// are in the batch: for a given number of rows (which sets the parts of the channel axis) the sum is the same for a row whatever its neighbours.  Two launches, P = x A^T in parts of the channel axis
// and Y = Y0 + s P B^T, which adds the parts in their order; a third in front sorts the rows by adapter when there are
// more than 64 of them (up to 64 the groups are formed by a ballot in every wavefront).  A few operations per byte of A, B,
// X and Y: bound by memory, or by the launches when few rows come.
//
// Both products are formed transposed (rank or output in the rows of the 16 x 16 accumulator, token in its columns), so a lane
// holds four consecutive ranks or outputs of one token and loads and stores 16 bytes.  A and B are bf16; fp32 X and the
// fp32 P enter the bf16 instruction as three terms that add up to all 24 bits (v = v1 + v2 + v3, each the rounded rest).  Rows where they do not (values
// below 1e-33 or so, the largest finite ones, infinities) are done again by the fp32 instruction, which for a whole call of such rows takes three times as
// long: 4099 rows 140 -> 465 us.  Looking whether there are any costs 1 to 3 %.
// Measured: 4099 rows of 4096 fp32 inputs, 14336 outputs, rank 64, 6 adapters: sorting 8.7 us, P 23 to 24 (67 MB of X, 2.8 TB/s), Y 106 to 109
// (470 MB of Y0 and Y, 4.4 TB/s; a plain copy reaches 5.3); 48 rows, 4096 by 4096, rank 16, 16 adapters 4.2 + 5.8.
#include "bf16_pair.h"
#include "aser_internal.h"

namespace {

typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

constexpr int kFewRows = 64;        // up to here groups are formed by ballot, in tiles of 16 rows
constexpr int kManyTiles = 2;       // beyond, a tile has so many times 16 rows
constexpr int kMaxAdapters = 4096;

struct AdArgs {
    const void* X; int64_t ldx; int64_t rows, n;
    const int32_t* id;
    const uint16_t* A; const uint16_t* B; const float* scale;
    int n_adapters, r, rp;          // rp: r rounded up to 16
    int64_t m;
    const float* Y0; int64_t ldy0; float* Y; int64_t ldy;
    float* P; int parts; int64_t part_n;     // [part][row][rp]; channels of a part (a multiple of 32)
    int4* tiles; int32_t* order;    // more than kFewRows rows: (adapter, first place in order, rows, 0), rows sorted by adapter
};

// Sorts the rows by adapter (rows without one last) and cuts the result into tiles.  One workgroup: counts per adapter, their
// running sums, places.  The rows of a prompt have one adapter: a wavefront whose rows agree counts them in one step.
__global__ __launch_bounds__(1024) void adapter_sort_kernel(AdArgs g, int tok, int max_tiles) {
    __shared__ int cnt[kMaxAdapters + 1], wave_rows[16], wave_tiles[16];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, na = g.n_adapters;
    auto take = [&](int64_t base, bool place) {        // 64 rows from base on
        const bool in = base + lane < g.rows;
        int a = in ? g.id[base + lane] : 0;
        if ((uint32_t)a >= (uint32_t)na) a = na;
        const int a0 = __builtin_amdgcn_readfirstlane(a);
        const uint64_t here = __ballot(in);
        int at;
        if (__ballot(in & (a == a0)) == here) {
            int first = 0;
            if (lane == 0) first = atomicAdd(&cnt[a0], __popcll(here));
            at = __builtin_amdgcn_readfirstlane(first) + lane;
        } else {
            at = in ? atomicAdd(&cnt[a], 1) : 0;
        }
        if (place && in) g.order[at] = (int32_t)(base + lane);
    };
    for (int i = tid; i <= na; i += 1024) cnt[i] = 0;
    __syncthreads();
    for (int64_t base = 64 * wave; base < g.rows; base += 1024) take(base, false);
    __syncthreads();
    // thread i owns `per` consecutive adapters
    const int per = (na + 1 + 1023) / 1024, lo = min(tid * per, na + 1), hi = min(lo + per, na + 1);
    int nr = 0, nt = 0;
    for (int i = lo; i < hi; ++i) { nr += cnt[i]; nt += (cnt[i] + tok - 1) / tok; }
    int r0 = nr, t0 = nt;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int x = __shfl_up(r0, o), y = __shfl_up(t0, o);
        r0 += lane >= o ? x : 0;
        t0 += lane >= o ? y : 0;
    }
    if (lane == 63) { wave_rows[wave] = r0; wave_tiles[wave] = t0; }
    __syncthreads();
    int total = 0;
    r0 -= nr;
    t0 -= nt;
    for (int w = 0; w < 16; ++w) {
        r0 += w < wave ? wave_rows[w] : 0;
        t0 += w < wave ? wave_tiles[w] : 0;
        total += wave_tiles[w];
    }
    for (int i = lo; i < hi; ++i) {
        const int c = cnt[i];
        for (int x = 0; x < c; x += tok) g.tiles[t0++] = make_int4(i < na ? i : -1, r0 + x, min(tok, c - x), 0);
        cnt[i] = r0;                                   // from here on: the next free place
        r0 += c;
    }
    for (int i = total + tid; i < max_tiles; i += 1024) g.tiles[i] = make_int4(-2, 0, 0, 0);
    __syncthreads();
    for (int64_t base = 64 * wave; base < g.rows; base += 1024) take(base, true);
}

// The rows of a workgroup's tile: adapter (-1: rows without one, -2: no such tile) and the rows in columns `col` (+ 16 ..), -1 past the last.
template <int NT>
struct TileRows {
    int adapter, row[NT];
    __device__ __forceinline__ TileRows(const AdArgs& g, int tile, int lane) {
        const int col = lane & 15;
        if constexpr (NT > 1) {
            const int4 t = g.tiles[tile];
            adapter = t.x;
#pragma unroll
            for (int x = 0; x < NT; ++x) row[x] = 16 * x + col < t.z ? g.order[t.y + 16 * x + col] : -1;
        } else {
            // tile = slots j + q: the rows whose adapter is row j's, if no earlier row has it; 16 q .. of them
            const int slots = (int)((g.rows + 15) / 16), j = tile / slots, skip = tile % slots * 16;
            int a = lane < g.rows ? g.id[lane] : -2;
            if (lane < g.rows && (uint32_t)a >= (uint32_t)g.n_adapters) a = -1;
            const int mine = __builtin_amdgcn_readlane(a, j);
            const uint64_t same = __ballot(a == mine && lane < g.rows);
            adapter = (int)(__ffsll((unsigned long long)same) - 1) == j && __popcll(same) > skip ? mine : -2;
            row[0] = -1;
            if (adapter == -2) return;
            uint64_t left = same;
            for (int i = 0, k = __popcll(same); i < k; ++i) {
                const int at = __ffsll((unsigned long long)left) - 1;
                left &= left - 1;
                if (i == skip + col) row[0] = at;
            }
        }
    }
};

__device__ __forceinline__ bf16x8_t pack8(const float x[8]) {
    return __builtin_bit_cast(bf16x8_t, make_uint4(bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3]), bf16_pair(x[4], x[5]), bf16_pair(x[6], x[7])));
}
// x as three bf16 terms.  Returns the bits of what they leave, 0 unless some value is out of their range: some last bits of one below 1e-33 or so fall under
// the smallest bf16 value, one above the largest rounds to an infinity, and from an infinity or a NaN nothing can be taken away.
__device__ __forceinline__ uint32_t three_terms(const float v[8], bf16x8_t t[3]) {
#pragma clang fp contract(off)                     // a product that v is the rounded value of would leave its own last bits
    float x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = v[j];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        t[k] = pack8(x);
        const uint4 w = __builtin_bit_cast(uint4, t[k]);
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            x[2 * j] -= __uint_as_float(u[j] << 16);
            x[2 * j + 1] -= __uint_as_float(u[j] & 0xFFFF0000u);
        }
    }
    uint32_t rest = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) rest |= __float_as_uint(x[j]);
    return rest;
}
// One step of 32 with the terms of x, and with x itself by eight fp32 instructions (each takes one of a lane's eight: the order of a step is free as long as
// both operands agree).  The second takes several times as long and is for columns whose x has no three terms.
__device__ __forceinline__ f32x4_t terms_step(bf16x8_t a, const bf16x8_t t[3], f32x4_t acc) {
#pragma unroll
    for (int k = 2; k >= 0; --k) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, t[k], acc, 0, 0, 0);
    return acc;
}
__device__ __forceinline__ f32x4_t exact_step(bf16x8_t a, const float x[8], f32x4_t acc) {
    const uint4 w = __builtin_bit_cast(uint4, a);
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(u[j] << 16), x[2 * j], acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(u[j] & 0xFFFF0000u), x[2 * j + 1], acc, 0, 0, 0);
    }
    return acc;
}
// Bit c: some lane of column c says so.  A column is decided by its own values, so a row's result does not depend on the other rows of its tile.
__device__ __forceinline__ uint32_t columns_where(bool lane_says) {
    const uint64_t b = __ballot(lane_says), h = b | b >> 32;
    return (uint32_t)(h | h >> 16) & 0xFFFFu;
}

// Eight consecutive values of a row of n, from column c on; zeros past its end.  Rows start where they like: the loads take 16 bytes from any
// element on.  last (the same for all lanes): the row may end inside or before these eight; then the row's last eight are loaded and moved down.
// Before, rows of other than a multiple of 8 values were read one by one: 315 rows of 258 inputs, 675 outputs, rank 128 33.6 us, with these loads 26.1;
// 1962 rows of 5035 outputs 51.5 and 39.4.
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));

__device__ __forceinline__ bf16x8_t row8(const uint16_t* row, int64_t c, int64_t n, bool last) {
    if (n < 8) {
        uint32_t u[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) u[j] = c + j < n ? row[c + j] : 0u;
        return __builtin_bit_cast(bf16x8_t, make_uint4(u[0] | u[1] << 16, u[2] | u[3] << 16, u[4] | u[5] << 16, u[6] | u[7] << 16));
    }
    const u32x4_any w = *(const u32x4_any*)(row + (c < n - 8 ? c : n - 8));
    uint64_t lo = w.x | (uint64_t)w.y << 32, hi = w.z | (uint64_t)w.w << 32;
    if (last) {
        const int64_t past = c - (n - 8);
        const int down = past < 0 ? 0 : past > 8 ? 8 : (int)past, bits = 16 * (down & 3);
        if (down & 4) { lo = hi; hi = 0; }
        lo = lo >> bits | (bits ? hi << (64 - bits) : 0);
        hi >>= bits;
        if (down == 8) lo = hi = 0;
    }
    return __builtin_bit_cast(bf16x8_t, make_uint4((uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)));
}
__device__ __forceinline__ void row8_f32(const float* row, int64_t c, int64_t n, bool last, float x[8]) {
    if (n < 8) {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = c + j < n ? row[c + j] : 0.f;
        return;
    }
    const float* at = row + (c < n - 8 ? c : n - 8);
    const f32x4_any a = *(const f32x4_any*)at, b = *(const f32x4_any*)(at + 4);
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    if (last) {
        const int64_t past = c - (n - 8);
        const int down = past < 0 ? 0 : past > 8 ? 8 : (int)past;
#pragma unroll
        for (int step = 8; step; step >>= 1)
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = (down & step) == 0 ? x[j] : j + step < 8 ? x[j + step] : 0.f;
    }
}

// P[part][row][.] = x A^T over the part's channels; the four wavefronts take every fourth step of 32 channels.
template <int RT, bool F32, int NT>
__global__ __launch_bounds__(256) void adapter_down_kernel(AdArgs g) {
    __shared__ f32x4_t sm[3][NT][RT][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, grp = lane >> 4;
    const int part = blockIdx.x % g.parts;
    const TileRows<NT> tr(g, blockIdx.x / g.parts, lane);
    if (tr.adapter < 0) return;
    const int64_t c0 = part * g.part_n, c1 = c0 + g.part_n < g.n ? c0 + g.part_n : g.n;
    const uint16_t* a_row = g.A + (int64_t)tr.adapter * g.r * g.n;
    f32x4_t acc[NT][RT];
#pragma unroll
    for (int x = 0; x < NT; ++x)
#pragma unroll
        for (int i = 0; i < RT; ++i) acc[x][i] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
    uint32_t rest[NT] = {};
    for (int64_t c = c0 + 32 * wave; c < c1; c += 128) {
        const int64_t at = c + 8 * grp;
        const bool last = c + 32 > g.n;
        bf16x8_t a[RT];
        float xf[NT][8];
        bf16x8_t xb[NT];
#pragma unroll
        for (int x = 0; x < NT; ++x) {
            const int64_t row = max(tr.row[x], 0);     // a column without a row is not stored
            if (F32) row8_f32((const float*)g.X + row * g.ldx, at, g.n, last, xf[x]);
            else xb[x] = row8((const uint16_t*)g.X + row * g.ldx, at, g.n, last);
        }
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            a[i] = row8(a_row + min(16 * i + col, g.r - 1) * g.n, at, g.n, last);
            if (16 * i + 16 > g.r && 16 * i + col >= g.r) a[i] = __builtin_bit_cast(bf16x8_t, make_uint4(0u, 0u, 0u, 0u));
        }
#pragma unroll
        for (int x = 0; x < NT; ++x) {
            if constexpr (F32) {
                bf16x8_t t[3];
                rest[x] |= three_terms(xf[x], t);
#pragma unroll
                for (int i = 0; i < RT; ++i) acc[x][i] = terms_step(a[i], t, acc[x][i]);
            } else {
#pragma unroll
                for (int i = 0; i < RT; ++i) acc[x][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[i], xb[x], acc[x][i], 0, 0, 0);
            }
        }
    }
    if constexpr (F32) {
#pragma unroll
        for (int x = 0; x < NT; ++x) {
            const uint32_t exact = columns_where(rest[x] != 0);
            if (exact == 0) continue;
            // rare: these columns again, with all bits, one tile of ranks after the other
            const float* x_row = (const float*)g.X + (int64_t)max(tr.row[x], 0) * g.ldx;
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                f32x4_t v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
                for (int64_t c = c0 + 32 * wave; c < c1; c += 128) {
                    float xs[8];
                    row8_f32(x_row, c + 8 * grp, g.n, c + 32 > g.n, xs);
                    v = exact_step(row8(a_row + min(16 * i + col, g.r - 1) * g.n, c + 8 * grp, g.n, c + 32 > g.n), xs, v);
                }
                acc[x][i] = exact >> col & 1 ? v : acc[x][i];
            }
        }
    }
    if (wave)
#pragma unroll
        for (int x = 0; x < NT; ++x)
#pragma unroll
            for (int i = 0; i < RT; ++i) sm[wave - 1][x][i][lane] = acc[x][i];
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int x = 0; x < NT; ++x) {
        if (tr.row[x] < 0) continue;
        float* dst = g.P + ((int64_t)part * g.rows + tr.row[x]) * g.rp;
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            f32x4_t v = acc[x][i];
#pragma unroll
            for (int w = 0; w < 3; ++w) v += sm[w][x][i][lane];
            if (16 * i < g.rp) *(f32x4_t*)(dst + 16 * i + 4 * grp) = v;
        }
    }
}

// Y = Y0 + s P B^T: a wavefront has 64 outputs, a workgroup 256 (several times as many for each wavefront, with P kept, were slower: 300 rows, 4096 outputs:
// 15.4 us, 22.8 with four).  The accumulators go through LDS, so that Y0 and Y are read and written 256 bytes of a row at a time (4099 rows of 14336: 113
// -> 106).
template <int KS, int NT>
__global__ __launch_bounds__(256, NT > 1 ? 3 : 4) void adapter_up_kernel(AdArgs g) {
    constexpr int ROWS = 16 * NT, PITCH = 68;      // floats of a row in LDS
    constexpr int SUMS = 4 * NT * KS * 2 * 64 * 4, TURN = 4 * ROWS * PITCH;
    __shared__ __align__(16) float sm[SUMS > TURN ? SUMS : TURN];
    const int blocks = (int)((g.m + 255) / 256), block = blockIdx.x % blocks;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, grp = lane >> 4;
    const TileRows<NT> tr(g, blockIdx.x / blocks, lane);
    if (tr.adapter == -2 || (tr.adapter == -1 && g.Y0 == g.Y)) return;
    const bool some = tr.adapter >= 0;
    // this lane's rows and outputs at the turn: rows 4 j + grp, four outputs from 4 col on.  Y0 is asked for first of all: 1962 rows of 5035 outputs
    // 39.4 -> 36.6 us.
    int out_row[4 * NT];
#pragma unroll
    for (int j = 0; j < 4 * NT; ++j) out_row[j] = __shfl(tr.row[j / 4], 4 * (j % 4) + grp);
    float* turn = sm + wave * ROWS * PITCH;
    const int64_t o0 = (int64_t)block * 256 + wave * 64;
    const int64_t o = o0 + 4 * col;
    const bool four = o + 4 <= g.m;
    f32x4_t y[4 * NT];
#pragma unroll
    for (int j = 0; j < 4 * NT; ++j) {
        y[j] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
        if (g.Y0 && out_row[j] >= 0 && o < g.m) {
            const float* y0 = g.Y0 + (int64_t)out_row[j] * g.ldy0 + o;
            if (four) y[j] = __builtin_nontemporal_load((const f32x4_any*)y0);
            else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (o + e < g.m) y[j][e] = y0[e];
            }
        }
    }
    bf16x8_t t[NT][KS][3];
    uint32_t exact[NT];                            // columns whose P has no three terms
    const uint16_t* b = g.B;
    const float s = some && g.scale ? g.scale[tr.adapter] : 1.f;
    if (some) {
        b += (int64_t)tr.adapter * g.m * g.r;
        f32x4_t* sums = (f32x4_t*)sm;              // [wave][NT][KS][2][lane]
        // a wavefront adds every fourth part, the four sums meet
#pragma unroll
        for (int x = 0; x < NT; ++x)
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                const int at = 32 * k + 8 * grp;
                f32x4_t u = {0.f, 0.f, 0.f, 0.f}, v = u;
                if (tr.row[x] >= 0 && at < g.rp) {
#pragma unroll 4
                    for (int part = wave; part < g.parts; part += 4) {
                        const float* src = g.P + ((int64_t)part * g.rows + tr.row[x]) * g.rp + at;
                        u += *(const f32x4_t*)src;
                        v += *(const f32x4_t*)(src + 4);
                    }
                }
                sums[(((wave * NT + x) * KS + k) * 2) * 64 + lane] = u;
                sums[(((wave * NT + x) * KS + k) * 2 + 1) * 64 + lane] = v;
            }
        __syncthreads();
#pragma unroll
        for (int x = 0; x < NT; ++x) {
            uint32_t rest = 0;
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                f32x4_t w[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const f32x4_t* at = sums + ((x * KS + k) * 2 + j) * 64 + lane;
                    constexpr int NEXT = NT * KS * 2 * 64;
                    w[j] = (at[0] + at[NEXT]) + (at[2 * NEXT] + at[3 * NEXT]);
                }
                const float p[8] = {w[0][0] * s, w[0][1] * s, w[0][2] * s, w[0][3] * s, w[1][0] * s, w[1][1] * s, w[1][2] * s, w[1][3] * s};
                rest |= three_terms(p, t[x][k]);
            }
            exact[x] = columns_where(rest != 0);
        }
        __syncthreads();                           // before the turns below overwrite the sums
    }
    if (o0 >= g.m) return;
    if (some) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f32x4_t acc[NT];
#pragma unroll
            for (int x = 0; x < NT; ++x) acc[x] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
            const int64_t row = min(o0 + 16 * i + col, g.m - 1);   // an output past the last is not stored
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                const bf16x8_t w = row8(b + row * g.r, 32 * k + 8 * grp, g.r, 32 * k + 32 > g.r);
#pragma unroll
                for (int x = 0; x < NT; ++x) acc[x] = terms_step(w, t[x][k], acc[x]);
            }
#pragma unroll
            for (int x = 0; x < NT; ++x) *(f32x4_t*)(turn + (16 * x + col) * PITCH + 16 * i + 4 * grp) = acc[x];
        }
#pragma unroll
        for (int x = 0; x < NT; ++x) {
            if (exact[x] == 0) continue;
            // rare: these columns again, with all bits; P from its parts once more, added in the same order
#pragma unroll 1
            for (int i = 0; i < 4; ++i) {
                f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
                for (int k0 = 0; k0 < g.r; k0 += 32) {
                    const int at = k0 + 8 * grp;
                    f32x4_t pair[2][2] = {};
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        f32x4_t u = {0.f, 0.f, 0.f, 0.f}, v = u;
#pragma unroll 1
                        for (int part = w; part < g.parts && tr.row[x] >= 0 && at < g.rp; part += 4) {
                            const float* src = g.P + ((int64_t)part * g.rows + tr.row[x]) * g.rp + at;
                            u += *(const f32x4_t*)src;
                            v += *(const f32x4_t*)(src + 4);
                        }
                        pair[w / 2][0] = w % 2 ? pair[w / 2][0] + u : u;
                        pair[w / 2][1] = w % 2 ? pair[w / 2][1] + v : v;
                    }
                    const f32x4_t lo = pair[0][0] + pair[1][0], hi = pair[0][1] + pair[1][1];
                    float p[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) p[j] = at + j < g.r ? (j < 4 ? lo[j % 4] : hi[j % 4]) * s : 0.f;   // behind the rank: an infinity of X has left NaN
                    acc = exact_step(row8(b + min(o0 + 16 * i + col, g.m - 1) * g.r, at, g.r, k0 + 32 > g.r), p, acc);
                }
                if (exact[x] >> col & 1) *(f32x4_t*)(turn + (16 * x + col) * PITCH + 16 * i + 4 * grp) = acc;
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int j = 0; j < 4 * NT; ++j) y[j] += *(const f32x4_t*)(turn + (4 * j + grp) * PITCH + 4 * col);
    }
#pragma unroll
    for (int j = 0; j < 4 * NT; ++j) {
        if (out_row[j] < 0) continue;
        float* dst = g.Y + (int64_t)out_row[j] * g.ldy + o;
        if (four) *(f32x4_any*)dst = y[j];
        else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (o + e < g.m) dst[e] = y[j][e];
        }
    }
}

struct AdPlan { int tok, tiles, parts; int64_t part_n; size_t p_bytes, order_bytes, tile_bytes; };

AdPlan plan_adapters(int64_t rows, int64_t n, int r) {
    AdPlan p;
    const bool few = rows <= kFewRows;
    p.tok = few ? 16 : 16 * kManyTiles;
    p.tiles = (int)(few ? ceil_div64(rows, p.tok) * rows : ceil_div64(rows, p.tok) + kMaxAdapters + 1);
    // parts of the channel axis: about 512 workgroups, at least 256 channels each (1024 workgroups: 4099 rows of 4096 inputs, 14336 outputs 140 -> 153 us,
    // whose many blocks of outputs add the parts each; 3434 rows of 7459 inputs, 869 outputs 64.5 -> 59.1)
    const int64_t groups = few ? rows : ceil_div64(rows, p.tok);
    int64_t parts = ceil_div64(512, groups);
    if (parts > ceil_div64(n, 256)) parts = ceil_div64(n, 256);
    if (parts > 16) parts = 16;
    p.part_n = align_up((size_t)ceil_div64(n, parts), 128);
    p.parts = (int)ceil_div64(n, p.part_n);
    p.p_bytes = align_up((size_t)p.parts * rows * align_up(r, 16) * 4, 256);
    p.order_bytes = few ? 0 : align_up((size_t)rows * 4, 256);
    p.tile_bytes = few ? 0 : align_up((size_t)p.tiles * 16, 256);
    return p;
}

template <int RT, int NT>
void launch_down(const AdArgs& g, bool f32, dim3 grid, hipStream_t st) {
    if (f32) adapter_down_kernel<RT, true, NT><<<grid, 256, 0, st>>>(g);
    else adapter_down_kernel<RT, false, NT><<<grid, 256, 0, st>>>(g);
}
template <int NT>
void launch_downs(const AdArgs& g, bool f32, dim3 grid, hipStream_t st) {
    if (g.r <= 16) launch_down<1, NT>(g, f32, grid, st);
    else if (g.r <= 32) launch_down<2, NT>(g, f32, grid, st);
    else if (g.r <= 64) launch_down<4, NT>(g, f32, grid, st);
    else launch_down<8, NT>(g, f32, grid, st);
}
template <int NT>
void launch_ups(const AdArgs& g, int64_t tiles, hipStream_t st) {
    const dim3 grid((unsigned)(tiles * ceil_div64(g.m, 256)));
    if (g.r <= 32) adapter_up_kernel<1, NT><<<grid, 256, 0, st>>>(g);
    else if (g.r <= 64) adapter_up_kernel<2, NT><<<grid, 256, 0, st>>>(g);
    else adapter_up_kernel<4, NT><<<grid, 256, 0, st>>>(g);
}

}  // namespace

extern "C" size_t aser_adapter_workspace_bytes(int64_t rows, int64_t n, int64_t m, int32_t r) {
    if (rows <= 0 || n <= 0 || m <= 0 || r <= 0) return kAserWsTail;
    const AdPlan p = plan_adapters(rows, n, r);
    return p.p_bytes + p.order_bytes + p.tile_bytes + kAserWsTail;
}

extern "C" int aser_adapter_forward(aser_ctx* ctx, const void* X, int x_dtype, int64_t rows, int64_t n, int64_t ldx, const int32_t* adapter,
                                    const uint16_t* A, const uint16_t* B, const float* scale, int32_t n_adapters, int32_t r, int64_t m,
                                    const float* Y0, int64_t ldy0, float* Y, int64_t ldy) {
    if (!ctx) return ASER_ERR_INVALID_ARG;
    if (!A || !B || (rows != 0 && (!X || !adapter || !Y))) ASER_FAIL(ctx, ASER_ERR_INVALID_ARG, "adapter_forward: null pointer");
    if (x_dtype != ASER_DTYPE_BF16 && x_dtype != ASER_DTYPE_F32) ASER_FAIL(ctx, ASER_ERR_DTYPE, "adapter_forward: dtype must be bf16 or f32");
    if (rows < 0 || rows > INT32_MAX / 32 || n <= 0 || m <= 0 || ldx < n || ldy < m || (Y0 && (ldy0 < m || (Y0 == Y && ldy0 != ldy))) || m > ((int64_t)1 << 23))
        ASER_FAIL(ctx, ASER_ERR_SHAPE, "adapter_forward: bad shape");
    if (r <= 0 || r > 128 || n_adapters <= 0 || n_adapters > kMaxAdapters) ASER_FAIL(ctx, ASER_ERR_SHAPE, "adapter_forward: r must be in [1, 128], n_adapters in [1, 4096]");
    const bool f32 = x_dtype == ASER_DTYPE_F32;
    if (((uintptr_t)X & (f32 ? 3 : 1)) || (((uintptr_t)A | (uintptr_t)B) & 1) || (((uintptr_t)Y | (uintptr_t)Y0 | (uintptr_t)scale | (uintptr_t)adapter) & 3))
        ASER_FAIL(ctx, ASER_ERR_INVALID_ARG, "adapter_forward: misaligned pointer");
    if (rows == 0) return ASER_OK;
    const AdPlan p = plan_adapters(rows, n, r);
    if (!ctx->ws || ctx->ws_bytes < p.p_bytes + p.order_bytes + p.tile_bytes + kAserWsTail) ASER_FAIL(ctx, ASER_ERR_WORKSPACE, "adapter_forward: workspace too small");
    AdArgs g{X, ldx, rows, n, adapter, A, B, scale, n_adapters, r, (int)align_up(r, 16), m, Y0, ldy0, Y, ldy, (float*)ctx->ws, p.parts, p.part_n, nullptr, nullptr};
    int tiles = p.tiles;
    ASER_TRY(aser_prepare_device(ctx));
    if (rows > kFewRows) {
        g.order = (int32_t*)((char*)ctx->ws + p.p_bytes);
        g.tiles = (int4*)((char*)ctx->ws + p.p_bytes + p.order_bytes);
        // no more tiles than full ones and one for each adapter, and for the rows without one, that is there
        const int64_t most = ceil_div64(rows, p.tok) + (n_adapters + 1 < rows ? n_adapters + 1 : rows);
        tiles = (int)(most < p.tiles ? most : p.tiles);
        adapter_sort_kernel<<<1, 1024, 0, ctx->stream>>>(g, p.tok, tiles);
        ASER_TRY(aser_check_launch(ctx, "adapter_sort_kernel"));
    }
    if (tiles * ceil_div64(m, 256) > INT32_MAX) ASER_FAIL(ctx, ASER_ERR_SHAPE, "adapter_forward: too many rows times outputs");
    const dim3 down((unsigned)(tiles * (int64_t)p.parts));       // neighbours read the same rows: consecutive memory, whatever the rows' distance
    if (rows > kFewRows) launch_downs<kManyTiles>(g, f32, down, ctx->stream);
    else launch_downs<1>(g, f32, down, ctx->stream);
    ASER_TRY(aser_check_launch(ctx, "adapter_down_kernel"));
    if (rows > kFewRows) launch_ups<kManyTiles>(g, tiles, ctx->stream);
    else launch_ups<1>(g, tiles, ctx->stream);
    return aser_check_launch(ctx, "adapter_up_kernel");
}
