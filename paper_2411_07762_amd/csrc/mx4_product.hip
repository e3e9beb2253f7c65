// Products of matrices in microscaled 4 bits, dense or one matrix for each group of rows (experts), with the low-rank branch and the gated form behind them:
//     Z[p][o] = sum_i x[row(p)][i] w_e[o][i] + sum_k P[p][k] L_A_e[o][k],   P[p][k] = sum_i x[row(p)][i] L_B_e[k][i].
//
// The matrix instruction multiplies 32 four-bit floats of a row by 32 of another and scales each such product by the two blocks' powers of two.  A
// lane holds 32 channels of one row, a block, so the layout of the codes in memory is the layout of its operands.  Which blocks the lanes of an
// instruction hold does not matter as long as both operands agree.
#include <type_traits>

#include "bf16_pair.h"
#include "mx4.h"

namespace {

typedef int v4i_t __attribute__((ext_vector_type(4)));
typedef int v8i_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

struct MxArgs {
    MxGroups groups;
    const uint8_t* xc; const uint32_t* xs; int64_t x_rows;
    const uint8_t* wc; const uint32_t* ws; int64_t m;      // rows of a weight matrix
    int64_t n; int words;
    const uint16_t* la; const uint16_t* lb; int r, rp;      // rp: r rounded up to 16
    float* P; int parts; int part_words;                    // [part][position][rp]
    void* Y; int64_t ldy; int64_t outs;                     // columns of Y
    bool vec;                                               // four columns of Y at a time
    bool la_vec, lb_vec;                                    // rows of the factors in 16-byte loads
};

// Four-bit operands are the first four registers of the instruction's eight.
__device__ __forceinline__ v8i_t wide(const v4i_t& v) { return v8i_t{v[0], v[1], v[2], v[3], 0, 0, 0, 0}; }
template <int B>
__device__ __forceinline__ f32x4_t mfma16(const v4i_t& a, uint32_t sa, const v4i_t& b, uint32_t sb, const f32x4_t& c) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wide(a), wide(b), c, 4, 4, B, (int)sa, B, (int)sb);
}

__device__ __forceinline__ float gated(float gate, float up) { return gate / (1.f + expf(-gate)) * up; }

template <bool F32>
__device__ __forceinline__ void store4(const MxArgs& g, int64_t p, int64_t o, const float* y) {
    const int64_t at = p * g.ldy + o;
    if (g.vec && o + 4 <= g.outs) {
        if (F32) *(float4*)((float*)g.Y + at) = make_float4(y[0], y[1], y[2], y[3]);
        else *(uint2*)((uint16_t*)g.Y + at) = make_uint2(bf16_pair(y[0], y[1]), bf16_pair(y[2], y[3]));
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (o + i >= g.outs) continue;
        if (F32) ((float*)g.Y)[at + i] = y[i];
        else ((uint16_t*)g.Y)[at + i] = (uint16_t)bf16_rne(y[i]);
    }
}

// ---------------------------------------------------------------------------------------------------------------- P = x L_B^T
// 16 positions a workgroup; four wavefronts share a part of the channels, a scale word at a time: lane group q = lane / 16 has block q of it, 32 channels of
// its token, which become bf16 (exactly) eight at a time and meet 64 bytes of each row of L_B.  Ranks are in the rows of the accumulator.
template <int RF>
__global__ __launch_bounds__(256) void mx4_down_kernel(MxArgs g) {
    __shared__ __align__(16) float part[4][RF][64][4];
    const int lane = threadIdx.x & 63, li = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int pt = blockIdx.x % g.parts;
    int e, rows;
    int64_t p0;
    if (!mx4_find_tile(g.groups, blockIdx.x / g.parts, 16, &e, &p0, &rows)) return;
    const int64_t row = mx4_row(g.groups, p0 + (li < rows ? li : rows - 1));
    const uint8_t* const xc = g.xc + row * g.words * 64 + 16 * q;
    const uint32_t* const xs = g.xs + row;
    const uint16_t* const lb = g.lb + (int64_t)e * g.r * g.n;
    f32x4_t acc[RF];
#pragma unroll
    for (int f = 0; f < RF; ++f) acc[f] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    const int first = pt * g.part_words, last = first + g.part_words < g.words ? first + g.part_words : g.words;
    for (int w = first + wave; w < last; w += 4) {
        const v4i_t codes = *(const v4i_t*)(xc + (int64_t)w * 64);
        const uint32_t byte = (xs[(int64_t)w * g.x_rows] >> (8 * q)) & 255u;
        const float scale = byte == 0 ? __uint_as_float(0x00400000u) : byte == 255 ? __uint_as_float(0x7FC00000u) : __uint_as_float(byte << 23);
        const int64_t c0 = (int64_t)w * kMxWord + 32 * q;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            typedef float pair_t __attribute__((ext_vector_type(2)));
            const uint32_t w4 = (uint32_t)codes[j];
            const pair_t v0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w4, 1.f, 0), v1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w4, 1.f, 1),
                         v2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w4, 1.f, 2), v3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w4, 1.f, 3);
            const uint4 xv = make_uint4(upper_halves(v0[0] * scale, v0[1] * scale), upper_halves(v1[0] * scale, v1[1] * scale),
                                        upper_halves(v2[0] * scale, v2[1] * scale), upper_halves(v3[0] * scale, v3[1] * scale));
            const bf16x8_t b = __builtin_bit_cast(bf16x8_t, xv);
            const int64_t c = c0 + 8 * j;
#pragma unroll
            for (int f = 0; f < RF; ++f) {
                const int k = 16 * f + li;
                uint4 a = make_uint4(0u, 0u, 0u, 0u);
                if (k < g.r) {
                    const uint16_t* src = lb + (int64_t)k * g.n + c;
                    if (g.lb_vec) {                          // n is a multiple of 8: eight channels are there or none
                        if (c < g.n) a = *(const uint4*)src;
                    } else {
                        uint32_t h[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) h[i] = c + i < g.n ? src[i] : 0u;
                        a = make_uint4(h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16);
                    }
                }
                acc[f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), b, acc[f], 0, 0, 0);
            }
        }
    }
#pragma unroll
    for (int f = 0; f < RF; ++f) *(f32x4_t*)part[wave][f][lane] = acc[f];
    __syncthreads();
    for (int f = wave; f < RF; f += 4) {                     // ranks 16 f + 4 q .. + 3 of token li
        f32x4_t sum = *(const f32x4_t*)part[0][f][lane];
#pragma unroll
        for (int w = 1; w < 4; ++w) sum += *(const f32x4_t*)part[w][f][lane];
        if (li < rows) *(f32x4_t*)(g.P + ((int64_t)pt * g.groups.positions + p0 + li) * g.rp + 16 * f + 4 * q) = sum;
    }
}

// ---------------------------------------------------------------------------------------------------------------- few rows of a matrix
// A workgroup has 16 outputs (of each half, if gated) of up to 16 NT positions; its W wavefronts share the channels in chunks of 512, of which lane
// group q has the four blocks of word 4 c + q: one word of scales for four instructions, 64 bytes of codes a lane.  Outputs are in the rows of the
// accumulator, so a lane has four neighbouring ones of a position.  The sums of the wavefronts meet in LDS in a fixed order.
template <int NA, int NT, int W, bool F32>
__global__ __launch_bounds__(64 * W) void mx4_few_kernel(MxArgs g) {
    extern __shared__ __align__(16) float part[];            // [wavefront][fragment][lane][4]
    const int lane = threadIdx.x & 63, li = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int e, rows;
    int64_t p0;
    if (!mx4_find_tile(g.groups, blockIdx.y, 16 * NT, &e, &p0, &rows)) return;
    const int64_t o0 = (int64_t)blockIdx.x * 16, o = o0 + li < g.outs ? o0 + li : g.outs - 1;     // past the end: the last one again, not stored
    const uint8_t* ac[NA];
    const uint32_t* as[NA];
#pragma unroll
    for (int a = 0; a < NA; ++a) {
        const int64_t row = o + a * g.outs;
        ac[a] = g.wc + ((int64_t)e * g.m + row) * g.words * 64;
        as[a] = g.ws + (int64_t)e * g.words * g.m + row;
    }
    const uint8_t* bc[NT];
    const uint32_t* bs[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int at = 16 * t + li;
        const int64_t row = mx4_row(g.groups, p0 + (at < rows ? at : rows - 1));
        bc[t] = g.xc + row * g.words * 64;
        bs[t] = g.xs + row;
    }
    f32x4_t acc[NA][NT];
#pragma unroll
    for (int a = 0; a < NA; ++a)
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[a][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    for (int c = wave; 4 * c < g.words; c += W) {
        const bool there = 4 * c + q < g.words;
        const int64_t w = there ? 4 * c + q : g.words - 1;
        v4i_t av[NA][4], bv[NT][4];
        uint32_t sa[NA], sb[NT];
#pragma unroll
        for (int a = 0; a < NA; ++a) {
            sa[a] = as[a][w * g.m];
#pragma unroll
            for (int j = 0; j < 4; ++j) av[a][j] = *(const v4i_t*)(ac[a] + w * 64 + 16 * j);
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            sb[t] = bs[t][w * g.x_rows];
#pragma unroll
            for (int j = 0; j < 4; ++j) bv[t][j] = *(const v4i_t*)(bc[t] + w * 64 + 16 * j);
        }
        if (!there) {                                        // words past the end: zeros, at scales that keep them so
#pragma unroll
            for (int a = 0; a < NA; ++a) {
                sa[a] = 0x7F7F7F7Fu;
#pragma unroll
                for (int j = 0; j < 4; ++j) av[a][j] = v4i_t{0, 0, 0, 0};
            }
#pragma unroll
            for (int t = 0; t < NT; ++t) sb[t] = 0x7F7F7F7Fu;
        }
#pragma unroll
        for (int a = 0; a < NA; ++a)
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                acc[a][t] = mfma16<0>(av[a][0], sa[a], bv[t][0], sb[t], acc[a][t]);
                acc[a][t] = mfma16<1>(av[a][1], sa[a], bv[t][1], sb[t], acc[a][t]);
                acc[a][t] = mfma16<2>(av[a][2], sa[a], bv[t][2], sb[t], acc[a][t]);
                acc[a][t] = mfma16<3>(av[a][3], sa[a], bv[t][3], sb[t], acc[a][t]);
            }
    }
    if (g.P) {                                               // four ranks an instruction, in fp32; the wavefronts share them
        const uint16_t* la = g.la + (int64_t)e * g.m * g.r;
        for (int k0 = 4 * wave; k0 < g.r; k0 += 4 * W) {
            const int k = k0 + q;
            float lv[NA], pv[NT];
#pragma unroll
            for (int a = 0; a < NA; ++a) lv[a] = k < g.r ? __uint_as_float((uint32_t)la[(o + a * g.outs) * g.r + k] << 16) : 0.f;
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const int at = 16 * t + li;
                const float* src = g.P + (p0 + (at < rows ? at : rows - 1)) * g.rp + k;
                pv[t] = 0.f;
                for (int p = 0; p < g.parts; ++p) pv[t] += src[(int64_t)p * g.groups.positions * g.rp];
            }
#pragma unroll
            for (int a = 0; a < NA; ++a)
#pragma unroll
                for (int t = 0; t < NT; ++t) acc[a][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(lv[a], pv[t], acc[a][t], 0, 0, 0);
        }
    }
    f32x4_t* const mine = (f32x4_t*)part + lane;
#pragma unroll
    for (int a = 0; a < NA; ++a)
#pragma unroll
        for (int t = 0; t < NT; ++t) mine[((wave * NA + a) * NT + t) * 64] = acc[a][t];
    __syncthreads();
    for (int t = wave; t < NT; t += W) {
        f32x4_t z[NA];
#pragma unroll
        for (int a = 0; a < NA; ++a) {
            z[a] = mine[(a * NT + t) * 64];
#pragma unroll
            for (int w = 1; w < W; ++w) z[a] += mine[((w * NA + a) * NT + t) * 64];
        }
        float y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = NA == 2 ? gated(z[0][i], z[NA - 1][i]) : z[0][i];
        const int at = 16 * t + li;
        if (at < rows) store4<F32>(g, p0 + at, o0 + 4 * q, y);
    }
}

// ---------------------------------------------------------------------------------------------------------------- many rows of a matrix
// A workgroup has 64 MF outputs of 64 NF positions, a wavefront (2 x 2 of them, one for each SIMD) 32 MF x 32 NF.  A step is a scale word, 128 channels: 64 bytes of
// codes of every row and a word of scales go straight from memory into LDS, in 16-byte chunks whose place in a row is turned by the row so that 32 rows' reads meet all banks; a ring of
// four stages keeps three steps of loads in flight, one barrier a step.  The loads are inline assembly because the compiler would
// make every LDS read wait for all of them.  Half h = lane / 32 of the lanes holds blocks h and 2 + h of a step, one for each of its two instructions
// per pair of fragments, whose scales are bytes 0 and 2 of its word shifted by h bytes.
// Gated, a wavefront's first MF / 2 fragments are gates and the others the values that belong to them.
// Workgroup b runs on XCD b % 8; an XCD's tiles are numbered in panels of kPanel tiles of positions, so that its 32 workgroups share few slabs of either operand.
constexpr int kStages = 4, kPanel = 4;

__device__ __forceinline__ int chunk_at(int r, int c) { return r * 64 + ((c ^ ((r >> 2) & 3)) << 4); }

template <int B>
__device__ __forceinline__ f32x16_t mfma32(const v4i_t& a, uint32_t sa, const v4i_t& b, uint32_t sb, const f32x16_t& c) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wide(a), wide(b), c, 4, 4, B, (int)sa, B, (int)sb);
}

template <int MF, int NF, bool GATED, bool F32>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(1, 1))) void mx4_tile_kernel(MxArgs g, int out_tiles) {
    extern __shared__ __align__(16) char smem[];
    constexpr int BM = 64 * MF, BN = 64 * NF;
    constexpr int A_BYTES = BM * 64, B_BYTES = BN * 64, SA = A_BYTES + B_BYTES, SB = SA + BM * 4, STAGE = SB + BN * 4;
    constexpr int LOADS = MF + NF + 2;                       // of a wavefront for a stage
    const int tid = threadIdx.x, lane = tid & 63, li = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wa = wave >> 1, wb = wave & 1;

    const int64_t tiles = mx4_tiles(g.groups, BN), total = tiles * out_tiles, per_xcd = (total + 7) / 8;
    const int64_t id = (int64_t)(blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
    if ((blockIdx.x >> 3) >= per_xcd || id >= total) return;
    const int64_t panel = id / (kPanel * (int64_t)out_tiles), in_panel = id - panel * kPanel * out_tiles;
    const int64_t high = tiles - panel * kPanel < kPanel ? tiles - panel * kPanel : kPanel;
    int e, rows;
    int64_t p0;
    if (!mx4_find_tile(g.groups, panel * kPanel + in_panel % high, BN, &e, &p0, &rows)) return;
    const int64_t o0 = (in_panel / high) * (GATED ? BM / 2 : BM);
    // weight row of row r of the tile; past the end the last one, whose sums are not stored
    auto weight_row = [&](int r) {
        int64_t o, base = 0;
        if (GATED) {
            const int in = r % (32 * MF);                    // of the wavefront's rows, the first half are gates
            base = in >= 16 * MF ? g.outs : 0;
            o = o0 + (r / (32 * MF)) * (16 * MF) + in % (16 * MF);
        } else {
            o = o0 + r;
        }
        return base + (o < g.outs ? o : g.outs - 1);
    };
    auto token_row = [&](int r) { return mx4_row(g.groups, p0 + (r < rows ? r : rows - 1)); };

    // what this lane fetches: chunk lane % 4 of a row's slab of 64 bytes, 16 rows an instruction, and words of scales, 64 rows an instruction
    const char *ga[MF], *gb[NF], *gs[2];
    const int64_t pitch = (int64_t)g.words * 64;
    const int ch = (lane & 3) ^ ((lane >> 4) & 3);
#pragma unroll
    for (int t = 0; t < MF; ++t) ga[t] = (const char*)g.wc + ((int64_t)e * g.m + weight_row(16 * (MF * wave + t) + (lane >> 2))) * pitch + 16 * ch;
#pragma unroll
    for (int t = 0; t < NF; ++t) gb[t] = (const char*)g.xc + token_row(16 * (NF * wave + t) + (lane >> 2)) * pitch + 16 * ch;
    gs[0] = (const char*)(g.ws + (int64_t)e * g.words * g.m + weight_row(64 * (wave % MF) + lane));
    gs[1] = (const char*)(g.xs + token_row(64 * (wave % NF) + lane));
    const int64_t sa_step = g.m * 4, sb_step = g.x_rows * 4;
    const uint32_t ring = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
    // load number t of a stage
    auto issue = [&](int64_t s, int t) {
        const uint32_t slot = ring + (uint32_t)(s & (kStages - 1)) * STAGE;
        if (t < MF) {
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" : : "s"(slot + (uint32_t)(MF * wave + t) * 1024), "v"(ga[t]) : "memory", "m0");
            ga[t] += 64;
        } else if (t < MF + NF) {
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" : : "s"(slot + A_BYTES + (uint32_t)(NF * wave + t - MF) * 1024), "v"(gb[t - MF]) : "memory", "m0");
            gb[t - MF] += 64;
        } else if (t == MF + NF) {
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" : : "s"(slot + SA + (uint32_t)(wave % MF) * 256), "v"(gs[0]) : "memory", "m0");
            gs[0] += sa_step;
        } else {
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" : : "s"(slot + SB + (uint32_t)(wave % NF) * 256), "v"(gs[1]) : "memory", "m0");
            gs[1] += sb_step;
        }
    };
    auto wait = [&](int stages) {                            // until at most the loads of so many later stages are in flight
        if (stages == 2) asm volatile("s_waitcnt vmcnt(%0)" : : "n"(2 * LOADS) : "memory");
        else if (stages == 1) asm volatile("s_waitcnt vmcnt(%0)" : : "n"(LOADS) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
    };

    int offa[MF], offb[NF];
#pragma unroll
    for (int i = 0; i < MF; ++i) offa[i] = chunk_at(wa * 32 * MF + 32 * i + li, h);
#pragma unroll
    for (int j = 0; j < NF; ++j) offb[j] = A_BYTES + chunk_at(wb * 32 * NF + 32 * j + li, h);
    const int offsa = SA + (wa * 32 * MF + li) * 4, offsb = SB + (wb * 32 * NF + li) * 4;
    f32x16_t acc[MF][NF];
#pragma unroll
    for (int i = 0; i < MF; ++i)
#pragma unroll
        for (int j = 0; j < NF; ++j)
#pragma unroll
            for (int k = 0; k < 16; ++k) acc[i][j][k] = 0.f;
    v4i_t a0[MF], a1[MF], b0[NF], b1[NF];
    uint32_t sa[MF], sb[NF], na[MF], nb[NF];
    auto read0 = [&](const char* st, int t) {                // operand t of a step's first instruction, then the words of scales
        if (t < MF) a0[t] = *(const v4i_t*)(st + offa[t]);
        else if (t < MF + NF) b0[t - MF] = *(const v4i_t*)(st + offb[t - MF]);
        else if (t < 2 * MF + NF) na[t - MF - NF] = *(const uint32_t*)(st + offsa + 128 * (t - MF - NF));
        else nb[t - 2 * MF - NF] = *(const uint32_t*)(st + offsb + 128 * (t - 2 * MF - NF));
    };
    auto read1 = [&](const char* st, int t) {                // the second's: the neighbouring pair of chunks
        if (t < MF) a1[t] = *(const v4i_t*)(st + (offa[t] ^ 32));
        else b1[t - MF] = *(const v4i_t*)(st + (offb[t - MF] ^ 32));
    };
    const int64_t steps = g.words;
    for (int64_t s = 0; s < kStages - 1 && s < steps; ++s)
#pragma unroll
        for (int t = 0; t < LOADS; ++t) issue(s, t);
    wait(steps >= 3 ? 2 : steps == 2 ? 1 : 0);
    __syncthreads();
#pragma unroll
    for (int t = 0; t < 2 * (MF + NF); ++t) read0(smem, t);
    constexpr int M = MF * NF;                               // instructions of a half step
    constexpr int R0 = 2 * (MF + NF), R1 = MF + NF;
    constexpr int W = M > 4 ? 1 : 0;                         // the barrier's place in the second half
    auto step = [&](int64_t s, auto steady_tag) {
        constexpr bool STEADY = decltype(steady_tag)::value;
        const char* st = smem + (int)(s & (kStages - 1)) * STAGE;
        const char* sn = smem + (int)((s + 1) & (kStages - 1)) * STAGE;
        const bool more = STEADY || s + 1 < steps, fetch = STEADY || s + kStages - 1 < steps;
#pragma unroll
        for (int i = 0; i < MF; ++i) sa[i] = na[i] >> (8 * h);
#pragma unroll
        for (int j = 0; j < NF; ++j) sb[j] = nb[j] >> (8 * h);
        // first half: the operands of the second are read under its first instructions
#pragma unroll
        for (int k = 0; k < M; ++k) {
            const int i = k / NF, j = k % NF;
            acc[i][j] = mfma32<0>(a0[i], sa[i], b0[j], sb[j], acc[i][j]);
#pragma unroll
            for (int t = 0; t < R1; ++t)
                if (t * (M / 2) / R1 == k) read1(st, t);
            __builtin_amdgcn_sched_barrier(0);
        }
        // second half: the wait for the next stage, the reads of its first half, the loads of stage s + 3
#pragma unroll
        for (int k = 0; k < M; ++k) {
            const int i = k / NF, j = k % NF;
            acc[i][j] = mfma32<2>(a1[i], sa[i], b1[j], sb[j], acc[i][j]);
            if (k == W && more) {
                wait((STEADY || s + 2 < steps) ? 1 : 0);
                __syncthreads();                             // everyone's share has landed, and everyone is done with stage s - 1
            }
#pragma unroll
            for (int t = 0; t < R0; ++t)
                if (more && W + 1 + t * (M / 2 - W) / R0 == k) read0(sn, t);
#pragma unroll
            for (int t = 0; t < LOADS; ++t)
                if (fetch && M / 2 + t * (M / 2) / LOADS == k) issue(s + kStages - 1, t);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    int64_t s = 0;
    for (; s + kStages - 1 < steps; ++s) step(s, std::true_type{});
    for (; s < steps; ++s) step(s, std::false_type{});

    if (g.P) {                                               // the low-rank branch on the same accumulators: P as three bf16 terms that hold all its bits
        const uint16_t* const la = g.la + (int64_t)e * g.m * g.r;
        const uint16_t* lr[MF];
#pragma unroll
        for (int i = 0; i < MF; ++i) lr[i] = la + weight_row(wa * 32 * MF + 32 * i + li) * g.r;
        const float* pr[NF];
#pragma unroll
        for (int j = 0; j < NF; ++j) {
            const int at = wb * 32 * NF + 32 * j + li;
            pr[j] = g.P + (p0 + (at < rows ? at : rows - 1)) * g.rp;
        }
        const int64_t part = g.groups.positions * g.rp;
#pragma nounroll
        for (int k0 = 0; k0 < g.r; k0 += 16) {
            const int k = k0 + 8 * h;
            bf16x8_t pv[NF][3];
#pragma unroll
            for (int j = 0; j < NF; ++j) {
                float v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = 0.f;
                for (int p = 0; p < g.parts; ++p) {
                    const float4 x = *(const float4*)(pr[j] + p * part + k), y = *(const float4*)(pr[j] + p * part + k + 4);
                    v[0] += x.x; v[1] += x.y; v[2] += x.z; v[3] += x.w; v[4] += y.x; v[5] += y.y; v[6] += y.z; v[7] += y.w;
                }
#pragma unroll
                for (int u = 0; u < 3; ++u) {
                    uint32_t w[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        w[i] = bf16_pair(v[2 * i], v[2 * i + 1]);
                        v[2 * i] -= __uint_as_float(w[i] << 16);
                        v[2 * i + 1] -= __uint_as_float(w[i] & 0xFFFF0000u);
                    }
                    pv[j][u] = __builtin_bit_cast(bf16x8_t, make_uint4(w[0], w[1], w[2], w[3]));
                }
            }
#pragma unroll
            for (int i = 0; i < MF; ++i) {
                uint4 a = make_uint4(0u, 0u, 0u, 0u);
                if (g.la_vec) {
                    if (k < g.r) a = *(const uint4*)(lr[i] + k);
                } else {
                    uint32_t q[8];
#pragma unroll
                    for (int u = 0; u < 8; ++u) q[u] = k + u < g.r ? lr[i][k + u] : 0u;
                    a = make_uint4(q[0] | q[1] << 16, q[2] | q[3] << 16, q[4] | q[5] << 16, q[6] | q[7] << 16);
                }
                const bf16x8_t av = __builtin_bit_cast(bf16x8_t, a);
#pragma unroll
                for (int j = 0; j < NF; ++j)
#pragma unroll
                    for (int u = 2; u >= 0; --u) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(av, pv[j][u], acc[i][j], 0, 0, 0);
            }
        }
    }
    // acc[i][j][k]: output 32 i + 8 (k / 4) + 4 h + k % 4, position 32 j + li of the wavefront's.  32 positions at a time are turned through LDS (the wavefront's own
    // part of it), so that rows of Y are written in whole lines.
    constexpr int OF = GATED ? MF / 2 : MF;                  // fragments of outputs
    constexpr int SIZE = F32 ? 4 : 2, ROW = OF * 32 * SIZE + 16;
    const int64_t ow = o0 + wa * 32 * OF;
    __syncthreads();
    char* const mine = smem + wave * (32 * ROW);
#pragma unroll
    for (int j = 0; j < NF; ++j) {
        const int first = wb * 32 * NF + 32 * j;
        const int here = rows - first;                       // positions of these 32 that are there
#pragma unroll
        for (int i = 0; i < OF; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float y[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) y[u] = GATED ? gated(acc[i][j][4 * k + u], acc[MF - OF + i][j][4 * k + u]) : acc[i][j][4 * k + u];
                const int o = 32 * i + 8 * k + 4 * h;
                if (!g.vec) {
                    if (li < here) store4<F32>(g, p0 + first + li, ow + o, y);
                } else if (F32) {
                    *(float4*)(mine + li * ROW + o * 4) = make_float4(y[0], y[1], y[2], y[3]);
                } else {
                    *(uint2*)(mine + li * ROW + o * 2) = make_uint2(bf16_pair(y[0], y[1]), bf16_pair(y[2], y[3]));
                }
            }
        if (!g.vec) continue;
        __builtin_amdgcn_wave_barrier();
        constexpr int EACH = 16 / SIZE, PER = OF * 32 / EACH, ROWS = 64 / PER;      // outputs of a lane, lanes of a row, rows an instruction
        const int o = (lane % PER) * EACH;
#pragma unroll
        for (int t = 0; t < 32; t += ROWS) {
            const int r = t + lane / PER;
            const uint4 v = *(const uint4*)(mine + r * ROW + o * SIZE);
            if (r >= here) continue;
            char* const dst = (char*)g.Y + ((p0 + first + r) * g.ldy + ow + o) * SIZE;
            if (ow + o + EACH <= g.outs) {
                *(uint4*)dst = v;
            } else {
                const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int u = 0; u < EACH; ++u) {
                    if (ow + o + u >= g.outs) continue;
                    if (F32) ((uint32_t*)dst)[u] = w[u % 4];
                    else ((uint16_t*)dst)[u] = (uint16_t)(w[(u / 2) % 4] >> (16 * (u & 1)));
                }
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
}

template <int NA, int NT, int W>
void launch_few(const MxArgs& g, dim3 grid, bool f32, hipStream_t s) {
    const size_t lds = (size_t)W * NA * NT * 1024;
    if (f32) mx4_few_kernel<NA, NT, W, true><<<grid, 64 * W, lds, s>>>(g);
    else mx4_few_kernel<NA, NT, W, false><<<grid, 64 * W, lds, s>>>(g);
}

template <int MF, int NF, bool GATED, bool F32>
int launch_tile_one(aser_ctx* ctx, const MxArgs& g) {
    constexpr int kRing = kStages * (64 * MF + 64 * NF) * 68, kTurn = 4 * 32 * ((GATED ? MF / 2 : MF) * 32 * (F32 ? 4 : 2) + 16), kLds = kRing > kTurn ? kRing : kTurn;
    static_assert(kLds <= 160 * 1024, "the ring and the turned outputs have to fit the LDS of a compute unit");
    const auto kernel = mx4_tile_kernel<MF, NF, GATED, F32>;
    ASER_HIP(ctx, hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, kLds));
    const int64_t out_tiles = ceil_div64(g.outs, GATED ? 32 * MF : 64 * MF), grid = ceil_div64(g.groups.most_tiles(64 * NF) * out_tiles, 8) * 8;
    if (grid > INT32_MAX) ASER_FAIL(ctx, ASER_ERR_SHAPE, "mx4: too many rows times outputs");
    kernel<<<(unsigned)grid, 256, kLds, ctx->stream>>>(g, (int)out_tiles);
    return aser_check_launch(ctx, "mx4_tile_kernel");
}
template <int MF, int NF>
int launch_tile(aser_ctx* ctx, const MxArgs& g, bool gated, bool f32) {
    if (gated) return f32 ? launch_tile_one<MF, NF, true, true>(ctx, g) : launch_tile_one<MF, NF, true, false>(ctx, g);
    return f32 ? launch_tile_one<MF, NF, false, true>(ctx, g) : launch_tile_one<MF, NF, false, false>(ctx, g);
}

struct Plan {
    int nt;                  // 16 nt positions a workgroup
    int nf;                  // not 0: 64 nf positions a workgroup, 256 outputs
    int parts, part_words;   // of the channels, for P
    size_t p_bytes;
};

Plan plan_product(int64_t positions, int64_t n, int32_t count, int32_t r) {
    Plan p{};
    const int64_t each = ceil_div64(positions, count < positions ? count : positions);
    p.nt = each <= 16 ? 1 : each <= 32 ? 2 : 4;
    p.nf = each <= 64 ? 0 : each <= 128 ? 2 : 4;
    const int64_t words = mx4_words(n), tiles = ceil_div64(positions, 16);
    int64_t parts = tiles >= 256 ? 1 : ceil_div64(256, tiles);
    if (parts > ceil_div64(words, 8)) parts = ceil_div64(words, 8);
    p.part_words = (int)ceil_div64(words, parts);
    p.parts = (int)ceil_div64(words, p.part_words);
    p.p_bytes = r > 0 ? align_up((size_t)p.parts * positions * align_up(r, 16) * 4, 256) : 0;
    return p;
}

template <int RF>
void launch_down(const MxArgs& g, unsigned grid, hipStream_t s) { mx4_down_kernel<RF><<<grid, 256, 0, s>>>(g); }

int run_product(aser_ctx* ctx, const char* who, const aser_mx4* x, const aser_mx4* w, const MxGroups& groups, const uint16_t* L_A, const uint16_t* L_B, int32_t r,
                int32_t swiglu, void* Y, int32_t y_dtype, int64_t ldy) {
    if (y_dtype != ASER_DTYPE_BF16 && y_dtype != ASER_DTYPE_F32) ASER_FAIL(ctx, ASER_ERR_DTYPE, "%s: dtype must be bf16 or f32", who);
    if (x->n != w->n || x->count != 1) ASER_FAIL(ctx, ASER_ERR_SHAPE, "%s: x must be one matrix with the channels of w", who);
    if (r < 0 || r > 128) ASER_FAIL(ctx, ASER_ERR_SHAPE, "%s: r must be in [0, 128]", who);
    if (r > 0 && (!L_A || !L_B)) ASER_FAIL(ctx, ASER_ERR_INVALID_ARG, "%s: null factors", who);
    if (swiglu && (w->rows & 1)) ASER_FAIL(ctx, ASER_ERR_SHAPE, "%s: gates and values need an even number of outputs", who);
    const int64_t outs = swiglu ? w->rows / 2 : w->rows;
    if (ldy < outs || w->rows > ((int64_t)1 << 24) || groups.positions > INT32_MAX / 32) ASER_FAIL(ctx, ASER_ERR_SHAPE, "%s: bad shape", who);
    const bool f32 = y_dtype == ASER_DTYPE_F32;
    if (((uintptr_t)Y & (f32 ? 3 : 1)) || (((uintptr_t)L_A | (uintptr_t)L_B) & 1)) ASER_FAIL(ctx, ASER_ERR_INVALID_ARG, "%s: misaligned pointer", who);
    if (groups.positions == 0) return ASER_OK;
    if (!Y) ASER_FAIL(ctx, ASER_ERR_INVALID_ARG, "%s: null pointer", who);
    const Plan p = plan_product(groups.positions, w->n, w->count, r);
    if (p.p_bytes && (!ctx->ws || ctx->ws_bytes < p.p_bytes + kAserWsTail)) ASER_FAIL(ctx, ASER_ERR_WORKSPACE, "%s: workspace too small", who);
    MxArgs g{};
    g.groups = groups;
    g.xc = x->codes; g.xs = (const uint32_t*)x->scales; g.x_rows = x->rows;
    g.wc = w->codes; g.ws = (const uint32_t*)w->scales; g.m = w->rows;
    g.n = w->n; g.words = (int)mx4_words(w->n);
    g.la = L_A; g.lb = L_B; g.r = r; g.rp = (int)align_up(r, 16);
    g.P = r > 0 ? (float*)ctx->ws : nullptr; g.parts = p.parts; g.part_words = p.part_words;
    g.Y = Y; g.ldy = ldy; g.outs = outs;
    // the kernel for many rows stores 16 bytes at a time, the other one four columns
    const int64_t unit = p.nf || f32 ? 16 : 8, size = f32 ? 4 : 2;
    g.vec = !((uintptr_t)Y & (unit - 1)) && !(ldy * size & (unit - 1));
    g.la_vec = !((uintptr_t)L_A & 15) && !(r & 7);
    g.lb_vec = !((uintptr_t)L_B & 15) && !(w->n & 7);
    const int64_t down = groups.most_tiles(16) * p.parts, tiles = groups.most_tiles(16 * p.nt);
    if (down > INT32_MAX || tiles > 65535) ASER_FAIL(ctx, ASER_ERR_SHAPE, "%s: too many rows", who);
    ASER_TRY(aser_prepare_device(ctx));
    if (r > 0) {
        switch (g.rp / 16) {
            case 1: launch_down<1>(g, (unsigned)down, ctx->stream); break;
            case 2: launch_down<2>(g, (unsigned)down, ctx->stream); break;
            case 3: launch_down<3>(g, (unsigned)down, ctx->stream); break;
            case 4: launch_down<4>(g, (unsigned)down, ctx->stream); break;
            case 5: launch_down<5>(g, (unsigned)down, ctx->stream); break;
            case 6: launch_down<6>(g, (unsigned)down, ctx->stream); break;
            case 7: launch_down<7>(g, (unsigned)down, ctx->stream); break;
            default: launch_down<8>(g, (unsigned)down, ctx->stream); break;
        }
        ASER_TRY(aser_check_launch(ctx, "mx4_down_kernel"));
    }
    if (p.nf) return p.nf == 2 ? launch_tile<4, 2>(ctx, g, swiglu, f32) : launch_tile<4, 4>(ctx, g, swiglu, f32);
    const dim3 grid((unsigned)ceil_div64(outs, 16), (unsigned)tiles);
    if (swiglu) {
        if (p.nt == 1) launch_few<2, 1, 8>(g, grid, f32, ctx->stream);
        else if (p.nt == 2) launch_few<2, 2, 4>(g, grid, f32, ctx->stream);
        else launch_few<2, 4, 4>(g, grid, f32, ctx->stream);
    } else {
        if (p.nt == 1) launch_few<1, 1, 8>(g, grid, f32, ctx->stream);
        else if (p.nt == 2) launch_few<1, 2, 4>(g, grid, f32, ctx->stream);
        else launch_few<1, 4, 4>(g, grid, f32, ctx->stream);
    }
    return aser_check_launch(ctx, "mx4_few_kernel");
}

}  // namespace

extern "C" size_t aser_mx4_forward_workspace_bytes(int64_t rows, int64_t n, int64_t m, int32_t r) {
    return aser_expert_forward_workspace_bytes(rows, n, m, 1, r);
}

extern "C" int aser_mx4_forward(aser_ctx* ctx, const aser_mx4* x, const aser_mx4* w, const uint16_t* L_A, const uint16_t* L_B, int32_t r, int32_t swiglu, void* Y,
                                int32_t y_dtype, int64_t ldy) {
    if (!ctx) return ASER_ERR_INVALID_ARG;
    ASER_TRY(aser_mx4_check(ctx, "mx4_forward", x, true));
    ASER_TRY(aser_mx4_check(ctx, "mx4_forward", w, false));
    if (w->count != 1) ASER_FAIL(ctx, ASER_ERR_SHAPE, "mx4_forward: w must be one matrix");
    return run_product(ctx, "mx4_forward", x, w, MxGroups{nullptr, nullptr, 1, 1, x->rows}, L_A, L_B, r, swiglu, Y, y_dtype, ldy);
}

extern "C" size_t aser_expert_forward_workspace_bytes(int64_t positions, int64_t n, int64_t m, int32_t n_experts, int32_t r) {
    if (positions <= 0 || n <= 0 || m <= 0 || n_experts <= 0) return kAserWsTail;
    return plan_product(positions, n, n_experts, r).p_bytes + kAserWsTail;
}

extern "C" int aser_expert_forward(aser_ctx* ctx, const aser_mx4* x, const aser_mx4* w, const aser_expert_plan* plan, int32_t gather, const uint16_t* L_A,
                                   const uint16_t* L_B, int32_t r, int32_t swiglu, void* Y, int32_t y_dtype, int64_t ldy) {
    if (!ctx) return ASER_ERR_INVALID_ARG;
    ASER_TRY(aser_mx4_check(ctx, "expert_forward", x, true));
    ASER_TRY(aser_mx4_check(ctx, "expert_forward", w, false));
    ASER_TRY(aser_plan_check(ctx, "expert_forward", plan));
    if (w->count != plan->n_experts) ASER_FAIL(ctx, ASER_ERR_SHAPE, "expert_forward: w must have a matrix for each expert");
    const int64_t positions = plan->rows * plan->top_k;
    if (x->rows != (gather ? plan->rows : positions)) ASER_FAIL(ctx, ASER_ERR_SHAPE, "expert_forward: x must have a row for each %s", gather ? "token" : "position");
    if (positions > 0 && (!plan->offsets || (gather && !plan->order))) ASER_FAIL(ctx, ASER_ERR_INVALID_ARG, "expert_forward: null offsets or order");
    return run_product(ctx, "expert_forward", x, w, MxGroups{plan->offsets, gather ? plan->order : nullptr, plan->n_experts, plan->top_k, positions}, L_A, L_B, r,
                       swiglu, Y, y_dtype, ldy);
}
