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
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

struct MxArgs {
    MxGroups groups;
    const uint8_t* xc; const uint32_t* xs;
    const uint8_t* wc; const uint32_t* ws; int64_t m, w_size;   // rows of a weight matrix, units from one to the next
    int words;
    const uint16_t* la; const uint16_t* lb; int r;
    int64_t la_ld, lb_ld;                                   // their rows: r and n, or what they are padded to
    float* P; int parts, part_words, rp;                    // few rows: [part][position][rp] fp32, rp: r rounded up to 16
    uint16_t* planes; int lr_steps;                         // many rows: [term][position][32 lr_steps / terms] bf16; steps of 32 ranks and one term
    float* exact; uint8_t* marks;                           // and P itself, fp32, [position][32 lr_steps / terms], where terms do not hold it: [position][8], a byte for 16 ranks
    void* Y; int64_t ldy; int64_t outs;                     // columns of Y
    bool vec;                                               // 16 bytes (few rows: four columns) of Y at a time
    bool la_four;                                           // four ranks of L_A in a load
};

// Four-bit operands are the first four registers of the instruction's eight.
__device__ __forceinline__ v8i_t wide(const v4i_t& v) { return v8i_t{v[0], v[1], v[2], v[3], 0, 0, 0, 0}; }
__device__ __forceinline__ f32x4_t mfma16(const v4i_t& a, uint32_t sa, const v4i_t& b, uint32_t sb, const f32x4_t& c) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wide(a), wide(b), c, 4, 4, 0, (int)sa, 0, (int)sb);
}

// gate / (1 + exp(-gate)) * up.  For a bf16 result the exponential and the reciprocal of the instructions do: the rounded product before the exponential makes the factor about
// |gate| 2^-24 off below zero, 2^-17 at most, the instructions 2^-22, where the result is rounded to 2^-8; gates below -87 count as 0, less than 1e-36 of up.  The functions of
// fp32 take five times as many instructions.
template <bool F32>
__device__ __forceinline__ float gated(float gate, float up) {
    if (F32) return gate / (1.f + expf(-gate)) * up;
    return gate * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(gate * -1.44269504f)) * up;
}

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
        else ((uint16_t*)g.Y)[at + i] = (uint16_t)bf16_pair(y[i], y[i]);
    }
}

// ---------------------------------------------------------------------------------------------------------------- P = x L_B^T
// 16 NT positions and 16 ranks a workgroup; W wavefronts share a part of the channels, a word at a time with the loads of U words in flight.  Ranks are in the
// rows of the accumulator; tokens become bf16 on the way, exactly.
// TERMS = 0, few rows: fp32 sums of the part.  L_B goes into the registers as it is: of each of a word's four blocks lane group q = lane / 16 has channels 8 q .. + 7.
// Otherwise the sum (of one part) as so many bf16 terms, each what the ones before leave, rounded: three hold its 24 bits, two leave 2^-17 of it, and are taken for
// bf16 outputs, whose own rounding is 2^-8 (a third would be half as many steps of ranks again).  Where they do
// not (below 1e-33 or so bits fall under the smallest bf16 value, the largest numbers round to an infinity) a token's 16 sums are marked and kept in fp32, and their terms are zeros.
// Lane group q has block q, and L_B is turned through LDS: lanes next to each
// other in the matrix instruction have different rows, and a load of 16 bytes from 64 places occupies a compute unit's address unit for 64 cycles where one of four rows'
// 256 bytes takes 16.  Without that 4099 tokens of 4096 channels and 64 ranks take 25 us; with L_B put in order by a launch of its own 10 and 4.7.  Latency bounds it: 16 ranks of 32
// tokens and two words ahead, two workgroups a compute unit, take 10.8; 32 ranks and four words, one workgroup, 12.8; eight wavefronts 13 to 15; 64 tokens 11.6 to 12.5.
template <int NT, int W, int U, int TERMS>
__global__ __launch_bounds__(64 * W) void mx4_down_kernel(MxArgs g, int rank_tiles) {
    extern __shared__ __align__(16) float part[];            // the wavefronts' rows of L_B, then the sums, [wavefront][tokens][lane][4]
    constexpr bool TURNED = TERMS > 0;
    const int lane = threadIdx.x & 63, li = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int rt = blockIdx.x % rank_tiles, rest = blockIdx.x / rank_tiles, pt = rest % g.parts;
    int e, rows;
    int64_t p0;
    if (!mx4_find_tile(g.groups, rest / g.parts, 16 * NT, &e, &p0, &rows)) return;
    int64_t xat[NT], xcode[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int64_t row = mx4_row(g.groups, p0 + (16 * t + li < rows ? 16 * t + li : rows - 1));
        xat[t] = mx4_at(row, g.words);
        xcode[t] = mx4_code(row, g.words) * 16;
    }
    const uint16_t* lrow[TURNED ? 4 : 1];                    // ranks that are not there: the last one again, and what becomes of them is not kept
    f32x4_t acc[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < (TURNED ? 4 : 1); ++j) {             // turned: load j has four rows, a lane a sixteenth of one's word
        const int k = 16 * rt + (TURNED ? 4 * j + q : li);
        lrow[j] = g.lb + ((int64_t)e * g.r + (k < g.r ? k : g.r - 1)) * g.lb_ld;
    }
    char* const turn = (char*)part + wave * (16 * 256);
    const int first = pt * g.part_words, last = first + g.part_words < g.words ? first + g.part_words : g.words;
    v4i_t codes[U][NT];
    uint32_t scale[U][NT];
    uint4 a[U][4];
    auto load = [&](int u, int w) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const uint8_t* const code = g.xc + xcode[t] + (int64_t)w * 1024;
            if (TURNED) codes[u][t] = *(const v4i_t*)(code + 256 * q);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (!TURNED) codes[u][t][j] = *(const int*)(code + 256 * j + 4 * q);
            scale[u][t] = g.xs[xat[t] + (int64_t)w * kMxNext];
        }
        // behind the last channel the last ones are read again, against zeros of x
        const int64_t c0 = (int64_t)w * kMxWord + 8 * (TURNED ? li : q);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t at = c0 + (TURNED ? 0 : 32 * j), c = at < g.lb_ld ? at : g.lb_ld - 8;
            a[u][j] = *(const uint4*)(lrow[TURNED ? j : 0] + c);
        }
    };
    auto multiply = [&](int u) {
        if (TURNED) {                                        // the sixteenths of a row change places by the row: a quarter of the cycles of LDS are conflicts all the same
#pragma unroll
            for (int j = 0; j < 4; ++j) *(uint4*)(turn + (4 * j + q) * 256 + ((li ^ (4 * j + q)) << 4)) = a[u][j];
            mx4_lanes_meet();
#pragma unroll
            for (int j = 0; j < 4; ++j) a[u][j] = *(const uint4*)(turn + li * 256 + (((4 * q + j) ^ li) << 4));
            mx4_lanes_meet();
        }
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float by = __uint_as_float(((scale[u][t] >> (8 * (TURNED ? q : j))) & 255u) << 23);      // the conversion takes the exponent field for a scale byte
                const uint32_t w4 = (uint32_t)codes[u][t][j];
                const bf16x2_t v0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w4, by, 0), v1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w4, by, 1),
                               v2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w4, by, 2), v3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w4, by, 3);
                const bf16x8_t b = {v0[0], v0[1], v1[0], v1[1], v2[0], v2[1], v3[0], v3[1]};
                acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a[u][j]), b, acc[t], 0, 0, 0);
            }
    };
    const int count = first + wave < last ? (last - first - wave + W - 1) / W : 0;
    auto word = [&](int i) { return first + wave + W * i; };
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (u < count) load(u, word(u));
    for (int i = 0; i < count; i += U) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (i + u < count) multiply(u);
            if (i + u + U < count) load(u, word(i + u + U));
        }
    }
    f32x4_t* const mine = (f32x4_t*)part + lane;
    if (TURNED) __syncthreads();
#pragma unroll
    for (int t = 0; t < NT; ++t) mine[(wave * NT + t) * 64] = acc[t];
    __syncthreads();
    for (int i = wave; i < NT; i += W) {                     // ranks 4 q .. + 3 of token li
        f32x4_t sum = mine[i * 64];
#pragma unroll
        for (int w = 1; w < W; ++w) sum += mine[(w * NT + i) * 64];
        const int k = 16 * rt + 4 * q, at = 16 * i + li;
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (k + u >= g.r) sum[u] = 0.f;
        if (TERMS == 0) {
            if (at < rows) *(f32x4_t*)(g.P + ((int64_t)pt * g.groups.positions + p0 + at) * g.rp + k) = sum;
            continue;
        }
        const int64_t width = g.lr_steps / (TERMS ? TERMS : 1) * 32;
        const f32x4_t whole = sum;
        uint2 term[TERMS ? TERMS : 1];
#pragma unroll
        for (int u = 0; u < TERMS; ++u) {
            term[u] = make_uint2(bf16_pair(sum[0], sum[1]), bf16_pair(sum[2], sum[3]));
            sum -= f32x4_t{__uint_as_float(term[u].x << 16), __uint_as_float(term[u].x & 0xFFFF0000u), __uint_as_float(term[u].y << 16), __uint_as_float(term[u].y & 0xFFFF0000u)};
        }
        bool held = true;
#pragma unroll
        for (int u = 0; u < 4; ++u) held = held && fabsf(sum[u]) <= (TERMS == 3 ? 0.f : 0x1p-17f * fabsf(whole[u]));      // not so for infinities and NaN
        const uint64_t lost = __ballot(!held);
        if (at >= rows) continue;
        const bool mark = (lost >> li) & 0x0001000100010001u;        // by the token's 16 sums, so that the other tokens of the tile do not matter
        uint16_t* dst = g.planes + (p0 + at) * width + k;
#pragma unroll
        for (int u = 0; u < TERMS; ++u, dst += g.groups.positions * width) *(uint2*)dst = mark ? make_uint2(0u, 0u) : term[u];
        if (mark) *(f32x4_t*)(g.exact + (p0 + at) * width + k) = whole;
        if (q == 0) g.marks[(p0 + at) * 8 + rt] = mark;
    }
}

// The tokens of the positions in their order, so that tiles read them as they read any matrix: on their own, 16 bytes of a row here and there would take
// the address unit four times as long.  A workgroup has a part of a panel, its threads the rows' blocks and words of scales.
constexpr int kGatherWords = 8;
__global__ __launch_bounds__(256) void mx4_gather_kernel(MxGroups groups, const uint8_t* __restrict__ xc, const uint32_t* __restrict__ xs, int words, uint8_t* __restrict__ oc, uint32_t* __restrict__ os) {
    const int li = threadIdx.x & 15;
    const int64_t p = (int64_t)blockIdx.x * 16 + li, row = mx4_row(groups, p < groups.positions ? p : groups.positions - 1);
    const uint4* const from = (const uint4*)xc + mx4_code(row, words);
    uint4* const to = (uint4*)oc + (int64_t)blockIdx.x * words * 64 + li;
    const int first = blockIdx.y * kGatherWords, last = first + kGatherWords < words ? first + kGatherWords : words;
    for (int i = 4 * first + (threadIdx.x >> 4); i < 4 * last; i += 16) to[16 * i] = from[16 * i];
    const int w = first + (threadIdx.x >> 4);
    if (w < last) os[((int64_t)blockIdx.x * words + w) * 16 + li] = xs[mx4_at(row, words) + (int64_t)w * kMxNext];
}

// A factor with its rows of r padded with zeros, where it cannot be read in pieces of 16 bytes as it is (L_B), or not in pieces of 64 (L_A of many rows).
__global__ __launch_bounds__(256) void mx4_pad_kernel(const uint16_t* __restrict__ la, int64_t rows, int64_t r, int64_t width, uint16_t* __restrict__ out) {
    const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8, row = i / width;
    const int64_t k = i - row * width;
    if (row >= rows) return;
    uint32_t v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = k + u < r ? la[row * r + k + u] : 0u;
    *(uint4*)(out + i) = make_uint4(v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
}

// ---------------------------------------------------------------------------------------------------------------- few rows of a matrix
// A workgroup has 16 FA rows of the weights (gated: half of them gates, the others their values) and up to 16 NT positions; its W wavefronts take the words of
// the channels in turn, U of them ahead.  A fragment of a word, a panel's 16 rows, is a kilobyte of memory in the order of the lanes; a lane's 16 bytes are block
// lane / 16 of row lane % 16.  Outputs are in the rows of the accumulator, so a lane has four neighbouring ones of a position.  The sums of the wavefronts meet in LDS in a fixed
// order.
constexpr int kMostParts = 4;                                // of the channels, for P of few rows

template <int FA, int NT, int W, int U, bool GATED, bool F32>
__global__ __launch_bounds__(64 * W, FA * NT <= 2 ? 5 : FA * NT <= 4 ? 4 : FA * NT <= 8 ? 3 : 2) void mx4_few_kernel(MxArgs g) {
    extern __shared__ __align__(16) float part[];            // [wavefront][fragment][lane][4]
    constexpr int OF = GATED ? FA / 2 : FA;                  // fragments of outputs
    const int lane = threadIdx.x & 63, li = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int e, rows;
    int64_t p0;
    if (!mx4_find_tile(g.groups, blockIdx.y, 16 * NT, &e, &p0, &rows)) return;
    const int64_t o0 = (int64_t)blockIdx.x * (16 * OF);
    int64_t arow[FA], aat[FA], bat[NT], acode[FA], bcode[NT];
#pragma unroll
    for (int a = 0; a < FA; ++a) {
        const int64_t o = o0 + 16 * (a % OF) + li;           // past the end: the last one again, not stored
        arow[a] = (a >= OF ? g.outs : 0) + (o < g.outs ? o : g.outs - 1);
        aat[a] = e * g.w_size + mx4_at(arow[a], g.words);
        acode[a] = e * g.w_size * 64 + mx4_code(arow[a], g.words) * 16 + 256 * q;
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int64_t row = mx4_row(g.groups, p0 + (16 * t + li < rows ? 16 * t + li : rows - 1));
        bat[t] = mx4_at(row, g.words);
        bcode[t] = mx4_code(row, g.words) * 16 + 256 * q;
    }
    f32x4_t acc[FA][NT];
#pragma unroll
    for (int a = 0; a < FA; ++a)
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[a][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    v4i_t av[U][FA], bv[U][NT];
    uint32_t sa[U][FA], sb[U][NT];
    auto load = [&](int u, int w) {
#pragma unroll
        for (int a = 0; a < FA; ++a) {
            av[u][a] = *(const v4i_t*)(g.wc + acode[a] + (int64_t)w * 1024);
            sa[u][a] = g.ws[aat[a] + (int64_t)w * kMxNext];
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            bv[u][t] = *(const v4i_t*)(g.xc + bcode[t] + (int64_t)w * 1024);
            sb[u][t] = g.xs[bat[t] + (int64_t)w * kMxNext];
        }
    };
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (wave + u * W < g.words) load(u, wave + u * W);
    // the low-rank branch: 16 ranks at a time, each such chunk by one wavefront, four ranks an instruction, in fp32.  P's parts are summed into LDS; lane group q has
    // ranks 4 q .. + 3 of a chunk, of its four outputs' rows of L_A here and of P later
    uint32_t lv[FA][2];
    auto ranks_of = [&](int k0) {
        const uint16_t* const la = g.la + (int64_t)e * g.m * g.r;
        const int k = k0 + 4 * q;
#pragma unroll
        for (int a = 0; a < FA; ++a) {
            const uint16_t* const src = la + arow[a] * g.r + k;
            if (g.la_four) {
                const uint2 v = *(const uint2*)(k < g.r ? src : la);
                lv[a][0] = k < g.r ? v.x : 0u;
                lv[a][1] = k < g.r ? v.y : 0u;
                continue;
            }
            uint32_t h[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) h[i] = k + i < g.r ? src[i] : 0u;
            lv[a][0] = h[0] | h[1] << 16;
            lv[a][1] = h[2] | h[3] << 16;
        }
    };
    if (g.P) {
        if (16 * wave < g.rp) ranks_of(16 * wave);
        const int four = g.rp / 4;
        const int64_t next = g.groups.positions * g.rp;
        for (int i = threadIdx.x; i < 16 * NT * four; i += 64 * W) {
            const int at = i / four, k = 4 * (i - at * four);
            const float* src = g.P + (p0 + (at < rows ? at : rows - 1)) * g.rp + k;
            f32x4_t sum = *(const f32x4_t*)src;
            f32x4_t more[kMostParts - 1];
#pragma unroll
            for (int p = 1; p < kMostParts; ++p) more[p - 1] = p < g.parts ? *(const f32x4_t*)(src + p * next) : f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int p = 1; p < kMostParts; ++p) sum += more[p - 1];
            *(f32x4_t*)(part + at * (g.rp + 4) + k) = sum;
        }
    }
    for (int w = wave; w < g.words; w += U * W) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (w + u * W < g.words) {
#pragma unroll
                for (int a = 0; a < FA; ++a)
#pragma unroll
                    for (int t = 0; t < NT; ++t) acc[a][t] = mfma16(av[u][a], sa[u][a] >> (8 * q), bv[u][t], sb[u][t] >> (8 * q), acc[a][t]);
            }
            if (w + (u + U) * W < g.words) load(u, w + (u + U) * W);
        }
    }
    if (g.P) {
        __syncthreads();
        for (int k0 = 16 * wave; k0 < g.rp; k0 += 16 * W) {
            if (k0 >= 16 * W) ranks_of(k0);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const f32x4_t pv = *(const f32x4_t*)(part + (16 * t + li) * (g.rp + 4) + k0 + 4 * q);
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int a = 0; a < FA; ++a)
                        acc[a][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(i & 1 ? lv[a][i >> 1] & 0xFFFF0000u : lv[a][i >> 1] << 16), pv[i], acc[a][t], 0, 0, 0);
            }
        }
        __syncthreads();
    }
    f32x4_t* const mine = (f32x4_t*)part + lane;
#pragma unroll
    for (int a = 0; a < FA; ++a)
#pragma unroll
        for (int t = 0; t < NT; ++t) mine[((wave * FA + a) * NT + t) * 64] = acc[a][t];
    __syncthreads();
    for (int i = wave; i < OF * NT; i += W) {
        const int a = i / NT, t = i % NT;
        f32x4_t z = mine[(a * NT + t) * 64], up = f32x4_t{0.f, 0.f, 0.f, 0.f};
        if (GATED) up = mine[((a + OF) * NT + t) * 64];
#pragma unroll
        for (int w = 1; w < W; ++w) {
            z += mine[((w * FA + a) * NT + t) * 64];
            if (GATED) up += mine[((w * FA + a + OF) * NT + t) * 64];
        }
        float y[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) y[u] = GATED ? gated<F32>(z[u], up[u]) : z[u];
        const int at = 16 * t + li;
        if (at < rows) store4<F32>(g, p0 + at, o0 + 16 * a + 4 * q, y);
    }
}

// ---------------------------------------------------------------------------------------------------------------- many rows of a matrix
// A workgroup has 64 MF outputs of 64 NF positions, a wavefront (2 x 2 of them, one for each SIMD) 32 MF x 32 NF.  A step is a word of the channels: 64 bytes of
// codes and a word of scales of every row go straight from memory into LDS, a panel's kilobyte as it is, block by block, so that 16 lanes read 256 bytes in a row; a ring
// of ST stages, one barrier a step.  The loads are inline assembly because the compiler would
// make every LDS read wait for all of them.  Half h = lane / 32 of the lanes holds blocks h and 2 + h of a step, one for each of its two instructions
// per pair of fragments, whose scales are bytes 0 and 2 of its word shifted by h bytes.
// Gated, a wavefront's first MF / 2 fragments are gates and the others the values that belong to them.
// Workgroup b runs on XCD b % 8; an XCD's tiles are numbered matrix by matrix in panels of kPanel tiles of positions, so that its workgroups share few slabs of either operand
// and a matrix is read once where its positions make no more than a panel.
constexpr int kPanel = 4;

__device__ __forceinline__ int block_at(int r, int q) { return (r >> 4) * 1024 + q * 256 + (r & 15) * 16; }
__device__ __forceinline__ int chunk_at(int r, int c) { return r * 64 + ((c ^ ((r >> 2) & 3)) << 4); }

template <int B>
__device__ __forceinline__ f32x16_t mfma32(const v4i_t& a, uint32_t sa, const v4i_t& b, uint32_t sb, const f32x16_t& c) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wide(a), wide(b), c, 4, 4, B, (int)sa, B, (int)sb);
}

__device__ __forceinline__ f32x16_t mfma32_bf16(const v4i_t& a, const v4i_t& b, const f32x16_t& c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}

template <int MF, int NF, int ST, int WG, bool GATED, bool F32>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(WG, WG))) void mx4_tile_kernel(MxArgs g, uint32_t out_tiles) {
    extern __shared__ __align__(16) char smem[];
    constexpr int BM = 64 * MF, BN = 64 * NF;
    constexpr int A_BYTES = BM * 64, B_BYTES = BN * 64, SA = A_BYTES + B_BYTES, SB = SA + BM * 4, STAGE = SB + BN * 4;
    constexpr int LOADS = MF + NF + 2;                       // of a wavefront for a stage
    const int tid = threadIdx.x, lane = tid & 63, li = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wa = wave >> 1, wb = wave & 1;

    const uint64_t total = (uint64_t)mx4_tiles(g.groups, BN) * out_tiles, per_xcd = (total + 7) / 8;
    const uint64_t id = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
    if ((blockIdx.x >> 3) >= per_xcd || id >= total) return;
    int e, count;
    int64_t first_p;
    uint32_t in;
    if (!mx4_find(g.groups, id, BN, out_tiles, &e, &first_p, &count, &in)) return;
    const uint32_t tiles = (uint32_t)(count + BN - 1) / BN, panel = in / (kPanel * out_tiles), in_panel = in - panel * kPanel * out_tiles;
    const uint32_t high = tiles - panel * kPanel < kPanel ? tiles - panel * kPanel : kPanel, across = in_panel / high;
    const int before = (int)(panel * kPanel + in_panel - across * high) * BN, rows = count - before < BN ? count - before : BN;
    const int64_t p0 = first_p + before, o0 = (int64_t)across * (GATED ? BM / 2 : BM);
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
    auto token_row = [&](int r) { return p0 + (r < rows ? r : rows - 1); };      // many rows: in order

    // what this lane fetches: 16 rows an instruction, of row lane % 16 block lane / 16, and words of scales, 64 rows an instruction
    const char *ga[MF], *gb[NF], *gs[2];
#pragma unroll
    for (int t = 0; t < MF; ++t) ga[t] = (const char*)g.wc + e * g.w_size * 64 + mx4_code(weight_row(16 * (MF * wave + t) + (lane & 15)), g.words) * 16 + 256 * (lane >> 4);
#pragma unroll
    for (int t = 0; t < NF; ++t) gb[t] = (const char*)g.xc + mx4_code(token_row(16 * (NF * wave + t) + (lane & 15)), g.words) * 16 + 256 * (lane >> 4);
    gs[0] = (const char*)(g.ws + e * g.w_size + mx4_at(weight_row(64 * (wave % MF) + lane), g.words));
    gs[1] = (const char*)(g.xs + mx4_at(token_row(64 * (wave % NF) + lane), g.words));
    int64_t next_a = kMxNext * 64, next_b = kMxNext * 64, next_s = kMxNext * 4;      // bytes to the following stage
    const uint32_t ring = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
    // load number t of a stage, to the slot at byte `at` of the ring
    auto issue = [&](uint32_t at, int t) {
        const uint32_t slot = ring + at;
        if (t < MF) {
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" : : "s"(slot + (uint32_t)(MF * wave + t) * 1024), "v"(ga[t]) : "memory", "m0");
            ga[t] += next_a;
        } else if (t < MF + NF) {
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" : : "s"(slot + A_BYTES + (uint32_t)(NF * wave + t - MF) * 1024), "v"(gb[t - MF]) : "memory", "m0");
            gb[t - MF] += next_b;
        } else if (t == MF + NF) {
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" : : "s"(slot + SA + (uint32_t)(wave % MF) * 256), "v"(gs[0]) : "memory", "m0");
            gs[0] += next_s;
        } else {
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" : : "s"(slot + SB + (uint32_t)(wave % NF) * 256), "v"(gs[1]) : "memory", "m0");
            gs[1] += next_s;
        }
    };
    auto wait_for = [&](auto most) { asm volatile("s_waitcnt vmcnt(%0)" : : "n"(decltype(most)::value) : "memory"); };       // until at most so many loads are in flight

    int offa[MF], offb[NF];
#pragma unroll
    for (int i = 0; i < MF; ++i) offa[i] = block_at(wa * 32 * MF + 32 * i + li, h);
#pragma unroll
    for (int j = 0; j < NF; ++j) offb[j] = A_BYTES + block_at(wb * 32 * NF + 32 * j + li, h);
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
    // the operands of a step's first instructions and the words of scales, in the order in which they are wanted
    auto read0 = [&](const char* st, int t) {
        if (t < NF) b0[t] = *(const v4i_t*)(st + offb[t]);
        else if (t == NF) a0[0] = *(const v4i_t*)(st + offa[0]);
        else if (t < 2 * NF + 1) nb[t - NF - 1] = *(const uint32_t*)(st + offsb + 128 * (t - NF - 1));
        else if (t < 2 * NF + MF + 1) na[t - 2 * NF - 1] = *(const uint32_t*)(st + offsa + 128 * (t - 2 * NF - 1));
        else a0[t - 2 * NF - MF] = *(const v4i_t*)(st + offa[t - 2 * NF - MF]);
    };
    auto read1 = [&](const char* st, int t, bool ranks) {    // the second's: two blocks on, or the neighbouring pair of chunks
        if (t < NF) b1[t] = *(const v4i_t*)(st + (ranks ? offb[t] ^ 32 : offb[t] + 512));
        else a1[t - NF] = *(const v4i_t*)(st + (ranks ? offa[t - NF] ^ 32 : offa[t - NF] + 512));
    };
    auto read_ranks = [&]() {                                // from here on stages of ranks are read
#pragma unroll
        for (int i = 0; i < MF; ++i) offa[i] = chunk_at(wa * 32 * MF + 32 * i + li, h);
#pragma unroll
        for (int j = 0; j < NF; ++j) offb[j] = A_BYTES + chunk_at(wb * 32 * NF + 32 * j + li, h);
    };
    // Behind the words of the channels come the steps of the low-rank branch, 32 ranks of L_A and of one term of P each: 64 bytes a row as well.
    constexpr int TERMS = F32 ? 3 : 2;
    const int words = g.words, steps = words + g.lr_steps;
    auto turn_to_ranks = [&]() {
        const int ch = (lane & 3) ^ ((lane >> 4) & 3);       // of row lane / 4 the chunk that goes to place lane % 4
        const int64_t width = 64 * (int64_t)(g.lr_steps / TERMS);        // bytes of a row of P
#pragma unroll
        for (int t = 0; t < MF; ++t) ga[t] = (const char*)g.la + ((int64_t)e * g.m + weight_row(16 * (MF * wave + t) + (lane >> 2))) * g.la_ld * 2 + 16 * ch;
#pragma unroll
        for (int t = 0; t < NF; ++t) {
            const int r = 16 * (NF * wave + t) + (lane >> 2);
            gb[t] = (const char*)g.planes + (p0 + (r < rows ? r : rows - 1)) * width + 16 * ch;
        }
        gs[0] -= next_s;                                     // scales are not looked at: the last word's again
        gs[1] -= next_s;
        next_s = 0;
    };
    // before the loads of stage s
    auto aim = [&](int s) {
        if (s < words) return;
        if (s == words) turn_to_ranks();
        const int term = (s - words) % TERMS;
        const int64_t plane = g.groups.positions * 64 * (int64_t)(g.lr_steps / TERMS);
        next_a = term == TERMS - 1 ? 64 : 0;
        next_b = term == TERMS - 1 ? 64 - (TERMS - 1) * plane : plane;
    };
    // Of a stage's loads the first EARLY are issued in the second half of a step, the others in the first half of the next: all at once they would wait for each other.
    // Three slots only leave no time for that.
    constexpr int EARLY = ST == 4 ? LOADS / 2 : LOADS;
    for (int s = 0; s < ST - 1 && s < steps; ++s) {
        aim(s);
#pragma unroll
        for (int t = 0; t < LOADS; ++t)
            if (s < ST - 2 || t < EARLY) issue((uint32_t)s * STAGE, t);
    }
    if (steps >= ST - 1) wait_for(std::integral_constant<int, (ST - 3) * LOADS + EARLY>{});
    else if (ST == 4 && steps == 2) wait_for(std::integral_constant<int, LOADS>{});
    else wait_for(std::integral_constant<int, 0>{});
    __syncthreads();
#pragma unroll
    for (int t = 0; t < 2 * (MF + NF); ++t) read0(smem, t);
    constexpr int M = MF * NF;                               // instructions of a half step
    constexpr int R0 = 2 * (MF + NF), R1 = MF + NF;
    constexpr int W = M > 4 ? 1 : 0;                         // the barrier's place in the second half
    uint32_t cur = 0;                                        // the step's slot
    auto step = [&](int s, auto steady_tag, auto ranks_tag) {
        constexpr bool STEADY = decltype(steady_tag)::value, RANKS = decltype(ranks_tag)::value;
        const uint32_t next = cur + STAGE == ST * STAGE ? 0 : cur + STAGE, put = cur == 0 ? (ST - 1) * STAGE : cur - STAGE;
        const char *st = smem + cur, *sn = smem + next;
        const bool more = STEADY || s + 1 < steps, fetch = STEADY || s + ST - 1 < steps;
        const bool rest = EARLY < LOADS && (STEADY || s + ST - 2 < steps);
        const uint32_t late = put == 0 ? (ST - 1) * STAGE : put - STAGE;      // the slot of the stage before
#pragma unroll
        for (int i = 0; i < MF; ++i) sa[i] = na[i] >> (8 * h);
#pragma unroll
        for (int j = 0; j < NF; ++j) sb[j] = nb[j] >> (8 * h);
        // first half: the operands of the second are read under its first instructions
#pragma unroll
        for (int k = 0; k < M; ++k) {
            const int i = k / NF, j = k % NF;
            acc[i][j] = RANKS ? mfma32_bf16(a0[i], b0[j], acc[i][j]) : mfma32<0>(a0[i], sa[i], b0[j], sb[j], acc[i][j]);
#pragma unroll
            for (int t = 0; t < R1; ++t)
                if (t * (M - 1) / R1 == k) read1(st, t, RANKS);
#pragma unroll
            for (int t = EARLY; t < LOADS; ++t)
                if (rest && (t - EARLY) * M / (LOADS - EARLY) == k) issue(late, t);
            __builtin_amdgcn_sched_barrier(0);
        }
        // second half: the wait for the next stage, the reads of its first half, loads of the last stage that has a slot
#pragma unroll
        for (int k = 0; k < M; ++k) {
            const int i = k / NF, j = k % NF;
            acc[i][j] = RANKS ? mfma32_bf16(a1[i], b1[j], acc[i][j]) : mfma32<2>(a1[i], sa[i], b1[j], sb[j], acc[i][j]);
            if (k == W && more) {
                if (ST == 4 && (STEADY || s + 2 < steps)) wait_for(std::integral_constant<int, LOADS>{});
                else wait_for(std::integral_constant<int, 0>{});
                __syncthreads();                             // everyone's share has landed, and everyone is done with stage s - 1
                if (!STEADY && fetch) aim(s + ST - 1);
                if (!STEADY && s + 1 == words) read_ranks();
            }
#pragma unroll
            for (int t = 0; t < R0; ++t)
                if (more && W + 1 + t * (M - W - 1) / R0 == k) read0(sn, t);
#pragma unroll
            for (int t = 0; t < EARLY; ++t)
                if (fetch && W + 1 + t * (M - W - 1) / EARLY == k) issue(put, t);
            __builtin_amdgcn_sched_barrier(0);
        }
        cur = next;
    };
    int s = 0;
    for (; s + ST - 1 < words; ++s) step(s, std::true_type{}, std::false_type{});
    for (; s < words; ++s) step(s, std::false_type{}, std::false_type{});
    if (g.lr_steps) {
        // sums of P that terms do not hold: the marks of this lane's positions, looked at when the steps of ranks are through
        uint64_t marked[NF], some = 0;
#pragma unroll
        for (int j = 0; j < NF; ++j) marked[j] = ((const uint64_t*)g.marks)[token_row(wb * 32 * NF + 32 * j + li)];
        for (; s < steps; ++s) step(s, std::false_type{}, std::true_type{});
#pragma unroll
        for (int j = 0; j < NF; ++j) {
            marked[j] = wb * 32 * NF + 32 * j + li < rows ? marked[j] & (~(uint64_t)0 >> (64 - 16 * (g.lr_steps / TERMS))) : 0;      // the bytes that were written
            some |= marked[j];
        }
        if (__ballot(some != 0)) {
            // rare: these by the fp32 instruction, half h of the lanes the second of two ranks; other positions get zeros.  A whole call of such rows takes twice as long (4099 x 4096 x
            // 14336, rank 64: 189 us to 352); the look whether there are any 0.2 % where the marks are on their way during the steps of ranks (loaded behind them 2 %)
            const int64_t width = 32 * (int64_t)(g.lr_steps / TERMS);
#pragma unroll 1
            for (int k0 = 0; k0 < g.r; k0 += 2) {
                const int k = k0 + h;
                float a[MF], b[NF];
                bool has = false;
#pragma unroll
                for (int j = 0; j < NF; ++j) {
                    const bool mine = k < g.r && (marked[j] >> (8 * (k >> 4)) & 1);
                    b[j] = mine ? g.exact[(p0 + wb * 32 * NF + 32 * j + li) * width + k] : 0.f;
                    has = has || mine;
                }
                if (!__ballot(has)) continue;
#pragma unroll
                for (int i = 0; i < MF; ++i) {
                    const uint16_t* const row = g.la + ((int64_t)e * g.m + weight_row(wa * 32 * MF + 32 * i + li)) * g.la_ld;
                    a[i] = k < g.r ? __uint_as_float((uint32_t)row[k] << 16) : 0.f;
                }
#pragma unroll
                for (int i = 0; i < MF; ++i)
#pragma unroll
                    for (int j = 0; j < NF; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], b[j], acc[i][j], 0, 0, 0);
            }
        }
    }

    // acc[i][j][k]: output 32 i + 8 (k / 4) + 4 h + k % 4, position 32 j + li of the wavefront's.  They are turned through the wavefront's part of the ring, as many
    // positions at a time as it holds, so that rows of Y are written in whole lines; the 16-byte chunks of a row change places by the row, which keeps most of the
    // writes and reads off each other's banks (of all cycles of LDS 3 to 13 % are conflicts).
    constexpr int OF = GATED ? MF / 2 : MF;                  // fragments of outputs
    constexpr int SIZE = F32 ? 4 : 2, ROW = OF * 32 * SIZE, CHUNKS = ROW / 16;
    constexpr int FIT = ST * STAGE / 4 / (32 * ROW), BATCH = FIT >= NF ? NF : FIT >= 2 && NF % 2 == 0 ? 2 : 1;
    static_assert(FIT >= 1, "the ring has to hold 32 positions of every wavefront");
    auto chunk_of = [](int r, int c) { return c ^ (CHUNKS >= 16 ? r & 15 : r / (16 / (CHUNKS < 16 ? CHUNKS : 16)) & (CHUNKS - 1)); };
    const int64_t ow = o0 + wa * 32 * OF;
    __syncthreads();
    char* const mine = smem + wave * (BATCH * 32 * ROW);
#pragma unroll
    for (int j0 = 0; j0 < NF; j0 += BATCH) {
#pragma unroll
        for (int jj = 0; jj < BATCH; ++jj) {
            const int j = j0 + jj;
            char* const row = mine + (32 * jj + li) * ROW;
#pragma unroll
            for (int i = 0; i < OF; ++i)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    float y[4];
#pragma unroll
                    for (int u = 0; u < 4; ++u) y[u] = GATED ? gated<F32>(acc[i][j][4 * k + u], acc[MF - OF + i][j][4 * k + u]) : acc[i][j][4 * k + u];
                    const int o = 32 * i + 8 * k + 4 * h;
                    if (F32) *(float4*)(row + 16 * chunk_of(li, o / 4)) = make_float4(y[0], y[1], y[2], y[3]);
                    else *(uint2*)(row + 16 * chunk_of(li, o / 8) + 8 * h) = make_uint2(bf16_pair(y[0], y[1]), bf16_pair(y[2], y[3]));
                }
        }
        mx4_lanes_meet();
        constexpr int EACH = 16 / SIZE, ROWS = 64 / CHUNKS;  // outputs of a lane, rows an instruction
        const int c = lane % CHUNKS, o = c * EACH, r0 = lane / CHUNKS, base = wb * 32 * NF + 32 * j0;
        char* dst = (char*)g.Y + ((p0 + base + r0) * g.ldy + ow + o) * SIZE;
        const int64_t next = ROWS * g.ldy * SIZE;
        if (g.vec && base + 32 * BATCH <= rows && ow + 32 * OF <= g.outs) {
#pragma unroll
            for (int t = 0; t < 32 * BATCH; t += ROWS, dst += next) *(uint4*)dst = *(const uint4*)(mine + (t + r0) * ROW + 16 * chunk_of((t + r0) & 31, c));
        } else {                                             // the last positions or outputs, or rows of Y that 16 bytes do not fit
#pragma nounroll
            for (int t = r0; t < 32 * BATCH && base + t < rows; t += ROWS, dst += next) {
                const uint4 v = *(const uint4*)(mine + t * ROW + 16 * chunk_of(t & 31, c));
                if (g.vec && ow + o + EACH <= g.outs) {
                    *(uint4*)dst = v;
                    continue;
                }
                const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int u = 0; u < EACH; ++u) {
                    if (ow + o + u >= g.outs) continue;
                    if (F32) ((uint32_t*)dst)[u] = w[u % 4];
                    else ((uint16_t*)dst)[u] = (uint16_t)(w[(u / 2) % 4] >> (16 * (u & 1)));
                }
            }
        }
        mx4_lanes_meet();
    }
}

template <int FA, int NT, int W, int U, bool GATED>
int launch_few_one(aser_ctx* ctx, const MxArgs& g, bool f32) {
    size_t lds = (size_t)W * FA * NT * 1024;                 // the sums of the wavefronts; before them P, if there is one
    const size_t ranks = g.P ? (size_t)16 * NT * (g.rp + 4) * 4 : 0;
    if (lds < ranks) lds = ranks;
    const int64_t tiles = g.groups.most_tiles(16 * NT);
    if (tiles > 65535) ASER_FAIL(ctx, ASER_ERR_SHAPE, "mx4: too many rows");
    const dim3 grid((unsigned)ceil_div64(g.outs, 16 * (GATED ? FA / 2 : FA)), (unsigned)tiles);
    const auto kernel = f32 ? mx4_few_kernel<FA, NT, W, U, GATED, true> : mx4_few_kernel<FA, NT, W, U, GATED, false>;
    if (lds > 65536) ASER_HIP(ctx, hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
    kernel<<<grid, 64 * W, lds, ctx->stream>>>(g);
    return aser_check_launch(ctx, "mx4_few_kernel");
}
template <int FA, int NT, int W, int U>
int launch_few(aser_ctx* ctx, const MxArgs& g, bool gated, bool f32) {
    return gated ? launch_few_one<FA, NT, W, U, true>(ctx, g, f32) : launch_few_one<FA, NT, W, U, false>(ctx, g, f32);
}

template <int MF, int NF, int ST, int WG, bool GATED, bool F32>
int launch_tile_one(aser_ctx* ctx, const MxArgs& g) {
    constexpr int kLds = ST * (64 * MF + 64 * NF) * 68;
    static_assert(kLds * WG <= 160 * 1024, "the rings have to fit the LDS of a compute unit");
    const auto kernel = mx4_tile_kernel<MF, NF, ST, WG, GATED, F32>;
    ASER_HIP(ctx, hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, kLds));
    const int64_t out_tiles = ceil_div64(g.outs, GATED ? 32 * MF : 64 * MF), grid = ceil_div64(g.groups.most_tiles(64 * NF) * out_tiles, 8) * 8;
    if (!mx4_fits(grid, 256)) ASER_FAIL(ctx, ASER_ERR_SHAPE, "mx4: too many rows times outputs");
    kernel<<<(unsigned)grid, 256, kLds, ctx->stream>>>(g, (uint32_t)out_tiles);
    return aser_check_launch(ctx, "mx4_tile_kernel");
}
template <int MF, int NF, int ST, int WG>
int launch_tile(aser_ctx* ctx, const MxArgs& g, bool gated, bool f32) {
    if (gated) return f32 ? launch_tile_one<MF, NF, ST, WG, true, true>(ctx, g) : launch_tile_one<MF, NF, ST, WG, true, false>(ctx, g);
    return f32 ? launch_tile_one<MF, NF, ST, WG, false, true>(ctx, g) : launch_tile_one<MF, NF, ST, WG, false, false>(ctx, g);
}

// Rows of the weights and of x of a workgroup, its wavefronts and words ahead, by how many workgroups there are: `tiles` of 16 nt rows, and 32 weight rows each.  Many of them fill
// the device by themselves and read x less often with 64 weight rows; few of them have to have more in flight.  Weights not in any cache, us (the other side):
//   one row or up to 16: <2, 1, 4, 3>, three words ahead and five wavefronts a SIMD, 1 x 4096 x 14336 twice, gated, rank 32 (1792 workgroups) 30.0, 48 rows on 64 experts,
//   1408 x 2048, with the weighted sum (4096) 33.6; four words ahead and four wavefronts 30.2, 36.7; <2, 1, 8, 2> and <4, 1, 4, 2> 1.7 to 7 more than these; one row, 14336 x 4096
//   (128) <1, 1, 8, 4> 9.4 (<2, 1, 8, 2> 9.6, <2, 1, 4, 4> 11.3)
//   24 rows, 4096 x 14336 (448) <2, 2, ..> 8.4 (<4, 2, ..> 9.2); 256 rows on 64 experts, 2048 x 2816 (5632) <4, 2, ..> 58 (77)
//   64 rows, 4096 x 14336 (448) <4, 4, ..> 14.4 (<2, 4, ..> 15.7); 128 rows, 4096 x 4096 (256) <2, 4, ..> 8.6 (9.5)
int run_few(aser_ctx* ctx, const MxArgs& g, int nt, int64_t matrices, bool gated, bool f32) {
    const int64_t tiles = ceil_div64(g.groups.positions, 16 * nt), workgroups = (matrices > tiles ? matrices : tiles) * ceil_div64(g.m, 32);
    if (nt == 1) {
        if (workgroups >= 512) return launch_few<2, 1, 4, 3>(ctx, g, gated, f32);
        return gated ? launch_few_one<2, 1, 8, 2, true>(ctx, g, f32) : launch_few_one<1, 1, 8, 4, false>(ctx, g, f32);
    }
    if (nt == 2) return workgroups >= 2048 ? launch_few<4, 2, 4, 2>(ctx, g, gated, f32) : launch_few<2, 2, 4, 2>(ctx, g, gated, f32);
    if (nt == 3) return workgroups >= 2048 ? launch_few<4, 3, 4, 2>(ctx, g, gated, f32) : launch_few<2, 3, 4, 2>(ctx, g, gated, f32);
    return workgroups >= 400 ? launch_few<4, 4, 4, 2>(ctx, g, gated, f32) : launch_few<2, 4, 4, 2>(ctx, g, gated, f32);
}

// Tiles of 128 x 128 where there are not enough larger ones.  Rows x channels x outputs, us: 2048 x 4096 x 4096 (256 of 256 x 128) 25.6, larger 29.8; 512 x 4096 x 14336 (224) 25.0, 31.2;
// 1024 x 4096 x 14336 (448) 47.6, 43.5.  128 x 64 is faster only where the kernel for few rows is faster still.
// 256 outputs x 256 positions, one workgroup a compute unit, move less for each product than 256 x 128, two of them, whose beginnings and ends cover each other: a word of the channels takes a
// round of 256 of them 0.88 us, beside 8.5 at its ends, and a round of 512 of the others 1.05 and 6 (4096 rows and 16384 outputs of 1024 to 8192 channels: 60.5 to 256 us against
// 55.9 to 286).  Which takes fewer such rounds' time decides: 4099 x 4096 x 14336 149 against 160, 1501 rows on 8 experts (375 each) 326 against 301.
int run_many(aser_ctx* ctx, const MxArgs& g, bool gated, bool f32) {
    const int64_t across = ceil_div64(g.m, 256), tiles = g.groups.most_tiles(128) * across;
    if (tiles < 384) return launch_tile<2, 2, 4, 2>(ctx, g, gated, f32);
    const int steps = g.words + g.lr_steps;
    const double large = (double)ceil_div64(g.groups.most_tiles(256) * across, 256) * (0.88 * steps + 8.5), small = (double)ceil_div64(tiles, 512) * (1.05 * steps + 6.0);
    return large < small ? launch_tile<4, 4, 3, 1>(ctx, g, gated, f32) : launch_tile<4, 2, 3, 2>(ctx, g, gated, f32);
}

struct Plan {
    int nt;                  // 16 nt positions a workgroup
    bool many;               // tiles through LDS instead
    int parts, part_words;   // few rows: of the channels, for P
    size_t x_bytes;                          // many rows of experts: their codes and scales in order
    size_t p_bytes, la_bytes, lb_bytes;      // P, and the factors should they have to be padded
    size_t all() const { return x_bytes + p_bytes + la_bytes + lb_bytes; }
};

Plan plan_product(int64_t positions, int64_t n, int64_t m, int32_t count, int32_t r, bool experts) {
    Plan p{};
    const int64_t each = ceil_div64(positions, count < positions ? count : positions);
    p.nt = (int)(each <= 64 ? ceil_div64(each, 16) : 4);
    // Tiles begin to pay where 64 rows by 64 outputs, which is what the other kernel takes at a time, make more workgroups than the device holds at once.  us, tiles (the other
    // kernel): 128 x 4096 x 14336 15.3 (14.1), 192: 17.3 (19.2); 512 x 4096 x 4096 12.9 (12.2), 1024: 16.6 (20.9); 256 x 14336 x 4096 40 (22)
    p.many = each > 64 && ceil_div64(positions, 64) * ceil_div64(m, 64) > 512;
    const int64_t words = mx4_words(n), tiles = ceil_div64(positions, 16);
    int64_t parts = p.many || tiles >= 256 ? 1 : ceil_div64(256, tiles);
    if (parts > ceil_div64(words, 8)) parts = ceil_div64(words, 8);
    if (parts > kMostParts) parts = kMostParts;
    p.part_words = (int)ceil_div64(words, parts);
    p.parts = (int)ceil_div64(words, p.part_words);
    if (p.many && experts) p.x_bytes = align_up((size_t)mx4_size(positions, words) * 68, 256);
    if (r <= 0) return p;
    p.lb_bytes = align_up((size_t)count * r * align_up(n, 8) * 2, 256);
    // Few rows, P: parts x positions, but what any fewer positions need as well, so that who asks for the largest batch has room for all: parts are at most 256 / tiles rounded up,
    // (255 + tiles) / tiles, of tiles of 16 positions
    const int64_t most_parts = words > 8 * kMostParts ? kMostParts : ceil_div64(words, 8);
    const int64_t sums = most_parts * positions < positions + 255 * 16 ? most_parts * positions : positions + 255 * 16;
    p.p_bytes = align_up((size_t)sums * align_up(r, 16) * 4, 256);
    if (p.many) {
        const size_t bytes = align_up((size_t)positions * align_up(r, 32) * (3 * 2 + 4) + (size_t)positions * 8, 256);      // terms, sums, marks
        if (p.p_bytes < bytes) p.p_bytes = bytes;
        p.la_bytes = align_up((size_t)count * m * align_up(r, 32) * 2, 256);
    }
    return p;
}

int pad_rows(aser_ctx* ctx, const uint16_t* f, int64_t rows, int64_t r, int64_t width, uint16_t* out) {
    const int64_t grid = ceil_div64(rows * width, 2048);
    if (!mx4_fits(grid, 256)) ASER_FAIL(ctx, ASER_ERR_SHAPE, "mx4: the factors are too large");
    mx4_pad_kernel<<<(unsigned)grid, 256, 0, ctx->stream>>>(f, rows, r, width, out);
    return aser_check_launch(ctx, "mx4_pad_kernel");
}

template <int NT, int W, int U, int TERMS>
int launch_down(aser_ctx* ctx, const MxArgs& g) {
    const int rank_tiles = (int)ceil_div64(TERMS ? g.lr_steps / (TERMS ? TERMS : 1) * 32 : g.rp, 16);
    const int64_t grid = g.groups.most_tiles(16 * NT) * g.parts * rank_tiles;
    if (!mx4_fits(grid, 64 * W)) ASER_FAIL(ctx, ASER_ERR_SHAPE, "mx4: too many rows");
    mx4_down_kernel<NT, W, U, TERMS><<<(unsigned)grid, 64 * W, (size_t)W * 1024 * (TERMS && NT < 4 ? 4 : NT), ctx->stream>>>(g, rank_tiles);
    return aser_check_launch(ctx, "mx4_down_kernel");
}

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
    const Plan p = plan_product(groups.positions, w->n, w->rows, w->count, r, groups.offsets != nullptr);
    if (r > 0 && p.many && !mx4_fits(groups.most_tiles(32) * (align_up(r, 32) / 16), 256)) ASER_FAIL(ctx, ASER_ERR_SHAPE, "%s: too many rows for this rank", who);
    if (p.all() > 0 && (!ctx->ws || ctx->ws_bytes < p.all() + kAserWsTail)) ASER_FAIL(ctx, ASER_ERR_WORKSPACE, "%s: workspace too small", who);
    MxArgs g{};
    g.groups = groups;
    g.words = (int)mx4_words(w->n);
    g.xc = x->codes; g.xs = (const uint32_t*)x->scales;
    g.wc = w->codes; g.ws = (const uint32_t*)w->scales; g.m = w->rows; g.w_size = mx4_size(w->rows, g.words);
    g.la = L_A; g.lb = L_B; g.r = r; g.la_ld = r; g.lb_ld = w->n;
    g.parts = p.parts; g.part_words = p.part_words; g.rp = (int)align_up(r, 16);
    g.Y = Y; g.ldy = ldy; g.outs = outs;
    const int64_t unit = p.many || f32 ? 16 : 8, size = f32 ? 4 : 2;
    g.vec = !((uintptr_t)Y & (unit - 1)) && !(ldy * size & (unit - 1));
    g.la_four = !((uintptr_t)L_A & 7) && !(r & 3);
    ASER_TRY(aser_prepare_device(ctx));
    char* const p_room = (char*)ctx->ws + p.x_bytes;
    if (r > 0 && (((uintptr_t)L_B & 15) || (w->n & 7))) {
        uint16_t* const padded = (uint16_t*)(p_room + p.p_bytes + p.la_bytes);
        g.lb_ld = align_up(w->n, 8);
        ASER_TRY(pad_rows(ctx, L_B, (int64_t)w->count * r, w->n, g.lb_ld, padded));
        g.lb = padded;
    }
    if (!p.many) {
        if (r > 0) {
            g.P = (float*)p_room;
            ASER_TRY((launch_down<1, 4, 2, 0>(ctx, g)));
        }
        return run_few(ctx, g, p.nt, w->count < groups.positions ? w->count : groups.positions, swiglu, f32);
    }
    if (groups.order) {
        uint8_t* const codes = (uint8_t*)ctx->ws;
        uint32_t* const scales = (uint32_t*)(codes + mx4_size(groups.positions, g.words) * 64);
        mx4_gather_kernel<<<dim3((unsigned)ceil_div64(groups.positions, 16), (unsigned)ceil_div64(g.words, kGatherWords)), 256, 0, ctx->stream>>>(groups, g.xc, g.xs, g.words, codes, scales);
        ASER_TRY(aser_check_launch(ctx, "mx4_gather_kernel"));
        g.xc = codes;
        g.xs = scales;
        g.groups.order = nullptr;
    }
    if (r > 0) {
        const int terms = f32 ? 3 : 2, width = (int)align_up(r, 32);
        g.planes = (uint16_t*)p_room;
        g.lr_steps = width / 32 * terms;
        g.exact = (float*)(g.planes + groups.positions * width * 3);
        g.marks = (uint8_t*)(g.exact + groups.positions * width);
        ASER_TRY(f32 ? (launch_down<2, 4, 2, 3>(ctx, g)) : (launch_down<2, 4, 2, 2>(ctx, g)));
        if (r != width || ((uintptr_t)L_A & 15)) {
            uint16_t* const padded = (uint16_t*)(p_room + p.p_bytes);
            ASER_TRY(pad_rows(ctx, L_A, w->rows * w->count, r, width, padded));
            g.la = padded;
            g.la_ld = width;
        }
    }
    return run_many(ctx, g, swiglu, f32);
}

}  // namespace

extern "C" size_t aser_mx4_forward_workspace_bytes(int64_t rows, int64_t n, int64_t m, int32_t r) {
    if (rows <= 0 || n <= 0 || m <= 0) return kAserWsTail;
    return plan_product(rows, n, m, 1, r, false).all() + kAserWsTail;
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
    return plan_product(positions, n, m, n_experts, r, true).all() + kAserWsTail;
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
