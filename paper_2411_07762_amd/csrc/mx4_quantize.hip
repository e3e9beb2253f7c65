// Rows of weights or activations to microscaled 4 bits: per block of 32 channels the power of two 2^e, e = floor(log2 max|u|) - 2, that takes the block's
// largest magnitude to [4, 8), and the nearest of the magnitudes 0, 0.5, 1, 1.5, 2, 3, 4, 6 to each u / 2^e.
//
// The maximum is taken of the bit patterns without sign, which orders magnitudes with infinities and NaN on top, and its exponent field less 2 is the
// scale byte: no logarithm.  u is scaled by a product with a power of two (exact: what leaves the range of fp32 below rounds to 0 anyway), rounded and packed two at a
// time by the conversion instruction.
// A group of 16 lanes has a scale word of a row, 128 channels, a lane 8 of them: 16 bytes of bf16 or twice 16 of fp32.  A workgroup has a panel's 16 rows, the
// next one the next word of them.  Bound by memory, with a division for each value by the instructions as well: 4096 x 11008 fp32 with their values written back 89 us (4.3 TB/s; panel
// after panel for a word before the next word: 101), 4099 x 4096 bf16 11 us, divided 16.  Two to eight words a thread, their loads together, changed nothing.
#include "bf16_pair.h"
#include "mx4.h"

namespace {

typedef float pair_t __attribute__((ext_vector_type(2)));

struct QuantArgs {
    const void* X; int64_t ldx;
    const float* m;
    uint8_t* codes; uint32_t* scales;
    void* values; int64_t ldv;
    int64_t rows, all_rows, n, words;        // rows of a matrix, of all of them
    bool vec;                                // rows of X and of values on 16-byte boundaries, m too
};

template <bool F32>
__device__ __forceinline__ void load8(const void* X, int64_t at, float* u) {
    if (F32) {
        const float4 a = *(const float4*)((const float*)X + at), b = *(const float4*)((const float*)X + at + 4);
        u[0] = a.x; u[1] = a.y; u[2] = a.z; u[3] = a.w; u[4] = b.x; u[5] = b.y; u[6] = b.z; u[7] = b.w;
    } else {
        const uint4 a = *(const uint4*)((const uint16_t*)X + at);
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            u[2 * i] = __uint_as_float(w[i] << 16);
            u[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
}

template <bool F32>
__device__ __forceinline__ float load1(const void* X, int64_t at) {
    return F32 ? ((const float*)X)[at] : __uint_as_float((uint32_t)((const uint16_t*)X)[at] << 16);
}

template <bool F32, bool M, bool VALUES>
__global__ __launch_bounds__(256) void mx4_quantize_kernel(QuantArgs g) {
    const uint32_t words = (uint32_t)g.words, id = blockIdx.y * (uint32_t)kMxAcross + blockIdx.x, tile = id / words, word = id - tile * words, row = tile * 16 + (threadIdx.x >> 4);
    if (row >= (uint32_t)g.all_rows) return;                 // the same for all lanes of a group
    const int li = threadIdx.x & 15;
    const int64_t c = (int64_t)word * kMxWord + 8 * li;
    const int here = (int)(c + 8 <= g.n ? 8 : c < g.n ? g.n - c : 0);
    float u[8];
    if (g.vec && here == 8) {
        load8<F32>(g.X, row * g.ldx + c, u);
        if (M) {
            float d[8];
            load8<true>(g.m, c, d);
#pragma unroll
            for (int i = 0; i < 8; ++i) u[i] = u[i] / d[i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            u[i] = i < here ? load1<F32>(g.X, row * g.ldx + c + i) : 0.f;
            if (M && i < here) u[i] = u[i] / g.m[c + i];
        }
    }
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t b = __float_as_uint(u[i]) & 0x7FFFFFFFu;
        top = b > top ? b : top;
    }
#pragma unroll
    for (int k = 1; k < 4; k *= 2) {
        const uint32_t v = __shfl_xor(top, k);
        top = v > top ? v : top;
    }
    const uint32_t expo = top >> 23;
    const bool bad = expo == 255;
    const uint32_t byte = bad ? 255u : expo > 2 ? expo - 2 : 0u;
    const float by = bad ? 0.f : __uint_as_float((254u - byte) << 23);       // 2^(127 - byte), 2^-125 to 2^127
    uint32_t codes = 0;
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, u[0] * by, u[1] * by, 1.f, 0);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, u[2] * by, u[3] * by, 1.f, 1);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, u[4] * by, u[5] * by, 1.f, 2);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, u[6] * by, u[7] * by, 1.f, 3);
    if (bad) codes = 0;
    uint32_t all = byte << (8 * (li >> 2));
    all |= __shfl_xor(all, 4);
    all |= __shfl_xor(all, 8);
    const uint32_t e = row / (uint32_t)g.rows;
    const int64_t in = row - e * (uint32_t)g.rows, matrix = e * mx4_size(g.rows, g.words);
    ((uint32_t*)g.codes)[(matrix * 4 + mx4_code(in, g.words) + word * 64 + 16 * (li >> 2)) * 4 + (li & 3)] = codes;
    if (li == 0) g.scales[matrix + mx4_at(in, g.words) + word * kMxNext] = all;
    if (!VALUES || here == 0) return;
    const pair_t v2[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.f, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.f, 1),
                          __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.f, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.f, 3)};
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = bad ? __uint_as_float(0x7FC00000u) : __builtin_ldexpf(v2[i >> 1][i & 1], (int)byte - 127);
    const int64_t at = row * g.ldv + c;
    if (g.vec && here == 8) {
        if (F32) {
            *(float4*)((float*)g.values + at) = make_float4(v[0], v[1], v[2], v[3]);
            *(float4*)((float*)g.values + at + 4) = make_float4(v[4], v[5], v[6], v[7]);
        } else {                                             // four bits are exact in bf16, also below its normal range
            *(uint4*)((uint16_t*)g.values + at) = make_uint4(upper_halves(v[0], v[1]), upper_halves(v[2], v[3]), upper_halves(v[4], v[5]), upper_halves(v[6], v[7]));
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (i >= here) continue;
        if (F32) ((float*)g.values)[at + i] = v[i];
        else ((uint16_t*)g.values)[at + i] = (uint16_t)(__float_as_uint(v[i]) >> 16);
    }
}

template <bool F32, bool M>
void launch(const QuantArgs& g, hipStream_t s) {
    const int64_t workgroups = ceil_div64(g.all_rows, 16) * g.words;        // below 2^31
    const dim3 grid((unsigned)(workgroups < kMxAcross ? workgroups : kMxAcross), (unsigned)ceil_div64(workgroups, kMxAcross));
    if (g.values) mx4_quantize_kernel<F32, M, true><<<grid, 256, 0, s>>>(g);
    else mx4_quantize_kernel<F32, M, false><<<grid, 256, 0, s>>>(g);
}

}  // namespace

int aser_mx4_check(aser_ctx* ctx, const char* who, const aser_mx4* t, bool may_be_empty) {
    if (!t) ASER_FAIL(ctx, ASER_ERR_INVALID_ARG, "%s: null matrix", who);
    if (t->rows < 0 || (t->rows == 0 && !may_be_empty) || t->n <= 0 || t->count <= 0 || t->n > ((int64_t)1 << 22) || t->rows > ((int64_t)1 << 27) || t->count > 65536 ||
        t->rows * t->count > ((int64_t)1 << 30))
        ASER_FAIL(ctx, ASER_ERR_SHAPE, "%s: bad shape of a matrix in 4 bits", who);
    if (t->rows == 0) return ASER_OK;
    if (!t->codes || !t->scales) ASER_FAIL(ctx, ASER_ERR_INVALID_ARG, "%s: null codes or scales", who);
    if (((uintptr_t)t->codes | (uintptr_t)t->scales) & 15) ASER_FAIL(ctx, ASER_ERR_INVALID_ARG, "%s: codes and scales must be 16-byte aligned", who);
    return ASER_OK;
}

extern "C" int aser_mx4_quantize(aser_ctx* ctx, const void* X, int x_dtype, int64_t ldx, const float* mdiag, const aser_mx4* out, void* values, int64_t ldv) {
    if (!ctx) return ASER_ERR_INVALID_ARG;
    if (x_dtype != ASER_DTYPE_BF16 && x_dtype != ASER_DTYPE_F32) ASER_FAIL(ctx, ASER_ERR_DTYPE, "mx4_quantize: dtype must be bf16 or f32");
    ASER_TRY(aser_mx4_check(ctx, "mx4_quantize", out, true));
    if (out->rows != 0 && !X) ASER_FAIL(ctx, ASER_ERR_INVALID_ARG, "mx4_quantize: null pointer");
    if (ldx < out->n || (values && ldv < out->n) || (values && values == X && ldv != ldx)) ASER_FAIL(ctx, ASER_ERR_SHAPE, "mx4_quantize: bad leading dimension");
    const bool f32 = x_dtype == ASER_DTYPE_F32;
    const uintptr_t unit = f32 ? 3 : 1;
    if ((((uintptr_t)X | (uintptr_t)values) & unit) || ((uintptr_t)mdiag & 3)) ASER_FAIL(ctx, ASER_ERR_INVALID_ARG, "mx4_quantize: misaligned pointer");
    if (out->rows == 0) return ASER_OK;
    const int64_t size = f32 ? 4 : 2;
    QuantArgs g{X, ldx, mdiag, out->codes, (uint32_t*)out->scales, values, ldv, out->rows, out->rows * out->count, out->n, mx4_words(out->n), false};
    g.vec = !(((uintptr_t)X | (uintptr_t)values | (uintptr_t)mdiag) & 15) && !(ldx * size & 15) && (!values || !(ldv * size & 15));
    if (ceil_div64(g.all_rows, 16) * g.words > INT32_MAX) ASER_FAIL(ctx, ASER_ERR_SHAPE, "mx4_quantize: too many values");
    ASER_TRY(aser_prepare_device(ctx));
    if (f32) mdiag ? launch<true, true>(g, ctx->stream) : launch<true, false>(g, ctx->stream);
    else mdiag ? launch<false, true>(g, ctx->stream) : launch<false, false>(g, ctx->stream);
    return aser_check_launch(ctx, "mx4_quantize_kernel");
}
