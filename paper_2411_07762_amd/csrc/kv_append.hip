// New tokens on their way from the projections into attention: queries and keys normalised per head and turned by their
// position, keys and values stored in the paged cache, all in one pass.
//     u = x rsqrt(mean x^2 + eps) w,   (a, b) -> (a c - b s, b c + a s) for the channel pairs of the rotated part.
// A value is read once and written once, a few operations each: bound by memory, or by the launch when few tokens come.
//
// D / 8 lanes hold a head (8 channels each, 16-byte accesses), so the sum of squares and the partner of a rotated
// channel (rot_dim / 2 channels away, a whole number of lanes) come by lane exchange.  A wavefront does 64 / (D / 8)
// heads at a time and stays with its token, whose angles it loads once; with few tokens the heads of a token are spread over
// several wavefronts instead.
// Measured: 11070 tokens of 5 prompts, fp32, 32 + 8 + 8 heads of 128 channels with norms and rotation 83 us, 5.0 TB/s (a plain copy
// reaches 5.3); into an int8 cache 11000 tokens of 5 prompts 81 us; 96 single tokens 6.7 us, one 4.5, of which an empty launch takes 2.
#include "bf16_pair.h"
#include "paged_kv.h"

namespace {

struct AppendArgs {
    PagedArgs p;
    const void* q; const void* k; const void* v;
    int64_t ldq, ldk, ldv, ldqo;
    uint16_t* q_out;
    const float* cos; const float* sin; const float* q_norm; const float* k_norm;
    float eps;
    int half_rot, n_heads, waves_per_token;      // n_heads: 0 without queries
    bool interleaved;
};

// Number of the request that owns row t: the last one that starts at or before t; -1: none.
__device__ __forceinline__ int request_of_row(const PagedArgs& g, int64_t t, int lane) {
    int at_or_before = 0;
    for (int base = 0; base <= g.n_seq; base += 64) {
        const int i = base + lane;
        at_or_before += __popcll(__ballot(i <= g.n_seq && (int64_t)g.start[i <= g.n_seq ? i : 0] <= t));
    }
    return at_or_before > g.n_seq ? -1 : at_or_before - 1;
}

template <bool F32>
__device__ __forceinline__ void load8(const void* base, int64_t i, float x[8]) {
    if (F32) {
        const float4 a = *(const float4*)((const float*)base + i), b = *(const float4*)((const float*)base + i + 4);
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
        x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    } else {
        const uint4 a = *(const uint4*)((const uint16_t*)base + i);
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            x[2 * j] = __uint_as_float(w[j] << 16);
            x[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
        }
    }
}

template <int D, bool F32, bool I8>
__global__ __launch_bounds__(256) void kv_append_kernel(AppendArgs g) {
    constexpr int L = D / 8, R = 64 / L, U = 4;
    const int lane = threadIdx.x & 63;
    const int64_t wave = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int64_t t = wave / g.waves_per_token;
    if (t >= g.p.tokens) return;
    const int part = (int)(wave % g.waves_per_token);
    const int s = request_of_row(g.p, t, lane);
    if (s < 0) return;
    int64_t first;
    const int64_t count = request_rows(g.p, s, &first);
    const int64_t pos = request_kv_len(g.p, s) - count + (t - first);
    if (t < first || t >= first + count || pos < 0) return;
    const int page = g.p.pages[s * g.p.ld_pages + (pos >> g.p.page_shift)];
    const bool have_page = (uint32_t)page < (uint32_t)g.p.n_pages;
    const int slot = (int)(pos & ((1 << g.p.page_shift) - 1));
    const int64_t in_cache = (int64_t)page * g.p.page_stride + slot * g.p.slot_stride;

    const int c0 = (lane % L) * 8;
    float cs[8], sn[8], wq[8], wk[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) { cs[j] = 1.f; sn[j] = 0.f; wq[j] = 1.f; wk[j] = 1.f; }
    int partner = lane;                           // lane that holds the other channels of this lane's pairs
    if (g.cos && c0 < 2 * g.half_rot) {
        const int64_t row = pos * g.half_rot;
        if (g.interleaved) {
            const float4 c = *(const float4*)(g.cos + row + c0 / 2), n = *(const float4*)(g.sin + row + c0 / 2);
            cs[0] = cs[1] = c.x; cs[2] = cs[3] = c.y; cs[4] = cs[5] = c.z; cs[6] = cs[7] = c.w;
            sn[1] = n.x; sn[3] = n.y; sn[5] = n.z; sn[7] = n.w;
            sn[0] = -n.x; sn[2] = -n.y; sn[4] = -n.z; sn[6] = -n.w;
        } else {
            const bool low = c0 < g.half_rot;
            const int64_t at = row + (low ? c0 : c0 - g.half_rot);
            load8<true>(g.cos, at, cs);
            load8<true>(g.sin, at, sn);
            if (low)
#pragma unroll
                for (int j = 0; j < 8; ++j) sn[j] = -sn[j];
            partner = low ? lane + g.half_rot / 8 : lane - g.half_rot / 8;
        }
    }
    if (g.q_norm) load8<true>(g.q_norm, c0, wq);
    if (g.k_norm) load8<true>(g.k_norm, c0, wk);

    const int heads = g.n_heads + 2 * g.p.n_kv, steps = (heads + R - 1) / R;
    const int per = (steps + g.waves_per_token - 1) / g.waves_per_token, end = (part + 1) * per < steps ? (part + 1) * per : steps;
    for (int step = part * per; step < end; step += U) {
        float x[U][8];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            int h = (step + u) * R + lane / L;
            if (h >= heads || step + u >= end) h = heads - 1;          // loaded and not used
            const bool isq = h < g.n_heads, isk = !isq && h < g.n_heads + g.p.n_kv;
            const void* base = isq ? g.q : (isk ? g.k : g.v);
            const int64_t at = isq ? t * g.ldq + h * D : (isk ? t * g.ldk + (h - g.n_heads) * D : t * g.ldv + (h - g.n_heads - g.p.n_kv) * D);
            load8<F32>(base, at + c0, x[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int h = (step + u) * R + lane / L;
            const bool live = h < heads && step + u < end, isq = h < g.n_heads, isk = !isq && h < g.n_heads + g.p.n_kv;
            if (g.q_norm || g.k_norm) {
                float ss = 0.f;
#pragma unroll
                for (int j = 0; j < 8; ++j) ss += x[u][j] * x[u][j];
#pragma unroll
                for (int o = 1; o < L; o <<= 1) ss += __shfl_xor(ss, o);
                const float inv = rsqrtf(ss * (1.0f / D) + g.eps);
                if (isq ? g.q_norm != nullptr : isk && g.k_norm != nullptr)
#pragma unroll
                    for (int j = 0; j < 8; ++j) x[u][j] *= inv * (isq ? wq[j] : wk[j]);
            }
            float y[8];
            if (g.cos) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float other = g.interleaved ? x[u][j ^ 1] : __shfl(x[u][j], partner);
                    y[j] = isq || isk ? x[u][j] * cs[j] + other * sn[j] : x[u][j];
                }
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) y[j] = x[u][j];
            }
            float scale = 1.f;
            if (I8) {
                // by their bits, so that an infinity is above every number and a NaN above that; either makes the scale NaN (top - top)
                uint32_t bits = 0;
#pragma unroll
                for (int j = 0; j < 8; ++j) bits = max(bits, __float_as_uint(y[j]) & 0x7FFFFFFFu);
#pragma unroll
                for (int o = 1; o < L; o <<= 1) bits = max(bits, (uint32_t)__shfl_xor((int)bits, o));
                const float top = __uint_as_float(bits);
                scale = top == 0.f ? 1.f : top / 127.f + (top - top);
            }
            if (!live) continue;
            if (isq || !I8) {
                const uint4 w = make_uint4(bf16_pair(y[0], y[1]), bf16_pair(y[2], y[3]), bf16_pair(y[4], y[5]), bf16_pair(y[6], y[7]));
                if (isq) *(uint4*)(g.q_out + t * g.ldqo + h * D + c0) = w;
                else if (have_page) {
                    const int kvh = h - g.n_heads - (isk ? 0 : g.p.n_kv);
                    *(uint4*)((uint16_t*)(isk ? g.p.k : g.p.v) + in_cache + kvh * g.p.head_stride + c0) = w;
                }
            } else if (have_page) {
                const int kvh = h - g.n_heads - (isk ? 0 : g.p.n_kv);
                uint32_t w[2] = {0u, 0u};
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int code = (int)fminf(fmaxf(rintf(y[j] / scale), -127.f), 127.f);
                    w[j >> 2] |= (uint32_t)(code & 0xFF) << (8 * (j & 3));
                }
                *(uint2*)((int8_t*)(isk ? g.p.k : g.p.v) + in_cache + kvh * g.p.head_stride + c0) = make_uint2(w[0], w[1]);
                if (c0 == 0) (isk ? g.p.k_scale : g.p.v_scale)[((((int64_t)page * g.p.n_kv + kvh) << g.p.page_shift)) + slot] = scale;
            }
        }
    }
}

template <int D>
void launch_append(const AppendArgs& g, bool f32, bool i8, dim3 grid, hipStream_t st) {
    if (f32) {
        if (i8) kv_append_kernel<D, true, true><<<grid, 256, 0, st>>>(g);
        else kv_append_kernel<D, true, false><<<grid, 256, 0, st>>>(g);
    } else {
        if (i8) kv_append_kernel<D, false, true><<<grid, 256, 0, st>>>(g);
        else kv_append_kernel<D, false, false><<<grid, 256, 0, st>>>(g);
    }
}

}  // namespace

extern "C" int aser_kv_append(aser_ctx* ctx, const void* q, int64_t ldq, int32_t n_heads, const void* k, int64_t ldk, const void* v, int64_t ldv,
                              int32_t x_dtype, const aser_qk_opts* opts, const aser_kv_cache* cache, const aser_kv_batch* batch,
                              uint16_t* q_out, int64_t ldqo) {
    if (!ctx) return ASER_ERR_INVALID_ARG;
    if (x_dtype != ASER_DTYPE_BF16 && x_dtype != ASER_DTYPE_F32) ASER_FAIL(ctx, ASER_ERR_DTYPE, "kv_append: dtype must be bf16 or f32");
    AppendArgs g{};
    ASER_TRY(aser_paged_args(ctx, "kv_append", cache, batch, q ? n_heads : (cache ? cache->n_kv : 1), &g.p));
    if (batch->tokens != 0 && (!k || !v || (q == nullptr) != (q_out == nullptr))) ASER_FAIL(ctx, ASER_ERR_INVALID_ARG, "kv_append: null pointer");
    const int D = cache->head_dim, size = x_dtype == ASER_DTYPE_F32 ? 4 : 2;
    if (ldk < (int64_t)cache->n_kv * D || ldv < (int64_t)cache->n_kv * D || (q && (ldq < (int64_t)n_heads * D || ldqo < (int64_t)n_heads * D)))
        ASER_FAIL(ctx, ASER_ERR_SHAPE, "kv_append: leading dimension below the heads' channels");
    if (!aser_rows_aligned(k, ldk, size) || !aser_rows_aligned(v, ldv, size) || (q && (!aser_rows_aligned(q, ldq, size) || !aser_rows_aligned(q_out, ldqo, 2))))
        ASER_FAIL(ctx, ASER_ERR_INVALID_ARG, "kv_append: rows must be 16-byte aligned");
    if (opts) {
        if ((opts->rope_cos == nullptr) != (opts->rope_sin == nullptr)) ASER_FAIL(ctx, ASER_ERR_INVALID_ARG, "kv_append: cosines and sines go together");
        if (((uintptr_t)opts->rope_cos | (uintptr_t)opts->rope_sin | (uintptr_t)opts->q_norm | (uintptr_t)opts->k_norm) & 15)
            ASER_FAIL(ctx, ASER_ERR_INVALID_ARG, "kv_append: tables and weights must be 16-byte aligned");
        if (opts->rope_cos) {
            if (opts->rot_dim <= 0 || opts->rot_dim > D || opts->rot_dim % 16) ASER_FAIL(ctx, ASER_ERR_SHAPE, "kv_append: rot_dim must be a multiple of 16 up to head_dim");
            if (opts->n_pos < batch->max_kv) ASER_FAIL(ctx, ASER_ERR_SHAPE, "kv_append: angles of fewer than max_kv positions");
            g.cos = opts->rope_cos;
            g.sin = opts->rope_sin;
            g.half_rot = opts->rot_dim / 2;
            g.interleaved = opts->interleaved != 0;
        }
        if ((opts->q_norm || opts->k_norm) && !(opts->eps >= 0.f)) ASER_FAIL(ctx, ASER_ERR_INVALID_ARG, "kv_append: eps must not be negative");
        g.q_norm = q ? opts->q_norm : nullptr;
        g.k_norm = opts->k_norm;
        g.eps = opts->eps;
    }
    if (batch->tokens == 0 || batch->max_kv == 0) return ASER_OK;
    g.q = q; g.k = k; g.v = v;
    g.ldq = ldq; g.ldk = ldk; g.ldv = ldv; g.ldqo = ldqo;
    g.q_out = q_out;
    g.n_heads = q ? n_heads : 0;
    // a wavefront per token once that fills the device, else a token's heads on as many as there are
    const int rows = 64 / (D / 8), steps = (g.n_heads + 2 * cache->n_kv + rows - 1) / rows;
    const int64_t want = ceil_div64(4096, batch->tokens);
    g.waves_per_token = want < steps ? (int)want : steps;
    const int64_t blocks = ceil_div64(batch->tokens * g.waves_per_token, 4);
    if (blocks > INT32_MAX) ASER_FAIL(ctx, ASER_ERR_SHAPE, "kv_append: too many tokens");
    ASER_TRY(aser_prepare_device(ctx));
    const dim3 grid((unsigned)blocks);
    const bool f32 = x_dtype == ASER_DTYPE_F32, i8 = cache->dtype == ASER_KV_INT8;
    if (D == 64) launch_append<64>(g, f32, i8, grid, ctx->stream);
    else if (D == 128) launch_append<128>(g, f32, i8, grid, ctx->stream);
    else launch_append<256>(g, f32, i8, grid, ctx->stream);
    return aser_check_launch(ctx, "kv_append_kernel");
}
