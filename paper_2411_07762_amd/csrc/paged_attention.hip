// Attention of new tokens over a paged cache, calls whose requests all have few rows (few_rows.h), and the entry points.
#include "few_rows.h"

namespace {

constexpr int kMaxSplits = 256;                   // a thread of the joining kernel for each

template <int D, bool I8, bool ONCE>
__global__ __launch_bounds__(256, D == 256 ? 2 : 3) void attn_few_kernel(AttnArgs g) {
    __shared__ FewShared<D> sm;
    few_rows<D, I8, ONCE>(g, blockIdx.x, blockIdx.y, sm);
}

// Joins the splits of one row: o = sum_s w_s o_s / sum_s w_s l_s, w_s = exp2(m_s - max m).  The maxima are asked for before the
// request's length says how many of them there are: one wait less in a kernel that is nothing but waits.
template <int D>
__global__ __launch_bounds__(256) void attn_join_kernel(AttnArgs g) {
    constexpr int CL = D / 4, SL = 256 / CL;      // lanes over channels (4 each), splits side by side
    __shared__ f32x4_t sm[SL][CL];
    __shared__ float sm_w[kMaxSplits], sm_m[4], sm_l[4];
    const int tid = threadIdx.x, cl = tid % CL, sl = tid / CL, r = blockIdx.y;
    const int tile = g.by_kv(blockIdx.x), kvh = blockIdx.x - tile * g.p.n_kv;
    const FewTile ft(g, tile);
    const int s = ft.seq, rt = ft.row_tile;
    const int64_t pr = (int64_t)blockIdx.x * g.splits * 16 + r;
    float2 ml = g.part_ml[pr + (int64_t)min(tid, g.splits - 1) * 16];
    int64_t row0;
    const int count = (int)request_rows(g.p, s, &row0), kv = request_kv_len(g.p, s), row = rt * 16 + r;
    if (row >= count * g.p.group || count * g.p.group > g.few_rows) return;
    const int last_row = min(rt * 16 + 15, count * g.p.group - 1);
    const KeyTiles<kTile> kt(max(kv - count + g.by_group(rt * 16), 0), kv - count + g.by_group(last_row), g.window, g.sinks);
    const int used = g.by_split(kt.total + g.tiles_per_split - 1);
    if (used <= 1) return;
    if (tid >= used) ml = make_float2(kNone, 0.f);
    float top = ml.x;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));
    if ((tid & 63) == 0) sm_m[tid >> 6] = top;
    __syncthreads();
    top = fmaxf(fmaxf(sm_m[0], sm_m[1]), fmaxf(sm_m[2], sm_m[3]));
    const float w = tid < used ? __builtin_amdgcn_exp2f(ml.x - top) : 0.f;
    float ll = w * ml.y;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) ll += __shfl_xor(ll, o);
    if ((tid & 63) == 0) sm_l[tid >> 6] = ll;
    sm_w[tid] = w;
    __syncthreads();
    f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int i = sl; i < used; i += SL) acc += *(const f32x4_t*)(g.part_o + (pr + (int64_t)i * 16) * D + 4 * cl) * sm_w[i];
    sm[sl][cl] = acc;
    __syncthreads();
    if (sl) return;
#pragma unroll
    for (int i = 1; i < SL; ++i) acc += sm[i][cl];
    ll = (sm_l[0] + sm_l[1]) + (sm_l[2] + sm_l[3]);
    const float inv = ll > 0.f ? 1.f / ll : 0.f;
    const int token = g.by_group(row);
    uint16_t* dst = g.out + (row0 + token) * g.ldo + (int64_t)(kvh * g.p.group + row - token * g.p.group) * D + 4 * cl;
    *(uint2*)dst = make_uint2(bf16_pair(acc[0] * inv, acc[1] * inv), bf16_pair(acc[2] * inv, acc[3] * inv));
}

constexpr int kFewRows = 64;                      // requests of more rows take the kernel for prompts

struct Plan { int most_splits, splits, tiles_per_split, row_tiles; };

// Splits of the key axis: several thousand workgroups even out requests of different lengths, as long as each of a workgroup's four
// wavefronts has 8 steps; a call of few requests takes shorter ones, down to two steps, to fill the device.  (Equal shares of all keys
// for a fixed number of workgroups came out no faster on ragged batches and slower on others.)  keys: the most that a row sees.
// Where a call has prompts too, most of the others are single tokens: one row tile of a request is counted (31 tokens over 8192 keys and a prompt of 1000
// 209 -> 203 us).  Workspace is there for most_splits, which grows with the keys (a window asks for no more than none does).
Plan plan_few(int64_t n_seq, int64_t n_kv, int64_t group, int64_t max_new, int64_t keys) {
    Plan p;
    const int64_t rows = max_new * group < kFewRows ? max_new * group : kFewRows;
    p.row_tiles = (int)ceil_div64(rows, 16);
    const int64_t tiles = keys / kTile + 3, pairs = n_seq * n_kv * (max_new * group > kFewRows ? 1 : p.row_tiles);
    int64_t splits = ceil_div64(4096, pairs);
    if (splits > tiles / 32) splits = tiles / 32;
    if (splits * pairs < 1024) {
        splits = ceil_div64(1024, pairs);
        if (splits > tiles / 8) splits = tiles / 8;
    }
    if (splits > kMaxSplits) splits = kMaxSplits;
    if (splits < 1) splits = 1;
    p.most_splits = (int)splits;
    p.tiles_per_split = (int)ceil_div64(tiles, splits);
    p.splits = (int)ceil_div64(tiles, p.tiles_per_split);
    return p;
}
int64_t keys_seen(int64_t max_kv, int64_t max_new, int64_t window, int64_t sinks) {
    const int64_t seen = window + sinks + max_new + 2 * kTile;  // the windows of a request's new tokens, in whole steps
    return window > 0 && seen < max_kv ? seen : max_kv;
}

// One row tile reads its keys once.  Then the hint that a line is not wanted again pays: 64 requests of up to 8192 tokens, 128 channels, bf16 242 -> 223 us,
// int8 138 -> 131; not where several row tiles share the keys (142 -> 195 with four).
template <int D>
int run_few(aser_ctx* ctx, const AttnArgs& g) {
    const dim3 grid((unsigned)((int64_t)g.p.n_seq * g.row_tiles * g.p.n_kv), (unsigned)g.splits);
    const bool once = g.row_tiles == 1;
    if (g.p.k_scale) {
        if (once) attn_few_kernel<D, true, true><<<grid, 256, 0, ctx->stream>>>(g);
        else attn_few_kernel<D, true, false><<<grid, 256, 0, ctx->stream>>>(g);
    } else {
        if (once) attn_few_kernel<D, false, true><<<grid, 256, 0, ctx->stream>>>(g);
        else attn_few_kernel<D, false, false><<<grid, 256, 0, ctx->stream>>>(g);
    }
    return aser_check_launch(ctx, "attn_few_kernel");
}
template <int D>
int join_few(aser_ctx* ctx, const AttnArgs& g, int64_t max_rows) {
    if (g.splits == 1) return ASER_OK;
    attn_join_kernel<D><<<dim3((unsigned)(g.p.n_seq * g.row_tiles * g.p.n_kv), (unsigned)(max_rows < 16 ? max_rows : 16)), 256, 0, ctx->stream>>>(g);
    return aser_check_launch(ctx, "attn_join_kernel");
}

size_t few_workspace(const Plan& p, int64_t n_seq, int64_t n_kv, int head_dim, size_t* o_bytes) {
    const size_t rows = p.most_splits > 1 ? (size_t)(n_seq * p.row_tiles * n_kv) * p.most_splits * 16 : 0;
    *o_bytes = align_up(rows * head_dim * 4, 256);
    return *o_bytes + align_up(rows * 8, 256);
}

}  // namespace

extern "C" size_t aser_paged_attention_workspace_bytes(const aser_kv_cache* c, const aser_kv_batch* b, int32_t n_heads) {
    if (!c || !b || c->n_kv <= 0 || n_heads < c->n_kv || b->n_seq <= 0 || b->tokens <= 0 || b->max_new <= 0 || b->max_kv <= 0 || c->head_dim <= 0) return kAserWsTail;
    const int64_t group = n_heads / c->n_kv;
    size_t o_bytes, need = few_workspace(plan_few(b->n_seq, c->n_kv, group, b->max_new, b->max_kv), b->n_seq, c->n_kv, c->head_dim, &o_bytes);
    if (b->max_new * group > kFewRows) need += aser_attention_prompt_workspace(b->tokens, b->n_seq, c->n_kv, group, c->head_dim, b->max_kv);
    return need + kAserWsTail;
}

extern "C" int aser_paged_attention(aser_ctx* ctx, const uint16_t* q, int64_t ldq, int32_t n_heads, const aser_kv_cache* cache,
                                    const aser_kv_batch* batch, float scale, int32_t window, int32_t sinks, uint16_t* out, int64_t ldo) {
    if (!ctx) return ASER_ERR_INVALID_ARG;
    if (!q || !out) ASER_FAIL(ctx, ASER_ERR_INVALID_ARG, "paged_attention: null pointer");
    AttnArgs g{};
    ASER_TRY(aser_paged_args(ctx, "paged_attention", cache, batch, n_heads, &g.p));
    const int64_t width = (int64_t)n_heads * cache->head_dim;
    if (ldq < width || ldo < width) ASER_FAIL(ctx, ASER_ERR_SHAPE, "paged_attention: leading dimension below the heads' channels");
    if (!aser_rows_aligned(q, ldq, 2) || !aser_rows_aligned(out, ldo, 2)) ASER_FAIL(ctx, ASER_ERR_INVALID_ARG, "paged_attention: rows must be 16-byte aligned");
    if (window < 0 || sinks < 0) ASER_FAIL(ctx, ASER_ERR_SHAPE, "paged_attention: negative window or sinks");
    if (!(scale - scale == 0.f)) ASER_FAIL(ctx, ASER_ERR_INVALID_ARG, "paged_attention: scale is not finite");
    if (batch->tokens == 0 || batch->max_new == 0) return ASER_OK;
    const int64_t keys = keys_seen(batch->max_kv, batch->max_new, window, window > 0 ? sinks : 0), max_rows = (int64_t)batch->max_new * g.p.group;
    const Plan plan = plan_few(g.p.n_seq, g.p.n_kv, g.p.group, batch->max_new, keys);
    g.q = q; g.ldq = ldq; g.out = out; g.ldo = ldo;
    g.by_group = Divider::by(g.p.group);
    g.by_kv = Divider::by(g.p.n_kv);
    g.c = scale * 1.4426950408889634f;
    g.window = window;
    g.sinks = window > 0 ? sinks : 0;
    g.few_rows = kFewRows;
    g.splits = plan.splits; g.tiles_per_split = plan.tiles_per_split; g.row_tiles = plan.row_tiles;
    g.by_tiles = Divider::by(g.row_tiles);
    g.by_split = Divider::by(g.tiles_per_split);
    if ((int64_t)g.p.n_seq * g.row_tiles * g.p.n_kv > INT32_MAX || batch->tokens * g.p.group > INT32_MAX)
        ASER_FAIL(ctx, ASER_ERR_SHAPE, "paged_attention: too many requests times rows");
    size_t o_bytes, need = few_workspace(plan, g.p.n_seq, g.p.n_kv, cache->head_dim, &o_bytes);
    const size_t few = need;
    if (max_rows > kFewRows) need += aser_attention_prompt_workspace(g.p.tokens, g.p.n_seq, g.p.n_kv, g.p.group, cache->head_dim, keys);
    if (need > 0 && (!ctx->ws || ctx->ws_bytes < need + kAserWsTail)) ASER_FAIL(ctx, ASER_ERR_WORKSPACE, "paged_attention: workspace too small");
    ASER_TRY(aser_prepare_device(ctx));
    g.part_o = (float*)ctx->ws;
    g.part_ml = (float2*)((char*)ctx->ws + o_bytes);
    if (max_rows > kFewRows) {
        if (g.p.n_seq == 1) g.few_rows = -1;      // one request: it is for the kernel for prompts, whatever it is
        ASER_TRY(aser_attention_prompt(ctx, g, cache->head_dim, keys, few));
        if (g.p.n_seq == 1) return ASER_OK;
    } else {
        ASER_TRY(cache->head_dim == 64 ? run_few<64>(ctx, g) : cache->head_dim == 128 ? run_few<128>(ctx, g) : run_few<256>(ctx, g));
    }
    return cache->head_dim == 64 ? join_few<64>(ctx, g, max_rows) : cache->head_dim == 128 ? join_few<128>(ctx, g, max_rows) : join_few<256>(ctx, g, max_rows);
}
