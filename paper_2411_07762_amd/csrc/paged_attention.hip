// Attention of new tokens over a paged cache, calls whose requests all have few rows (few_rows.h), and the entry points.
#include "few_rows.h"

namespace {

template <int D, bool I8, bool ONCE>
__global__ __launch_bounds__(256, D == 256 ? 2 : 3) void attn_few_kernel(AttnArgs g) {
    __shared__ FewShared<D> sm;
    few_rows<D, I8, ONCE>(g, blockIdx.x, blockIdx.y, sm);
}

template <int D>
__global__ __launch_bounds__(256) void attn_join_kernel(AttnArgs g) {
    __shared__ FewJoin<D> x;
    few_join<D>(g, blockIdx.x, blockIdx.y, x);
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
int run_few(aser_ctx* ctx, const AttnArgs& g, int64_t max_rows) {
    const dim3 grid((unsigned)((int64_t)g.p.n_seq * g.row_tiles * g.p.n_kv), (unsigned)g.splits);
    const bool once = g.row_tiles == 1;
    if (g.p.k_scale) {
        if (once) attn_few_kernel<D, true, true><<<grid, 256, 0, ctx->stream>>>(g);
        else attn_few_kernel<D, true, false><<<grid, 256, 0, ctx->stream>>>(g);
    } else {
        if (once) attn_few_kernel<D, false, true><<<grid, 256, 0, ctx->stream>>>(g);
        else attn_few_kernel<D, false, false><<<grid, 256, 0, ctx->stream>>>(g);
    }
    ASER_TRY(aser_check_launch(ctx, "attn_few_kernel"));
    if (g.splits == 1) return ASER_OK;
    attn_join_kernel<D><<<dim3(grid.x, (unsigned)(max_rows < 16 ? max_rows : 16)), 256, 0, ctx->stream>>>(g);
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
    AttnArgs g{};
    ASER_TRY(aser_paged_args(ctx, "paged_attention", cache, batch, n_heads, &g.p));
    if (batch->tokens != 0 && (!q || !out)) ASER_FAIL(ctx, ASER_ERR_INVALID_ARG, "paged_attention: null pointer");
    const int64_t width = (int64_t)n_heads * cache->head_dim;
    if (ldq < width || ldo < width) ASER_FAIL(ctx, ASER_ERR_SHAPE, "paged_attention: leading dimension below the heads' channels");
    if (!aser_rows_aligned(q, ldq, 2) || !aser_rows_aligned(out, ldo, 2)) ASER_FAIL(ctx, ASER_ERR_INVALID_ARG, "paged_attention: rows must be 16-byte aligned");
    if (window < 0 || sinks < 0) ASER_FAIL(ctx, ASER_ERR_SHAPE, "paged_attention: negative window or sinks");
    if (!(scale - scale == 0.f)) ASER_FAIL(ctx, ASER_ERR_INVALID_ARG, "paged_attention: scale is not finite");
    if (batch->tokens == 0 || batch->max_new == 0) return ASER_OK;
    // A window that no key can fall out of is none.  Beside tokens in front of position 0 the first key of a wider one would leave 32 bits.
    if (window >= batch->max_kv) window = 0;
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
        return aser_attention_prompt(ctx, g, cache->head_dim, keys, few);
    }
    if (cache->head_dim == 64) return run_few<64>(ctx, g, max_rows);
    if (cache->head_dim == 128) return run_few<128>(ctx, g, max_rows);
    return run_few<256>(ctx, g, max_rows);
}
