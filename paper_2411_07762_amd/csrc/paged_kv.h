// The paged cache and the batch of requests as the kernels take them, and the checks that both entry points share.
#pragma once
#include "aser_internal.h"

struct PagedArgs {
    void* k; void* v;
    float* k_scale; float* v_scale;              // null: bf16
    const int32_t* start; const int32_t* kv_len; const int32_t* pages;
    int64_t page_stride, head_stride, slot_stride, ld_pages, tokens;
    int n_pages, page_shift, n_kv, n_seq, max_kv, group;   // group: query heads of a key/value head
};

// Rows of request s, [*first, *first + count): what `start` says, clamped so that no row outside the matrices is touched.
__device__ __forceinline__ int64_t request_rows(const PagedArgs& g, int s, int64_t* first) {
    int64_t a = g.start[s], b = g.start[s + 1];
    a = a < 0 ? 0 : (a > g.tokens ? g.tokens : a);
    b = b < a ? a : (b > g.tokens ? g.tokens : b);
    *first = a;
    return b - a;
}
__device__ __forceinline__ int request_kv_len(const PagedArgs& g, int s) {
    const int n = g.kv_len[s];
    return n < 0 ? 0 : (n > g.max_kv ? g.max_kv : n);
}

// Checks everything of the cache and the batch that the host can see, and fills the kernels' arguments.
static inline int aser_paged_args(aser_ctx* ctx, const char* who, const aser_kv_cache* c, const aser_kv_batch* b, int32_t n_heads, PagedArgs* out) {
    if (!c || !b || !c->k || !c->v || !b->start || !b->kv_len || !b->pages) ASER_FAIL(ctx, ASER_ERR_INVALID_ARG, "%s: null pointer", who);
    if (c->dtype != ASER_KV_BF16 && c->dtype != ASER_KV_INT8) ASER_FAIL(ctx, ASER_ERR_DTYPE, "%s: unknown cache dtype %d", who, c->dtype);
    const bool i8 = c->dtype == ASER_KV_INT8;
    if (i8 && (!c->k_scale || !c->v_scale)) ASER_FAIL(ctx, ASER_ERR_INVALID_ARG, "%s: an int8 cache needs scales", who);
    if (((uintptr_t)c->k | (uintptr_t)c->v) & 15) ASER_FAIL(ctx, ASER_ERR_INVALID_ARG, "%s: cache must be 16-byte aligned", who);
    if (i8 && (((uintptr_t)c->k_scale | (uintptr_t)c->v_scale) & 15)) ASER_FAIL(ctx, ASER_ERR_INVALID_ARG, "%s: scales must be 16-byte aligned", who);
    if (((uintptr_t)b->start | (uintptr_t)b->kv_len | (uintptr_t)b->pages) & 3) ASER_FAIL(ctx, ASER_ERR_INVALID_ARG, "%s: misaligned batch array", who);
    if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) ASER_FAIL(ctx, ASER_ERR_SHAPE, "%s: head_dim must be 64, 128 or 256, got %d", who, c->head_dim);
    int shift = 0;
    while (shift < 8 && (1 << shift) != c->page_size) ++shift;
    if (shift < 4 || (1 << shift) != c->page_size) ASER_FAIL(ctx, ASER_ERR_SHAPE, "%s: page_size must be 16, 32, 64, 128 or 256, got %d", who, c->page_size);
    if (c->n_kv <= 0 || n_heads <= 0 || n_heads % c->n_kv || n_heads > 65535)
        ASER_FAIL(ctx, ASER_ERR_SHAPE, "%s: %d query heads over %d key/value heads", who, n_heads, c->n_kv);
    if (c->n_pages <= 0 || c->n_pages > INT32_MAX) ASER_FAIL(ctx, ASER_ERR_SHAPE, "%s: bad number of pages", who);
    if (c->page_stride < 0 || c->head_stride < 0 || c->slot_stride < c->head_dim || ((c->page_stride | c->head_stride | c->slot_stride) & 15))
        ASER_FAIL(ctx, ASER_ERR_SHAPE, "%s: cache strides must be multiples of 16, slots at least head_dim apart", who);
    if (c->slot_stride > ((int64_t)1 << 22)) ASER_FAIL(ctx, ASER_ERR_SHAPE, "%s: slots more than 2^22 elements apart", who);
    if (b->n_seq <= 0 || b->n_seq > 65535 || b->tokens < 0 || b->tokens > INT32_MAX || b->max_new < 0 || b->max_kv < 0)
        ASER_FAIL(ctx, ASER_ERR_SHAPE, "%s: bad batch shape", who);
    if (b->max_kv > (1 << 30) || b->ld_pages < ceil_div64(b->max_kv, c->page_size)) ASER_FAIL(ctx, ASER_ERR_SHAPE, "%s: ld_pages * page_size < max_kv", who);
    *out = PagedArgs{c->k, c->v, i8 ? c->k_scale : nullptr, i8 ? c->v_scale : nullptr, b->start, b->kv_len, b->pages, c->page_stride, c->head_stride,
                     c->slot_stride, b->ld_pages, b->tokens, (int)c->n_pages, shift, c->n_kv, b->n_seq, b->max_kv, n_heads / c->n_kv};
    return ASER_OK;
}

// True when rows of `ld` elements of `size` bytes at p start on 16-byte boundaries.
static inline bool aser_rows_aligned(const void* p, int64_t ld, int size) { return (((uintptr_t)p | (uintptr_t)(ld * size)) & 15) == 0; }
