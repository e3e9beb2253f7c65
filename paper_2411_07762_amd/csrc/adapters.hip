// Low-rank adapters of many requests beside a projection that they share:
//     Y[t] = Y0[t] + s_a (x_t A_a^T) B_a^T,   a the adapter of row t.
// Rows with the same adapter are taken 16 at a time, so that an adapter is read once for 16 of its rows, wherever they are in
// the batch: the sum is the same for a row whatever its neighbours.  Two launches, P = x A^T in parts of the channel axis
// and Y = Y0 + s P B^T, which adds the parts in their order; a third in front sorts the rows by adapter when there are
// more than 64 of them (up to 64 the groups are formed by a ballot in every wavefront).  A few operations per byte of A, B,
// X and Y: bound by memory, or by the launches when few rows come.
//
// Both products are formed transposed (rank or output in the rows of the 16 x 16 accumulator, token in its columns), so a lane
// holds four consecutive ranks or outputs of one token and loads and stores 16 bytes.  A and B are bf16; fp32 X and the
// fp32 P enter the bf16 instruction as three terms that add up to all 24 bits (v = v1 + v2 + v3, each the rounded rest).
#include "bf16_pair.h"
#include "aser_internal.h"

namespace {

typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

constexpr int kTok = 16;            // rows of a tile
constexpr int kFewRows = 64;        // up to here groups are formed by ballot
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
// running sums, places.
__global__ __launch_bounds__(1024) void adapter_sort_kernel(AdArgs g, int max_tiles) {
    __shared__ int cnt[kMaxAdapters + 1], tile_at[1024], row_at[1024];
    const int tid = threadIdx.x, na = g.n_adapters;
    for (int i = tid; i <= na; i += 1024) cnt[i] = 0;
    __syncthreads();
    for (int64_t t = tid; t < g.rows; t += 1024) {
        const int a = g.id[t];
        atomicAdd(&cnt[(uint32_t)a < (uint32_t)na ? a : na], 1);
    }
    __syncthreads();
    // thread i owns `per` consecutive adapters
    const int per = (na + 1 + 1023) / 1024, lo = min(tid * per, na + 1), hi = min(lo + per, na + 1);
    int nr = 0, nt = 0;
    for (int i = lo; i < hi; ++i) { nr += cnt[i]; nt += (cnt[i] + kTok - 1) / kTok; }
    row_at[tid] = nr;
    tile_at[tid] = nt;
    __syncthreads();
    for (int o = 1; o < 1024; o <<= 1) {
        const int a = tid >= o ? row_at[tid - o] : 0, b = tid >= o ? tile_at[tid - o] : 0;
        __syncthreads();
        row_at[tid] += a;
        tile_at[tid] += b;
        __syncthreads();
    }
    const int total = tile_at[1023];
    int r0 = row_at[tid] - nr, t0 = tile_at[tid] - nt;
    for (int i = lo; i < hi; ++i) {
        const int c = cnt[i];
        for (int x = 0; x < c; x += kTok) g.tiles[t0++] = make_int4(i < na ? i : -1, r0 + x, min(kTok, c - x), 0);
        cnt[i] = r0;                                   // from here on: the next free place
        r0 += c;
    }
    for (int i = total + tid; i < max_tiles; i += 1024) g.tiles[i] = make_int4(-2, 0, 0, 0);
    __syncthreads();
    for (int64_t t = tid; t < g.rows; t += 1024) {
        const int a = g.id[t];
        g.order[atomicAdd(&cnt[(uint32_t)a < (uint32_t)na ? a : na], 1)] = (int32_t)t;
    }
}

// The rows of a workgroup's tile: adapter (-1: rows without one, -2: no such tile) and the row in column `col`, -1 past the last.
struct TileRows {
    int adapter, row;
    __device__ __forceinline__ TileRows(const AdArgs& g, int tile, int lane) {
        const int col = lane & 15;
        if (g.tiles) {
            const int4 t = g.tiles[tile];
            adapter = t.x;
            row = col < t.z ? g.order[t.y + col] : -1;
            return;
        }
        // tile = slots j + q: the rows whose adapter is row j's, if no earlier row has it; 16 q .. of them
        const int slots = (int)((g.rows + kTok - 1) / kTok), j = tile / slots, skip = tile % slots * kTok;
        int a = lane < g.rows ? g.id[lane] : -2;
        if (lane < g.rows && (uint32_t)a >= (uint32_t)g.n_adapters) a = -1;
        const int mine = __shfl(a, j);
        const uint64_t same = __ballot(a == mine && lane < g.rows);
        adapter = (int)(__ffsll((unsigned long long)same) - 1) == j && __popcll(same) > skip ? mine : -2;
        row = -1;
        uint64_t left = same;
        for (int i = 0, k = __popcll(same); i < k; ++i) {
            const int at = __ffsll((unsigned long long)left) - 1;
            left &= left - 1;
            if (i == skip + col) row = at;
        }
    }
};

__device__ __forceinline__ bf16x8_t pack8(const float x[8]) {
    return __builtin_bit_cast(bf16x8_t, make_uint4(bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3]), bf16_pair(x[4], x[5]), bf16_pair(x[6], x[7])));
}
// x as three bf16 terms
__device__ __forceinline__ void three_terms(float x[8], bf16x8_t t[3]) {
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
}

// Eight consecutive bf16 of a row of n, from column c on; zeros past its end.  VEC: rows are 16-byte aligned and n is a multiple of 8.
template <bool VEC>
__device__ __forceinline__ bf16x8_t row8(const uint16_t* row, int64_t c, int64_t n, bool live) {
    uint4 w = make_uint4(0u, 0u, 0u, 0u);
    if (VEC) {
        if (live && c < n) w = *(const uint4*)(row + c);
    } else if (live) {
        uint32_t u[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) u[j] = c + j < n ? row[c + j] : 0u;
        w = make_uint4(u[0] | u[1] << 16, u[2] | u[3] << 16, u[4] | u[5] << 16, u[6] | u[7] << 16);
    }
    return __builtin_bit_cast(bf16x8_t, w);
}
template <bool VEC>
__device__ __forceinline__ void row8_f32(const float* row, int64_t c, int64_t n, bool live, float x[8]) {
    if (VEC) {
        float4 a = make_float4(0.f, 0.f, 0.f, 0.f), b = a;
        if (live && c < n) { a = *(const float4*)(row + c); b = *(const float4*)(row + c + 4); }
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
        x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = live && c + j < n ? row[c + j] : 0.f;
    }
}

// P[part][row][.] = x A^T over the part's channels; the four wavefronts take every fourth step of 32 channels.
template <int RT, bool F32, bool VEC>
__global__ __launch_bounds__(256) void adapter_down_kernel(AdArgs g) {
    __shared__ f32x4_t sm[3][RT][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, grp = lane >> 4;
    const TileRows tr(g, blockIdx.x, lane);
    if (tr.adapter < 0) return;
    const bool live = tr.row >= 0;
    const int64_t row = live ? tr.row : 0;
    const int64_t c0 = blockIdx.y * g.part_n, c1 = c0 + g.part_n < g.n ? c0 + g.part_n : g.n;
    const uint16_t* a_row = g.A + (int64_t)tr.adapter * g.r * g.n;
    f32x4_t acc[RT];
#pragma unroll
    for (int i = 0; i < RT; ++i) acc[i] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
    for (int64_t c = c0 + 32 * wave; c < c1; c += 128) {
        const int64_t at = c + 8 * grp;
        bf16x8_t x[3], a[RT];
        float xf[8];
        if (F32) row8_f32<VEC>((const float*)g.X + row * g.ldx, at, g.n, live, xf);
        else x[0] = row8<VEC>((const uint16_t*)g.X + row * g.ldx, at, g.n, live);
#pragma unroll
        for (int i = 0; i < RT; ++i) a[i] = row8<VEC>(a_row + (16 * i + col) * g.n, at, g.n, 16 * i + col < g.r);
        if (F32) three_terms(xf, x);
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
            for (int k = F32 ? 2 : 0; k >= 0; --k) acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[i], x[k], acc[i], 0, 0, 0);
    }
    if (wave)
#pragma unroll
        for (int i = 0; i < RT; ++i) sm[wave - 1][i][lane] = acc[i];
    __syncthreads();
    if (wave || !live) return;
    float* dst = g.P + ((int64_t)blockIdx.y * g.rows + row) * g.rp;
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        f32x4_t v = acc[i];
#pragma unroll
        for (int w = 0; w < 3; ++w) v += sm[w][i][lane];
        if (16 * i < g.rp) *(f32x4_t*)(dst + 16 * i + 4 * grp) = v;
    }
}

// Y = Y0 + s P B^T: a wavefront has 64 outputs, a workgroup 256.  ALIGNED: four outputs of a row at a time.
template <int KS, bool VEC>
__global__ __launch_bounds__(256) void adapter_up_kernel(AdArgs g, bool aligned) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, grp = lane >> 4;
    const TileRows tr(g, blockIdx.x, lane);
    if (tr.adapter == -2 || (tr.adapter == -1 && g.Y0 == g.Y)) return;
    const bool live = tr.row >= 0;
    const int64_t row = live ? tr.row : 0, o0 = (int64_t)blockIdx.y * 256 + wave * 64;
    if (o0 >= g.m) return;
    f32x4_t acc[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
    if (tr.adapter >= 0) {
        const float s = g.scale ? g.scale[tr.adapter] : 1.f;
        const uint16_t* b = g.B + (int64_t)tr.adapter * g.m * g.r;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            const int at = 32 * k + 8 * grp;
            float p[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) p[j] = 0.f;
            if (live && at < g.rp)
                for (int part = 0; part < g.parts; ++part) {
                    const float* src = g.P + ((int64_t)part * g.rows + row) * g.rp + at;
                    const float4 u = *(const float4*)src, v = *(const float4*)(src + 4);
                    p[0] += u.x; p[1] += u.y; p[2] += u.z; p[3] += u.w;
                    p[4] += v.x; p[5] += v.y; p[6] += v.z; p[7] += v.w;
                }
#pragma unroll
            for (int j = 0; j < 8; ++j) p[j] *= s;
            bf16x8_t t[3];
            three_terms(p, t);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int64_t o = o0 + 16 * i + col;
                const bf16x8_t w = row8<VEC>(b + o * g.r, at, g.r, o < g.m);
#pragma unroll
                for (int x = 2; x >= 0; --x) acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, t[x], acc[i], 0, 0, 0);
            }
        }
    }
    if (!live) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t o = o0 + 16 * i + 4 * grp;
        float* y = g.Y + row * g.ldy + o;
        const float* y0 = g.Y0 ? g.Y0 + row * g.ldy0 + o : nullptr;
        if (aligned && o + 4 <= g.m) {
            f32x4_t v = acc[i];
            if (y0) v += *(const f32x4_t*)y0;
            *(f32x4_t*)y = v;
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (o + e < g.m) y[e] = acc[i][e] + (y0 ? y0[e] : 0.f);
        }
    }
}

struct AdPlan { int tiles, parts; int64_t part_n; size_t p_bytes, order_bytes, tile_bytes; };

AdPlan plan_adapters(int64_t rows, int64_t n, int r) {
    AdPlan p;
    const bool few = rows <= kFewRows;
    p.tiles = (int)(few ? ceil_div64(rows, kTok) * rows : ceil_div64(rows, kTok) + kMaxAdapters + 1);
    // parts of the channel axis: about 512 workgroups, at least 256 channels each
    const int64_t groups = few ? rows : ceil_div64(rows, kTok);
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

template <int RT>
void launch_down(const AdArgs& g, bool f32, bool vec, dim3 grid, hipStream_t st) {
    if (f32) {
        if (vec) adapter_down_kernel<RT, true, true><<<grid, 256, 0, st>>>(g);
        else adapter_down_kernel<RT, true, false><<<grid, 256, 0, st>>>(g);
    } else {
        if (vec) adapter_down_kernel<RT, false, true><<<grid, 256, 0, st>>>(g);
        else adapter_down_kernel<RT, false, false><<<grid, 256, 0, st>>>(g);
    }
}
template <int KS>
void launch_up(const AdArgs& g, bool vec, bool aligned, dim3 grid, hipStream_t st) {
    if (vec) adapter_up_kernel<KS, true><<<grid, 256, 0, st>>>(g, aligned);
    else adapter_up_kernel<KS, false><<<grid, 256, 0, st>>>(g, aligned);
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
    if (!X || !adapter || !A || !B || !Y) ASER_FAIL(ctx, ASER_ERR_INVALID_ARG, "adapter_forward: null pointer");
    if (x_dtype != ASER_DTYPE_BF16 && x_dtype != ASER_DTYPE_F32) ASER_FAIL(ctx, ASER_ERR_DTYPE, "adapter_forward: dtype must be bf16 or f32");
    if (rows < 0 || rows > INT32_MAX / 32 || n <= 0 || m <= 0 || ldx < n || ldy < m || (Y0 && ldy0 < m) || (Y0 == Y && ldy0 != ldy) || m > ((int64_t)1 << 23)) ASER_FAIL(ctx, ASER_ERR_SHAPE, "adapter_forward: bad shape");
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
        const int64_t most = ceil_div64(rows, kTok) + (n_adapters + 1 < rows ? n_adapters + 1 : rows);
        tiles = (int)(most < p.tiles ? most : p.tiles);
        adapter_sort_kernel<<<1, 1024, 0, ctx->stream>>>(g, tiles);
        ASER_TRY(aser_check_launch(ctx, "adapter_sort_kernel"));
    }
    const int xw = f32 ? 3 : 7;                          // elements of 16 bytes, less one
    const bool vec_a = n % 8 == 0 && ((uintptr_t)A & 15) == 0 && ((uintptr_t)X & 15) == 0 && (ldx & xw) == 0;
    const bool vec_b = r % 8 == 0 && ((uintptr_t)B & 15) == 0;
    const bool aligned = (ldy & 3) == 0 && ((uintptr_t)Y & 15) == 0 && (!Y0 || ((ldy0 & 3) == 0 && ((uintptr_t)Y0 & 15) == 0));
    const dim3 down((unsigned)tiles, (unsigned)p.parts), up((unsigned)tiles, (unsigned)ceil_div64(m, 256));
    if (r <= 16) launch_down<1>(g, f32, vec_a, down, ctx->stream);
    else if (r <= 32) launch_down<2>(g, f32, vec_a, down, ctx->stream);
    else if (r <= 64) launch_down<4>(g, f32, vec_a, down, ctx->stream);
    else launch_down<8>(g, f32, vec_a, down, ctx->stream);
    ASER_TRY(aser_check_launch(ctx, "adapter_down_kernel"));
    if (r <= 32) launch_up<1>(g, vec_b, aligned, up, ctx->stream);
    else if (r <= 64) launch_up<2>(g, vec_b, aligned, up, ctx->stream);
    else launch_up<4>(g, vec_b, aligned, up, ctx->stream);
    return aser_check_launch(ctx, "adapter_up_kernel");
}
