// Attention of prompts over the paged cache: the formulas and the transposed products of paged_attention.hip on tiles that the
// matrix instructions bound instead of memory, 4 D operations per visible key, row and head.
//
// A wavefront owns 32 RB rows (a row: one query head of one new token; the heads that share a key/value head lie next to each
// other, so a tile spans few positions and little of it is masked) and goes through the keys 32 at a time with
// v_mfma_f32_32x32x16_bf16:  S^T = K Q^T leaves a query row in each column and 16 keys in the registers of a lane, which
// rounded to bf16 are, 8 at a time, the operand of O^T += V^T P^T as they stand (keys 4 h .. and 8 + 4 h .., h = lane / 32).
// The workgroup's wavefronts share the keys and values through LDS: stages of KEYS keys, copied by global_load_lds_dwordx4
// (pages that are not there and keys that nobody sees come from a chunk of zeros), three stages in flight, one barrier per stage.
// K is read as rows (16 bytes of a key), V through ds_read_b64_tr_b16 (four keys of a channel); the chunks of a row are
// swizzled so that neither meets bank conflicts.  8-bit caches go through registers, which widen the codes on their way to LDS; the
// scales multiply logits and probabilities.
#include "attention.h"

namespace {

typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef short s16x8_t __attribute__((ext_vector_type(8)));

__device__ const uint4 g_zeros = {0u, 0u, 0u, 0u};

__device__ __forceinline__ bf16x8_t lds_tr(const char* lo, const char* hi) {
    typedef s16x4_t __attribute__((address_space(3))) * lds_s4p;
    const s16x4_t a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4p)lo);
    const s16x4_t b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4p)hi);
    return __builtin_bit_cast(bf16x8_t, (s16x8_t)__builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

// The u-th row tile of BM rows, counted from the last request's last one (later rows see more keys: long tiles start first).
struct RowTile {
    int seq, tile;
    __device__ __forceinline__ RowTile(const AttnArgs& g, int u, int bm, int lane) {
        int total = 0;
        for (int pass = 0; pass < 2; ++pass) {
            int before = 0;
            seq = -1;
            for (int base = 0; base < g.p.n_seq; base += 64) {
                int nt = 0;
                if (base + lane < g.p.n_seq) {
                    int64_t first;
                    const int64_t rows = request_rows(g.p, base + lane, &first) * g.p.group;
                    nt = rows > g.few_rows ? (int)((rows + bm - 1) / bm) : 0;
                }
                int upto = nt;
#pragma unroll
                for (int o = 1; o < 64; o <<= 1) {
                    const int x = __shfl_up(upto, o);
                    upto += lane >= o ? x : 0;
                }
                if (pass == 1) {
                    const int t = total - 1 - u;
                    const uint64_t mine = __ballot((before + upto > t) & (before + upto - nt <= t));
                    if (mine) {
                        const int l = __ffsll((unsigned long long)mine) - 1;
                        seq = base + l;
                        tile = t - (before + __shfl(upto - nt, l));
                        return;
                    }
                }
                before += __shfl(upto, 63);
            }
            total = before;
            if (u >= total) return;
        }
    }
};

template <int D, bool I8, int RB, int W>
__global__ __launch_bounds__(64 * W, W / 4) void attn_prompt_kernel(AttnArgs g) {
    constexpr int KEYS = D == 256 ? 32 : 64, SUB = KEYS / 32, CH = D / 8, KS = D / 16, DB = D / 32;
    constexpr int PITCH = 2 * D, HALF = KEYS * PITCH, STAGE = 2 * HALF, NST = 4, BM = 32 * RB * W;
    constexpr int GR = KEYS / W;                  // keys that a wavefront stages, all on one page
    constexpr int LOADS = GR * CH / 64;           // 16-byte loads of a lane for them, of K and of V each
    static_assert(LOADS >= 1, "a wavefront stages at least one load");
    extern __shared__ __align__(16) char smem[];
    int* sm_there = (int*)(smem + NST * STAGE);   // [stage][wave]: the page of its keys is there
    float* sm_ks = (float*)(sm_there + NST * W);  // int8: [stage][key] scales of K, then of V
    float* sm_vs = sm_ks + NST * KEYS;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 31, h = lane >> 5;
    const int kvh = blockIdx.x % g.p.n_kv;
    const RowTile rt(g, blockIdx.x / g.p.n_kv, BM, lane);
    const int s = __builtin_amdgcn_readfirstlane(rt.seq);
    if (s < 0) return;
    int64_t row0;
    const int count = (int)request_rows(g.p, s, &row0), kv = request_kv_len(g.p, s), rows = count * g.p.group, group = g.p.group;
    const int first = __builtin_amdgcn_readfirstlane(rt.tile) * BM, base_pos = kv - count;
    const int p_lo = max(base_pos + first / group, 0), p_hi = base_pos + min(first + BM - 1, rows - 1) / group;
    const int low_all = g.window > 0 ? base_pos + first / group - g.window + 1 : 0;
    const KeyTiles<KEYS> kt(p_lo, p_hi, g.window, g.sinks);

    // rows of this wavefront
    const int wfirst = first + wave * 32 * RB;
    const bool idle = wfirst >= rows;
    const int wp_lo = base_pos + min(wfirst, rows - 1) / group, wp_hi = base_pos + min(wfirst + 32 * RB - 1, rows - 1) / group;
    int pos[RB];
    bf16x8_t q[RB][KS];
    const uint32_t flip = g.c < 0.f ? 0x80008000u : 0u;                      // a negative scale turns the queries round
    const float c = fmaxf(fabsf(g.c), 1e-37f);                               // 0: every logit is as good as 0, masked ones stay -inf
#pragma unroll
    for (int b = 0; b < RB; ++b) {
        const int r = min(wfirst + 32 * b + col, rows - 1);
        pos[b] = base_pos + r / group;
        const uint16_t* src = g.q + (row0 + r / group) * g.ldq + (int64_t)(kvh * group + r % group) * D + 8 * h;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            uint4 w = *(const uint4*)(src + 16 * k);
            w.x ^= flip; w.y ^= flip; w.z ^= flip; w.w ^= flip;
            q[b][k] = __builtin_bit_cast(bf16x8_t, w);
        }
    }
    f32x16_t o[RB][DB];
    float m[RB], l[RB];
#pragma unroll
    for (int b = 0; b < RB; ++b) {
        m[b] = kNone;
        l[b] = 0.f;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[b][d][e] = 0.f;
    }

    // staging: wavefront w has keys GR w .. of a stage; lane: row lane / CH (+ 64 / CH per load), slot lane % CH
    const int* table = g.p.pages + s * g.p.ld_pages;
    const int page_mask = (1 << g.p.page_shift) - 1;
    const int64_t head_at = kvh * g.p.head_stride;
    const uint32_t ring = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem + wave * GR * PITCH;
    auto k_swizzle = [](int r) { return D == 64 ? (r >> 1) & 7 : r & 15; };
    auto v_swizzle = [](int r) { return D == 64 ? 4 * ((r >> 1) & 1) : 4 * (r & 3); };
    auto page_of = [&](int i) -> int {
        const int key = kt.first_key(i) + GR * wave;
        return i < kt.total && key < kv ? table[key >> g.p.page_shift] : -1;
    };
    uint4 held[I8 ? LOADS : 1];                    // int8: codes on their way (one 16-byte load is two chunks of a row)
    float held_scale = 0.f;
    auto issue = [&](int i, int page) {            // stage i of the list into slot i % NST
        const int st = i & (NST - 1), key0 = kt.first_key(i) + GR * wave;
        const bool there = (uint32_t)page < (uint32_t)g.p.n_pages;
        const int64_t at = (int64_t)(there ? page : 0) * g.p.page_stride + head_at + (int64_t)(key0 & page_mask) * g.p.slot_stride;
        if (lane == 0) sm_there[st * W + wave] = there ? 1 : 0;
        if constexpr (!I8) {
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int t = 0; t < LOADS; ++t) {
                    const int r = t * (64 / CH) + lane / CH, slot = lane % CH, rr = GR * wave + r, key = key0 + r;
                    const int chunk = slot ^ (half ? v_swizzle(rr) : k_swizzle(rr));
                    const bool used = there & (key <= p_hi) & ((key >= low_all) | (key < g.sinks));
                    const char* src = (const char*)((half ? (const uint16_t*)g.p.v : (const uint16_t*)g.p.k) + at + r * g.p.slot_stride + 8 * chunk);
                    if (!used) src = (const char*)&g_zeros;
                    const uint32_t dst = ring + st * STAGE + half * HALF + t * 1024;
                    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" : : "s"(dst), "v"(src) : "memory", "m0");
                }
        } else {
            // a lane takes 16 codes (two chunks) of row lane / (CH / 2): first the loads of K, then of V
#pragma unroll
            for (int t = 0; t < LOADS; ++t) {
                const int x = t * 64 + lane, half = x / (GR * CH / 2), y = x % (GR * CH / 2), r = y / (CH / 2), key = key0 + r;
                const bool used = there & (key <= p_hi) & ((key >= low_all) | (key < g.sinks));
                const int8_t* src = (half ? (const int8_t*)g.p.v : (const int8_t*)g.p.k) + at + r * g.p.slot_stride + 16 * (y % (CH / 2));
                held[t] = make_uint4(0u, 0u, 0u, 0u);
                if (used) held[t] = *(const uint4*)src;
            }
            if (lane < 2 * GR) {
                const int r = lane % GR, key = key0 + r;
                const bool used = there & (key <= p_hi) & ((key >= low_all) | (key < g.sinks));
                const float* src = (lane < GR ? g.p.k_scale : g.p.v_scale) + (((int64_t)(there ? page : 0) * g.p.n_kv + kvh) << g.p.page_shift) + (key0 & page_mask) + r;
                held_scale = used ? *src : 0.f;
            }
        }
    };
    auto land = [&](int i) {                       // int8: what issue(i) has fetched goes to LDS, widened
        if constexpr (I8) {
            const int st = i & (NST - 1);
            char* dst = smem + st * STAGE + wave * GR * PITCH;
#pragma unroll
            for (int t = 0; t < LOADS; ++t) {
                const int x = t * 64 + lane, half = x / (GR * CH / 2), y = x % (GR * CH / 2), r = y / (CH / 2), ch = 2 * (y % (CH / 2)), rr = GR * wave + r;
                const int sw = half ? v_swizzle(rr) : k_swizzle(rr);
                char* row = dst + half * HALF + r * PITCH;
                const uint4 w = held[t];
                *(uint4*)(row + ((ch ^ sw) << 4)) = make_uint4(codes_pair<0>(w.x), codes_pair<2>(w.x), codes_pair<0>(w.y), codes_pair<2>(w.y));
                *(uint4*)(row + (((ch + 1) ^ sw) << 4)) = make_uint4(codes_pair<0>(w.z), codes_pair<2>(w.z), codes_pair<0>(w.w), codes_pair<2>(w.w));
            }
            if (lane < 2 * GR) (lane < GR ? sm_ks : sm_vs)[st * KEYS + GR * wave + lane % GR] = held_scale;
        }
    };

    // operand offsets inside a stage
    int k_off[KS], v_off[DB];
#pragma unroll
    for (int k = 0; k < KS; ++k) k_off[k] = col * PITCH + (((2 * k + h) ^ k_swizzle(col)) << 4);
    {
        const int i = lane & 15, r = 4 * h + (i >> 2);
#pragma unroll
        for (int d = 0; d < DB; ++d) v_off[d] = HALF + r * PITCH + (((4 * d + 2 * ((lane >> 4) & 1) + ((i & 3) >> 1)) ^ v_swizzle(r)) << 4) + 8 * (i & 1);
    }

    const int t0 = 0, t1 = kt.total;
    int page_next = -1;
    if constexpr (!I8) {
#pragma unroll
        for (int i = 0; i < NST - 1; ++i) {
            const int page = page_of(t0 + i);
            if (t0 + i < t1) issue(t0 + i, page);
        }
        page_next = page_of(t0 + NST - 1);
    } else {
        if (t0 < t1) { issue(t0, page_of(t0)); land(t0); }
        if (t0 + 1 < t1) issue(t0 + 1, page_of(t0 + 1));
        page_next = page_of(t0 + 2);
    }
    for (int i = t0; i < t1; ++i) {
        if constexpr (!I8) {
            // stages i + 1 and i + 2 may still be on their way
            const int behind = min(t1 - 1 - i, NST - 2);
            if (behind == 2) __builtin_amdgcn_s_waitcnt(0x0070 | (4 * LOADS & 15) | ((4 * LOADS >> 4) << 14));
            else if (behind == 1) __builtin_amdgcn_s_waitcnt(0x0070 | (2 * LOADS & 15) | ((2 * LOADS >> 4) << 14));
            else __builtin_amdgcn_s_waitcnt(0x0070);
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            if (i + NST - 1 < t1) {
                issue(i + NST - 1, page_next);
                page_next = page_of(i + NST);
            }
        } else {
            __syncthreads();
            if (i + 1 < t1) land(i + 1);
            if (i + 2 < t1) {
                issue(i + 2, page_next);
                page_next = page_of(i + 3);
            }
        }
        const char* stage = smem + (i & (NST - 1)) * STAGE;
        const int st = i & (NST - 1);
#pragma unroll
        for (int u = 0; u < SUB; ++u) {
            const int key0 = kt.first_key(i) + 32 * u;
            const int wlow = g.window > 0 ? wp_lo - g.window + 1 : 0;
            if (idle || key0 > wp_hi || (key0 + 31 < wlow && key0 >= g.sinks)) continue;
            f32x16_t st_acc[RB];
#pragma unroll
            for (int b = 0; b < RB; ++b)
#pragma unroll
                for (int e = 0; e < 16; ++e) st_acc[b][e] = 0.f;
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                const bf16x8_t kf = *(const bf16x8_t*)(stage + k_off[k] + u * 32 * PITCH);
#pragma unroll
                for (int b = 0; b < RB; ++b) st_acc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, q[b][k], st_acc[b], 0, 0, 0);
            }
            if constexpr (I8) {
#pragma unroll
                for (int e4 = 0; e4 < 4; ++e4) {
                    const f32x4_t ks = *(const f32x4_t*)(sm_ks + st * KEYS + 32 * u + 8 * e4 + 4 * h);
#pragma unroll
                    for (int b = 0; b < RB; ++b)
#pragma unroll
                        for (int e = 0; e < 4; ++e) st_acc[b][4 * e4 + e] *= ks[e];
                }
            }
            int there = 1;
#pragma unroll
            for (int x = 0; x < 32 / GR; ++x) there &= sm_there[st * W + u * (32 / GR) + x];
            there = __builtin_amdgcn_readfirstlane(there);
            const bool plain = there && key0 + 31 <= wp_lo && (g.window <= 0 || key0 >= wp_hi - g.window + 1 || key0 + 32 <= g.sinks);
            if (!plain) {
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int off = 8 * (e >> 2) + 4 * h + (e & 3), key = key0 + off;
                    const bool page_there = sm_there[st * W + (32 * u + off) / GR] != 0;
#pragma unroll
                    for (int b = 0; b < RB; ++b) {
                        const bool seen = page_there & (key <= pos[b]) & ((key >= pos[b] - g.window + 1) | (key < g.sinks) | (g.window <= 0));
                        st_acc[b][e] = seen ? st_acc[b][e] : -INFINITY;
                    }
                }
            }
            bf16x8_t pb[RB][2];
#pragma unroll
            for (int b = 0; b < RB; ++b) {
                float top = st_acc[b][0];
#pragma unroll
                for (int e = 1; e < 16; ++e) top = fmaxf(top, st_acc[b][e]);
                top *= c;
                // the maximum moves only when a logit is 8 above it: until then p <= 2^8, which neither fp32 sums nor bf16 mind
                if (__ballot(top > m[b] + 8.f)) {
                    top = fmaxf(top, __shfl_xor(top, 32));
                    const float m_new = fmaxf(m[b], top), r = __builtin_amdgcn_exp2f(m[b] - m_new);
                    m[b] = m_new;
                    l[b] *= r;
#pragma unroll
                    for (int d = 0; d < DB; ++d) o[b][d] *= r;
                }
                float p[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    p[e] = __builtin_amdgcn_exp2f(fmaf(st_acc[b][e], c, -m[b]));
                    l[b] += p[e];
                }
                if constexpr (I8) {
#pragma unroll
                    for (int e4 = 0; e4 < 4; ++e4) {
                        const f32x4_t vs = *(const f32x4_t*)(sm_vs + st * KEYS + 32 * u + 8 * e4 + 4 * h);
#pragma unroll
                        for (int e = 0; e < 4; ++e) p[4 * e4 + e] *= vs[e];
                    }
                }
#pragma unroll
                for (int x = 0; x < 2; ++x)
                    pb[b][x] = __builtin_bit_cast(bf16x8_t, make_uint4(bf16_pair(p[8 * x], p[8 * x + 1]), bf16_pair(p[8 * x + 2], p[8 * x + 3]),
                                                                       bf16_pair(p[8 * x + 4], p[8 * x + 5]), bf16_pair(p[8 * x + 6], p[8 * x + 7])));
            }
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                    const char* v = stage + v_off[d] + (32 * u + 16 * x) * PITCH;
                    const bf16x8_t vf = lds_tr(v, v + 8 * PITCH);
#pragma unroll
                    for (int b = 0; b < RB; ++b) o[b][d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pb[b][x], o[b][d], 0, 0, 0);
                }
        }
    }
#pragma unroll
    for (int b = 0; b < RB; ++b) {
        const int r = wfirst + 32 * b + col;
        l[b] += __shfl_xor(l[b], 32);
        if (r >= rows) continue;
        const float inv = l[b] > 0.f ? 1.f / l[b] : 0.f;
        uint16_t* dst = g.out + (row0 + r / group) * g.ldo + (int64_t)(kvh * group + r % group) * D + 4 * h;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int e = 0; e < 16; e += 4)
                *(uint2*)(dst + 32 * d + 2 * e) = make_uint2(bf16_pair(o[b][d][e] * inv, o[b][d][e + 1] * inv), bf16_pair(o[b][d][e + 2] * inv, o[b][d][e + 3] * inv));
    }
}

template <int D, bool I8, int RB, int W>
int launch_prompt(aser_ctx* ctx, const AttnArgs& g) {
    constexpr int KEYS = D == 256 ? 32 : 64, BM = 32 * RB * W;
    constexpr size_t lds = 4 * (2 * KEYS * 2 * D) + 4 * W * 4 + (I8 ? 4 * KEYS * 8 : 0);
    const int64_t tiles = ceil_div64(g.p.tokens * g.p.group, BM) + g.p.n_seq;
    if (tiles * g.p.n_kv > INT32_MAX) ASER_FAIL(ctx, ASER_ERR_SHAPE, "paged_attention: too many rows");
    auto kernel = attn_prompt_kernel<D, I8, RB, W>;
    ASER_HIP(ctx, hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
    kernel<<<dim3((unsigned)(tiles * g.p.n_kv)), 64 * W, lds, ctx->stream>>>(g);
    return aser_check_launch(ctx, "attn_prompt_kernel");
}

}  // namespace

int aser_attention_prompt(aser_ctx* ctx, AttnArgs g, int head_dim, int64_t max_rows, float* part, size_t part_bytes) {
    const bool i8 = g.p.k_scale != nullptr;
    (void)max_rows; (void)part; (void)part_bytes;
    if (head_dim == 64) return i8 ? launch_prompt<64, true, 1, 8>(ctx, g) : launch_prompt<64, false, 1, 8>(ctx, g);
    if (head_dim == 128) return i8 ? launch_prompt<128, true, 1, 8>(ctx, g) : launch_prompt<128, false, 1, 8>(ctx, g);
    return i8 ? launch_prompt<256, true, 1, 4>(ctx, g) : launch_prompt<256, false, 1, 4>(ctx, g);
}
