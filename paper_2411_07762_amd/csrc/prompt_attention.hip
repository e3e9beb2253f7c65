// Attention of prompts over the paged cache: the formulas and the transposed products of few_rows.h on tiles that the
// matrix instructions bound instead of memory, 4 D operations per visible key, row and head.
//
// A wavefront owns 32 rows (a row: one query head of one new token; the heads that share a key/value head lie next to each
// other, so a tile spans few positions and little of it is masked) and goes through the keys 32 at a time with
// v_mfma_f32_32x32x16_bf16:  S^T = K Q^T leaves a query row in each column and 16 keys in the registers of a lane, which
// rounded to bf16 are, 8 at a time, the operand of O^T += V^T P^T as they stand (keys 4 h .. and 8 + 4 h .., h = lane / 32).
// A workgroup's four wavefronts share the keys and values through LDS: stages of KEYS keys, copied by global_load_lds_dwordx4, the
// keys of a stage a step before its values, one barrier per stage.  K is read as rows (16 bytes of a key), V through
// ds_read_b64_tr_b16 (four keys of a channel); the chunks of a row are swizzled so that neither meets bank conflicts.  8-bit caches
// go through registers, which widen the codes on their way to LDS; the scales multiply logits and probabilities.
//
// Roundings: probabilities to bf16 for the second product (8 bits; their sum keeps the unrounded ones), results to bf16.
//
// Measured (32 query heads over 8): 8192 tokens of 128 channels 493 to 522 us on different devices, 1.05 to 1.11 PFLOP/s (525 to 562 back to back under a trace); the same
// matrix instructions alone, without loads and softmax, take 362 us: at this length the clock gives way to the power that they draw, 1.7 GHz against 2.2 for 1024
// tokens (28 us), where the length of a step counts: 600 cycles to begin the copies, 1050 for the softmax, 1130 for the products.
// Two prompts of 6001 and 3034 tokens under a window of 1024: 171 to 176 us.  64 channels: 8192 tokens 290 to 307 us, bound by the vector unit: the 32
// exponentials of a step alone take as long as its products (512 cycles each), and the rest of the softmax comes on top.  256 channels (16 heads), 4096 tokens:
// 233 us, one wavefront a SIMD, so that nothing runs beside its softmax.  int8 pays 60 vector instructions a step of 280 for widening: 4096 tokens of 128
// channels 187 us.
#include "few_rows.h"

namespace {

typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef short s16x8_t __attribute__((ext_vector_type(8)));

__device__ __forceinline__ bf16x8_t lds_tr(const char* lo, const char* hi) {
    typedef s16x4_t __attribute__((address_space(3))) * lds_s4p;
    const s16x4_t a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4p)lo);
    const s16x4_t b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4p)hi);
    return __builtin_bit_cast(bf16x8_t, (s16x8_t)__builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

// The u-th row tile of `bm` rows, counted from the last request's last one (later rows see more keys: long tiles start first), and its request: rows
// row0 .. row0 + count - 1, kv keys.  Every lane looks at one request, up to 64 of them once.
struct RowTile {
    int seq = -1, tile = 0, row0 = 0, count = 0, kv = 0;
    __device__ __forceinline__ RowTile(const AttnArgs& g, int u, int bm, int lane) {
        int my_row0, my_count, my_kv, tiles, upto, in_all = 0;
        auto look = [&](int base) {
            my_row0 = my_count = my_kv = tiles = 0;
            if (base + lane < g.p.n_seq) {
                int64_t at;
                my_count = (int)request_rows(g.p, base + lane, &at);
                my_row0 = (int)at;
                my_kv = request_kv_len(g.p, base + lane);
                const int64_t rows = (int64_t)my_count * g.p.group;
                tiles = rows > g.few_rows ? (int)((rows + bm - 1) / bm) : 0;
            }
            const int n = min(g.p.n_seq - base, 64);
            upto = tiles;
            for (int o = 1; o < n; o <<= 1) {
                const int x = __shfl_up(upto, o);
                upto += lane >= o ? x : 0;
            }
            in_all = __builtin_amdgcn_readlane(upto, n - 1);
        };
        auto pick = [&](int base, int t) {         // tile t of these requests
            const int l = __ffsll((unsigned long long)__ballot((upto > t) & (upto - tiles <= t))) - 1;
            seq = base + l;
            tile = t - __builtin_amdgcn_readlane(upto - tiles, l);
            row0 = __builtin_amdgcn_readlane(my_row0, l);
            count = __builtin_amdgcn_readlane(my_count, l);
            kv = __builtin_amdgcn_readlane(my_kv, l);
        };
        if (g.p.n_seq <= 64) {
            look(0);
            if (u < in_all) pick(0, in_all - 1 - u);
            return;
        }
        int total = 0;
        for (int base = 0; base < g.p.n_seq; base += 64) { look(base); total += in_all; }
        int t = total - 1 - u;
        for (int base = 0; t >= 0 && base < g.p.n_seq; base += 64) {
            look(base);
            if (t < in_all) { pick(base, t); return; }
            t -= in_all;
        }
    }
};

constexpr int W = 4;                              // wavefronts of a workgroup
constexpr int kRows = 32 * W;                     // rows of its tile

// Keys of a stage, and slots for stages in LDS: two workgroups of up to 128 channels fit a compute unit, of 256 one does and has more stages on
// their way.  Stages of 32 keys for 128 channels: 8192 tokens 519 -> 539 us, 1024 28 -> 33, 4096 on an int8 cache 188 -> 214, only under the window 172 -> 164;
// four slots for 64 channels: 8192 tokens 307 -> 339.
constexpr int keys_of(int d) { return d == 256 ? 32 : 64; }
constexpr int slots_of(int d) { return d == 256 ? 4 : 2; }

// Stages of each of `splits` parts of a row tile's list.
__device__ __forceinline__ int stages_per_split(int total, int splits) { return max((total + splits - 1) / splits, 1); }

template <int D, bool I8>
__global__ __launch_bounds__(64 * W, D == 256 ? 1 : D == 64 ? 3 : 2) void attn_prompt_kernel(AttnArgs g) {
    constexpr int KEYS = keys_of(D), SUB = KEYS / 32, CH = D / 8, KS = D / 16, DB = D / 32;
    constexpr int PITCH = 2 * D, HALF = KEYS * PITCH, STAGE = 2 * HALF, NST = slots_of(D), AHEAD = NST == 4 || I8 ? 3 : 2, NSC = 8, BM = kRows;
    constexpr int GR = KEYS / W;                  // keys that a wavefront stages, all on one page
    constexpr int LOADS = GR * CH / 64;           // 16-byte loads of a lane for them, of K and of V each
    static_assert(LOADS >= 1, "a wavefront stages at least one load");
    extern __shared__ __align__(16) char smem[];
    int* sm_missing = (int*)(smem + NST * STAGE); // some page of these keys is not there
    float* sm_ks = (float*)(sm_missing + 4);      // int8: [stage % NSC][key] scales of K, then of V
    float* sm_vs = sm_ks + NSC * KEYS;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 31, h = lane >> 5;
    if ((int)blockIdx.x >= g.prompt_all) {         // behind the prompts: the rows of requests that have few
        const int b = blockIdx.x - g.prompt_all, split = g.by_pairs(b);
        few_rows<D, I8, false>(g, b - split * (g.p.n_seq * g.row_tiles * g.p.n_kv), split, *(FewShared<D>*)smem);
        return;
    }
    const int part = g.by_blocks(blockIdx.x), block = blockIdx.x - part * g.prompt_blocks, u = g.by_kv(block), kvh = block - u * g.p.n_kv;
    const RowTile rt(g, u, BM, lane);
    if (rt.seq < 0) return;
    const int s = rt.seq, count = rt.count, kv = rt.kv, rows = count * g.p.group, group = g.p.group;
    const int64_t row0 = rt.row0;
    const int first = rt.tile * BM, base_pos = kv - count;
    const int p_lo = max(base_pos + g.by_group(first), 0), p_hi = base_pos + g.by_group(min(first + BM - 1, rows - 1));
    const int low_all = g.window > 0 ? base_pos + g.by_group(first) - g.window + 1 : 0;
    // stages of the tile, and this workgroup's: t0 .. t0 + t1 - 1, numbered from 0 below
    const KeyTiles<KEYS> kt(p_lo, p_hi, g.window, g.sinks);
    const int per_split = stages_per_split(kt.total, g.prompt_splits), t0 = part * per_split, t1 = min(kt.total - t0, per_split);
    if (t1 <= 0 && part > 0) return;
    auto first_key = [&](int i) -> int { return kt.first_key(t0 + i); };

    // rows of this wavefront
    const int wfirst = first + 32 * wave;
    const bool idle = wfirst >= rows;
    const int wp_lo = base_pos + g.by_group(min(wfirst, rows - 1)), wp_hi = base_pos + g.by_group(min(wfirst + 31, rows - 1));
    const int q_r = min(wfirst + col, rows - 1), q_token = g.by_group(q_r), pos = base_pos + q_token;
    bf16x8_t q[KS];
    const uint32_t flip = g.c < 0.f ? 0x80008000u : 0u;                      // a negative scale turns the queries round
    const float c = fmaxf(fabsf(g.c), 1e-37f);                               // 0: every logit is as good as 0, masked ones stay -inf
    const uint16_t* q_row = g.q + (row0 + q_token) * g.ldq + (int64_t)(kvh * group + q_r - q_token * group) * D + 8 * h;
#pragma unroll
    for (int k = 0; k < KS; ++k) {
        uint4 w = *(const uint4*)(q_row + 16 * k);
        w.x ^= flip; w.y ^= flip; w.z ^= flip; w.w ^= flip;
        q[k] = __builtin_bit_cast(bf16x8_t, w);
    }
    f32x16_t o[DB];
    float m = kNone, l = 0.f;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[d][e] = 0.f;

    // staging: wavefront w has keys GR w .. of a stage; lane: row lane / CH (+ 64 / CH per load), slot lane % CH
    const ScalarInts table = scalar_ints(g.p.pages + s * g.p.ld_pages);
    const int page_mask = (1 << g.p.page_shift) - 1;
    const int64_t head_at = kvh * g.p.head_stride;
    const uint32_t ring = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem + wave * GR * PITCH;
    auto k_swizzle = [](int r) { return D == 64 ? (r >> 1) & 7 : r & 15; };
    auto v_swizzle = [](int r) { return D == 64 ? 4 * ((r >> 1) & 1) : 4 * (r & 3); };
    // Where this wavefront's keys of a stage are, the same for all lanes; page_of(i) is asked for a step before it is needed.
    struct Place { int64_t at; int key, page; bool there, all; };   // elements from the head's first; first key; all: the tile sees every one
    auto page_of = [&](int i) -> int {
        return table[min(first_key(i) + GR * wave, kv - 1) >> g.p.page_shift];                         // kv > 0 where there are stages
    };
    auto place_of = [&](int i, int page) -> Place {
        Place x;
        x.key = first_key(i) + GR * wave;
        x.page = page;
        x.there = (i < t1) & (x.key < kv) & ((uint32_t)page < (uint32_t)g.p.n_pages);
        x.at = (int64_t)(x.there ? page : 0) * g.p.page_stride + (int64_t)((x.key & page_mask) * (uint32_t)g.p.slot_stride);
        x.all = x.there && x.key + GR - 1 <= p_hi && (x.key >= low_all || x.key + GR <= g.sinks);
        return x;
    };
    // what nobody of this tile sees is not looked at
    auto wanted = [&](const Place& x, int r) -> bool { return x.there & (x.key + r <= p_hi) & ((x.key + r >= low_all) | (x.key + r < g.sinks)); };
    uint32_t lane_off[2][LOADS];                   // bytes from a wavefront's first slot to the chunk that a lane copies
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int t = 0; t < LOADS; ++t) {
            const int r = t * (64 / CH) + lane / CH, rr = GR * wave + r;
            lane_off[half][t] = 2 * (r * (uint32_t)g.p.slot_stride + 8 * ((lane % CH) ^ (half ? v_swizzle(rr) : k_swizzle(rr))));
        }
    const char* k_head = (const char*)((const uint16_t*)g.p.k + head_at);
    const char* v_head = (const char*)((const uint16_t*)g.p.v + head_at);
    // bf16: the n-th of 2 LOADS copies of a step, of this wavefront's part of the keys (first LOADS) or values, on its way into slot i % NST.  Lanes
    // whose key nobody of the tile sees copy nothing: such a key's logit does not matter, and its value, whose probability is 0, is set to 0 before.
    struct Part { int64_t at; uint64_t lanes[LOADS]; bool whole, clear; };     // whole: no copy is without lanes; clear: values are to be set to 0
    auto part_of = [&](int i, const Place& x) -> Part {
        Part y;
        y.clear = !x.all && i < t1;
        y.at = 2 * x.at;
        y.whole = true;
#pragma unroll
        for (int t = 0; t < LOADS; ++t) y.lanes[t] = ~0ull;
        if (!x.all) {
#pragma unroll
            for (int t = 0; t < LOADS; ++t) {
                y.lanes[t] = __ballot(wanted(x, t * (64 / CH) + lane / CH));
                y.whole &= y.lanes[t] != 0;
            }
        }
        return y;
    };
    auto copy = [&](int i, const Part& y, int n) {
        const int half = n >= LOADS, t = n % LOADS;
        const char* base = (half ? v_head : k_head) + y.at;
        const uint32_t slot = ring + (i & (NST - 1)) * STAGE + half * HALF + t * 1024;
        asm volatile("s_mov_b32 m0, %0\n\ts_mov_b64 exec, %3\n\tglobal_load_lds_dwordx4 %1, %2\n\ts_mov_b64 exec, -1"
                     : : "s"(slot), "v"(lane_off[half][t]), "s"(base), "s"(y.lanes[t]) : "memory", "m0");
    };
    auto clear_values = [&](int i) {
#pragma unroll
        for (int t = 0; t < LOADS; ++t)
            *(uint4*)(smem + (i & (NST - 1)) * STAGE + HALF + wave * GR * PITCH + t * 1024 + lane * 16) = make_uint4(0u, 0u, 0u, 0u);
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0xC07F);        // lgkmcnt(0): before the copies
        asm volatile("" ::: "memory");
    };
    // int8: codes and scales of the keys of stage i (half 0) or its values (half 1) into registers, and from there, widened, to LDS.  A load is 16
    // codes (two chunks) of a row.
    uint4 held[2][I8 ? LOADS / 2 : 1];
    float held_scale[2] = {0.f, 0.f};
    bool held_there[2] = {false, false};
    uint32_t code_off[I8 ? LOADS / 2 : 1];
#pragma unroll
    for (int t = 0; t < LOADS / 2; ++t) {
        const int z = t * 64 + lane;
        code_off[t] = z / (CH / 2) * (uint32_t)g.p.slot_stride + 16 * (z % (CH / 2));
    }
    auto fetch = [&](const Place& x, int half) {
        // any code is finite: those of keys that nobody sees need no care beside a scale of 0
        const int8_t* src = (half ? (const int8_t*)g.p.v : (const int8_t*)g.p.k) + head_at + x.at;
#pragma unroll
        for (int t = 0; t < LOADS / 2; ++t) held[half][t] = *(const uint4*)(src + code_off[t]);
        const float* scale = (half ? g.p.v_scale : g.p.k_scale) + (((int64_t)(x.there ? x.page : 0) * g.p.n_kv + kvh) << g.p.page_shift) + (x.key & page_mask);
        held_scale[half] = scale[lane & (GR - 1)];
        held_there[half] = wanted(x, lane & (GR - 1));
    };
    auto land = [&](int i, int half) {
        char* dst = smem + (i & (NST - 1)) * STAGE + half * HALF + wave * GR * PITCH;
#pragma unroll
        for (int t = 0; t < LOADS / 2; ++t) {
            const int z = t * 64 + lane, r = z / (CH / 2), ch = 2 * (z % (CH / 2)), rr = GR * wave + r, sw = half ? v_swizzle(rr) : k_swizzle(rr);
            const uint4 w = held[half][t];
            *(uint4*)(dst + r * PITCH + ((ch ^ sw) << 4)) = make_uint4(codes_pair<0>(w.x), codes_pair<2>(w.x), codes_pair<0>(w.y), codes_pair<2>(w.y));
            *(uint4*)(dst + r * PITCH + (((ch + 1) ^ sw) << 4)) = make_uint4(codes_pair<0>(w.z), codes_pair<2>(w.z), codes_pair<0>(w.w), codes_pair<2>(w.w));
        }
        if (lane < GR) (half ? sm_vs : sm_ks)[(i & (NSC - 1)) * KEYS + GR * wave + lane] = held_there[half] ? held_scale[half] : 0.f;
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

    const int mine = idle ? 0 : max(min(kt.count_up_to(wp_hi) - t0, t1), 0);     // stages that this wavefront works on: those behind lie past its rows
    bool missing = false;                          // some page that the tile may look at is not there
    bool far = false;                              // some row's maximum is beyond 2^24
    f32x16_t sc[SUB];                              // logits of a stage, rows and keys as S^T has them
    bf16x8_t pb[SUB][2];                           // its probabilities
    auto logits = [&](int i) {
        const char* stage = smem + (i & (NST - 1)) * STAGE;
#pragma unroll
        for (int u = 0; u < SUB; ++u) {
            bf16x8_t kf[KS];
#pragma unroll
            for (int k = 0; k < KS; ++k) kf[k] = *(const bf16x8_t*)(stage + k_off[k] + u * 32 * PITCH);
#pragma unroll
                for (int e = 0; e < 16; ++e) sc[u][e] = 0.f;
#pragma unroll
            for (int k = 0; k < KS; ++k)
                sc[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[k], q[k], sc[u], 0, 0, 0);
        }
    };
    auto softmax = [&](int i) {
        const int key0 = first_key(i), fl = i & (NSC - 1);
        if constexpr (I8) {
#pragma unroll
            for (int u = 0; u < SUB; ++u)
#pragma unroll
                for (int e4 = 0; e4 < 4; ++e4) {
                    const f32x4_t ks = *(const f32x4_t*)(sm_ks + fl * KEYS + 32 * u + 8 * e4 + 4 * h);
#pragma unroll
                    for (int e = 0; e < 4; ++e) sc[u][4 * e4 + e] *= ks[e];
                }
        }
        const bool plain = !missing && key0 + KEYS - 1 <= wp_lo && (g.window <= 0 || key0 >= wp_hi - g.window + 1 || key0 + KEYS <= g.sinks);
        if (!plain) {
            // a row sees the keys from `low` to `high`, and those below `sink`, counted from this lane's first
            const int first = key0 + 4 * h, sink = g.window > 0 ? g.sinks - first : 0;
            int high = pos - first, low = g.window > 0 ? high - g.window + 1 : INT32_MIN;
            asm volatile("" : "+v"(high), "+v"(low));   // nothing of this rare piece is worth registers outside of it
#pragma unroll
            for (int u = 0; u < SUB; ++u)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int off = 32 * u + 8 * (e >> 2) + (e & 3);
                    const bool seen = (off <= high) & ((off >= low) | (off < sink));
                    sc[u][e] = seen ? sc[u][e] : -INFINITY;
                }
            if (missing) {
                const int key = min(key0 + lane, kv - 1);
                const uint64_t there = __ballot((uint32_t)g.p.pages[s * g.p.ld_pages + (key >> g.p.page_shift)] < (uint32_t)g.p.n_pages) >> (4 * h);
#pragma unroll
                for (int u = 0; u < SUB; ++u)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const bool seen = (there >> (32 * u + 8 * (e >> 2) + (e & 3)) & 1) != 0;
                        sc[u][e] = seen ? sc[u][e] : -INFINITY;
                    }
            }
        }
        float top = sc[0][0];
#pragma unroll
        for (int u = 0; u < SUB; ++u)
#pragma unroll
            for (int e = 0; e < 16; ++e) top = fmaxf(top, sc[u][e]);
        top *= c;
        // the maximum moves only when a logit is 8 above it: until then p <= 2^8, which neither fp32 sums nor bf16 mind
        if (__ballot(top > m + 8.f)) {
            const float m_new = fmaxf(m, fmaxf(top, __shfl_xor(top, 32))), shrink = __builtin_amdgcn_exp2f(m - m_new);
            m = m_new;
            l *= shrink;
#pragma unroll
            for (int d = 0; d < DB; ++d) o[d] *= shrink;
            far = __ballot((fabsf(m) > 0x1p24f) & (m > kNone)) != 0;
        }
        // The maximum has been rounded, the products below are not: up to 2^24 that is a factor of 2 for all keys alike, beyond 2^31 it would take
        // every exponential out of range.  So there the logits are rounded as the maximum is.
        float factor = c;
        if (far) {
#pragma unroll
            for (int u = 0; u < SUB; ++u)
#pragma unroll
                for (int e = 0; e < 16; ++e) sc[u][e] *= c;
            factor = 1.f;
        }
        float sum[2] = {0.f, 0.f};                 // of the unrounded probabilities
#pragma unroll
        for (int u = 0; u < SUB; ++u) {
            uint32_t w[8];
#pragma unroll
            for (int e4 = 0; e4 < 4; ++e4) {
                float p[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) p[e] = __builtin_amdgcn_exp2f(fmaf(sc[u][4 * e4 + e], factor, -m));
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[e & 1] += p[e];
                if constexpr (I8) {
                    const f32x4_t vs = *(const f32x4_t*)(sm_vs + fl * KEYS + 32 * u + 8 * e4 + 4 * h);
#pragma unroll
                    for (int e = 0; e < 4; ++e) p[e] *= vs[e];
                }
                w[2 * e4] = bf16_pair(p[0], p[1]);
                w[2 * e4 + 1] = bf16_pair(p[2], p[3]);
            }
#pragma unroll
            for (int x = 0; x < 2; ++x) pb[u][x] = __builtin_bit_cast(bf16x8_t, make_uint4(w[4 * x], w[4 * x + 1], w[4 * x + 2], w[4 * x + 3]));
        }
        l += sum[0] + sum[1];
        __builtin_amdgcn_sched_barrier(0);         // all of it in this phase
    };
    auto outputs = [&](int i) {
        const char* stage = smem + (i & (NST - 1)) * STAGE;
#pragma unroll
        for (int u = 0; u < SUB; ++u)
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                    const char* v = stage + v_off[d] + (32 * u + 16 * x) * PITCH;
                    const bf16x8_t vf = lds_tr(v, v + 8 * PITCH);
                    o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pb[u][x], o[d], 0, 0, 0);
                }
    };
    // outputs(i) and logits(i + 1) in one piece.  Nothing but the order of instructions hides the latency of the LDS reads here, so it is
    // laid down: behind each instruction the operand of the one four further on is asked for, into the registers that it has read.
    auto products = [&](int i) {
        const char* stage = smem + (i & (NST - 1)) * STAGE;
        const char* next = smem + ((i + 1) & (NST - 1)) * STAGE;
        constexpr int PV = 2 * SUB * DB, ALL = PV + KS * SUB;
        bf16x8_t fr[4];
        auto ask = [&](int n, bf16x8_t& f) {
            if (n < PV) {
                const char* v = stage + v_off[n % DB] + 16 * (n / DB) * PITCH;
                f = lds_tr(v, v + 8 * PITCH);
            } else {
                f = *(const bf16x8_t*)(next + k_off[(n - PV) / SUB] + (n - PV) % SUB * 32 * PITCH);
            }
        };
        auto multiply = [&](int n, const bf16x8_t& f) {
            if (n < PV) {
                o[n % DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, pb[n / DB / 2][n / DB % 2], o[n % DB], 0, 0, 0);
            } else {
                const int k = (n - PV) / SUB, u = (n - PV) % SUB;
                f32x16_t zero = {};
                sc[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, q[k], k ? sc[u] : zero, 0, 0, 0);
            }
        };
#pragma unroll
        for (int n = 0; n < 4; ++n) ask(n, fr[n]);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int n = 0; n < ALL; ++n) {
            multiply(n, fr[n % 4]);
            if (n + 4 < ALL) ask(n + 4, fr[n % 4]);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // Ends a step: waits for this wavefront's LDS accesses and its copies, all or (four slots, `later`) all but those begun in this step, then for the others.
    // later: every copy of this step has lanes, so that the counter has it.
    auto meet = [&](bool later) {
        if (I8) __builtin_amdgcn_s_waitcnt(0xC07F);                                                     // lgkmcnt(0)
        else if (NST == 4 && later) __builtin_amdgcn_s_waitcnt(0x0070 | (2 * LOADS & 15) | ((2 * LOADS >> 4) << 14));
        else __builtin_amdgcn_s_waitcnt(0x0070);
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };

    // What the first steps need from the page table is asked for at once, and whether all pages of the keys that the tile may see are there: those of
    // the sinks, then those from the window's first.
    int pages[AHEAD + 1];
#pragma unroll
    for (int i = 0; i <= AHEAD; ++i) pages[i] = t1 > 0 ? page_of(i) : -1;
    const int last_page = p_hi < 0 ? -1 : min(p_hi, kv - 1) >> g.p.page_shift;
    const int sink_pages = g.window > 0 ? min((min(g.sinks, p_hi + 1) + page_mask) >> g.p.page_shift, last_page + 1) : 0;
    const int skipped = max((max(low_all, 0) >> g.p.page_shift) - sink_pages, 0);
    auto page_word = [&](int x) -> uint32_t {      // 0 behind the last one
        x += x < sink_pages ? 0 : skipped;
        return x <= last_page ? (uint32_t)g.p.pages[s * g.p.ld_pages + x] : 0u;
    };
    const uint32_t my_page = page_word(tid);
    int page_k = pages[AHEAD];
    Place place_v;                                 // int8
    Part part_k, part_v;                           // bf16: copied in this step, of stages i + AHEAD and i + AHEAD - 1
    if constexpr (!I8) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            part_k = part_of(i, place_of(i, pages[i]));
#pragma unroll
            for (int n = 0; n < LOADS; ++n) copy(i, part_k, n);
            if (i > 0) {
                if (part_v.clear) clear_values(i - 1);
#pragma unroll
                for (int n = LOADS; n < 2 * LOADS; ++n) copy(i - 1, part_v, n);
            }
            part_v = part_k;
        }
    } else {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {          // stages past the last come with scales of 0
            const Place x = place_of(i, pages[i]);
            fetch(x, 0);
            if (i > 0) fetch(place_v, 1);
            if (i < 2) land(i, 0);
            if (i == 1) land(0, 1);
            place_v = x;
        }
    }
    missing = my_page >= (uint32_t)g.p.n_pages;
    for (int x = tid + 64 * W; x <= last_page - skipped; x += 64 * W) missing |= page_word(x) >= (uint32_t)g.p.n_pages;
    if (tid == 0) *sm_missing = 0;
    __syncthreads();
    if (missing) *sm_missing = 1;
    meet(false);
    missing = __builtin_amdgcn_readfirstlane(*sm_missing) != 0;
    if (mine > 0) logits(0);
    // Where two slots are all, step 0 writes keys to the slot that this has read: nobody may before everybody has.
    if constexpr (NST == 2) {
        __builtin_amdgcn_s_waitcnt(0xC07F);        // lgkmcnt(0)
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    }
    // Step i: copies of the keys of stage i + AHEAD and the values of the stage before it begun, into slots that were read last in step i - 1;
    // softmax of stage i; products P V of stage i and K Q of stage i + 1; what step i + 1 needs waited for; barrier.  int8: the keys of stage i + 2 and
    // the values of stage i + 1 land, the next ones are fetched.  While one workgroup of the compute unit is at its softmax (vector unit), the other
    // one may be at its products (matrix unit).  One workgroup of eight wavefronts whose halves a second barrier kept half a step apart took 523 us for 8192
    // tokens (without that barrier 571) and 46 for 3 x 200 behind 1500, where this takes 31.
    // Copies spread over the softmax took as long as together before it.
    auto begin = [&](int i) {                      // of a step, before its softmax: copies on their way
        if constexpr (!I8) {
            part_k = part_of(i + AHEAD, place_of(i + AHEAD, page_k));
            if (part_v.clear) clear_values(i + AHEAD - 1);
#pragma unroll
            for (int n = 0; n < 2 * LOADS; ++n) copy(n < LOADS ? i + AHEAD : i + AHEAD - 1, n < LOADS ? part_k : part_v, n);
            page_k = page_of(i + AHEAD + 1);
        }
    };
    auto refill = [&](int i) -> bool {
        if constexpr (!I8) {
            const bool later = part_k.whole && part_v.whole;
            part_v = part_k;
            return later;
        } else {                                   // behind the softmax, which has hidden the loads' latency
            const Place x = place_of(i + AHEAD, page_k);
            page_k = page_of(i + AHEAD + 1);
            land(i + 2, 0);
            land(i + 1, 1);
            fetch(x, 0);
            fetch(place_v, 1);
            place_v = x;
            return false;
        }
    };
    // The last step by itself: where paths meet the compiler moves all accumulators from one set of registers to another.
    int i = 0;
    for (; i < mine - 1; ++i) {
        begin(i);
        softmax(i);
        const bool later = refill(i);
        __builtin_amdgcn_s_setprio(1);
        products(i);
        __builtin_amdgcn_s_setprio(0);
        meet(later);
    }
    if (i < mine) {
        begin(i);
        softmax(i);
        const bool later = refill(i);
        outputs(i);
        meet(later);
        ++i;
    }
    for (; i < t1; ++i) {
        begin(i);
        const bool later = refill(i);
        meet(later);
    }
    const int r = wfirst + col;
    l += __shfl_xor(l, 32);
    if (r >= rows) return;
    if (per_split >= kt.total) {
        const float inv = l > 0.f ? 1.f / l : 0.f;
        const int token = g.by_group(r);
        uint16_t* dst = g.out + (row0 + token) * g.ldo + (int64_t)(kvh * group + r - token * group) * D + 4 * h;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int e = 0; e < 16; e += 4)
                *(uint2*)(dst + 32 * d + 2 * e) = make_uint2(bf16_pair(o[d][e] * inv, o[d][e + 1] * inv), bf16_pair(o[d][e + 2] * inv, o[d][e + 3] * inv));
    } else {
        const int64_t pr = ((int64_t)block * g.prompt_splits + part) * BM + (r - first);
        if (h == 0) g.prompt_ml[pr] = make_float2(m, l);
        float* dst = g.prompt_o + pr * D + 4 * h;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int e = 0; e < 16; e += 4) *(f32x4_t*)(dst + 32 * d + 2 * e) = (f32x4_t){o[d][e], o[d][e + 1], o[d][e + 2], o[d][e + 3]};
    }
}

// Joins the splits of a row tile: o = sum_s w_s o_s / sum_s w_s l_s, w_s = exp2(m_s - max m); four channels of a row per thread.  Behind the prompts'
// workgroups come those of the rows of requests that have few.
template <int D>
constexpr int join_blocks = kRows / (256 / (D / 4));       // of a row tile and head

template <int D>
__global__ __launch_bounds__(256) void attn_prompt_join_kernel(AttnArgs g) {
    constexpr int CL = D / 4, R = 256 / CL, BM = kRows;
    __shared__ FewJoin<D> few;
    if ((int)blockIdx.x >= g.prompt_joins) {
        const int b = blockIdx.x - g.prompt_joins;
        few_join<D>(g, b >> 4, b & 15, few);
        return;
    }
    const int tid = threadIdx.x, block = blockIdx.x / join_blocks<D>, c = tid % CL * 4, in_tile = blockIdx.x % join_blocks<D> * R + tid / CL;
    const int u = g.by_kv(block), kvh = block - u * g.p.n_kv;
    const RowTile rt(g, u, BM, tid & 63);
    if (rt.seq < 0) return;
    const int rows = rt.count * g.p.group, group = g.p.group;
    const int first = rt.tile * BM, base_pos = rt.kv - rt.count, r = first + in_tile;
    const KeyTiles<keys_of(D)> kt(max(base_pos + g.by_group(first), 0), base_pos + g.by_group(min(first + BM - 1, rows - 1)), g.window, g.sinks);
    const int per = stages_per_split(kt.total, g.prompt_splits);
    if (per >= kt.total || r >= rows) return;
    const int used = (kt.total + per - 1) / per;
    const int64_t pr = (int64_t)block * g.prompt_splits * BM + in_tile;
    float top = kNone;
    for (int i = 0; i < used; ++i) top = fmaxf(top, g.prompt_ml[pr + (int64_t)i * BM].x);
    f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
    float l = 0.f;
#pragma unroll 4
    for (int i = 0; i < used; ++i) {
        const float2 ml = g.prompt_ml[pr + (int64_t)i * BM];
        const float w = __builtin_amdgcn_exp2f(ml.x - top);
        l += w * ml.y;
        acc += *(const f32x4_t*)(g.prompt_o + (pr + (int64_t)i * BM) * D + c) * w;
    }
    const float inv = l > 0.f ? 1.f / l : 0.f;
    const int token = g.by_group(r);
    uint16_t* dst = g.out + (rt.row0 + (int64_t)token) * g.ldo + (int64_t)(kvh * group + r - token * group) * D + c;
    *(uint2*)dst = make_uint2(bf16_pair(acc[0] * inv, acc[1] * inv), bf16_pair(acc[2] * inv, acc[3] * inv));
}

// Sizes of a launch.  Two workgroups per compute unit are what the device holds (one with 256 channels); when the row tiles are fewer than half of that, the
// keys are split, 6 stages at least to a workgroup, and the parts joined by a second launch (300 tokens behind 6000: 47 us; split twice as far 61).
// Splits also where the device is full, to even out long and short tiles, cost more than they gave but on 8-bit caches of 64 channels: 3000 tokens
// 85 -> 108 us, 2048 53 -> 60, ragged int8 pieces 94 -> 81.
struct PromptPlan { int64_t tiles; int splits; size_t o_bytes, bytes; };

PromptPlan plan_prompt(int64_t tokens, int64_t n_seq, int64_t n_kv, int64_t group, int head_dim, int64_t keys) {
    PromptPlan p;
    p.tiles = ceil_div64(tokens * group, kRows) + n_seq;
    const int64_t stages = keys / keys_of(head_dim) + 2, full = head_dim == 256 ? 256 : 512;
    int64_t splits = full / (p.tiles * n_kv);
    if (splits > stages / 6) splits = stages / 6;
    if (splits < 1) splits = 1;
    p.splits = (int)splits;
    const size_t rows = splits > 1 ? (size_t)(p.tiles * n_kv) * p.splits * kRows : 0;
    p.o_bytes = align_up(rows * head_dim * 4, 256);
    p.bytes = p.o_bytes + align_up(rows * 8, 256);
    return p;
}

template <int D, bool I8>
int launch_prompt(aser_ctx* ctx, AttnArgs& g, const PromptPlan& p) {
    constexpr int KEYS = keys_of(D);
    constexpr size_t lds = slots_of(D) * (2 * KEYS * 2 * D) + 16 + (I8 ? 8 * KEYS * 8 : 0);
    static_assert(sizeof(FewShared<D>) <= lds, "the few rows' sums lie where the stages do");
    const int64_t blocks = p.tiles * g.p.n_kv, pairs = (int64_t)g.p.n_seq * g.row_tiles * g.p.n_kv;
    const int64_t all = blocks * p.splits + (g.few_rows > 0 ? pairs * g.splits : 0);
    if (all > INT32_MAX) ASER_FAIL(ctx, ASER_ERR_SHAPE, "paged_attention: too many rows");
    g.prompt_blocks = (int)blocks;
    g.prompt_all = (int)(blocks * p.splits);
    g.by_blocks = Divider::by((uint32_t)blocks);
    g.by_pairs = Divider::by((uint32_t)pairs);
    auto kernel = attn_prompt_kernel<D, I8>;
    ASER_HIP(ctx, hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
    kernel<<<(unsigned)all, 64 * W, lds, ctx->stream>>>(g);
    ASER_TRY(aser_check_launch(ctx, "attn_prompt_kernel"));
    const int64_t joins = p.splits > 1 ? blocks * join_blocks<D> : 0, few = g.few_rows > 0 && g.splits > 1 ? pairs * 16 : 0;
    if (joins + few == 0) return ASER_OK;
    if (joins + few > INT32_MAX) ASER_FAIL(ctx, ASER_ERR_SHAPE, "paged_attention: too many rows");
    g.prompt_joins = (int)joins;
    attn_prompt_join_kernel<D><<<(unsigned)(joins + few), 256, 0, ctx->stream>>>(g);
    return aser_check_launch(ctx, "attn_prompt_join_kernel");
}

}  // namespace

size_t aser_attention_prompt_workspace(int64_t tokens, int64_t n_seq, int64_t n_kv, int64_t group, int head_dim, int64_t keys) {
    return plan_prompt(tokens, n_seq, n_kv, group, head_dim, keys).bytes;
}

int aser_attention_prompt(aser_ctx* ctx, AttnArgs g, int head_dim, int64_t keys, size_t ws_at) {
    const bool i8 = g.p.k_scale != nullptr;
    const PromptPlan p = plan_prompt(g.p.tokens, g.p.n_seq, g.p.n_kv, g.p.group, head_dim, keys);
    g.prompt_splits = p.splits;
    g.prompt_o = (float*)((char*)ctx->ws + ws_at);
    g.prompt_ml = (float2*)((char*)ctx->ws + ws_at + p.o_bytes);
    if (head_dim == 64) return i8 ? launch_prompt<64, true>(ctx, g, p) : launch_prompt<64, false>(ctx, g, p);
    if (head_dim == 128) return i8 ? launch_prompt<128, true>(ctx, g, p) : launch_prompt<128, false>(ctx, g, p);
    return i8 ? launch_prompt<256, true>(ctx, g, p) : launch_prompt<256, false>(ctx, g, p);
}
