// Attention of new tokens over a paged cache:
//     o = sum_j p_j v_j / sum_j p_j,   p_j = exp2(c (q . k_j) - m),   c = scale log2 e,
// in one pass over the keys with a running maximum m and running sums.  Query heads that share a key/value head are rows of
// the same tile (row = new token * group + head of the group), so a key is read once for all of them.
//
// Few rows (a wavefront per 16 rows, this file; prompts: prompt_attention.hip).  The products are formed transposed: S^T = K Q^T has a query row per
// column of the 16 x 16 accumulator, four keys in the registers of a lane; two such tiles are, as they stand, the operand of
// the next product O^T = V^T P^T (8 keys per lane, in the order 4 g .. 4 g + 3 of the first 16 keys, then of the second 16;
// g = lane / 16).  The sum over keys does not care for their order, so the values are simply fetched in that order and no
// probability changes lanes.  V^T wants 8 keys of one channel in a lane where memory has 8 channels of one key: a lane loads
// D / 16 channels of its 8 keys and a byte permute per pair of keys turns them round.
// Bound by reading the cache: 4 D bytes per key and head against 64 D / 16 matrix operations of 16 columns.  The keys of a request are cut
// into parts for different workgroups, whose results a second launch joins: a single request would otherwise keep a workgroup per
// key/value head busy and no more.  Probabilities enter the second product as two bf16 terms (16 bits; one term puts an error of up to 2^-8
// where the results' own rounding is 2^-8 too, and the second costs nothing beside the loads).
// Measured: 64 requests of 1600 to 8192 tokens, 128 channels, 32 query heads over 8: 214 us, 6.0 TB/s (a plain read reaches 6.65); one request of
// 32771 tokens 23 us + 4.5 to join; 40 requests of up to 12003 on an int8 cache of 64 channels 64 us, 5.1 TB/s, where widening the codes counts too;
// 16 requests with 4 new tokens each, 32 heads over 32, under a window of 2048 with 4 sinks 86 us, 6.3 TB/s.
#pragma once
#include "attention.h"

constexpr int kTile = 32;                         // keys of a step
constexpr int kMaxSplits = 256;                   // parts of a request's keys: a thread of the join for each

// Loads N words; ONCE: and says that nobody reads them again.
template <int N, bool ONCE>
__device__ __forceinline__ void load_words(const char* p, uint32_t* w) {
    typedef uint32_t words_t __attribute__((ext_vector_type(N)));
    words_t v;
    if constexpr (ONCE) v = __builtin_nontemporal_load((const words_t*)p);
    else v = *(const words_t*)p;
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = v[i];
}

template <int D>
struct FewShared { float o[4][16][D + 4], m[4][16], l[4][16]; };

// One of a request's tiles of 16 rows and part `split` of its keys; block: (request, row tile, key/value head).  ONCE: no other row tile reads these keys.
template <int D, bool I8, bool ONCE>
__device__ __forceinline__ void few_rows(const AttnArgs& g, int block, int split, FewShared<D>& sm) {
    constexpr int KS = D / 32;                    // steps of 32 channels in K Q^T
    constexpr int NB = D / 16;                    // channels of a lane in V^T, and accumulators of O^T
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, grp = lane >> 4;
    const int tile = g.by_kv(block), kvh = block - tile * g.p.n_kv;
    const FewTile ft(g, tile);
    const int s = ft.seq, rt = ft.row_tile;
    int64_t row0;
    const int count = (int)request_rows(g.p, s, &row0), kv = request_kv_len(g.p, s);
    const int rows = count * g.p.group - rt * 16;                            // rows of this tile, if positive
    if (rows <= 0 || count * g.p.group > g.few_rows) return;
    const int my_row = min(rt * 16 + n, count * g.p.group - 1), my_tok = g.by_group(my_row), my_head = my_row - my_tok * g.p.group;
    const int my_pos = kv - count + my_tok;
    const int last_row = min(rt * 16 + 15, count * g.p.group - 1);
    const int p_lo = max(kv - count + g.by_group(rt * 16), 0), p_hi = kv - count + g.by_group(last_row);
    const KeyTiles<kTile> kt(p_lo, p_hi, g.window, g.sinks);
    const int t0 = split * g.tiles_per_split, t1 = min(t0 + g.tiles_per_split, kt.total);
    if (t0 >= t1 && split > 0) return;
    const int low_all = g.window > 0 ? kv - count + g.by_group(rt * 16) - g.window + 1 : 0;   // the same for the tile's first row
    const int my_low = g.window > 0 ? my_pos - g.window + 1 : 0;             // keys below are seen up to sinks only

    // the row's query: B operand of K Q^T, channels 32 step + 8 grp ..; int8: 64 (step / 2) + 16 grp + 8 (step % 2) .., so that a load is 16 codes
    bf16x8_t q[KS];
    const int64_t q_at = (row0 + my_tok) * g.ldq + (int64_t)(kvh * g.p.group + my_head) * D;
#pragma unroll
    for (int k = 0; k < KS; ++k) q[k] = __builtin_bit_cast(bf16x8_t, *(const uint4*)(g.q + q_at + (I8 ? 64 * (k / 2) + 16 * grp + 8 * (k % 2) : 32 * k + 8 * grp)));

    f32x4_t o[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) o[b] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
    float m = kNone, l = 0.f;
    const ScalarInts table = scalar_ints(g.p.pages + s * g.p.ld_pages);
    const int page_mask = (1 << g.p.page_shift) - 1;
    // a lane's offsets in bytes inside 16 slots; everything else of an address is the same for the wavefront
    constexpr int ES = I8 ? 1 : 2, KL = I8 ? D / 64 : KS;                    // bytes of an element; 16-byte loads of K for 16 keys
    constexpr int VW = I8 ? NB / 4 : NB / 2;                                 // words of a lane's channels of a key
    constexpr int VK = I8 && D < 256 ? 256 / D : 1;                          // int8: keys that 16 lanes cover with 16-byte loads of V
    const uint32_t pitch = (uint32_t)g.p.slot_stride * ES;
    const uint32_t k_off = n * pitch + 16 * grp;
    const uint32_t v_off = VK > 1 ? (4 * grp + n / (16 / VK)) * pitch + 16 * (n % (16 / VK)) : 4 * grp * pitch + NB * n * ES;
    const int64_t page_bytes = g.p.page_stride * ES;
    const char* k_head = (const char*)g.p.k + kvh * g.p.head_stride * ES;
    const char* v_head = (const char*)g.p.v + kvh * g.p.head_stride * ES;

    // A step's keys and values.  Enough of them are on their way because 16 wavefronts of a compute unit do this; fetching a step ahead instead
    // takes the registers of half of those and was slower (int8, 64 channels: 80 -> 97 us).
    struct Step {
        uint32_t kw[2][KL][4], vw[8 * VW];            // of key e (0 .. 3 of the first 16, then of the second): vw[VW e ..]
        float ks[I8 ? 8 : 1], vs[I8 ? 8 : 1];
        int key0;
        bool there[2];
    };
    auto page_at = [&](int i, int h) -> int {
        const int k0 = kt.first_key(min(i, t1 - 1)) + 16 * h;
        return k0 < kv ? table[k0 >> g.p.page_shift] : -1;                   // the table has columns for kv tokens only
    };
    int page_next[2] = {-1, -1};                                             // asked for a step ahead of the fetch that needs them
    auto fetch = [&](Step& f, int i) {
        f.key0 = kt.first_key(i);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int k0 = f.key0 + 16 * h;
            f.there[h] = (uint32_t)page_next[h] < (uint32_t)g.p.n_pages;
            const int page = f.there[h] ? page_next[h] : 0;
            const int64_t at = page * page_bytes + (int64_t)(k0 & page_mask) * pitch;
            // in scalar registers as they stand: the loads then add the lane's offset themselves
            const char *k_at = k_head + at, *v_at = v_head + at, *v_next;
            asm volatile("" : "+s"(k_at), "+s"(v_at));
            // keys: A operand, row n
#pragma unroll
            for (int k = 0; k < KL; ++k) load_words<4, ONCE>(k_at + k_off + 64 * k, f.kw[h][k]);
            // values: the lane's channels of keys 4 grp + e; int8 of fewer than 256 channels: 16 codes of every VK-th key, see regroup()
#pragma unroll
            for (int e = 0; e < 4; e += VK, v_at = v_next) {
                v_next = v_at + VK * pitch;
                asm volatile("" : "+s"(v_next));
                if constexpr (VK > 1) {
                    load_words<4, ONCE>(v_at + v_off, f.vw + (4 * h + e) * VW);
                } else {
#pragma unroll
                    for (int x = 0; x < VW; x += 4) load_words<(VW < 4 ? VW : 4), ONCE>(v_at + v_off + 4 * x, f.vw + (4 * h + e) * VW + x);
                }
            }
            if constexpr (I8) {
                const int64_t sc = (((int64_t)page * g.p.n_kv + kvh) << g.p.page_shift) + (k0 & page_mask) + 4 * grp;
                const float4 a = *(const float4*)(g.p.k_scale + sc), b = *(const float4*)(g.p.v_scale + sc);
                f.ks[4 * h] = a.x; f.ks[4 * h + 1] = a.y; f.ks[4 * h + 2] = a.z; f.ks[4 * h + 3] = a.w;
                f.vs[4 * h] = b.x; f.vs[4 * h + 1] = b.y; f.vs[4 * h + 2] = b.z; f.vs[4 * h + 3] = b.w;
            }
        }
        page_next[0] = page_at(i + 4, 0);
        page_next[1] = page_at(i + 4, 1);
    };
    // int8 of 64 or 128 channels: 16 lanes have loaded VK keys together, lane n 16 codes of key n / (16 / VK).  The VK lanes with the same codes'
    // places turn that round, so that each has 16 / VK of the codes of all VK keys: its own keys' words stay in order.
    auto regroup = [&](Step& f) {
        if constexpr (VK > 1) {
#pragma unroll
            for (int x = 0; x < 8; x += VK) {
                uint32_t* v = f.vw + x * VW;
                const uint32_t w0 = v[0], w1 = v[1], w2 = v[2], w3 = v[3];
                const bool odd = n & 4, high = n & 8;
                if constexpr (VK == 4) {           // a 4 x 4 transpose over lanes n, n ^ 4, n ^ 8, n ^ 12
                    const uint32_t a0 = __builtin_amdgcn_ds_swizzle(odd ? w0 : w1, 0x101F), a1 = __builtin_amdgcn_ds_swizzle(odd ? w2 : w3, 0x101F);
                    const uint32_t b0 = odd ? a0 : w0, b1 = odd ? w1 : a0, b2 = odd ? a1 : w2, b3 = odd ? w3 : a1;
                    const uint32_t c0 = __builtin_amdgcn_ds_swizzle(high ? b0 : b2, 0x201F), c1 = __builtin_amdgcn_ds_swizzle(high ? b1 : b3, 0x201F);
                    v[0] = high ? c0 : b0;
                    v[1] = high ? c1 : b1;
                    v[2] = high ? b2 : c0;
                    v[3] = high ? b3 : c1;
                } else {                           // pairs of words between lanes n and n ^ 8
                    const uint32_t a0 = __builtin_amdgcn_ds_swizzle(high ? w0 : w2, 0x201F), a1 = __builtin_amdgcn_ds_swizzle(high ? w1 : w3, 0x201F);
                    v[0] = high ? a0 : w0;
                    v[1] = high ? a1 : w1;
                    v[2] = high ? w2 : a0;
                    v[3] = high ? w3 : a1;
                }
            }
        }
    };
    auto use = [&](Step& f) {
        regroup(f);
        const int key0 = f.key0;
        f32x4_t st[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            st[h] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                const uint32_t* x = I8 ? f.kw[h][k / 2] + 2 * (k % 2) : f.kw[h][k];
                uint4 w;
                if constexpr (I8) w = make_uint4(codes_pair<0>(x[0]), codes_pair<2>(x[0]), codes_pair<0>(x[1]), codes_pair<2>(x[1]));
                else w = make_uint4(x[0], x[1], x[2], x[3]);
                st[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, w), q[k], st[h], 0, 0, 0);
            }
        }
        // logits in units of log2, masked to -inf
        float x[8];
        const bool plain = key0 + kTile <= p_lo + 1 && f.there[0] && f.there[1] && (g.window <= 0 || key0 >= p_hi - g.window + 1 || key0 + kTile <= g.sinks);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = st[e >> 2][e & 3] * (I8 ? g.c * f.ks[e] : g.c);
        if (!plain) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int h = e >> 2, key = key0 + 16 * h + 4 * grp + (e & 3);
                // one comparison after the other, no branches: this compiler has lost the first of several masked values in branches
                const bool seen = f.there[h] & (key <= my_pos) & ((key >= my_low) | (key < g.sinks));
                x[e] = seen ? x[e] : -INFINITY;
                // what nobody of this tile sees does not count, whatever the slot holds
                const bool used = f.there[h] & (key <= p_hi) & ((key >= low_all) | (key < g.sinks));
                if (I8) f.vs[e] = used ? f.vs[e] : 0.f;
#pragma unroll
                for (int w = 0; w < VW; ++w) f.vw[e * VW + w] = used ? f.vw[e * VW + w] : 0u;
            }
        }
        float top = x[0];
#pragma unroll
        for (int e = 1; e < 8; ++e) top = fmaxf(top, x[e]);
        // The maximum moves only when a logit is 8 above it: until then p <= 2^8, which neither fp32 sums nor bf16 mind.
        if (__ballot(top > m + 8.f)) {
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float m_new = fmaxf(m, top), r = __builtin_amdgcn_exp2f(m - m_new);
            m = m_new;
            l *= r;
#pragma unroll
            for (int b = 0; b < NB; ++b) o[b] *= r;
        }
        float p[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            p[e] = __builtin_amdgcn_exp2f(x[e] - m);
            l += p[e];
            if (I8) p[e] *= f.vs[e];
        }
        // two bf16 terms, 2^-16 together: the second product is far from bounding this kernel
        const uint4 p1 = make_uint4(bf16_pair(p[0], p[1]), bf16_pair(p[2], p[3]), bf16_pair(p[4], p[5]), bf16_pair(p[6], p[7]));
        const uint32_t pw[4] = {p1.x, p1.y, p1.z, p1.w};
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] -= __uint_as_float(e & 1 ? pw[e >> 1] & 0xFFFF0000u : pw[e >> 1] << 16);
        const bf16x8_t pb = __builtin_bit_cast(bf16x8_t, p1);
        const bf16x8_t pr = __builtin_bit_cast(bf16x8_t, make_uint4(bf16_pair(p[0], p[1]), bf16_pair(p[2], p[3]), bf16_pair(p[4], p[5]), bf16_pair(p[6], p[7])));
#pragma unroll
        for (int w = 0; w < NB / 2; ++w) {                                    // channels 2 w and 2 w + 1 of the lane
            uint32_t v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = I8 ? ((w & 1) ? codes_pair<2>(f.vw[e * VW + w / 2]) : codes_pair<0>(f.vw[e * VW + w / 2])) : f.vw[e * VW + w];
            uint4 even, odd;
            even = make_uint4(__builtin_amdgcn_perm(v[1], v[0], 0x05040100u), __builtin_amdgcn_perm(v[3], v[2], 0x05040100u),
                              __builtin_amdgcn_perm(v[5], v[4], 0x05040100u), __builtin_amdgcn_perm(v[7], v[6], 0x05040100u));
            odd = make_uint4(__builtin_amdgcn_perm(v[1], v[0], 0x07060302u), __builtin_amdgcn_perm(v[3], v[2], 0x07060302u),
                             __builtin_amdgcn_perm(v[5], v[4], 0x07060302u), __builtin_amdgcn_perm(v[7], v[6], 0x07060302u));
            o[2 * w] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, even), pr, o[2 * w], 0, 0, 0);
            o[2 * w + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, odd), pr, o[2 * w + 1], 0, 0, 0);
            o[2 * w] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, even), pb, o[2 * w], 0, 0, 0);
            o[2 * w + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, odd), pb, o[2 * w + 1], 0, 0, 0);
        }
    };
    const int mine = t1 > t0 + wave ? (t1 - t0 - wave + 3) / 4 : 0, i0 = t0 + wave;      // steps of this wavefront: i0, i0 + 4, ..
    if (mine > 0) {
        Step f;
        page_next[0] = page_at(i0, 0);
        page_next[1] = page_at(i0, 1);
        for (int j = 0; j < mine; ++j) {
            fetch(f, i0 + 4 * j);
            use(f);
        }
    }

    // the four wavefronts' results meet: row n, of lane x = 4 grp + e of V^T the channels from first(x) on
    auto first = [](int x) { return VK > 1 ? 16 * (x % (16 / VK)) + NB * (x / (16 / VK)) : NB * x; };
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (lane < 16) { sm.m[wave][n] = m; sm.l[wave][n] = l; }
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int b = 0; b < NB; b += 4)
            *(f32x4_t*)&sm.o[wave][n][first(4 * grp + e) + b] = (f32x4_t){o[b][e], o[b + 1][e], o[b + 2][e], o[b + 3][e]};
    __syncthreads();
    constexpr int PER = D / 16;                                              // channels of a thread: 16 threads per row
    const int r = tid >> 4, ch = (tid & 15) * PER;
    if (r >= rows) return;
    float mm = sm.m[0][r];
#pragma unroll
    for (int w = 1; w < 4; ++w) mm = fmaxf(mm, sm.m[w][r]);
    float ll = 0.f, acc[PER];
#pragma unroll
    for (int c = 0; c < PER; ++c) acc[c] = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const float f = __builtin_amdgcn_exp2f(sm.m[w][r] - mm);
        ll += sm.l[w][r] * f;
#pragma unroll
        for (int c = 0; c < PER; ++c) acc[c] += sm.o[w][r][ch + c] * f;
    }
    const int used = g.by_split(kt.total + g.tiles_per_split - 1);  // splits that have keys
    if (used <= 1) {
        const float inv = ll > 0.f ? 1.f / ll : 0.f;
        const int row = rt * 16 + r;
        const int token = g.by_group(row);
        uint16_t* dst = g.out + (row0 + token) * g.ldo + (int64_t)(kvh * g.p.group + row - token * g.p.group) * D + ch;
#pragma unroll
        for (int c = 0; c < PER; c += 4) *(uint2*)(dst + c) = make_uint2(bf16_pair(acc[c] * inv, acc[c + 1] * inv), bf16_pair(acc[c + 2] * inv, acc[c + 3] * inv));
    } else {
        const int64_t pr = ((int64_t)block * g.splits + split) * 16 + r;
        if ((tid & 15) == 0) g.part_ml[pr] = make_float2(mm, ll);
#pragma unroll
        for (int c = 0; c < PER; c += 4) *(f32x4_t*)(g.part_o + pr * D + ch + c) = (f32x4_t){acc[c], acc[c + 1], acc[c + 2], acc[c + 3]};
    }
}

// Joins the splits of one row: o = sum_s w_s o_s / sum_s w_s l_s, w_s = exp2(m_s - max m).  The maxima are asked for before the
// request's length says how many of them there are: one wait less in a kernel that is nothing but waits.
template <int D>
struct FewJoin { f32x4_t sm[1024 / D][D / 4]; float w[kMaxSplits], m[4], l[4]; };

// block: as in few_rows; r: row of the tile
template <int D>
__device__ __forceinline__ void few_join(const AttnArgs& g, int block, int r, FewJoin<D>& x) {
    constexpr int CL = D / 4, SL = 256 / CL;      // lanes over channels (4 each), splits side by side
    const int tid = threadIdx.x, cl = tid % CL, sl = tid / CL;
    const int tile = g.by_kv(block), kvh = block - tile * g.p.n_kv;
    const FewTile ft(g, tile);
    const int s = ft.seq, rt = ft.row_tile;
    const int64_t pr = (int64_t)block * g.splits * 16 + r;
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
    if ((tid & 63) == 0) x.m[tid >> 6] = top;
    __syncthreads();
    top = fmaxf(fmaxf(x.m[0], x.m[1]), fmaxf(x.m[2], x.m[3]));
    const float w = tid < used ? __builtin_amdgcn_exp2f(ml.x - top) : 0.f;
    float ll = w * ml.y;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) ll += __shfl_xor(ll, o);
    if ((tid & 63) == 0) x.l[tid >> 6] = ll;
    x.w[tid] = w;
    __syncthreads();
    f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int i = sl; i < used; i += SL) acc += *(const f32x4_t*)(g.part_o + (pr + (int64_t)i * 16) * D + 4 * cl) * x.w[i];
    x.sm[sl][cl] = acc;
    __syncthreads();
    if (sl) return;
#pragma unroll
    for (int i = 1; i < SL; ++i) acc += x.sm[i][cl];
    ll = (x.l[0] + x.l[1]) + (x.l[2] + x.l[3]);
    const float inv = ll > 0.f ? 1.f / ll : 0.f;
    const int token = g.by_group(row);
    uint16_t* dst = g.out + (row0 + token) * g.ldo + (int64_t)(kvh * g.p.group + row - token * g.p.group) * D + 4 * cl;
    *(uint2*)dst = make_uint2(bf16_pair(acc[0] * inv, acc[1] * inv), bf16_pair(acc[2] * inv, acc[3] * inv));
}
