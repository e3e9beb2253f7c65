// Routing of rows to experts, and the weighted sum of what the experts made of them.
//
// Routing: a wavefront or 16 of its lanes have a row, lane i the experts i, i + 64 (16), ...  Scores are computed in 64 bits, so that experts are told apart where fp32 would
// round their scores to one number.  The top_k largest are found one after the other, by the upper halves of keys of 64 bits that order as the numbers do; only where lanes
// agree in them the lower halves are looked at.  A workgroup has 32 rows: bit t of an expert's word says that row t chose it,
// so the number of a pair among its expert's pairs is a count of bits, and the order by expert is the same whatever the timing.  Up
// to 32 rows are ordered in the same launch; more in two further ones, a running sum over the workgroups for each expert and the placing.
#include "bf16_pair.h"
#include "mx4.h"

namespace {

constexpr int kTok = 32, kWaves = 16;         // rows of a workgroup, its wavefronts
constexpr double kMinus = -__builtin_huge_val();

struct RouteArgs {
    const void* logits; int64_t ldl;
    const float* bias;
    aser_route_opts o;
    int32_t* ids; float* weights; int32_t* offsets; int32_t* order; int32_t* place;
    int64_t rows;
    int top_k, experts;
    int32_t* counts;      // [expert][workgroup]; more than one workgroup
    int32_t* totals;      // [expert]
    int groups;           // workgroups
    int per_bits;         // 2^per_bits lanes look at a group of experts
    float per_expert;     // 1 / experts of a group
};

// Steps of a reduction over a wavefront by the data-parallel moves: after the six of them lane 63 has the result of all.  Lanes that a move does not reach get `idle`.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t moved(uint32_t v, uint32_t idle) { return (uint32_t)__builtin_amdgcn_update_dpp((int)idle, (int)v, CTRL, ROWS, 15, false); }
template <class F>
__device__ __forceinline__ uint32_t wave_reduce(uint32_t v, uint32_t idle, F join) {
    v = join(v, moved<0x111, 15>(v, idle));       // from 1, 2, 4, 8 lanes below within a row of 16, then from the rows before
    v = join(v, moved<0x112, 15>(v, idle));
    v = join(v, moved<0x114, 15>(v, idle));
    v = join(v, moved<0x118, 15>(v, idle));
    v = join(v, moved<0x142, 10>(v, idle));
    v = join(v, moved<0x143, 12>(v, idle));
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) { return wave_reduce(v, 0u, [](uint32_t a, uint32_t b) { return a > b ? a : b; }); }
template <int CTRL, int ROWS>
__device__ __forceinline__ double moved(double v) {                 // 0 where no lane is reached
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint64_t lo = moved<CTRL, ROWS>((uint32_t)b, 0u), hi = moved<CTRL, ROWS>((uint32_t)(b >> 32), 0u);
    return __builtin_bit_cast(double, lo | hi << 32);
}
__device__ __forceinline__ double lane_value(double v, int lane) {
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint64_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)b, lane), hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), lane);
    return __builtin_bit_cast(double, lo | hi << 32);
}
__device__ __forceinline__ double wave_sum(double v) {
    v += moved<0x111, 15>(v);
    v += moved<0x112, 15>(v);
    v += moved<0x114, 15>(v);
    v += moved<0x118, 15>(v);
    v += moved<0x142, 10>(v);
    v += moved<0x143, 12>(v);
    return lane_value(v, 63);
}
// Numbers of 64 bits as whole numbers in the same order; no number that is not -inf or NaN has a key below 2^52.
__device__ __forceinline__ uint64_t key_of(double v) {
    const uint64_t b = __builtin_bit_cast(uint64_t, v + 0.0);       // one zero
    return b >> 63 ? ~b : b | (uint64_t)1 << 63;
}

// x[j] <= 0 to exp(x[j]) in 64 bits, -746 and less (and NaN) to 0: x = k ln 2 + r, |r| <= ln 2 / 2, and the Taylor series of exp(r) to r^13 / 13!, whose rest is below 2^-57 of it.  All
// numbers of a lane at once, so that the constants are there once; half the instructions of the library's function, which a third of the routing's time went into.
template <int V>
__device__ __forceinline__ void exp64(double* x) {
    constexpr double kOver[12] = {1.0 / 479001600.0, 1.0 / 39916800.0, 1.0 / 3628800.0, 1.0 / 362880.0, 1.0 / 40320.0, 1.0 / 5040.0,
                                  1.0 / 720.0,       1.0 / 120.0,      1.0 / 24.0,      1.0 / 6.0,      0.5,           1.0};
    double k[V], r[V], p[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const double v = fmax(x[j], -746.0);
        k[j] = rint(v * 1.4426950408889634);
        r[j] = fma(-k[j], 2.3190468138462996e-17, fma(-k[j], 0.6931471805599453, v));      // ln 2 as the nearest number of 64 bits and what it leaves
        p[j] = 1.0 / 6227020800.0;
    }
#pragma unroll
    for (int i = 0; i < 12; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) p[j] = fma(p[j], r[j], kOver[i]);
#pragma unroll
    for (int j = 0; j < V; ++j) x[j] = __builtin_amdgcn_ldexp(fma(p[j], r[j], 1.0), (int)k[j]);
}
// 1 / x for x in [1, 1024]: the instruction's approximation and two steps of Newton's method.
__device__ __forceinline__ double reciprocal64(double x) {
    double y = __builtin_amdgcn_rcp(x);
    y = fma(fma(-x, y, 1.0), y, y);
    return fma(fma(-x, y, 1.0), y, y);
}
// The sigmoid 1 / (1 + exp(-l)) from t = exp(-|l|): 1 / (1 + t), below zero t / (1 + t), which has its own value down to the smallest numbers.  0 where exp(-l) is
// above the largest number of 64 bits, exp(709.7827...), as the definition evaluated in 64 bits is.
__device__ __forceinline__ double sigmoid64(float l, double t) {
    const double s = (l < 0.f ? t : 1.0) * reciprocal64(1.0 + t);
    return (double)l < -709.782712893384 ? 0.0 : s;
}

// Running sum over the experts: offs[e] = sum of count(e') for e' < e, offs[experts] the total.  One wavefront.
template <class COUNT>
__device__ __forceinline__ void sum_experts(int experts, int32_t* offs, COUNT count) {
    const int lane = threadIdx.x & 63;
    int32_t before = 0;
    for (int e0 = 0; e0 < experts; e0 += 64) {
        const int32_t mine = e0 + lane < experts ? count(e0 + lane) : 0;
        const int32_t upto = (int32_t)mx4_sums_upto((uint32_t)mine);
        if (e0 + lane < experts) offs[e0 + lane] = before + upto - mine;
        before += __builtin_amdgcn_readlane(upto, 63);
    }
    if (lane == 0) offs[experts] = before;
}

// Places the pairs of 32 rows: marks[e] has the rows that chose e, first[e] the position of the first of them.
__device__ __forceinline__ void place_pairs(const RouteArgs& g, int64_t row0, const uint32_t* marks, const int32_t* first, int32_t total) {
    const int64_t left = (g.rows - row0) * g.top_k, pairs = g.rows * g.top_k;
    const int here = left < kTok * g.top_k ? (int)left : kTok * g.top_k;
    for (int i = threadIdx.x; i < here; i += kWaves * 64) {
        const int64_t pair = row0 * g.top_k + i;
        const int32_t e = g.ids[pair];
        const int t = i / g.top_k;
        int32_t at = -1;
        if (e >= 0) {
            at = first[e] + __popc(marks[e] & ((1u << t) - 1u));
            g.order[at] = (int32_t)pair;
        }
        g.place[pair] = at;
        if (pair >= total && pair < pairs) g.order[pair] = -1;
    }
}

template <int V, bool F32>
__global__ __launch_bounds__(kWaves * 64) void route_kernel(RouteArgs g) {
    extern __shared__ __align__(16) char smem[];
    double* const cbuf = (double*)smem;                                     // [wavefront][expert], if there are groups
    uint32_t* const marks = (uint32_t*)(smem + (g.o.n_groups > 1 ? (size_t)kWaves * g.experts * 8 : 0));
    int32_t* const first = (int32_t*)(marks + g.experts);                   // experts + 1
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t row0 = (int64_t)blockIdx.x * kTok;
    float bias[V];
#pragma unroll
    for (int j = 0; j < V; ++j) bias[j] = g.bias && lane + 64 * j < g.experts ? g.bias[lane + 64 * j] : 0.f;
    for (int e = threadIdx.x; e < g.experts; e += kWaves * 64) marks[e] = 0;
    __syncthreads();
    const bool by_logit = !g.bias && (g.o.n_groups == 1 || g.o.group_top == 1);
    for (int t = wave; t < kTok && row0 + t < g.rows; t += kWaves) {
        const int64_t row = row0 + t;
        double s[V], c[V];
        float l[V], top = -__builtin_huge_valf();
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int e = lane + 64 * j;
            l[j] = -__builtin_huge_valf();
            if (e < g.experts) l[j] = F32 ? ((const float*)g.logits)[row * g.ldl + e] : __uint_as_float((uint32_t)((const uint16_t*)g.logits)[row * g.ldl + e] << 16);
            if (!(l[j] == l[j])) l[j] = -__builtin_huge_valf();
            if (l[j] > 3.402823466e38f) l[j] = 3.402823466e38f;
            top = fmaxf(top, l[j]);
        }
        // the largest logit, by the keys of 32 bits that order floats
        double l_top = 0.0;
        if (!g.o.sigmoid) {
            const uint32_t tb = __float_as_uint(top + 0.f), most = wave_max(tb >> 31 ? ~tb : tb | 0x80000000u);
            l_top = __uint_as_float(most >> 31 ? most & 0x7FFFFFFFu : ~most);
        }
#pragma unroll
        for (int j = 0; j < V; ++j) s[j] = g.o.sigmoid ? -fabs((double)l[j]) : (double)l[j] - l_top;
        exp64<V>(s);
        if (g.o.sigmoid) {
#pragma unroll
            for (int j = 0; j < V; ++j) s[j] = sigmoid64(l[j], s[j]);
        } else {
            double sum = 0.0;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                if (l[j] == -__builtin_huge_valf()) s[j] = 0.0;
                sum += s[j];
            }
            sum = wave_sum(sum);
            const double by = reciprocal64(sum > 0.0 ? sum : 1.0);       // the largest of the terms is 1
#pragma unroll
            for (int j = 0; j < V; ++j) s[j] *= by;
        }
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const double v = by_logit ? (double)l[j] : s[j] + (double)bias[j];
            c[j] = l[j] == -__builtin_huge_valf() || !(v == v) ? kMinus : v;
        }
        if (g.o.n_groups > 1) {
            double* const mine = cbuf + (size_t)wave * g.experts;
            const int size = g.experts / g.o.n_groups;
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (lane + 64 * j < g.experts) mine[lane + 64 * j] = c[j];
            mx4_lanes_meet();
            // `per` lanes look at a group's members in turn, and join what they found
            const int per = 1 << g.per_bits, group = lane >> g.per_bits;
            double worth = kMinus, second = kMinus;
            if (group < g.o.n_groups)
                for (int i = lane & (per - 1); i < size; i += per) {
                    const double v = mine[group * size + i];
                    second = fmax(second, fmin(worth, v));
                    worth = fmax(worth, v);
                }
            for (int d = 1; d < per; d *= 2) {
                const double w2 = __shfl_xor(worth, d), s2 = __shfl_xor(second, d);
                second = fmax(fmax(second, s2), fmin(worth, w2));
                worth = fmax(worth, w2);
            }
            if (g.o.group_top == 2 && second > kMinus) worth += second;
            int ahead = 0;
            for (int i = 0; i < g.o.n_groups; ++i) {
                const double v = lane_value(worth, i << g.per_bits);
                ahead += v > worth || (v == worth && i < group);
            }
            const uint64_t open = __ballot(group < g.o.n_groups && ahead < g.o.top_groups);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const int e = lane + 64 * j;
                const int of = (int)(((float)e + 0.5f) * g.per_expert);          // e / size: far from a whole number for what e < 1024 can be
                if (e < g.experts && !((open >> (of << g.per_bits)) & 1)) c[j] = kMinus;
            }
        }
        uint32_t high[V], low[V];                            // halves of the keys, 0: not to be chosen, or chosen
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const uint64_t key = c[j] > kMinus ? key_of(c[j]) : 0;
            high[j] = (uint32_t)(key >> 32);
            low[j] = (uint32_t)key;
        }
        int my_id = -1;
        for (int k = 0; k < g.top_k; ++k) {
            uint32_t best = high[0];
#pragma unroll
            for (int j = 1; j < V; ++j) best = high[j] > best ? high[j] : best;
            best = wave_max(best);
            if (best == 0) break;                            // nothing is left: keys of numbers are above 2^32
            uint64_t who[V];
            int agree = 0, e = 0;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                who[j] = __ballot(high[j] == best);
                agree += __popcll(who[j]);
                if (who[j]) e = 64 * j + __builtin_ctzll(who[j]);
            }
            if (agree > 1) {                                 // several agree in the upper half: the lower one, then the lowest expert
                uint32_t below = 0;
#pragma unroll
                for (int j = 0; j < V; ++j)
                    if (high[j] == best && low[j] > below) below = low[j];
                below = wave_max(below);
#pragma unroll
                for (int j = V - 1; j >= 0; --j) {
                    const uint64_t same = __ballot(high[j] == best && low[j] == below);
                    if (same) e = 64 * j + __builtin_ctzll(same);
                }
#pragma unroll
                for (int j = 0; j < V; ++j) who[j] = e >> 6 == j ? (uint64_t)1 << (e & 63) : 0;
            }
#pragma unroll
            for (int j = 0; j < V; ++j)
                if ((who[j] >> lane) & 1) high[j] = 0;
            if (lane == k) my_id = e;
        }
        double my_s = 0.0;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const double v = __shfl(s[j], my_id & 63);
            if (my_id >> 6 == j) my_s = v;                   // none: -1 is nobody's
        }
        const double total = wave_sum(my_s);
        if (g.o.renormalize && total > 0.0) my_s /= total;
        if (lane < g.top_k) {
            g.ids[row * g.top_k + lane] = my_id;
            g.weights[row * g.top_k + lane] = (float)(my_s * (double)g.o.scale);
            if (my_id >= 0) atomicOr(&marks[my_id], 1u << t);
        }
    }
    __syncthreads();
    if (g.groups > 1) {
        for (int e = threadIdx.x; e < g.experts; e += kWaves * 64) g.counts[(int64_t)e * g.groups + blockIdx.x] = __popc(marks[e]);
        return;
    }
    if (wave == 0) sum_experts(g.experts, first, [&](int e) { return __popc(marks[e]); });
    __syncthreads();
    for (int e = threadIdx.x; e <= g.experts; e += kWaves * 64) g.offsets[e] = first[e];
    place_pairs(g, row0, marks, first, first[g.experts]);
}

// More than 32 rows, up to 384 experts: 16 lanes have a row, a lane the experts lane, lane + 16, ...  With a wavefront for a row the steps of its reductions, most of its
// instructions, serve that row alone.  us a call (a wavefront for a row): 8191 rows of 256 experts, top 8 of 4 of 8 groups, sigmoid 25.7 (28.5; both 1.4 less since the running sums need no LDS), 64 rows 21.5 (24.0); 32000 rows of
// 64 experts without groups 29.1 (44.4), 100 rows, softmax 10.1 (12.3); 3627 rows of 384 experts 30.1 (36.8), 4000 of 512 no less (39.0).
constexpr int kManyWaves = kTok / 4;
template <int CTRL>
__device__ __forceinline__ uint32_t turned(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 15, 15, true); }
template <int CTRL>
__device__ __forceinline__ double turned(double v) {
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint64_t lo = turned<CTRL>((uint32_t)b), hi = turned<CTRL>((uint32_t)(b >> 32));
    return __builtin_bit_cast(double, lo | hi << 32);
}
// Every lane of 16 gets what all of them make: pairs, pairs of pairs, then halves and rows in the mirror.  Both sides of each step join the same two, so a rounded sum is the same
// in all lanes (turns by 1, 2, 4 and 8 lanes would add in another order in each).
template <class T, class F>
__device__ __forceinline__ T row_reduce(T v, F join) {
    v = join(v, turned<0xB1>(v));
    v = join(v, turned<0x4E>(v));
    v = join(v, turned<0x141>(v));
    return join(v, turned<0x140>(v));
}
__device__ __forceinline__ uint32_t row_max(uint32_t v) { return row_reduce(v, [](uint32_t a, uint32_t b) { return a > b ? a : b; }); }
__device__ __forceinline__ uint32_t row_min(uint32_t v) { return row_reduce(v, [](uint32_t a, uint32_t b) { return a < b ? a : b; }); }
__device__ __forceinline__ double row_sum(double v) { return row_reduce(v, [](double a, double b) { return a + b; }); }

template <int V, bool F32>
__global__ __launch_bounds__(kManyWaves * 64) void route_many_kernel(RouteArgs g) {
    extern __shared__ __align__(16) char smem[];
    const int room = g.experts + 16;                                        // of a row: neighbouring ones begin on other banks
    double* const cbuf = (double*)smem;                                     // [row][expert]
    uint32_t* const marks = (uint32_t*)(cbuf + (size_t)kTok * room);
    const int lane = threadIdx.x & 63, sub = lane & 15, t = threadIdx.x >> 4;
    const int64_t row0 = (int64_t)blockIdx.x * kTok;
    const bool there = row0 + t < g.rows;
    const int64_t row = there ? row0 + t : g.rows - 1;                      // behind the last row: that one again, not stored
    float l[V], top = -__builtin_huge_valf();
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const int e = sub + 16 * j;
        l[j] = -__builtin_huge_valf();
        if (e < g.experts) l[j] = F32 ? ((const float*)g.logits)[row * g.ldl + e] : __uint_as_float((uint32_t)((const uint16_t*)g.logits)[row * g.ldl + e] << 16);
    }
    for (int e = threadIdx.x; e < g.experts; e += kManyWaves * 64) marks[e] = 0;
    __syncthreads();
    const bool by_logit = !g.bias && (g.o.n_groups == 1 || g.o.group_top == 1);
#pragma unroll
    for (int j = 0; j < V; ++j) {
        if (!(l[j] == l[j])) l[j] = -__builtin_huge_valf();
        if (l[j] > 3.402823466e38f) l[j] = 3.402823466e38f;
        top = fmaxf(top, l[j]);
    }
    double s[V], c[V], l_top = 0.0;
    if (!g.o.sigmoid) {
        const uint32_t tb = __float_as_uint(top + 0.f), most = row_max(tb >> 31 ? ~tb : tb | 0x80000000u);
        l_top = __uint_as_float(most >> 31 ? most & 0x7FFFFFFFu : ~most);
    }
#pragma unroll
    for (int j = 0; j < V; ++j) s[j] = g.o.sigmoid ? -fabs((double)l[j]) : (double)l[j] - l_top;
#pragma unroll
    for (int j = 0; j < V; j += 4) exp64<4>(s + j);
    if (g.o.sigmoid) {
#pragma unroll
        for (int j = 0; j < V; ++j) s[j] = sigmoid64(l[j], s[j]);
    } else {
        double sum = 0.0;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            if (l[j] == -__builtin_huge_valf()) s[j] = 0.0;
            sum += s[j];
        }
        sum = row_sum(sum);
        const double by = reciprocal64(sum > 0.0 ? sum : 1.0);
#pragma unroll
        for (int j = 0; j < V; ++j) s[j] *= by;
    }
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const double v = by_logit ? (double)l[j] : s[j] + (double)(g.bias && sub + 16 * j < g.experts ? g.bias[sub + 16 * j] : 0.f);
        c[j] = l[j] == -__builtin_huge_valf() || !(v == v) ? kMinus : v;
    }
    double* const mine = cbuf + (size_t)t * room;
    if (g.o.n_groups > 1) {
        const int size = g.experts / g.o.n_groups;
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (sub + 16 * j < g.experts) mine[sub + 16 * j] = c[j];
        mx4_lanes_meet();
        // `per` lanes look at a group's members in turn, and join what they found
        const int per = 1 << g.per_bits, group = sub >> g.per_bits;
        double worth = kMinus, second = kMinus;
        if (group < g.o.n_groups)
            for (int i = sub & (per - 1); i < size; i += per) {
                const double v = mine[group * size + i];
                second = fmax(second, fmin(worth, v));
                worth = fmax(worth, v);
            }
        for (int d = 1; d < per; d *= 2) {
            const double w2 = __shfl_xor(worth, d), s2 = __shfl_xor(second, d);
            second = fmax(fmax(second, s2), fmin(worth, w2));
            worth = fmax(worth, w2);
        }
        if (g.o.group_top == 2 && second > kMinus) worth += second;
        int ahead = 0;
        for (int i = 0; i < g.o.n_groups; ++i) {
            const double v = __shfl(worth, (lane & 48) + (i << g.per_bits));
            ahead += v > worth || (v == worth && i < group);
        }
        const uint32_t open = (uint32_t)(__ballot(group < g.o.n_groups && ahead < g.o.top_groups) >> (lane & 48));
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int e = sub + 16 * j;
            const int of = (int)(((float)e + 0.5f) * g.per_expert);              // e / size: far from a whole number for what e < 1024 can be
            if (e < g.experts && !((open >> (of << g.per_bits)) & 1)) c[j] = kMinus;
        }
        mx4_lanes_meet();
    }
    uint32_t high[V], low[V];                                    // halves of the keys, 0: not to be chosen, or chosen
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const uint64_t key = c[j] > kMinus ? key_of(c[j]) : 0;
        high[j] = (uint32_t)(key >> 32);
        low[j] = (uint32_t)key;
        if (sub + 16 * j < g.experts) mine[sub + 16 * j] = s[j];
    }
    int my_id = -1;
    for (int k = 0; k < g.top_k; ++k) {
        uint32_t best = high[0];
#pragma unroll
        for (int j = 1; j < V; ++j) best = high[j] > best ? high[j] : best;
        best = row_max(best);
        const uint64_t open = __ballot(best != 0);
        if (!open) break;                                        // nothing is left: keys of numbers are above 2^32
        const uint32_t want = best ? best : 0xFFFFFFFFu;         // nobody's key
        uint32_t e = 0xFFFFFFFFu;
        int agree = 0;
#pragma unroll
        for (int j = V - 1; j >= 0; --j) {
            agree += __popcll(__ballot(high[j] == want));
            if (high[j] == want) e = sub + 16 * j;
        }
        if (16 * agree > __popcll(open)) {                       // in some row several agree in the upper half: the lower one, then the lowest expert
            uint32_t below = 0;
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (high[j] == want && low[j] > below) below = low[j];
            below = row_max(below);
            e = 0xFFFFFFFFu;
#pragma unroll
            for (int j = V - 1; j >= 0; --j)
                if (high[j] == want && low[j] == below) e = sub + 16 * j;
        }
        e = row_min(e);
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (e == (uint32_t)(sub + 16 * j)) high[j] = 0;
        if (sub == k) my_id = (int)e;
    }
    mx4_lanes_meet();
    double my_s = my_id >= 0 ? mine[my_id] : 0.0;
    const double total = row_sum(my_s);
    if (g.o.renormalize && total > 0.0) my_s /= total;
    if (there && sub < g.top_k) {
        g.ids[row * g.top_k + sub] = my_id;
        g.weights[row * g.top_k + sub] = (float)(my_s * (double)g.o.scale);
        if (my_id >= 0) atomicOr(&marks[my_id], 1u << t);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < g.experts; e += kManyWaves * 64) g.counts[(int64_t)e * g.groups + blockIdx.x] = __popc(marks[e]);
}

// counts[e][*] to the numbers of pairs in the workgroups before, totals[e] their sum.  A wavefront has an expert.
__global__ __launch_bounds__(64) void route_sum_kernel(RouteArgs g) {
    const int lane = threadIdx.x;
    int32_t* const mine = g.counts + (int64_t)blockIdx.x * g.groups;
    int32_t before = 0;
    for (int i0 = 0; i0 < g.groups; i0 += 64) {
        const int32_t v = i0 + lane < g.groups ? mine[i0 + lane] : 0;
        const int32_t upto = (int32_t)mx4_sums_upto((uint32_t)v);
        if (i0 + lane < g.groups) mine[i0 + lane] = before + upto - v;
        before += __builtin_amdgcn_readlane(upto, 63);
    }
    if (lane == 0) g.totals[blockIdx.x] = before;
}

__global__ __launch_bounds__(kWaves * 64) void route_place_kernel(RouteArgs g) {
    extern __shared__ __align__(16) char smem[];
    uint32_t* const marks = (uint32_t*)smem;
    int32_t* const first = (int32_t*)(marks + g.experts);
    const int64_t row0 = (int64_t)blockIdx.x * kTok;
    for (int e = threadIdx.x; e < g.experts; e += kWaves * 64) marks[e] = 0;
    __syncthreads();
    const int64_t left = (g.rows - row0) * g.top_k;
    const int here = left < kTok * g.top_k ? (int)left : kTok * g.top_k;
    for (int i = threadIdx.x; i < here; i += kWaves * 64) {
        const int32_t e = g.ids[row0 * g.top_k + i];
        if (e >= 0) atomicOr(&marks[e], 1u << (i / g.top_k));
    }
    if (threadIdx.x < 64) sum_experts(g.experts, first, [&](int e) { return g.totals[e]; });
    __syncthreads();
    const int32_t total = first[g.experts];
    if (blockIdx.x == 0)
        for (int e = threadIdx.x; e <= g.experts; e += kWaves * 64) g.offsets[e] = first[e];
    __syncthreads();
    for (int e = threadIdx.x; e < g.experts; e += kWaves * 64) first[e] += g.counts[(int64_t)e * g.groups + blockIdx.x];
    __syncthreads();
    place_pairs(g, row0, marks, first, total);
}

__global__ __launch_bounds__(256) void route_none_kernel(int32_t* offsets, int n) {
    for (int e = threadIdx.x; e <= n; e += 256) offsets[e] = 0;
}

template <int V>
int launch_route(aser_ctx* ctx, const RouteArgs& g, bool f32) {
    const size_t lds = (g.o.n_groups > 1 ? (size_t)kWaves * g.experts * 8 : 0) + (2 * (size_t)g.experts + 1) * 4;
    auto kernel = f32 ? route_kernel<V, true> : route_kernel<V, false>;
    if (lds > 65536) ASER_HIP(ctx, hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
    kernel<<<(unsigned)g.groups, kWaves * 64, lds, ctx->stream>>>(g);
    return aser_check_launch(ctx, "route_kernel");
}

template <int V>
int launch_route_many(aser_ctx* ctx, const RouteArgs& g, bool f32) {
    const size_t lds = (size_t)kTok * (g.experts + 16) * 8 + (size_t)g.experts * 4;
    auto kernel = f32 ? route_many_kernel<V, true> : route_many_kernel<V, false>;
    if (lds > 65536) ASER_HIP(ctx, hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
    kernel<<<(unsigned)g.groups, kManyWaves * 64, lds, ctx->stream>>>(g);
    return aser_check_launch(ctx, "route_many_kernel");
}

// ---------------------------------------------------------------------------------------------------------------- the weighted sum
struct CombineArgs {
    const void* Y; int64_t ldy, m;
    const int32_t* place; const float* weights;
    int64_t rows, positions;
    int top_k;
    const void* Y0; int64_t ldy0;
    void* out; int64_t ldo;
    bool vec;
};

template <bool F32>
__device__ __forceinline__ float element(const void* p, int64_t at) {
    return F32 ? ((const float*)p)[at] : __uint_as_float((uint32_t)((const uint16_t*)p)[at] << 16);
}
template <bool F32>
__device__ __forceinline__ void eight(const void* p, int64_t at, int here, bool vec, float* v) {
    if (vec && here == 8) {
        if (F32) {
            const float4 a = *(const float4*)((const float*)p + at), b = *(const float4*)((const float*)p + at + 4);
            v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        } else {
            const uint4 a = *(const uint4*)((const uint16_t*)p + at);
            const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[2 * i] = __uint_as_float(w[i] << 16);
                v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
            }
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < here ? element<F32>(p, at + i) : 0.f;
}

// A workgroup has 2048 columns of a token, a thread eight.
template <bool YF32, bool OF32>
__global__ __launch_bounds__(256) void combine_kernel(CombineArgs g) {
    const int64_t t = blockIdx.z * kMxAcross + blockIdx.x, c = ((int64_t)blockIdx.y * 256 + threadIdx.x) * 8;
    if (t >= g.rows || c >= g.m) return;
    const int here = (int)(g.m - c < 8 ? g.m - c : 8);
    float sum[8];
    if (g.Y0) eight<OF32>(g.Y0, t * g.ldy0 + c, here, g.vec, sum);
    else {
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] = 0.f;
    }
    for (int j = 0; j < g.top_k; ++j) {
        const int32_t at = g.place[t * g.top_k + j];
        if (at < 0 || at >= g.positions) continue;
        const float w = g.weights[t * g.top_k + j];
        float v[8];
        eight<YF32>(g.Y, (int64_t)at * g.ldy + c, here, g.vec, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] = fmaf(w, v[i], sum[i]);
    }
    const int64_t o = t * g.ldo + c;
    if (g.vec && here == 8) {
        if (OF32) {
            *(float4*)((float*)g.out + o) = make_float4(sum[0], sum[1], sum[2], sum[3]);
            *(float4*)((float*)g.out + o + 4) = make_float4(sum[4], sum[5], sum[6], sum[7]);
        } else {
            *(uint4*)((uint16_t*)g.out + o) = make_uint4(bf16_pair(sum[0], sum[1]), bf16_pair(sum[2], sum[3]), bf16_pair(sum[4], sum[5]), bf16_pair(sum[6], sum[7]));
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (i >= here) continue;
        if (OF32) ((float*)g.out)[o + i] = sum[i];
        else ((uint16_t*)g.out)[o + i] = (uint16_t)bf16_pair(sum[i], sum[i]);
    }
}

bool row16(const void* p, int64_t ld, int64_t size) { return !((uintptr_t)p & 15) && !(ld * size & 15); }

}  // namespace

int aser_plan_check(aser_ctx* ctx, const char* who, const aser_expert_plan* p) {
    if (!p) ASER_FAIL(ctx, ASER_ERR_INVALID_ARG, "%s: null plan", who);
    if (p->rows < 0 || p->n_experts <= 0 || p->n_experts > 1024 || p->top_k <= 0 || p->top_k > 32 || p->top_k > p->n_experts || p->rows > INT32_MAX / 32 / p->top_k)
        ASER_FAIL(ctx, ASER_ERR_SHAPE, "%s: needs 1 to 1024 experts, 1 to 32 of them for a row, and less than 2^26 pairs", who);
    if (((uintptr_t)p->ids | (uintptr_t)p->weights | (uintptr_t)p->offsets | (uintptr_t)p->order | (uintptr_t)p->place) & 3)
        ASER_FAIL(ctx, ASER_ERR_INVALID_ARG, "%s: misaligned plan", who);
    return ASER_OK;
}

extern "C" size_t aser_route_workspace_bytes(int64_t rows, int32_t n_experts, int32_t top_k) {
    (void)top_k;
    if (rows <= kTok || n_experts <= 0) return kAserWsTail;
    return align_up((size_t)(ceil_div64(rows, kTok) + 1) * n_experts * 4, 256) + kAserWsTail;
}

extern "C" int aser_route_experts(aser_ctx* ctx, const void* logits, int32_t x_dtype, int64_t ldl, const float* bias, const aser_route_opts* opts,
                                  const aser_expert_plan* plan) {
    if (!ctx) return ASER_ERR_INVALID_ARG;
    if (!opts) ASER_FAIL(ctx, ASER_ERR_INVALID_ARG, "route_experts: null options");
    if (x_dtype != ASER_DTYPE_BF16 && x_dtype != ASER_DTYPE_F32) ASER_FAIL(ctx, ASER_ERR_DTYPE, "route_experts: dtype must be bf16 or f32");
    ASER_TRY(aser_plan_check(ctx, "route_experts", plan));
    const int experts = plan->n_experts;
    if (opts->n_groups < 1 || opts->n_groups > 64 || experts % opts->n_groups || opts->top_groups < 1 || opts->top_groups > opts->n_groups || opts->group_top < 1 ||
        opts->group_top > 2)
        ASER_FAIL(ctx, ASER_ERR_SHAPE, "route_experts: 1 to 64 groups of as many experts, 1 to n_groups of them open, a group worth its one or two best");
    if (!(opts->scale - opts->scale == 0.f)) ASER_FAIL(ctx, ASER_ERR_INVALID_ARG, "route_experts: scale is not finite");
    if (!plan->offsets || (plan->rows != 0 && (!logits || !plan->ids || !plan->weights || !plan->order || !plan->place)))
        ASER_FAIL(ctx, ASER_ERR_INVALID_ARG, "route_experts: null pointer");
    if (ldl < experts) ASER_FAIL(ctx, ASER_ERR_SHAPE, "route_experts: leading dimension below the number of experts");
    const bool f32 = x_dtype == ASER_DTYPE_F32;
    if (((uintptr_t)logits & (f32 ? 3 : 1)) || ((uintptr_t)bias & 3)) ASER_FAIL(ctx, ASER_ERR_INVALID_ARG, "route_experts: misaligned pointer");
    if (plan->rows == 0) {
        ASER_TRY(aser_prepare_device(ctx));
        route_none_kernel<<<1, 256, 0, ctx->stream>>>(plan->offsets, experts);
        return aser_check_launch(ctx, "route_none_kernel");
    }
    const size_t need = aser_route_workspace_bytes(plan->rows, experts, plan->top_k);
    RouteArgs g{logits, ldl, bias, *opts, plan->ids, plan->weights, plan->offsets, plan->order, plan->place, plan->rows, plan->top_k, experts, nullptr, nullptr,
                (int)ceil_div64(plan->rows, kTok)};
    const bool sixteen = g.groups > 1 && experts <= 384 && opts->n_groups <= 16 && plan->top_k <= 16;
    while ((opts->n_groups << (g.per_bits + 1)) <= (sixteen ? 16 : 64)) ++g.per_bits;
    g.per_expert = (float)opts->n_groups / (float)experts;
    if (g.groups > 1) {
        if (!ctx->ws || ctx->ws_bytes < need) ASER_FAIL(ctx, ASER_ERR_WORKSPACE, "route_experts: workspace too small");
        g.counts = (int32_t*)ctx->ws;
        g.totals = g.counts + (int64_t)g.groups * experts;
    }
    ASER_TRY(aser_prepare_device(ctx));
    if (sixteen) ASER_TRY(experts <= 64 ? launch_route_many<4>(ctx, g, f32) : experts <= 128 ? launch_route_many<8>(ctx, g, f32) : experts <= 256 ? launch_route_many<16>(ctx, g, f32) : launch_route_many<24>(ctx, g, f32));
    else if (experts <= 64) ASER_TRY(launch_route<1>(ctx, g, f32));
    else if (experts <= 128) ASER_TRY(launch_route<2>(ctx, g, f32));
    else if (experts <= 256) ASER_TRY(launch_route<4>(ctx, g, f32));
    else if (experts <= 512) ASER_TRY(launch_route<8>(ctx, g, f32));
    else ASER_TRY(launch_route<16>(ctx, g, f32));
    if (g.groups == 1) return ASER_OK;
    route_sum_kernel<<<(unsigned)experts, 64, 0, ctx->stream>>>(g);
    ASER_TRY(aser_check_launch(ctx, "route_sum_kernel"));
    route_place_kernel<<<(unsigned)g.groups, kWaves * 64, (2 * (size_t)experts + 1) * 4, ctx->stream>>>(g);
    return aser_check_launch(ctx, "route_place_kernel");
}

extern "C" int aser_expert_combine(aser_ctx* ctx, const void* Y, int32_t y_dtype, int64_t ldy, int64_t m, const aser_expert_plan* plan, const void* Y0, int64_t ldy0,
                                   void* out, int32_t out_dtype, int64_t ldo) {
    if (!ctx) return ASER_ERR_INVALID_ARG;
    if ((y_dtype != ASER_DTYPE_BF16 && y_dtype != ASER_DTYPE_F32) || (out_dtype != ASER_DTYPE_BF16 && out_dtype != ASER_DTYPE_F32))
        ASER_FAIL(ctx, ASER_ERR_DTYPE, "expert_combine: dtypes must be bf16 or f32");
    ASER_TRY(aser_plan_check(ctx, "expert_combine", plan));
    if (plan->rows != 0 && (!Y || !out || !plan->place || !plan->weights)) ASER_FAIL(ctx, ASER_ERR_INVALID_ARG, "expert_combine: null pointer");
    if (m <= 0 || m > ((int64_t)1 << 24) || ldy < m || ldo < m || (Y0 && (ldy0 < m || (Y0 == out && ldy0 != ldo)))) ASER_FAIL(ctx, ASER_ERR_SHAPE, "expert_combine: bad shape");
    const bool yf = y_dtype == ASER_DTYPE_F32, of = out_dtype == ASER_DTYPE_F32;
    if (((uintptr_t)Y & (yf ? 3 : 1)) || (((uintptr_t)Y0 | (uintptr_t)out) & (of ? 3 : 1))) ASER_FAIL(ctx, ASER_ERR_INVALID_ARG, "expert_combine: misaligned pointer");
    if (plan->rows == 0) return ASER_OK;
    CombineArgs g{Y, ldy, m, plan->place, plan->weights, plan->rows, plan->rows * plan->top_k, plan->top_k, Y0, ldy0, out, ldo, false};
    g.vec = row16(Y, ldy, yf ? 4 : 2) && row16(out, ldo, of ? 4 : 2) && (!Y0 || row16(Y0, ldy0, of ? 4 : 2));
    const dim3 grid((unsigned)(plan->rows < kMxAcross ? plan->rows : kMxAcross), (unsigned)ceil_div64(m, 2048), (unsigned)ceil_div64(plan->rows, kMxAcross));
    ASER_TRY(aser_prepare_device(ctx));
    if (yf) of ? combine_kernel<true, true><<<grid, 256, 0, ctx->stream>>>(g) : combine_kernel<true, false><<<grid, 256, 0, ctx->stream>>>(g);
    else of ? combine_kernel<false, true><<<grid, 256, 0, ctx->stream>>>(g) : combine_kernel<false, false><<<grid, 256, 0, ctx->stream>>>(g);
    return aser_check_launch(ctx, "combine_kernel");
}
