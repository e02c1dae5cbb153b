// dash_choose.hip -- the experts of every row and their gates from a router's logits (public values: the features that a circuit is routed by).
// Of a row's logits l and the bias b:
//     scores s = softmax(l) or sigmoid(l);  choice values c = s + b, without a bias the order of l;
//     of n_groups equal groups of experts the top_groups with the largest c (or the largest sum of two);  of their experts the top_k largest c;
//     w = scale s (renormalise: / sum of the chosen s);  gate = w 2^gate_bits, to the nearest integer, ties to the even.
// Everything that a comparison or a rounding decides on is held in 64 bits; where a quotient stands next to the middle of two gates, its remainder decides.
#include <limits.h>
#include <math.h>
#include <string.h>

#include "dash_internal.h"

namespace dash {

struct ChooseArgs {
    const void* logits;
    const float* bias;
    const uint8_t* valid;
    int32_t* experts;
    int32_t* gates;
    float* weights;
    int64_t row_stride, first, n;       // first: the launch's first row
    int E, top_k, n_groups, group_n, share_log2, top_groups, dtype;     // group_n: experts of a group; 2^share_log2 lanes look through one
    int pair, renormalise;
    double scale, two;                  // two: 2^gate_bits
};

// Values x and y of neighbouring lanes, blocks of lanes from step 2 on, one of them the lane's own (or its block's): after the steps 0 to 3 every lane of 16 has met all others, after the steps 0 to 5 of 64.
template <class T> __device__ __forceinline__ void meet(T v, int step, T& x, T& y) {
    constexpr int n = sizeof(T) / 4;
    int w[n], o[n];
    __builtin_memcpy(w, &v, sizeof(T));
#pragma unroll
    for (int i = 0; i < n; i++) {
        if (step == 0) o[i] = __builtin_amdgcn_update_dpp(0, w[i], 0xB1, 0xf, 0xf, true);               // quad_perm:[1,0,3,2]
        else if (step == 1) o[i] = __builtin_amdgcn_update_dpp(0, w[i], 0x4E, 0xf, 0xf, true);          // quad_perm:[2,3,0,1]
        else if (step == 2) o[i] = __builtin_amdgcn_update_dpp(0, w[i], 0x141, 0xf, 0xf, true);         // row_half_mirror
        else if (step == 3) o[i] = __builtin_amdgcn_update_dpp(0, w[i], 0x140, 0xf, 0xf, true);         // row_mirror
        else {
            const auto r = step == 4 ? __builtin_amdgcn_permlane16_swap(w[i], w[i], false, false) : __builtin_amdgcn_permlane32_swap(w[i], w[i], false, false);
            w[i] = (int)r[0]; o[i] = (int)r[1];
        }
    }
    __builtin_memcpy(&x, w, sizeof(T));
    __builtin_memcpy(&y, o, sizeof(T));
}
__device__ __forceinline__ int larger(int a, int b) { return a > b ? a : b; }
__device__ __forceinline__ float larger(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ double larger(double a, double b) { return fmax(a, b); }
__device__ __forceinline__ float smaller(float a, float b) { return fminf(a, b); }
__device__ __forceinline__ double smaller(double a, double b) { return fmin(a, b); }
// of the L lanes of a row
template <int L, class T> __device__ __forceinline__ T row_max(T v) {
#pragma unroll
    for (int s = 0; 1 << s < L; s++) { T x, y; meet(v, s, x, y); v = larger(x, y); }
    return v;
}
template <int L> __device__ __forceinline__ int row_min(int v) {
#pragma unroll
    for (int s = 0; 1 << s < L; s++) { int x, y; meet(v, s, x, y); v = x < y ? x : y; }
    return v;
}
template <int L> __device__ __forceinline__ double row_sum(double v) {
#pragma unroll
    for (int s = 0; 1 << s < L; s++) { double x, y; meet(v, s, x, y); v = x + y; }
    return v;
}
// e^a for a <= 0: a = n ln 2 + r, |r| <= ln 2 / 2, and the series of e^r up to r^13 / 13! (what follows is below 2^-57); off by 1.5 units in the last place at most.
// What is below e^-690 counts as zero: quotients of scores hold all their bits.
// The coefficients stand in scalar registers: as literals each costs two moves in front of its sum, and in vector registers a wave less fits.
struct Series {
    double c[13];
    __device__ __forceinline__ Series() : c{1.0 / 6227020800.0, 1.0 / 479001600, 1.0 / 39916800, 1.0 / 3628800, 1.0 / 362880, 1.0 / 40320, 1.0 / 5040, 1.0 / 720, 1.0 / 120, 1.0 / 24, 1.0 / 6, 0.5, 1.0} {
#pragma unroll
        for (int i = 0; i < 11; i++) asm("" : "+s"(c[i]));
    }
};
__device__ __forceinline__ double exp_of(double a, const Series& S) {
    a = a < -690.0 ? -3000.0 : a;                           // (0 in the end)
    const double n = rint(a * 1.4426950408889634074);
    double r = fma(n, -0x1.62e42fefa39efp-1, a);            // ln 2 to 53 bits, and what is left of it
    r = fma(n, -0x1.abc9e3b39803fp-56, r);
    double s = S.c[0];
#pragma unroll
    for (int i = 1; i < 13; i++) s = fma(s, r, S.c[i]);
    s = fma(s, r, 1.0);
    return ldexp(s, (int)n);
}
// 1 / v, 2^-1000 < v < 2^1000: an estimate of at least 20 bits and two steps of Newton's
__device__ __forceinline__ double inverse_of(double v) {
    double y = __builtin_amdgcn_rcp(v);
    y = fma(fma(-v, y, 1.0), y, y);
    return fma(fma(-v, y, 1.0), y, y);
}
// not a number: -infinity; infinity: the largest number
__device__ __forceinline__ float clean_logit(float l) { return l == l ? fminf(l, 3.4028234663852886e38f) : -INFINITY; }
__device__ __forceinline__ float half_logit(uint16_t v, int dtype) {
    return dtype == DASH_BF16 ? __uint_as_float((uint32_t)v << 16) : (float)__builtin_bit_cast(_Float16, v);
}

// L lanes a row, V neighbouring experts a lane.  BIAS: choice values are sums in 64 bits, else the logits themselves.
// A row's choice values stand in LDS, the lanes' runs of V, and every lane keeps the largest of its run.  A round: the largest of these (four to six steps between lanes), the first run that
// holds it; the lanes look through that run together for the first place of it and for what is largest without it.  A row lies within a wave: no barriers.  (Each
// lane through its own run again in registers: 65536 rows of 256 experts, eight chosen, 84.5 us.)  The rounds compare 32-bit integers: the logits, or the sums rounded to float32, which keeps
// their order but for sums that it makes equal; a wave that meets equal ones among its largest does its rounds again with the sums themselves (rounds in 64 bits for all: 44.1 us).
// Bound by vector instructions where rows are many, a third of them the exponentials (13 steps in 64 bits an expert; a float32 sum would move a choice or a gate): 65536 rows of 256 experts,
// eight chosen, 40.5 us, 64 % of the cycles, 39.8 MB read and written in 8.2 us at a copy's rate.  Few rows: the steps of one row's lanes one after the other, which more lanes make fewer.
// 4096 rows of 256 in eight groups, four of them: 9.5 us; 1000 rows of 160 in eight groups: 5.9; one row of 8: 4.7.
// What looks for gates next to a middle costs 0.05 to 0.1 us, 0.35 where 65536 rows of 16 are chosen from without renormalisation (7.6 -> 7.95); a quotient by division 0.15 more there.
constexpr int kChooseThreads = 256;
template <int L, int V, bool BIAS, bool GROUPS, bool SIGMOID>
__global__ __launch_bounds__(kChooseThreads) void k_choose(const ChooseArgs A) {
    typedef typename std::conditional<BIAS, double, float>::type Key;
    constexpr int R = kChooseThreads / L, P = V + (V > 1 ? 1 : 0);      // P: a run and a word, against bank conflicts
    constexpr Key kNone = -(Key)INFINITY;
    __shared__ Key s_key[R][P * L];
    const int lane = threadIdx.x % L, rr = threadIdx.x / L;
    const int64_t row_ = A.first + (int64_t)blockIdx.x * R + rr, row = row_ < A.n ? row_ : A.n - 1;
    const bool use = !A.valid || A.valid[row];
    auto lds_order = [&]() __attribute__((always_inline)) { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); __builtin_amdgcn_wave_barrier(); };
    float l[V];
    {
        const int e0 = lane * V, have = A.E - e0;
        const int64_t at = row * A.row_stride + e0;
        if (have >= V) {
            if (A.dtype == DASH_F32) {
                float x[V];
                __builtin_memcpy(x, (const float*)A.logits + at, sizeof(x));
#pragma unroll
                for (int v = 0; v < V; v++) l[v] = clean_logit(x[v]);
            } else {
                uint16_t x[V];
                __builtin_memcpy(x, (const uint16_t*)A.logits + at, sizeof(x));
#pragma unroll
                for (int v = 0; v < V; v++) l[v] = clean_logit(half_logit(x[v], A.dtype));
            }
        } else {
#pragma unroll
            for (int v = 0; v < V; v++)
                l[v] = v < have ? clean_logit(A.dtype == DASH_F32 ? ((const float*)A.logits)[at + v] : half_logit(((const uint16_t*)A.logits)[at + v], A.dtype)) : -INFINITY;
        }
    }
    float m = l[0];
#pragma unroll
    for (int v = 1; v < V; v++) m = fmaxf(m, l[v]);
    m = row_max<L>(m);
    const double top = m > -INFINITY ? (double)m : 0.0;
    double whole = 1;                           // softmax: the sum that every score is divided by, and its inverse
    double common = 1;
    const Series series;
    // score times `whole`
    auto part = [&](float x) __attribute__((always_inline)) -> double {
        if (!SIGMOID) return exp_of((double)x - top, series);
        const double t = exp_of(-fabs((double)x), series);
        return (x >= 0 ? 1.0 : t) * inverse_of(1 + t);
    };
    auto score = [&](float x) __attribute__((always_inline)) -> double { return SIGMOID ? part(x) : part(x) * common; };
    const bool sum_wanted = !SIGMOID && (BIAS || A.pair || !A.renormalise);     // (renormalised and of no other use: any common factor)
    Key key[V];
    // an expert that may be chosen (a bias that is no number makes its sum none)
    auto able = [&](int v) __attribute__((always_inline)) { return l[v] > -INFINITY && (!BIAS || key[v] > kNone); };
    if constexpr (BIAS) {
        double s[V], sum = 0;
        float b[V];
        if (A.E - lane * V >= V) __builtin_memcpy(b, A.bias + lane * V, sizeof(b));
        else
#pragma unroll
            for (int v = 0; v < V; v++) b[v] = A.bias[lane * V + v < A.E ? lane * V + v : A.E - 1];
#pragma unroll
        for (int v = 0; v < V; v++) { s[v] = score(l[v]); sum += s[v]; }
        if (sum_wanted) {
            whole = sum = row_sum<L>(sum);
            common = sum > 0 ? inverse_of(sum) : 0.0;
        }
#pragma unroll
        for (int v = 0; v < V; v++) {
            key[v] = fma(s[v], common, (double)b[v]);
            if (GROUPS) key[v] = able(v) ? key[v] : kNone;
        }
    } else {
        if (sum_wanted) {
            double sum = 0;
#pragma unroll
            for (int v = 0; v < V; v++) sum += exp_of((double)l[v] - top, series);
            whole = sum = row_sum<L>(sum);
            common = sum > 0 ? inverse_of(sum) : 0.0;
        }
#pragma unroll
        for (int v = 0; v < V; v++) key[v] = l[v];
    }

    // a bit of every lane of the row
    typedef typename std::conditional<L == 64, uint64_t, uint32_t>::type Bits;
    auto row_bits = [&](bool x) __attribute__((always_inline)) {
        if constexpr (L == 64) return (Bits)__ballot(x);
        else return (Bits)(__ballot(x) >> (threadIdx.x & (64 - L))) & (Bits)((1ull << L) - 1);
    };
    auto lowest = [](Bits x) __attribute__((always_inline)) { return L == 64 ? __builtin_ctzll(x) : __builtin_ctz((uint32_t)x); };
    if constexpr (GROUPS) {
        // kBatch of the LDS's values at a time, the last in the place of those past the end (which count for nothing): one wait each
        constexpr int kBatch = 8;
        __shared__ double s_group[R][64];
#pragma unroll
        for (int v = 0; v < V; v++) s_key[rr][lane * P + v] = key[v];
        lds_order();
        const int n = A.group_n;
        // share_log2: 2^share_log2 neighbouring lanes find a group's two largest, all L lanes at work
        const int share = 1 << A.share_log2;
        for (int g = lane >> A.share_log2; g < A.n_groups; g += L >> A.share_log2) {
            Key a = kNone, b = kNone;
            for (int i = lane & (share - 1); i < n; i += share * kBatch) {
                Key k[kBatch];
#pragma unroll
                for (int j = 0; j < kBatch; j++) {
                    const int e = g * n + (i + j * share < n ? i + j * share : n - 1);
                    k[j] = s_key[rr][e / V * P + e % V];
                }
#pragma unroll
                for (int j = 0; j < kBatch; j++) {
                    k[j] = i + j * share < n ? k[j] : kNone;
                    b = larger(b, smaller(a, k[j]));
                    a = larger(a, k[j]);
                }
            }
#pragma unroll
            for (int step = 0; 1 << step < L; step++) {
                if (step >= A.share_log2) break;
                Key a0, a1, b0, b1;
                meet(a, step, a0, a1); meet(b, step, b0, b1);
                b = larger(smaller(a0, a1), larger(b0, b1));
                a = larger(a0, a1);
            }
            double value = a;
            if (A.pair && a > kNone) {
                // (without a bias keys are logits, of which scores follow)
                value = BIAS ? (double)a : score((float)a);
                if (b > kNone) value += BIAS ? (double)b : score((float)b);
            }
            s_group[rr][g] = value;
        }
        lds_order();
        uint64_t kept = 0;
        for (int g0 = 0; g0 < A.n_groups; g0 += L) {
            const int g = g0 + lane;
            const double mine = s_group[rr][g < A.n_groups ? g : 0];
            int rank = 0;
            for (int i = 0; i < A.n_groups; i += kBatch) {
                double o[kBatch];
#pragma unroll
                for (int j = 0; j < kBatch; j++) o[j] = s_group[rr][i + j < A.n_groups ? i + j : 0];
#pragma unroll
                for (int j = 0; j < kBatch; j++) rank += i + j < A.n_groups && (o[j] > mine || (o[j] == mine && i + j < g)) ? 1 : 0;
            }
            kept |= (uint64_t)row_bits(g < A.n_groups && rank < A.top_groups) << g0;
        }
        lds_order();
        int g = lane * V / n, in = lane * V - g * n;
#pragma unroll
        for (int v = 0; v < V; v++) {
            if (!(g < A.n_groups && (kept >> (g & 63) & 1))) key[v] = kNone;
            if (++in == n) { in = 0; g++; }
        }
    }

    // lane j mod L keeps number j
    constexpr int kMine = (DASH_MAX_TOP_K + L - 1) / L;
    int mine[kMine];
#pragma unroll
    for (int i = 0; i < kMine; i++) mine[i] = -1;
    constexpr int kPer = (V + L - 1) / L;       // of a run, per lane
    bool equal = false;
    {
        // integers in the order of the floats (without a second zero); none: the lowest
        int* const to = (int*)s_key[rr];
        int best = INT_MIN;
#pragma unroll
        for (int v = 0; v < V; v++) {
            const float c = BIAS ? (float)key[v] : (float)key[v] + 0.0f;        // (a sum that rounds to -0 is below zero)
            const int bits = __float_as_int(c), k = c > -INFINITY && (!BIAS || GROUPS || l[v] > -INFINITY) ? bits ^ ((bits >> 31) & 0x7fffffff) : INT_MIN;
            to[lane * P + v] = k;
            best = k > best ? k : best;
        }
        lds_order();
        for (int j = 0; j < A.top_k; j++) {
            const int most = row_max<L>(best);
            if (most == INT_MIN || !use) break;         // (a row's lanes leave together)
            const Bits runs = row_bits(best == most);
            const int run = lowest(runs);
            int k[kPer], rest = INT_MIN;
            Bits there = 0;
            int first = 0;
#pragma unroll
            for (int i = 0; i < kPer; i++) k[i] = i * L + lane < V ? to[run * P + i * L + lane] : INT_MIN;
            bool several = (runs & (runs - 1)) != 0;
#pragma unroll
            for (int i = 0; i < kPer; i++) {
                const Bits bits = row_bits(k[i] == most);
                several |= (bits & (bits - 1)) != 0 || (bits && there);
                if (bits && !there) first = i * L + lowest(bits);
                there |= bits;
            }
#pragma unroll
            for (int i = 0; i < kPer; i++) {
                if (i * L + lane == first) to[run * P + first] = INT_MIN;
                else rest = k[i] > rest ? k[i] : rest;
            }
            rest = row_max<L>(rest);
            lds_order();
            if (lane == run) best = rest;
            if (j % L == lane) mine[j / L] = run * V + first;
            equal |= several;
        }
    }
    if (BIAS && __any(equal)) {
        lds_order();
#pragma unroll
        for (int i = 0; i < kMine; i++) mine[i] = -1;
        Key best = kNone;
#pragma unroll
        for (int v = 0; v < V; v++) {
            const Key k = GROUPS || able(v) ? key[v] : kNone;
            s_key[rr][lane * P + v] = k;
            best = larger(best, k);
        }
        lds_order();
        for (int j = 0; j < A.top_k; j++) {
            const Key most = row_max<L>(best);
            if (!(most > kNone) || !use) break;
            const int run = row_min<L>(best == most ? lane : L);
            Key rest = kNone, k[kPer];
            int first = V;
#pragma unroll
            for (int i = 0; i < kPer; i++) {
                const int at = i * L + lane;
                k[i] = at < V ? s_key[rr][run * P + at] : kNone;
                if (k[i] == most && first == V) first = at;
            }
            first = row_min<L>(first);
#pragma unroll
            for (int i = 0; i < kPer; i++) {
                const int at = i * L + lane;
                if (at == first) s_key[rr][run * P + at] = kNone;
                else rest = larger(rest, k[i]);
            }
            rest = row_max<L>(rest);
            lds_order();
            if (lane == run) best = rest;
            if (j % L == lane) mine[j / L] = run * V + first;
        }
    }
    // scores, softmax's times `whole`
    double s[kMine];
#pragma unroll
    for (int i = 0; i < kMine; i++) {
        s[i] = 0;
        if (mine[i] >= 0) {
            const int64_t at = row * A.row_stride + mine[i];
            s[i] = part(clean_logit(A.dtype == DASH_F32 ? ((const float*)A.logits)[at] : half_logit(((const uint16_t*)A.logits)[at], A.dtype)));
        }
    }
    double inverse = common;                    // of what s are divided by
    if (A.renormalise) {
        const double sum = row_sum<L>(kMine == 2 ? s[0] + s[kMine - 1] : s[0]);
        inverse = sum > 0 ? inverse_of(sum) : 0.0;
    }
    double w[kMine], gate[kMine];
    bool near = false;                          // gates next to the middle of two integers (what was rounded until here is below 2^-19 of a gate)
#pragma unroll
    for (int i = 0; i < kMine; i++) {
        if (i * L >= A.top_k) break;
        w[i] = s[i] * inverse * A.scale;
        const double t = w[i] * A.two;
        gate[i] = rint(t);
        near |= fabs(fabs(t - gate[i]) - 0.5) < 0x1p-18;
    }
    if (A.gates && __any(near)) {
        // Equal scores share as integers do, and a rounded quotient would take the middle of two gates to either side: the sign of scale 2^gate_bits s - (m + 1/2) sum
        // decides, without a rounding.  A sum of chosen scores is held in two numbers for that: it is exact where they are equal.
        double high = s[0], low = 0;
        auto add = [&](double x, double y) __attribute__((always_inline)) {
            high = x + y;
            const double t = high - x;
            low += (x - (high - t)) + (y - t);
        };
        if (A.renormalise) {
            if (kMine == 2) add(s[0], s[kMine - 1]);
#pragma unroll
            for (int step = 0; 1 << step < L; step++) {
                double x, y, a, b;
                meet(high, step, x, y); meet(low, step, a, b);
                low = a + b;
                add(x, y);
            }
        } else high = whole;
#pragma unroll
        for (int i = 0; i < kMine; i++) {
            if (i * L >= A.top_k) break;
            const double t = w[i] * A.two, m = floor(t), middle = m + 0.5, p = middle * high;
            if (!(fabs(t - middle) < 0x1p-18)) continue;
            // (each of these is exact: the products leave less than 40 bits next to p)
            const double over = fma(A.scale * A.two, s[i], -p) - fma(middle, low, fma(middle, high, -p));
            gate[i] = over > 0 || (over == 0 && (int)m & 1) ? m + 1 : m;
        }
    }
    if (row_ >= A.n) return;
#pragma unroll
    for (int i = 0; i < kMine; i++) {
        const int j = i * L + lane;
        if (j >= A.top_k) break;
        const int64_t to = row * A.top_k + j;
        A.experts[to] = mine[i];
        if (A.gates) A.gates[to] = (int32_t)gate[i];
        if (A.weights) A.weights[to] = (float)w[i];
    }
}

}  // namespace dash

using namespace dash;

extern "C" {

int dash_choose(dash_ctx* c, const dash_router* r, const void* logits, int dtype, int64_t row_stride, int64_t n, const uint8_t* valid, int32_t* experts,
                int32_t* gates, float* weights, void* stream) {
    if (!c || !r || n < 0 || dtype < DASH_F32 || dtype > DASH_F16) return DASH_EINVAL;
    const int E = r->n_experts, G = r->n_groups;
    if (E < 1 || G < 1 || E % G || r->top_groups < 1 || r->top_groups > G || r->top_k < 1 || r->top_k > r->top_groups * (E / G)) return DASH_EINVAL;
    if (r->score < DASH_SOFTMAX || r->score > DASH_SIGMOID || r->group_score < DASH_GROUP_MAX || r->group_score > DASH_GROUP_PAIR) return DASH_EINVAL;
    if (!(r->scale > 0) || r->gate_bits < 0 || r->gate_bits > 30 || !(ldexp((double)r->scale, r->gate_bits) <= 1073741824.0)) return DASH_EINVAL;
    if (E > DASH_MAX_ROUTED || r->top_k > DASH_MAX_TOP_K || G > 64) return DASH_ESIZE;
    if (n == 0) return DASH_OK;
    const uintptr_t unaligned = dtype == DASH_F32 ? 3 : 1;
    if (!logits || ((uintptr_t)logits & unaligned) || row_stride < E || !experts) return DASH_EINVAL;
    if (((uintptr_t)experts & 3) || ((uintptr_t)gates & 3) || ((uintptr_t)weights & 3) || ((uintptr_t)r->bias & 3)) return DASH_EINVAL;
    ChooseArgs A;
    memset(&A, 0, sizeof(A));
    A.logits = logits; A.bias = r->bias; A.valid = valid; A.experts = experts; A.gates = gates; A.weights = weights;
    A.row_stride = row_stride; A.n = n; A.E = E; A.top_k = r->top_k; A.n_groups = G; A.group_n = E / G; A.top_groups = r->top_groups; A.dtype = dtype;
    A.pair = r->group_score == DASH_GROUP_PAIR && r->top_groups < G; A.renormalise = r->renormalise != 0;
    A.scale = r->scale; A.two = ldexp(1.0, r->gate_bits);
    auto launch = [&](auto lanes, auto v) {
        constexpr int L = decltype(lanes)::value, V = decltype(v)::value, R = kChooseThreads / L;
        constexpr int64_t most = 0xffffffffll / kChooseThreads;
        const bool groups = r->top_groups < G;
        while (G << (A.share_log2 + 1) <= L) A.share_log2++;
        auto kernel = [&](auto sigmoid) -> void (*)(ChooseArgs) {
            constexpr bool S = decltype(sigmoid)::value;
            if (r->bias) return groups ? k_choose<L, V, true, true, S> : k_choose<L, V, true, false, S>;
            if (groups) return k_choose<L, V, false, true, S>;
            if constexpr (L == 16 || V == 16) return k_choose<L, V, false, false, S>;
            return nullptr;                     // (by the rule below none)
        };
        const auto k = r->score == DASH_SIGMOID ? kernel(std::true_type{}) : kernel(std::false_type{});
        const int64_t blocks = (n + R - 1) / R;
        for (int64_t first = 0; first < blocks; first += most) {
            A.first = first * R;
            hipLaunchKernelGGL(k, dim3((uint32_t)(blocks - first < most ? blocks - first : most)), dim3(kChooseThreads), 0, (hipStream_t)stream, A);
        }
    };
    using std::integral_constant;
    constexpr integral_constant<int, 16> l16{};
    constexpr integral_constant<int, 32> l32{};
    constexpr integral_constant<int, 64> l64{};
    // Lanes of a row (times without the search for gates next to a middle, which adds 0.05 to 0.1 us to each).  What they do for their own experts one after the other takes the time where rows are few, and with sums in 64 bits and groups of many experts also where they are many; each
    // round costs instructions by the lane.  us with 16, 32, 64 lanes, eight chosen of 256 experts with a bias and groups (sigmoid): 1 row 9.5, 7.2, 6.2; 1000: 10.2, 7.7, 6.7; 2048: 10.2, 7.9, 7.9;
    // 4096: 10.3, 9.8, 10.7; 8192: 14.0, 13.5, 16.8; 65536: 66.6, 67.7, 103; with neither: 4.0, 3.9, 4.1 for one row, 18.6, 27.7, 49.1 for 65536.  Of 128: 1000 rows 7.7, 6.4, 6.4;
    // 8192: 10.2, 10.5, 15.6.  Of 512: 1000 rows 15.9, 10.3, 8.0; 2048: 16.0, 10.3, 9.9; 4096: 16.2, 14.1, 13.8; 16384: 41.6, 33.7, 36.4; with neither 1 row 5.1, 3.9, 4.1, 65536: 30.4, 32.1, 52.8.  Of 1024, 32 and 64: 1000 rows 15.8, 10.4;
    // 65536: 253, 211.
    const bool much = r->bias || r->top_groups < G;
    if (E <= 16) launch(l16, integral_constant<int, 1>{});
    else if (E <= 32) launch(l16, integral_constant<int, 2>{});
    else if (E <= 64) launch(l16, integral_constant<int, 4>{});
    else if (E <= 128) much && n <= 2048 ? launch(l32, integral_constant<int, 4>{}) : launch(l16, integral_constant<int, 8>{});
    else if (E <= 256) much && n <= 1024 ? launch(l64, integral_constant<int, 4>{}) : much && n <= 8192 ? launch(l32, integral_constant<int, 8>{}) : launch(l16, integral_constant<int, 16>{});
    else if (E <= 512) much && n <= 2048 ? launch(l64, integral_constant<int, 8>{}) : launch(l32, integral_constant<int, 16>{});
    else launch(l64, integral_constant<int, 16>{});
    DASH_HIP(hipGetLastError());
    return DASH_OK;
}

}  // extern "C"
