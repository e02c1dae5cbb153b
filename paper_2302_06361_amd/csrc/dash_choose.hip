// dash_choose.hip -- the experts of every row and their gates from a router's logits (public values: the features that a circuit is routed by).
// Of a row's logits l and the bias b:
//     scores s = softmax(l) or sigmoid(l);  choice values c = s + b, without a bias the order of l;
//     of n_groups equal groups of experts the top_groups with the largest c (or the largest sum of two);  of their experts the top_k largest c;
//     w = scale s (renormalise: / sum of the chosen s);  gate = w 2^gate_bits, to the nearest integer, ties to the even.
// Everything that a comparison or a rounding decides on is held in 64 bits.
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
    int E, top_k, n_groups, top_groups, dtype;
    int sigmoid, pair, renormalise;
    double scale, two;                  // two: 2^gate_bits
};
constexpr int kRowLanes = 16;           // lanes of a row

// the values of the lanes that differ from one another by the bits 1, 2, 4, 8 joined: a row's 16 lanes
template <class T> __device__ __forceinline__ T from_lane(T v, int step) {
    constexpr int n = sizeof(T) / 4;
    int w[n];
    __builtin_memcpy(w, &v, sizeof(T));
#pragma unroll
    for (int i = 0; i < n; i++)
        w[i] = step == 0 ? __builtin_amdgcn_update_dpp(0, w[i], 0xB1, 0xf, 0xf, true)           // quad_perm:[1,0,3,2]
             : step == 1 ? __builtin_amdgcn_update_dpp(0, w[i], 0x4E, 0xf, 0xf, true)           // quad_perm:[2,3,0,1]
             : step == 2 ? __builtin_amdgcn_update_dpp(0, w[i], 0x141, 0xf, 0xf, true)          // row_half_mirror
                         : __builtin_amdgcn_update_dpp(0, w[i], 0x140, 0xf, 0xf, true);         // row_mirror
    __builtin_memcpy(&v, w, sizeof(T));
    return v;
}
template <class T> __device__ __forceinline__ T row_max(T v) {
#pragma unroll
    for (int s = 0; s < 4; s++) { const T o = from_lane(v, s); v = o > v ? o : v; }
    return v;
}
__device__ __forceinline__ int row_min(int v) {
#pragma unroll
    for (int s = 0; s < 4; s++) { const int o = from_lane(v, s); v = o < v ? o : v; }
    return v;
}
__device__ __forceinline__ double row_sum(double v) {
#pragma unroll
    for (int s = 0; s < 4; s++) v += from_lane(v, s);
    return v;
}
// not a number: -infinity; infinity: the largest number
__device__ __forceinline__ float read_logit(const ChooseArgs& A, int64_t at) {
    float l;
    if (A.dtype == DASH_F32) l = ((const float*)A.logits)[at];
    else if (A.dtype == DASH_BF16) l = __uint_as_float((uint32_t)((const uint16_t*)A.logits)[at] << 16);
    else l = (float)((const _Float16*)A.logits)[at];
    return l == l ? fminf(l, 3.4028234663852886e38f) : -INFINITY;
}

// 16 lanes a row, V neighbouring experts a lane.  BIAS: choice values are sums in 64 bits, else the logits themselves.
template <int V, bool BIAS, bool GROUPS>
__global__ __launch_bounds__(V == 64 ? 64 : 256) void k_choose(const ChooseArgs A) {
    typedef typename std::conditional<BIAS, double, float>::type Key;
    constexpr int T = V == 64 ? 64 : 256, R = T / kRowLanes;
    constexpr Key kNone = -(Key)INFINITY;
    const int lane = threadIdx.x % kRowLanes, rr = threadIdx.x / kRowLanes;
    const int64_t row_ = A.first + (int64_t)blockIdx.x * R + rr, row = row_ < A.n ? row_ : A.n - 1;
    const bool use = !A.valid || A.valid[row];
    float l[V];
#pragma unroll
    for (int v = 0; v < V; v++) l[v] = lane * V + v < A.E ? read_logit(A, row * A.row_stride + lane * V + v) : -INFINITY;
    float m = l[0];
#pragma unroll
    for (int v = 1; v < V; v++) m = fmaxf(m, l[v]);
    m = row_max(m);
    const double top = m > -INFINITY ? (double)m : 0.0;
    double inverse = 0;
    if (!A.sigmoid && (BIAS || A.pair || !A.renormalise)) {
        double sum = 0;
#pragma unroll
        for (int v = 0; v < V; v++) sum += exp((double)l[v] - top);
        sum = row_sum(sum);
        inverse = sum > 0 ? 1 / sum : 0;
    } else inverse = 1;         // (renormalised and of no other use: any common factor)
    auto score = [&](float x) { return A.sigmoid ? 1 / (1 + exp(-(double)x)) : exp((double)x - top) * inverse; };
    Key key[V];
#pragma unroll
    for (int v = 0; v < V; v++) {
        const int e = lane * V + v;
        Key c = l[v];
        if constexpr (BIAS) {
            const double x = score(l[v]) + (double)A.bias[e < A.E ? e : A.E - 1];
            c = x == x ? x : kNone;
        }
        key[v] = use && l[v] > -INFINITY ? c : kNone;
    }

    if constexpr (GROUPS) {
        // keys and, for sums of two, scores through LDS; a lane per group
        __shared__ Key s_key[R][V * kRowLanes];
        __shared__ float s_logit[R][BIAS ? 1 : V * kRowLanes];
        __shared__ double s_group[R][64];
        __shared__ uint8_t s_kept[R][64];
        const int n = A.E / A.n_groups;
#pragma unroll
        for (int v = 0; v < V; v++) {
            s_key[rr][lane * V + v] = key[v];
            if (!BIAS) s_logit[rr][lane * V + v] = l[v];
        }
        __syncthreads();
        for (int g = lane; g < A.n_groups; g += kRowLanes) {
            Key a = kNone, b = kNone;       // the two largest
            for (int i = 0; i < n; i++) {
                const Key k = s_key[rr][g * n + i];
                if (k > a) { b = a; a = k; } else if (k > b) b = k;
            }
            double value = a;
            if (A.pair && a > kNone) {
                // (without a bias keys are logits, of which scores follow)
                value = BIAS ? (double)a : score((float)a);
                if (b > kNone) value += BIAS ? (double)b : score((float)b);
            }
            s_group[rr][g] = value;
        }
        __syncthreads();
        for (int g = lane; g < A.n_groups; g += kRowLanes) {
            const double mine = s_group[rr][g];
            int rank = 0;
            for (int i = 0; i < A.n_groups; i++) {
                const double o = s_group[rr][i];
                rank += o > mine || (o == mine && i < g) ? 1 : 0;
            }
            s_kept[rr][g] = rank < A.top_groups;
        }
        __syncthreads();
#pragma unroll
        for (int v = 0; v < V; v++) {
            const int e = lane * V + v;
            if (!s_kept[rr][e < A.E ? e / n : 0]) key[v] = kNone;
        }
    }

    // top_k rounds: the row's largest, the lowest number of it, out; lane j mod 16 keeps number j
    int mine[2] = {-1, -1};
    float logit[2] = {-INFINITY, -INFINITY};
    for (int j = 0; j < A.top_k; j++) {
        Key best = key[0];
        int at = 0;
        float bl = l[0];
#pragma unroll
        for (int v = 1; v < V; v++) if (key[v] > best) { best = key[v]; at = v; bl = l[v]; }
        const Key most = row_max(best);
        if (!(most > kNone)) break;
        const int e = row_min(best == most ? lane * V + at : 0x7fffffff);
        const bool won = e / V == lane;
#pragma unroll
        for (int v = 0; v < V; v++) if (won && v == at) key[v] = kNone;
        const float el = __shfl(bl, e / V, kRowLanes);
        if (j % kRowLanes == lane) {
            if (j < kRowLanes) { mine[0] = e; logit[0] = el; } else { mine[1] = e; logit[1] = el; }
        }
    }
    double s[2];
#pragma unroll
    for (int i = 0; i < 2; i++) s[i] = mine[i] >= 0 ? score(logit[i]) : 0.0;
    double factor = A.scale;
    if (A.renormalise) {
        const double sum = row_sum(s[0] + s[1]);
        factor = sum > 0 ? A.scale / sum : 0.0;
    }
    if (row_ >= A.n) return;
#pragma unroll
    for (int i = 0; i < 2; i++) {
        const int j = i * kRowLanes + lane;
        if (j >= A.top_k) break;
        const int64_t to = row * A.top_k + j;
        const double w = s[i] * factor;
        A.experts[to] = mine[i];
        if (A.gates) A.gates[to] = (int32_t)rint(w * A.two);
        if (A.weights) A.weights[to] = (float)w;
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
    A.row_stride = row_stride; A.n = n; A.E = E; A.top_k = r->top_k; A.n_groups = G; A.top_groups = r->top_groups; A.dtype = dtype;
    A.sigmoid = r->score == DASH_SIGMOID; A.pair = r->group_score == DASH_GROUP_PAIR && r->top_groups < G; A.renormalise = r->renormalise != 0;
    A.scale = r->scale; A.two = ldexp(1.0, r->gate_bits);
    auto launch = [&](auto v) {
        constexpr int V = decltype(v)::value, T = V == 64 ? 64 : 256, R = T / kRowLanes;
        constexpr int64_t most = 0xffffffffll / 256;
        const int64_t blocks = (n + R - 1) / R;
        for (int64_t first = 0; first < blocks; first += most) {
            A.first = first * R;
            const dim3 grid((uint32_t)(blocks - first < most ? blocks - first : most));
            const bool groups = r->top_groups < G;
            if (r->bias && groups) hipLaunchKernelGGL((k_choose<V, true, true>), grid, dim3(T), 0, (hipStream_t)stream, A);
            else if (r->bias) hipLaunchKernelGGL((k_choose<V, true, false>), grid, dim3(T), 0, (hipStream_t)stream, A);
            else if (groups) hipLaunchKernelGGL((k_choose<V, false, true>), grid, dim3(T), 0, (hipStream_t)stream, A);
            else hipLaunchKernelGGL((k_choose<V, false, false>), grid, dim3(T), 0, (hipStream_t)stream, A);
        }
    };
    using std::integral_constant;
    if (E <= 16) launch(integral_constant<int, 1>{});
    else if (E <= 32) launch(integral_constant<int, 2>{});
    else if (E <= 64) launch(integral_constant<int, 4>{});
    else if (E <= 128) launch(integral_constant<int, 8>{});
    else if (E <= 256) launch(integral_constant<int, 16>{});
    else if (E <= 512) launch(integral_constant<int, 32>{});
    else launch(integral_constant<int, 64>{});
    DASH_HIP(hipGetLastError());
    return DASH_OK;
}

}  // extern "C"
