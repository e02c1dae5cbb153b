// dash_experts.hip -- layers whose matrix depends on the row, on LabelTensors (Sec. Arithmetic Garbled Circuits: free addition and
// multiplication by a public constant).  Per CRT prime p
//     experts:  out[r][j][digit] = sum_i W_e(r)[j][i] * in[r / top_k][i][digit]  (+ bias_e(r)[j] * one[digit])   mod p
//     combine:  out[t][v][digit] = sum_j gate[t][j] * in[t * top_k + j][v][digit]                                mod p
// The expert e(r) of a row is public; rows of no expert get all-zero labels.  The garbler applies both to zero labels, the evaluator to
// active labels.
//
//   k_route_count / _scan / _fill : rows sorted by expert, in order inside an expert
//   k_weights8_prepare            : signed bytes into the tiles of the products
//   k_mx4_quantise                : weights to 4-bit floats with a power of two for every 32, into the tiles of the products
//   (the products: dash_experts_gemm.hip)
//   k_combine                     : the weighted sums
#include <hip/hip_bf16.h>
#include <string.h>

#include "dash_experts.h"

namespace dash {

constexpr int kWaves = kThreads / 64;

// ---- routing -----------------------------------------------------------------------------------
struct RouteArgs {
    const int32_t* experts;
    int64_t n;
    int E, k;
    uint8_t nchunk[DASH_MAX_PRIMES];
    RoutingView to;
};
__device__ __forceinline__ bool route_match(int32_t id, int e, int E) { return e < E ? id == e : (uint32_t)id >= (uint32_t)E; }

// A wave per expert (E + 1 of them: the last is "none") counts its rows.
__global__ __launch_bounds__(kThreads) void k_route_count(const RouteArgs A) {
    const int e = (int)(blockIdx.x * kWaves + threadIdx.x / 64), lane = threadIdx.x & 63;
    if (e > A.E) return;
    int32_t count = 0;
    for (int64_t r0 = 0; r0 < A.n; r0 += 64) {
        const bool hit = r0 + lane < A.n && route_match(A.experts[r0 + lane], e, A.E);
        count += __popcll(__ballot(hit));
    }
    if (lane == 0) A.to.offsets[e + 1] = count;
}
__device__ __forceinline__ int32_t route_tiles(const RouteArgs& A, int32_t rows, int groups) {
    int32_t t = 0;
    for (int i = 0; i < A.k; i++) t += (int32_t)(((int64_t)rows * A.nchunk[i] + groups - 1) / groups);
    return t;
}
// One block: counts to offsets and to first tiles.
__global__ __launch_bounds__(kThreads) void k_route_scan(const RouteArgs A) {
    __shared__ int32_t part[1 + kTileSizes][kThreads];
    const int n = A.E + 1, per = (n + kThreads - 1) / kThreads, e0 = threadIdx.x * per, e1 = e0 + per < n ? e0 + per : n;
    int32_t sum[1 + kTileSizes] = {};
    for (int e = e0; e < e1; e++) {
        const int32_t rows = A.to.offsets[e + 1];
        sum[0] += rows;
        for (int s = 0; s < kTileSizes; s++) sum[1 + s] += route_tiles(A, rows, kTileGroups[s]);
    }
    for (int s = 0; s < 1 + kTileSizes; s++) part[s][threadIdx.x] = sum[s];
    __syncthreads();
    if (threadIdx.x < 1 + kTileSizes) {
        int32_t at = 0;
        for (int i = 0; i < kThreads; i++) { const int32_t v = part[threadIdx.x][i]; part[threadIdx.x][i] = at; at += v; }
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        A.to.offsets[0] = 0;
        for (int s = 0; s < kTileSizes; s++) A.to.first_tile[s][0] = 0;
    }
    for (int s = 0; s < 1 + kTileSizes; s++) sum[s] = part[s][threadIdx.x];
    for (int e = e0; e < e1; e++) {
        const int32_t rows = A.to.offsets[e + 1];
        sum[0] += rows;
        A.to.offsets[e + 1] = sum[0];
        for (int s = 0; s < kTileSizes; s++) { sum[1 + s] += route_tiles(A, rows, kTileGroups[s]); A.to.first_tile[s][e + 1] = sum[1 + s]; }
    }
}
// The wave of an expert writes its rows in ascending order, and its tiles.
__global__ __launch_bounds__(kThreads) void k_route_fill(const RouteArgs A) {
    const int e = (int)(blockIdx.x * kWaves + threadIdx.x / 64), lane = threadIdx.x & 63;
    if (e > A.E) return;
    const int32_t start = A.to.offsets[e], count = A.to.offsets[e + 1] - start;
    int32_t at = start;
    for (int64_t r0 = 0; r0 < A.n; r0 += 64) {
        const bool hit = r0 + lane < A.n && route_match(A.experts[r0 + lane], e, A.E);
        const uint64_t m = __ballot(hit);
        if (hit) A.to.rows[at + __popcll(m & ((1ull << lane) - 1))] = (int32_t)(r0 + lane);
        at += __popcll(m);
    }
    for (int s = 0; s < kTileSizes; s++) {
        int32_t t0 = A.to.first_tile[s][e];
        for (int i = 0; i < A.k; i++) {
            const int32_t tiles = (int32_t)(((int64_t)count * A.nchunk[i] + kTileGroups[s] - 1) / kTileGroups[s]);
            for (int32_t t = lane; t < tiles; t += 64) A.to.tiles[s][t0 + t] = RouteTile{(uint32_t)e | (uint32_t)i << 24, start, count, t * kTileGroups[s]};
            t0 += tiles;
        }
    }
}

// ---- weights -----------------------------------------------------------------------------------
struct PrepArgs8 {
    const int8_t* w;
    int64_t row_stride, expert_stride, tiles;       // tiles of all experts
    int M, K;
    uint8_t* out;
};
// a lane per 16-byte piece of a tile
__global__ __launch_bounds__(kThreads) void k_weights8_prepare(const PrepArgs8 A) {
    const int64_t idx = (int64_t)blockIdx.x * kThreads + threadIdx.x, tile = idx / (kW8Tile / 16);
    if (tile >= A.tiles) return;
    const int piece = (int)(idx % (kW8Tile / 16)), r = piece / 4, q = piece % 4;
    const int64_t kt = col_tiles(A.K), mt = row_tiles(A.M), e = tile / (mt * kt), at = tile - e * mt * kt;
    const int64_t row = at / kt * kTileRows + r, col = at % kt * kTileCols + 16 * q;
    uint32_t v[4] = {0, 0, 0, 0};
    if (row < A.M) {
        const int8_t* src = A.w + e * A.expert_stride + row * A.row_stride + col;
        for (int i = 0; i < 16; i++)
            if (col + i < A.K) v[i / 4] |= (uint32_t)(uint8_t)src[i] << (8 * (i % 4));
    }
    *(uint4*)(A.out + tile * kW8Tile + w8_at(r, 16 * q)) = make_uint4(v[0], v[1], v[2], v[3]);
}

struct QuantArgs {
    const void* w;
    int64_t row_stride, expert_stride, tiles;
    int M, K, base, max_shift;
    uint8_t* out;
    void* values;
};
template <class T> __device__ __forceinline__ float to_float(T v) { return (float)v; }
template <> __device__ __forceinline__ float to_float(__hip_bfloat16 v) { return __bfloat162float(v); }
template <class T> __device__ __forceinline__ T from_float(float v) { return (T)v; }
template <> __device__ __forceinline__ __hip_bfloat16 from_float(float v) { return __float2bfloat16(v); }

// a lane per block of 32 weights
template <class T>
__global__ __launch_bounds__(kThreads) void k_mx4_quantise(const QuantArgs A) {
    const int64_t idx = (int64_t)blockIdx.x * kThreads + threadIdx.x, tile = idx / 64;
    if (tile >= A.tiles) return;
    const int r = (int)(idx % 64) / 2, b = (int)(idx % 2);
    const int64_t kt = col_tiles(A.K), mt = row_tiles(A.M), e = tile / (mt * kt), at = tile - e * mt * kt;
    const int64_t row = at / kt * kTileRows + r, col = at % kt * kTileCols + 32 * b;
    float v[32];
    uint32_t amax = 0;
    for (int i = 0; i < 32; i++) {
        float x = 0;
        if (row < A.M && col + i < A.K) x = to_float<T>(((const T*)A.w)[e * A.expert_stride + row * A.row_stride + col + i]);
        x = x != x ? 0.0f : __builtin_fminf(__builtin_fmaxf(x, -3.402823466e38f), 3.402823466e38f);
        v[i] = x;
        const uint32_t a = __float_as_uint(x) & 0x7fffffffu;
        amax = a > amax ? a : amax;
    }
    // floor(log2) of a normal number is its exponent; smaller numbers are below every base
    int E = (int)(amax >> 23) - 127 - 2;
    E = E > A.base + A.max_shift ? A.base + A.max_shift : E;
    E = E < A.base ? A.base : E;
    const float inv = __uint_as_float((uint32_t)(127 - E) << 23);                                     // E in [-126, 125]
    const float two = __uint_as_float((uint32_t)(127 + E) << 23);
    uint32_t code[4] = {0, 0, 0, 0};
    for (int i = 0; i < 32; i++) {
        const float a = __builtin_fabsf(v[i]) * inv;
        // number of the e2m1 magnitude nearest to a, ties to the even one
        const uint32_t m = (a > 0.25f) + (a >= 0.75f) + (a > 1.25f) + (a >= 1.75f) + (a > 2.5f) + (a >= 3.5f) + (a > 5.0f);
        const uint32_t c = m ? m | (v[i] < 0 ? 8u : 0u) : 0u;
        code[(i & 15) / 4] |= c << (8 * (i & 3) + (i >= 16 ? 4 : 0));
        if (A.values && row < A.M && col + i < A.K) {
            const float mag = m < 4 ? 0.5f * (float)m : m == 7 ? 6.0f : (float)(m - 2);
            ((T*)A.values)[(e * A.M + row) * A.K + col + i] = from_float<T>((v[i] < 0 ? -mag : mag) * two);
        }
    }
    uint8_t* dst = A.out + tile * kMx4Tile;
    *(uint4*)(dst + 32 * r + 16 * b) = make_uint4(code[0], code[1], code[2], code[3]);
    dst[kMx4Codes + 2 * r + b] = (uint8_t)(E - A.base);
}

__device__ __forceinline__ uint32_t signed_mod(int32_t v, const ModInfo& M) {
    const int32_t r = v % (int32_t)M.m;
    return (uint32_t)(r < 0 ? r + (int32_t)M.m : r);
}

// ---- weighted sums -----------------------------------------------------------------------------
struct CombPrime { uint32_t p; LView in, out; };
struct CombArgs {
    const ModInfo* mods;
    const int32_t* gates;
    int64_t n;
    int V, top_k;
    CombPrime pr[DASH_MAX_PRIMES];
};
// a lane per output word; blockIdx.y = prime
__global__ __launch_bounds__(kThreads) void k_combine(const CombArgs A) {
    const CombPrime& P = A.pr[blockIdx.y];
    const ModInfo M = A.mods[P.p];
    const int64_t idx = (int64_t)blockIdx.x * kThreads + threadIdx.x, per = A.n * A.V;
    if (idx >= per * M.nchunk) return;
    const int64_t ch = idx / per, o = idx - ch * per, t = o / A.V, v = o - t * A.V;
    uint32_t acc[16] = {};
    for (int j = 0; j < A.top_k; j++) {
        const uint32_t g = signed_mod(A.gates[t * A.top_k + j], M);
        const uint4 x = *(const uint4*)(P.in.p + ch * P.in.cs + ((t * A.top_k + j) * A.V + v) * 16);
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
        for (int d = 0; d < 16; d++) acc[d] += mul24(g, byte_of(w[d / 4], d % 4));
    }
    uint32_t w[4] = {0, 0, 0, 0};
    for (int d = 0; d < 16; d++) w[d / 4] |= mod_m(acc[d], M) << (8 * (d % 4));
    *(uint4*)(P.out.p + ch * P.out.cs + o * 16) = make_uint4(w[0], w[1], w[2], w[3]);
}

// ---- host side ---------------------------------------------------------------------------------
static int check_bundle(const dash_ctx* c, const dash_labels* t, int64_t n) {
    if (!t || t->n_elem < n) return DASH_EINVAL;
    for (int i = 0; i < c->k; i++)
        if (!t->data[i] || ((uintptr_t)t->data[i] & 15) || (t->chunk_stride[i] & 15) || t->chunk_stride[i] < 16 * n) return DASH_EINVAL;
    return DASH_OK;
}
static uint32_t blocks_of(int64_t lanes) { return (uint32_t)((lanes + kThreads - 1) / kThreads); }
constexpr int64_t kMaxLanes = 0x7fffffffll * kThreads;

int experts_layer(dash_ctx* c, const dash_layer* L, bool garble, const dash_labels* in, dash_labels* out, hipStream_t s) {
    int st = layer_sizes(c, L, nullptr, nullptr, nullptr);
    if (st) return st;
    if (!L->weights || ((uintptr_t)L->weights & 15) || (L->weight_format != DASH_W8 && L->weight_format != DASH_MX4)) return DASH_EINVAL;
    const int64_t n = L->n_elem, T = n / L->top_k;
    const int M = L->out_c, K = L->in_c, E = L->n_experts;
    if (T > 0x7fffffff / K || n > 0x7fffffff / M) return DASH_ESIZE;
    if (L->routing) {
        if (!L->routing->data || L->routing->ctx != c || L->routing->n != n || L->routing->n_experts != E) return DASH_EINVAL;
    } else if (E != 1) return DASH_EINVAL;
    if ((st = check_bundle(c, in, T * K)) || (st = check_bundle(c, out, n * M))) return st;
    // int32 accumulators must not overflow: bytes up to 128 in magnitude on an offset of as much, residues otherwise
    for (int i = 0; i < c->k; i++) {
        const uint64_t p1 = (uint64_t)c->prime[i] - 1, w = L->weight_format == DASH_W8 ? 256 : p1;
        if (w * p1 * (uint64_t)K + p1 >= (1ull << 31)) return DASH_ESIZE;
    }
    if (n == 0) return DASH_OK;
    ExpertsCall call{(const uint8_t*)L->weights, L->bias, nullptr, n, M, K, E, L->top_k, L->weight_format, garble};
    RoutingView R;
    if (L->routing) { R = routing_view(c, L->routing->data, n, E); call.routing = &R; }
    return experts_mfma(c, call, in, out, s);
}

int combine_layer(dash_ctx* c, const dash_layer* L, const dash_labels* in, dash_labels* out, hipStream_t s) {
    int st = layer_sizes(c, L, nullptr, nullptr, nullptr);
    if (st) return st;
    if (L->top_k > 1024) return DASH_ESIZE;            // (p - 1)^2 top_k below 2^24: one step to the residue
    const int64_t n = L->n_elem;
    const int V = L->in_c;
    if (!L->gates) return DASH_EINVAL;
    if (n > 0x7fffffff / V / L->top_k) return DASH_ESIZE;
    if ((st = check_bundle(c, in, n * L->top_k * V)) || (st = check_bundle(c, out, n * V))) return st;
    if (n == 0) return DASH_OK;
    CombArgs A;
    memset(&A, 0, sizeof(A));
    A.mods = c->d_mods; A.gates = L->gates; A.n = n; A.V = V; A.top_k = L->top_k;
    int64_t lanes = 0;
    double macs = 0, bytes = 0;
    for (int i = 0; i < c->k; i++) {
        const ModInfo& Mi = c->mods[c->prime[i]];
        A.pr[i] = CombPrime{(uint32_t)c->prime[i], view_of(in, i), view_of(out, i)};
        lanes = n * V * Mi.nchunk > lanes ? n * V * Mi.nchunk : lanes;
        macs += (double)n * V * L->top_k * Mi.lam;
        bytes += (double)n * V * (L->top_k + 1) * Mi.lam;
    }
    ProfScope ps(c->prof, DASH_PROF_LINEAR, s, macs, bytes);
    hipLaunchKernelGGL(k_combine, dim3(blocks_of(lanes), c->k), dim3(kThreads), 0, s, A);
    DASH_HIP(hipGetLastError());
    return DASH_OK;
}

// tiles of n_experts matrices whose rows and experts lie row_stride and expert_stride elements apart; 0: refused
static int64_t weight_tiles(const void* w, int64_t row_stride, int64_t expert_stride, int n_experts, int out_c, int K, const void* prepared) {
    if (!w || !prepared || ((uintptr_t)prepared & 15) || n_experts < 1 || out_c < 1 || K < 1 || row_stride < K || expert_stride < 0) return 0;
    return row_tiles(out_c) * col_tiles(K) * n_experts;
}

}  // namespace dash

using namespace dash;

extern "C" {

size_t dash_expert_weights_bytes(int format, int n_experts, int out_c, int K) {
    if ((format != DASH_W8 && format != DASH_MX4) || n_experts < 1 || out_c < 1 || K < 1) return 0;
    return (size_t)n_experts * (size_t)matrix_bytes(format, out_c, K);
}

int dash_weights8_prepare(dash_ctx* c, const int8_t* w, int64_t row_stride, int64_t expert_stride, int n_experts, int out_c, int K, void* prepared,
                          void* stream) {
    if (!c) return DASH_EINVAL;
    const int64_t tiles = weight_tiles(w, row_stride, expert_stride, n_experts, out_c, K, prepared);
    if (!tiles) return DASH_EINVAL;
    const int64_t lanes = tiles * (kW8Tile / 16);
    if (lanes > kMaxLanes) return DASH_ESIZE;
    const PrepArgs8 A{w, row_stride, expert_stride, tiles, out_c, K, (uint8_t*)prepared};
    hipLaunchKernelGGL(k_weights8_prepare, dim3(blocks_of(lanes)), dim3(kThreads), 0, (hipStream_t)stream, A);
    DASH_HIP(hipGetLastError());
    return DASH_OK;
}

int dash_mx4_quantise(dash_ctx* c, const void* w, int dtype, int64_t row_stride, int64_t expert_stride, int n_experts, int out_c, int K, int base,
                      int max_shift, void* prepared, void* values, void* stream) {
    if (!c || dtype < DASH_F32 || dtype > DASH_F16 || base < -126 || base > 125 || max_shift < 0 || max_shift > 255) return DASH_EINVAL;
    const uintptr_t unaligned = dtype == DASH_F32 ? 3 : 1;
    if (((uintptr_t)w & unaligned) || ((uintptr_t)values & unaligned)) return DASH_EINVAL;
    const int64_t tiles = weight_tiles(w, row_stride, expert_stride, n_experts, out_c, K, prepared);
    if (!tiles) return DASH_EINVAL;
    const int64_t lanes = tiles * 64;
    if (lanes > kMaxLanes) return DASH_ESIZE;
    const QuantArgs A{w, row_stride, expert_stride, tiles, out_c, K, base, max_shift, (uint8_t*)prepared, values};
    auto kernel = dtype == DASH_F32 ? k_mx4_quantise<float> : dtype == DASH_BF16 ? k_mx4_quantise<__hip_bfloat16> : k_mx4_quantise<_Float16>;
    hipLaunchKernelGGL(kernel, dim3(blocks_of(lanes)), dim3(kThreads), 0, (hipStream_t)stream, A);
    DASH_HIP(hipGetLastError());
    return DASH_OK;
}

size_t dash_route_bytes(const dash_ctx* c, int64_t n, int n_experts) {
    if (!c || n < 0 || n > 0x7fffffff || n_experts < 1 || n_experts > kMaxExperts) return 0;
    const RoutingView v = routing_view(c, nullptr, n, n_experts);
    for (int s = 0; s < kTileSizes; s++) if (v.max_tiles[s] > 0x7fffffff) return 0;
    return v.bytes;
}

int dash_route(dash_ctx* c, const int32_t* experts, int64_t n, int n_experts, void* data, dash_routing* routing, void* stream) {
    if (!c || !data || ((uintptr_t)data & 15) || !routing || n < 0 || n_experts < 1 || (n > 0 && !experts)) return DASH_EINVAL;
    if (!dash_route_bytes(c, n, n_experts)) return DASH_ESIZE;
    RouteArgs A;
    memset(&A, 0, sizeof(A));
    A.experts = experts; A.n = n; A.E = n_experts; A.k = c->k;
    for (int i = 0; i < c->k; i++) A.nchunk[i] = (uint8_t)c->mods[c->prime[i]].nchunk;
    A.to = routing_view(c, data, n, n_experts);
    const dim3 grid((uint32_t)((n_experts + 1 + kWaves - 1) / kWaves));
    hipLaunchKernelGGL(k_route_count, grid, dim3(kThreads), 0, (hipStream_t)stream, A);
    hipLaunchKernelGGL(k_route_scan, dim3(1), dim3(kThreads), 0, (hipStream_t)stream, A);
    hipLaunchKernelGGL(k_route_fill, grid, dim3(kThreads), 0, (hipStream_t)stream, A);
    DASH_HIP(hipGetLastError());
    routing->data = data; routing->ctx = c; routing->n = n; routing->n_experts = n_experts;
    return DASH_OK;
}

}  // extern "C"
