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
//   k_f8_quantise, k_f8_scales    : weights to 8-bit floats with an integer scale for every 128 x 128, into the same tiles as bytes
//   (the products: dash_experts_gemm.hip)
//   k_combine                     : the weighted sums
#include <math.h>
#include <string.h>

#include "dash_experts.h"
#include "dash_experts_rule.h"

namespace dash {

constexpr int kWaves = kThreads / 64;

// ---- routing -----------------------------------------------------------------------------------
// Three launches, once for all layers over the same rows; no atomics, so that the order is the same every time.  Bound by latency: 11 us for 1 to 16 rows, 17 us for 1000 rows of 64 experts, 52 for 10000; from there the waves that walk all rows, 500 us for 100000 rows of 8 or 4096 experts.
// A lane counts the tiles of one (kind, part of the primes) instead of the wave one after the other, 8 of the rows' loads are under way instead of one (16, 23, 77, 880 to 970 us
// with five kinds of tiles, 27, 36, 91, 970 to 1040 with eight).
constexpr int kMaxPairs = 128;
static_assert(2 + 6 * DASH_MAX_PRIMES <= kMaxPairs && kTileKinds <= 8, "pairs of a tile kind and a part of the primes");
struct RouteArgs {
    const int32_t* experts;
    int64_t n;
    int E, pairs;
    int kind_first[kTileKinds + 1];                 // first pair of every kind
    struct { uint8_t kind, part; uint16_t first, last; } pair[kMaxPairs];        // a kind's tiles of the chunks first .. last - 1
    RoutingView to;
};
__device__ __forceinline__ bool route_match(int32_t id, int e, int E) { return e < E ? id == e : (uint32_t)id >= (uint32_t)E; }
// Which of the rows r0 + 64 i + lane are of expert e: the loads of a step are under way together, as nothing else hides their latency
constexpr int kRouteRows = 8;
__device__ __forceinline__ void route_hits(const RouteArgs& A, int64_t r0, int e, int lane, bool (&hit)[kRouteRows]) {
    int32_t id[kRouteRows];
#pragma unroll
    for (int i = 0; i < kRouteRows; i++) id[i] = A.experts[r0 + 64 * i + lane < A.n ? r0 + 64 * i + lane : 0];
#pragma unroll
    for (int i = 0; i < kRouteRows; i++) hit[i] = r0 + 64 * i + lane < A.n && route_match(id[i], e, A.E);
}
__device__ __forceinline__ int32_t wave_scan(int32_t v, int lane) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) { const int32_t o = __shfl_up(v, d); v += lane >= d ? o : 0; }
    return v;
}
// Tiles that an expert of `rows` rows has before every pair: to[0 .. pairs] (a wave's own; a lane per pair)
__device__ __forceinline__ void route_pairs(const RouteArgs& A, int32_t rows, int lane, int32_t* to) {
    int32_t before = 0;
    for (int q0 = 0; q0 < A.pairs; q0 += 64) {
        const int q = q0 + lane;
        int32_t t = 0;
        if (q < A.pairs) {
            const auto P = A.pair[q];
            const int groups = kTileKind[P.kind].groups;
            t = (int32_t)(((int64_t)rows * (P.last - P.first) + groups - 1) / groups);
        }
        const int32_t up_to = before + wave_scan(t, lane);
        if (q < A.pairs) to[q] = up_to - t;
        before = __shfl(up_to, 63);
    }
    if (lane == 0) to[A.pairs] = before;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// A wave per expert (E + 1 of them: the last is "none") counts its rows and its tiles of every kind.
__global__ __launch_bounds__(kThreads) void k_route_count(const RouteArgs A) {
    __shared__ int32_t s_pairs[kWaves][kMaxPairs + 1];
    const int e = (int)(blockIdx.x * kWaves + threadIdx.x / 64), lane = threadIdx.x & 63;
    if (e > A.E) return;
    int32_t count = 0;
    for (int64_t r0 = 0; r0 < A.n; r0 += 64 * kRouteRows) {
        bool hit[kRouteRows];
        route_hits(A, r0, e, lane, hit);
#pragma unroll
        for (int i = 0; i < kRouteRows; i++) count += __popcll(__ballot(hit[i]));
    }
    int32_t* const first = s_pairs[threadIdx.x / 64];
    route_pairs(A, count, lane, first);
    if (lane == 0) A.to.offsets[e + 1] = count;
    if (lane < kTileKinds) A.to.first_tile[lane][e + 1] = first[A.kind_first[lane + 1]] - first[A.kind_first[lane]];
}
// One block: counts to offsets and to first tiles.
__global__ __launch_bounds__(kThreads) void k_route_scan(const RouteArgs A) {
    __shared__ int32_t part[1 + kTileKinds][kThreads];
    const int n = A.E + 1, per = (n + kThreads - 1) / kThreads, e0 = threadIdx.x * per, e1 = e0 + per < n ? e0 + per : n;
    int32_t sum[1 + kTileKinds] = {};
    for (int e = e0; e < e1; e++) {
        sum[0] += A.to.offsets[e + 1];
        for (int s = 0; s < kTileKinds; s++) sum[1 + s] += A.to.first_tile[s][e + 1];
    }
    for (int s = 0; s < 1 + kTileKinds; s++) part[s][threadIdx.x] = sum[s];
    __syncthreads();
    // a wave per sum, four threads' parts a lane
    const int lane = threadIdx.x & 63;
    for (int s = threadIdx.x / 64; s < 1 + kTileKinds; s += kWaves) {
        int32_t v[kWaves], all = 0;
        for (int i = 0; i < kWaves; i++) { v[i] = part[s][lane * kWaves + i]; all += v[i]; }
        int32_t at = wave_scan(all, lane) - all;
        for (int i = 0; i < kWaves; i++) { part[s][lane * kWaves + i] = at; at += v[i]; }
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        A.to.offsets[0] = 0;
        for (int s = 0; s < kTileKinds; s++) A.to.first_tile[s][0] = 0;
    }
    for (int s = 0; s < 1 + kTileKinds; s++) sum[s] = part[s][threadIdx.x];
    for (int e = e0; e < e1; e++) {
        sum[0] += A.to.offsets[e + 1];
        A.to.offsets[e + 1] = sum[0];
        for (int s = 0; s < kTileKinds; s++) { sum[1 + s] += A.to.first_tile[s][e + 1]; A.to.first_tile[s][e + 1] = sum[1 + s]; }
    }
}
// The wave of an expert writes its rows in ascending order, and its tiles, a lane each.
__global__ __launch_bounds__(kThreads) void k_route_fill(const RouteArgs A) {
    __shared__ int32_t s_pairs[kWaves][kMaxPairs + 1];
    const int e = (int)(blockIdx.x * kWaves + threadIdx.x / 64), lane = threadIdx.x & 63;
    if (e > A.E) return;
    const int32_t start = A.to.offsets[e], count = A.to.offsets[e + 1] - start;
    int32_t at = start;
    for (int64_t r0 = 0; r0 < A.n; r0 += 64 * kRouteRows) {
        bool hit[kRouteRows];
        route_hits(A, r0, e, lane, hit);
#pragma unroll
        for (int i = 0; i < kRouteRows; i++) {
            const uint64_t m = __ballot(hit[i]);
            if (hit[i]) A.to.rows[at + __popcll(m & ((1ull << lane) - 1))] = (int32_t)(r0 + 64 * i + lane);
            at += __popcll(m);
        }
    }
    int32_t* const first = s_pairs[threadIdx.x / 64];
    route_pairs(A, count, lane, first);
    if (first[A.pairs] > 16 * A.pairs) {            // many tiles: pair after pair (0.3 us each) instead of a search (1 us for 64 tiles)
        for (int q = 0; q < A.pairs; q++) {
            const auto P = A.pair[q];
            const int s = P.kind, groups = kTileKind[s].groups;
            RouteTile* const to = A.to.tiles[s] + A.to.first_tile[s][e] + first[q] - first[A.kind_first[s]];
            for (int32_t t = lane; t < first[q + 1] - first[q]; t += 64)
                to[t] = RouteTile{(uint32_t)e | (uint32_t)P.part << 24, start, count, P.first * count + t * groups};
        }
        return;
    }
    struct Pair { RouteTile* to; int32_t block; uint16_t part, groups; };           // where tile i of the expert goes, less i
    __shared__ Pair s_to[kWaves][kMaxPairs];
    Pair* const to = s_to[threadIdx.x / 64];
    for (int q = lane; q < A.pairs; q += 64) {
        const auto P = A.pair[q];
        const int s = P.kind;
        to[q] = Pair{A.to.tiles[s] + A.to.first_tile[s][e] - first[A.kind_first[s]], P.first * count, P.part, (uint16_t)kTileKind[s].groups};
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    for (int32_t i = lane; i < first[A.pairs]; i += 64) {
        int q = 0;                                  // the last pair that begins at i or before (of those of no tiles, the one behind them)
#pragma unroll
        for (int d = kMaxPairs / 2; d; d /= 2) if (q + d < A.pairs && first[q + d] <= i) q += d;
        const Pair P = to[q];
        P.to[i] = RouteTile{(uint32_t)e | (uint32_t)P.part << 24, start, count, P.block + (i - first[q]) * P.groups};
    }
}

// ---- weights -----------------------------------------------------------------------------------
struct PrepArgs8 {
    const int8_t* w;
    int64_t row_stride, expert_stride, tiles;       // tiles of all experts
    int64_t first;                                  // the launch's first lane
    int64_t expert_bytes;                           // of a prepared matrix
    int M, K, f8;
    uint8_t* out;
};
// a lane per 16-byte piece of a tile
__global__ __launch_bounds__(kThreads) void k_weights8_prepare(const PrepArgs8 A) {
    const int64_t idx = A.first + (int64_t)blockIdx.x * kThreads + threadIdx.x, tile = idx / (kW8Tile / 16);
    if (tile >= A.tiles) return;
    const int piece = (int)(idx % (kW8Tile / 16)), r = piece / 4, q = piece % 4;
    const int64_t kt = col_tiles(A.K), mt = row_tiles(A.M), e = tile / (mt * kt), at = tile - e * mt * kt;
    const int64_t row = at / kt * kTileRows + r, col = at % kt * kTileCols + 16 * q;
    uint32_t v[4] = {0, 0, 0, 0};
    if (row < A.M) {
        const int8_t* src = A.w + e * A.expert_stride + row * A.row_stride + col;
        if (col + 16 <= A.K) __builtin_memcpy(v, src, 16);          // (at any address)
        else
            for (int i = 0; i < 16; i++)
                if (col + i < A.K) v[i / 4] |= (uint32_t)(uint8_t)src[i] << (8 * (i % 4));
        if (A.f8)
            for (int i = 0; i < 4; i++) {
                // codes of no number (all seven bits) to zeros: the carry of 1 to the sign's place, and 0x80 - 1 with it
                const uint32_t none = ((v[i] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
                v[i] &= ~(none | (none - (none >> 7)));
            }
    }
    *(uint4*)(A.out + e * A.expert_bytes + at * kW8Tile + w8_at(r, 16 * q)) = make_uint4(v[0], v[1], v[2], v[3]);
}

struct QuantArgs {
    const void* w;
    int64_t row_stride, expert_stride;
    uint32_t first;             // the launch's first tile
    int M, K, base, max_shift;
    uint8_t* out;
    void* values;
};
typedef float v2f __attribute__((ext_vector_type(2)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef uint16_t v8s __attribute__((ext_vector_type(8)));
// V elements of a lane (16 bytes, at any address) as floats, and back
struct QuantF32 {
    static constexpr int V = 4;
    typedef float T;
    typedef v4f Vec;
    typedef v4f VecAny __attribute__((aligned(4)));
    static __device__ __forceinline__ float to(float v) { return v; }
    static __device__ __forceinline__ float from(float v) { return v; }
    static __device__ __forceinline__ float round(float v) { return v; }
};
struct QuantBF16 {
    static constexpr int V = 8;
    typedef uint16_t T;
    typedef v8s Vec;
    typedef v8s VecAny __attribute__((aligned(2)));
    static __device__ __forceinline__ float to(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
    static __device__ __forceinline__ uint16_t from(float v) { return (uint16_t)(__float_as_uint(v) >> 16); }       // two significant bits: exact
    static __device__ __forceinline__ uint16_t round(float v) { const uint32_t b = __float_as_uint(v); return (uint16_t)((b + 0x7fffu + (b >> 16 & 1)) >> 16); }     // to the nearest, ties to the even
};
struct QuantF16 {
    static constexpr int V = 8;
    typedef uint16_t T;
    typedef v8s Vec;
    typedef v8s VecAny __attribute__((aligned(2)));
    static __device__ __forceinline__ float to(uint16_t v) { return (float)__builtin_bit_cast(_Float16, v); }
    static __device__ __forceinline__ uint16_t from(float v) { return __builtin_bit_cast(uint16_t, (_Float16)v); }
    static __device__ __forceinline__ uint16_t round(float v) { return from(v); }
};
// nibbles 0..3 of n to the low halves of the four bytes
__device__ __forceinline__ uint32_t spread4(uint32_t n) {
    n = (n | n << 8) & 0x00ff00ffu;
    return (n | n << 4) & 0x0f0f0f0fu;
}

// A block per tile of 32 rows x 64 columns, 8 rows a wave (a wave for all 32 rows ran four times the code in a row: 4096 x 4096 as fast,
// matrices of a few tiles 6.9 us instead of 4.1): a lane reads 16 bytes of a row (V weights), the 32 / V lanes of a block find its largest
// magnitude among themselves, v_cvt_scalef32_pk_fp4_f32 rounds two weights at a time (nearest, ties to even, saturating).  Codes and
// shifts go through LDS, so that a tile is written 16 bytes a lane.  Bound by HBM: 4096 x 4096 bfloat16 with the values written, 76 MB, in 13.0 us
// (5.8 TB/s; a large copy moves 4.9).  (A lane per block of 32 weights, each walking its own cache lines with scalar loads: 111 us.)
template <class Q>
__global__ __launch_bounds__(kThreads) void k_mx4_quantise(const QuantArgs A) {
    constexpr int V = Q::V, kLanes = 32 / V, kRowLanes = 64 / V, kRows = 64 / kRowLanes, kSteps = kTileRows / kWaves / kRows;      // lanes of a block, of a row; rows at a time
    typedef typename Q::T T;
    __shared__ __attribute__((aligned(16))) uint8_t to[kMx4Tile];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t tile = A.first + blockIdx.x;
    const uint32_t kt = (uint32_t)col_tiles(A.K), mt = (uint32_t)row_tiles(A.M);
    const uint32_t rt = tile / kt, e = rt / mt;
    const int r0 = wave * (kTileRows / kWaves) + lane / kRowLanes;
    const int row0 = (int)(rt - e * mt) * kTileRows + r0, col = (int)(tile - rt * kt) * kTileCols + lane % kRowLanes * V;
    const T* const src = (const T*)A.w + (int64_t)e * A.expert_stride;
    const int have = A.K - col;                      // columns from the lane's first to the end
    // all loads go out before the first is waited for: no branch but the one on the tile; rows and columns past the end read the last
    typename Q::Vec in[kSteps];
    if (columns_inside((int)(tile - rt * kt) * kTileCols, kTileCols, A.K)) {
#pragma unroll
        for (int s = 0; s < kSteps; s++) {
            const int row = row0 + kRows * s < A.M ? row0 + kRows * s : A.M - 1;
            in[s] = *(const typename Q::VecAny*)(src + (int64_t)row * A.row_stride + col);
        }
    } else {
#pragma unroll
        for (int s = 0; s < kSteps; s++) {
            const int row = row0 + kRows * s < A.M ? row0 + kRows * s : A.M - 1;
#pragma unroll
            for (int i = 0; i < V; i++) in[s][i] = src[(int64_t)row * A.row_stride + (i < have ? col + i : A.K - 1)];
        }
    }
    T* const values = A.values ? (T*)A.values + ((int64_t)e * A.M + row0) * A.K + col : nullptr;
#pragma unroll
    for (int s = 0; s < kSteps; s++) {
        float x[V];
        uint32_t amax = 0;
#pragma unroll
        for (int i = 0; i < V; i++) {
            x[i] = Q::to(in[s][i]);
            x[i] = x[i] == x[i] && i < have && row0 + kRows * s < A.M ? x[i] : 0.0f;
            const uint32_t a = __float_as_uint(x[i]) & 0x7fffffffu;
            amax = a > amax ? a : amax;
        }
#pragma unroll
        for (int d = kLanes / 2; d; d /= 2) {
            const uint32_t o = d == 4 ? (uint32_t)__builtin_amdgcn_ds_swizzle((int)amax, (4 << 10) | 0x1f)                              // lane ^ 4
                             : d == 2 ? (uint32_t)__builtin_amdgcn_update_dpp(0, (int)amax, 0x4E, 0xf, 0xf, true)                       // quad_perm:[2,3,0,1]
                                      : (uint32_t)__builtin_amdgcn_update_dpp(0, (int)amax, 0xB1, 0xf, 0xf, true);                      // quad_perm:[1,0,3,2]
            amax = o > amax ? o : amax;
        }
        // floor(log2) of a normal number is its exponent; smaller numbers are below every base, an infinity counts as the largest number
        int E = (int)(amax >> 23) - 127 - 2;
        E = E > 125 ? 125 : E;
        E = E > A.base + A.max_shift ? A.base + A.max_shift : E;
        E = E < A.base ? A.base : E;
        const float two = __uint_as_float((uint32_t)(127 + E) << 23);                                                 // E in [-126, 125]
        uint32_t n = 0;
        n = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(n, x[0], x[1], two, 0);
        n = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(n, x[2], x[3], two, 1);
        if constexpr (V == 8) {
            n = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(n, x[4], x[5], two, 2);
            n = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(n, x[6], x[7], two, 3);
        }
        n &= 0x77777777u | ((n | n >> 1 | n >> 2) & 0x11111111u) << 3;                                                // no sign of a zero
        const int r = r0 + kRows * s, b = lane % kRowLanes / kLanes, at = lane % kLanes;
        // the lanes of a row's first block take the codes of its second into the high halves
        if constexpr (V == 4) {
            const uint32_t c = spread4(n), o = (uint32_t)__builtin_amdgcn_ds_swizzle((int)c, (8 << 10) | 0x1f);             // lane ^ 8
            if (b == 0) *(uint32_t*)(to + 32 * r + 4 * at) = c | o << 4;
        } else {
            const uint32_t c0 = spread4(n & 0xffffu), c1 = spread4(n >> 16);
            const uint32_t o0 = (uint32_t)__builtin_amdgcn_ds_swizzle((int)c0, (4 << 10) | 0x1f), o1 = (uint32_t)__builtin_amdgcn_ds_swizzle((int)c1, (4 << 10) | 0x1f);
            if (b == 0) *(uint2*)(to + 32 * r + 8 * at) = make_uint2(c0 | o0 << 4, c1 | o1 << 4);
        }
        if (at == 0) to[kMx4Codes + 2 * r + b] = (uint8_t)(E - A.base);
        if (values && row0 + kRows * s < A.M) {
            typename Q::Vec out;
            const v2f v0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(n, two, 0), v1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(n, two, 1);
            out[0] = Q::from(v0[0]); out[1] = Q::from(v0[1]); out[2] = Q::from(v1[0]); out[3] = Q::from(v1[1]);
            if constexpr (V == 8) {
                const v2f v2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(n, two, 2), v3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(n, two, 3);
                out[4] = Q::from(v2[0]); out[5] = Q::from(v2[1]); out[6] = Q::from(v3[0]); out[7] = Q::from(v3[1]);
            }
            T* const p = values + (int64_t)(kRows * s) * A.K;
            if (have >= V) *(typename Q::VecAny*)p = out;
            else
#pragma unroll
                for (int i = 0; i < V - 1; i++) if (i < have) p[i] = out[i];
        }
    }
    __syncthreads();
    uint8_t* const dst = A.out + (int64_t)tile * kMx4Tile;
    if (threadIdx.x < kMx4Tile / 16) *(uint4*)(dst + 16 * threadIdx.x) = *(const uint4*)(to + 16 * threadIdx.x);
}

constexpr int kF8Threads = 512;
struct QuantF8Args {
    const void* w;
    int64_t row_stride, expert_stride, expert_bytes;
    uint32_t first;             // the launch's first block of 128 x 128
    int M, K, max_scale;
    float unit, inverse;        // 2^base, 2^-base
    uint8_t* out;
    void* values;
};
// A block per 128 x 128 weights: they are read once, 16 bytes a lane, all loads out before the first is waited for, and stay in registers while the block finds its largest
// magnitude.  Quotients: with y = 1 / S rounded to nearest, q = x y and the remainder x - q S, exact, q + (x - q S) y is x / S rounded to nearest (Markstein); of 24 bits by
// 15 that is the middle of two e4m3 values only where x / S is.  v_cvt_pk_fp8_f32 rounds two at a time (nearest, ties to even); a lane's codes are neighbours in their tile.
// Bound by HBM: 4096 x 4096 bfloat16 in 15.7 us, 5.35 TB/s with the values written (74 us with a block's weights read twice, an element a lane); 10 x 128: 5.6 us, a launch and the
// chain of loads, maximum and stores.  values may be the weights themselves: a block has read its own before it writes.
template <class Q>
__global__ __launch_bounds__(kF8Threads) void k_f8_quantise(const QuantF8Args A) {
    constexpr int V = Q::V, kRowLanes = kScaleBlock / V, kRows = kF8Threads / kRowLanes, kSteps = kScaleBlock / kRows;
    typedef typename Q::T T;
    typedef typename Q::VecAny VecAny;
    const uint32_t block = A.first + blockIdx.x, kb = (uint32_t)scale_blocks(A.K), mb = (uint32_t)scale_blocks(A.M);
    const uint32_t rb = block / kb, e = rb / mb;
    const int row0 = (int)(rb - e * mb) * kScaleBlock, col0 = (int)(block - rb * kb) * kScaleBlock;
    const int r0 = threadIdx.x / kRowLanes, col = col0 + (int)threadIdx.x % kRowLanes * V, have = A.K - col;
    const int rows = A.M - row0 < kScaleBlock ? A.M - row0 : kScaleBlock;
    const T* const src = (const T*)A.w + (int64_t)e * A.expert_stride + (int64_t)row0 * A.row_stride;
    __shared__ uint32_t part[kF8Threads / 64];
    typename Q::Vec in[kSteps];
    if (columns_inside(col0, kScaleBlock, A.K)) {
#pragma unroll
        for (int s = 0; s < kSteps; s++)
            if (s * kRows < rows) in[s] = *(const VecAny*)(src + (int64_t)(r0 + s * kRows < rows ? r0 + s * kRows : rows - 1) * A.row_stride + col);
    } else {
#pragma unroll
        for (int s = 0; s < kSteps; s++)
            if (s * kRows < rows) {
#pragma unroll
                for (int i = 0; i < V; i++) in[s][i] = src[(int64_t)(r0 + s * kRows < rows ? r0 + s * kRows : rows - 1) * A.row_stride + (i < have ? col + i : A.K - 1)];
            }
    }
    // (rows and columns past the end repeat others: the magnitude is theirs)
    auto number = [](float x) __attribute__((always_inline)) { return x == x ? x : 0.0f; };
    float top = 0;
#pragma unroll
    for (int s = 0; s < kSteps; s++)
        if (s * kRows < rows) {
#pragma unroll
            for (int i = 0; i < V; i++) top = fmaxf(top, fabsf(Q::to(in[s][i])));       // (fmaxf leaves out what is not a number)
        }
    uint32_t amax = __float_as_uint(top);
#pragma unroll
    for (int d = 32; d; d /= 2) {
        const uint32_t o = d == 2 ? (uint32_t)__builtin_amdgcn_update_dpp(0, (int)amax, 0x4E, 0xf, 0xf, true) : d == 1 ? (uint32_t)__builtin_amdgcn_update_dpp(0, (int)amax, 0xB1, 0xf, 0xf, true)
                         : (uint32_t)__shfl_xor((int)amax, d);
        amax = o > amax ? o : amax;
    }
    if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = amax;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kF8Threads / 64; i++) amax = part[i] > amax ? part[i] : amax;
    amax = (uint32_t)__builtin_amdgcn_readfirstlane((int)amax);
    // the smallest S with 448 S >= a: 448 * 32767 < 2^24, so both sides are exact
    const float a = fminf(__uint_as_float(amax), 3.4028234663852886e38f) * A.inverse;
    float S = fminf(ceilf(a / 448.0f), (float)A.max_scale);
    if (S > 1 && 448.0f * (S - 1) >= a) S -= 1;
    if (448.0f * S < a) S += 1;
    S = fminf(fmaxf(S, 1.0f), (float)A.max_scale);
    uint8_t* const out = A.out + (int64_t)e * A.expert_bytes;
    if (threadIdx.x == 0) ((int32_t*)(out + scales_at(A.M, A.K)))[(rb - e * mb) * kb + (block - rb * kb)] = (int32_t)S;
    const int64_t kt = col_tiles(A.K);
    const float y = 1.0f / S, most = 448.0f * S, unit = S * A.unit;
    const int tile_rows = (rows + kTileRows - 1) / kTileRows * kTileRows;
    const bool tile_there = col / kTileCols < kt;
    T* const values = A.values ? (T*)A.values + ((int64_t)e * A.M + row0) * A.K + col : nullptr;
#pragma unroll
    for (int s = 0; s < kSteps; s++) {
        if (s * kRows >= tile_rows) break;
        const int r = r0 + s * kRows;
        uint32_t n[V / 4];
#pragma unroll
        for (int i = 0; i < V; i += 4) {
            float q[4];
#pragma unroll
            for (int j = 0; j < 4; j++) {
                const float w = number(Q::to(in[s][i + j])), x = fminf(fmaxf((i + j < have && r < rows ? w : 0.0f) * A.inverse, -most), most), q0 = x * y;
                q[j] = fmaf(fmaf(-q0, S, x), y, q0);
            }
            uint32_t c = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false);
            c = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], (int)c, true);
            n[i / 4] = c & (0x7f7f7f7fu | ((c & 0x7f7f7f7fu) + 0x7f7f7f7fu));          // no sign of a zero
        }
        if (r < tile_rows && tile_there)
            __builtin_memcpy(out + ((int64_t)((row0 + r) / kTileRows) * kt + col / kTileCols) * kW8Tile + w8_at(r % kTileRows, col % kTileCols), n, V);
        if (values && r < rows) {
            typename Q::Vec v;
#pragma unroll
            for (int i = 0; i < V; i += 4) {
                const v2f lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)n[i / 4], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)n[i / 4], true);
                v[i] = Q::round(lo[0] * unit); v[i + 1] = Q::round(lo[1] * unit); v[i + 2] = Q::round(hi[0] * unit); v[i + 3] = Q::round(hi[1] * unit);
            }
            T* const p = values + (int64_t)r * A.K;
            if (have >= V) *(VecAny*)p = v;
            else
#pragma unroll
                for (int i = 0; i < V - 1; i++) if (i < have) p[i] = v[i];
        }
    }
}
struct ScalesArgs {
    const int32_t* scales;
    int64_t at, expert_bytes;   // of the scales in a matrix; bytes of a matrix
    int64_t first, total;
    uint32_t blocks;            // of a matrix
    uint8_t* out;
};
__global__ __launch_bounds__(kThreads) void k_f8_scales(const ScalesArgs A) {
    const int64_t i = A.first + (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (i >= A.total) return;
    const int64_t e = i / A.blocks;
    ((int32_t*)(A.out + e * A.expert_bytes + A.at))[i - e * A.blocks] = A.scales[i];
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
    int64_t first, n;           // the launch's first lane; batch elements
    int V, top_k;
    CombPrime pr[DASH_MAX_PRIMES];
};
// A lane per output word: the top_k words of its inputs are neighbours of its neighbours' and each is read once.  blockIdx.y = prime.  Bound by
// HBM: four rows each of 128 batch elements, 4096 values, 12 primes, 1.64 GB, in 287 us (5.7 TB/s).
__global__ __launch_bounds__(kThreads) void k_combine(const CombArgs A) {
    const CombPrime& P = A.pr[blockIdx.y];
    const ModInfo M = A.mods[P.p];
    const int64_t idx = A.first + (int64_t)blockIdx.x * kThreads + threadIdx.x, per = A.n * A.V;
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
constexpr int64_t kMaxLanes = 0x7fffffffll * kThreads;
// launch(first, n) for blocks first .. first + n - 1: a direction of a grid holds fewer than 2^32 threads.  (A second direction instead, with the
// grid's size read by the kernel: 84 values, 16 batch elements: 4.3 -> 4.5 us a call; quantisation of 4096 x 4096: 13.65 -> 13.9.)
template <int Threads = kThreads, class Launch> static void in_launches(int64_t blocks, Launch launch) {
    constexpr int64_t most = 0xffffffffll / Threads;
    for (int64_t first = 0; first < blocks; first += most) launch(first, (uint32_t)(blocks - first < most ? blocks - first : most));
}

static bool weight_format(int f) { return f == DASH_W8 || f == DASH_MX4 || f == DASH_F8; }

int experts_layer(dash_ctx* c, const dash_layer* L, bool garble, const dash_labels* in, dash_labels* out, hipStream_t s) {
    int st = layer_sizes(c, L, nullptr, nullptr, nullptr);
    if (st) return st;
    if (L->n_elem == 0) return DASH_OK;         // (empty bundles and gates may have no address)
    if (!L->weights || ((uintptr_t)L->weights & 15) || !weight_format(L->weight_format)) return DASH_EINVAL;
    const int64_t n = L->n_elem, T = n / L->top_k;
    const int M = L->out_c, K = L->in_c, E = L->n_experts;
    // (offsets inside a row of weights or a row's labels, and the ends of blocks of 256 outputs: 32 bits)
    if (T > 0x7fffffff / K || n > 0x7fffffff / M || K > 1 << 26 || M > 0x7fffffff - 255) return DASH_ESIZE;
    if (L->routing) {
        if (!L->routing->data || L->routing->ctx != c || L->routing->n != n || L->routing->n_experts != E) return DASH_EINVAL;
    } else if (E != 1) return DASH_EINVAL;
    if ((st = check_bundle(c, in, T * K)) || (st = check_bundle(c, out, n * M))) return st;
    // int32 accumulators must not overflow: bytes up to 128 in magnitude on an offset of as much, residues otherwise
    for (int i = 0; i < c->k; i++) {
        const uint64_t p1 = (uint64_t)c->prime[i] - 1, w = L->weight_format == DASH_MX4 ? p1 : 256;
        if (w * p1 * (uint64_t)K + p1 >= (1ull << 31)) return DASH_ESIZE;
    }
    ExpertsCall call{(const uint8_t*)L->weights, L->bias, nullptr, n, M, K, E, L->top_k, L->weight_format, garble};
    RoutingView R;
    if (L->routing) { R = routing_view(c, L->routing->data, n, E); call.routing = &R; }
    return experts_mfma(c, call, in, out, s);
}

int combine_layer(dash_ctx* c, const dash_layer* L, const dash_labels* in, dash_labels* out, hipStream_t s) {
    int st = layer_sizes(c, L, nullptr, nullptr, nullptr);
    if (st) return st;
    if (L->n_elem == 0) return DASH_OK;         // (empty bundles and gates may have no address)
    if (L->top_k > 1024) return DASH_ESIZE;            // (p - 1)^2 top_k below 2^24: one step to the residue
    const int64_t n = L->n_elem;
    const int V = L->in_c;
    if (!L->gates) return DASH_EINVAL;
    if (n > 0x7fffffff / V / L->top_k) return DASH_ESIZE;
    if ((st = check_bundle(c, in, n * L->top_k * V)) || (st = check_bundle(c, out, n * V))) return st;
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
    in_launches((lanes + kThreads - 1) / kThreads, [&](int64_t first, uint32_t blocks) {
        A.first = first * kThreads;
        hipLaunchKernelGGL(k_combine, dim3(blocks, c->k), dim3(kThreads), 0, s, A);
    });
    DASH_HIP(hipGetLastError());
    return DASH_OK;
}

// tiles of n_experts matrices whose rows and experts lie row_stride and expert_stride elements apart; 0: refused
static int64_t weight_tiles(const void* w, int64_t row_stride, int64_t expert_stride, int n_experts, int out_c, int K, const void* prepared) {
    if (!w || !prepared || ((uintptr_t)prepared & 15) || n_experts < 1 || out_c < 1 || K < 1 || row_stride < K || expert_stride < 0) return 0;
    const int64_t tiles = row_tiles(out_c) * col_tiles(K), most = 1ll << 50;        // (more than any call takes)
    return tiles > most / n_experts ? most : tiles * n_experts;
}

// bytes, or 8-bit codes, into their tiles
static int lay_out_bytes(int format, const int8_t* w, int64_t row_stride, int64_t expert_stride, int64_t tiles, int out_c, int K, void* prepared, hipStream_t s) {
    const int64_t lanes = tiles * (kW8Tile / 16);
    if (lanes > kMaxLanes) return DASH_ESIZE;
    PrepArgs8 A{w, row_stride, expert_stride, tiles, 0, matrix_bytes(format, out_c, K), out_c, K, format == DASH_F8, (uint8_t*)prepared};
    in_launches((lanes + kThreads - 1) / kThreads, [&](int64_t first, uint32_t blocks) {
        A.first = first * kThreads;
        hipLaunchKernelGGL(k_weights8_prepare, dim3(blocks), dim3(kThreads), 0, s, A);
    });
    DASH_HIP(hipGetLastError());
    return DASH_OK;
}

}  // namespace dash

using namespace dash;

extern "C" {

size_t dash_expert_weights_bytes(int format, int n_experts, int out_c, int K) {
    if (!weight_format(format) || n_experts < 1 || out_c < 1 || K < 1) return 0;
    return (size_t)n_experts * (size_t)matrix_bytes(format, out_c, K);
}

int dash_weights8_prepare(dash_ctx* c, const int8_t* w, int64_t row_stride, int64_t expert_stride, int n_experts, int out_c, int K, void* prepared,
                          void* stream) {
    if (!c) return DASH_EINVAL;
    const int64_t tiles = weight_tiles(w, row_stride, expert_stride, n_experts, out_c, K, prepared);
    if (!tiles) return DASH_EINVAL;
    return lay_out_bytes(DASH_W8, w, row_stride, expert_stride, tiles, out_c, K, prepared, (hipStream_t)stream);
}

int dash_f8_prepare(dash_ctx* c, const uint8_t* codes, int64_t row_stride, int64_t expert_stride, const int32_t* scales, int n_experts, int out_c, int K,
                    void* prepared, void* stream) {
    if (!c || !scales || ((uintptr_t)scales & 3)) return DASH_EINVAL;
    const int64_t tiles = weight_tiles(codes, row_stride, expert_stride, n_experts, out_c, K, prepared);
    if (!tiles) return DASH_EINVAL;
    const int64_t per = scale_blocks(out_c) * scale_blocks(K);
    if (per > 0x7fffffff) return DASH_ESIZE;
    const int st = lay_out_bytes(DASH_F8, (const int8_t*)codes, row_stride, expert_stride, tiles, out_c, K, prepared, (hipStream_t)stream);
    if (st) return st;
    ScalesArgs A{scales, scales_at(out_c, K), matrix_bytes(DASH_F8, out_c, K), 0, per * n_experts, (uint32_t)per, (uint8_t*)prepared};
    in_launches((A.total + kThreads - 1) / kThreads, [&](int64_t first, uint32_t blocks) {
        A.first = first * kThreads;
        hipLaunchKernelGGL(k_f8_scales, dim3(blocks), dim3(kThreads), 0, (hipStream_t)stream, A);
    });
    DASH_HIP(hipGetLastError());
    return DASH_OK;
}

int dash_f8_quantise(dash_ctx* c, const void* w, int dtype, int64_t row_stride, int64_t expert_stride, int n_experts, int out_c, int K, int base,
                     int max_scale, void* prepared, void* values, void* stream) {
    if (!c || dtype < DASH_F32 || dtype > DASH_F16 || base < -64 || base > 64 || max_scale < 1 || max_scale > 32767) return DASH_EINVAL;
    const uintptr_t unaligned = dtype == DASH_F32 ? 3 : 1;
    if (((uintptr_t)w & unaligned) || ((uintptr_t)values & unaligned)) return DASH_EINVAL;
    if (!weight_tiles(w, row_stride, expert_stride, n_experts, out_c, K, prepared)) return DASH_EINVAL;
    const int64_t per = scale_blocks(out_c) * scale_blocks(K), blocks = per * n_experts;
    if (per > 0x7fffffff / n_experts) return DASH_ESIZE;
    QuantF8Args A{w, row_stride, expert_stride, matrix_bytes(DASH_F8, out_c, K), 0, out_c, K, max_scale, ldexpf(1.0f, base), ldexpf(1.0f, -base), (uint8_t*)prepared, values};
    auto kernel = dtype == DASH_F32 ? k_f8_quantise<QuantF32> : dtype == DASH_BF16 ? k_f8_quantise<QuantBF16> : k_f8_quantise<QuantF16>;
    in_launches<kF8Threads>(blocks, [&](int64_t first, uint32_t n) {
        A.first = (uint32_t)first;
        hipLaunchKernelGGL(kernel, dim3(n), dim3(kF8Threads), 0, (hipStream_t)stream, A);
    });
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
    if (tiles > 0x7fffffff) return DASH_ESIZE;
    QuantArgs A{w, row_stride, expert_stride, 0, out_c, K, base, max_shift, (uint8_t*)prepared, values};
    auto kernel = dtype == DASH_F32 ? k_mx4_quantise<QuantF32> : dtype == DASH_BF16 ? k_mx4_quantise<QuantBF16> : k_mx4_quantise<QuantF16>;
    in_launches(tiles, [&](int64_t first, uint32_t blocks) {
        A.first = (uint32_t)first;
        hipLaunchKernelGGL(kernel, dim3(blocks), dim3(kThreads), 0, (hipStream_t)stream, A);
    });
    DASH_HIP(hipGetLastError());
    return DASH_OK;
}

size_t dash_route_bytes(const dash_ctx* c, int64_t n, int n_experts) {
    // (groups and tiles are numbered in 32 bits)
    if (!c || n < 0 || n_experts < 1 || n_experts > kMaxExperts || n > 0x7fffffff / (total_chunks(c) + 64)) return 0;
    const RoutingView v = routing_view(c, nullptr, n, n_experts);
    for (int s = 0; s < kTileKinds; s++) if (v.max_tiles[s] > 0x7fffffff) return 0;
    return v.bytes;
}

int dash_route(dash_ctx* c, const int32_t* experts, int64_t n, int n_experts, void* data, dash_routing* routing, void* stream) {
    if (!c || !data || ((uintptr_t)data & 15) || !routing || n < 0 || n_experts < 1 || (n > 0 && !experts)) return DASH_EINVAL;
    if (!dash_route_bytes(c, n, n_experts)) return DASH_ESIZE;
    RouteArgs A;
    memset(&A, 0, sizeof(A));
    A.experts = experts; A.n = n; A.E = n_experts;
    const PrimeClasses classes = prime_classes(c);
    for (int s = 0; s < kTileKinds; s++) {
        const TileParts parts = kTileKind[s].parts;
        int chunk = 0;
        for (int i = 0; i < (parts == PARTS_NONE ? 1 : parts == PARTS_PRIMES ? c->k : classes.n); i++) {
            const int first = chunk;
            chunk = parts == PARTS_NONE ? (int)total_chunks(c) : parts == PARTS_PRIMES ? chunk + (int)c->mods[c->prime[i]].nchunk : classes.chunk_first[i + 1];
            A.pair[A.pairs++] = {(uint8_t)s, (uint8_t)i, (uint16_t)first, (uint16_t)chunk};
        }
        A.kind_first[s + 1] = A.pairs;
    }
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
