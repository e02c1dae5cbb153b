// dash_experts.h -- layouts shared by the host and device code of expert layers: prepared weights, the routing of rows
#pragma once
#include <stdint.h>

#include "dash_internal.h"

namespace dash {

// ---- prepared weights: tiles of 32 rows x 64 columns, row tiles outermost ----
constexpr int kTileRows = 32, kTileCols = 64;
constexpr int kW8Tile = 2048, kMx4Codes = 1024, kMx4Tile = kMx4Codes + 64;
__host__ __device__ inline int64_t row_tiles(int M) { return ((int64_t)M + kTileRows - 1) / kTileRows; }
__host__ __device__ inline int64_t col_tiles(int K) { return ((int64_t)K + kTileCols - 1) / kTileCols; }
__host__ __device__ inline int tile_bytes(int format) { return format == DASH_MX4 ? kMx4Tile : kW8Tile; }
__host__ __device__ inline int64_t matrix_bytes(int format, int M, int K) { return row_tiles(M) * col_tiles(K) * tile_bytes(format); }
// Where the 16-byte piece of columns 16 q .. 16 q + 15 (q = 0..3) of a row stands among the row's four: the pieces of one q in 8 or 16
// consecutive rows, which a wave reads together, then lie in different banks.
__host__ __device__ inline int w8_piece(int row, int q) { return q ^ ((row >> 1) & 3) ^ ((row >> 3) & 1); }
__host__ __device__ inline int w8_at(int row, int col) { return 64 * row + 16 * w8_piece(row, col >> 4) + (col & 15); }

// ---- routing: rows sorted by expert, and the tiles of the products ----
// A group is 16 digits (a chunk) of one row; the groups of an expert's rows for one prime are numbered chunk by chunk.  A tile is up to
// kTileGroups[s] consecutive groups of one expert and prime; tiles are sorted by expert, prime, first group.
constexpr int kTileSizes = 2;
constexpr int kTileGroups[kTileSizes] = {16, 8};
struct RouteTile {          // (read as a uint4)
    uint32_t expert_prime;  // expert (n_experts: none) | index of the prime << 24
    int32_t start, count;   // the expert's rows: rows[start .. start + count - 1]
    int32_t first;          // first group
};
constexpr int kMaxExperts = (1 << 24) - 2;
// offsets int32[E + 2] (expert E: rows of no expert), rows int32[n]; per tile size: first tile of every expert int32[E + 2], tiles
struct RoutingView {
    int32_t* offsets;
    int32_t* rows;
    int32_t* first_tile[kTileSizes];
    RouteTile* tiles[kTileSizes];
    int64_t max_tiles[kTileSizes];
    size_t bytes;
};
// tiles that n rows can make: every expert of a row leaves at most one of them partly filled for a prime
inline int64_t max_tiles(const dash_ctx* c, int64_t n, int E, int groups) {
    int64_t t = 0;
    const int64_t busy = n < E + 1 ? n : E + 1;
    for (int i = 0; i < c->k; i++) t += (int64_t)c->mods[c->prime[i]].nchunk * n / groups + busy;
    return t;
}
inline RoutingView routing_view(const dash_ctx* c, void* data, int64_t n, int E) {
    RoutingView v;
    size_t at = 0;
    auto take = [&](size_t bytes) { uint8_t* p = (uint8_t*)data + at; at += (bytes + 63) / 64 * 64; return p; };
    v.offsets = (int32_t*)take(sizeof(int32_t) * (size_t)(E + 2));
    v.rows = (int32_t*)take(sizeof(int32_t) * (size_t)n);
    for (int s = 0; s < kTileSizes; s++) {
        v.max_tiles[s] = max_tiles(c, n, E, kTileGroups[s]);
        v.first_tile[s] = (int32_t*)take(sizeof(int32_t) * (size_t)(E + 2));
        v.tiles[s] = (RouteTile*)take(sizeof(RouteTile) * (size_t)v.max_tiles[s]);
    }
    v.bytes = at;
    return v;
}

// ---- products (dash_experts_gemm.hip) ----
struct ExpertsCall {
    const uint8_t* w;
    const int32_t* bias;
    const RoutingView* routing;     // NULL: every row through matrix 0
    int64_t n;
    int M, K, E, top_k, format;
    bool garble;
};
int experts_mfma(dash_ctx* c, const ExpertsCall& L, const dash_labels* in, dash_labels* out, hipStream_t s);

}  // namespace dash
