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
// A group is 16 digits (a chunk) of one row.  The groups of an expert are numbered prime by prime, chunk by chunk, row by row.  A tile is up to
// `groups` consecutive ones of one expert (byte weights: the operand is the same for every prime) or of one expert and prime (4-bit weights);
// tiles are sorted by expert and first group.
struct TileKind { int groups; bool one_prime; };
constexpr int kTileKinds = 5;
constexpr TileKind kTileKind[kTileKinds] = {{16, false}, {8, false}, {16, true}, {8, true}, {4, true}};
struct RouteTile {          // (read as a uint4)
    uint32_t expert_prime;  // expert (n_experts: none) | index of the prime << 24 (one_prime; else 0)
    int32_t start, count;   // the expert's rows: rows[start .. start + count - 1]
    int32_t first;          // first group
};
constexpr int kMaxExperts = (1 << 24) - 2;
// offsets int32[E + 2] (expert E: rows of no expert), rows int32[n]; per tile kind: first tile of every expert int32[E + 2], tiles
struct RoutingView {
    int32_t* offsets;
    int32_t* rows;
    int32_t* first_tile[kTileKinds];
    RouteTile* tiles[kTileKinds];
    int64_t max_tiles[kTileKinds];
    size_t bytes;
};
inline int64_t total_chunks(const dash_ctx* c) {
    int64_t n = 0;
    for (int i = 0; i < c->k; i++) n += c->mods[c->prime[i]].nchunk;
    return n;
}
inline RoutingView routing_view(const dash_ctx* c, void* data, int64_t n, int E) {
    RoutingView v;
    size_t at = 0;
    auto take = [&](size_t bytes) { uint8_t* p = (uint8_t*)data + at; at += (bytes + 63) / 64 * 64; return p; };
    v.offsets = (int32_t*)take(sizeof(int32_t) * (size_t)(E + 2));
    v.rows = (int32_t*)take(sizeof(int32_t) * (size_t)n);
    // an expert with rows leaves at most one tile (one_prime: one a prime) partly filled
    const int64_t busy = n < (int64_t)E + 1 ? n : (int64_t)E + 1, chunks = total_chunks(c);
    for (int s = 0; s < kTileKinds; s++) {
        v.max_tiles[s] = chunks * n / kTileKind[s].groups + busy * (kTileKind[s].one_prime ? c->k : 1);
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
