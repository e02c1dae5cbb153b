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

// ---- routing: rows sorted by expert ----
// offsets int32[E + 2] (expert E: rows of no expert), rows int32[n]
struct RoutingView {
    int32_t* offsets;
    int32_t* rows;
    size_t bytes;
};
inline RoutingView routing_view(void* data, int64_t n, int E) {
    RoutingView v;
    size_t at = 0;
    auto take = [&](size_t bytes) { uint8_t* p = (uint8_t*)data + at; at += (bytes + 63) / 64 * 64; return p; };
    v.offsets = (int32_t*)take(sizeof(int32_t) * (size_t)(E + 2));
    v.rows = (int32_t*)take(sizeof(int32_t) * (size_t)n);
    v.bytes = at;
    return v;
}

}  // namespace dash
