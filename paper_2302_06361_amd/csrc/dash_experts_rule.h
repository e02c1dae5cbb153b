// dash_experts_rule.h -- which tile the products of an expert layer take, as a function of its sizes alone, and the grid of the launch (host code); the columns of a block
#pragma once
#include <stdint.h>

namespace dash {

// 256 digits x 256 features a block; 128 x 128; for 4-bit weights also 64 x 128 with the inputs dealt out to two sets of waves, and 128 x 256
enum ExpertsTile { EXPERTS_BY_SIZE = 0, EXPERTS_BIG = 1, EXPERTS_NARROW = 2, EXPERTS_FEW = 3, EXPERTS_WIDE = 4, EXPERTS_WIDE_CLASS = 5, EXPERTS_SMALL = 6 };       // (the last two: 8-bit floats)

struct ExpertsShape {
    int64_t rows;           // of all experts
    int experts, M, K;
    bool mx4;
    int k;                  // primes, and the 16-digit chunks of their labels
    int chunks[16];
};
// Rows are taken to be spread evenly over the experts (the host does not see the routing).  A group is a chunk of a row.
inline double experts_groups(const ExpertsShape& S, double* busy) {
    *busy = S.rows < S.experts ? (double)S.rows : (double)S.experts;
    double c = 0;
    for (int i = 0; i < S.k; i++) c += S.chunks[i];
    return c * (double)S.rows / *busy;
}
// tiles of `groups` groups an expert makes: across primes for byte weights, for every prime for 4-bit weights
inline double experts_tiles(const ExpertsShape& S, int groups) {
    double busy, t = 0;
    const double all = experts_groups(S, &busy);
    auto up = [&](double g) { const double q = g / groups; const int64_t f = (int64_t)q; return (double)(f + (q - (double)f > 1e-9 ? 1 : 0)); };
    if (!S.mx4) t = up(all);
    else for (int i = 0; i < S.k; i++) t += up(S.chunks[i] * (double)S.rows / busy);
    return t * busy;
}
// Time in us: a launch, and on the fullest CU what a block takes beside its stages of 64 inputs, and the stages, at the rate of one block's
// latency or of what shares the CU.  Constants fitted to runs over these 18 layers (us of repeated calls: bytes big, narrow | 4-bit big, narrow, few, wide):
//   1 row, 784 -> 128, 8 primes: 12.7, 5.8 | 12.5, 7.7, 7, 10.8
//   1 row, 4096 -> 4096, 12 primes: 37.4, 16 | 43, 26.8, 25.2, 33.8
//   4 rows, 4096 -> 4096, 12 primes: 41.4, 41.5 | 47.4, 50.1, 59.5, 53.6
//   16 rows, 4096 -> 4096, 12 primes: 131, 141 | 149, 158, 229, 140
//   128 rows, 4096 -> 4096, 12 primes: 991, 1230 | 1029, 1246, 1765, 1076
//   16 rows, 8 experts, 400 -> 120, 8 primes: 10.2, 5.2 | 11.2, 6.4, 6.2, 8.7
//   256 rows, 32 experts, 1024 -> 2048, 12 primes: 325, 376 | 414, 425, 667, 355
//   128 rows, 16 experts, 512 -> 768, 9 primes: 41.7, 41.8 | 48, 50.3, 80.5, 41.2
//   64 rows, 12 experts, 4096 -> 256, 12 primes: 43.7, 43.7 | 52.8, 51.8, 69.4, 54.1
//   64 rows, 64 experts, 1024 -> 1024, 12 primes: 49.2, 50.6 | 109, 77.9, 102, 67
//   64 rows, 16 experts, 1024 -> 1024, 12 primes: 47.7, 48 | 62.5, 59.8, 91.1, 52.8
//   2 rows, 2048 -> 2048, 12 primes: 22, 9.4 | 25.5, 14.1, 16.5, 19.6
//   8 rows, 256 -> 4096, 8 primes: 11.3, 11.4 | 18.7, 13.4, 22.7, 11.6
//   39 rows, 4 experts, 81 -> 29, 12 primes: 8.2, 4.6 | 8.3, 5.1, 6.6, 6.7
//   65 rows, 4 experts, 228 -> 12, 7 primes: 8.9, 4.8 | 9.5, 5.6, 7.3, 7.7
//   12 rows, 6 experts, 3833 -> 172, 9 primes: 35.6, 14.4 | 45.5, 22.3, 17.1, 32.4
//   256 rows, 2048 -> 64, 12 primes: 73.7, 60.6 | 88.7, 64, 76.8, 80.5
//   200 rows, 8 experts, 100 -> 1500, 9 primes: 61.5, 86.4 | 79.9, 88.6, 171, 66.3
// Over 441 drawn layers the choice took over 5 % more than the fastest tile in 25, over 10 % in 15, at most 37 % (bytes, 24 rows,
// 15 experts, 1170 -> 570: 20.0 us with the big tile, 14.6 with the narrow one).
inline double experts_us(const ExpertsShape& S, ExpertsTile tile) {
    const int groups = tile == EXPERTS_BIG ? 16 : tile == EXPERTS_FEW ? 4 : 8, features = tile == EXPERTS_BIG || tile == EXPERTS_WIDE ? 256 : 128;
    double block, latency, rate, busy, resident = tile == EXPERTS_BIG ? 1 : tile == EXPERTS_FEW ? 1.3 : 2;       // (blocks that start side by side)
    const double tiles = experts_tiles(S, groups), fill = experts_groups(S, &busy) * busy / (tiles * groups);
    if (!S.mx4) {
        block = tile == EXPERTS_BIG ? 4.4 : 3.4; latency = tile == EXPERTS_BIG ? 0.46 : 0.18; rate = tile == EXPERTS_BIG ? 0.75 : 0.25;
    } else if (tile == EXPERTS_BIG) { block = 5.0; latency = 0.60; rate = 0.70; }
    else if (tile == EXPERTS_NARROW) { block = 1.8 + 1.8 * fill; latency = 0.28; rate = 0.14 + 0.115 * fill; }      // (products of missing groups are left out)
    else if (tile == EXPERTS_WIDE) { block = 4.4; latency = 0.43; rate = 0.38; }
    else { block = 2.0 + 1.2 * fill; latency = 0.18; rate = 0.165; }
    double per_cu = tiles * (double)((S.M + features - 1) / features) / 256;
    if (per_cu <= 4) per_cu = (double)(int64_t)(per_cu + 1 - 1e-9);
    if (per_cu < 1) per_cu = 1;
    const double stages = (double)(((int64_t)S.K + 63) / 64), rounds = per_cu / resident < 1 ? 1 : per_cu / resident;
    return 2 + block * rounds + stages * (latency > rate * per_cu ? latency : rate * per_cu);
}
inline ExpertsTile experts_tile(int forced, const ExpertsShape& S) {
    if (forced == EXPERTS_BIG || forced == EXPERTS_NARROW || ((forced == EXPERTS_FEW || forced == EXPERTS_WIDE) && S.mx4)) return (ExpertsTile)forced;
    int best = EXPERTS_BIG;
    for (int t = EXPERTS_NARROW; t <= (S.mx4 ? EXPERTS_WIDE : EXPERTS_NARROW); t++)
        if (experts_us(S, (ExpertsTile)t) < experts_us(S, (ExpertsTile)best)) best = t;
    return (ExpertsTile)best;
}

// ---- 8-bit floats ----
struct ExpertsShape8 {
    int64_t rows;           // of all experts
    int experts, M, K;
    int k;                  // primes, and the 16-digit chunks of their labels
    int chunks[16];
    int classes;            // of primes, and the chunks of theirs
    int class_chunks[16];
};
struct ExpertsRate8 {
    int groups, features;
    bool by_class;
    double call, block, latency, rate, empty, resident;     // empty: of a group that a tile has room for
};
inline ExpertsRate8 experts_rate8(ExpertsTile tile) {
    switch (tile) {
        case EXPERTS_BIG: return {32, 128, false, 0.5, 5.96, 0.394, 0.881, 0.61, 1};
        case EXPERTS_WIDE: return {16, 128, false, 2.67, 2.35, 0.518, 0.523, 0.46, 1};
        case EXPERTS_WIDE_CLASS: return {16, 128, true, 2.99, 2.69, 0.531, 0.508, 0.49, 1};
        case EXPERTS_FEW: return {8, 128, true, 0.74, 5.15, 0.335, 0.453, 0.82, 1};
        case EXPERTS_SMALL: return {8, 64, true, 1.87, 3.84, 0.336, 0.261, 0.39, 1.5};
        default: return {8, 128, true, 3.26, 1.27, 0.5, 0.367, 0.74, 1};
    }
}
// Time in us, as above: a call, what a block takes beside its stages of 64 inputs (a set's, where there are two), and the stages.  Constants fitted to runs over 120 layers, these 18 among them
// (us of repeated calls with the tiles big, wide, class, narrow, few, small):
//   1 row, 784 -> 128, 8 primes: 13.6, 10.7, 12.1, 10.6, 11.3, 9.9
//   1 row, 4096 -> 4096, 12 primes: 89.5, 50.5, 40.8, 37.6, 34.8, 37.2
//   4 rows, 4096 -> 4096, 12 primes: 93.4, 59.9, 61.5, 74.6, 98.2, 96.5
//   16 rows, 4096 -> 4096, 12 primes: 165, 167, 176, 251, 335, 322
//   128 rows, 4096 -> 4096, 12 primes: 1141, 1238, 1385, 1887, 2607, 2513
//   16 rows, 8 experts, 400 -> 120, 8 primes: 10.4, 9.1, 9.2, 7.9, 9.1, 8.3
//   256 rows, 32 experts, 1024 -> 2048, 12 primes: 542, 423, 453, 539, 962, 948
//   128 rows, 16 experts, 512 -> 768, 9 primes: 55.8, 45.9, 47.5, 54.5, 107, 104
//   64 rows, 12 experts, 4096 -> 256, 12 primes: 94.4, 65, 65.5, 76.3, 99.5, 99.9
//   64 rows, 64 experts, 1024 -> 1024, 12 primes: 327, 160, 103, 93.9, 167, 164
//   64 rows, 16 experts, 1024 -> 1024, 12 primes: 96.2, 66.5, 69.5, 78.1, 124, 122
//   2 rows, 2048 -> 2048, 12 primes: 27, 22.6, 23.3, 21.1, 20.4, 21.3
//   8 rows, 256 -> 4096, 8 primes: 19.1, 17.3, 15.3, 14.9, 26.9, 28.4
//   39 rows, 4 experts, 81 -> 29, 12 primes: 8.4, 6.7, 6.8, 5.7, 6.8, 6.2
//   65 rows, 4 experts, 228 -> 12, 7 primes: 10, 7.9, 7.9, 6.6, 8, 7
//   12 rows, 6 experts, 3833 -> 172, 9 primes: 46.1, 38, 38.3, 36.3, 32.7, 27.2
//   256 rows, 2048 -> 64, 12 primes: 78.7, 72, 70.3, 73.5, 99.4, 72.9
//   200 rows, 8 experts, 100 -> 1500, 9 primes: 90.5, 75.8, 73.5, 80.6, 220, 223
// Over the 120 the choice took over 5 % more than the fastest tile in 5, over 10 % in 2, at most 20 % (141 rows, 2 experts, 3578 -> 162, 7 primes: 102.6 us with the narrow
// tile, 85.3 with the one across classes), 0.7 % in the mean; over 40 drawn layers that were not fitted 0.7 % in the mean, 8 % at most.
inline double experts_us8(const ExpertsShape8& S, ExpertsTile tile) {
    const ExpertsRate8 R = experts_rate8(tile);
    const double busy = S.rows < S.experts ? (double)S.rows : (double)S.experts, rows = (double)S.rows / busy;
    double tiles = 0, groups = 0;
    const int parts = R.by_class ? S.classes : S.k;
    for (int i = 0; i < parts; i++) {
        const double g = rows * (R.by_class ? S.class_chunks[i] : S.chunks[i]), q = g / R.groups;
        const int64_t f = (int64_t)q;
        tiles += (double)(f + (q - (double)f > 1e-9 ? 1 : 0));
        groups += g;
    }
    const double fill = groups / (tiles * R.groups);
    double per_cu = tiles * busy * (double)((S.M + R.features - 1) / R.features) / 256;
    if (per_cu <= 4) per_cu = (double)(int64_t)(per_cu + 1 - 1e-9);
    if (per_cu < 1) per_cu = 1;
    const double stages = (double)(((int64_t)S.K + 63) / 64), rounds = per_cu / R.resident < 1 ? 1 : per_cu / R.resident;
    const double rate = R.rate * (R.empty + (1 - R.empty) * fill) * per_cu;
    return R.call + R.block * rounds + stages * (R.latency > rate ? R.latency : rate);
}
inline ExpertsTile experts_tile8(int forced, const ExpertsShape8& S) {
    if (forced >= EXPERTS_BIG && forced <= EXPERTS_SMALL) return (ExpertsTile)forced;
    int best = EXPERTS_BIG;
    for (int t = EXPERTS_NARROW; t <= EXPERTS_SMALL; t++)
        if (experts_us8(S, (ExpertsTile)t) < experts_us8(S, (ExpertsTile)best)) best = t;
    return (ExpertsTile)best;
}

// whether the columns first .. first + n - 1 of a row of K all exist (K up to 2^31 - 1: their end may pass 31 bits)
constexpr bool columns_inside(int first, int n, int K) { return K - first >= n; }

// At least `blocks` blocks of `threads` threads as x times y, x a multiple of the 8 XCDs: a direction of a grid holds fewer than 2^32 threads.
struct BlockGrid { uint32_t x, y; };
inline BlockGrid block_grid(int64_t blocks, int threads) {
    const int64_t most = 0xffffffffll / threads / 8 * 8, y = (blocks + most - 1) / most, x = (blocks + y - 1) / y;
    return BlockGrid{(uint32_t)((x + 7) / 8 * 8), (uint32_t)y};
}

}  // namespace dash
