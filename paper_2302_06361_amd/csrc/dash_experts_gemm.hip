// dash_experts_gemm.hip -- the products of expert layers as int8 MFMA contractions (dash_experts.hip has the formulas).
//
// Shape.  A group is 16 digits (a chunk) of one row: in memory K words of 16 bytes, word i = the 16 digits of input i.  For all groups
// of one expert and prime the layer is one matrix product  Out^T (16 groups x M) = X^T (16 groups x K) * W^T (K x M).  The labels are
// the A operand and the weights the B operand of v_mfma_i32_32x32x32_i8: a lane then holds, for ONE output feature, 4 consecutive
// digits in 4 consecutive accumulators, so the result needs no turning around: pack 4 bytes, swap halves of the wave (2 groups a
// tile), store 16 bytes a lane, neighbouring lanes neighbouring features.
//
// Loads.  Everything comes by loads that write LDS directly (global_load_lds: no registers, no LDS write instructions).  64 words of a
// group are 1 KB in a row, one instruction; prepared weights are laid out in tiles for the same.  Labels are turned around (the MFMA
// wants 16 consecutive inputs of one digit) by the LDS itself: ds_read_b64_tr_b8 gives lane l of 16 the byte l of 8 words.
// A ring of S stages of 64 inputs; each wave waits for its own loads of the next stage (vmcnt counts down in order, all stages issue the
// same number), then one barrier a stage.
//
// Weights.  Signed bytes are the operand as they are, for every prime: the sums start at a multiple of p that keeps them positive and
// are reduced once.  4-bit floats: 2 e2m1 2^shift mod p by table: the 8 magnitudes of a shift and their negatives are 16 bytes of
// LDS, a v_perm picks four of them by four 3-bit codes at a time; a stage's tile is expanded once a block, a stage ahead, into the
// layout of the byte weights.
#include <string.h>

#include "dash_experts.h"

#pragma clang diagnostic ignored "-Winline-asm"       // (m0 as a clobber)

namespace dash {

typedef int v2i __attribute__((ext_vector_type(2)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v16i __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) uint8_t* lds_ptr;
typedef __attribute__((address_space(3))) v2i* lds_v2i;

// WD x WF waves (along digits, along features), a wave DA x FB tiles of 32 digits x 32 features; S stages of 64 inputs in LDS
template <int WD_, int WF_, int DA_, int FB_, int S_, int WPE_, int SIZE_>
struct ETile {
    static constexpr int WD = WD_, WF = WF_, DA = DA_, FB = FB_, S = S_, WPE = WPE_, SIZE = SIZE_;
    static constexpr int NW = WD * WF, T = 64 * NW;
    static constexpr int G = 2 * WD * DA;          // groups per block
    static constexpr int FT = WF * FB, F = 32 * FT;  // feature tiles, features per block
    static constexpr int GP = G / NW;              // groups that a wave loads
    static constexpr int NL = GP + 2;              // loads per wave and stage
    static_assert(G == kTileGroups[SIZE] && GP * NW == G && FT == NW, "a wave loads GP groups and one tile of weights");
};
typedef ETile<2, 4, 4, 2, 4, 2, 0> EBig;           // 256 digits x 256 features
typedef ETile<1, 4, 4, 1, 4, 2, 1> ENarrow;        // 128 digits x 128 features

struct ExpPrime {
    uint32_t p, nchunk;
    uint32_t mmagic;            // ceil(2^32 / p)
    uint32_t pow12;             // 4096 mod p
    uint32_t start;             // multiple of p that the sums start at
    uint32_t two_step;          // sums are too large for one multiplication by mmagic
    const uint8_t* one;         // chunked label of the constant-one wire, or NULL
    LView in, out;
};
struct ExpArgs {
    const uint8_t* w;
    int64_t expert_bytes;
    const int32_t* bias;
    const int32_t* rows;                // routing, or NULL
    const RouteTile* tiles;
    const int32_t* n_tiles;
    int M, K, E, n, top_k;
    int col_blocks, row_blocks;         // blocks along the groups (at most) and along the features
    int lg_st, lg_sty, gy;              // block -> tile: log2 of the blocks of a super-tile and of its rows, super-tile rows
    int st_total;
    int first[DASH_MAX_PRIMES + 1];     // without routing: first block along the groups of every prime
    ExpPrime pr[DASH_MAX_PRIMES];
};

// 16 (4) bytes a lane from base + off to LDS at `to` + 16 (4) * lane.  In flight until a wait on vmcnt; nothing in registers.
__device__ __forceinline__ void load_lds16(uint32_t to, const uint8_t* base, uint32_t off) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(off), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ void load_lds4(uint32_t to, const uint8_t* base, uint32_t off) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(to), "v"(off), "s"(base) : "memory", "m0");
}
// at most N loads of the wave outstanding, its LDS accesses done; then the block's barrier
template <int N> __device__ __forceinline__ void wait_and_barrier() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}
template <int N> __device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
__device__ __forceinline__ const uint8_t* uniform(const uint8_t* p) {
    const uint64_t a = (uint64_t)p;
    return (const uint8_t*)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)a) |
                            (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(a >> 32)) << 32);
}

template <int FMT, class TL>
__global__ __launch_bounds__(TL::T, TL::WPE) void k_experts_mfma(const ExpArgs A) {
    constexpr int G = TL::G, DA = TL::DA, FB = TL::FB, S = TL::S, GP = TL::GP, NL = TL::NL, FT = TL::FT, T = TL::T;
    constexpr bool kMx4 = FMT == DASH_MX4;
    // ---- block -> tile ----
    const int xcd = blockIdx.x & 7, seq = blockIdx.x >> 3;
    const int st = (seq >> A.lg_st) * 8 + xcd, within = seq & ((1 << A.lg_st) - 1);
    if (st >= A.st_total) return;
    const int by = (st % A.gy << A.lg_sty) + (within & ((1 << A.lg_sty) - 1)), bx = (st / A.gy << (A.lg_st - A.lg_sty)) + (within >> A.lg_sty);
    if (by >= A.row_blocks || bx >= A.col_blocks) return;
    int e = 0, pi = 0, start = 0, count = A.n, first;
    if (A.tiles) {
        if (bx >= *A.n_tiles) return;
        const RouteTile t = A.tiles[bx];
        e = (int)(t.expert_prime & 0xffffffu); pi = (int)(t.expert_prime >> 24);
        start = t.start; count = t.count; first = t.first;
    } else {
        while (bx >= A.first[pi + 1]) pi++;
        first = (bx - A.first[pi]) * G;
    }
    const ExpPrime& P = A.pr[pi];
    const int M = A.M, K = A.K;
    const uint32_t prime = P.p, mmagic = P.mmagic;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wd = wave / TL::WF, wf = wave % TL::WF;

    constexpr int kDig = G * 1024, kRaw = kMx4 ? 1280 : 2048;       // bytes of a stage's labels; of a stage's weights per feature tile, as loaded
    constexpr int kExp = FT * 2048;                                 // 4-bit: bytes of an expanded stage
    // one array: its address goes into the loads, so that the compiler takes all of it to change at their waits and barriers
    __shared__ __attribute__((aligned(1024))) uint8_t smem[S * kDig + S * FT * kRaw + (kMx4 ? 2 * kExp : 0)];
    uint8_t* const s_dig = smem;
    uint8_t* const s_raw = smem + S * kDig;
    uint8_t* const s_exp = s_raw + S * FT * kRaw;
    __shared__ u32x4 s_lut[kMx4 ? 256 : 1];
    __shared__ u32x4 s_one[G];
    __shared__ const uint8_t* s_src[G];
    __shared__ uint8_t* s_dst[G];

    // ---- the groups of the tile ----
    const int n_groups = (int)P.nchunk * count;
    if (tid < G) {
        const bool valid = first + tid < n_groups;
        const int g = valid ? first + tid : first;                  // (a group past the end loads the tile's first and stores nothing)
        const int ch = g / count, t = g - ch * count, row = A.rows ? A.rows[start + t] : t;
        s_src[tid] = P.in.p + (int64_t)ch * P.in.cs + (int64_t)(row / A.top_k) * K * 16;
        s_dst[tid] = valid ? P.out.p + (int64_t)ch * P.out.cs + (int64_t)row * M * 16 : nullptr;
        if (A.bias) s_one[tid] = *(const u32x4*)(P.one + 16 * ch);
    }
    if (kMx4 && tid < 256) {
        // 2^tid mod p, times the eight magnitudes, and p minus that
        uint32_t two = 1 % prime, sq = 2 % prime;
        for (uint32_t b = tid; b; b >>= 1) {
            if (b & 1) { two *= sq; two -= mul24(mulhi(two, mmagic), prime); }
            sq *= sq; sq -= mul24(mulhi(sq, mmagic), prime);
        }
        uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
        for (int m = 0; m < 8; m++) {
            uint32_t r = two * (uint32_t)(m < 4 ? m : m == 7 ? 12 : 2 * m - 4);
            r -= mul24(mulhi(r, mmagic), prime);
            w[m / 4] |= r << (8 * (m % 4));
            w[2 + m / 4] |= (r ? prime - r : 0) << (8 * (m % 4));
        }
        s_lut[tid] = u32x4{w[0], w[1], w[2], w[3]};
    }
    __syncthreads();
    if (e >= A.E) {         // rows of no expert: the value 0 on both sides
        for (int i = tid; i < G * TL::F; i += T) {
            uint8_t* const dst = s_dst[i / TL::F];
            const int j = by * TL::F + i % TL::F;
            if (dst && j < M) *(u32x4*)(dst + (int64_t)j * 16) = u32x4{0, 0, 0, 0};
        }
        return;
    }

    // ---- loads ----
    const int nk = (K + 63) / 64;
    const uint8_t* src[GP];
#pragma unroll
    for (int i = 0; i < GP; i++) src[i] = uniform(s_src[wave * GP + i]);
    const int row_tiles_ = (M + 31) / 32, rt = by * FT + wave < row_tiles_ ? by * FT + wave : row_tiles_ - 1;       // (tiles past the end: the last again)
    constexpr int kTileBytes = kMx4 ? kMx4Tile : kW8Tile;
    const uint8_t* const wsrc = uniform(A.w + (int64_t)e * A.expert_bytes + (int64_t)rt * nk * kTileBytes);
    const uint32_t dig0 = (uint32_t)(uintptr_t)(lds_ptr)s_dig, raw0 = (uint32_t)(uintptr_t)(lds_ptr)s_raw;
    // stage kt into slot kt % S; past the end the last stage again, so that every stage counts the same loads
    auto issue = [&](int kt) __attribute__((always_inline)) {
        const int slot = kt % S, k = kt < nk ? kt : nk - 1;
        const int last = K - 1 - 64 * k;                            // words past K: the last again (their weights are zero)
        const uint32_t off = 16u * (uint32_t)(lane < last ? lane : last);
#pragma unroll
        for (int i = 0; i < GP; i++) load_lds16(dig0 + slot * kDig + (wave * GP + i) * 1024, src[i] + (int64_t)k * 1024, off);
        const uint8_t* const w = wsrc + (int64_t)k * kTileBytes;
        const uint32_t to = raw0 + (slot * FT + wave) * kRaw;
        load_lds16(to, w, 16u * lane);
        if constexpr (kMx4) load_lds4(to + 1024, w + kMx4Codes, 4u * (lane & 15));
        else load_lds16(to + 1024, w + 1024, 16u * lane);
    };
    // 4-bit: the wave's tile of stage kt, a block of 32 weights a lane, as bytes
    auto expand = [&](int kt) __attribute__((always_inline)) {
        if constexpr (kMx4) {
            const uint8_t* const raw = s_raw + ((kt % S) * FT + wave) * kRaw;
            const u32x4 code = *(const u32x4*)(raw + 16 * lane);
            const u32x4 lut = s_lut[raw[1024 + lane]];
            uint8_t* const to = s_exp + (kt & 1) * kExp + wave * 2048 + 64 * (lane >> 1);
#pragma unroll
            for (int half = 0; half < 2; half++) {
                uint32_t r[4];
#pragma unroll
                for (int d = 0; d < 4; d++) {
                    const uint32_t x = half ? code[d] >> 4 : code[d], sel = x & 0x07070707u;
                    const uint32_t neg = __builtin_amdgcn_perm(0, 0, ((x >> 3) & 0x01010101u) | 0x0c0c0c0cu);    // selector 12: 0x00, 13: 0xff
                    const uint32_t a = __builtin_amdgcn_perm(lut[1], lut[0], sel), b = __builtin_amdgcn_perm(lut[3], lut[2], sel);
                    r[d] = (a & ~neg) | (b & neg);
                }
                *(u32x4*)(to + 16 * w8_piece(lane >> 1, 2 * (lane & 1) + half)) = u32x4{r[0], r[1], r[2], r[3]};
            }
        }
    };

    // ---- products ----
    v16i acc[DA][FB];
#pragma unroll
    for (int d = 0; d < DA; d++)
#pragma unroll
        for (int f = 0; f < FB; f++)
#pragma unroll
            for (int r = 0; r < 16; r++) acc[d][f][r] = kMx4 ? 0 : (int)P.start;
    const int h = lane >> 5, j32 = lane & 31, l16 = lane & 15;
    const int da = wd * DA * 2048 + ((lane >> 4) & 1) * 1024 + h * 256 + (l16 >> 1) * 16 + (l16 & 1) * 8;
    const int fb0 = wf * FB * 2048 + 64 * j32 + 16 * w8_piece(j32, h), fb1 = wf * FB * 2048 + 64 * j32 + 16 * w8_piece(j32, 2 + h);
    auto multiply = [&](const uint8_t* dig, const uint8_t* wgt) __attribute__((always_inline)) {
#pragma unroll
        for (int s = 0; s < 2; s++) {
            v4i b[FB], a[DA];
#pragma unroll
            for (int f = 0; f < FB; f++) b[f] = *(const v4i*)(wgt + (s ? fb1 : fb0) + f * 2048);
#pragma unroll
            for (int d = 0; d < DA; d++) {
                const uint8_t* const at = dig + da + d * 2048 + s * 512;
                const v2i lo = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_v2i)(at)), hi = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_v2i)(at + 128));
                a[d] = v4i{lo[0], lo[1], hi[0], hi[1]};
            }
#pragma unroll
            for (int d = 0; d < DA; d++)
#pragma unroll
                for (int f = 0; f < FB; f++) acc[d][f] = __builtin_amdgcn_mfma_i32_32x32x32_i8(a[d], b[f], acc[d][f], 0, 0, 0);
        }
    };
#pragma unroll
    for (int kt = 0; kt < S - 1; kt++) issue(kt);
    if constexpr (kMx4) {
        // Stage kt: labels in slot kt % S, expanded weights in half kt & 1.  The barrier of stage kt stands behind the expansion of stage kt,
        // behind every read of stage kt - 1, and behind the arrival of stage kt + 1.
        wait_loads<(S - 2) * NL>();
        expand(0);          // (what a wave expands, it has loaded itself)
        for (int kt = 0; kt < nk; kt++) {
            wait_and_barrier<(S - 3) * NL>();
            issue(kt + S - 1);
            expand(kt + 1);
            multiply(s_dig + (kt % S) * kDig, s_exp + (kt & 1) * kExp);
        }
    } else {
        for (int kt = 0; kt < nk; kt++) {
            wait_and_barrier<(S - 2) * NL>();       // stage kt has arrived, stage kt - 1 has been read
            issue(kt + S - 1);
            multiply(s_dig + (kt % S) * kDig, s_raw + (kt % S) * FT * kRaw);
        }
    }
    wait_loads<0>();

    // ---- reduction mod p, 16 bytes a lane ----
    const uint32_t pow12 = P.pow12;
    const bool two_step = P.two_step != 0;
    auto red1 = [&](uint32_t v) __attribute__((always_inline)) { return v - mul24(mulhi(v, mmagic), prime); };
#pragma unroll
    for (int d = 0; d < DA; d++) {
        const int g0 = (wd * DA + d) * 2;
        uint8_t* const dst = s_dst[g0 + h];
#pragma unroll
        for (int f = 0; f < FB; f++) {
            const int j = by * TL::F + (wf * FB + f) * 32 + j32;
            uint32_t w[4];          // digits 4 h .. and 8 + 4 h .. of the first group, of the second
            uint32_t bm = 0;
            if (A.bias) {
                const int32_t b = j < M ? A.bias[(int64_t)e * M + j] % (int32_t)prime : 0;
                bm = (uint32_t)(b < 0 ? b + (int32_t)prime : b);
            }
#pragma unroll
            for (int q = 0; q < 4; q++) {
                uint32_t v[4];
#pragma unroll
                for (int r = 0; r < 4; r++) v[r] = (uint32_t)acc[d][f][4 * q + r];
                if (two_step) {
#pragma unroll
                    for (int r = 0; r < 4; r++) v[r] = mul24(red1(v[r] >> 12), pow12) + (v[r] & 4095u);
                }
                if (A.bias) {
                    const uint32_t one = s_one[g0 + q / 2][2 * (q % 2) + h];
#pragma unroll
                    for (int r = 0; r < 4; r++) v[r] = red1(v[r]) + mul24(bm, (one >> (8 * r)) & 0xffu);
                }
                w[q] = red1(v[0]) | red1(v[1]) << 8 | red1(v[2]) << 16 | red1(v[3]) << 24;
            }
            // lanes 0-31 hold dwords 0, 2 of both groups, lanes 32-63 dwords 1, 3: after the swaps the first half holds the first group
            const auto lo = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false), hi = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
            if (dst && j < M) *(u32x4*)(dst + (int64_t)j * 16) = u32x4{lo[0], lo[1], hi[0], hi[1]};
        }
    }
}

int experts_mfma(dash_ctx* c, const ExpertsCall& L, const dash_labels* in, dash_labels* out, hipStream_t s) {
    ExpArgs A;
    memset(&A, 0, sizeof(A));
    A.w = L.w; A.expert_bytes = matrix_bytes(L.format, L.M, L.K); A.bias = L.bias;
    A.M = L.M; A.K = L.K; A.E = L.E; A.n = (int)L.n; A.top_k = L.top_k;
    double macs = 0, bytes = (double)L.E * A.expert_bytes;
    int64_t blocks_big = 0;
    for (int i = 0; i < c->k; i++) {
        ExpPrime& P = A.pr[i];
        const ModInfo& Mi = c->mods[c->prime[i]];
        P.p = c->prime[i]; P.nchunk = Mi.nchunk; P.mmagic = Mi.mmagic; P.pow12 = 4096u % P.p;
        P.one = L.bias ? (L.garble ? c->d_one0[i] : c->d_one[i]) : nullptr;
        P.in = view_of(in, i); P.out = view_of(out, i);
        const uint64_t p1 = P.p - 1;
        uint64_t vmax = p1 * p1 * (uint64_t)L.K;
        if (L.format == DASH_W8) {
            P.start = (uint32_t)((128 * p1 * (uint64_t)L.K + P.p - 1) / P.p * P.p);
            vmax = P.start + 127 * p1 * (uint64_t)L.K;
        }
        // v / p = mulhi(v, mmagic) as long as v times the rounding of mmagic stays below 2^32; the quotient goes into a 24-bit product
        const uint64_t over = (uint64_t)P.mmagic * P.p - (1ull << 32);
        P.two_step = vmax * over >= (1ull << 32) || vmax / P.p >= (1u << 24);
        macs += (double)L.n * L.M * L.K * Mi.lam;
        bytes += ((double)(L.n / L.top_k) * L.K + (double)L.n * L.M) * Mi.lam;
        blocks_big += (int64_t)Mi.nchunk * L.n / EBig::G;
    }
    blocks_big *= (L.M + EBig::F - 1) / EBig::F;
    const bool big = c->experts_tile ? c->experts_tile == 1 : blocks_big >= 256;
    auto launch = [&](auto tl) -> int {
        typedef decltype(tl) TL;
        int64_t cols = 0;
        if (L.routing) {
            cols = L.routing->max_tiles[TL::SIZE];
            A.rows = L.routing->rows; A.tiles = L.routing->tiles[TL::SIZE]; A.n_tiles = L.routing->first_tile[TL::SIZE] + L.E + 1;
        } else
            for (int i = 0; i < c->k; i++) {
                A.first[i] = (int)cols;
                cols += ((int64_t)A.pr[i].nchunk * L.n + TL::G - 1) / TL::G;
                A.first[i + 1] = (int)cols;
            }
        const int64_t rows = (L.M + TL::F - 1) / TL::F;
        if (cols * rows > (1 << 30)) return DASH_ESIZE;
        // Work-groups go to the 8 XCDs in turn; the blocks of an XCD at one time share panels of weights and labels through its L2: super-tiles
        // of up to 4 x 8 blocks, smaller ones where there are too few blocks for all XCDs.
        int lg = 5;
        while (lg > 0 && (cols * rows) >> lg < 16) lg--;
        int lgy = 2;
        while (lgy > 0 && (1 << lgy) > rows) lgy--;
        if (lgy > lg) lgy = lg;
        A.lg_st = lg; A.lg_sty = lgy;
        A.col_blocks = (int)cols; A.row_blocks = (int)rows;
        A.gy = (int)((rows + (1 << lgy) - 1) >> lgy);
        const int64_t st = A.gy * ((cols + (1 << (lg - lgy)) - 1) >> (lg - lgy));
        A.st_total = (int)st;
        const int64_t grid = (st + 7) / 8 * 8 << lg;
        if (grid > 0x7fffffff) return DASH_ESIZE;
        ProfScope ps(c->prof, DASH_PROF_LINEAR, s, macs, bytes);
        auto kernel = L.format == DASH_MX4 ? k_experts_mfma<DASH_MX4, TL> : k_experts_mfma<DASH_W8, TL>;
        hipLaunchKernelGGL(kernel, dim3((uint32_t)grid), dim3(TL::T), 0, s, A);
        return DASH_OK;
    };
    const int st = big ? launch(EBig{}) : launch(ENarrow{});
    if (st) return st;
    DASH_HIP(hipGetLastError());
    return DASH_OK;
}

}  // namespace dash
