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

#include <type_traits>

#include "dash_experts.h"

#pragma clang diagnostic ignored "-Winline-asm"       // (m0 as a clobber)

namespace dash {

typedef int v2i __attribute__((ext_vector_type(2)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v16i __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) uint8_t* lds_ptr;
typedef __attribute__((address_space(3))) v2i* lds_v2i;

// WK sets of WD x WF waves (along the inputs; along digits, along features), a wave DA x FB tiles of 32 digits x 32 features; S stages of 64
// inputs in LDS for each set; WPE: waves per SIMD that the registers are held to; KIND: tiles of the routing (byte weights; + 2: 4-bit)
template <int WK_, int WD_, int WF_, int DA_, int FB_, int S_, int WPE_, int KIND_>
struct ETile {
    static constexpr int WK = WK_, WD = WD_, WF = WF_, DA = DA_, FB = FB_, S = S_, WPE = WPE_, KIND = KIND_;
    static constexpr int NW = WD * WF, T = 64 * NW * WK;
    static constexpr int G = 2 * WD * DA;            // groups per block
    static constexpr int FT = WF * FB, F = 32 * FT;  // feature tiles, features per block
    static constexpr int GP = G / NW, WT = FT / NW;  // groups and tiles of weights that a wave loads
    static_assert(G == kTileKind[KIND].groups && GP * NW == G && WT * NW == FT, "loader roles");
};
typedef ETile<1, 2, 4, 4, 2, 4, 2, 0> EBig;          // 256 digits x 256 features
typedef ETile<1, 2, 2, 2, 2, 4, 2, 1> ENarrow;       // 128 digits x 128 features
typedef ETile<2, 2, 2, 2, 2, 4, 2, 1> EDeep;         // the same by two sets of waves

struct ExpPrime {
    uint32_t p;
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
    int M, K, E, n, top_k, k;
    int cols, row_blocks, sty;          // blocks along the groups (without routing) and along the features; rows of a band
    int first[DASH_MAX_PRIMES + 1];     // without routing, 4-bit: first block along the groups of every prime
    int chunk_first[DASH_MAX_PRIMES + 1];   // first chunk of every prime in the numbering of all; past the last prime: a number no chunk has
    ExpPrime pr[DASH_MAX_PRIMES];
};

// 16 (4) bytes a lane from base + off to LDS at `to` + 16 (4) * lane.  In flight until a wait on vmcnt; nothing in registers.
__device__ __forceinline__ void load_lds16(uint32_t to, const uint8_t* base, uint32_t off) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(off), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ void load_lds4(uint32_t to, const uint8_t* base, uint32_t off) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(to), "v"(off), "s"(base) : "memory", "m0");
}
// the wave's LDS accesses done, then the block's barrier (loads stay in flight)
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
// at most N loads of the wave outstanding
template <int N> __device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
__device__ __forceinline__ const uint8_t* uniform(const uint8_t* p) {
    const uint64_t a = (uint64_t)p;
    return (const uint8_t*)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)a) |
                            (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(a >> 32)) << 32);
}

template <int FMT, class TL>
__global__ __launch_bounds__(TL::T, TL::WPE) void k_experts_mfma(const ExpArgs A) {
    constexpr int G = TL::G, DA = TL::DA, FB = TL::FB, S = TL::S, GP = TL::GP, WT = TL::WT, FT = TL::FT, NW = TL::NW, WK = TL::WK, T = TL::T;
    constexpr bool kMx4 = FMT == DASH_MX4;
    // ---- block -> tile ----
    // Work-groups go to the 8 XCDs in turn, each with an L2 of its own: an XCD takes a run of consecutive tiles, numbered in bands of `sty`
    // row blocks, row block after row block, then column after column.  The blocks on an XCD at one time then share a band's weights, which
    // stay in its L2 while the labels pass once.
    const int cols = A.tiles ? *A.n_tiles : A.cols, total = cols * A.row_blocks, run = (total + 7) >> 3;
    const int seq = blockIdx.x >> 3, at = (int)(blockIdx.x & 7) * run + seq;
    if (seq >= run || at >= total) return;
    const int band = at / (A.sty * cols), in_band = at - band * (A.sty * cols);
    const int height = A.row_blocks - band * A.sty < A.sty ? A.row_blocks - band * A.sty : A.sty;
    const int bx = in_band / height, by = band * A.sty + in_band - bx * height;
    int e = 0, pi = 0, start = 0, count = A.n, first;
    if (A.tiles) {
        const RouteTile t = A.tiles[bx];
        e = (int)(t.expert_prime & 0xffffffu); pi = (int)(t.expert_prime >> 24);
        start = t.start; count = t.count; first = t.first;
    } else if (kMx4) {
        while (bx >= A.first[pi + 1]) pi++;
        first = A.chunk_first[pi] * count + (bx - A.first[pi]) * G;
    } else first = bx * G;
    const int end = A.chunk_first[kMx4 ? pi + 1 : A.k] * count;        // groups of the tile: first .. min(first + G, end) - 1
    const int M = A.M, K = A.K;
    const int tid = threadIdx.x, lane = tid & 63, wave_ = __builtin_amdgcn_readfirstlane(tid >> 6), ws = wave_ / NW, wave = wave_ % NW;
    const int wd = wave / TL::WF, wf = wave % TL::WF;

    constexpr int kDig = G * 1024, kRaw = kMx4 ? 1280 : 2048;       // bytes of a stage's labels; of a stage's weights per feature tile, as loaded
    constexpr int kExp = FT * 2048;                                 // 4-bit: bytes of an expanded stage
    // one array: its address goes into the loads, so that the compiler takes all of it to change at their waits and barriers
    constexpr int kSet = S * kDig + S * FT * kRaw + (kMx4 ? 2 * kExp : 0);      // of a set of waves
    __shared__ __attribute__((aligned(1024))) uint8_t smem[WK * kSet];
    static_assert((WK - 1) * NW * TL::DA * TL::FB * 4096 <= WK * kSet, "the sums of the sets are added up in it");
    uint8_t* const s_dig = smem + ws * kSet;
    uint8_t* const s_raw = s_dig + S * kDig;
    uint8_t* const s_exp = s_raw + S * FT * kRaw;
    __shared__ u32x4 s_lut[kMx4 ? 256 : 1];
    __shared__ u32x4 s_one[G];
    __shared__ const uint8_t* s_src[G];
    __shared__ uint8_t* s_dst[G];
    __shared__ int s_prime[G];

    // ---- the groups of the tile ----
    if (tid < G) {
        const bool valid = first + tid < end;
        const int g = valid ? first + tid : first;                  // (a group past the end loads the tile's first and stores nothing)
        const int chunk = g / count, t = g - chunk * count, row = A.rows ? A.rows[start + t] : t;
        int p = 0;
#pragma unroll
        for (int i = 1; i < DASH_MAX_PRIMES; i++) p += chunk >= A.chunk_first[i] ? 1 : 0;
        const ExpPrime& P = A.pr[p];
        const int ch = chunk - A.chunk_first[p];
        s_src[tid] = P.in.p + (int64_t)ch * P.in.cs + (int64_t)(row / A.top_k) * K * 16;
        s_dst[tid] = valid ? P.out.p + (int64_t)ch * P.out.cs + (int64_t)row * M * 16 : nullptr;
        s_prime[tid] = p;
        if (A.bias) s_one[tid] = *(const u32x4*)(P.one + 16 * ch);
    }
    if (kMx4 && tid < 256) {
        // 2^tid mod p, times the eight magnitudes, and p minus that
        const uint32_t prime = A.pr[pi].p, mmagic = A.pr[pi].mmagic;
        uint32_t two = 1, sq = prime == 2 ? 0 : 2;
#pragma unroll
        for (int b = 0; b < 8; b++) {
            const uint32_t t = two * sq;
            if (tid >> b & 1) two = t - mul24(mulhi(t, mmagic), prime);
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
    // (a wave whose groups lie past the end loads weights alone; large tiles are rarely short)
    const bool loads_labels = DA > 2 || __builtin_amdgcn_readfirstlane(first + wave * GP < end);
    const int row_tiles_ = (M + 31) / 32;
    constexpr int kTileBytes = kMx4 ? kMx4Tile : kW8Tile;
    const uint8_t* wsrc[WT];
#pragma unroll
    for (int i = 0; i < WT; i++) {
        const int rt = by * FT + wave * WT + i;                     // (tiles past the end: the last again)
        wsrc[i] = uniform(A.w + (int64_t)e * A.expert_bytes + (int64_t)(rt < row_tiles_ ? rt : row_tiles_ - 1) * nk * kTileBytes);
    }
    const uint32_t dig0 = (uint32_t)(uintptr_t)(lds_ptr)s_dig, raw0 = (uint32_t)(uintptr_t)(lds_ptr)s_raw;
    // A set takes every WK-th stage of 64 inputs: its stage t are the inputs from 64 (WK t + ws).  Stage t goes into slot t % S; past the end
    // the last one again, so that every stage counts the same loads.  A stage's loads come in two parts, one for each half of the work on a stage.
    constexpr int kParts = 2 * WT + GP, kPart0 = (kParts + 1) / 2;
    // words 8 .. 15 of every 16 of a group with an odd number stand before words 0 .. 7: the reads of two groups meet different banks
    auto load_piece = [&](int t, int i) __attribute__((always_inline)) {
        const int slot = t % S, k = WK * t + ws < nk ? WK * t + ws : nk - 1;
        if (i < 2 * WT) {
            const uint8_t* const w = wsrc[i / 2] + (int64_t)k * kTileBytes;
            const uint32_t to = raw0 + (slot * FT + wave * WT + i / 2) * kRaw;
            if (i % 2 == 0) load_lds16(to, w, 16u * lane);
            else if constexpr (kMx4) load_lds4(to + 1024, w + kMx4Codes, 4u * (lane & 15));
            else load_lds16(to + 1024, w + 1024, 16u * lane);
        } else if (loads_labels) {
            const int g = i - 2 * WT, last = K - 1 - 64 * k, word = lane ^ (g & 1) * 8;     // words past K: the last again (their weights are zero)
            load_lds16(dig0 + slot * kDig + (wave * GP + g) * 1024, src[g] + (int64_t)k * 1024, 16u * (uint32_t)(word < last ? word : last));
        }
    };
    auto issue = [&](int t, int part) __attribute__((always_inline)) {
#pragma unroll
        for (int i = part ? kPart0 : 0; i < (part ? kParts : kPart0); i++) load_piece(t, i);
    };
    // at most N stages of the wave's loads outstanding
    auto arrived = [&](auto n) __attribute__((always_inline)) {
        constexpr int N = decltype(n)::value;
        if (loads_labels) wait_loads<N * kParts>(); else wait_loads<N * 2 * WT>();
    };
    // 4-bit: the wave's tiles of a stage, a block of 32 weights a lane: codes and shift, table entry (fetch), then bytes, 4 at a time (expand)
    u32x4 code[WT], lut[WT], bytes[WT];
    uint32_t shift[WT];
    auto fetch_codes = [&](int t) __attribute__((always_inline)) {
        if constexpr (kMx4) {
#pragma unroll
            for (int i = 0; i < WT; i++) {
                const uint8_t* const raw = s_raw + ((t % S) * FT + wave * WT + i) * kRaw;
                code[i] = *(const u32x4*)(raw + 16 * lane);
                shift[i] = raw[1024 + lane];
            }
        }
    };
    auto fetch_table = [&]() __attribute__((always_inline)) {
        if constexpr (kMx4) {
#pragma unroll
            for (int i = 0; i < WT; i++) lut[i] = s_lut[shift[i]];
        }
    };
    constexpr int kSteps = 8 * WT;
    auto expand = [&](int t, int step) __attribute__((always_inline)) {
        if constexpr (kMx4) {
            const int i = step / 8, half = step / 4 % 2, d = step % 4;
            const uint32_t x = half ? code[i][d] >> 4 : code[i][d], sel = x & 0x07070707u;
            const uint32_t neg = __builtin_amdgcn_perm(0, 0, ((x >> 3) & 0x01010101u) | 0x0c0c0c0cu);    // selector 12: 0x00, 13: 0xff
            const uint32_t a = __builtin_amdgcn_perm(lut[i][1], lut[i][0], sel), b = __builtin_amdgcn_perm(lut[i][3], lut[i][2], sel);
            bytes[i][d] = (a & ~neg) | (b & neg);
            if (d == 3) *(u32x4*)(s_exp + (t & 1) * kExp + (wave * WT + i) * 2048 + 64 * (lane >> 1) + 16 * w8_piece(lane >> 1, 2 * (lane & 1) + half)) = bytes[i];
        }
    };

    // ---- products ----
    v16i acc[DA][FB];
#pragma unroll
    for (int d = 0; d < DA; d++) {
        const int g0 = (wd * DA + d) * 2;
        const int s0 = kMx4 || ws ? 0 : (int)A.pr[__builtin_amdgcn_readfirstlane(s_prime[g0])].start, s1 = kMx4 || ws ? 0 : (int)A.pr[__builtin_amdgcn_readfirstlane(s_prime[g0 + 1])].start;
#pragma unroll
        for (int f = 0; f < FB; f++)
#pragma unroll
            for (int r = 0; r < 16; r++) acc[d][f][r] = r < 8 ? s0 : s1;
    }
    const int h = lane >> 5, j32 = lane & 31, l16 = lane & 15;
    const int odd = (lane >> 4) & 1;
    const int da = wd * DA * 2048 + odd * 1024 + h * 256 + (l16 >> 1) * 16 + (l16 & 1) * 8, da0 = da + odd * 128, da1 = da + 128 - odd * 128;
    const int fb0 = wf * FB * 2048 + 64 * j32 + 16 * w8_piece(j32, h), fb1 = wf * FB * 2048 + 64 * j32 + 16 * w8_piece(j32, 2 + h);
    // operands of one half (32 inputs) of stage t, in FB + 2 DA reads
    struct Operands { v4i b[FB]; v2i a[DA][2]; };
    auto read = [&](Operands& o, int t, int half, int i) __attribute__((always_inline)) {
        const uint8_t* const wgt = (kMx4 ? s_exp + (t & 1) * kExp : s_raw + (t % S) * FT * kRaw) + (half ? fb1 : fb0);
        const uint8_t* const dig = s_dig + (t % S) * kDig + half * 512;
        if (i < FB) o.b[i] = *(const v4i*)(wgt + i * 2048);
        else {
            const int d = (i - FB) / 2, second = (i - FB) % 2;
            o.a[d][second] = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_v2i)(dig + (second ? da1 : da0) + d * 2048));
        }
    };
    auto multiply = [&](const Operands& o, int i) __attribute__((always_inline)) {
        const int d = i / FB, f = i % FB;
        const v4i a = {o.a[d][0][0], o.a[d][0][1], o.a[d][1][0], o.a[d][1][1]};
        acc[d][f] = __builtin_amdgcn_mfma_i32_32x32x32_i8(a, o.b[f], acc[d][f], 0, 0, 0);
    };
    // Stage t in two halves of 32 inputs; the operands of its first half are in registers when it starts:
    //   products of the first half  | reads of the second half's operands; the second part of the loads of stage t - 1 + S; 4-bit: the
    //                                 second half of the expansion of stage t + 1
    //   wait for the loads of stage t + 1 (4-bit: t + 2), barrier
    //   products of the second half | the first part of the loads of stage t + S into the slot that stage t has left; reads of the first half
    //                                 of stage t + 1;
    //                                 4-bit: codes and table entries of stage t + 2, the first half of its expansion
    // The barrier stands behind all reads of stage t (each wave waits for its own), behind the expansion of stage t + 1, and behind
    // the arrival of stage t + 1.
    // The order inside a half is fixed: behind each product two reads (done well before the half ends), the loads far apart (a load that
    // cannot go out holds up the products behind it).
    using std::integral_constant;
    constexpr integral_constant<int, 0> k0{};
    constexpr integral_constant<int, 1> k1{};
    constexpr integral_constant<int, kMx4 ? S - 3 : S - 2> k_ahead{};
    const int stages = (nk + WK - 1) / WK;
    auto loop = [&](auto dn) __attribute__((always_inline)) {
        constexpr int kProducts = dn * FB, kReads = FB + 2 * dn;
        Operands o0, o1;
        auto half = [&](const Operands& now, Operands& next, bool there, int t_read, int half_read, int t_load, auto part, int t_expand) __attribute__((always_inline)) {
            constexpr int kSlots = kProducts > 4 ? kProducts : 4, kLoads = part ? kParts - kPart0 : kPart0;
#pragma unroll
            for (int m = 0; m < kSlots; m++) {
                if (m < kProducts && there) multiply(now, m);
#pragma unroll
                for (int i = 0; i < kReads; i++) if (i / 2 == m || (m == kSlots - 1 && i / 2 > m)) read(next, t_read, half_read, i);
                // (4-bit: the first half of an expansion follows its table entry, the second half has a half of products to itself)
                if constexpr (!part) {
                    if (m == 0) fetch_codes(t_expand);
                    if (m == kSlots / 4) fetch_table();
#pragma unroll
                    for (int i = 0; i < kSteps / 2; i++) if (kSlots / 2 + i * kSlots / kSteps == m) expand(t_expand, i);
                } else {
#pragma unroll
                    for (int i = 0; i < kSteps / 2; i++) if (i * 2 * kSlots / kSteps == m) expand(t_expand, kSteps / 2 + i);
                }
#pragma unroll
                for (int i = 0; i < kLoads; i++) if ((2 * i + 1) * kSlots / (2 * kLoads) == m) load_piece(t_load, (part ? kPart0 : 0) + i);
                __builtin_amdgcn_sched_barrier(0);
            }
        };
#pragma unroll
        for (int i = 0; i < kReads; i++) read(o0, 0, 0, i);
        fetch_codes(1);
        fetch_table();
#pragma unroll
        for (int i = 0; i < kSteps / 2; i++) expand(1, i);
        for (int t = 0; t < stages; t++) {
            const bool there = WK == 1 || WK * t + ws < nk;         // (the last round may be short of a stage for some sets)
            half(o0, o1, there, t, 1, t - 1 + S, k1, t + 1);
            arrived(k_ahead);
            lds_barrier();
            half(o1, o0, there, t + 1, 0, t + S, k0, t + 2);
        }
    };
#pragma unroll
    for (int t = 0; t < S; t++) { issue(t, 0); if (t < S - 1) issue(t, 1); }
    // (stages 0 and, 4-bit, 1; the last stage's second part is not out yet)
    auto first_arrived = [&](auto n) __attribute__((always_inline)) {
        constexpr int N = decltype(n)::value * kParts - (kParts - kPart0), NW8 = decltype(n)::value * 2 * WT - (2 * WT > kPart0 ? 2 * WT - kPart0 : 0);
        if (loads_labels) wait_loads<N>(); else wait_loads<NW8>();
    };
    if constexpr (kMx4) {
        first_arrived(integral_constant<int, S - 1>{});
        fetch_codes(0);
        fetch_table();
#pragma unroll
        for (int i = 0; i < kSteps; i++) expand(0, i);              // (what a wave expands, it has loaded itself)
        first_arrived(integral_constant<int, S - 2>{});
    } else first_arrived(integral_constant<int, S - 1>{});
    lds_barrier();
    if constexpr (DA > 2) loop(integral_constant<int, DA>{});
    else {
        // waves whose digits lie past the tile's groups, in part or whole, leave out those products
        const int mine = ((end - first + 1) >> 1) - wd * DA;
        if (mine >= DA) loop(integral_constant<int, DA>{});
        else if (mine > 0) loop(k1);
        else loop(k0);
    }
    wait_loads<0>();
    if constexpr (WK > 1) {
        // the sums of the other sets come through LDS
        lds_barrier();
        u32x4* const part = (u32x4*)smem + wave * DA * FB * 256 + lane;
#pragma unroll
        for (int s = 1; s < WK; s++) {
            if (ws == s) {
#pragma unroll
                for (int i = 0; i < DA * FB * 4; i++) {
                    const v16i& v = acc[i / 4 / FB][i / 4 % FB];
                    part[((s - 1) * NW * DA * FB * 4 + i) * 64] = u32x4{(uint32_t)v[i % 4 * 4], (uint32_t)v[i % 4 * 4 + 1], (uint32_t)v[i % 4 * 4 + 2], (uint32_t)v[i % 4 * 4 + 3]};
                }
            }
        }
        lds_barrier();
        if (ws) return;
#pragma unroll
        for (int s = 1; s < WK; s++)
#pragma unroll
            for (int i = 0; i < DA * FB * 4; i++) {
                const u32x4 v = part[((s - 1) * NW * DA * FB * 4 + i) * 64];
#pragma unroll
                for (int r = 0; r < 4; r++) acc[i / 4 / FB][i / 4 % FB][i % 4 * 4 + r] += (int)v[r];
            }
    }

    // ---- reduction mod p, 16 bytes a lane ----
#pragma unroll
    for (int d = 0; d < DA; d++) {
        const int g0 = (wd * DA + d) * 2;
        if (first + g0 >= end) break;
        uint8_t* const dst = s_dst[g0 + h];
        const ExpPrime* const P[2] = {&A.pr[__builtin_amdgcn_readfirstlane(s_prime[g0])], &A.pr[__builtin_amdgcn_readfirstlane(s_prime[g0 + 1])]};
#pragma unroll
        for (int f = 0; f < FB; f++) {
            const int j = by * TL::F + (wf * FB + f) * 32 + j32;
            uint32_t w[4];          // digits 4 h .. and 8 + 4 h .. of the first group, of the second
#pragma unroll
            for (int g = 0; g < 2; g++) {
                const uint32_t prime = P[g]->p, mmagic = P[g]->mmagic, pow12 = P[g]->pow12;
                auto red1 = [&](uint32_t v) __attribute__((always_inline)) { return v - mul24(mulhi(v, mmagic), prime); };
                uint32_t v[8];
#pragma unroll
                for (int r = 0; r < 8; r++) v[r] = (uint32_t)acc[d][f][8 * g + r];
                if (P[g]->two_step) {
#pragma unroll
                    for (int r = 0; r < 8; r++) v[r] = mul24(red1(v[r] >> 12), pow12) + (v[r] & 4095u);
                }
                if (A.bias) {
                    const int32_t b = j < M ? A.bias[(int64_t)e * M + j] % (int32_t)prime : 0;
                    const uint32_t bm = (uint32_t)(b < 0 ? b + (int32_t)prime : b);
#pragma unroll
                    for (int r = 0; r < 8; r++) v[r] = red1(v[r]) + mul24(bm, (s_one[g0 + g][2 * (r / 4) + h] >> (8 * (r % 4))) & 0xffu);
                }
#pragma unroll
                for (int q = 0; q < 2; q++) w[2 * g + q] = red1(v[4 * q]) | red1(v[4 * q + 1]) << 8 | red1(v[4 * q + 2]) << 16 | red1(v[4 * q + 3]) << 24;
            }
            // lanes 0-31 hold dwords 0, 2 of both groups, lanes 32-63 dwords 1, 3: after the swaps the first half holds the first group
            const auto lo = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false), hi = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
            if (dst && j < M) *(u32x4*)(dst + (int64_t)j * 16) = u32x4{lo[0], lo[1], hi[0], hi[1]};
            __builtin_amdgcn_sched_barrier(0);      // (else all accumulators are read at once)
        }
    }
}

int experts_mfma(dash_ctx* c, const ExpertsCall& L, const dash_labels* in, dash_labels* out, hipStream_t s) {
    ExpArgs A;
    memset(&A, 0, sizeof(A));
    A.w = L.w; A.expert_bytes = matrix_bytes(L.format, L.M, L.K); A.bias = L.bias;
    A.M = L.M; A.K = L.K; A.E = L.E; A.n = (int)L.n; A.top_k = L.top_k;
    double macs = 0, bytes = (double)L.E * A.expert_bytes;
    A.k = c->k;
    for (int i = 0; i <= DASH_MAX_PRIMES; i++) A.chunk_first[i] = 0x7fffffff;
    A.chunk_first[0] = 0;
    for (int i = 0; i < c->k; i++) {
        ExpPrime& P = A.pr[i];
        const ModInfo& Mi = c->mods[c->prime[i]];
        A.chunk_first[i + 1] = A.chunk_first[i] + (int)Mi.nchunk;
        P.p = c->prime[i]; P.mmagic = Mi.mmagic; P.pow12 = 4096u % P.p;
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
    }
    const int64_t groups = (int64_t)A.chunk_first[c->k] * L.n;
    if (groups > 0x7fffffff - 64) return DASH_ESIZE;
    auto launch = [&](auto tl) -> int {
        typedef decltype(tl) TL;
        const bool mx4 = L.format == DASH_MX4;
        int64_t cols = 0;
        if (L.routing) {
            const int s = TL::KIND + (mx4 ? 2 : 0);
            cols = L.routing->max_tiles[s];
            A.rows = L.routing->rows; A.tiles = L.routing->tiles[s]; A.n_tiles = L.routing->first_tile[s] + L.E + 1;
        } else if (mx4)
            for (int i = 0; i < c->k; i++) {
                A.first[i] = (int)cols;
                cols += ((int64_t)(A.chunk_first[i + 1] - A.chunk_first[i]) * L.n + TL::G - 1) / TL::G;
                A.first[i + 1] = (int)cols;
            }
        else cols = (groups + TL::G - 1) / TL::G;
        A.cols = (int)cols;
        A.row_blocks = (L.M + TL::F - 1) / TL::F;
        A.sty = 4;
        const int64_t total = cols * A.row_blocks;
        if (cols * A.sty > 0x7fffffff || total > 0x7fffff00) return DASH_ESIZE;
        ProfScope ps(c->prof, DASH_PROF_LINEAR, s, macs, bytes);
        auto kernel = mx4 ? k_experts_mfma<DASH_MX4, TL> : k_experts_mfma<DASH_W8, TL>;
        hipLaunchKernelGGL(kernel, dim3((uint32_t)((total + 7) / 8 * 8)), dim3(TL::T), 0, s, A);
        return DASH_OK;
    };
    const int64_t blocks_big = groups / EBig::G * ((L.M + EBig::F - 1) / EBig::F), blocks_narrow = (groups + 7) / 8 * ((L.M + 127) / 128);
    const int tile = c->experts_tile ? c->experts_tile : blocks_big >= 256 ? 1 : blocks_narrow <= 256 ? 3 : 2;
    const int st = tile == 1 ? launch(EBig{}) : tile == 3 ? launch(EDeep{}) : launch(ENarrow{});
    if (st) return st;
    DASH_HIP(hipGetLastError());
    return DASH_OK;
}

}  // namespace dash
