// dash_experts_kernel.h -- the products of expert layers as int8 MFMA contractions (dash_experts.hip has the formulas): the kernel and its launch;
// dash_experts_gemm.hip has the tiles of byte and 4-bit weights, dash_experts_f8.hip those of 8-bit floats.
//
// Shape.  A group is 16 digits (a chunk) of one row: in memory K words of 16 bytes, word i = the 16 digits of input i.  For all groups
// of one expert and prime the layer is one matrix product  Out^T (16 groups x M) = X^T (16 groups x K) * W^T (K x M).  The labels are
// the A operand and the weights the B operand of v_mfma_i32_32x32x32_i8: a lane then holds, for ONE output feature, 4 consecutive
// digits in 4 consecutive accumulators, so the result needs no turning around: pack 4 bytes, swap halves of the wave (2 groups a
// tile), store 16 bytes a lane, neighbouring lanes neighbouring features.
//
// Loads.  Everything comes by buffer loads that write LDS directly: no registers, no LDS write instructions, and what lies past the end of a
// row of inputs or of a row of weight tiles is left out by the buffer's size.  64 words of a group are 1 KB in a row, one instruction;
// prepared weights are laid out in tiles for the same.  Labels are turned around (the MFMA wants 16 consecutive inputs of one digit) by the
// LDS itself: ds_read_b64_tr_b8 gives lane l of 16 the byte l of 8 words.  A ring of S stages of 64 inputs, the loop unrolled over its
// slots; each wave waits for its own loads of the stages ahead (vmcnt counts down in order, all stages issue the same number), then
// one barrier a stage.  (With loads through registers and byte permutes, as the dense layers have them, the same product takes
// 1 096 us; with the slots as run-time numbers small tiles issued twice the instructions: one row, 4096 -> 4096: 40 us,
// unrolled 27 at that step.)
//
// Weights.  Signed bytes are the operand as they are, for every prime: a tile goes across primes, the sums start at a multiple of p that
// keeps them positive and are reduced once.  4-bit floats: 2 e2m1 2^shift mod p by table: the 8 magnitudes of a shift and their
// negatives are 16 bytes of LDS; two v_perm pick four of each by four 3-bit codes, a third picks by the signs: 6.5 instructions for
// four weights.  The largest tiles expand a stage's weights once a block, through LDS, into the layout of the byte weights; in the others a
// wave's weights are its own and stay in registers.
//
// What bounds it (us).  128 rows, 4096 -> 4096, 12 primes: 960 to 1 025 with bytes from box to box (2.3 to 2.5 POP/s counted over the label digits, 2.6 to
// 2.8 with the zero digits of the last chunks; a library's int8 product of 16384 reaches 2.4): power, the matrix pipe is busy 76 % of the cycles and the clock falls
// from 2.7 to 1.6 GHz.  4-bit: 1 010 to 1 060, the expansion beside it.  32 experts, 256 rows, 1024 -> 2048, 4-bit: 358 to 367 with 128 x 256 tiles, two
// blocks a CU (256 x 256, one block: 412): vector instructions of the expansion in 65 % of the cycles, the matrix pipe in 39 %.  One row,
// 4096 -> 4096, 4-bit: 26; latency of the stages, about 110 instructions by two to four waves a SIMD.  One row, 784 -> 128, 4-bit: 7.1 to 7.4,
// 4.8 of them for a single stage: launch, the chain of loads to the first labels, results.
//
// 8-bit floats.  512 e4m3 S mod m by a table of 256 bytes in LDS, one for every scale (128 inputs) that a block passes: a byte read a weight (64 lanes in 4.3
// clocks, bank conflicts among them; 2.8 with the signs apart in 128 entries, whose instructions cost more than that saves), joined by two v_perm and a v_or for four.  An operand
// holds 32 features, so what a table read serves is the tile's digits: 512 of them where the weights are expanded once a block, 256 or 128 where a wave's
// weights are its own.  m is a prime of the tile, or the product (up to 240: signed bytes) of a class of primes whose digits then share a tile and its reads: 2, 3, 5,
// ... 37 are 6 classes, one row of them 7 tiles of 128 digits instead of 12.  The sums take either sign and start at a multiple of p, as with bytes.
//   Where many blocks wait, residues of single primes are better, as bytes up to 37 leave more of the power to the clock (128 rows, 4096 -> 4096, largest tile:
// 1 137 us, classes 1 271).
//   What bounds it.  128 rows, 4096 -> 4096, 12 primes: 1 127, of the cycles the LDS busy in 49 %, the matrix pipe in 49, vector instructions in 30, at 1.7 to 2.2 GHz.  With
// 128 x 128 tiles the table reads: LDS 84 %, 1 638.  32 experts, 256 rows, 1024 -> 2048: 455 (256 x 128).  One row, 4096 -> 4096: 34.0, a stage 0.43
// us in each of 224 blocks, the time of its LDS accesses (tables 550 clocks, labels 256, codes and loads 190), 0.185 without the expansion.  One row, 784 -> 128: 10.6, 5.9 for a single
// stage, then 0.65 for two.
//   The compiler must not see accesses that could be LDS or scalar loads near the loop: from then on it waits for all LDS results at once (narrow tiles 1 702 -> 1 638).
#pragma once
#include <string.h>

#include <type_traits>

#include "dash_experts.h"
#include "dash_experts_rule.h"

#pragma clang diagnostic ignored "-Winline-asm"       // (m0 as a clobber)

namespace dash {

typedef int v2i __attribute__((ext_vector_type(2)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v16i __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) uint8_t* lds_ptr;
typedef __attribute__((address_space(3))) v2i* lds_v2i;
// addresses that come as numbers are device memory's (of accesses that could be LDS the compiler waits for all of LDS, lgkmcnt(0), from there on)
typedef __attribute__((address_space(1))) uint8_t* global_ptr;
typedef __attribute__((address_space(1))) u32x4* global_u32x4;
typedef const __attribute__((address_space(1))) uint32_t* global_u32;

// WK sets of WD x WF waves (along the inputs; along digits, along features), a wave DA x FB tiles of 32 digits x 32 features; S stages of 64
// inputs in LDS for each set; KIND: tiles of the routing; PERSIST: a block takes tile after tile (one block per CU)
template <int WK_, int WD_, int WF_, int DA_, int FB_, int S_, int KIND_, bool PERSIST_>
struct ETile {
    static constexpr int WK = WK_, WD = WD_, WF = WF_, DA = DA_, FB = FB_, S = S_, KIND = KIND_;
    static constexpr bool PERSIST = PERSIST_;
    static constexpr int NW = WD * WF, T = 64 * NW * WK;
    static constexpr int G = 2 * WD * DA;            // groups per block
    static constexpr int FT = WF * FB, F = 32 * FT;  // feature tiles, features per block
    static constexpr int GP = G / NW, WT = FT / NW;  // groups and tiles of weights that a wave loads
    static constexpr bool HALF = FT * 2 == NW;       // a wave loads half a tile of weights
    static_assert(G == kTileKind[KIND].groups && GP * NW == G && (HALF || WT * NW == FT), "loader roles");
    static_assert(!PERSIST || WK == 1, "the sets' sums go through the slots");
};

constexpr int kCus = 256;       // (a multiple of the 8 XCDs)

struct ExpPrime {
    uint32_t p;
    uint32_t mmagic;            // ceil(2^32 / p)
    uint32_t pow12;             // 4096 mod p
    uint32_t start;             // multiple of p that the sums start at
    int32_t chunk_first;        // first chunk in the numbering of all
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
    int plain;                          // no bias, and every sum v below the bound up to which v / p is one multiplication by mmagic
    int cols, row_blocks, sty;          // blocks along the groups (without routing) and along the features; rows of a band
    int first[DASH_MAX_PRIMES + 1];     // without routing, 4-bit: first block along the groups of every prime
    int chunk_first[DASH_MAX_PRIMES + 1];   // first chunk of every prime in the numbering of all; past the last prime: a number no chunk has
    ExpPrime pr[DASH_MAX_PRIMES];
    // 8-bit floats: the parts, primes or classes of them (the primes above then stand in their order)
    int part_first[DASH_MAX_PRIMES + 1];    // first chunk of every part
    struct { uint32_t m, magic; } part[DASH_MAX_PRIMES];     // a part's modulus and ceil(2^32 / m)
};

// 16 (4) bytes a lane from offset `off` + At of the buffer to LDS at `to` + Slot + At + 16 (4) * lane; a lane whose offset lies past the end of
// the buffer reads nothing.  In flight until a wait on vmcnt; no registers.  A buffer's words that a vector instruction has written (a readfirstlane,
// a spilled word's way back) may be read five wait states later at the earliest, and the compiler does not look after that in front of an assembly
// block: the block brings all five, whatever stands in front of it.
template <int Slot, int At> __device__ __forceinline__ void load_lds16(uint32_t to, const v4i& buffer, uint32_t off) {
    asm volatile("s_add_u32 m0, %0, %3\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %2, 0 offen offset:%4 lds" ::"s"(to), "v"(off), "s"(buffer), "n"(Slot), "n"(At) : "memory", "m0", "scc");
}
template <int Slot> __device__ __forceinline__ void load_lds4(uint32_t to, const v4i& buffer, uint32_t off) {
    asm volatile("s_add_u32 m0, %0, %3\n\ts_nop 3\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(to), "v"(off), "s"(buffer), "n"(Slot) : "memory", "m0", "scc");
}
// a buffer of `bytes` bytes without a format (raw, stride 0)
__device__ __forceinline__ v4i buffer_of(const uint8_t* p, uint32_t bytes) {
    const uint64_t a = (uint64_t)p;
    return v4i{__builtin_amdgcn_readfirstlane((int)(uint32_t)a), __builtin_amdgcn_readfirstlane((int)(uint32_t)(a >> 32) & 0xffff),
               __builtin_amdgcn_readfirstlane((int)bytes), 0x00020000};
}
__device__ __forceinline__ uint32_t lane_of(uint32_t v, int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)v, lane); }
__device__ __forceinline__ uint64_t lane_of(uint64_t v, int lane) { return lane_of((uint32_t)v, lane) | (uint64_t)lane_of((uint32_t)(v >> 32), lane) << 32; }
// The wave's LDS accesses done, then the block's barrier (loads stay in flight).  The wait behind it has nothing to wait for: it tells the compiler, which does not see the other,
// that no scalar load is out, whose end it would have to expect before every LDS result (lgkmcnt(0) everywhere, fresh reads waited for in front of products).
__device__ __forceinline__ void lds_barrier() {
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xc07f);
}
// at most N loads of the wave outstanding
template <int N> __device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
template <int FMT, class TL>
__global__ __launch_bounds__(TL::T, 2) void k_experts_mfma(const ExpArgs A) {
    constexpr int G = TL::G, DA = TL::DA, FB = TL::FB, S = TL::S, GP = TL::GP, WT = TL::HALF ? 1 : TL::WT, FT = TL::FT, NW = TL::NW, WK = TL::WK;
    constexpr bool kMx4 = FMT == DASH_MX4, kF8 = FMT == DASH_F8;
    constexpr bool kPart = kMx4 || kF8;                 // residues of the weights: a tile is of one prime or class
    constexpr bool kDirect = kPart && TL::WD == 1;      // a wave's weights are its own: expanded in registers
    constexpr bool kHalfTile = TL::HALF;
    constexpr bool kClass = kTileKind[TL::KIND].parts == PARTS_CLASSES;
    static_assert(!kHalfTile || (kF8 && !kDirect), "loader roles");
    static_assert(!kF8 || WK <= 2, "a round of the sets' stages is of one block of 128 inputs or half of one");
    static_assert(!kF8 || kDirect || kHalfTile, "steps of the expansion");
    const int M = A.M, K = A.K, nk = (K + 63) / 64;
    const int tid = threadIdx.x, lane = tid & 63, wave_ = __builtin_amdgcn_readfirstlane(tid >> 6), ws = wave_ / NW, wave = wave_ % NW;
    const int wd = wave / TL::WF, wf = wave % TL::WF;

    // ---- block -> tiles ----
    // Work-groups go to the 8 XCDs in turn, each with an L2 of its own: an XCD takes a run of consecutive tiles, numbered in bands of `sty`
    // row blocks, row block after row block, then column after column.  The blocks on an XCD at one time then share a band's weights, which
    // stay in its L2 while the labels pass once.
    const int cols = A.tiles ? __builtin_amdgcn_readfirstlane(*A.n_tiles) : A.cols, total = cols * A.row_blocks, run = (total + 7) >> 3, run0 = (int)(blockIdx.x & 7) * run;
    struct Tile { int by, e, pi, start, count, first, n_groups; };      // n_groups: groups first .. first + n_groups - 1, at most G
    auto decode = [&](int seq, Tile& t) __attribute__((always_inline)) -> bool {
        const int at = run0 + seq;
        if (seq >= run || at >= total) return false;
        const int band = at / (A.sty * cols), in_band = at - band * (A.sty * cols);
        const int height = A.row_blocks - band * A.sty < A.sty ? A.row_blocks - band * A.sty : A.sty;
        const int bx = in_band / height;
        t.by = band * A.sty + in_band - bx * height;
        t.e = 0; t.pi = 0; t.start = 0; t.count = A.n;
        if (A.tiles) {
            const RouteTile r = A.tiles[bx];
            const uint32_t ep = (uint32_t)__builtin_amdgcn_readfirstlane((int)r.expert_prime);
            t.e = (int)(ep & 0xffffffu); t.pi = (int)(ep >> 24);
            t.start = __builtin_amdgcn_readfirstlane(r.start); t.count = __builtin_amdgcn_readfirstlane(r.count);
            t.first = __builtin_amdgcn_readfirstlane(r.first);
        } else if (kPart) {
            while (bx >= A.first[t.pi + 1]) t.pi++;
            t.first = (kF8 ? A.part_first : A.chunk_first)[t.pi] * t.count + (bx - A.first[t.pi]) * G;
        } else t.first = bx * G;
        const int end = (kF8 ? A.part_first[t.pi + 1] : A.chunk_first[kMx4 ? t.pi + 1 : A.k]) * t.count;
        t.n_groups = end - t.first < G ? end - t.first : G;
        return true;
    };

    constexpr int kDig = G * 1024, kRaw = kMx4 ? 1280 : 2048;       // bytes of a stage's labels; of a stage's weights per feature tile, as loaded
    constexpr int kExp = kPart && !kDirect ? FT * 2048 : 0;         // bytes of an expanded stage
    // one array: its address goes into the loads, so that the compiler takes all of it to change at their waits and barriers
    constexpr int kSet = S * kDig + S * FT * kRaw + 2 * kExp;       // of a set of waves
    __shared__ __attribute__((aligned(1024))) uint8_t smem[WK * kSet];
    static_assert((WK - 1) * NW * DA * FB * 4096 <= WK * kSet, "the sums of the sets are added up in it");
    uint8_t* const s_dig = smem + ws * kSet;
    uint8_t* const s_raw = s_dig + S * kDig;
    uint8_t* const s_exp = s_raw + S * FT * kRaw;
    __shared__ u32x4 s_lut[kMx4 ? 256 : 1];
    static_assert(!kF8 || kScaleBlock % TL::F == 0, "a block's features have one row of scales");
    __shared__ __attribute__((aligned(256))) uint8_t s_f8[kF8 ? 512 : 16];      // tables of two blocks of 128 inputs

    // the primes, for lanes that each want another
    struct PrimeLds { uint64_t in, in_cs, out, out_cs, one; uint32_t p, mmagic, pow12, start, chunk_first, pad; };
    __shared__ PrimeLds s_pr[DASH_MAX_PRIMES];
    if (tid < A.k) {
        const ExpPrime& P = A.pr[tid];
        s_pr[tid] = PrimeLds{(uint64_t)P.in.p, (uint64_t)P.in.cs, (uint64_t)P.out.p, (uint64_t)P.out.cs, (uint64_t)P.one, P.p, P.mmagic, P.pow12, P.start, (uint32_t)P.chunk_first, 0};
    }

    // ---- the groups of a tile: group g of it in lane g of every wave ----
    struct Begun { int chunk, row; };           // chunk in the numbering of all, row (a load in flight)
    auto begin = [&](const Tile& t) __attribute__((always_inline)) -> Begun {
        const int g = t.first + (lane < t.n_groups ? lane : 0), chunk = g / t.count, at = g - chunk * t.count;
        return Begun{chunk, A.rows ? A.rows[t.start + at] : at};
    };
    struct Groups { uint64_t src, dst, one; uint32_t prime, magic, pow12, start; };
    auto groups_of = [&](const Begun& b) __attribute__((always_inline)) -> Groups {
        int p = 0;
#pragma unroll
        for (int i = 1; i < DASH_MAX_PRIMES; i++) p += b.chunk >= A.chunk_first[i] ? 1 : 0;
        const PrimeLds& P = s_pr[p];
        const int64_t ch = b.chunk - (int)P.chunk_first;
        Groups g;
        g.src = P.in + ch * P.in_cs + (int64_t)(b.row / A.top_k) * K * 16;
        g.dst = P.out + ch * P.out_cs + (int64_t)b.row * M * 16;
        g.one = P.one + 16 * ch;
        g.prime = P.p; g.magic = P.mmagic; g.pow12 = P.pow12; g.start = P.start;
        return g;
    };
    // rows of no expert: the value 0 on both sides
    auto zeros = [&](const Tile& t) __attribute__((always_inline)) {
        const Groups z = groups_of(begin(t));
        for (int g = wave_; g < t.n_groups; g += NW * WK) {
            const global_ptr dst = (global_ptr)lane_of(z.dst, g);
            for (int j = t.by * TL::F + lane; j < M && j < t.by * TL::F + TL::F; j += 64) *(global_u32x4)(dst + (int64_t)j * 16) = u32x4{0, 0, 0, 0};
        }
    };
    // the block's next tile with an expert
    int seq = (int)(blockIdx.x >> 3) + ((int)blockIdx.y - (int)gridDim.y) * (int)(gridDim.x >> 3);
    auto next_tile = [&](Tile& t) __attribute__((always_inline)) -> bool {
        for (;;) {
            seq += (int)gridDim.y * (int)(gridDim.x >> 3);
            if (!decode(seq, t)) return false;
            if (t.e < A.E) return true;
            zeros(t);
        }
    };

    // ---- loads ----
    constexpr int kTileBytes = kMx4 ? kMx4Tile : kW8Tile;
    v4i lab[GP], wgt[WT];
    uint32_t off_w, off_s, off_l;
    auto open_weights = [&](const Tile& t) __attribute__((always_inline)) {
        const uint8_t* const wexp = A.w + (int64_t)t.e * A.expert_bytes;
#pragma unroll
        for (int i = 0; i < WT; i++) {                              // (tiles past the last: empty buffers)
            const int rt = t.by * FT + (kHalfTile ? wave >> 1 : wave * WT + i);
            wgt[i] = buffer_of(wexp + (int64_t)rt * nk * kTileBytes, rt < (M + 31) / 32 ? (uint32_t)(nk * kTileBytes) : 0u);
        }
        off_w = 16u * lane + ws * kTileBytes + (kHalfTile ? (wave & 1) * 1024u : 0u); off_s = 4u * (lane & 15) + kMx4Codes + ws * kTileBytes;
    };
    auto open_labels = [&](const Tile& t, const Groups& g) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < GP; i++) lab[i] = buffer_of((const uint8_t*)lane_of(g.src, wave * GP + i), wave * GP + i < t.n_groups ? (uint32_t)K * 16u : 0u);
        off_l = (16u * lane ^ (GP % 2 ? (wave & 1) * 128u : 0u)) + ws * 1024;
    };
    const uint32_t dig0 = (uint32_t)(uintptr_t)(lds_ptr)s_dig + wave * GP * 1024, raw0 = (uint32_t)(uintptr_t)(lds_ptr)s_raw + (kHalfTile ? wave * 1024 : wave * WT * kRaw);
    // A set takes every WK-th stage of 64 inputs: its stage t, the inputs from 64 (WK t + ws), goes into slot t % S.  Stages past the end load nothing (their offsets lie past the buffers) but count.  A
    // lane's offsets run along with the stages.
    // Words 8 .. 15 of every 16 of a group with an odd number stand before words 0 .. 7: the reads of two groups meet different banks.
    constexpr int kWLoads = kHalfTile ? 1 : 2 * WT, kParts = kWLoads + GP;       // loads of a stage: weights, then labels
    auto load_weights = [&](auto slot, int i) __attribute__((always_inline)) {
        constexpr int kSlot = decltype(slot)::value % S * FT * kRaw;
        const uint32_t to = raw0 + i / 2 * kRaw;
        if (i % 2 == 0) load_lds16<kSlot, 0>(to, wgt[i / 2], off_w);
        else if constexpr (kMx4) load_lds4<kSlot + kMx4Codes>(to, wgt[i / 2], off_s);
        else load_lds16<kSlot, 1024>(to, wgt[i / 2], off_w);
        if (i == kWLoads - 1) { off_w += WK * kTileBytes; off_s += WK * kTileBytes; }
    };
    auto load_labels = [&](auto slot, int i) __attribute__((always_inline)) {
        constexpr int kSlot = decltype(slot)::value % S * kDig;
        load_lds16<kSlot, 0>(dig0 + i * 1024, lab[i], i % 2 ? off_l ^ 128u : off_l);          // (the wave's second group has an odd number; with one group a wave, see open)
        if (i == GP - 1) off_l += WK * 1024;
    };

    // ---- 4-bit weights ----
    const int h = lane >> 5, j32 = lane & 31, l16 = lane & 15;
    auto make_table = [&](int pi) __attribute__((always_inline)) {
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
    };
    // ---- 8-bit floats ----
    // Code c under the scale S: 512 e4m3(c) S mod m, m the prime of the tile or the product of the primes of its class, a byte of a table of 256 for every 128 inputs.  Thread c
    // keeps its code's residue and multiplies it by the scale's; lane l of every wave keeps the residue of one of 64 scales.  (Scales by scalar loads where they are
    // wanted: waits for memory in front of the barriers, 128 rows, 4096 -> 4096: 1158 us.)
    uint32_t f8_residue = 0, f8_mod = 0, f8_magic = 0, f8_scale = 0;
    const int32_t* f8_scales = nullptr;
    const int f8_blocks = (K + kScaleBlock - 1) / kScaleBlock;
    int32_t f8_loaded = 0;
    // A window of the scales: 64 of the tile's row of them, from number `first` (past the end: the last), number i in lane i % 64; a load in flight
    auto load_scales = [&](int first) __attribute__((always_inline)) {
        if constexpr (kF8) {
            const int i = first + ((lane - first) & 63);
            f8_loaded = f8_scales[i < f8_blocks ? i : f8_blocks - 1];
        }
    };
    auto open_scales = [&](const Tile& t) __attribute__((always_inline)) {
        if constexpr (kF8) {
            f8_scales = (const int32_t*)(A.w + (int64_t)t.e * A.expert_bytes + scales_at(M, K)) + (int64_t)(t.by * TL::F / kScaleBlock) * f8_blocks;
            load_scales(0);
        }
    };
    auto take_scales = [&]() __attribute__((always_inline)) {
        if constexpr (kF8) {
            // |S| up to 2^31 in two steps
            const int32_t v = f8_loaded;
            const uint32_t a = v < 0 ? 0u - (uint32_t)v : (uint32_t)v, pow12 = 4096u - mul24(mulhi(4096u, f8_magic), f8_mod);
            auto red1 = [&](uint32_t n) __attribute__((always_inline)) { return n - mul24(mulhi(n, f8_magic), f8_mod); };
            const uint32_t r = red1(mul24(red1(a >> 12), pow12) + (a & 4095u));
            f8_scale = v < 0 && r ? f8_mod - r : r;
        }
    };
    auto open_table = [&](const Tile& t) __attribute__((always_inline)) {
        if constexpr (kF8) {
            f8_mod = A.part[t.pi].m; f8_magic = A.part[t.pi].magic;
            const uint32_t mag = f8_magnitude(tid & 0x7f) % f8_mod;
            f8_residue = (tid & 0x80) && mag ? f8_mod - mag : mag;
            take_scales();
        }
    };
    // the table of inputs 128 kb .. 128 kb + 127 (past the end: any)
    auto make_f8 = [&](int kb) __attribute__((always_inline)) {
        if constexpr (kF8) {
            // (without a branch for the waves past the fourth, which write the same again: a branch amid the products makes the reads around it be waited for)
            const uint32_t v = mul24(f8_residue, lane_of(f8_scale, kb & 63)), r = v - mul24(mulhi(v, f8_magic), f8_mod);
            s_f8[(kb & 1) * 256 + (tid & 255)] = (uint8_t)(kClass && 2 * r > f8_mod ? r - f8_mod : r);
        }
    };
    // four codes' bytes; base: the table's address in LDS (a multiple of 256, below 2^24)
    auto look4 = [&](uint32_t (&r)[4], uint32_t x, uint32_t base) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 4; i++) r[i] = *(lds_ptr)(uintptr_t)__builtin_amdgcn_perm(x, base, 0x0c020104u + (uint32_t)i);
    };
    auto join4 = [&](const uint32_t (&r)[4]) __attribute__((always_inline)) -> uint32_t {
        return __builtin_amdgcn_perm(r[1], r[0], 0x0c0c0400u) | __builtin_amdgcn_perm(r[3], r[2], 0x04000c0cu);
    };
    const uint32_t f8_base = (uint32_t)(uintptr_t)(lds_ptr)s_f8;
    constexpr int kUnroll = S == 3 ? 6 : S;         // stages of a round of the loop: slots and parities are known in each
    // A lane's 16 bytes of codes are 16 weights of a row's first block of 32 and 16 of its second (low and high halves of the bytes); shifts of
    // both blocks, table entries of both, then four weights at a time as bytes.
    // In registers (a wave's weights are its own: kDirect): lane (j32, h) holds what it multiplies, two stages in the making.
    // Else through LDS: lane (row, half) = (lane / 2, lane % 2).
    constexpr int kMaking = kDirect ? 2 : 1;
    u32x4 code[kMaking][WT], lut[2][WT], bytes[WT];
    uint32_t shift[WT];
    const uint8_t* const raw_codes = s_raw + wave * WT * kRaw + 16 * (kDirect ? 2 * j32 + h : lane);
    const uint8_t* const raw_shifts = s_raw + wave * WT * kRaw + kMx4Codes + 2 * (kDirect ? j32 : lane >> 1);
    // (8-bit floats: the codes of half `b` of a stage)
    // (through LDS: the lane's 16 codes of the stage)
    const uint8_t* const raw_f8 = kHalfTile ? s_raw + wave * 1024 + 16 * lane : s_raw + wave * WT * kRaw + 64 * j32;
    auto fetch_codes = [&](auto slot, int b) __attribute__((always_inline)) {
        if constexpr (kF8 && !kDirect) code[0][0] = *(const u32x4*)(raw_f8 + decltype(slot)::value % S * FT * kRaw);
        else if constexpr (kF8) {
#pragma unroll
            for (int i = 0; i < WT; i++) code[b][i] = *(const u32x4*)(raw_f8 + 16 * w8_piece(j32, 2 * b + h) + (decltype(slot)::value % S * FT + i) * kRaw);
        }
        if constexpr (kMx4) {
#pragma unroll
            for (int i = 0; i < WT; i++) {
                code[b][i] = *(const u32x4*)(raw_codes + (decltype(slot)::value * FT + i) * kRaw);
                shift[i] = *(const uint16_t*)(raw_shifts + (decltype(slot)::value * FT + i) * kRaw);
            }
        }
    };
    auto fetch_table = [&](int block) __attribute__((always_inline)) {
        if constexpr (kMx4) {
#pragma unroll
            for (int i = 0; i < WT; i++) lut[block][i] = s_lut[block ? shift[i] >> 8 : shift[i] & 255u];
        }
    };
    uint32_t k3210 = 0x03020100u;
    asm volatile("" : "+v"(k3210));             // (in a register: one instruction takes one literal)
    auto four = [&](uint32_t x, const u32x4& l, int block) __attribute__((always_inline)) -> uint32_t {
        // (v_bitop3_b32 takes half the time of v_and_or_b32: one row, 4096 -> 4096: 25.7 -> 24.3 us)
        const uint32_t sel = (block ? x >> 4 : x) & 0x07070707u, sign = __builtin_amdgcn_bitop3_b32(block ? x >> 5 : x >> 1, 0x04040404u, k3210, 0xea);     // a & b | c
        return __builtin_amdgcn_perm(__builtin_amdgcn_perm(l[3], l[2], sel), __builtin_amdgcn_perm(l[1], l[0], sel), sign);
    };
    constexpr int kSteps = kHalfTile ? 4 : 8 * WT;
    uint8_t* const exp_to0 = s_exp + wave * WT * 2048 + 64 * (lane >> 1) + 16 * w8_piece(lane >> 1, lane & 1);
    uint8_t* const exp_to1 = s_exp + wave * WT * 2048 + 64 * (lane >> 1) + 16 * w8_piece(lane >> 1, 2 + (lane & 1));
    // (steps of the first block of every tile, then of the second)
    auto expand = [&](int parity, int step) __attribute__((always_inline)) {
        if constexpr (kMx4 && !kDirect) {
            const int block = step / (4 * WT), i = step / 4 % WT, d = step % 4;
            bytes[i][d] = four(code[0][i][d], lut[block][i], block);
            if (d == 3) *(u32x4*)((block ? exp_to1 : exp_to0) + parity * kExp + i * 2048) = bytes[i];
        }
    };

    uint8_t* const exp8_to = s_exp + wave * 1024 + 16 * lane;
    auto expand8 = [&](int parity, uint32_t base) __attribute__((always_inline)) {
        if constexpr (kF8 && !kDirect) {
#pragma unroll
            for (int i = 0; i < 4; i++) {
                uint32_t look[4];
                look4(look, code[0][0][i], base);
                bytes[0][i] = join4(look);
            }
            *(u32x4*)(exp8_to + parity * kExp) = bytes[0];
        }
    };

    // ---- products ----
    const int odd = (lane >> 4) & 1;
    const uint8_t* const da = s_dig + wd * DA * 2048 + odd * 1024 + h * 256 + (l16 >> 1) * 16 + (l16 & 1) * 8;
    const uint8_t* const da0 = da + odd * 128;
    const uint8_t* const da1 = da + 128 - odd * 128;
    const uint8_t* const fb = (kPart ? s_exp : s_raw) + wf * FB * 2048 + 64 * j32;
    const uint8_t* const fb0 = fb + 16 * w8_piece(j32, h);
    const uint8_t* const fb1 = fb + 16 * w8_piece(j32, 2 + h);
    // operands of one half (32 inputs) of a stage, in FB + 2 DA reads
    struct Operands { v4i b[FB]; v2i a[DA][2]; };
    auto read = [&](Operands& o, auto slot, int half, int i) __attribute__((always_inline)) {
        constexpr int kSlot = decltype(slot)::value;
        if (i < FB) {
            if constexpr (!kDirect) o.b[i] = *(const v4i*)((half ? fb1 : fb0) + (kPart ? (kSlot & 1) * kExp : kSlot * FT * kRaw) + i * 2048);
        } else {
            const int d = (i - FB) / 2, second = (i - FB) % 2;
            o.a[d][second] = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_v2i)((second ? da1 : da0) + kSlot % S * kDig + half * 512 + d * 2048));
        }
    };
    // Stage t in two halves of 32 inputs; the operands of its first half are in registers when it starts:
    //   products of the first half  | reads of the second half's operands; loads of the labels of stage t - 1 + S
    //   wait for the loads of stage t + 1 (4-bit: and the weights of stage t + 2), barrier
    //   products of the second half | loads of the weights of stage t + S; reads of the first half of stage t + 1
    // The barrier stands behind all reads of stage t (each wave waits for its own) and behind the arrival of stage t + 1: slot t % S may be
    // loaded again, slot (t + 1) % S be read.
    // 4-bit weights through LDS: codes, table entries and the first blocks' expansion of stage t + 2 in the second half of stage t, the second
    // blocks' in the first half of stage t + 1; half (t + 2) % 2 of the expanded weights is free behind the barrier of stage t.
    // In registers: codes and first entry of stage t + 1 in the first half of stage t, its first expansion and second entry in the second half,
    // its second expansion in its own first half.
    // The order inside a half is fixed: behind each product two reads (done well before the half ends), the loads far apart (a load that
    // cannot go out holds up the products behind it).
    using std::integral_constant;
    constexpr integral_constant<int, 0> k0{};
    constexpr integral_constant<int, 1> k1{};
    // loads that may be in flight at the barrier of stage t: those behind the labels of stage t + 1, 4-bit: behind the weights of stage t + 2
    static_assert(S == 4 || (kF8 && S == 3), "the loop's slots; parities of stages follow from slots; the waits of the first stages");
    constexpr int kInFlight = kPart ? (S - 3) * kParts + GP : (S - 2) * kParts;
    // the first stages: all weights, then labels (these wait for the rows' numbers), but for the labels of stage S - 1
    auto fill_weights = [&](auto self, auto u) __attribute__((always_inline)) -> void {
        if constexpr (decltype(u)::value < S) {
#pragma unroll
            for (int i = 0; i < kWLoads; i++) load_weights(u, i);
            self(self, integral_constant<int, decltype(u)::value + 1>{});
        }
    };
    auto fill_labels = [&](auto self, auto u) __attribute__((always_inline)) -> void {
        if constexpr (decltype(u)::value < S - 1) {
#pragma unroll
            for (int i = 0; i < GP; i++) load_labels(u, i);
            self(self, integral_constant<int, decltype(u)::value + 1>{});
        }
    };
    Tile tile;
    Groups g;
    bool more = true;
    // Products and results of the tile whose first loads are out; before the results, the first loads of the block's next tile.  dn: the wave's
    // tiles of 32 digits that hold groups
    auto work = [&](auto dn) __attribute__((always_inline)) {
        constexpr int kProducts = dn * FB, kReads = FB + 2 * dn, kSlots = kProducts > 4 ? kProducts : 4;
        Tile next = tile;
        Begun begun = {0, 0};
        make_table(tile.pi); open_table(tile); make_f8(0);
        // (behind the barrier at the end of the last tile's products, before the one in front of this one's)
        more = TL::PERSIST && next_tile(next);
        if (more) begun = begin(next);
        wait_loads<(S - 2) * GP>();         // all weights and the labels of stage 0
        lds_barrier();
        if constexpr (kPart && !kDirect) {
            fetch_codes(k0, 0);
            fetch_table(0); fetch_table(1);
#pragma unroll
            for (int i = 0; i < kSteps; i++) expand(0, i);
            if constexpr (kF8) expand8(0, f8_base);
            lds_barrier();
        }
        int zero = 0;
        asm volatile("" : "+s"(zero));          // (known zeros make the compiler keep a second set of sums)
        v16i acc[dn][FB];
#pragma unroll
        for (int d = 0; d < dn; d++) {
            const int g0 = (wd * DA + d) * 2;
            const int s0 = kMx4 || ws ? zero : (int)lane_of(g.start, g0), s1 = kMx4 || ws ? zero : (int)lane_of(g.start, g0 + 1);
#pragma unroll
            for (int f = 0; f < FB; f++)
#pragma unroll
                for (int r = 0; r < 16; r++) acc[d][f][r] = r < 8 ? s0 : s1;
        }
        auto multiply = [&](const auto& o, int i) __attribute__((always_inline)) {
            const int d = i / FB, f = i % FB;
            const v4i a = {o.a[d][0][0], o.a[d][0][1], o.a[d][1][0], o.a[d][1][1]};
            acc[d][f] = __builtin_amdgcn_mfma_i32_32x32x32_i8(a, o.b[f], acc[d][f], 0, 0, 0);
        };
        Operands o0, o1;
        int t = 0;
        uint32_t look[kF8 && kDirect ? 4 * FB : 4][4];
        auto half = [&](const Operands& now, Operands& next, bool there, auto u, auto second) __attribute__((always_inline)) {
            constexpr int U = decltype(u)::value, kHalf = decltype(second)::value, kLoads = kHalf ? kWLoads : GP;
            constexpr integral_constant<int, (U + 1) % kUnroll> u1{};
            constexpr integral_constant<int, (U + 2) % kUnroll> u2{};
            constexpr integral_constant<int, (U + S - 1) % S> before{};
#pragma unroll
            for (int m = 0; m < kSlots; m++) {
                if (m < kProducts && there) multiply(now, m);
#pragma unroll
                for (int i = 0; i < kReads; i++)
                    if (i / 2 == m || (m == kSlots - 1 && i / 2 > m)) { if constexpr (kHalf) read(next, u1, 0, i); else read(next, u, 1, i); }
                if constexpr (kF8 && !kDirect) {
                    // The lane's 16 codes of stage t + 2 come in the second half of stage t, half of them are looked up in it, half in the first half of stage t + 1, at the end of
                    // which their bytes go out; the tables of the 128 inputs that stage t + 2 (even) begins are made in the first half of stage t.
                    if (m == 0 && !kHalf && !(U & 1)) make_f8((t >> 1) + 1);
                    if (kHalf && m == 0) fetch_codes(u2, 0);
                    const uint32_t base = f8_base + ((uint32_t)(t + kHalf + 1) >> 1 & 1) * 256;         // of stage t + 2, in the first half of stage t + 1
#pragma unroll
                    for (int i = 0; i < 2; i++) {
                        const int dword = 2 * !kHalf + i;
                        if (m == (kHalf ? kSlots * 3 / 8 : 0) + i * kSlots / 8) look4(look[i], code[0][0][dword], base);
                        if (m == (kHalf ? kSlots - 1 : kSlots * 5 / 8)) {
                            bytes[0][dword] = join4(look[i]);
                            if (kHalf) asm volatile("" : "+v"(bytes[0][dword]));          // (here, not in the next stage, where it would be waited for at once)
                        }
                    }
                    if (!kHalf && m == kSlots - 2) *(u32x4*)(exp8_to + ((U + 1) & 1) * kExp) = bytes[0];
                } else if constexpr (kF8) {
                    // Codes of the next stage's half of the same number, and the bytes of the half whose codes are there.  The tables of the 128 inputs that
                    // the next stage begins are made in the first half, in front of the barrier.
                    static_assert(FB == WT, "a wave expands what it multiplies");
                    if (m == 0) fetch_codes(u1, kHalf);
                    if (m == 0 && !kHalf && (WK > 1 || (U & 1))) make_f8((WK * (t + 1)) >> 1);
                    const uint32_t kb = (uint32_t)(WK * (t + kHalf) + ws) >> 1;            // of the half that is expanded
                    // (in the first slots, the results taken some slots later)
#pragma unroll
                    for (int i = 0; i < 4 * FB; i++) {
                        const int s = i * kSlots / (8 * FB);
                        if (s == m) look4(look[i], code[!kHalf][i / 4][i % 4], f8_base + (kb & 1) * 256);
                        if (s + kSlots / 2 == m) {
                            next.b[i / 4][i % 4] = (int)join4(look[i]);
                            if (kHalf) asm volatile("" : "+v"(next.b[i / 4][i % 4]));
                        }
                    }
                } else if constexpr (kDirect) {
                    static_assert(FB == WT, "a wave expands what it multiplies");
                    if (m == 0 && !kHalf) fetch_codes(u1, (U + 1) & 1);
#pragma unroll
                    for (int i = 0; i < 4 * FB; i++)
                        if (i * kSlots / (4 * FB) == m) next.b[i / 4][i % 4] = (int)four(code[(U + kHalf) & 1][i / 4][i % 4], lut[!kHalf][i / 4], !kHalf);
                    if (m == kSlots / 2) fetch_table(kHalf);
                } else if constexpr (kMx4) {
                    if constexpr (kHalf) {
                        if (m == 0) fetch_codes(u2, 0);
                        if (m == kSlots / 4) { fetch_table(0); fetch_table(1); }
#pragma unroll
                        for (int i = 0; i < kSteps / 2; i++) if (kSlots / 2 + i * kSlots / kSteps == m) expand(U & 1, i);
                    } else {
#pragma unroll
                        for (int i = 0; i < kSteps / 2; i++) if (i * 2 * kSlots / kSteps == m) expand((U + 1) & 1, kSteps / 2 + i);
                    }
                }
#pragma unroll
                for (int i = 0; i < kLoads; i++)
                    if ((2 * i + 1) * kSlots / (2 * kLoads) == m) { if constexpr (kHalf) load_weights(u, i); else load_labels(before, i); }
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        // one stage in slot u; false: it was the last
        auto stage = [&](auto u) __attribute__((always_inline)) -> bool {
            const bool there = WK == 1 || WK * t + ws < nk;         // (the last round may be short of a stage for some sets)
            half(o0, o1, there, u, k0);
            // (of the first stages the weights went out first: fewer loads stand behind the labels of stage t + 1)
            constexpr int U = decltype(u)::value;
            constexpr int kEarly = kPart ? S - 3 : S - 2;
            if (U < kEarly && t == U) wait_loads<(S - 2) * GP + (U < kEarly ? U : 0) * kWLoads>();
            else wait_loads<kInFlight>();
            lds_barrier();
            half(o1, o0, there, u, k1);
            t++;
            if constexpr (kF8) {
                // stage t makes the table of scale number 64, 96, 128 ...: that one and 31 behind it in place of the 32 oldest (the one before it is still in use)
                constexpr int kPer = 64 / WK, kAt = kPer - (kDirect ? 1 : 2);
                if (__builtin_expect((t & (kPer - 1)) == kAt && t > kPer, 0)) { load_scales(32 * (t / kPer)); take_scales(); }
            }
            return t < (nk + WK - 1) / WK;
        };
#pragma unroll
        for (int i = 0; i < kReads; i++) read(o0, k0, 0, i);
        if constexpr (kF8 && !kDirect) {
            fetch_codes(k1, 0);
#pragma unroll
            for (int i = 0; i < 2; i++) {
                look4(look[i], code[0][0][i], f8_base);
                bytes[0][i] = join4(look[i]);
            }
        } else if constexpr (kF8) {
            fetch_codes(k0, 0);
            fetch_codes(k0, 1);
#pragma unroll
            for (int i = 0; i < 4 * FB; i++) {
                uint32_t look[4];
                look4(look, code[0][i / 4][i % 4], f8_base + (ws >> 1) * 256);
                o0.b[i / 4][i % 4] = (int)join4(look);
            }
        } else if constexpr (kDirect) {
            fetch_codes(k0, 0);
            fetch_table(0); fetch_table(1);
#pragma unroll
            for (int i = 0; i < 4 * FB; i++) o0.b[i / 4][i % 4] = (int)four(code[0][i / 4][i % 4], lut[0][i / 4], 0);
        } else if constexpr (kMx4) {
            fetch_codes(k1, 0);
            fetch_table(0); fetch_table(1);
#pragma unroll
            for (int i = 0; i < kSteps / 2; i++) expand(1, i);
        }
        constexpr integral_constant<int, 2> k2{};
        constexpr integral_constant<int, 3> k3{};
        if constexpr (kUnroll == 6) while (stage(k0) && stage(k1) && stage(k2) && stage(k3) && stage(integral_constant<int, 4>{}) && stage(integral_constant<int, 5>{})) {}
        else while (stage(k0) && stage(k1) && stage(k2) && stage(k3)) {}
        wait_loads<0>();
        if constexpr (WK > 1) {
            // the sums of the other sets come through LDS
            lds_barrier();
            u32x4* const part = (u32x4*)smem + wave * DA * FB * 256 + lane;
#pragma unroll
            for (int s = 1; s < WK; s++) {
                if (ws == s) {
#pragma unroll
                    for (int i = 0; i < dn * FB * 4; i++) {
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
                for (int i = 0; i < dn * FB * 4; i++) {
                    const u32x4 v = part[((s - 1) * NW * DA * FB * 4 + i) * 64];
#pragma unroll
                    for (int r = 0; r < 4; r++) acc[i / 4 / FB][i / 4 % FB][i % 4 * 4 + r] += (int)v[r];
                }
        }
        const Tile done = tile;
        const Groups gd = g;
        if (more) {
            lds_barrier();          // (the slots and the table are free)
            tile = next;
            open_weights(tile);
            fill_weights(fill_weights, k0);
            g = groups_of(begun);
            open_labels(tile, g);
            fill_labels(fill_labels, k0);
        }

        // ---- reduction mod p, 16 bytes a lane ----
        // (plain: no bias, every sum takes one multiplication; the common case, without branches)
        auto finish = [&](auto plain) __attribute__((always_inline)) {
#pragma unroll
            for (int d = 0; d < dn; d++) {
                const int g0 = (wd * DA + d) * 2;
                if (g0 >= done.n_groups) break;
                const uint64_t dst0 = lane_of(gd.dst, g0), dst1 = lane_of(gd.dst, g0 + 1);
                const global_ptr dst = (global_ptr)(h ? dst1 : dst0);
                const bool valid = g0 + h < done.n_groups;
#pragma unroll
                for (int f = 0; f < FB; f++) {
                    const int j = done.by * TL::F + (wf * FB + f) * 32 + j32;
                    uint32_t w[4];          // digits 4 h .. and 8 + 4 h .. of the first group, of the second
#pragma unroll
                    for (int g = 0; g < 2; g++) {
                        const uint32_t prime = lane_of(gd.prime, g0 + g), mmagic = lane_of(gd.magic, g0 + g);
                        auto red1 = [&](uint32_t v) __attribute__((always_inline)) { return v - __umul24(mulhi(v, mmagic), prime); };
                        uint32_t v[8];
#pragma unroll
                        for (int r = 0; r < 8; r++) v[r] = (uint32_t)acc[d][f][8 * g + r];
                        if constexpr (!plain) {
                            const uint32_t pow12 = lane_of(gd.pow12, g0 + g);
#pragma unroll
                            for (int r = 0; r < 8; r++) v[r] = __umul24(red1(v[r] >> 12), pow12) + (v[r] & 4095u);
                            if (A.bias) {
                                const int32_t b = j < M ? A.bias[(int64_t)done.e * M + j] % (int32_t)prime : 0;
                                const uint32_t bm = (uint32_t)(b < 0 ? b + (int32_t)prime : b);
                                const global_u32 one = (global_u32)lane_of(gd.one, g0 + g);
#pragma unroll
                                for (int r = 0; r < 8; r++) v[r] = red1(v[r]) + __umul24(bm, (one[2 * (r / 4) + h] >> (8 * (r % 4))) & 0xffu);
                            }
                        }
#pragma unroll
                        for (int q = 0; q < 2; q++) w[2 * g + q] = red1(v[4 * q]) | red1(v[4 * q + 1]) << 8 | red1(v[4 * q + 2]) << 16 | red1(v[4 * q + 3]) << 24;
                    }
                    // lanes 0-31 hold dwords 0, 2 of both groups, lanes 32-63 dwords 1, 3: after the swaps the first half holds the first group
                    const auto lo = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false), hi = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
                    if (valid && j < M) *(global_u32x4)(dst + (int64_t)j * 16) = u32x4{lo[0], lo[1], hi[0], hi[1]};
                    __builtin_amdgcn_sched_barrier(0);      // (else all accumulators are read at once)
                }
            }
        };
        if (A.plain) finish(k1); else finish(k0);
    };
    __syncthreads();
    if (!next_tile(tile)) return;
    const Begun begun0 = begin(tile);
    open_scales(tile);
    open_weights(tile);
    fill_weights(fill_weights, k0);
    g = groups_of(begun0);
    open_labels(tile, g);
    fill_labels(fill_labels, k0);
    do {
        // waves whose digits lie past the tile's groups, in part or whole, leave out those products (large tiles are rarely short)
        const int mine = ((tile.n_groups + 1) >> 1) - wd * DA;
        if (DA > 4 && mine > 2 && mine <= 4) work(integral_constant<int, 4>{});
        else if (TL::PERSIST || mine > 2 || (DA == 2 && mine == 2)) work(integral_constant<int, DA>{});
        else if (DA > 2 && mine == 2) work(integral_constant<int, 2>{});
        else work(k1);
    } while (more);
}

// what the launches of every tile share; work and bytes for the profile
struct ExpWork { ExpArgs A; double macs, bytes; PrimeClasses classes; };
inline int experts_args(const dash_ctx* c, const ExpertsCall& L, const dash_labels* in, dash_labels* out, ExpWork& work, bool by_class = false) {
    ExpArgs& A = work.A;
    memset(&A, 0, sizeof(A));
    A.w = L.w; A.expert_bytes = matrix_bytes(L.format, L.M, L.K); A.bias = L.bias;
    A.M = L.M; A.K = L.K; A.E = L.E; A.n = (int)L.n; A.top_k = L.top_k;
    double &macs = work.macs, &bytes = work.bytes;
    macs = 0; bytes = (double)L.E * A.expert_bytes;
    A.k = c->k;
    A.plain = L.bias == nullptr;
    for (int i = 0; i <= DASH_MAX_PRIMES; i++) A.chunk_first[i] = 0x7fffffff;
    A.chunk_first[0] = 0;
    work.classes = {};
    if (by_class) {
        const PrimeClasses& C = work.classes = prime_classes(c);
        for (int i = 0; i <= C.n; i++) A.part_first[i] = C.chunk_first[i];
        for (int i = 0; i < C.n; i++) {
            const uint32_t m = (uint32_t)C.modulus[i];
            A.part[i] = {m, (uint32_t)(((1ull << 32) + m - 1) / m)};
        }
    }
    for (int at = 0; at < c->k; at++) {
        const int i = by_class ? work.classes.order[at] : at;
        ExpPrime& P = A.pr[at];
        const ModInfo& Mi = c->mods[c->prime[i]];
        A.chunk_first[at + 1] = A.chunk_first[at] + (int)Mi.nchunk;
        P.chunk_first = A.chunk_first[at];
        P.p = c->prime[i]; P.mmagic = Mi.mmagic; P.pow12 = 4096u % P.p;
        if (!by_class) {
            A.part_first[at + 1] = A.chunk_first[at + 1];
            A.part[at] = {P.p, P.mmagic};
        }
        P.one = L.bias ? (L.garble ? c->d_one0[i] : c->d_one[i]) : nullptr;
        P.in = view_of(in, i); P.out = view_of(out, i);
        const uint64_t p1 = P.p - 1;
        uint64_t vmax = p1 * p1 * (uint64_t)L.K;
        if (L.format != DASH_MX4) {
            P.start = (uint32_t)((128 * p1 * (uint64_t)L.K + P.p - 1) / P.p * P.p);
            vmax = P.start + 127 * p1 * (uint64_t)L.K;
        }
        // v / p = mulhi(v, mmagic) as long as v times the rounding of mmagic stays below 2^32; the quotient goes into a 24-bit product
        const uint64_t over = (uint64_t)P.mmagic * P.p - (1ull << 32);
        if (vmax * over >= (1ull << 32) || vmax / P.p >= (1u << 24)) A.plain = 0;
        macs += (double)L.n * L.M * L.K * Mi.lam;
        bytes += ((double)(L.n / L.top_k) * L.K + (double)L.n * L.M) * Mi.lam;
    }
    return (int64_t)A.chunk_first[c->k] * L.n > 0x7fffffff - 64 ? DASH_ESIZE : DASH_OK;
}
template <int FMT, class TL> int launch_experts(dash_ctx* c, const ExpertsCall& L, ExpWork& work, hipStream_t s) {
    ExpArgs& A = work.A;
    constexpr TileParts parts = kTileKind[TL::KIND].parts;
    static_assert((FMT == DASH_W8) == (parts == PARTS_NONE) && (FMT != DASH_MX4 || parts == PARTS_PRIMES), "tiles of the format");
    int64_t cols = 0;
    if (L.routing) {
        constexpr int s = TL::KIND;
        cols = L.routing->max_tiles[s];
        A.rows = L.routing->rows; A.tiles = L.routing->tiles[s]; A.n_tiles = L.routing->first_tile[s] + L.E + 1;
    } else if (parts != PARTS_NONE) {
        const int* const chunks = parts == PARTS_CLASSES ? A.part_first : A.chunk_first;
        for (int i = 0; i < (parts == PARTS_CLASSES ? work.classes.n : c->k); i++) {
            A.first[i] = (int)cols;
            cols += ((int64_t)(chunks[i + 1] - chunks[i]) * L.n + TL::G - 1) / TL::G;
            A.first[i + 1] = (int)cols;
        }
    }
    else cols = ((int64_t)A.chunk_first[c->k] * L.n + TL::G - 1) / TL::G;
    A.cols = (int)cols;
    A.row_blocks = (L.M + TL::F - 1) / TL::F;
    A.sty = 4;
    const int64_t total = cols * A.row_blocks;
    if (cols * A.sty > 0x7fffffff || total > 0x7fffff00) return DASH_ESIZE;
    ProfScope ps(c->prof, DASH_PROF_LINEAR, s, work.macs, work.bytes);
    const BlockGrid grid = block_grid(TL::PERSIST && total > kCus ? kCus : total, TL::T);
    hipLaunchKernelGGL((k_experts_mfma<FMT, TL>), dim3(grid.x, grid.y), dim3(TL::T), 0, s, A);
    DASH_HIP(hipGetLastError());
    return DASH_OK;
}
inline ExpertsShape experts_shape(const dash_ctx* c, const ExpertsCall& L) {
    ExpertsShape shape{L.n, L.E, L.M, L.K, L.format != DASH_W8, c->k, {}};
    for (int i = 0; i < c->k; i++) shape.chunks[i] = (int)c->mods[c->prime[i]].nchunk;
    return shape;
}

}  // namespace dash
