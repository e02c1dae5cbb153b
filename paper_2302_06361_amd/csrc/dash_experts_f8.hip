// dash_experts_f8.hip -- tiles of the products of expert layers with 8-bit floating point weights (dash_experts_kernel.h has the kernel).
#include "dash_experts_kernel.h"

namespace dash {

// Three stages: four and six change nothing for a lone block, whose stages wait for LDS, not for memory.  Each tile's home (us, and the best of the other tiles):
typedef ETile<1, 4, 2, 4, 2, 3, 6, false> EBig8;         // 512 digits x 128 features, weights expanded once a block, through LDS (128 rows, 4096 -> 4096, 12 primes: 1 127; 1 215)
typedef ETile<1, 1, 4, 8, 1, 3, 2, false> EWide8;        // 256 x 128, expanded in registers as in the others (256 rows, 32 experts, 1024 -> 2048: 423; 453)
typedef ETile<1, 1, 4, 8, 1, 3, 7, false> EWideClass8;   // the same, tiles across a class of primes (256 rows, 2048 -> 64: 70.3; 72.0)
typedef ETile<1, 1, 4, 4, 1, 3, 5, false> ENarrow8;      // 128 x 128, classes (64 rows, 64 experts, 1024 -> 1024: 93.9; 102.9)
typedef ETile<2, 1, 4, 4, 1, 3, 5, false> EFew8;         // 128 x 128 by two sets of waves, classes (1 row, 4096 -> 4096: 34.8; 37.2)
typedef ETile<2, 1, 2, 4, 1, 3, 5, false> ESmall8;       // 128 x 64 by two sets of waves, classes (12 rows, 6 experts, 3833 -> 172, 9 primes: 27.2; 32.7)

int experts_mfma_f8(dash_ctx* c, const ExpertsCall& L, const dash_labels* in, dash_labels* out, hipStream_t s) {
    auto launch = [&](auto tl) -> int {
        typedef decltype(tl) TL;
        ExpWork W;
        const int st = experts_args(c, L, in, out, W, kTileKind[TL::KIND].parts == PARTS_CLASSES);
        return st ? st : launch_experts<DASH_F8, TL>(c, L, W, s);
    };
    ExpertsShape8 shape{L.n, L.E, L.M, L.K, c->k, {}, 0, {}};
    const PrimeClasses C = prime_classes(c);
    for (int i = 0; i < c->k; i++) shape.chunks[i] = (int)c->mods[c->prime[i]].nchunk;
    shape.classes = C.n;
    for (int i = 0; i < C.n; i++) shape.class_chunks[i] = C.chunk_first[i + 1] - C.chunk_first[i];
    switch (experts_tile8(c->experts_tile, shape)) {
        case EXPERTS_BIG: return launch(EBig8{});
        case EXPERTS_WIDE: return launch(EWide8{});
        case EXPERTS_WIDE_CLASS: return launch(EWideClass8{});
        case EXPERTS_FEW: return launch(EFew8{});
        case EXPERTS_SMALL: return launch(ESmall8{});
        default: return launch(ENarrow8{});
    }
}

}  // namespace dash
