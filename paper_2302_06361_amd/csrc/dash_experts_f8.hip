// dash_experts_f8.hip -- tiles of the products of expert layers with 8-bit floating point weights (dash_experts_kernel.h has the kernel).
#ifndef DASH_F8_COMPUTED
#define DASH_F8_COMPUTED 2
#endif
#include "dash_experts_kernel.h"

namespace dash {

// A stage's codes take as much LDS as byte weights: three stages.
typedef ETile<1, 4, 2, 4, 2, 3, 6, false> EBig8;         // 512 digits x 128 features, weights expanded once a block, through LDS
typedef ETile<1, 4, 2, 4, 2, 3, 7, false> EBigClass8;    // the same, tiles across a class of primes
typedef ETile<1, 1, 4, 4, 1, 3, 3, false> ENarrow8;      // 128 x 128
typedef ETile<1, 1, 4, 4, 1, 3, 5, false> ENarrowClass8;
typedef ETile<2, 1, 4, 4, 1, 3, 5, false> EFew8;         // 128 x 128 by two sets of waves

int experts_mfma_f8(dash_ctx* c, const ExpertsCall& L, const dash_labels* in, dash_labels* out, hipStream_t s) {
    ExpWork W;
    auto launch = [&](auto tl) -> int {
        typedef decltype(tl) TL;
        const int st = experts_args(c, L, in, out, W, kTileKind[TL::KIND].parts == PARTS_CLASSES);
        return st ? st : launch_experts<DASH_F8, TL>(c, L, W, s);
    };
    const ExpertsTile tile = experts_tile(c->experts_tile, experts_shape(c, L));
    bool small = true;          // primes to 37
    for (int i = 0; i < c->k; i++) small &= c->prime[i] <= 37;
    if (tile == EXPERTS_FEW) return launch(EFew8{});
    if (tile == EXPERTS_NARROW) return small ? launch(ENarrow8{}) : launch(ENarrowClass8{});
    return tile == EXPERTS_BIG ? launch(EBig8{}) : launch(EBigClass8{});
}

}  // namespace dash
