// dash_experts_f8.hip -- tiles of the products of expert layers with 8-bit floating point weights (dash_experts_kernel.h has the kernel).
#include "dash_experts_kernel.h"

namespace dash {

// A stage's codes take as much LDS as byte weights: three stages.
typedef ETile<1, 4, 2, 4, 2, 3, 6, false> EBig8;         // 512 digits x 128 features, weights expanded once a block, through LDS
typedef ETile<1, 1, 4, 4, 1, 3, 5, false> ENarrow8;      // 128 x 128
typedef ETile<1, 1, 4, 4, 2, 3, 5, false> EWide8;        // 128 x 256
typedef ETile<2, 1, 4, 4, 1, 3, 5, false> EFew8;         // 128 x 128 by two sets of waves

int experts_mfma_f8(dash_ctx* c, const ExpertsCall& L, const dash_labels* in, dash_labels* out, hipStream_t s) {
    ExpWork W;
    const int st = experts_args(c, L, in, out, W);
    if (st) return st;
    const ExpertsTile tile = experts_tile(c->experts_tile, experts_shape(c, L, W.A));
    return tile == EXPERTS_FEW ? launch_experts<DASH_F8, EFew8>(c, L, W, s) : tile == EXPERTS_NARROW ? launch_experts<DASH_F8, ENarrow8>(c, L, W, s)
         : tile == EXPERTS_BIG ? launch_experts<DASH_F8, EBig8>(c, L, W, s) : launch_experts<DASH_F8, EWide8>(c, L, W, s);
}

}  // namespace dash
