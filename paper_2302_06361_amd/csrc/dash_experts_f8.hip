// dash_experts_f8.hip -- tiles of the products of expert layers with 8-bit floating point weights (dash_experts_kernel.h has the kernel).
#include "dash_experts_kernel.h"

namespace dash {

// 8-bit floats: a stage's codes take as much LDS as byte weights, three stages leave room for two blocks per CU
typedef ETile<1, 1, 4, 4, 1, 3, 3, false> ENarrow8;
typedef ETile<1, 1, 4, 4, 2, 3, 3, false> EWide8;
typedef ETile<2, 1, 4, 2, 1, 3, 4, false> EFew8;

int experts_mfma_f8(dash_ctx* c, const ExpertsCall& L, const dash_labels* in, dash_labels* out, hipStream_t s) {
    ExpWork W;
    const int st = experts_args(c, L, in, out, W);
    if (st) return st;
    const ExpertsTile tile = experts_tile(c->experts_tile, experts_shape(c, L, W.A));
    return tile == EXPERTS_FEW ? launch_experts<DASH_F8, EFew8>(c, L, W, s) : tile == EXPERTS_NARROW ? launch_experts<DASH_F8, ENarrow8>(c, L, W, s)
         : launch_experts<DASH_F8, EWide8>(c, L, W, s);
}

}  // namespace dash
