// dash_experts_gemm.hip -- tiles of the products of expert layers with byte and 4-bit weights (dash_experts_kernel.h has the kernel).
#include "dash_experts_kernel.h"

namespace dash {

typedef ETile<1, 2, 4, 4, 2, 4, 0, true> EBig;       // 256 digits x 256 features
typedef ETile<1, 2, 4, 4, 2, 4, 2, false> EBig4;     // the same for 4-bit weights (tile after tile: 2 % at 16 stages, but 8 % lost at two)
typedef ETile<1, 2, 2, 2, 2, 4, 1, false> ENarrow;   // 128 digits x 128 features
typedef ETile<1, 1, 4, 4, 1, 4, 3, false> ENarrow4;  // the same for 4-bit weights
typedef ETile<1, 1, 4, 4, 2, 4, 3, false> EWide4;    // 128 digits x 256 features, weights expanded in registers, two blocks per CU (256 rows, 32 experts, 1024 -> 2048: 414 -> 355 us; 128 rows, 4096 -> 4096: 1029 -> 1076)
typedef ETile<2, 1, 4, 2, 1, 4, 4, false> EFew4;     // 64 digits x 128 features by two sets of waves, 4-bit weights

int experts_mfma(dash_ctx* c, const ExpertsCall& L, const dash_labels* in, dash_labels* out, hipStream_t s) {
    if (L.format == DASH_F8) return experts_mfma_f8(c, L, in, out, s);
    ExpWork W;
    const int st = experts_args(c, L, in, out, W);
    if (st) return st;
    const ExpertsTile tile = experts_tile(c->experts_tile, experts_shape(c, L));
    if (L.format == DASH_W8) return tile == EXPERTS_BIG ? launch_experts<DASH_W8, EBig>(c, L, W, s) : launch_experts<DASH_W8, ENarrow>(c, L, W, s);
    return tile == EXPERTS_BIG ? launch_experts<DASH_MX4, EBig4>(c, L, W, s) : tile == EXPERTS_FEW ? launch_experts<DASH_MX4, EFew4>(c, L, W, s)
         : tile == EXPERTS_WIDE ? launch_experts<DASH_MX4, EWide4>(c, L, W, s) : launch_experts<DASH_MX4, ENarrow4>(c, L, W, s);
}

}  // namespace dash
