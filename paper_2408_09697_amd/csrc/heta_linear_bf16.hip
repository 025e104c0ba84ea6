// heta_linear and heta_linear_bwd on bf16 operands.
#include "heta_linear.h"

namespace heta {

template <bool A_RC, bool B_RC> using Large = TileShape<bf16_t, 2, 1, A_RC, B_RC, kDirect, 2, 4, 4, 2, 64, 2, 1>;       // 256 x 256
template <bool A_RC, bool B_RC> using Small = TileShape<bf16_t, 2, 1, A_RC, B_RC, kDirect, 2, 2, 1, 1, 64, 3, 2>;       // 64 x 64
template <bool A_RC, bool B_RC> using StagedLarge = TileShape<bf16_t, 2, 1, A_RC, B_RC, kStaged, 4, 2, 2, 2, 64, 2, 1>; // 256 x 128
template <bool A_RC, bool B_RC> using StagedSmall = TileShape<bf16_t, 2, 1, A_RC, B_RC, kStaged, 2, 2, 1, 1, 64, 2, 2>; // 64 x 64

template <bool B_RC, typename O, bool SLOPES> static heta_status launch(const Launch &l, const LinearExtra &x)
{
    return launch_linear<Large<false, B_RC>, Large<false, B_RC>, Small<false, B_RC>, StagedLarge<false, B_RC>, StagedSmall<false, B_RC>, O, SLOPES>(l, 2, x);
}
heta_status launch_linear_bf16(const Launch &l, bool input_gradient, heta_dtype out_dt, const LinearExtra &x)
{
    if (input_gradient) return launch<false, bf16_t, true>(l, x);
    return out_dt == HETA_F32 ? launch<true, float, false>(l, x) : launch<true, bf16_t, false>(l, x);
}
heta_status launch_grad_w_bf16(const Launch &l, float *part) { return launch_grad_w<Large<true, true>, Small<true, true>, StagedLarge<true, true>, StagedSmall<true, true>>(l, 2, part); }

} // namespace heta
