// heta_linear and heta_linear_bwd on bf16 operands.
#include "heta_linear.h"

namespace heta {

template <bool A_RC, bool B_RC> using Large = TileShape<bf16_t, 2, 1, A_RC, B_RC, kDirect, 2, 4, 4, 2, 64, 2, 1>;       // 256 x 256
template <bool A_RC, bool B_RC> using Small = TileShape<bf16_t, 2, 1, A_RC, B_RC, kDirect, 2, 2, 1, 1, 64, 3, 2>;       // 64 x 64
template <bool A_RC, bool B_RC> using Elements = TileShape<bf16_t, 2, 1, A_RC, B_RC, kElements, 2, 2, 2, 2, 32, 2, 1>;  // 128 x 128

heta_status launch_linear_bf16(const Launch &l, bool input_gradient, heta_dtype out_dt, const LinearExtra &x)
{
    if (input_gradient) return launch_linear<Large<false, false>, Large<false, false>, Small<false, false>, Elements<false, false>, bf16_t, true>(l, 2, x);
    if (out_dt == HETA_F32) return launch_linear<Large<false, true>, Large<false, true>, Small<false, true>, Elements<false, true>, float, false>(l, 2, x);
    return launch_linear<Large<false, true>, Large<false, true>, Small<false, true>, Elements<false, true>, bf16_t, false>(l, 2, x);
}
heta_status launch_grad_w_bf16(const Launch &l, float *part) { return launch_grad_w<Large<true, true>, Small<true, true>, Elements<true, true>>(l, 2, part); }

} // namespace heta
