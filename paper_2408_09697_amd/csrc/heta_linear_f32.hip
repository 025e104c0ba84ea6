// heta_linear and heta_linear_bwd on fp32 operands: split into three bf16 terms on their way through registers into LDS.
#include "heta_linear.h"

namespace heta {

template <bool A_RC, bool B_RC> using Large = TileShape<float, 2, 3, A_RC, B_RC, kStaged, 4, 2, 2, 2, 32, 2, 1>; // 256 x 128
template <bool A_RC, bool B_RC> using Small = TileShape<float, 2, 3, A_RC, B_RC, kStaged, 2, 2, 1, 1, 32, 2, 2>; // 64 x 64

template <bool B_RC, bool SLOPES> static heta_status launch(const Launch &l, const LinearExtra &x)
{
    return launch_linear<Large<false, B_RC>, Large<false, B_RC>, Large<false, B_RC>, Small<false, B_RC>, Large<false, B_RC>, Small<false, B_RC>, float, SLOPES>(l, 4, x);
}
heta_status launch_linear_f32(const Launch &l, bool input_gradient, const LinearExtra &x) { return input_gradient ? launch<false, true>(l, x) : launch<true, false>(l, x); }
heta_status launch_grad_w_f32(const Launch &l, float *part) { return launch_grad_w<Large<true, true>, Small<true, true>, Large<true, true>, Small<true, true>>(l, 4, part); }

} // namespace heta
