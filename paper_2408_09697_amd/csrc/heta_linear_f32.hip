// heta_linear and heta_linear_bwd on fp32 operands: split into three bf16 terms on their way into LDS.
#include "heta_linear.h"

namespace heta {

template <bool A_RC, bool B_RC> using Large = TileShape<float, 2, 3, A_RC, B_RC, kStaged, 4, 2, 2, 2, 32, 2, 1>;      // 256 x 128
template <bool A_RC, bool B_RC> using Small = TileShape<float, 2, 3, A_RC, B_RC, kStaged, 2, 2, 1, 1, 32, 2, 2>;      // 64 x 64
template <bool A_RC, bool B_RC> using Elements = TileShape<float, 2, 3, A_RC, B_RC, kElements, 2, 2, 1, 1, 32, 2, 2>; // 64 x 64

heta_status launch_linear_f32(const Launch &l, bool input_gradient, const LinearExtra &x)
{
    if (input_gradient) return launch_linear<Large<false, false>, Large<false, false>, Small<false, false>, Elements<false, false>, float, true>(l, 4, x);
    return launch_linear<Large<false, true>, Large<false, true>, Small<false, true>, Elements<false, true>, float, false>(l, 4, x);
}
heta_status launch_grad_w_f32(const Launch &l, float *part) { return launch_grad_w<Large<true, true>, Small<true, true>, Elements<true, true>>(l, 4, part); }

} // namespace heta
