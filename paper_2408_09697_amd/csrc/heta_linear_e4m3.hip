// heta_linear on 8-bit operands: widened to bf16 behind LDS, or (coarse sums) on the 8-bit matrix instruction.
#include "heta_linear.h"

namespace heta {

template <bool WIDEN> using Large = TileShape<uint8_t, 1, 1, false, false, kDirect, 2, 4, 4, 2, 128, 2, 1, WIDEN>;      // 256 x 256
template <bool WIDEN> using Small = TileShape<uint8_t, 1, 1, false, false, kDirect, 2, 2, 1, 1, 128, 3, 2, WIDEN>;      // 64 x 64
template <bool WIDEN> using Elements = TileShape<uint8_t, 1, 1, false, false, kElements, 2, 2, 2, 2, 64, 2, 1, WIDEN>;  // 128 x 128

heta_status launch_linear_e4m3(const Launch &l, heta_dtype out_dt, bool coarse, const LinearExtra &x)
{
    auto with = [&](auto tag) {
        using O = decltype(tag);
        return coarse ? launch_linear<Large<false>, Small<false>, Elements<false>, O, false>(l, 1, x) : launch_linear<Large<true>, Small<true>, Elements<true>, O, false>(l, 1, x);
    };
    return out_dt == HETA_F32 ? with(float{}) : with(bf16_t{});
}

} // namespace heta
