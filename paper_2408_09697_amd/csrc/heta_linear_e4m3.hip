// heta_linear on 8-bit operands: widened to bf16 behind LDS, or (coarse sums) on the 8-bit matrix instruction.
#include "heta_linear.h"

namespace heta {

// 256 x 256; 256 x 128 for epilogues that read or take any width, which do not fit the registers beside 256 x 256 (with a residual, 200,000 x 1,024 x 4,096: 1,760 us,
// 1,730 with spilled registers; 100,000 x 1,024 x 1,024 191 / 226; 300,000 x 256 x 512 210 / 226)
template <bool WIDEN> using Large = TileShape<uint8_t, 1, 1, false, false, kDirect, 2, 4, 4, 2, 128, 2, 1, WIDEN>;
template <bool WIDEN> using Half = TileShape<uint8_t, 1, 1, false, false, kDirect, 4, 2, 2, 2, 128, 2, 1, WIDEN>;
template <bool WIDEN> using Small = TileShape<uint8_t, 1, 1, false, false, kDirect, 2, 2, 1, 1, 128, 3, 2, WIDEN>;       // 64 x 64
template <bool WIDEN> using StagedLarge = TileShape<uint8_t, 1, 1, false, false, kStaged, 4, 2, 2, 2, 128, 2, 1, WIDEN>; // 256 x 128
template <bool WIDEN> using StagedSmall = TileShape<uint8_t, 1, 1, false, false, kStaged, 2, 2, 1, 1, 128, 2, 2, WIDEN>; // 64 x 64

heta_status launch_linear_e4m3(const Launch &l, heta_dtype out_dt, bool coarse, const LinearExtra &x)
{
    auto with = [&](auto tag, auto widen) {
        using O = decltype(tag);
        constexpr bool W = decltype(widen)::value;
        return launch_linear<Large<W>, Half<W>, Half<W>, Small<W>, StagedLarge<W>, StagedSmall<W>, O, false>(l, 1, x);
    };
    if (out_dt == HETA_F32) return coarse ? with(float{}, std::false_type{}) : with(float{}, std::true_type{});
    return coarse ? with(bf16_t{}, std::false_type{}) : with(bf16_t{}, std::true_type{});
}

} // namespace heta
