// heta_linear and heta_linear_bwd on bf16 operands.
#include "heta_linear.h"

namespace heta {

template <bool A_RC, bool B_RC> using Large = TileShape<bf16_t, 2, 1, A_RC, B_RC, kDirect, 2, 4, 4, 2, 64, 2, 1>;       // 256 x 256
template <bool A_RC, bool B_RC> using Ragged = TileShape<bf16_t, 2, 1, A_RC, B_RC, kDirect, 4, 2, 2, 2, 64, 2, 1>;      // 256 x 128: for epilogues of any width
template <bool A_RC, bool B_RC> using Small = TileShape<bf16_t, 2, 1, A_RC, B_RC, kDirect, 2, 2, 1, 1, 64, 3, 2>;       // 64 x 64
template <bool A_RC, bool B_RC> using StagedLarge = TileShape<bf16_t, 2, 1, A_RC, B_RC, kStaged, 4, 2, 2, 2, 64, 2, 1>; // 256 x 128
template <bool A_RC, bool B_RC> using StagedSmall = TileShape<bf16_t, 2, 1, A_RC, B_RC, kStaged, 2, 2, 1, 1, 64, 2, 2>; // 64 x 64

template <bool B_RC, typename O, bool SLOPES> static heta_status launch(const Launch &l, const LinearExtra &x)
{
    return launch_linear<Large<false, B_RC>, Large<false, B_RC>, Ragged<false, B_RC>, Small<false, B_RC>, StagedLarge<false, B_RC>, StagedSmall<false, B_RC>, O, SLOPES>(l, 2, x);
}
heta_status launch_linear_bf16(const Launch &l, bool input_gradient, heta_dtype out_dt, const LinearExtra &x)
{
    if (input_gradient) return launch<false, bf16_t, true>(l, x);
    return out_dt == HETA_F32 ? launch<true, float, false>(l, x) : launch<true, bf16_t, false>(l, x);
}
heta_status launch_grad_w_bf16(const Launch &l, float *part) { return launch_grad_w<Large<true, true>, Small<true, true>, StagedLarge<true, true>, StagedSmall<true, true>>(l, 2, part); }

// A workgroup copies 32 rows, a thread eight columns at a time with four loads in flight; the columns that fill the last eight up are zero.
static __global__ void __launch_bounds__(256) align_rows_kernel(const bf16_t *src, int64_t ld, int64_t rows, uint32_t d, uint32_t chunks, bf16_t *dst, unsigned first)
{
    const int64_t r0 = (static_cast<int64_t>(blockIdx.x) + first) * 32;
    const uint32_t total = static_cast<uint32_t>(min(rows - r0, static_cast<int64_t>(32))) * chunks;
    const bf16_t *base = src + r0 * ld;
    bf16_t *to = dst + r0 * chunks * 8;
    for (uint32_t q0 = threadIdx.x; q0 < total; q0 += 1024) {
        union { uintx4 u; bf16_t s[8]; } v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t q = min(q0 + 256 * j, total - 1), row = q / chunks, c = (q - row * chunks) * 8;
            const bf16_t *from = base + row * ld + c;
            if (c + 8 <= d) {
                v[j].u = load16(from);
            } else {
#pragma unroll
                for (uint32_t e = 0; e < 8; ++e) v[j].s[e] = c + e < d ? from[e] : static_cast<bf16_t>(0);
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (q0 + 256 * j < total) store16<false>(to + static_cast<int64_t>(q0 + 256 * j) * 8, v[j].u);
    }
}

// Through registers, 16-byte accesses that start anywhere cost far more than loads straight into LDS, once for every tile that reads
// the operand; a copy costs one pass at 5.3 TB/s and a launch.  It pays for operands of 32 MB and more where both are unaligned or the one
// that is, is read by at least two tiles (staged ones are 256 x 128).  us staged / copied:
//   one unaligned, read by 2 to 4 tiles: 100,000 x 789 x 512 319 / 187, 512 x 789 208 / 178, 789 x 256 173 / 130, 10^6 x 101 x 512 1,129 / 364
//   both: 300,000 x 301 x 301 612 / 285, 10^6 x 101 x 103 497 / 323;  below 32 MB: 9,000 x 257 x 259 25 / 38, 4,000 x 1,030 x 1,030 67 / 74
//   one, read by one tile: 100,000 x 789 x 64 89 / 114, 100,000 x 256 x 789 116 / 129
// At most 1 GiB is copied.
size_t align_grad_w_bytes(const Launch &l)
{
    const TileItem &it = l.it;
    const bool a_in = direct_rows(it.A, it.lda, 2), b_in = direct_rows(it.B, it.ldb, 2);
    const int64_t a_ld = (it.M + 7) / 8 * 8, b_ld = (it.N + 7) / 8 * 8;
    const size_t bytes = static_cast<size_t>(it.K) * ((a_in ? 0 : a_ld) + (b_in ? 0 : b_ld)) * 2;
    if (!l.large() || bytes < (size_t(32) << 20) || bytes > (size_t(1) << 30)) return 0;
    if ((a_in && it.M <= 256) || (b_in && it.N <= 128)) return 0;
    if (a_ld * 2 >= (int64_t(1) << 23) || b_ld * 2 >= (int64_t(1) << 23)) return 0; // the copies could not go straight into LDS either
    return bytes;
}

heta_status align_grad_w_bf16(Launch &l, char *to)
{
    TileItem &it = l.it;
    const bool a_in = direct_rows(it.A, it.lda, 2), b_in = direct_rows(it.B, it.ldb, 2);
    const int64_t a_ld = (it.M + 7) / 8 * 8, b_ld = (it.N + 7) / 8 * 8;
    const int64_t rows = it.K;
    auto copy = [&](const void *&p, int64_t &ld, int64_t cols, int64_t ld_to) {
        ProfScope prof("align_rows_kernel", l.st, 4.0 * rows * cols, 0);
        const uint32_t chunks = static_cast<uint32_t>(ld_to / 8);
        launch_pieces((rows + 31) / 32, 256, [&](unsigned first, unsigned count) {
            hipLaunchKernelGGL(align_rows_kernel, dim3(count), dim3(256), 0, l.st, static_cast<const bf16_t *>(p), ld, rows, static_cast<uint32_t>(cols), chunks,
                               reinterpret_cast<bf16_t *>(to), first);
        });
        p = to;
        ld = ld_to;
        to += static_cast<size_t>(rows) * ld_to * 2;
    };
    if (!a_in) copy(it.A, it.lda, it.M, a_ld);
    if (!b_in) copy(it.B, it.ldb, it.N, b_ld);
    HETA_LAUNCH_CHECK("align_rows_kernel");
    return HETA_OK;
}

} // namespace heta
