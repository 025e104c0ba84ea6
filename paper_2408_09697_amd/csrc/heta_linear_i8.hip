// heta_linear on rows and weights of 8-bit whole numbers, and how both are made.
//
//     q_ij = round(127 x_ij / max_j |x_ij|), scale_i = max_j |x_ij| / 127      (rows; weights: the columns of W)
//     pre_ij = scale_i w_scale_j sum_k q_ik p_jk + bias_j
//
// The integer matrix instruction adds exactly and takes 32 k-values in the time of 16 in bf16: the products are those of the e4m3 kernels with coarse
// sums in rate, and of those with exact ones in their sums.
#include "heta_linear.h"

namespace heta {

template <int WM, int WN, int MI, int NJ, int LOAD, int ST, int OCC> using Shape = TileShape<uint8_t, 1, 1, false, false, LOAD, WM, WN, MI, NJ, 128, ST, OCC, false, true>;
// 256 x 256 and 256 x 128 by eight wavefronts as for e4m3 (200,000 x 1,024 x 4,096, us: 1,200; two workgroups of four wavefronts a CU, 256 x 128: 1,364, 128 x 128: 1,520; LDS is read
// and written for as long as the matrix pipe works, and smaller tiles read more of it)
using Large = Shape<2, 4, 4, 2, kDirect, 2, 1>;       // 256 x 256
using Ragged = Shape<4, 2, 2, 2, kDirect, 2, 1>;      // 256 x 128: for epilogues of any width
// 128 x 128 by four wavefronts, two workgroups a CU, for epilogues that read: they wait for it while the other multiplies (200,000 x 1,024 x 4,096 with a residual 1,901 -> 1,716 us, 100,000 x
// 4,096 x 1,024 823 -> 748)
using Reading = Shape<2, 2, 2, 2, kDirect, 2, 2>;
using Small = Shape<2, 2, 1, 1, kDirect, 3, 2>;       // 64 x 64
using StagedLarge = Shape<4, 2, 2, 2, kStaged, 2, 1>; // 256 x 128
using StagedSmall = Shape<2, 2, 1, 1, kStaged, 2, 2>; // 64 x 64

// Rows of 8-bit values, `chunks` pieces of 16 bytes each, the last one filled up with zeros.
// Two operands in one launch (no rows of one that needs no copy), at most 2^26 pieces.
struct CodeRows {
    const uint8_t *p;
    uint8_t *to;
    int64_t ld;
    uint32_t rows;
};
static __global__ void __launch_bounds__(256) align_codes_kernel(CodeRows a, CodeRows b, int32_t d, uint32_t chunks)
{
    const uint32_t first = a.rows * chunks, total = first + b.rows * chunks;
    for (uint32_t at = blockIdx.x * 256 + threadIdx.x; at < total; at += gridDim.x * 256) {
        const CodeRows &x = at < first ? a : b;
        const uint32_t q = at < first ? at : at - first, r = q / chunks;
        const int c = static_cast<int>(q - r * chunks) * 16;
        const uint8_t *from = x.p + r * x.ld + c;
        uintx4 v = {0u, 0u, 0u, 0u};
        if (c + 16 <= d) {
            v = load16(from);
        } else {
#pragma unroll
            for (int e = 0; e < 16; ++e)
                if (c + e < d) v[e / 4] |= static_cast<uint32_t>(from[e]) << (8 * (e & 3));
        }
        store16(x.to + static_cast<int64_t>(q) * 16, v);
    }
}

// Large products of rows that start anywhere read copies of them in aligned rows (of at most 1 GiB, and only where there is room): through registers, every
// tile pays for the accesses (100,000 x 789 x 349: 141 us, 90 with the copy).
static heta_status align_operands(Launch &l)
{
    TileItem &it = l.it;
    const bool a_in = direct_rows(it.A, it.lda, 1), b_in = direct_rows(it.B, it.ldb, 1);
    const int64_t ld = (it.K + 15) / 16 * 16;
    const size_t a_bytes = a_in ? 0 : static_cast<size_t>(it.M) * ld, b_bytes = b_in ? 0 : static_cast<size_t>(it.N) * ld, bytes = (a_bytes + 255) / 256 * 256 + b_bytes;
    if ((a_in && b_in) || !l.large() || bytes > (size_t(1) << 30) || ld >= (int64_t(1) << 23)) return HETA_OK;
    if ((l.g->ws_refused > 0 && bytes >= l.g->ws_refused) || ensure_workspace(l.g, bytes) != HETA_OK) return HETA_OK;
    char *to = static_cast<char *>(l.g->d_ws);
    ProfScope prof("align_codes_kernel", l.st, 2.0 * bytes, 0);
    char *const to_b = to + (a_bytes + 255) / 256 * 256;
    const CodeRows a{static_cast<const uint8_t *>(it.A), reinterpret_cast<uint8_t *>(to), it.lda, a_in ? 0u : static_cast<uint32_t>(it.M)},
        b{static_cast<const uint8_t *>(it.B), reinterpret_cast<uint8_t *>(to_b), it.ldb, b_in ? 0u : static_cast<uint32_t>(it.N)};
    const uint32_t chunks = static_cast<uint32_t>(ld / 16);
    hipLaunchKernelGGL(align_codes_kernel, dim3(std::min(((a.rows + b.rows) * chunks + 255) / 256, 16384u)), dim3(256), 0, l.st, a, b, static_cast<int32_t>(it.K), chunks);
    if (!a_in) it.A = to, it.lda = ld;
    if (!b_in) it.B = to_b, it.ldb = ld;
    HETA_LAUNCH_CHECK("align_codes_kernel");
    return HETA_OK;
}

heta_status launch_linear_i8(Launch l, heta_dtype out_dt, const LinearExtra &x)
{
    HETA_TRY(align_operands(l));
    // a quarter of 256 columns a tile or more would be beyond the last (100,000 x 800 x 320 and x 384, 20,000 x 4,096 x 384, 100,000 x 256 x 384, us: 74.3, 74.5, 55.8 and 35.6 by
    // 256 x 256, 64.4, 68.3, 36.5 and 29.3 by 128 x 128; a sixth, x 640: 96.6 and 98.4)
    const int64_t columns = (l.it.N + 255) / 256 * 256;
    const bool narrow = (columns - l.it.N) * 4 >= columns;
    auto go = [&](auto o) {
        using O = decltype(o);
        return narrow ? launch_linear<Reading, Reading, Ragged, Small, StagedLarge, StagedSmall, O, false>(l, 1, x)
                      : launch_linear<Large, Reading, Ragged, Small, StagedLarge, StagedSmall, O, false>(l, 1, x);
    };
    return out_dt == HETA_F32 ? go(float{}) : go(bf16_t{});
}

// ---- rows ----------------------------------------------------------------------------------------------
// A row lies in the registers of 8 to 64 lanes, eight consecutive columns a lane and chunk; longer ones are walked twice by a workgroup.
template <typename T, int LANES, int NV> __global__ void __launch_bounds__(256) rows_i8_kernel(const T *x, int64_t ld_x, int64_t n_rows, int32_t d, int8_t *out, int64_t ld_out, float *scale)
{
    constexpr int GROUPS = 256 / LANES;
    const int l = threadIdx.x % LANES, grp = threadIdx.x / LANES;
    // the last columns of a row that is no multiple of eight wide are the last eight, some of which another lane has as well
    auto first = [&](int i) {
        const int c = (i * LANES + l) * 8;
        return c < d && c + 8 > d && d >= 8 ? d - 8 : c;
    };
    for (int64_t r = static_cast<int64_t>(blockIdx.x) * GROUPS + grp; r < n_rows; r += static_cast<int64_t>(gridDim.x) * GROUPS) {
        float v[NV][8];
#pragma unroll
        for (int i = 0; i < NV; ++i) load8(x + r * ld_x + first(i), d - first(i), v[i]);
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) top = max(top, magnitude(v[i][e]));
#pragma unroll
        for (int o = LANES / 2; o > 0; o >>= 1) top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), o)));
        const float amax = __uint_as_float(top), f = i8_factor(amax);
        if (l == 0) scale[r] = i8_scale(amax);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = first(i);
            store_codes(reinterpret_cast<uint8_t *>(out) + r * ld_out + c, d - c,
                        Codes8{{four_i8(v[i][0] * f, v[i][1] * f, v[i][2] * f, v[i][3] * f), four_i8(v[i][4] * f, v[i][5] * f, v[i][6] * f, v[i][7] * f)}});
        }
    }
}
template <typename T> __global__ void __launch_bounds__(256) rows_i8_wide_kernel(const T *x, int64_t ld_x, int64_t n_rows, int32_t d, int8_t *out, int64_t ld_out, float *scale)
{
    __shared__ uint32_t tops[4];
    const uint32_t width = static_cast<uint32_t>(d); // unsigned: a step past the widest row, of 2^31 - 1,024, is still ahead
    for (int64_t r = blockIdx.x; r < n_rows; r += gridDim.x) {
        const T *row = x + r * ld_x;
        uint32_t top = 0;
        for (uint32_t c = threadIdx.x * 8; c < width; c += 2048) {
            float v[8];
            load8(row + c, static_cast<int>(width - c), v);
#pragma unroll
            for (int e = 0; e < 8; ++e) top = max(top, magnitude(v[e]));
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), o)));
        __syncthreads();
        if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
        __syncthreads();
        const float amax = __uint_as_float(max(max(tops[0], tops[1]), max(tops[2], tops[3]))), f = i8_factor(amax);
        if (threadIdx.x == 0) scale[r] = i8_scale(amax);
        for (uint32_t c = threadIdx.x * 8; c < width; c += 2048) {
            float v[8];
            load8(row + c, static_cast<int>(width - c), v);
            store_codes(reinterpret_cast<uint8_t *>(out) + r * ld_out + c, static_cast<int>(width - c), Codes8{{four_i8(v[0] * f, v[1] * f, v[2] * f, v[3] * f), four_i8(v[4] * f, v[5] * f, v[6] * f, v[7] * f)}});
        }
    }
}

// ---- weights -------------------------------------------------------------------------------------------
// Column j of W [d_in, d_out] becomes row j of the packed matrix.  Once per set of weights: one wavefront per column.
template <typename T> __global__ void __launch_bounds__(256) pack_i8_kernel(const T *W, int64_t ld_w, int32_t d_in, int32_t d_out, int8_t *out, int64_t ld_out, float *scale, unsigned first)
{
    const int64_t j = (static_cast<int64_t>(blockIdx.x) + first) * 4 + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    if (j >= d_out) return;
    uint32_t top = 0;
    for (int k = lane; k < d_in; k += 64) top = max(top, magnitude(widen(W[k * ld_w + j])));
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), o)));
    const float amax = __uint_as_float(top), f = i8_factor(amax);
    for (int k = lane; k < d_in; k += 64) out[j * ld_out + k] = static_cast<int8_t>(one_i8(widen(W[k * ld_w + j]) * f));
    if (lane == 0) scale[j] = i8_scale(amax);
}

template <typename T> static void launch_rows(const T *x, int64_t ld_x, int64_t n, int32_t d, int8_t *out, int64_t ld_out, float *scale, hipStream_t st)
{
    auto go = [&](auto lanes, auto nv) {
        constexpr int L = decltype(lanes)::value, NV = decltype(nv)::value;
        const int64_t blocks = (n + 256 / L - 1) / (256 / L);
        hipLaunchKernelGGL((rows_i8_kernel<T, L, NV>), dim3(static_cast<unsigned>(std::min<int64_t>(blocks, 1 << 20))), dim3(256), 0, st, x, ld_x, n, d, out, ld_out, scale);
    };
    using std::integral_constant;
    if (d <= 64) go(integral_constant<int, 8>{}, integral_constant<int, 1>{});
    else if (d <= 128) go(integral_constant<int, 16>{}, integral_constant<int, 1>{});
    else if (d <= 256) go(integral_constant<int, 32>{}, integral_constant<int, 1>{});
    else if (d <= 512) go(integral_constant<int, 64>{}, integral_constant<int, 1>{});
    else if (d <= 1024) go(integral_constant<int, 64>{}, integral_constant<int, 2>{});
    else if (d <= 2048) go(integral_constant<int, 64>{}, integral_constant<int, 4>{});
    else hipLaunchKernelGGL(rows_i8_wide_kernel<T>, dim3(static_cast<unsigned>(std::min<int64_t>(n, 1 << 20))), dim3(256), 0, st, x, ld_x, n, d, out, ld_out, scale);
}

} // namespace heta

using namespace heta;

extern "C" heta_status heta_linear_rows_i8(int64_t n_rows, int32_t d, const void *x, heta_dtype x_dt, int64_t ld_x, void *out, int64_t ld_out, float *scale, void *hip_stream)
{
    const char *who = "heta_linear_rows_i8";
    if (n_rows < 0 || d <= 0) return fail(HETA_ERR_SHAPE, "%s: need n_rows >= 0 and d > 0", who);
    if (d > kWidest) return fail(HETA_ERR_UNSUPPORTED, "%s: rows too wide", who);
    if (!valid_dtype(x_dt)) return fail(HETA_ERR_INVALID_ARG, "%s: bad dtype", who);
    HETA_TRY(check_rows(who, "x", x, n_rows, ld_x, d, dtype_size(x_dt)));
    HETA_TRY(check_rows(who, "out", out, n_rows, ld_out, d, 1));
    if ((!scale && n_rows > 0) || (reinterpret_cast<uintptr_t>(scale) & 3u)) return fail(HETA_ERR_INVALID_ARG, "%s: bad scale", who);
    const RowRange rx(x, n_rows, ld_x, d, dtype_size(x_dt)), ro(out, n_rows, ld_out, d, 1), rs(scale, 1, n_rows, n_rows, 4);
    if (ro.overlaps(rx) || rs.overlaps(rx) || rs.overlaps(ro)) return fail(HETA_ERR_INVALID_ARG, "%s: an output overlaps an operand or another output", who);
    if (n_rows == 0) return HETA_OK;
    hipStream_t st = as_stream(hip_stream);
    ProfScope prof("rows_i8_kernel", st, static_cast<double>(n_rows) * (d * (dtype_size(x_dt) + 1.0) + 4), 0);
    if (x_dt == HETA_F32) launch_rows(static_cast<const float *>(x), ld_x, n_rows, d, static_cast<int8_t *>(out), ld_out, scale, st);
    else launch_rows(static_cast<const bf16_t *>(x), ld_x, n_rows, d, static_cast<int8_t *>(out), ld_out, scale, st);
    HETA_LAUNCH_CHECK("rows_i8_kernel");
    return HETA_OK;
}

extern "C" heta_status heta_linear_pack_i8(const void *W, heta_dtype w_dt, int64_t ld_w, int32_t d_in, int32_t d_out, void *packed, int64_t ld_packed, float *scale, void *hip_stream)
{
    const char *who = "heta_linear_pack_i8";
    if (!valid_dtype(w_dt)) return fail(HETA_ERR_INVALID_ARG, "%s: bad dtype", who);
    if (d_in <= 0 || d_out <= 0) return fail(HETA_ERR_SHAPE, "%s: need widths > 0", who);
    if (std::max(d_in, d_out) > kWidest) return fail(HETA_ERR_UNSUPPORTED, "%s: rows too wide", who);
    HETA_TRY(check_rows(who, "W", W, 1, ld_w, d_out, dtype_size(w_dt)));
    HETA_TRY(check_rows(who, "packed", packed, 1, ld_packed, d_in, 1));
    if (!scale || (reinterpret_cast<uintptr_t>(scale) & 3u)) return fail(HETA_ERR_INVALID_ARG, "%s: bad scale", who);
    const RowRange w(W, d_in, ld_w, d_out, dtype_size(w_dt)), o(packed, d_out, ld_packed, d_in, 1), s(scale, 1, d_out, d_out, 4);
    if (o.overlaps(w) || s.overlaps(w) || s.overlaps(o)) return fail(HETA_ERR_INVALID_ARG, "%s: an output overlaps an operand or another output", who);
    hipStream_t st = as_stream(hip_stream);
    ProfScope prof("pack_i8_kernel", st, static_cast<double>(d_in) * d_out * (2.0 * dtype_size(w_dt) + 1.0), 0);
    launch_pieces((d_out + 3) / 4, 256, [&](unsigned first, unsigned count) {
        int8_t *const to = static_cast<int8_t *>(packed);
        if (w_dt == HETA_F32) hipLaunchKernelGGL(pack_i8_kernel<float>, dim3(count), dim3(256), 0, st, static_cast<const float *>(W), ld_w, d_in, d_out, to, ld_packed, scale, first);
        else hipLaunchKernelGGL(pack_i8_kernel<bf16_t>, dim3(count), dim3(256), 0, st, static_cast<const bf16_t *>(W), ld_w, d_in, d_out, to, ld_packed, scale, first);
    });
    HETA_LAUNCH_CHECK("pack_i8_kernel");
    return HETA_OK;
}
