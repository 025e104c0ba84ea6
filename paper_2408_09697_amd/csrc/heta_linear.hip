// Products with a fused epilogue (bias, activation, residual) over rows of node embeddings, and their backward pass: the two
// matrices of a feed-forward block that follows a layer's relation aggregation.
//
//     pre = s_i w_j (in . W) + bias,  out = act(pre) + residual          s, w: scales of 8-bit rows / columns, else 1
//     grad_pre = grad_out * act'(pre),  grad_bias = sum of its rows,  grad_in = (grad_pre . W^T) * act_in'(pre_in),
//     grad_W = in^T . grad_pre
//
// All three products are the tile kernel of heta_tiles.h: bf16 operands straight into LDS; e4m3 operands too, widened to
// bf16 behind LDS or, where the caller allows coarser sums, on the 8-bit matrix instruction at twice the rate (block scales 1;
// the scales of rows and columns come in the epilogue); 8-bit integers on the integer instruction; fp32 operands as three bf16 terms.  grad_W is split over the rows (long
// unaligned bf16 operands of it are copied to aligned rows first); the partial products are added in a fixed order.
#include <algorithm>

#include "heta_linear.h"

namespace heta {

// ---- sums of partials --------------------------------------------------------------------------------
// 256 threads: 256 / CH groups of four columns, CH chains over the partials each, joined through LDS in order.  A chain keeps
// sixteen loads in flight: with eight, and 32 chains for 256 columns of 2,048 partials, the sum took 36 us of a norm's 340.  Four columns
// come by one load at whatever place they start (a width that is no multiple of four shifts them from partial to partial).
typedef float float4_any __attribute__((ext_vector_type(4), aligned(4)));
template <int CH, typename O> __global__ void __launch_bounds__(256) fold_partials_kernel(const float *part, int64_t n_part, int64_t total, O *out, int32_t width, int64_t ld, const float *factor)
{
    constexpr int G = 256 / CH;
    __shared__ float sums[CH][G][4];
    const int gq = threadIdx.x % G, ch = threadIdx.x / G;
    const int64_t c = (static_cast<int64_t>(blockIdx.x) * G + gq) * 4;
    const int valid = static_cast<int>(min(total - c, static_cast<int64_t>(4)));
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    if (valid > 0) {
        // chain ch takes every CH-th partial
        if (valid == 4) {
            const float *p = part + c + ch * total;
            const int64_t n = ch < n_part ? (n_part - ch + CH - 1) / CH : 0, step = CH * total;
            int64_t i = 0;
            for (; i + 16 <= n; i += 16, p += 16 * step) {
                float4_any x[16];
#pragma unroll
                for (int q = 0; q < 16; ++q) x[q] = *reinterpret_cast<const float4_any *>(p + q * step);
#pragma unroll
                for (int q = 0; q < 16; ++q) {
                    s[0] += x[q].x; s[1] += x[q].y; s[2] += x[q].z; s[3] += x[q].w;
                }
            }
#pragma unroll 4
            for (; i < n; ++i, p += step) {
                const float4_any x = *reinterpret_cast<const float4_any *>(p);
                s[0] += x.x; s[1] += x.y; s[2] += x.z; s[3] += x.w;
            }
        } else {
#pragma unroll 8
            for (int64_t i = ch; i < n_part; i += CH) {
                const float *p = part + i * total + c;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (e < valid) s[e] += p[e];
            }
        }
    }
    if constexpr (CH > 1) {
#pragma unroll
        for (int e = 0; e < 4; ++e) sums[ch][gq][e] = s[e];
        __syncthreads();
        if (ch != 0) return;
#pragma unroll
        for (int i = 1; i < CH; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[e] += sums[i][gq][e];
    }
    if (factor) {
        const float f = *factor;
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] *= f;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e < valid) {
            const int64_t row = (c + e) / width, col = (c + e) - row * width;
            if constexpr (sizeof(O) == 2) out[row * ld + col] = to_bf16(s[e]);
            else out[row * ld + col] = s[e];
        }
}

template <typename O> static void fold_launch(const float *part, int64_t n_part, int64_t total, O *out, int32_t width, int64_t ld, hipStream_t st, const float *factor)
{
    const int64_t groups = (total + 3) / 4;
    // few columns: the chains are what keeps loads in flight
    if (groups < 2048 && n_part >= 64)
        hipLaunchKernelGGL((fold_partials_kernel<128, O>), dim3((unsigned)((groups + 1) / 2)), dim3(256), 0, st, part, n_part, total, out, width, ld, factor);
    else if (groups < 16384 && n_part >= 16)
        hipLaunchKernelGGL((fold_partials_kernel<16, O>), dim3((unsigned)((groups + 15) / 16)), dim3(256), 0, st, part, n_part, total, out, width, ld, factor);
    else
        hipLaunchKernelGGL((fold_partials_kernel<4, O>), dim3((unsigned)((groups + 63) / 64)), dim3(256), 0, st, part, n_part, total, out, width, ld, factor);
}

heta_status fold_partials(const float *part, int64_t n_part, int64_t total, void *out, heta_dtype out_dt, int32_t width, int64_t ld, hipStream_t st, const float *factor)
{
    if (total > kFoldMost) return fail(HETA_ERR_UNSUPPORTED, "sum of partials: too many columns for one launch");
    ProfScope prof("fold_partials_kernel", st, static_cast<double>(total) * (4.0 * n_part + dtype_size(out_dt)), static_cast<double>(total) * n_part);
    if (out_dt == HETA_F32) fold_launch(part, n_part, total, static_cast<float *>(out), width, ld, st, factor);
    else fold_launch(part, n_part, total, static_cast<bf16_t *>(out), width, ld, st, factor);
    HETA_LAUNCH_CHECK("fold_partials_kernel");
    return HETA_OK;
}

// ---- gradient through the activation, and the bias's ---------------------------------------------------
// A workgroup takes a slab of rows of 256 columns: 32 lanes of eight columns, 8 rows at a time; every lane keeps the sums of
// its columns, which are joined through LDS into the slab's row of the partials.  Four rows are read before the first is
// worked on.  ACT = NONE: sums alone.
template <typename E, int ACT, bool STREAM> __global__ void __launch_bounds__(256) act_grad_kernel(const E *go, int64_t ld_go, const E *pre, int64_t ld_pre, E *gp, int64_t ld_gp,
                                                                                                  int64_t n_rows, int32_t d, int64_t rows_each, float *part, uint32_t first)
{
    __shared__ float sums[8][256 + 8];
    constexpr bool ACTS = ACT != HETA_ACT_NONE;
    const int lx = threadIdx.x & 31, ly = threadIdx.x >> 5;
    const uint32_t strips = (d + 255) / 256, b = first + blockIdx.x;
    const int64_t slab = b / strips;
    const int c = static_cast<int>(b % strips) * 256 + lx * 8, valid = min(d - c, 8);
    float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (valid > 0) {
        const int64_t end = min(n_rows, (slab + 1) * rows_each);
        auto rows = [&](int64_t r, auto count) {
            constexpr int N = decltype(count)::value;
            float g[N][8], x[ACTS ? N : 1][8];
#pragma unroll
            for (int i = 0; i < N; ++i) {
                load8<STREAM>(go + (r + 8 * i) * ld_go + c, valid, g[i]);
                if constexpr (ACTS) load8<STREAM>(pre + (r + 8 * i) * ld_pre + c, valid, x[i]);
            }
#pragma unroll
            for (int i = 0; i < N; ++i) {
                if constexpr (ACTS) {
                    times_slopes(g[i], x[i], ACT);
                    store8<STREAM>(gp + (r + 8 * i) * ld_gp + c, valid, g[i]);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) s[e] += g[i][e];
            }
        };
        int64_t r = slab * rows_each + ly;
        for (; r + 24 < end; r += 32) rows(r, std::integral_constant<int, 4>{});
        for (; r < end; r += 8) rows(r, std::integral_constant<int, 1>{});
    }
    if (!part) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[ly][lx * 8 + e] = s[e];
    __syncthreads();
    const int col = static_cast<int>(b % strips) * 256 + threadIdx.x;
    if (col >= d) return;
    float t = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) t += sums[i][threadIdx.x];
    part[slab * d + col] = t;
}

// ---- weights in 8 bits -------------------------------------------------------------------------------
// Column j of W [d_in, d_out] becomes row j of the packed matrix [d_out, d_in], e4m3 with the scale max|W[:, j]| / 448.  Once per
// set of weights: one wavefront per column.
template <typename E> __global__ void __launch_bounds__(256) pack_e4m3_kernel(const E *W, int64_t ld_w, int32_t d_in, int32_t d_out, uint8_t *out, int64_t ld_out, float *scale, unsigned first)
{
    const int64_t j = (static_cast<int64_t>(blockIdx.x) + first) * 4 + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    if (j >= d_out) return;
    uint32_t top = 0;
    for (int k = lane; k < d_in; k += 64) top = max(top, magnitude(widen(W[k * ld_w + j])));
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), o)));
    const float amax = __uint_as_float(top), inv = e4m3_factor(amax);
    for (int k = lane; k < d_in; k += 64) {
        const float x = widen(W[k * ld_w + j]) * inv;
        out[j * ld_out + k] = static_cast<uint8_t>(__builtin_amdgcn_cvt_pk_fp8_f32(x, x, 0, false) & 0xff);
    }
    if (lane == 0) scale[j] = e4m3_scale(amax);
}

// ---- host side ---------------------------------------------------------------------------------------
static bool valid_act(int a) { return a >= HETA_ACT_NONE && a <= HETA_ACT_SILU; }

} // namespace heta

using namespace heta;

extern "C" heta_status heta_linear(heta_graph *g, const heta_linear_args *a, void *hip_stream)
{
    const char *who = "heta_linear";
    if (!g || !a) return fail(HETA_ERR_INVALID_ARG, "%s: null arguments", who);
    if (a->n_rows < 0 || a->d_in <= 0 || a->d_out <= 0) return fail(HETA_ERR_SHAPE, "%s: need n_rows >= 0 and widths > 0", who);
    if (std::max(a->d_in, a->d_out) > kWidest) return fail(HETA_ERR_UNSUPPORTED, "%s: rows too wide", who);
    if (!valid_act(a->act)) return fail(HETA_ERR_INVALID_ARG, "%s: bad act", who);
    const bool whole = a->in_dt == HETA_I8, q = a->in_dt == HETA_E4M3 || whole;
    if (!q && !valid_dtype(a->in_dt)) return fail(HETA_ERR_INVALID_ARG, "%s: bad dtype", who);
    if (!valid_dtype(a->out_dt)) return fail(HETA_ERR_INVALID_ARG, "%s: outputs are fp32 or bf16", who);
    if (a->w_dt != a->in_dt || (a->in_dt == HETA_F32 && a->out_dt != HETA_F32))
        return fail(HETA_ERR_UNSUPPORTED, "%s: in and W have one type, and fp32 operands an fp32 output", who);
    // no rows, no scales of theirs: an empty array's address may be null
    if ((q ? !a->in_scale && a->n_rows > 0 : a->in_scale != nullptr) || q != (a->w_scale != nullptr))
        return fail(HETA_ERR_INVALID_ARG, "%s: scales belong to 8-bit operands, and those need them", who);
    if ((!q || whole) && a->coarse_sums) return fail(HETA_ERR_INVALID_ARG, "%s: coarse sums are those of HETA_E4M3 operands", who);
    if (whole && a->d_in >= 1 << 17) return fail(HETA_ERR_UNSUPPORTED, "%s: 2^17 products of 8-bit integers and more may pass 32 bits", who);
    const size_t esz = q ? 1 : dtype_size(a->in_dt), osz = dtype_size(a->out_dt);
    HETA_TRY(check_rows(who, "in", a->in, a->n_rows, a->ld_in, a->d_in, esz));
    HETA_TRY(check_rows(who, "W", a->W, 1, a->ld_w, q ? a->d_in : a->d_out, esz));
    HETA_TRY(check_rows(who, "out", a->out, a->n_rows, a->ld_out, a->d_out, osz));
    if (a->residual) HETA_TRY(check_rows(who, "residual", a->residual, a->n_rows, a->ld_res, a->d_out, osz));
    if (a->pre) HETA_TRY(check_rows(who, "pre", a->pre, a->n_rows, a->ld_pre, a->d_out, osz));
    for (const float *v : {a->bias, a->in_scale, a->w_scale})
        if (reinterpret_cast<uintptr_t>(v) & 3u) return fail(HETA_ERR_INVALID_ARG, "%s: pointer not aligned to its element size", who);
    const RowRange out(a->out, a->n_rows, a->ld_out, a->d_out, osz), pre(a->pre, a->n_rows, a->ld_pre, a->d_out, osz);
    const RowRange in(a->in, a->n_rows, a->ld_in, a->d_in, esz), w(a->W, q ? a->d_out : a->d_in, a->ld_w, q ? a->d_in : a->d_out, esz);
    const RowRange res(a->residual, a->n_rows, a->ld_res, a->d_out, osz);
    const bool same_rows = a->residual == a->out && a->ld_res == a->ld_out; // read and written by the same lane
    if (out.overlaps(in) || out.overlaps(w) || out.overlaps(pre) || pre.overlaps(in) || pre.overlaps(w) || pre.overlaps(res) || (out.overlaps(res) && !same_rows))
        return fail(HETA_ERR_INVALID_ARG, "%s: an output overlaps an operand or another output", who);
    for (const RowRange &v : {RowRange(a->bias, 1, a->d_out, a->d_out, 4), RowRange(a->in_scale, 1, a->n_rows, a->n_rows, 4), RowRange(a->w_scale, 1, a->d_out, a->d_out, 4)})
        if (out.overlaps(v) || pre.overlaps(v)) return fail(HETA_ERR_INVALID_ARG, "%s: bias or a scale overlaps an output", who);
    if (a->n_rows == 0) return HETA_OK;
    const LinearExtra x{a->bias, a->in_scale, a->w_scale, a->residual, a->pre, a->out, a->ld_res, a->ld_pre, a->ld_out, a->act, HETA_ACT_NONE};
    const double bytes = static_cast<double>(a->n_rows) * (a->d_in * esz + a->d_out * osz * (1.0 + !!a->residual + !!a->pre)) + static_cast<double>(a->d_in) * a->d_out * esz;
    const Launch l{g, who, "linear_kernel", TileItem{a->in, a->W, a->ld_in, a->ld_w, 0, 0, a->n_rows, a->d_out, a->d_in, a->d_in, 1, 0, 0, 0, 0, 0}, bytes,
                   2.0 * a->n_rows * a->d_in * a->d_out, as_stream(hip_stream)};
    if (whole) return launch_linear_i8(l, a->out_dt, x);
    if (q) return launch_linear_e4m3(l, a->out_dt, a->coarse_sums != 0, x);
    return a->in_dt == HETA_F32 ? launch_linear_f32(l, false, x) : launch_linear_bf16(l, false, a->out_dt, x);
}

extern "C" heta_status heta_linear_bwd(heta_graph *g, const heta_linear_bwd_args *a, void *hip_stream)
{
    const char *who = "heta_linear_bwd";
    if (!g || !a) return fail(HETA_ERR_INVALID_ARG, "%s: null arguments", who);
    if (a->n_rows < 0 || a->d_in <= 0 || a->d_out <= 0) return fail(HETA_ERR_SHAPE, "%s: need n_rows >= 0 and widths > 0", who);
    if (std::max(a->d_in, a->d_out) > kWidest) return fail(HETA_ERR_UNSUPPORTED, "%s: rows too wide", who);
    if (!valid_act(a->act) || !valid_act(a->in_act)) return fail(HETA_ERR_INVALID_ARG, "%s: bad act", who);
    if (!valid_dtype(a->dt) || (a->dW && !valid_dtype(a->dw_dt))) return fail(HETA_ERR_INVALID_ARG, "%s: bad dtype", who);
    if (a->dt == HETA_F32 && a->dW && a->dw_dt != HETA_F32) return fail(HETA_ERR_UNSUPPORTED, "%s: fp32 operands have an fp32 weight gradient", who);
    const bool acts = a->act != HETA_ACT_NONE, fused = a->in_act != HETA_ACT_NONE;
    const size_t esz = dtype_size(a->dt);
    const int64_t n = a->n_rows;
    HETA_TRY(check_rows(who, "grad_out", a->grad_out, n, a->ld_go, a->d_out, esz));
    if (acts) {
        HETA_TRY(check_rows(who, "pre", a->pre, n, a->ld_pre, a->d_out, esz));
        HETA_TRY(check_rows(who, "grad_pre", a->grad_pre, n, a->ld_gp, a->d_out, esz));
    }
    if (a->grad_in) {
        HETA_TRY(check_rows(who, "grad_in", a->grad_in, n, a->ld_gi, a->d_in, esz));
        HETA_TRY(check_rows(who, "W", a->W, 1, a->ld_w, a->d_out, esz));
        if (fused) HETA_TRY(check_rows(who, "in_pre", a->in_pre, n, a->ld_ip, a->d_in, esz));
    }
    if (a->dW) {
        HETA_TRY(check_rows(who, "in", a->in, n, a->ld_in, a->d_in, esz));
        HETA_TRY(check_rows(who, "dW", a->dW, 1, a->ld_dw, a->d_out, dtype_size(a->dw_dt)));
    }
    if (reinterpret_cast<uintptr_t>(a->dbias) & 3u) return fail(HETA_ERR_INVALID_ARG, "%s: pointer not aligned to its element size", who);
    const RowRange go(a->grad_out, n, a->ld_go, a->d_out, esz), pre(acts ? a->pre : nullptr, n, a->ld_pre, a->d_out, esz);
    const RowRange gp(acts ? a->grad_pre : nullptr, n, a->ld_gp, a->d_out, esz), gi(a->grad_in, n, a->ld_gi, a->d_in, esz);
    const RowRange w(a->grad_in ? a->W : nullptr, a->d_in, a->ld_w, a->d_out, esz), in(a->dW ? a->in : nullptr, n, a->ld_in, a->d_in, esz);
    const RowRange ip(a->grad_in && fused ? a->in_pre : nullptr, n, a->ld_ip, a->d_in, esz);
    const RowRange dw(a->dW, a->d_in, a->ld_dw, a->d_out, a->dW ? dtype_size(a->dw_dt) : 4), db(a->dbias, 1, a->d_out, a->d_out, 4);
    const bool over_go = a->grad_pre == a->grad_out && a->ld_gp == a->ld_go, over_pre = a->grad_pre == a->pre && a->ld_gp == a->ld_pre;
    const bool over_ip = a->grad_in == a->in_pre && a->ld_gi == a->ld_ip; // each read and written by the same lane
    const RowRange outs[4] = {gp, gi, dw, db}, ins[5] = {go, pre, w, in, ip};
    for (int i = 0; i < 4; ++i) {
        for (int j = 0; j < i; ++j)
            if (outs[i].overlaps(outs[j])) return fail(HETA_ERR_INVALID_ARG, "%s: two outputs overlap", who);
        for (int j = 0; j < 5; ++j)
            if (outs[i].overlaps(ins[j]) && !(i == 0 && ((j == 0 && over_go) || (j == 1 && over_pre))) && !(i == 1 && j == 4 && over_ip))
                return fail(HETA_ERR_INVALID_ARG, "%s: an output overlaps an operand", who);
    }
    hipStream_t st = as_stream(hip_stream);

    // workspace: partial sums of the bias gradient and partial products of the weight gradient
    const int64_t strips = (a->d_out + 255) / 256;
    const int64_t slabs = std::max<int64_t>(1, std::min<int64_t>((n + 63) / 64, 2048 / strips));
    const int64_t rows_each = std::max<int64_t>(1, (n + slabs - 1) / slabs);
    const int64_t bias_elems = a->dbias ? slabs * a->d_out : 0;
    const int64_t bias_off = (bias_elems + 3) / 4 * 4;
    const int64_t w_tiles = tiles_of(a->d_in, a->d_out, 256, 256);
    int64_t n_split = 0, k_per_split = 0;
    if (a->dW && n > 0) {
        const int64_t most = std::max<int64_t>(1, 256 / w_tiles); // one workgroup per CU
        k_per_split = (std::max<int64_t>((n + most - 1) / most, 256) + 63) / 64 * 64;
        n_split = (n + k_per_split - 1) / k_per_split;
    }
    const int64_t w_elems = n_split * a->d_in * a->d_out;
    const void *gpre = acts ? a->grad_pre : a->grad_out;
    const int64_t ld_gpre = acts ? a->ld_gp : a->ld_go;
    const double flops = 2.0 * n * a->d_in * a->d_out;
    const double in_bytes = (static_cast<double>(n) * (a->d_in * (fused ? 2 : 1) + a->d_out) + static_cast<double>(a->d_in) * a->d_out) * esz;
    const Launch in_l{g, who, "linear_grad_in_kernel", TileItem{gpre, a->W, ld_gpre, a->ld_w, 0, 0, n, a->d_in, a->d_out, a->d_out, 1, 0, 0, 0, 0, 0}, in_bytes, flops, st};
    Launch w_l{g, who, "linear_grad_w_kernel", TileItem{a->in, gpre, a->ld_in, ld_gpre, 0, 0, a->d_in, a->d_out, n, k_per_split, static_cast<int32_t>(n_split), 0, 0, 0, 0, 0},
               static_cast<double>(n) * (a->d_in + a->d_out) * esz + 4.0 * w_elems, flops, st};

    // Everything that can fail comes before the first launch.  The copies to aligned rows are only faster: without room for them the
    // operands are read as they are.
    if (a->dW && (n >= (int64_t(1) << 31) || static_cast<int64_t>(a->d_in) * a->d_out > kFoldMost))
        return fail(HETA_ERR_UNSUPPORTED, "%s: weight gradient of too many rows or elements", who);
    size_t need = static_cast<size_t>(bias_off + w_elems) * sizeof(float);
    const size_t copies_at = (need + 255) / 256 * 256;
    size_t copies = a->dW && n > 0 && a->dt == HETA_BF16 ? align_grad_w_bytes(w_l) : 0;
    if (a->grad_in && n > 0) need = std::max(need, plan_split(in_l, esz).bytes);
    const size_t most = std::max(need, copies_at + copies);
    if (copies > 0 && ((g->ws_refused > 0 && most >= g->ws_refused) || ensure_workspace(g, most) != HETA_OK)) copies = 0;
    if (need > 0) HETA_TRY(ensure_workspace(g, need));
    float *ws = static_cast<float *>(g->d_ws);

    // gradient at the pre-activation
    if (n > 0 && (acts || a->dbias)) {
        const double bytes = static_cast<double>(n) * a->d_out * esz * (acts ? 3 : 1);
        ProfScope prof("act_grad_kernel", st, bytes, static_cast<double>(n) * a->d_out);
        auto go = [&](auto tag, auto act, auto stream) {
            using E = decltype(tag);
            launch_pieces(slabs * strips, 256, [&](unsigned first, unsigned count) {
                hipLaunchKernelGGL((act_grad_kernel<E, decltype(act)::value, decltype(stream)::value>), dim3(count), dim3(256), 0, st, static_cast<const E *>(a->grad_out), a->ld_go,
                                   static_cast<const E *>(a->pre), a->ld_pre, static_cast<E *>(a->grad_pre), a->ld_gp, n, a->d_out, rows_each, a->dbias ? ws : nullptr, first);
            });
            return HETA_OK;
        };
        auto with = [&](auto tag) { return with_act(a->act, [&](auto act) { return streams(bytes) ? go(tag, act, std::true_type{}) : go(tag, act, std::false_type{}); }); };
        (void)(a->dt == HETA_F32 ? with(float{}) : with(bf16_t{}));
        HETA_LAUNCH_CHECK("act_grad_kernel");
    }
    if (a->dbias) HETA_TRY(fold_partials(ws, n > 0 ? slabs : 0, a->d_out, a->dbias, HETA_F32, a->d_out, a->d_out, st));

    if (a->grad_in && n > 0) {
        const LinearExtra x{nullptr, nullptr, nullptr, fused ? a->in_pre : nullptr, nullptr, a->grad_in, a->ld_ip, 0, a->ld_gi, HETA_ACT_NONE, a->in_act};
        HETA_TRY(a->dt == HETA_F32 ? launch_linear_f32(in_l, true, x) : launch_linear_bf16(in_l, true, HETA_BF16, x));
    }
    if (a->dW) {
        float *part = ws + bias_off;
        if (copies > 0) HETA_TRY(align_grad_w_bf16(w_l, static_cast<char *>(g->d_ws) + copies_at));
        if (n > 0) HETA_TRY(a->dt == HETA_F32 ? launch_grad_w_f32(w_l, part) : launch_grad_w_bf16(w_l, part));
        HETA_TRY(fold_partials(part, n_split, static_cast<int64_t>(a->d_in) * a->d_out, a->dW, a->dw_dt, a->d_out, a->ld_dw, st));
    }
    return HETA_OK;
}

extern "C" heta_status heta_linear_pack_e4m3(const void *W, heta_dtype w_dt, int64_t ld_w, int32_t d_in, int32_t d_out, void *packed, int64_t ld_packed, float *scale, void *hip_stream)
{
    const char *who = "heta_linear_pack_e4m3";
    if (!valid_dtype(w_dt)) return fail(HETA_ERR_INVALID_ARG, "%s: bad dtype", who);
    if (d_in <= 0 || d_out <= 0) return fail(HETA_ERR_SHAPE, "%s: need widths > 0", who);
    if (std::max(d_in, d_out) > kWidest) return fail(HETA_ERR_UNSUPPORTED, "%s: rows too wide", who);
    HETA_TRY(check_rows(who, "W", W, 1, ld_w, d_out, dtype_size(w_dt)));
    HETA_TRY(check_rows(who, "packed", packed, 1, ld_packed, d_in, 1));
    if (!scale || (reinterpret_cast<uintptr_t>(scale) & 3u)) return fail(HETA_ERR_INVALID_ARG, "%s: bad scale", who);
    const RowRange w(W, d_in, ld_w, d_out, dtype_size(w_dt)), o(packed, d_out, ld_packed, d_in, 1), s(scale, 1, d_out, d_out, 4);
    if (o.overlaps(w) || s.overlaps(w) || s.overlaps(o)) return fail(HETA_ERR_INVALID_ARG, "%s: an output overlaps an operand or another output", who);
    hipStream_t st = as_stream(hip_stream);
    ProfScope prof("pack_e4m3_kernel", st, static_cast<double>(d_in) * d_out * (2.0 * dtype_size(w_dt) + 1.0), 0);
    launch_pieces((d_out + 3) / 4, 256, [&](unsigned first, unsigned count) {
        uint8_t *const to = static_cast<uint8_t *>(packed);
        if (w_dt == HETA_F32) hipLaunchKernelGGL(pack_e4m3_kernel<float>, dim3(count), dim3(256), 0, st, static_cast<const float *>(W), ld_w, d_in, d_out, to, ld_packed, scale, first);
        else hipLaunchKernelGGL(pack_e4m3_kernel<bf16_t>, dim3(count), dim3(256), 0, st, static_cast<const bf16_t *>(W), ld_w, d_in, d_out, to, ld_packed, scale, first);
    });
    HETA_LAUNCH_CHECK("pack_e4m3_kernel");
    return HETA_OK;
}
