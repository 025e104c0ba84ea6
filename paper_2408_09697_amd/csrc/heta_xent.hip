// Softmax cross entropy of rows through an output product, and its gradients, without the logits in memory.
//
//     z = in . W + bias,  lse_i = log sum_j exp z_ij,  loss_i = lse_i - z_i,label(i)   (0 for a row without a label)
//     D_ij = g_i (exp(z_ij - lse_i) - [j = label(i)]),  grad_in = F D W^T,  grad_W = F in^T D,  grad_bias = F sum_i D_i
//
// Forward: the product of heta_tiles.h with an epilogue that leaves, of a row's logits in a wavefront's columns, their largest and the sum of
// the exponentials below it, 8 bytes for 64 logits; a second kernel joins a row's.  The label's logit is taken from the registers it is in.
// Backward: the logits are formed again (2 d operations each; kept in 4 bytes they would cost as long to write and read at d = 1,024 and
// longer below), their epilogue makes D of them, and two products read D.  D is made in pieces of 512 MB, of about as many rows as classes,
// since every further piece along the classes adds n d partial sums of grad_in, and every one along the rows d V of grad_W (8,192 x 512 x 131,072, us:
// 5,044; 192 MB, which the last-level cache holds, but with more products, split further, 5,602; 256 MB 5,507, 1 GB 5,103, all at once 5,277).
// D is stored in the operands' type: the matrix instruction reads 16 bits, and its rounding (2^-9 of each D, to and fro) is below that of a gradient
// in 16 bits.  F, which all rows share (scale, over the number of labelled rows), multiplies the sums: in D, its rounding would be the same for all labels' elements
// (8,192 x 512 x 131,072: gradients 3.7e-3 of their norm off, 1.7e-3 this way, their own rounding).  grad_bias is added up from the unrounded D in the epilogue's registers.
// Logits are held in units of log 2, z log2(e), from one fused operation with the bias, so that exponentials are the hardware's 2^x.
//
// A row without a label has D = 0 whatever it holds; where it holds NaN or infinities (a padded batch), 0 times those would reach grad_W, which then reads
// a copy of the rows with zeros in their place.  Such rows have an lse that is not finite, which is how they are found.
#include <algorithm>
#include <cmath>

#include "heta_linear.h"
#include "heta_test_hooks.h"

namespace heta {

constexpr float kLn2 = 0.6931471805599453f;
// In the place of a largest logit of -infinity or infinity: beyond every other, and its difference to any is finite.
constexpr float kBeyond = 1e30f, kNothing = -kBeyond;

// ---- forward: a tile's logits ----------------------------------------------------------------------------
struct XentPart {
    float top, sum; // in units of log 2; sum over j of 2^(z_j - top)
};
// top is kept finite; with a logit of +infinity the sum is infinite, whatever it is joined with
__device__ __forceinline__ float finite_top(float t) { return __builtin_amdgcn_fmed3f(t, kNothing, kBeyond); }
__device__ __forceinline__ XentPart join(XentPart a, XentPart b)
{
    const float t = fmaxf(a.top, b.top);
    return {t, a.sum * __builtin_amdgcn_exp2f(a.top - t) + b.sum * __builtin_amdgcn_exp2f(b.top - t)};
}

// Sums start from the bias (nullable); register 4 q + e of block jj is column 32 jj + 8 q + 4 (lane / 32) + e of the strip.
template <typename C, typename Acc> __device__ __forceinline__ void begin_with(const float *bias, int64_t n0, int64_t N, Acc (&acc)[C::MI][C::NJ], int lane)
{
    int here = lane;
    asm volatile("" : "+v"(here)); // not kept through the products
    const int half = here >> 5;
#pragma unroll
    for (int jj = 0; jj < C::NJ; ++jj)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            float b[4] = {0.f, 0.f, 0.f, 0.f};
            if (bias) {
                const int64_t n = n0 + 32 * jj + 8 * q + 4 * half;
                if (n0 + 32 * C::NJ <= N) {
                    const uintx4 w = load16(bias + n);
#pragma unroll
                    for (int e = 0; e < 4; ++e) b[e] = __uint_as_float(w[e]);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) b[e] = bias[min(n + e, N - 1)];
                }
            }
#pragma unroll
            for (int i = 0; i < C::MI; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][jj][4 * q + e] = b[e];
        }
}
struct XentForward {
    const float *bias;     // nullable
    const int64_t *labels;
    XentPart *part;        // [strips of columns][n]
    float *target;         // [n]: the label's logit
};
struct XentForwardEpi {
    static constexpr int kItems = 1;
    static constexpr bool kTile = true;
    template <typename C> static constexpr int kStrip = 0;
    using Extra = XentForward;
    __device__ __forceinline__ static void choose(const Extra &, TileItem &) {}
    template <typename C, typename Acc> __device__ __forceinline__ static void begin(const Extra &x, const TileItem &it, Acc (&acc)[C::MI][C::NJ], const TilePlace &now, int wave, int lane)
    {
        begin_with<C>(x.bias, now.n0 + (wave % C::WN) * (32 * C::NJ), it.N, acc, lane);
    }
    template <typename C, typename Acc>
    __device__ __forceinline__ static void tile(const Extra &x, const TileItem &it, Acc (&acc)[C::MI][C::NJ], float *, const TilePlace &now, int wave, int lane)
    {
        constexpr int MI = C::MI, NJ = C::NJ;
        int here = lane;
        asm volatile("" : "+v"(here)); // not kept through the products
        const int half = here >> 5, l32 = here & 31;
        const int64_t m0 = now.m0 + (wave / C::WN) * (32 * MI) + l32, n0 = now.n0 + (wave % C::WN) * (32 * NJ);
        if (n0 >= it.N) return;
        const int n_here = static_cast<int>(min(it.N - n0, static_cast<int64_t>(32 * NJ))); // columns of this strip
        // columns 32 jj + 8 q + 4 half + e of the strip are a lane's; edge: some are beyond the last class, where acc may hold anything
        auto strip_part = [&](auto edge) {
            constexpr bool EDGE = decltype(edge)::value;
#pragma unroll
            for (int i = 0; i < MI; ++i) {
                const int64_t m = m0 + 32 * i, label = x.labels[min(m, it.M - 1)] - n0;
                const int at = label >= 0 && label < n_here ? static_cast<int>(label) - 4 * half : -64; // the label's column
                XentPart p;
#pragma unroll
                for (int jj = 0; jj < NJ; ++jj) {
                    __builtin_amdgcn_sched_barrier(0); // one block at a time: the registers hold no more beside the sums
                    int beyond = n_here - 4 * half - 32 * jj;
                    asm volatile("" : "+v"(beyond)); // compared here, not once for all rows: that takes two scalar registers a column
                    auto &z = acc[i][jj];
                    float top = -INFINITY, sum = 0.f;
#pragma unroll
                    for (int v = 0; v < 16; ++v) {
                        if constexpr (EDGE) z[v] = 8 * (v / 4) + v % 4 < beyond ? z[v] : -INFINITY;
                        top = fmaxf(top, z[v]);
                    }
                    top = finite_top(top * kLog2e);
#pragma unroll
                    for (int v = 0; v < 16; ++v) sum += __builtin_amdgcn_exp2f(fmaf(z[v], kLog2e, -top));
                    p = jj == 0 ? XentPart{top, sum} : join(p, {top, sum});
                    const int c = at - 32 * jj;
                    if (__any(c >= 0 && c < 32 && (c & 4) == 0)) {
                        float t = 0.f;
#pragma unroll
                        for (int v = 0; v < 16; ++v) t = c == 8 * (v / 4) + v % 4 ? z[v] : t;
                        if (c >= 0 && c < 32 && (c & 4) == 0 && m < it.M) x.target[m] = t * kLog2e;
                    }
                }
                p = join(p, {__shfl_xor(p.top, 32), __shfl_xor(p.sum, 32)});
                if (half == 0 && m < it.M) x.part[n0 / (32 * NJ) * it.M + m] = p;
            }
        };
        if (n_here == 32 * NJ) strip_part(std::false_type{});
        else strip_part(std::true_type{});
    }
};

// Row m's parts of every G-th strip from `first` on, eight loads in flight.
template <int G> __device__ __forceinline__ XentPart join_strips(const XentPart *part, int64_t first, int64_t end, int64_t n, int64_t m)
{
    XentPart p{kNothing, 0.f};
    for (int64_t s = first; s < end; s += 8 * G) {
        XentPart q[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) q[u] = s + u * G < end ? part[(s + u * G) * n + m] : XentPart{kNothing, 0.f};
#pragma unroll
        for (int u = 0; u < 8; ++u) p = join(p, q[u]);
    }
    return p;
}

// ---- forward: many parts of few rows joined to fewer -------------------------------------------------------
// A workgroup takes `each` strips of R rows; out: [chunks][n].
template <int R> __global__ void __launch_bounds__(256) xent_join_kernel(const XentPart *part, int64_t strips, int64_t each, int64_t n, int64_t row_groups, XentPart *out)
{
    constexpr int G = 256 / R;
    __shared__ XentPart parts[G][R];
    const int r = threadIdx.x % R, g = threadIdx.x / R;
    const int64_t chunk = blockIdx.x / row_groups, m = (blockIdx.x - chunk * row_groups) * R + r, end = min(strips, (chunk + 1) * each);
    XentPart p{kNothing, 0.f};
    if (m < n) p = join_strips<G>(part, chunk * each + g, end, n, m);
    parts[g][r] = p;
    __syncthreads();
    for (int h = G / 2; h > 0; h /= 2) {
        if (g < h) parts[g][r] = join(parts[g][r], parts[g + h][r]);
        __syncthreads();
    }
    if (g == 0 && m < n) out[chunk * n + m] = parts[0][r];
}

// ---- forward: a row's parts joined -------------------------------------------------------------------------
// R rows a workgroup, 256 / R threads a row.  sums: of the workgroup's losses, and how many rows have a label; a single workgroup writes the mean at once.
struct XentSum {
    double loss, rows;
};
__device__ __forceinline__ void mean_of(XentSum s, float *mean)
{
    mean[0] = s.rows > 0 ? static_cast<float>(s.loss / s.rows) : 0.f;
    mean[1] = static_cast<float>(s.rows);
}
template <int R> __global__ void __launch_bounds__(256) xent_rows_kernel(const XentPart *part, int64_t strips, const float *target, const int64_t *labels, int64_t n, int64_t n_classes,
                                                                        float *loss, float *lse, XentSum *sums, float *mean)
{
    constexpr int G = 256 / R;
    __shared__ XentPart parts[G][R];
    __shared__ XentSum waves[4];
    const int r = threadIdx.x % R, g = threadIdx.x / R;
    const int64_t m = static_cast<int64_t>(blockIdx.x) * R + r;
    XentPart p{kNothing, 0.f};
    if (m < n) p = join_strips<G>(part, g, strips, n, m);
    parts[g][r] = p;
    __syncthreads();
    for (int h = G / 2; h > 0; h /= 2) {
        if (g < h) parts[g][r] = join(parts[g][r], parts[g + h][r]);
        __syncthreads();
    }
    XentSum s{0., 0.};
    if (g == 0 && m < n) {
        p = parts[0][r];
        const float l2 = p.top + __builtin_amdgcn_logf(p.sum);
        const int64_t label = labels[m];
        const bool has = label >= 0 && label < n_classes;
        const float mine = has ? (l2 - target[m]) * kLn2 : 0.f;
        lse[m] = l2 * kLn2;
        if (loss) loss[m] = mine;
        s = {mine, has ? 1. : 0.};
    }
    if (!mean) return;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) s = {s.loss + __shfl_xor(s.loss, o), s.rows + __shfl_xor(s.rows, o)};
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        s = waves[0];
        for (int i = 1; i < 4; ++i) s = {s.loss + waves[i].loss, s.rows + waves[i].rows};
        if (sums) sums[blockIdx.x] = s;
        else mean_of(s, mean);
    }
}
__global__ void __launch_bounds__(256) xent_mean_kernel(const XentSum *sums, int64_t n, float *mean)
{
    __shared__ XentSum all[256];
    XentSum s{0., 0.};
#pragma unroll 4
    for (int64_t i = threadIdx.x; i < n; i += 256) s = {s.loss + sums[i].loss, s.rows + sums[i].rows};
    all[threadIdx.x] = s;
    __syncthreads();
    for (int h = 128; h > 0; h /= 2) {
        if (threadIdx.x < static_cast<unsigned>(h)) all[threadIdx.x] = {all[threadIdx.x].loss + all[threadIdx.x + h].loss, all[threadIdx.x].rows + all[threadIdx.x + h].rows};
        __syncthreads();
    }
    if (threadIdx.x == 0) mean_of(all[0], mean);
}

// ---- backward: what a row's D needs ------------------------------------------------------------------------
struct XentRow {
    float lse;  // in units of log 2
    float f;    // the row's grad_loss; 0: its D is 0
    int64_t label;
};
// call: this call's number.  *poison becomes it where a row without a gradient holds something that 0 does not clear.
__global__ void __launch_bounds__(256) xent_prepare_kernel(const int64_t *labels, const float *lse, const float *grad_loss, const float *mean, float scale, int64_t n, int64_t n_classes,
                                                           XentRow *rows, float *factor, uint32_t *poison, uint32_t call)
{
    const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (i == 0) *factor = !mean ? scale : mean[1] > 0.f ? scale / mean[1] : 0.f;
    if (i >= n) return;
    const int64_t label = labels[i];
    const bool has = label >= 0 && label < n_classes;
    const float f = grad_loss ? grad_loss[i] : 1.f, l = lse[i];
    rows[i] = {l * kLog2e, has ? f : 0.f, has ? label : -1};
    if (!(has && f != 0.f) && !(fabsf(l) < INFINITY)) *poison = call; // all that write write the same
}
// The rows for grad_W: with zeros in those without a gradient.  Unless always, only where *poison says that there is need.
template <typename E> __global__ void __launch_bounds__(256) xent_clean_kernel(const E *in, int64_t ld, int64_t n, int32_t d, const XentRow *rows, E *out, int64_t ld_out, bool always,
                                                                               const uint32_t *poison, uint32_t call)
{
    if (!always && *poison != call) return;
    const int chunks = static_cast<int>(ld_out / 8);
    const int64_t total = n * chunks;
    for (int64_t q = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; q < total; q += static_cast<int64_t>(gridDim.x) * 256) {
        const int64_t r = q / chunks;
        const int c = static_cast<int>(q - r * chunks) * 8;
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (rows[r].f != 0.f) load8(in + r * ld + c, d - c, v);
        store8(out + r * ld_out + c, 8, v);
    }
}

// Both for few rows, in one launch: LANES lanes a row, which is copied whatever it holds.
template <typename E, int LANES> __global__ void __launch_bounds__(256) xent_prepare_rows_kernel(const int64_t *labels, const float *lse, const float *grad_loss, const float *mean, float scale,
                                                                                                int64_t n, int64_t n_classes, XentRow *rows, float *factor, uint32_t *poison, uint32_t call,
                                                                                                const E *in, int64_t ld, int32_t d, E *out, int64_t ld_out)
{
    const int64_t i = static_cast<int64_t>(blockIdx.x) * (256 / LANES) + threadIdx.x / LANES;
    const int l = threadIdx.x % LANES;
    if (i == 0 && l == 0) {
        *factor = !mean ? scale : mean[1] > 0.f ? scale / mean[1] : 0.f;
        *poison = call;
    }
    if (i >= n) return;
    const int64_t label = labels[i];
    const bool has = label >= 0 && label < n_classes;
    const float f = has ? (grad_loss ? grad_loss[i] : 1.f) : 0.f;
    if (l == 0) rows[i] = {lse[i] * kLog2e, f, has ? label : -1};
    for (int c = l * 8; c < ld_out; c += LANES * 8) {
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (f != 0.f) load8(in + i * ld + c, d - c, v);
        store8(out + i * ld_out + c, 8, v);
    }
}

// ---- backward: a tile of D -----------------------------------------------------------------------------------
struct XentBackward {
    const float *bias;   // nullable
    const XentRow *rows; // of the piece
    void *D;
    int64_t ld;
    float *sums;         // [strips of rows][N]: D's sums over them; nullable
    int64_t first;       // the piece's first class
    const float *factor; // of the sums (a single strip's are the result); nullable
};
template <typename O> struct XentBackwardEpi {
    static constexpr int kItems = 1;
    static constexpr bool kTile = true;
    // a wavefront's columns side by side: 64 columns of 16 bits are stored as whole lines (a quarter of 8,192 x 512 x 131,072 441 us by 32 columns, 420; 700,000 x 256 x 349 353, 325)
    template <typename C> static constexpr int kStrip = 4096 * C::NJ;
    using Extra = XentBackward;
    __device__ __forceinline__ static void choose(const Extra &, TileItem &) {}
    template <typename C, typename Acc> __device__ __forceinline__ static void begin(const Extra &x, const TileItem &it, Acc (&acc)[C::MI][C::NJ], const TilePlace &now, int wave, int lane)
    {
        begin_with<C>(x.bias, now.n0 + (wave % C::WN) * (32 * C::NJ), it.N, acc, lane);
    }
    template <typename C, typename Acc>
    __device__ __forceinline__ static void tile(const Extra &x, const TileItem &it, Acc (&acc)[C::MI][C::NJ], float *strip, const TilePlace &now, int wave, int lane)
    {
        constexpr int MI = C::MI, NJ = C::NJ, COLS = 32 * NJ, W = 16 / (int)sizeof(O), LPR = COLS / W, RPP = 64 / LPR, ROUNDS = 32 / RPP;
        int here = lane;
        asm volatile("" : "+v"(here)); // not kept through the products
        const int sr = here / LPR, sc = here % LPR, half = here >> 5, l32 = here & 31;
        const int64_t mw = now.m0 + (wave / C::WN) * (32 * MI), nw = now.n0 + (wave % C::WN) * (32 * NJ), m0 = mw + sr, n0 = nw + sc * W;
        float sum[W];
#pragma unroll
        for (int e = 0; e < W; ++e) sum[e] = 0.f;
        // a row a lane, as the sums lie; all of them here: a load behind the stores below waits for them
        float lse[MI], factor[MI];
        int at[MI]; // the label's column
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            const XentRow row = x.rows[min(mw + 32 * i + l32, it.M - 1)];
            const int64_t label = row.label - x.first - nw;
            lse[i] = row.lse;
            factor[i] = mw + 32 * i + l32 < it.M ? row.f : 0.f;
            at[i] = label >= 0 && label < 32 * NJ ? static_cast<int>(label) : -64;
        }
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            const float f = factor[i];
#pragma unroll
            for (int jj = 0; jj < NJ; ++jj)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    float y[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float p = __builtin_amdgcn_exp2f(fmaf(acc[i][jj][4 * q + e], kLog2e, -lse[i])) * f;
                        y[e] = f != 0.f ? p : 0.f;
                    }
                    *strip_at<COLS>(strip, l32, 8 * jj + 2 * q + half) = make_float4(y[0], y[1], y[2], y[3]);
                }
            if (half == 0 && at[i] >= 0) reinterpret_cast<float *>(strip_at<COLS>(strip, l32, at[i] / 4))[at[i] & 3] -= f;
#pragma unroll
            for (int r = 0; r < ROUNDS; ++r) {
                const int64_t m = m0 + 32 * i + RPP * r;
                float y[W];
#pragma unroll
                for (int h = 0; h < W / 4; ++h) {
                    const float4 v = *strip_at<COLS>(strip, RPP * r + sr, sc * (W / 4) + h);
                    y[4 * h] = v.x; y[4 * h + 1] = v.y; y[4 * h + 2] = v.z; y[4 * h + 3] = v.w;
                }
#pragma unroll
                for (int e = 0; e < W; ++e) sum[e] += y[e];
                // D's rows are padded to whole pieces; what lies behind the classes is read by nothing that is stored
                if (m < it.M && n0 < x.ld) store16(static_cast<O *>(x.D) + m * x.ld + n0, pack16<O>(y));
            }
        }
        if (!x.sums || mw >= it.M) return;
        const float whole = x.factor ? *x.factor : 1.f;
#pragma unroll
        for (int e = 0; e < W; ++e) {
            float s = sum[e];
#pragma unroll
            for (int o = LPR; o < 64; o <<= 1) s += __shfl_xor(s, o);
            if (sr == 0 && n0 + e < it.N) x.sums[mw / (32 * MI) * it.N + n0 + e] = s * whole;
        }
    }
};

// ---- backward: the products that read D -------------------------------------------------------------------
// Their partial sums, or, where a contraction is whole, the results.  grad_W's rows are read from their clean copy where there is need of it.
struct XentProduct {
    void *out;           // [splits][M][ld]
    int64_t ld;
    const float *factor; // nullable
    const void *clean;
    int64_t ld_clean;
    const uint32_t *poison; // nullable: no copy
    uint32_t call;
};
template <typename O> struct XentProductEpi {
    static constexpr int kItems = 1;
    static constexpr bool kTile = true;
    template <typename C> static constexpr int kStrip = 4096;
    using Extra = XentProduct;
    __device__ __forceinline__ static void choose(const Extra &x, TileItem &it)
    {
        if (!x.poison || *x.poison != x.call) return;
        it.A = x.clean;
        it.lda = x.ld_clean;
    }
    template <typename C, typename Acc> __device__ __forceinline__ static void begin(const Extra &, const TileItem &, Acc (&acc)[C::MI][C::NJ], const TilePlace &, int, int)
    {
#pragma unroll
        for (int i = 0; i < C::MI; ++i)
#pragma unroll
            for (int jj = 0; jj < C::NJ; ++jj)
#pragma unroll
                for (int v = 0; v < 16; ++v) acc[i][jj][v] = 0.f;
    }
    template <typename C, typename Acc>
    __device__ __forceinline__ static void tile(const Extra &x, const TileItem &it, Acc (&acc)[C::MI][C::NJ], float *strip, const TilePlace &now, int wave, int lane)
    {
        constexpr int MI = C::MI, NJ = C::NJ, W = 16 / (int)sizeof(O), LPR = 32 / W, RPP = 64 / LPR, ROUNDS = 32 / RPP;
        int here = lane;
        asm volatile("" : "+v"(here)); // not kept through the products
        const int sr = here / LPR, sc = here % LPR, half = here >> 5, l32 = here & 31;
        const int64_t m0 = now.m0 + (wave / C::WN) * (32 * MI) + sr, n0 = now.n0 + (wave % C::WN) * (32 * NJ) + sc * W;
        O *const out = static_cast<O *>(x.out) + now.split * it.M * x.ld;
        // awaited here: left to the branches below, a load is awaited behind every store so far at each of its uses (grad_in of 700,000 x 256 x 349 288 us that way, 249 this way; partial
        // sums of a quarter of 8,192 x 512 x 131,072 338 and 267)
        float f = x.factor ? *x.factor : 1.f;
        asm volatile("" : "+v"(f));
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int jj = 0; jj < NJ; ++jj) {
                const int64_t n = n0 + 32 * jj;
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    *strip_at(strip, l32, 2 * q + half) = make_float4(acc[i][jj][4 * q], acc[i][jj][4 * q + 1], acc[i][jj][4 * q + 2], acc[i][jj][4 * q + 3]);
#pragma unroll
                for (int r = 0; r < ROUNDS; ++r) {
                    const int64_t m = m0 + 32 * i + RPP * r;
                    float y[W];
#pragma unroll
                    for (int h = 0; h < W / 4; ++h) {
                        const float4 v = *strip_at(strip, RPP * r + sr, sc * (W / 4) + h);
                        y[4 * h] = v.x * f; y[4 * h + 1] = v.y * f; y[4 * h + 2] = v.z * f; y[4 * h + 3] = v.w * f;
                    }
                    if (m < it.M && n < it.N) store_piece(out + m * x.ld + n, static_cast<int>(min(it.N - n, static_cast<int64_t>(W))), pack16<O>(y));
                }
            }
    }
};

// ---- host side ---------------------------------------------------------------------------------------------
template <typename E, bool A_RC, bool B_RC, bool LARGE, bool STAGED> struct XentShape;
// grad_in's 256 x 256 (8,192 x 512 x 32,768 and 700,000 x 256 x 349, us, before their epilogue took a fifth less: 337 and 282; 256 x 128 by two workgroups a CU 387 and 348, 256 x 128 by one 460 and 377, four wavefronts with
// 128 x 128 each 313 and 326) and grad_W's, whose operands are both read transposed, 256 x 128 by two workgroups a CU, a wavefront 64 x 128 (261 and 219; 256 x 256 320 and 248, 64
// columns a wavefront 331 and 256).
template <> struct XentShape<bf16_t, false, false, true, false> { using type = TileShape<bf16_t, 2, 1, false, false, kDirect, 2, 4, 4, 2, 64, 2, 1>; };
template <> struct XentShape<bf16_t, true, true, true, false> { using type = TileShape<bf16_t, 2, 1, true, true, kDirect, 4, 1, 2, 4, 32, 2, 2>; };
// Logits of up to 32 rows: the weights are read once, 512 consecutive bytes at a time (4 x 1,024 x 1,100,000, forward, us: 380, 5.9 TB/s; 64 x 64 463, 32 x 128 398, 64 x 128 391, deeper
// rings by one workgroup a CU 389 to 405; 16 x 256 x 4,096 11.2, 64 x 64 21.3).
using XentSkinnyForwardTiles = TileShape<bf16_t, 2, 1, false, true, kDirect, 1, 4, 1, 2, 64, 2, 2>; // 32 x 256
using XentSkinnyBackwardTiles = TileShape<bf16_t, 2, 1, false, true, kDirect, 1, 4, 1, 2, 64, 2, 1>;
// The logits' tiles: 256 x 128 by four wavefronts, two workgroups on a CU, so that one's exponentials run beside the other's products (forward + both gradients of 700,000 x
// 256 x 349 and of 8,192 x 512 x 131,072, us: 1,414 and 5,630; one workgroup of eight wavefronts with 256 x 256 1,544 and 5,597, with 256 x 128 1,555 and 6,060; two with
// 128 x 128 1,526 and 6,090; each when its sums started from zero instead of the bias: 1,581 and 6,186 for this one).
using XentForwardTiles = TileShape<bf16_t, 2, 1, false, true, kDirect, 2, 2, 4, 2, 32, 3, 2>;
using XentBackwardTiles = TileShape<bf16_t, 2, 1, false, true, kDirect, 2, 2, 4, 2, 32, 2, 2>;
// grad_W's where 256 x 128 would have more beyond its rows
template <typename E> struct XentTurned { using type = TileShape<float, 2, 3, true, true, kStaged, 2, 4, 2, 2, 32, 2, 1>; };                 // 128 x 256
template <> struct XentTurned<bf16_t> { using type = TileShape<bf16_t, 2, 1, true, true, kDirect, 1, 4, 4, 2, 32, 2, 2>; };
template <bool A_RC, bool B_RC> struct XentShape<bf16_t, A_RC, B_RC, false, false> { using type = TileShape<bf16_t, 2, 1, A_RC, B_RC, kDirect, 2, 2, 1, 1, 64, 3, 2>; };  // 64 x 64
template <bool A_RC, bool B_RC, bool LARGE> struct XentShape<bf16_t, A_RC, B_RC, LARGE, true> { using type = TileShape<bf16_t, 2, 1, A_RC, B_RC, kStaged, 2, 2, 1, 1, 64, 2, 2>; };
template <bool A_RC, bool B_RC, bool STAGED> struct XentShape<float, A_RC, B_RC, true, STAGED> { using type = TileShape<float, 2, 3, A_RC, B_RC, kStaged, 4, 2, 2, 2, 32, 2, 1>; };  // 256 x 128
template <bool A_RC, bool B_RC, bool STAGED> struct XentShape<float, A_RC, B_RC, false, STAGED> { using type = TileShape<float, 2, 3, A_RC, B_RC, kStaged, 2, 2, 1, 1, 32, 2, 2>; }; // 64 x 64

static int64_t round_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

// Regions of the workspace, 256 bytes apart.
struct Regions {
    size_t bytes = 0;
    size_t take(size_t b)
    {
        const size_t at = bytes;
        bytes += (b + 255) / 256 * 256;
        return at;
    }
};

// What a row operand or the weights are read from: themselves, or a copy of them with aligned rows.
struct Operand {
    const void *p;
    int64_t ld;
};

// How the products of bf16 operands read them (those of fp32 go through registers, their addresses are 64 bits wide).  Straight into LDS goes what lies in rows that start at 16 bytes
// and whose offsets from a tile's first row stay below 2^32 bytes: kTileRows rows where a row's consecutive elements are contracted over (both operands of the logits but W, and W for
// grad_in), kTileDepth of them where a row is one k-value (W for the logits; in and D for grad_W).  D's offsets do, being within a piece.
constexpr int64_t kTileRows = 256, kTileDepth = 64;
static bool aligned_rows(const void *p, int64_t ld) { return aligned16(p) && ld % 8 == 0; }
static bool offsets_fit(int64_t rows, int64_t ld) { return rows * ld * 2 < (int64_t(1) << 32); }
// Whether the products are worth aligned copies of operands whose rows start anywhere: a copy of the weights is a pass over them, tiles that read them through registers take longer the more of
// them there are.  Forward + gradients, us, with copies / without: 256 x 30,011 by 256 rows 31 + 75 / 24 + 70, 384 28 + 97 / 31 + 107, 512 29 + 100 / 34 + 117, 4,096 97 + 318 / 178 +
// 579; 512 x 300,001 by 128 rows 218 + 484 / 138 + 488, 256 239 + 587 / 238 + 813, 512 314 + 876 / 435 + 1,391; 256 x 349 by 512 rows 18 + 30 / 16 + 30.  In between, down to
// some 300 rows over many classes, copies would already pay.
static bool copies_pay(int64_t n) { return n >= 512; }
struct XentReads {
    bool copy_w = false, copy_in = false;                 // to aligned rows first: of W, as many classes as a piece has
    bool logits = false, grad_in = false, grad_w = false; // products whose operands go straight into LDS
    int64_t ld_w = 0, ld_in = 0;                          // of what the products read
};
// `classes`: those of a piece, which a copy of W holds at a time.  A forward pass reads W for the logits alone.
static XentReads xent_reads(int64_t n, int64_t d, int64_t classes, const void *in, int64_t ld_in, const void *W, int64_t ld_w, bool backward)
{
    XentReads r;
    const int64_t ld_wc = round_up(classes, 8), ld_ic = round_up(d, 8), w_rows = backward ? kTileRows : kTileDepth;
    const bool w = aligned_rows(W, ld_w), x = aligned_rows(in, ld_in) && offsets_fit(kTileRows, ld_in);
    r.copy_w = copies_pay(n) && !(w && offsets_fit(w_rows, ld_w)) && offsets_fit(w_rows, ld_wc);
    r.copy_in = copies_pay(n) && !x && offsets_fit(kTileRows, ld_ic);
    r.ld_w = r.copy_w ? ld_wc : ld_w;
    r.ld_in = r.copy_in ? ld_ic : ld_in;
    r.grad_w = x || r.copy_in;
    // rows of 8 MB and more, forward + input gradient of n x 256 x 5,000,000, us, straight into LDS / through registers: 4 rows 461 + 1,140 / 601 + 1,251, 32 504 + 1,227 / 629 + 1,306,
    // 64 790 + 2,095 / 684 + 1,681, 128 1,003 + 2,252 / 1,132 + 2,817, 511 2,085 + 5,232 / 4,340 + 10,114
    const bool registers = n > 32 && n <= 64 && !offsets_fit(512, r.ld_w);
    r.logits = r.grad_w && (w || r.copy_w) && offsets_fit(kTileDepth, r.ld_w) && !registers;
    r.grad_in = (w || r.copy_w) && offsets_fit(kTileRows, r.ld_w) && !registers;
    return r;
}

template <typename E> __global__ void __launch_bounds__(256) xent_align_kernel(const E *in, int64_t ld, int64_t n, int32_t d, E *out, int64_t ld_out)
{
    const int chunks = static_cast<int>(ld_out / 8);
    const int64_t total = n * chunks;
    for (int64_t q = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; q < total; q += static_cast<int64_t>(gridDim.x) * 256) {
        const int64_t r = q / chunks;
        const int c = static_cast<int>(q - r * chunks) * 8;
        float v[8];
        load8(in + r * ld + c, d - c, v);
        store8(out + r * ld_out + c, 8, v);
    }
}
static unsigned walk(int64_t items) { return static_cast<unsigned>(std::min<int64_t>((items + 255) / 256, 16384)); }

template <typename C> constexpr bool offsets_as_ruled() { return C::LOAD != kDirect || (C::BK <= kTileDepth && C::BM <= kTileRows && C::BN <= kTileRows); }

enum XentTiles { kTilesLarge, kTilesTurned, kTilesSmall, kTilesSkinny, kTilesStaged };
// The tiles of a product: staged where bf16 rows are not aligned, large where they give every second CU one and are not mostly beyond the last row or column.
// Those of the logits: a tile for few rows too.
template <typename E> static XentTiles logit_tiles_for(bool direct, int64_t M, int64_t N)
{
    if (sizeof(E) == 2 && !direct) return kTilesStaged;
    if (sizeof(E) == 2 && M <= 32) return kTilesSkinny;
    return M > 64 && N > 64 && tiles_of(M, N, 256, 256) >= 128 ? kTilesLarge : kTilesSmall;
}
// f(shape)
template <typename T> struct Tag { using type = T; };
template <typename E, bool A_RC, bool B_RC, typename Epi, typename F> static heta_status with_tiles(XentTiles t, F f)
{
    if (t == kTilesStaged) return f(XentShape<E, A_RC, B_RC, false, true>{});
    constexpr bool FORWARD = sizeof(E) == 2 && std::is_same<Epi, XentForwardEpi>::value, BACKWARD = sizeof(E) == 2 && std::is_same<Epi, XentBackwardEpi<bf16_t>>::value;
    if constexpr (FORWARD)
        if (t == kTilesSkinny) return f(Tag<XentSkinnyForwardTiles>{});
    if constexpr (BACKWARD)
        if (t == kTilesSkinny) return f(Tag<XentSkinnyBackwardTiles>{});
    if (t == kTilesSmall) return f(XentShape<E, A_RC, B_RC, false, false>{});
    if constexpr (A_RC && B_RC)
        if (t == kTilesTurned) return f(XentTurned<E>{});
    if constexpr (FORWARD) return f(Tag<XentForwardTiles>{});
    else if constexpr (BACKWARD) return f(Tag<XentBackwardTiles>{});
    else return f(XentShape<E, A_RC, B_RC, true, false>{});
}
template <typename E, bool A_RC, bool B_RC, typename Epi> static heta_status go_tiles(const Launch &l, XentTiles t, const typename Epi::Extra &x)
{
    return with_tiles<E, A_RC, B_RC, Epi>(t, [&](auto shape) {
        using C = typename decltype(shape)::type;
        static_assert(offsets_as_ruled<C>(), "xent_reads() knows tiles of kTileRows and kTileDepth");
        return l.go<C, Epi>(x);
    });
}
// rows and columns of a wavefront's sums
template <typename E, typename Epi> static void strip_of(XentTiles t, int64_t *rows, int64_t *cols)
{
    (void)with_tiles<E, false, true, Epi>(t, [&](auto shape) {
        using C = typename decltype(shape)::type;
        *rows = 32 * C::MI;
        *cols = 32 * C::NJ;
        return HETA_OK;
    });
}

// Sums over the parts of a contraction, after those of earlier pieces (nullable): out[i / width][i % width] for i < total, in a fixed order.
template <typename O> __global__ void __launch_bounds__(256) xent_add_kernel(const float *so_far, const float *part, int splits, int64_t total, O *out, int32_t width, int64_t ld, const float *factor)
{
    const int64_t i = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) * 4;
    if (i >= total) return;
    const int valid = static_cast<int>(min(total - i, static_cast<int64_t>(4)));
    float y[4] = {0.f, 0.f, 0.f, 0.f};
    auto add = [&](const float *p) {
        const uintx4 q = load_piece(p + i, valid);
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] += __uint_as_float(q[e]);
    };
    if (so_far) add(so_far);
#pragma unroll 4
    for (int s = 0; s < splits; ++s) add(part + s * total);
    if (factor) {
        const float f = *factor;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] *= f;
    }
    const int64_t row = i / width;
    int32_t c = static_cast<int32_t>(i - row * width);
    O *to = out + row * ld;
    if (c + 4 <= width && valid == 4) {
        if constexpr (sizeof(O) == 4) store16(to + c, uintx4{__float_as_uint(y[0]), __float_as_uint(y[1]), __float_as_uint(y[2]), __float_as_uint(y[3])});
        else __builtin_memcpy(to + c, (const uint32_t[2]){pack2_bf16(y[0], y[1]), pack2_bf16(y[2], y[3])}, 8);
        return;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (e >= valid) continue;
        if constexpr (sizeof(O) == 4) to[c] = y[e];
        else to[c] = to_bf16(y[e]);
        if (++c == width) {
            c = 0;
            to += ld;
        }
    }
}
// Sums of D's columns over the strips of rows: where there are many, first over `each` of them at a time.  part: [slots][cols], out: [chunks][cols].
__global__ void __launch_bounds__(256) xent_column_sums_kernel(const float *part, int64_t slots, int64_t each, int64_t cols, int64_t column_groups, float *out)
{
    const int64_t chunk = blockIdx.x / column_groups, c = (blockIdx.x - chunk * column_groups) * 256 + threadIdx.x, end = min(slots, (chunk + 1) * each);
    if (c >= cols) return;
    float y = 0.f;
    for (int64_t s = chunk * each; s < end; s += 8) {
        float q[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) q[u] = s + u < end ? part[(s + u) * cols + c] : 0.f;
#pragma unroll
        for (int u = 0; u < 8; ++u) y += q[u];
    }
    out[chunk * cols + c] = y;
}

static heta_status xent_add(const float *so_far, const float *part, int splits, int64_t total, void *out, heta_dtype dt, int32_t width, int64_t ld, const float *factor, hipStream_t st)
{
    const int64_t blocks = (total + 1023) / 1024;
    ProfScope prof("xent_add_kernel", st, static_cast<double>(total) * (4.0 * (splits + !!so_far) + dtype_size(dt)), 0);
    if (dt == HETA_F32) hipLaunchKernelGGL(xent_add_kernel<float>, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, st, so_far, part, splits, total, static_cast<float *>(out), width, ld, factor);
    else hipLaunchKernelGGL(xent_add_kernel<bf16_t>, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, st, so_far, part, splits, total, static_cast<bf16_t *>(out), width, ld, factor);
    HETA_LAUNCH_CHECK("xent_add_kernel");
    return HETA_OK;
}

constexpr int64_t kXentPiece = int64_t(512) << 20; // bytes at a time: of D, and of a forward pass's parts

template <typename E> static heta_status xent_forward(heta_graph *g, const heta_linear_xent_args &a, hipStream_t st)
{
    const char *who = "heta_linear_xent";
    const int64_t n = a.n_rows, d = a.d, V = a.n_classes;
    Regions ws;
    const bool bf16 = sizeof(E) == 2;
    const XentReads reads = bf16 ? xent_reads(n, d, V, a.in, a.ld_in, a.W, a.ld_w, false) : XentReads{};
    const size_t w_at = ws.take(reads.copy_w ? static_cast<size_t>(d) * reads.ld_w * 2 : 0), in_at = ws.take(reads.copy_in ? static_cast<size_t>(n) * reads.ld_in * 2 : 0);
    const size_t target_at = ws.take(static_cast<size_t>(n) * 4);
    const XentTiles tiles = logit_tiles_for<E>(reads.logits, n, V);
    int64_t strip_rows = 0, strip_cols = 0;
    strip_of<E, XentForwardEpi>(tiles, &strip_rows, &strip_cols);
    const int64_t strips = (V + strip_cols - 1) / strip_cols;
    // rows at a time: all of them, or as many as leave kXentPiece bytes of parts
    const int64_t most = std::max<int64_t>(256, kXentPiece / static_cast<int64_t>(sizeof(XentPart)) / strips / 256 * 256), R = std::min(n, most);
    const size_t part_at = ws.take(static_cast<size_t>(strips) * R * sizeof(XentPart));
    // rows of a workgroup: few where there are few rows and many strips; and where there are very many, they are joined in two steps
    const int per_group = strips <= 16 ? 256 : R >= 4096 || strips <= 64 ? 32 : 4;
    const int64_t groups = (n + per_group - 1) / per_group;
    const int64_t each = std::max<int64_t>(256 / per_group * 8, (strips + 1023) / 1024), chunks = per_group == 4 && strips > 2 * each ? (strips + each - 1) / each : 0;
    const size_t joined_at = ws.take(static_cast<size_t>(chunks) * R * sizeof(XentPart));
    const size_t sums_at = ws.take(a.mean && groups > 1 ? static_cast<size_t>(groups) * sizeof(XentSum) : 0);
    HETA_TRY(ensure_workspace(g, ws.bytes));
    char *base = static_cast<char *>(g->d_ws);
    Operand W{a.W, a.ld_w}, in{a.in, a.ld_in};
    if (reads.copy_w) {
        hipLaunchKernelGGL(xent_align_kernel<bf16_t>, dim3(walk(d * reads.ld_w / 8)), dim3(256), 0, st, static_cast<const bf16_t *>(a.W), a.ld_w, d, a.n_classes, reinterpret_cast<bf16_t *>(base + w_at),
                           reads.ld_w);
        W = {base + w_at, reads.ld_w};
    }
    if (reads.copy_in) {
        hipLaunchKernelGGL(xent_align_kernel<bf16_t>, dim3(walk(n * reads.ld_in / 8)), dim3(256), 0, st, static_cast<const bf16_t *>(a.in), a.ld_in, n, a.d, reinterpret_cast<bf16_t *>(base + in_at),
                           reads.ld_in);
        in = {base + in_at, reads.ld_in};
    }
    HETA_LAUNCH_CHECK("xent_align_kernel");
    // Weights that an XCD's L2 does not hold are read by four row blocks at a time (8,192 x 512 x 131,072: 1,250 us one by one, 1,187; eight 1,188, sixteen 1,228).  D's tiles, which
    // write their rows, lose by it (433 us for a quarter of the classes, 474), and so do weights that fit (700,000 x 256 x 349: 231, 238).
    const int32_t group = d * V * static_cast<int64_t>(sizeof(E)) > int64_t(4) << 20 ? 4 : 0;
    XentSum *sums = a.mean && groups > 1 ? reinterpret_cast<XentSum *>(base + sums_at) : nullptr;
    for (int64_t r0 = 0; r0 < n; r0 += R) { // a piece starts at a multiple of 256 rows, and so at a workgroup's first of xent_rows_kernel
        const int64_t rn = std::min(R, n - r0), here = (rn + per_group - 1) / per_group;
        const Launch l{g, who, "xent_kernel", TileItem{static_cast<const E *>(in.p) + r0 * in.ld, W.p, in.ld, W.ld, 0, 0, rn, V, d, d, 1, 0, 0, 0, 0, 0, group},
                       (static_cast<double>(rn) * d + static_cast<double>(d) * V) * sizeof(E), 2.0 * rn * d * V, st};
        const XentForward x{a.bias, a.labels + r0, reinterpret_cast<XentPart *>(base + part_at), reinterpret_cast<float *>(base + target_at) + r0};
        HETA_TRY((go_tiles<E, false, true, XentForwardEpi>(l, tiles, x)));
        const XentPart *parts = x.part;
        int64_t n_parts = strips;
        if (chunks > 0) {
            XentPart *joined = reinterpret_cast<XentPart *>(base + joined_at);
            hipLaunchKernelGGL(xent_join_kernel<4>, dim3(static_cast<unsigned>(chunks * here)), dim3(256), 0, st, x.part, strips, each, rn, here, joined);
            HETA_LAUNCH_CHECK("xent_join_kernel");
            parts = joined;
            n_parts = chunks;
        }
        ProfScope prof("xent_rows_kernel", st, static_cast<double>(rn) * (8.0 * n_parts + 20), 0);
        auto go = [&](auto per) {
            hipLaunchKernelGGL(xent_rows_kernel<decltype(per)::value>, dim3(static_cast<unsigned>(here)), dim3(256), 0, st, parts, n_parts, x.target, x.labels, rn, V,
                               a.loss ? a.loss + r0 : nullptr, a.lse + r0, sums ? sums + r0 / per_group : nullptr, a.mean);
        };
        if (per_group == 256) go(std::integral_constant<int, 256>{});
        else if (per_group == 32) go(std::integral_constant<int, 32>{});
        else go(std::integral_constant<int, 4>{});
        HETA_LAUNCH_CHECK("xent_rows_kernel");
    }
    if (sums) hipLaunchKernelGGL(xent_mean_kernel, dim3(1), dim3(256), 0, st, sums, groups, a.mean);
    HETA_LAUNCH_CHECK("xent_mean_kernel");
    return HETA_OK;
}

// A product whose contraction over K may be split: as many parts as fill the chip once, counted in the tiles that are used (forward and both gradients, us: fp32 5,003 x 300 x 2,983 378
// where 256 x 256 were counted for all and grad_W had 256 x 128 only, 338; 3,000 x 100 x 5,000 187, 163; bf16 700,000 x 256 x 349 1,024, 998; 200,000 x 512 x 100 296, 306).
struct SplitProduct {
    XentTiles tiles;
    int32_t splits;
    int64_t k_each;
};
// bm x bn: the large tiles, `slots` of which the chip holds at a time
template <typename E> static SplitProduct split_product(bool direct, int64_t M, int64_t N, int64_t K, int64_t least, XentTiles large, int bm, int bn, int64_t slots, int32_t at_most)
{
    const int64_t tiles = tiles_of(M, N, bm, bn), most = std::max<int64_t>(1, slots / tiles);
    SplitProduct p;
    p.k_each = round_up(std::max((K + most - 1) / most, least), 64);
    p.splits = static_cast<int32_t>((K + p.k_each - 1) / p.k_each);
    if (p.splits > at_most) {
        p.k_each = round_up((K + at_most - 1) / at_most, 64);
        p.splits = static_cast<int32_t>((K + p.k_each - 1) / p.k_each);
    }
    p.tiles = sizeof(E) == 2 && !direct ? kTilesStaged : M > 64 && N > 64 && tiles * p.splits * 2 >= slots ? large : kTilesSmall;
    return p;
}
template <typename E> static SplitProduct grad_in_product(bool direct, int64_t n, int64_t d, int64_t V, int32_t at_most)
{
    return split_product<E>(direct, n, d, V, 512, kTilesLarge, 256, sizeof(E) == 2 ? 256 : 128, 256, at_most);
}
// 256 x 128 tiles or 128 x 256, whichever have less beyond the result
template <typename E> static SplitProduct grad_w_product(bool direct, int64_t n, int64_t d, int64_t V, int32_t at_most)
{
    const int64_t slots = sizeof(E) == 2 ? 512 : 256;
    if (round_up(d, 128) * round_up(V, 256) < round_up(d, 256) * round_up(V, 128)) return split_product<E>(direct, d, V, n, 256, kTilesTurned, 128, 256, slots, at_most);
    return split_product<E>(direct, d, V, n, 256, kTilesLarge, 256, 128, slots, at_most);
}

// Partial sums that pieces of rows leave, one after another, until there is no room for more (if `bounded`): then they are added up into the first place, in order.
struct Partials {
    float *at; // [most, and one place in front of them if bounded][total]
    int64_t total, most;
    int32_t width; // a divisor of total
    bool bounded;
    float *joined; // [64][total], for sums of many parts of few columns; nullable
    int64_t parts = 0, in_joined = 0;
    bool added = false; // the first place holds a sum
    float *next() const { return at + (bounded + parts) * total; }
    heta_status make_room(int64_t n, hipStream_t st)
    {
        if (parts + n <= most) return HETA_OK;
        HETA_TRY(join(st));
        HETA_TRY(xent_add(nullptr, first(), static_cast<int>(count()), total, at, HETA_F32, width, width, nullptr, st));
        parts = in_joined = 0;
        added = true;
        return HETA_OK;
    }
    // Many parts are first added up 64 ways: 5,469 strips of 349 columns take 27 us in one step, few workgroups of which have columns.
    heta_status join(hipStream_t st)
    {
        if (!joined || count() <= 256) return HETA_OK;
        const int64_t slots = count(), each = (slots + 63) / 64, groups = (total + 255) / 256, chunks = (slots + each - 1) / each;
        hipLaunchKernelGGL(xent_column_sums_kernel, dim3(static_cast<unsigned>(chunks * groups)), dim3(256), 0, st, first(), slots, each, total, groups, joined);
        HETA_LAUNCH_CHECK("xent_column_sums_kernel");
        in_joined = chunks;
        return HETA_OK;
    }
    const float *first() const { return in_joined > 0 ? joined : added ? at : at + bounded * total; }
    int64_t count() const { return in_joined > 0 ? in_joined : parts + added; }
};

// Rows and classes of a piece of D: all of them, or kXentPiece bytes of pieces of one size.
struct PieceOfD {
    int64_t rows, classes;
};
static PieceOfD piece_of_d(int64_t n, int64_t V, size_t elt)
{
    const int64_t room = kXentPiece / static_cast<int64_t>(elt);
    int64_t R = n, Vc = V;
    if (n * round_up(V, 8) > room) {
        const int64_t side = static_cast<int64_t>(std::sqrt(static_cast<double>(room)));
        R = std::min(n, std::max(side, room / round_up(V, 8)));
        R = round_up((n + (n + R - 1) / R - 1) / ((n + R - 1) / R), 256); // pieces of one size
        const int64_t most = std::max<int64_t>(256, room / R);
        Vc = round_up((V + (V + most - 1) / most - 1) / ((V + most - 1) / most), 256);
        R = std::min(R, n);
        Vc = std::min(Vc, V);
    }
    return {R, Vc};
}

template <typename E> static heta_status xent_backward(heta_graph *g, const heta_linear_xent_bwd_args &a, hipStream_t st)
{
    const char *who = "heta_linear_xent_bwd";
    const int64_t n = a.n_rows, d = a.d, V = a.n_classes;
    const bool bf16 = sizeof(E) == 2;
    const heta_dtype dt = bf16 ? HETA_BF16 : HETA_F32;
    const auto [R, Vc] = piece_of_d(n, V, sizeof(E));
    const int64_t n_r = (n + R - 1) / R, n_v = (V + Vc - 1) / Vc;
    // rows of D are not multiples of 1,024 bytes apart (8,192 x 512 x 130,072: 5,760 us at 65,536 bytes, 5,515 with 128 bytes more)
    const int64_t ld_d = round_up(Vc, 8) + (round_up(Vc, 8) * static_cast<int64_t>(sizeof(E)) % 1024 == 0 ? 64 : 0);
    const XentReads reads = bf16 ? xent_reads(n, d, Vc, a.in, a.ld_in, a.W, a.ld_w, true) : XentReads{};
    const int64_t ld_ic = round_up(d, 8);
    const int32_t in_splits = grad_in_product<E>(reads.grad_in, R, d, Vc, INT32_MAX).splits, w_splits = grad_w_product<E>(reads.grad_w, R, d, Vc, INT32_MAX).splits;
    Regions ws;
    const size_t poison_at = ws.take(8), rows_at = ws.take(static_cast<size_t>(n) * sizeof(XentRow));
    const size_t w_at = ws.take(reads.copy_w ? static_cast<size_t>(d) * reads.ld_w * 2 : 0), in_at = ws.take(a.dW || reads.copy_in ? static_cast<size_t>(n) * ld_ic * sizeof(E) : 0);
    const size_t d_at = ws.take(static_cast<size_t>(R) * ld_d * sizeof(E));
    // partial sums of one piece of rows at least, of all of them at most, between these 64 MB of D's columns' and 512 MB of grad_W's
    const int64_t strips = (R + 31) / 32, all_sums = strips * n_r, most_sums = std::min(all_sums, std::max(strips, kXentPiece / 8 / (Vc * 4)));
    const int64_t all_dw = w_splits * n_r, most_dw = std::min(all_dw, std::max<int64_t>(w_splits, kXentPiece / (d * Vc * 4)));
    const size_t sums_at = ws.take(a.dbias ? static_cast<size_t>(most_sums + (most_sums < all_sums)) * Vc * 4 : 0);
    const size_t joined_at = ws.take(a.dbias ? static_cast<size_t>(64) * Vc * 4 : 0);
    const size_t dw_at = ws.take(a.dW && (w_splits > 1 || n_r > 1) ? static_cast<size_t>(most_dw + (most_dw < all_dw)) * d * Vc * 4 : 0);
    // grad_in's sums over the classes so far, and in front of each piece's partial products
    const size_t di_at = ws.take(a.grad_in && (in_splits > 1 || n_v > 1) ? static_cast<size_t>(in_splits + (n_v > 1 ? n_r : 0)) * R * d * 4 : 0);
    if (a.grad_in && (n_v > 1 || in_splits > 1) && R * d > max_blocks(256) * 1024) return fail(HETA_ERR_UNSUPPORTED, "%s: input gradient too large for one launch", who);
    HETA_TRY(ensure_workspace(g, ws.bytes));
    char *base = static_cast<char *>(g->d_ws);
    uint32_t *poison = reinterpret_cast<uint32_t *>(base + poison_at);
    float *factor = reinterpret_cast<float *>(poison) + 1;
    XentRow *rows = reinterpret_cast<XentRow *>(base + rows_at);
    const uint32_t call = ++g->xent_calls;
    E *clean = reinterpret_cast<E *>(base + in_at);
    // few rows: their copy is made at once, and taken whatever they hold (a launch less: 11 x 47 x 3, forward and gradients, 37.7 us for 35.0)
    const bool at_once = (a.dW || reads.copy_in) && n * ld_ic * static_cast<int64_t>(sizeof(E)) <= int64_t(8) << 20;
    {
        ProfScope prof("xent_prepare_kernel", st, 32.0 * n, 0);
        if (at_once && d >= 128)
            hipLaunchKernelGGL((xent_prepare_rows_kernel<E, 64>), dim3(static_cast<unsigned>((n + 3) / 4)), dim3(256), 0, st, a.labels, a.lse, a.grad_loss, a.mean, a.scale, n, V, rows, factor, poison, call,
                               static_cast<const E *>(a.in), a.ld_in, a.d, clean, ld_ic);
        else if (at_once)
            hipLaunchKernelGGL((xent_prepare_rows_kernel<E, 8>), dim3(static_cast<unsigned>((n + 31) / 32)), dim3(256), 0, st, a.labels, a.lse, a.grad_loss, a.mean, a.scale, n, V, rows, factor, poison, call,
                               static_cast<const E *>(a.in), a.ld_in, a.d, clean, ld_ic);
        else
            hipLaunchKernelGGL(xent_prepare_kernel, dim3(static_cast<unsigned>((n + 255) / 256)), dim3(256), 0, st, a.labels, a.lse, a.grad_loss, a.mean, a.scale, n, V, rows, factor, poison, call);
        HETA_LAUNCH_CHECK("xent_prepare_kernel");
    }
    Operand in{a.in, a.ld_in};
    if ((reads.copy_in || a.dW) && !at_once)
        hipLaunchKernelGGL(xent_clean_kernel<E>, dim3(walk(n * ld_ic / 8)), dim3(256), 0, st, static_cast<const E *>(a.in), a.ld_in, n, a.d, rows, clean, ld_ic, reads.copy_in, poison, call);
    if (reads.copy_in) in = {clean, ld_ic};
    HETA_LAUNCH_CHECK("xent_clean_kernel");

    for (int64_t v = 0; v < n_v; ++v) {
        const int64_t v0 = v * Vc, cols = std::min(Vc, V - v0);
        const E *Wv = static_cast<const E *>(a.W) + v0;
        const int64_t ld_w = reads.copy_w ? reads.ld_w : a.ld_w;
        if (reads.copy_w) { // of this piece's classes: rows of any length are short ones here
            bf16_t *const copy = reinterpret_cast<bf16_t *>(base + w_at);
            hipLaunchKernelGGL(xent_align_kernel<bf16_t>, dim3(walk(d * ld_w / 8)), dim3(256), 0, st, reinterpret_cast<const bf16_t *>(Wv), a.ld_w, d, static_cast<int32_t>(cols), copy, ld_w);
            HETA_LAUNCH_CHECK("xent_align_kernel");
            Wv = reinterpret_cast<const E *>(copy);
        }
        Partials sums{reinterpret_cast<float *>(base + sums_at), cols, most_sums, static_cast<int32_t>(cols), most_sums < all_sums, reinterpret_cast<float *>(base + joined_at)};
        Partials dw{reinterpret_cast<float *>(base + dw_at), d * cols, most_dw, static_cast<int32_t>(cols), most_dw < all_dw, nullptr};
        for (int64_t r = 0; r < n_r; ++r) {
            const int64_t r0 = r * R, rn = std::min(R, n - r0);
            const E *in_r = static_cast<const E *>(in.p) + r0 * in.ld;
            const double product = 2.0 * rn * d * cols;
            {
                const Launch l{g, who, "xent_logit_grad_kernel", TileItem{in_r, Wv, in.ld, ld_w, 0, 0, rn, cols, d, d, 1, 0, 0, 0, 0, 0, 0},
                               (static_cast<double>(rn) * (d + cols) + static_cast<double>(d) * cols) * sizeof(E), product, st};
                const XentTiles tiles = logit_tiles_for<E>(reads.logits, rn, cols);
                int64_t strip_rows = 0, strip_cols = 0;
                strip_of<E, XentBackwardEpi<E>>(tiles, &strip_rows, &strip_cols);
                const int64_t strips_here = (rn + strip_rows - 1) / strip_rows;
                const bool single = a.dbias && n_r == 1 && strips_here == 1;
                if (a.dbias && !single) HETA_TRY(sums.make_room(strips_here, st));
                const XentBackward x{a.bias ? a.bias + v0 : nullptr, rows + r0, base + d_at, ld_d, single ? a.dbias + v0 : a.dbias ? sums.next() : nullptr, v0,
                                     single ? factor : nullptr};
                HETA_TRY((go_tiles<E, false, true, XentBackwardEpi<E>>(l, tiles, x)));
                if (a.dbias && !single) sums.parts += strips_here; // none without dbias: nothing is added up below
            }
            if (a.grad_in) {
                const auto [tiles, splits, k_each] = grad_in_product<E>(reads.grad_in, rn, d, cols, in_splits);
                const Launch l{g, who, "xent_grad_in_kernel", TileItem{base + d_at, Wv, ld_d, ld_w, 0, 0, rn, d, cols, k_each, splits, 0, 0, 0, 0, 0},
                               (static_cast<double>(rn) * (d + cols) + static_cast<double>(d) * cols) * sizeof(E), product, st};
                float *so_far = reinterpret_cast<float *>(base + di_at) + (n_v > 1 ? r * R * d : 0), *part = reinterpret_cast<float *>(base + di_at) + (n_v > 1 ? n_r * R * d : 0);
                E *out = static_cast<E *>(a.grad_in) + r0 * a.ld_gi;
                if (splits == 1 && n_v == 1) {
                    HETA_TRY((go_tiles<E, false, false, XentProductEpi<E>>(l, tiles, XentProduct{out, a.ld_gi, factor, nullptr, 0, nullptr, 0})));
                } else {
                    const bool last = v + 1 == n_v;
                    HETA_TRY((go_tiles<E, false, false, XentProductEpi<float>>(l, tiles, XentProduct{part, d, nullptr, nullptr, 0, nullptr, 0})));
                    HETA_TRY(xent_add(v > 0 ? so_far : nullptr, part, splits, rn * d, last ? static_cast<void *>(out) : so_far, last ? dt : HETA_F32, a.d, last ? a.ld_gi : d,
                                      last ? factor : nullptr, st));
                }
            }
            if (a.dW) {
                const auto [tiles, splits, k_each] = grad_w_product<E>(reads.grad_w, rn, d, cols, w_splits);
                // a column's row blocks one after the other, where the contraction is whole: they share its part of D (all gradients of 8,192 x 512 x 131,072: 3,783 us row block by
                // row block, 3,741 this way; of 700,000 x 256 x 349, which is split, the same)
                const Launch l{g, who, "xent_grad_w_kernel", TileItem{in_r, base + d_at, in.ld, ld_d, 0, 0, d, cols, rn, k_each, splits, 0, 0, 0, 0, 0, 64},
                               (static_cast<double>(rn) * (d + cols)) * sizeof(E) + 4.0 * splits * d * cols, product, st};
                XentProduct x{nullptr, cols, nullptr, clean + r0 * ld_ic, ld_ic, poison, call};
                if (splits == 1 && n_r == 1) {
                    x.out = static_cast<char *>(a.dW) + v0 * dtype_size(a.dw_dt);
                    x.ld = a.ld_dw;
                    x.factor = factor;
                    if (a.dw_dt == HETA_F32) HETA_TRY((go_tiles<E, true, true, XentProductEpi<float>>(l, tiles, x)));
                    else HETA_TRY((go_tiles<E, true, true, XentProductEpi<bf16_t>>(l, tiles, x)));
                } else {
                    HETA_TRY(dw.make_room(splits, st));
                    x.out = dw.next();
                    HETA_TRY((go_tiles<E, true, true, XentProductEpi<float>>(l, tiles, x)));
                    dw.parts += splits;
                }
            }
        }
        HETA_TRY(sums.join(st));
        if (sums.count() > 0) HETA_TRY(fold_partials(sums.first(), sums.count(), cols, a.dbias + v0, HETA_F32, static_cast<int32_t>(cols), cols, st, factor));
        if (dw.count() > 0) {
            char *to = static_cast<char *>(a.dW) + v0 * dtype_size(a.dw_dt);
            HETA_TRY(fold_partials(dw.first(), dw.count(), d * cols, to, a.dw_dt, static_cast<int32_t>(cols), a.ld_dw, st, factor));
        }
    }
    return HETA_OK;
}

} // namespace heta

using namespace heta;

extern "C" heta_status heta_linear_xent(heta_graph *g, const heta_linear_xent_args *a, void *hip_stream)
{
    const char *who = "heta_linear_xent";
    if (!g || !a) return fail(HETA_ERR_INVALID_ARG, "%s: null arguments", who);
    if (a->n_rows < 0 || a->d <= 0 || a->n_classes <= 0) return fail(HETA_ERR_SHAPE, "%s: need n_rows >= 0, a width and classes", who);
    if (std::max(a->d, a->n_classes) > kWidest || a->n_rows >= int64_t(1) << 31) return fail(HETA_ERR_UNSUPPORTED, "%s: too many rows, columns or classes", who);
    if (!valid_dtype(a->dt)) return fail(HETA_ERR_INVALID_ARG, "%s: bad dtype", who);
    const size_t esz = dtype_size(a->dt);
    const int64_t n = a->n_rows;
    HETA_TRY(check_rows(who, "in", a->in, n, a->ld_in, a->d, esz));
    HETA_TRY(check_rows(who, "W", a->W, 1, a->ld_w, a->n_classes, esz));
    if (n > 0 && (!a->labels || !a->lse)) return fail(HETA_ERR_INVALID_ARG, "%s: null labels or lse", who);
    if (reinterpret_cast<uintptr_t>(a->labels) & 7u) return fail(HETA_ERR_INVALID_ARG, "%s: pointer not aligned to its element size", who);
    for (const float *v : {a->bias, static_cast<const float *>(a->loss), static_cast<const float *>(a->lse), static_cast<const float *>(a->mean)})
        if (reinterpret_cast<uintptr_t>(v) & 3u) return fail(HETA_ERR_INVALID_ARG, "%s: pointer not aligned to its element size", who);
    const RowRange outs[3] = {RowRange(a->loss, 1, n, n, 4), RowRange(a->lse, 1, n, n, 4), RowRange(a->mean, 1, 2, 2, 4)};
    const RowRange ins[4] = {RowRange(a->in, n, a->ld_in, a->d, esz), RowRange(a->W, a->d, a->ld_w, a->n_classes, esz), RowRange(a->bias, 1, a->n_classes, a->n_classes, 4),
                             RowRange(a->labels, 1, n, n, 8)};
    for (int i = 0; i < 3; ++i) {
        for (int j = 0; j < i; ++j)
            if (outs[i].overlaps(outs[j])) return fail(HETA_ERR_INVALID_ARG, "%s: two outputs overlap", who);
        for (const RowRange &in : ins)
            if (outs[i].overlaps(in)) return fail(HETA_ERR_INVALID_ARG, "%s: an output overlaps an operand", who);
    }
    hipStream_t st = as_stream(hip_stream);
    if (n == 0) {
        if (a->mean) hipLaunchKernelGGL(xent_mean_kernel, dim3(1), dim3(256), 0, st, nullptr, 0, a->mean);
        HETA_LAUNCH_CHECK("xent_mean_kernel");
        return HETA_OK;
    }
    return a->dt == HETA_F32 ? xent_forward<float>(g, *a, st) : xent_forward<bf16_t>(g, *a, st);
}

extern "C" heta_status heta_linear_xent_bwd(heta_graph *g, const heta_linear_xent_bwd_args *a, void *hip_stream)
{
    const char *who = "heta_linear_xent_bwd";
    if (!g || !a) return fail(HETA_ERR_INVALID_ARG, "%s: null arguments", who);
    if (a->n_rows < 0 || a->d <= 0 || a->n_classes <= 0) return fail(HETA_ERR_SHAPE, "%s: need n_rows >= 0, a width and classes", who);
    if (std::max(a->d, a->n_classes) > kWidest || a->n_rows >= int64_t(1) << 31) return fail(HETA_ERR_UNSUPPORTED, "%s: too many rows, columns or classes", who);
    if (!valid_dtype(a->dt) || (a->dW && !valid_dtype(a->dw_dt))) return fail(HETA_ERR_INVALID_ARG, "%s: bad dtype", who);
    if (a->dt == HETA_F32 && a->dW && a->dw_dt != HETA_F32) return fail(HETA_ERR_UNSUPPORTED, "%s: fp32 operands have an fp32 weight gradient", who);
    const size_t esz = dtype_size(a->dt);
    const int64_t n = a->n_rows, V = a->n_classes;
    HETA_TRY(check_rows(who, "in", a->in, n, a->ld_in, a->d, esz));
    HETA_TRY(check_rows(who, "W", a->W, 1, a->ld_w, V, esz));
    if (a->grad_in) HETA_TRY(check_rows(who, "grad_in", a->grad_in, n, a->ld_gi, a->d, esz));
    if (a->dW) HETA_TRY(check_rows(who, "dW", a->dW, 1, a->ld_dw, V, dtype_size(a->dw_dt)));
    if (n > 0 && (!a->labels || !a->lse)) return fail(HETA_ERR_INVALID_ARG, "%s: null labels or lse", who);
    if (reinterpret_cast<uintptr_t>(a->labels) & 7u) return fail(HETA_ERR_INVALID_ARG, "%s: pointer not aligned to its element size", who);
    for (const float *v : {a->bias, a->lse, a->grad_loss, a->mean, static_cast<const float *>(a->dbias)})
        if (reinterpret_cast<uintptr_t>(v) & 3u) return fail(HETA_ERR_INVALID_ARG, "%s: pointer not aligned to its element size", who);
    if (a->dW && static_cast<int64_t>(a->d) * V > kFoldMost) return fail(HETA_ERR_UNSUPPORTED, "%s: weight gradient of too many elements", who);
    const RowRange outs[3] = {RowRange(a->grad_in, n, a->ld_gi, a->d, esz), RowRange(a->dW, a->d, a->ld_dw, V, a->dW ? dtype_size(a->dw_dt) : 4), RowRange(a->dbias, 1, V, V, 4)};
    const RowRange ins[7] = {RowRange(a->in, n, a->ld_in, a->d, esz), RowRange(a->W, a->d, a->ld_w, V, esz), RowRange(a->bias, 1, V, V, 4), RowRange(a->labels, 1, n, n, 8),
                             RowRange(a->lse, 1, n, n, 4), RowRange(a->grad_loss, 1, n, n, 4), RowRange(a->mean, 1, 2, 2, 4)};
    for (int i = 0; i < 3; ++i) {
        for (int j = 0; j < i; ++j)
            if (outs[i].overlaps(outs[j])) return fail(HETA_ERR_INVALID_ARG, "%s: two outputs overlap", who);
        for (const RowRange &in : ins)
            if (outs[i].overlaps(in)) return fail(HETA_ERR_INVALID_ARG, "%s: an output overlaps an operand", who);
    }
    hipStream_t st = as_stream(hip_stream);
    if (n == 0) {
        if (a->dbias) HETA_TRY(fold_partials(nullptr, 0, V, a->dbias, HETA_F32, a->n_classes, V, st));
        if (a->dW) HETA_TRY(fold_partials(nullptr, 0, a->d * V, a->dW, a->dw_dt, a->n_classes, a->ld_dw, st));
        return HETA_OK;
    }
    if (!a->grad_in && !a->dW && !a->dbias) return HETA_OK;
    return a->dt == HETA_F32 ? xent_backward<float>(g, *a, st) : xent_backward<bf16_t>(g, *a, st);
}

extern "C" heta_status heta_xent_reads(const heta_linear_xent_bwd_args *a, int32_t backward, int64_t *out)
{
    if (!a || !out) return fail(HETA_ERR_INVALID_ARG, "heta_xent_reads: null arguments");
    const int64_t classes = backward ? piece_of_d(a->n_rows, a->n_classes, 2).classes : a->n_classes;
    const XentReads r = xent_reads(a->n_rows, a->d, classes, a->in, a->ld_in, a->W, a->ld_w, backward != 0);
    // bytes from the first row to behind the last one of a tile of so many, `there` of which exist
    auto reach = [](bool direct, int64_t rows, int64_t there, int64_t ld) { return direct ? std::min(rows, there) * ld * 2 : 0; };
    out[0] = r.copy_w;
    out[1] = r.copy_in;
    out[2] = r.logits;
    out[3] = backward ? r.grad_in : 0;
    out[4] = backward ? r.grad_w : 0;
    out[5] = classes;
    out[6] = std::max(reach(r.logits, kTileDepth, a->d, r.ld_w), reach(out[3] != 0, kTileRows, a->d, r.ld_w));
    out[7] = std::max(reach(r.logits, kTileRows, a->n_rows, r.ld_in), reach(out[4] != 0, kTileDepth, a->n_rows, r.ld_in));
    return HETA_OK;
}
