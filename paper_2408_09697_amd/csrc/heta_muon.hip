// Orthogonalised momentum (Muon: Jordan et al. 2024) for the weight matrices of a model, all of them in one call.
//
//     m <- mu m + g,   u = g + mu m (Nesterov) or m,   X_0 = u / (|u|_F + eps)
//     X <- a X + (b A + c A A) X,  A = X X^T   (steps times; a quintic that drives every singular value towards 1)
//     W <- (1 - lr wd) W - lr sqrt(max(1, cols / rows)) X
//
// The matrices [rows, cols] are those of a product in . W.  X lies with its shorter side k as rows (a tall matrix is
// transposed on its way in and out, by the element-wise kernels), so a step is three products for every item: k x k Gram
// matrix, k x k polynomial, k x l update.  They are the tile kernel of heta_tiles.h on the bf16 matrix pipe with every
// matrix held as bf16 terms, three for fp32 weights (24 bits, the rounding of fp32: a state of 32 bits or more), two for
// bf16 weights (16 bits: the update is lr times X and the weight it is subtracted from keeps 8); the epilogue that makes
// a matrix writes it as terms, so that the next product loads them straight into LDS.
// |u| is summed per 64 x 64 tile, then over the tiles in a fixed order by every workgroup that needs it.
#include <algorithm>
#include <cmath>

#include "heta_rows.h"
#include "heta_tiles.h"

namespace heta {

constexpr int kMuonItems = 12; // per launch
constexpr float kNsA = 3.4445f, kNsB = -4.7750f, kNsC = 2.0315f;

struct MuonItem {
    void *W;
    float *m;
    const void *grad;
    int64_t ld_w, ld_m, ld_grad;
    int32_t rows, cols;
    int32_t tall;      // rows > cols: X is the transpose
    int32_t grad_bf16;
    bf16_t *x;         // terms of X
    int64_t ld_x, plane; // elements
    float *part;       // sums of squares, one per tile
    uint32_t block0, tiles;
};
struct MuonArgs {
    int n;
    float mu, keep, step_size, eps; // keep = 1 - lr wd, step_size = lr
    int nesterov;
    MuonItem item[kMuonItems];
};
static_assert(sizeof(MuonArgs) <= 3584, "kernel arguments are limited to 4 KB");

__device__ __forceinline__ int muon_item(const MuonArgs &p)
{
    int i = 0;
    while (i + 1 < p.n && blockIdx.x >= p.item[i + 1].block0) ++i;
    return i;
}
__device__ __forceinline__ float muon_grad(const MuonItem &it, int64_t r, int64_t c)
{
    return it.grad_bf16 ? widen(static_cast<const bf16_t *>(it.grad)[r * it.ld_grad + c]) : static_cast<const float *>(it.grad)[r * it.ld_grad + c];
}

// One workgroup per 64 x 64 tile: momentum, and the sum of squares of u.
__global__ void __launch_bounds__(256) muon_momentum_kernel(MuonArgs p)
{
    __shared__ float sums[4];
    const MuonItem &it = p.item[muon_item(p)];
    const uint32_t b = blockIdx.x - it.block0, tc = (it.cols + 63) / 64;
    const int64_t r0 = static_cast<int64_t>(b / tc) * 64, c = static_cast<int64_t>(b % tc) * 64 + (threadIdx.x & 63);
    float ss = 0.f;
    if (c < it.cols) {
#pragma unroll 4
        for (int64_t r = r0 + (threadIdx.x >> 6); r < min(r0 + 64, static_cast<int64_t>(it.rows)); r += 4) {
            const float g = muon_grad(it, r, c);
            const float m = fmaf(p.mu, it.m[r * it.ld_m + c], g);
            it.m[r * it.ld_m + c] = m;
            const float u = p.nesterov ? fmaf(p.mu, m, g) : m;
            ss += u * u;
        }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) ss += __shfl_xor(ss, o);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = ss;
    __syncthreads();
    if (threadIdx.x == 0) it.part[b] = (sums[0] + sums[1]) + (sums[2] + sums[3]);
}

template <int T> __device__ __forceinline__ void store_terms(bf16_t *p, int64_t plane, float v)
{
#pragma unroll
    for (int t = 0; t < T; ++t) {
        const bf16_t h = to_bf16(v);
        p[t * plane] = h;
        v -= widen(h);
    }
}

// X_0 as terms; a tall matrix goes through LDS so that both its reads and its writes are along rows.
template <int T> __global__ void __launch_bounds__(256) muon_start_kernel(MuonArgs p)
{
    __shared__ float tile[64][65];
    __shared__ float sums[4];
    const MuonItem &it = p.item[muon_item(p)];
    float ss = 0.f;
    for (uint32_t i = threadIdx.x; i < it.tiles; i += 256) ss += it.part[i];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) ss += __shfl_xor(ss, o);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = ss;
    __syncthreads();
    const float inv = 1.f / (sqrtf((sums[0] + sums[1]) + (sums[2] + sums[3])) + p.eps);
    const uint32_t b = blockIdx.x - it.block0, tc = (it.cols + 63) / 64;
    const int64_t r0 = static_cast<int64_t>(b / tc) * 64, c0 = static_cast<int64_t>(b % tc) * 64;
    const int lx = threadIdx.x & 63, ly = threadIdx.x >> 6;
#pragma unroll 4
    for (int i = ly; i < 64; i += 4) {
        const int64_t r = r0 + i, c = c0 + lx;
        if (r >= it.rows || c >= it.cols) continue;
        const float m = it.m[r * it.ld_m + c];
        const float x = (p.nesterov ? fmaf(p.mu, m, muon_grad(it, r, c)) : m) * inv;
        if (it.tall) tile[i][lx] = x;
        else store_terms<T>(it.x + r * it.ld_x + c, it.plane, x);
    }
    if (!it.tall) return; // uniform
    __syncthreads();
#pragma unroll 4
    for (int i = ly; i < 64; i += 4)
        if (c0 + i < it.cols && r0 + lx < it.rows) store_terms<T>(it.x + (c0 + i) * it.ld_x + r0 + lx, it.plane, tile[lx][i]);
}

// W <- keep W - step X
template <int T, typename E> __global__ void __launch_bounds__(256) muon_update_kernel(MuonArgs p)
{
    __shared__ float tile[64][65];
    const MuonItem &it = p.item[muon_item(p)];
    const uint32_t b = blockIdx.x - it.block0, tc = (it.cols + 63) / 64;
    const int64_t r0 = static_cast<int64_t>(b / tc) * 64, c0 = static_cast<int64_t>(b % tc) * 64;
    const int lx = threadIdx.x & 63, ly = threadIdx.x >> 6;
    auto value = [&](int64_t at) {
        float v = widen(it.x[at]);
#pragma unroll
        for (int t = 1; t < T; ++t) v += widen(it.x[at + t * it.plane]);
        return v;
    };
    if (it.tall) {
#pragma unroll 4
        for (int i = ly; i < 64; i += 4)
            if (c0 + i < it.cols && r0 + lx < it.rows) tile[lx][i] = value((c0 + i) * it.ld_x + r0 + lx);
        __syncthreads();
    }
    const float step = p.step_size * sqrtf(fmaxf(1.f, static_cast<float>(it.cols) / static_cast<float>(it.rows)));
    E *W = static_cast<E *>(it.W);
#pragma unroll 4
    for (int i = ly; i < 64; i += 4) {
        const int64_t r = r0 + i, c = c0 + lx;
        if (r >= it.rows || c >= it.cols) continue;
        const float x = it.tall ? tile[i][lx] : value(r * it.ld_x + c);
        const float w = fmaf(-step, x, p.keep * widen(W[r * it.ld_w + c]));
        if constexpr (sizeof(E) == 2) W[r * it.ld_w + c] = to_bf16(w);
        else W[r * it.ld_w + c] = w;
    }
}

// out = beta old + alpha A B, as terms
struct TermsExtra {
    const bf16_t *old; // nullable
    bf16_t *out;
    int64_t ld_old, old_plane, ld_out, out_plane; // elements
};
template <int T> struct TermsEpi {
    static constexpr int kItems = kMuonItems;
    static constexpr bool kStrip = false;
    using Out = bf16_t;
    struct Extra : TermsExtra {
        float alpha, beta;
    };
    __device__ __forceinline__ static void put(const Extra &x, const TileItem &, int64_t m, int64_t n, int valid, const float (&v)[8], int)
    {
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = x.alpha * v[e];
        if (x.old) {
            float o[8], s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int t = T - 1; t >= 0; --t) { // smallest first
                load8(x.old + t * x.old_plane + m * x.ld_old + n, valid, true, o);
#pragma unroll
                for (int e = 0; e < 8; ++e) s[e] += o[e];
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = fmaf(x.beta, s[e], y[e]);
        }
#pragma unroll
        for (int t = 0; t < T; ++t) {
            uint32_t w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                w[j] = pack2_bf16(y[2 * j], y[2 * j + 1]);
                y[2 * j] -= __uint_as_float(w[j] << 16);
                y[2 * j + 1] -= __uint_as_float(w[j] & 0xffff0000u);
            }
            bf16_t *to = x.out + t * x.out_plane + m * x.ld_out + n;
            if (valid >= 8) {
                *reinterpret_cast<uint4 *>(to) = make_uint4(w[0], w[1], w[2], w[3]);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (e < valid) to[e] = static_cast<bf16_t>(w[e / 2] >> (16 * (e & 1)));
            }
        }
    }
};

// ---- host side ---------------------------------------------------------------------------------------
template <int T, bool B_RC> using NsSmall = TileShape<bf16_t, 2, T, false, B_RC, kDirect, 2, 2, 1, 1, 32, 3, 2>;
template <int T, bool B_RC> using NsLarge = TileShape<bf16_t, 2, T, false, B_RC, kDirect, 2, 2, 2, 2, 32, 2, 1>;

template <int T, bool B_RC> static heta_status launch_terms(const char *who, TileArgs<TermsEpi<T>> &p, hipStream_t st)
{
    double bytes = 0, flops = 0;
    int64_t tiles = 0;
    for (int i = 0; i < p.n_items; ++i) {
        const TileItem &it = p.item[i];
        bytes += 2.0 * T * (static_cast<double>(it.M) * it.K + static_cast<double>(it.K) * it.N + static_cast<double>(it.M) * it.N);
        flops += 2.0 * it.M * it.N * it.K;
        tiles += (it.M + 127) / 128 * ((it.N + 127) / 128);
    }
    if (tiles >= 256) return launch_tiles<NsLarge<T, B_RC>>(who, "muon_product_kernel", p, bytes, flops, st);
    return launch_tiles<NsSmall<T, B_RC>>(who, "muon_product_kernel", p, bytes, flops, st);
}

static int64_t pad8(int64_t n) { return (n + 7) / 8 * 8; }
struct MuonPlan { // places in the workspace, in bytes, of one item
    int64_t k, l, tiles;
    int64_t ld_x, ld_g, x_plane, g_plane; // elements
    int64_t x[2], gram, poly, part, end;
    MuonPlan(int32_t rows, int32_t cols, int terms, int64_t at)
        : k(std::min(rows, cols)), l(std::max(rows, cols)), tiles(int64_t((rows + 63) / 64) * ((cols + 63) / 64)), ld_x(pad8(l)), ld_g(pad8(k)), x_plane(k * ld_x), g_plane(k * ld_g)
    {
        auto take = [&](int64_t bytes) {
            const int64_t p = at;
            at += (bytes + 255) / 256 * 256;
            return p;
        };
        x[0] = take(x_plane * terms * 2);
        x[1] = take(x_plane * terms * 2);
        gram = take(g_plane * terms * 2);
        poly = take(g_plane * terms * 2);
        part = take(tiles * 4);
        end = at;
    }
};

template <int T, typename E>
static heta_status muon_group(const char *who, heta_graph *g, const std::vector<const heta_muon_item *> &items, float lr, float mu, int nesterov, float wd, float eps, int steps,
                              hipStream_t st)
{
    int64_t at = 0;
    std::vector<MuonPlan> plan;
    for (const heta_muon_item *it : items) {
        plan.emplace_back(it->rows, it->cols, T, at);
        at = plan.back().end;
    }
    HETA_TRY(ensure_workspace(g, static_cast<size_t>(at)));
    char *ws = static_cast<char *>(g->d_ws);
    const int n = static_cast<int>(items.size());
    MuonArgs a{};
    a.n = n;
    a.mu = mu;
    a.keep = static_cast<float>(1.0 - static_cast<double>(lr) * wd);
    a.step_size = lr;
    a.eps = eps;
    a.nesterov = nesterov;
    int64_t blocks = 0;
    double elems = 0, esz = 0;
    for (int i = 0; i < n; ++i) {
        const heta_muon_item &q = *items[i];
        const MuonPlan &pl = plan[i];
        a.item[i] = MuonItem{q.W, q.m, q.grad, q.ld_w, q.ld_m, q.ld_grad, q.rows, q.cols, q.rows > q.cols, q.grad_dt == HETA_BF16, reinterpret_cast<bf16_t *>(ws + pl.x[0]), pl.ld_x,
                             pl.x_plane, reinterpret_cast<float *>(ws + pl.part), static_cast<uint32_t>(blocks), static_cast<uint32_t>(pl.tiles)};
        blocks += pl.tiles;
        elems += static_cast<double>(q.rows) * q.cols;
        esz = static_cast<double>(dtype_size(q.grad_dt));
        if (blocks > max_blocks(256)) return fail(HETA_ERR_UNSUPPORTED, "%s: too many elements for one launch", who);
    }
    const dim3 grid(static_cast<unsigned>(blocks));
    {
        ProfScope prof("muon_momentum_kernel", st, elems * (8 + esz), 0);
        hipLaunchKernelGGL(muon_momentum_kernel, grid, dim3(256), 0, st, a);
        HETA_LAUNCH_CHECK("muon_momentum_kernel");
    }
    {
        ProfScope prof("muon_start_kernel", st, elems * (4 + esz + 2 * T), 0);
        hipLaunchKernelGGL(muon_start_kernel<T>, grid, dim3(256), 0, st, a);
        HETA_LAUNCH_CHECK("muon_start_kernel");
    }
    for (int s = 0; s < steps; ++s) {
        TileArgs<TermsEpi<T>> gram{}, poly{}, apply{};
        gram.n_items = poly.n_items = apply.n_items = n;
        for (int i = 0; i < n; ++i) {
            const MuonPlan &pl = plan[i];
            char *x = ws + pl.x[s & 1], *y = ws + pl.x[(s & 1) ^ 1], *A = ws + pl.gram, *P = ws + pl.poly;
            auto terms = [](char *p) { return reinterpret_cast<bf16_t *>(p); };
            gram.item[i] = TileItem{x, x, pl.ld_x, pl.ld_x, pl.x_plane * 2, pl.x_plane * 2, pl.k, pl.k, pl.l, pl.l, 1, 0, 0, 0, 0};
            poly.item[i] = TileItem{A, A, pl.ld_g, pl.ld_g, pl.g_plane * 2, pl.g_plane * 2, pl.k, pl.k, pl.k, pl.k, 1, 0, 0, 0, 0};
            apply.item[i] = TileItem{P, x, pl.ld_g, pl.ld_x, pl.g_plane * 2, pl.x_plane * 2, pl.k, pl.l, pl.k, pl.k, 1, 0, 0, 0, 0};
            gram.extra[i] = {{nullptr, terms(A), 0, 0, pl.ld_g, pl.g_plane}, 1.f, 0.f};
            poly.extra[i] = {{terms(A), terms(P), pl.ld_g, pl.g_plane, pl.ld_g, pl.g_plane}, kNsC, kNsB};
            apply.extra[i] = {{terms(x), terms(y), pl.ld_x, pl.x_plane, pl.ld_x, pl.x_plane}, 1.f, kNsA};
        }
        HETA_TRY((launch_terms<T, false>(who, gram, st)));
        HETA_TRY((launch_terms<T, false>(who, poly, st)));
        HETA_TRY((launch_terms<T, true>(who, apply, st)));
    }
    for (int i = 0; i < n; ++i) a.item[i].x = reinterpret_cast<bf16_t *>(ws + plan[i].x[steps & 1]);
    ProfScope prof("muon_update_kernel", st, elems * (2 * T + 2 * sizeof(E)), 0);
    hipLaunchKernelGGL((muon_update_kernel<T, E>), grid, dim3(256), 0, st, a);
    HETA_LAUNCH_CHECK("muon_update_kernel");
    return HETA_OK;
}

} // namespace heta

using namespace heta;

extern "C" heta_status heta_muon_multi(heta_graph *g, int32_t n_items, const heta_muon_item *items, float lr, float momentum, int32_t nesterov, float weight_decay, float eps,
                                       int32_t steps, void *hip_stream)
{
    const char *who = "heta_muon_multi";
    if (!g || n_items < 0 || (n_items > 0 && !items)) return fail(HETA_ERR_INVALID_ARG, "%s: bad handle or item list", who);
    if (!(momentum >= 0.f && momentum < 1.f) || !(eps > 0.f) || steps < 0 || steps > 64 || !(weight_decay >= 0.f) || !std::isfinite(lr))
        return fail(HETA_ERR_INVALID_ARG, "%s: need 0 <= momentum < 1, eps > 0, weight_decay >= 0, 0 <= steps <= 64 and a finite lr", who);
    std::vector<ItemRange> outs, ins;
    for (int32_t i = 0; i < n_items; ++i) {
        const heta_muon_item &q = items[i];
        if (!valid_dtype(q.dt) || !valid_dtype(q.grad_dt)) return fail(HETA_ERR_INVALID_ARG, "%s: item %d: bad dtype", who, i);
        if (q.rows <= 0 || q.cols <= 0 || q.ld_w < q.cols || q.ld_m < q.cols || q.ld_grad < q.cols)
            return fail(HETA_ERR_SHAPE, "%s: item %d: need 0 < cols <= every leading dimension and rows > 0", who, i);
        if (!q.W || !q.m || !q.grad) return fail(HETA_ERR_INVALID_ARG, "%s: item %d: null pointer", who, i);
        const size_t esz = dtype_size(q.dt), gsz = dtype_size(q.grad_dt);
        if (reinterpret_cast<uintptr_t>(q.W) % esz || reinterpret_cast<uintptr_t>(q.m) % 4 || reinterpret_cast<uintptr_t>(q.grad) % gsz)
            return fail(HETA_ERR_INVALID_ARG, "%s: item %d: pointer not aligned to its element size", who, i);
        if (static_cast<int64_t>((q.rows + 63) / 64) * ((q.cols + 63) / 64) > (1 << 22)) return fail(HETA_ERR_UNSUPPORTED, "%s: item %d: matrix too large", who, i);
        const RowRange w(q.W, q.rows, q.ld_w, q.cols, esz), m(q.m, q.rows, q.ld_m, q.cols, 4), gr(q.grad, q.rows, q.ld_grad, q.cols, gsz);
        if (gr.overlaps(w) || gr.overlaps(m)) return fail(HETA_ERR_INVALID_ARG, "%s: item %d: the gradient overlaps an output", who, i);
        outs.emplace_back(i, w);
        outs.emplace_back(i, m);
        ins.emplace_back(i, gr);
    }
    if (items_collide(outs, ins)) return fail(HETA_ERR_INVALID_ARG, "%s: an output overlaps another item's arrays", who);
    hipStream_t st = as_stream(hip_stream);
    for (const heta_dtype dt : {HETA_F32, HETA_BF16}) {
        std::vector<const heta_muon_item *> some;
        for (int32_t i = 0; i <= n_items; ++i) {
            if (i < n_items && items[i].dt == dt) some.push_back(&items[i]);
            if (some.empty() || (i < n_items && some.size() < static_cast<size_t>(kMuonItems))) continue;
            HETA_TRY((dt == HETA_F32 ? muon_group<3, float>(who, g, some, lr, momentum, nesterov != 0, weight_decay, eps, steps, st)
                                     : muon_group<2, bf16_t>(who, g, some, lr, momentum, nesterov != 0, weight_decay, eps, steps, st)));
            some.clear();
        }
    }
    return HETA_OK;
}
