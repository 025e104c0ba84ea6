// Orthogonalised momentum (Muon: Jordan et al. 2024) for the weight matrices of a model, all of them in one call.
//
//     m <- mu m + g,   u = g + mu m (Nesterov) or m,   X_0 = u / (|u|_F + eps)
//     X <- a X + (b A + c A A) X,  A = X X^T   (steps times; a quintic that drives every singular value towards 1)
//     W <- (1 - lr wd) W - lr sqrt(max(1, cols / rows)) X
//
// The matrices [rows, cols] are those of a product in . W.  X lies with its shorter side k as rows (a tall matrix is
// transposed on its way in and out, by the element-wise kernels), so a step is three products for every item: k x k Gram
// matrix, k x k polynomial, k x l update.  They are the tile kernel of heta_tiles.h on the bf16 matrix pipe with every
// matrix held as bf16 terms, three for fp32 weights and two for bf16 ones; the epilogue that makes a matrix writes it as terms, so that
// the next product loads them straight into LDS.  Gram matrix and polynomial are symmetric: only the tiles on and above the diagonal are formed.
// |u| is summed per part of 32 x 64, then over the parts in a fixed order by every workgroup that needs it.
#include <algorithm>
#include <cmath>
#include <new>

#include "heta_tiles.h"

namespace heta {

constexpr int kMuonItems = 12; // per launch
// T, bf16 terms of a matrix.  Three hold fp32 (the update misses the one of exact products by 2.3e-7 of its norm), two 16 bits (2.5e-5) at half
// the products: enough for weights that are rounded to 8 bits behind the update, 2^-9 of their own, and for a caller who asks for it.
// One: 1.3e-2.
static int muon_terms(int dt, int flags) { return dt == HETA_F32 && !(flags & HETA_MUON_COARSE) ? 3 : 2; }
constexpr float kNsA = 3.4445f, kNsB = -4.7750f, kNsC = 2.0315f;

struct MuonItem {
    void *W;
    float *m;
    const void *grad;
    int64_t ld_w, ld_m, ld_grad;
    int32_t rows, cols;
    int32_t tall;      // rows > cols: X is the transpose
    int32_t grad_bf16, w_bf16;
    bf16_t *x;         // terms of X
    int64_t ld_x, plane; // elements
    float *part;       // sums of squares, one per part
    uint32_t block0, parts; // first workgroup and number of its 32 x 64 parts
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

// Momentum, and the sum of squares of u: one workgroup per part of 32 x 64.  Every load comes before the first store: a
// small matrix has one workgroup's latency to wait for.
__global__ void __launch_bounds__(256) muon_momentum_kernel(MuonArgs p)
{
    __shared__ float sums[4];
    const MuonItem &it = p.item[muon_item(p)];
    const uint32_t b = blockIdx.x - it.block0, tc = (it.cols + 63) / 64;
    const int lx = threadIdx.x & 63, ly = threadIdx.x >> 6;
    const int64_t r0 = static_cast<int64_t>(b / tc) * 32 + ly, c = static_cast<int64_t>(b % tc) * 64 + lx;
    float g[8], m[8], ss = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int64_t r = r0 + 4 * i;
        const bool in = r < it.rows && c < it.cols;
        g[i] = in ? muon_grad(it, r, c) : 0.f;
        m[i] = in ? it.m[r * it.ld_m + c] : 0.f;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int64_t r = r0 + 4 * i;
        m[i] = fmaf(p.mu, m[i], g[i]);
        const float u = p.nesterov ? fmaf(p.mu, m[i], g[i]) : m[i];
        ss += u * u;
        if (r < it.rows && c < it.cols) it.m[r * it.ld_m + c] = m[i];
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) ss += __shfl_xor(ss, o);
    if (lx == 0) sums[ly] = ss;
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

// X_0 as terms; a tall matrix goes through LDS so that both its reads and its writes are along
// rows.  The sums of squares come in while the part does.
template <int T> __global__ void __launch_bounds__(256) muon_start_kernel(MuonArgs p)
{
    __shared__ float tile[32][65];
    __shared__ float sums[4];
    const MuonItem &it = p.item[muon_item(p)];
    const uint32_t b = blockIdx.x - it.block0, tc = (it.cols + 63) / 64;
    const int64_t r0 = static_cast<int64_t>(b / tc) * 32, c0 = static_cast<int64_t>(b % tc) * 64;
    const int lx = threadIdx.x & 63, ly = threadIdx.x >> 6;
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int64_t r = r0 + 4 * i + ly, c = c0 + lx;
        x[i] = 0.f;
        if (r < it.rows && c < it.cols) {
            x[i] = it.m[r * it.ld_m + c];
            if (p.nesterov) x[i] = fmaf(p.mu, x[i], muon_grad(it, r, c));
        }
    }
    float ss = 0.f;
    for (uint32_t i = threadIdx.x; i < it.parts; i += 256) ss += it.part[i];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) ss += __shfl_xor(ss, o);
    if (lx == 0) sums[ly] = ss;
    __syncthreads();
    const float inv = 1.f / (sqrtf((sums[0] + sums[1]) + (sums[2] + sums[3])) + p.eps);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int64_t r = r0 + 4 * i + ly, c = c0 + lx;
        if (it.tall) tile[4 * i + ly][lx] = x[i] * inv;
        else if (r < it.rows && c < it.cols) store_terms<T>(it.x + r * it.ld_x + c, it.plane, x[i] * inv);
    }
    if (!it.tall) return; // uniform
    __syncthreads();
    const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (c0 + 8 * i + ty < it.cols && r0 + tx < it.rows) store_terms<T>(it.x + (c0 + 8 * i + ty) * it.ld_x + r0 + tx, it.plane, tile[tx][8 * i + ty]);
}

// W <- keep W - step X
template <int T> __global__ void __launch_bounds__(256) muon_update_kernel(MuonArgs p)
{
    __shared__ float tile[32][65];
    const MuonItem &it = p.item[muon_item(p)];
    const uint32_t b = blockIdx.x - it.block0, tc = (it.cols + 63) / 64;
    const int64_t r0 = static_cast<int64_t>(b / tc) * 32, c0 = static_cast<int64_t>(b % tc) * 64;
    const int lx = threadIdx.x & 63, ly = threadIdx.x >> 6, tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
    auto value = [&](int64_t at) {
        float v = widen(it.x[at]);
#pragma unroll
        for (int t = 1; t < T; ++t) v += widen(it.x[at + t * it.plane]);
        return v;
    };
    float w[8], x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int64_t r = r0 + 4 * i + ly, c = c0 + lx, at = r * it.ld_w + c;
        const bool in = r < it.rows && c < it.cols;
        w[i] = in ? (it.w_bf16 ? widen(static_cast<const bf16_t *>(it.W)[at]) : static_cast<const float *>(it.W)[at]) : 0.f;
        if (it.tall) x[i] = c0 + 8 * i + ty < it.cols && r0 + tx < it.rows ? value((c0 + 8 * i + ty) * it.ld_x + r0 + tx) : 0.f;
        else x[i] = in ? value(r * it.ld_x + c) : 0.f;
    }
    if (it.tall) { // uniform
#pragma unroll
        for (int i = 0; i < 8; ++i) tile[tx][8 * i + ty] = x[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = tile[4 * i + ly][lx];
    }
    const float step = p.step_size * sqrtf(fmaxf(1.f, static_cast<float>(it.cols) / static_cast<float>(it.rows)));
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int64_t r = r0 + 4 * i + ly, c = c0 + lx, at = r * it.ld_w + c;
        if (r >= it.rows || c >= it.cols) continue;
        const float v = fmaf(-step, x[i], p.keep * w[i]);
        if (it.w_bf16) static_cast<bf16_t *>(it.W)[at] = to_bf16(v);
        else static_cast<float *>(it.W)[at] = v;
    }
}

// out = beta old + alpha A B, as terms.  A symmetric product's tiles beside the diagonal are written twice, the second time
// with rows and columns exchanged.
struct TermsExtra {
    const bf16_t *old; // nullable
    bf16_t *out;
    int64_t ld_old, old_plane, ld_out, out_plane; // elements
    float alpha, beta;
};
template <int T> struct TermsEpi {
    static constexpr int kItems = kMuonItems;
    static constexpr bool kBlocks = true;
    using Extra = TermsExtra;
    // eight results of row r, columns c, c + 1, ... (valid of them there; rows of the terms are 16-byte aligned)
    __device__ __forceinline__ static void put(const Extra &x, int64_t r, int64_t c, int valid, float (&y)[8])
    {
#pragma unroll
        for (int t = 0; t < T; ++t) {
            uint32_t w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                w[j] = pack2_bf16(y[2 * j], y[2 * j + 1]);
                y[2 * j] -= __uint_as_float(w[j] << 16);
                y[2 * j + 1] -= __uint_as_float(w[j] & 0xffff0000u);
            }
            bf16_t *to = x.out + t * x.out_plane + r * x.ld_out + c;
            if (valid >= 8) {
                *reinterpret_cast<uint4 *>(to) = make_uint4(w[0], w[1], w[2], w[3]);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (e < valid) to[e] = static_cast<bf16_t>(w[e / 2] >> (16 * (e & 1)));
            }
        }
    }
    __device__ __forceinline__ static void block(const Extra &x, const TileItem &it, float *strip, int64_t m0, int64_t n0, bool off_diagonal, int lane)
    {
        const int sr = lane / 4, sc = lane % 4;
        const bool mirror = it.symmetric && off_diagonal;
        const int64_t n = n0 + 8 * sc;
        const int valid = static_cast<int>(min(it.N - n, static_cast<int64_t>(8)));
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int row = 16 * h + sr;
            const int64_t m = m0 + row;
            const float4 lo = *strip_at(strip, row, 2 * sc), hi = *strip_at(strip, row, 2 * sc + 1);
            float y[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] *= x.alpha;
            if (x.old && m < it.M && valid > 0) {
                float o[8], s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int t = T - 1; t >= 0; --t) { // smallest first
                    load8(x.old + t * x.old_plane + m * x.ld_old + n, valid, o);
#pragma unroll
                    for (int e = 0; e < 8; ++e) s[e] += o[e];
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = fmaf(x.beta, s[e], y[e]);
            }
            if (mirror) { // back into the strip, to be read by columns
                *strip_at(strip, row, 2 * sc) = make_float4(y[0], y[1], y[2], y[3]);
                *strip_at(strip, row, 2 * sc + 1) = make_float4(y[4], y[5], y[6], y[7]);
            }
            if (m < it.M && valid > 0) put(x, m, n, valid, y);
        }
        if (!mirror) return;
        const int64_t c = m0 + 8 * sc; // column of the mirrored block
        const int there = static_cast<int>(min(it.M - c, static_cast<int64_t>(8)));
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int col = 16 * h + sr;
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int row = 8 * sc + e;
                y[e] = reinterpret_cast<const float *>(strip_at(strip, row, col / 4))[col % 4];
            }
            if (n0 + col < it.N && there > 0) put(x, n0 + col, c, there, y);
        }
    }
};

// ---- host side ---------------------------------------------------------------------------------------
// Tiles by how much LDS the terms' stages take.
template <int T, bool B_RC> struct Ns;
template <bool B_RC> struct Ns<2, B_RC> {
    using Deep = TileShape<bf16_t, 2, 2, false, B_RC, kDirect, 2, 2, 1, 1, 64, 4, 1>;  // 64 x 64, one per CU
    using Small = TileShape<bf16_t, 2, 2, false, B_RC, kDirect, 2, 2, 1, 1, 64, 2, 1>; // 64 x 64, two per CU
    using Large = TileShape<bf16_t, 2, 2, false, B_RC, kDirect, 2, 4, 2, 1, 64, 2, 1>; // 128 x 128
};
template <bool B_RC> struct Ns<3, B_RC> {
    using Deep = TileShape<bf16_t, 2, 3, false, B_RC, kDirect, 2, 2, 1, 1, 64, 3, 1>;
    using Small = TileShape<bf16_t, 2, 3, false, B_RC, kDirect, 2, 2, 1, 1, 32, 2, 1>;
    using Large = TileShape<bf16_t, 2, 3, false, B_RC, kDirect, 2, 4, 2, 1, 32, 2, 1>;
};
constexpr int64_t kTileRows = 128; // of an operand of any of them, at most
static_assert(Ns<2, false>::Large::BM <= kTileRows && Ns<3, false>::Large::BM <= kTileRows, "the size check of heta_muon_multi counts rows of a tile");

template <int T, bool B_RC> static heta_status launch_terms(const char *who, TileArgs<TermsEpi<T>> &p, hipStream_t st)
{
    double bytes = 0, flops = 0;
    int64_t large = 0, small = 0;
    for (int i = 0; i < p.n_items; ++i) {
        const TileItem &it = p.item[i];
        bytes += 2.0 * T * (static_cast<double>(it.M) * it.K + static_cast<double>(it.K) * it.N + static_cast<double>(it.M) * it.N);
        flops += (it.symmetric ? 1.0 : 2.0) * it.M * it.N * it.K;
        auto tiles = [&](int64_t b) {
            const int64_t mt = (it.M + b - 1) / b, nt = (it.N + b - 1) / b;
            return it.symmetric ? mt * (mt + 1) / 2 : mt * nt;
        };
        large += tiles(128);
        small += tiles(64);
    }
    // Large tiles once they occupy a good third of the chip.  Below, 64 x 64: with a workgroup per CU at most, the ring takes the CU's
    // whole LDS and the first 256 k-values are on their way at once (7 matrices of 128 x 256, two terms: 138 -> 121 us); with more of
    // them, two share a CU (2 matrices of 1,024 x 4,096, two terms: 709 us, 871 with the deep ring).
    if (large >= 96) return launch_tiles<typename Ns<T, B_RC>::Large>(who, "muon_product_kernel", p, bytes, flops, st);
    if (small <= 256) return launch_tiles<typename Ns<T, B_RC>::Deep>(who, "muon_product_kernel", p, bytes, flops, st);
    return launch_tiles<typename Ns<T, B_RC>::Small>(who, "muon_product_kernel", p, bytes, flops, st);
}

static int64_t pad8(int64_t n) { return (n + 7) / 8 * 8; }
struct MuonPlan { // places in the workspace, in bytes, of one item
    int64_t k, l, parts;
    int64_t ld_x, ld_g, x_plane, g_plane; // elements
    int64_t x[2], gram, poly, part, end;
    MuonPlan(int32_t rows, int32_t cols, int terms, int64_t at)
        : k(std::min(rows, cols)), l(std::max(rows, cols)), parts((int64_t(rows) + 31) / 32 * ((int64_t(cols) + 63) / 64)), ld_x(pad8(l)), ld_g(pad8(k)), x_plane(k * ld_x), g_plane(k * ld_g)
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
        part = take(parts * 4);
        end = at;
    }
};

// Items that share their launches: those of a list with as many terms, as many as fit kMuonItems and the parts of a grid.
struct MuonGroup {
    std::vector<const heta_muon_item *> items;
    std::vector<MuonPlan> plan;
    int64_t bytes = 0, parts = 0; // of workspace, and workgroups of the element-wise kernels
    int terms;
    bool add(const heta_muon_item &q)
    {
        const MuonPlan p(q.rows, q.cols, terms, bytes);
        if (static_cast<int>(items.size()) == kMuonItems || parts + p.parts > max_blocks(256)) return false; // never the first: an item's parts are bounded
        items.push_back(&q);
        plan.push_back(p);
        bytes = p.end;
        parts += p.parts;
        return true;
    }
};

// Launches alone: what it needs has been checked, and the workspace is there.
template <int T>
static heta_status muon_group(const char *who, heta_graph *g, const MuonGroup &group, float lr, float mu, int nesterov, float wd, float eps, int steps, hipStream_t st)
{
    const std::vector<MuonPlan> &plan = group.plan;
    const int n = static_cast<int>(plan.size());
    char *ws = static_cast<char *>(g->d_ws);
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
        const heta_muon_item &q = *group.items[i];
        const MuonPlan &pl = plan[i];
        a.item[i] = MuonItem{q.W, q.m, q.grad, q.ld_w, q.ld_m, q.ld_grad, q.rows, q.cols, q.rows > q.cols, q.grad_dt == HETA_BF16, q.dt == HETA_BF16, reinterpret_cast<bf16_t *>(ws + pl.x[0]), pl.ld_x,
                             pl.x_plane, reinterpret_cast<float *>(ws + pl.part), static_cast<uint32_t>(blocks), static_cast<uint32_t>(pl.parts)};
        blocks += pl.parts;
        elems += static_cast<double>(q.rows) * q.cols;
        esz = static_cast<double>(dtype_size(q.grad_dt));
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
            gram.item[i] = TileItem{x, x, pl.ld_x, pl.ld_x, pl.x_plane * 2, pl.x_plane * 2, pl.k, pl.k, pl.l, pl.l, 1, 0, 0, 1, 0, 0};
            poly.item[i] = TileItem{A, A, pl.ld_g, pl.ld_g, pl.g_plane * 2, pl.g_plane * 2, pl.k, pl.k, pl.k, pl.k, 1, 0, 0, 1, 0, 0};
            apply.item[i] = TileItem{P, x, pl.ld_g, pl.ld_x, pl.g_plane * 2, pl.x_plane * 2, pl.k, pl.l, pl.k, pl.k, 1, 0, 0, 0, 0, 0};
            gram.extra[i] = {nullptr, terms(A), 0, 0, pl.ld_g, pl.g_plane, 1.f, 0.f};
            poly.extra[i] = {terms(A), terms(P), pl.ld_g, pl.g_plane, pl.ld_g, pl.g_plane, kNsC, kNsB};
            apply.extra[i] = {terms(x), terms(y), pl.ld_x, pl.x_plane, pl.ld_x, pl.x_plane, 1.f, kNsA};
        }
        HETA_TRY((launch_terms<T, false>(who, gram, st)));
        HETA_TRY((launch_terms<T, false>(who, poly, st)));
        HETA_TRY((launch_terms<T, true>(who, apply, st)));
    }
    for (int i = 0; i < n; ++i) a.item[i].x = reinterpret_cast<bf16_t *>(ws + plan[i].x[steps & 1]);
    ProfScope prof("muon_update_kernel", st, elems * (2 * T + 2 * esz), 0);
    hipLaunchKernelGGL(muon_update_kernel<T>, grid, dim3(256), 0, st, a);
    HETA_LAUNCH_CHECK("muon_update_kernel");
    return HETA_OK;
}

} // namespace heta

using namespace heta;

static heta_status muon_multi(heta_graph *g, int32_t n_items, const heta_muon_item *items, float lr, float momentum, int32_t flags, float weight_decay, float eps, int32_t steps,
                              void *hip_stream)
{
    const char *who = "heta_muon_multi";
    if (!g || n_items < 0 || (n_items > 0 && !items)) return fail(HETA_ERR_INVALID_ARG, "%s: bad handle or item list", who);
    if (!(momentum >= 0.f && momentum < 1.f) || !(eps > 0.f) || steps < 0 || steps > 64 || !(weight_decay >= 0.f) || !std::isfinite(lr))
        return fail(HETA_ERR_INVALID_ARG, "%s: need 0 <= momentum < 1, eps > 0, weight_decay >= 0, 0 <= steps <= 64 and a finite lr", who);
    if (flags & ~(HETA_MUON_NESTEROV | HETA_MUON_COARSE)) return fail(HETA_ERR_INVALID_ARG, "%s: unknown flags", who);
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
        // a tile's rows (of the shorter side, 128 at most) are loaded by 32-bit offsets from its first one
        const int64_t k = std::min(q.rows, q.cols), row_bytes = pad8(std::max(q.rows, q.cols)) * 2;
        if ((int64_t(q.rows) + 31) / 32 * ((int64_t(q.cols) + 63) / 64) > (1 << 22) || (std::min<int64_t>(k, kTileRows) - 1) * row_bytes > (int64_t(1) << 32) - 1024)
            return fail(HETA_ERR_UNSUPPORTED, "%s: item %d: matrix too large", who, i);
        const RowRange w(q.W, q.rows, q.ld_w, q.cols, esz), m(q.m, q.rows, q.ld_m, q.cols, 4), gr(q.grad, q.rows, q.ld_grad, q.cols, gsz);
        if (gr.overlaps(w) || gr.overlaps(m)) return fail(HETA_ERR_INVALID_ARG, "%s: item %d: the gradient overlaps an output", who, i);
        outs.emplace_back(i, w);
        outs.emplace_back(i, m);
        ins.emplace_back(i, gr);
    }
    if (items_collide(outs, ins)) return fail(HETA_ERR_INVALID_ARG, "%s: an output overlaps another item's arrays", who);
    // every group's workspace before the first group's launches: a call that fails has updated nothing
    std::vector<MuonGroup> groups;
    int64_t need = 0;
    for (const int terms : {3, 2}) {
        bool open = false;
        for (int32_t i = 0; i < n_items; ++i) {
            if (muon_terms(items[i].dt, flags) != terms) continue;
            if (!open || !groups.back().add(items[i])) {
                groups.emplace_back();
                groups.back().terms = terms;
                groups.back().add(items[i]);
                open = true;
            }
        }
    }
    for (const MuonGroup &group : groups) need = std::max(need, group.bytes);
    if (need > 0) HETA_TRY(ensure_workspace(g, static_cast<size_t>(need)));
    hipStream_t st = as_stream(hip_stream);
    for (const MuonGroup &group : groups) {
        const auto run = group.terms == 3 ? muon_group<3> : muon_group<2>;
        HETA_TRY(run(who, g, group, lr, momentum, flags & HETA_MUON_NESTEROV, weight_decay, eps, steps, st));
    }
    return HETA_OK;
}

// No exception crosses the boundary: host containers may throw std::bad_alloc.
extern "C" heta_status heta_muon_multi(heta_graph *g, int32_t n_items, const heta_muon_item *items, float lr, float momentum, int32_t flags, float weight_decay, float eps,
                                       int32_t steps, void *hip_stream)
{
    try {
        return muon_multi(g, n_items, items, lr, momentum, flags, weight_decay, eps, steps, hip_stream);
    } catch (const std::bad_alloc &) {
        return fail(HETA_ERR_OOM, "heta_muon_multi: host allocation failed");
    }
}
