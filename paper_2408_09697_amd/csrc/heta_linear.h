// Epilogues and launches of heta_linear and heta_linear_bwd, shared by the translation units that hold the kernels of one
// operand type each (not part of the ABI).
#pragma once

#include <algorithm>

#include "heta_tiles.h"

namespace heta {

// ---- activations: x * sigmoid(z(x)); GELU in its tanh form, 0.5 (1 + tanh(u)) = sigmoid(2 u) --------------------
constexpr float kGelu2 = 1.5957691216057308f; // 2 sqrt(2 / pi)
constexpr float kGeluCubic = 0.044715f;
constexpr float kLog2e = 1.4426950408889634f;

// 1 / (1 + exp(-z)) by the hardware's 2^x and reciprocal (one unit in the last place each)
__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * z)); }

// -inf takes the value of the lowest finite number, -0, where -inf * 0 would be NaN; NaN stays, by the sigmoid.
template <int ACT> __device__ __forceinline__ float activate(float x)
{
    if constexpr (ACT == HETA_ACT_RELU) return x > 0.f ? x : (x != x ? x : 0.f);
    const float s = sigmoid(ACT == HETA_ACT_GELU ? x * fmaf(kGelu2 * kGeluCubic, x * x, kGelu2) : x);
    return fmaxf(x, -3.402823466e38f) * s;
}
// s + x s (1 - s) z'(x).  Where x is beyond what fp32 tells from a slope of 1 or 0, s (1 - s) is zero, and neither x nor z' may be
// infinite beside it; NaN stays, by s.
template <int ACT> __device__ __forceinline__ float activation_slope(float x)
{
    if constexpr (ACT == HETA_ACT_RELU) return x > 0.f ? 1.f : (x != x ? x : 0.f);
    const float xx = x * x;
    const float s = sigmoid(ACT == HETA_ACT_GELU ? x * fmaf(kGelu2 * kGeluCubic, xx, kGelu2) : x);
    const float t = __builtin_amdgcn_fmed3f(x, -1e30f, 1e30f) * s * (1.f - s);
    if constexpr (ACT == HETA_ACT_GELU) return fmaf(t, fminf(fmaf(3.f * kGelu2 * kGeluCubic, xx, kGelu2), 1e30f), s);
    return t + s;
}
// Several elements per (uniform) branch: chosen element by element, the choice costs more than the function.
template <int N> __device__ __forceinline__ void activate_all(float (&y)[N], int act)
{
    if (act == HETA_ACT_SILU) {
#pragma unroll
        for (int e = 0; e < N; ++e) y[e] = activate<HETA_ACT_SILU>(y[e]);
    } else if (act == HETA_ACT_GELU) {
#pragma unroll
        for (int e = 0; e < N; ++e) y[e] = activate<HETA_ACT_GELU>(y[e]);
    } else if (act == HETA_ACT_RELU) {
#pragma unroll
        for (int e = 0; e < N; ++e) y[e] = activate<HETA_ACT_RELU>(y[e]);
    }
}
template <int N> __device__ __forceinline__ void times_slopes(float (&y)[N], const float (&x)[N], int act)
{
    if (act == HETA_ACT_SILU) {
#pragma unroll
        for (int e = 0; e < N; ++e) y[e] *= activation_slope<HETA_ACT_SILU>(x[e]);
    } else if (act == HETA_ACT_GELU) {
#pragma unroll
        for (int e = 0; e < N; ++e) y[e] *= activation_slope<HETA_ACT_GELU>(x[e]);
    } else if (act == HETA_ACT_RELU) {
#pragma unroll
        for (int e = 0; e < N; ++e) y[e] *= activation_slope<HETA_ACT_RELU>(x[e]);
    }
}

// ---- epilogues ---------------------------------------------------------------------------------------
struct LinearExtra {
    const float *bias, *in_scale, *w_scale; // nullable
    const void *other;                      // nullable: the residual, or the producer's pre-activation whose slope multiplies
    void *pre, *out_p;                      // pre nullable
    int64_t ld_other, ld_pre, ld_out;
    int act, slope_act;                     // slope_act != NONE: other is a pre-activation
};
// O: type of the outputs and of what is read in their shape.  SCALED: 8-bit operands.  ACT, SLOPE: which activation, and whose
// slope, or kAnyAct for a choice at run time (small tiles, and outputs of any width): with it the epilogue of a large tile is 11,000 instructions long
// and takes longer than the product.  READS: whether `other` may be there.  WHOLE: the output is whole 16-byte pieces wide (without
// it the epilogues of large tiles cost 5 to 14 % of a product).
constexpr int kAnyAct = -1;
template <typename O, bool SCALED, int ACT = kAnyAct, int SLOPE = kAnyAct, bool READS = true, bool WHOLE = false> struct LinearEpi {
    static constexpr int kItems = 1;
    static constexpr bool kBlocks = false, kReads = READS, kPre = SLOPE <= 0, kWhole = WHOLE;
    using Out = O;
    using Extra = LinearExtra;
    static constexpr int W = 16 / (int)sizeof(O);
    // Columns and rows beyond the matrix take the values of its last ones (they are not stored): no lane is masked here, see heta_tiles.h.
    struct Cols {
        float bias[W], scale[SCALED ? W : 1];
        __device__ __forceinline__ static void floats(const float *v, int64_t n, int64_t N, float (&y)[W])
        {
#pragma unroll
            for (int h = 0; h < W; h += 4) {
                if constexpr (WHOLE) {
                    const uintx4 q = load16(v + min(n, N - W) + h);
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[h + e] = __uint_as_float(q[e]);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[h + e] = v[min(n + h + e, N - 1)];
                }
            }
        }
        __device__ __forceinline__ void load(const Extra &x, int64_t n, int64_t N)
        {
            if (x.bias) {
                floats(x.bias, n, N, bias);
            } else {
#pragma unroll
                for (int e = 0; e < W; ++e) bias[e] = 0.f;
            }
            if constexpr (SCALED) floats(x.w_scale, n, N, scale);
        }
    };
    struct Row {
        float scale;
        __device__ __forceinline__ void load(const Extra &x, int64_t m, int64_t M)
        {
            if constexpr (SCALED) scale = x.in_scale[min(m, M - 1)];
        }
    };
    __device__ __forceinline__ static O *out(const Extra &x, const TileItem &, int) { return static_cast<O *>(x.out_p); }
    __device__ __forceinline__ static void first(const Cols &c, const Row &r, float (&y)[W])
    {
#pragma unroll
        for (int e = 0; e < W; ++e) {
            if constexpr (SCALED) y[e] = fmaf(y[e], r.scale * c.scale[e], c.bias[e]);
            else y[e] += c.bias[e];
        }
    }
    template <int N> __device__ __forceinline__ static void second(const Extra &x, float (&y)[N], const float (&t)[N])
    {
        activate_all(y, ACT == kAnyAct ? x.act : ACT);
        const int slope = SLOPE == kAnyAct ? x.slope_act : SLOPE;
        if (slope != HETA_ACT_NONE) {
            times_slopes(y, t, slope);
        } else if (READS && x.other) {
#pragma unroll
            for (int e = 0; e < N; ++e) y[e] += t[e];
        }
    }
};

// partial products of a contraction that is split over its rows: [split][M][N] fp32
struct PartialEpi {
    static constexpr int kItems = 1;
    static constexpr bool kBlocks = false, kReads = false, kPre = false, kWhole = false;
    using Out = float;
    struct Extra {
        float *part;
        int64_t ld_out; // N
    };
    struct Cols {
        __device__ __forceinline__ void load(const Extra &, int64_t, int64_t) {}
    };
    using Row = Cols;
    __device__ __forceinline__ static float *out(const Extra &x, const TileItem &it, int split) { return x.part + split * it.M * it.N; }
    __device__ __forceinline__ static void first(const Cols &, const Row &, float (&)[4]) {}
    __device__ __forceinline__ static void second(const Extra &, float (&)[4], const float (&)[4]) {}
};

// The rest of a product whose contraction was split: the partial products of 16 bytes of outputs added in order, and the epilogue.
template <typename O, bool SCALED> __global__ void __launch_bounds__(256) linear_finish_kernel(LinearExtra x, const float *part, int n_split, int64_t M, int64_t N)
{
    using Epi = LinearEpi<O, SCALED>;
    constexpr int W = Epi::W;
    const int64_t per_row = (N + W - 1) / W, at = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x, m = at / per_row, n = (at - m * per_row) * W;
    if (m >= M) return;
    const int valid = static_cast<int>(min(N - n, static_cast<int64_t>(W)));
    typename Epi::Cols cols;
    typename Epi::Row row;
    cols.load(x, n, N);
    row.load(x, m, M);
    float y[W], t[W];
#pragma unroll
    for (int e = 0; e < W; ++e) y[e] = 0.f;
#pragma unroll 4
    for (int s = 0; s < n_split; ++s)
#pragma unroll
        for (int h = 0; h < W; h += 4) {
            const uintx4 q = load_piece(part + (s * M + m) * N + n + h, valid - h);
#pragma unroll
            for (int e = 0; e < 4; ++e) y[h + e] += __uint_as_float(q[e]);
        }
    unpack16<O>(x.other ? load_piece(static_cast<const O *>(x.other) + m * x.ld_other + n, valid) : uintx4{0u, 0u, 0u, 0u}, t);
    Epi::first(cols, row, y);
    if (x.pre) store_piece(static_cast<O *>(x.pre) + m * x.ld_pre + n, valid, pack16<O>(y));
    Epi::second(x, y, t);
    store_piece(static_cast<O *>(x.out_p) + m * x.ld_out + n, valid, pack16<O>(y));
}

// rows that can go straight into LDS: 16-byte aligned, and a tile's rows within 32-bit offsets
inline bool direct_rows(const void *p, int64_t ld, size_t elt) { return aligned16(p) && (ld * static_cast<int64_t>(elt)) % 16 == 0 && ld * static_cast<int64_t>(elt) < (int64_t(1) << 23); }

inline int64_t tiles_of(int64_t M, int64_t N, int bm, int bn) { return (M + bm - 1) / bm * ((N + bn - 1) / bn); }

// One product; large tiles where they give every second CU one.
struct Launch {
    heta_graph *g;
    const char *who, *name;
    TileItem it;
    double bytes, flops;
    hipStream_t st;
    template <typename C, typename Epi> heta_status go(const typename Epi::Extra &x) const
    {
        TileArgs<Epi> p{1, 0, 0, {it}, {x}};
        return launch_tiles<C>(who, name, p, bytes, flops, st);
    }
    bool direct(size_t elt) const { return direct_rows(it.A, it.lda, elt) && direct_rows(it.B, it.ldb, elt); }
    bool large() const { return tiles_of(it.M, it.N, 256, 256) * it.n_split >= 128; }
};
// How a product of few tiles and a long contraction is split: so that a workgroup has about eight k-tiles and most of the chip one
// workgroup; a second launch adds the parts up and does the epilogue (114 x 1,611 x 7: 114 -> 15 us).  Small tiles are 64 x 64 of 128 bytes of k-values.
struct SplitPlan {
    int64_t k_per_split = 0;
    int32_t n_split = 1; // 1: not split
    size_t bytes = 0;    // of partial products
};
inline SplitPlan plan_split(const Launch &l, size_t elt)
{
    SplitPlan s;
    const int64_t bk = 128 / static_cast<int64_t>(elt), tiles = tiles_of(l.it.M, l.it.N, 64, 64), k_tiles = (l.it.K + bk - 1) / bk;
    const int64_t splits = l.large() ? 0 : std::min(k_tiles / 8, 256 / tiles);
    if (splits < 2) return s;
    s.k_per_split = (k_tiles + splits - 1) / splits * bk;
    s.n_split = static_cast<int32_t>((l.it.K + s.k_per_split - 1) / s.k_per_split);
    s.bytes = static_cast<size_t>(s.n_split) * l.it.M * l.it.N * sizeof(float);
    return s;
}
// f(std::integral_constant<int, a>) for activation a
template <typename F> inline heta_status with_act(int a, F f)
{
    if (a == HETA_ACT_RELU) return f(std::integral_constant<int, HETA_ACT_RELU>{});
    if (a == HETA_ACT_GELU) return f(std::integral_constant<int, HETA_ACT_GELU>{});
    if (a == HETA_ACT_SILU) return f(std::integral_constant<int, HETA_ACT_SILU>{});
    return f(std::integral_constant<int, HETA_ACT_NONE>{});
}
// in . W (B_RC = true; the output's activation) or grad . W^T (the slope's activation), and the split in^T . grad
heta_status launch_linear_f32(const Launch &l, bool input_gradient, const LinearExtra &x);
heta_status launch_linear_bf16(const Launch &l, bool input_gradient, heta_dtype out_dt, const LinearExtra &x);
heta_status launch_linear_e4m3(const Launch &l, heta_dtype out_dt, bool coarse, const LinearExtra &x);
heta_status launch_grad_w_f32(const Launch &l, float *part);
// Bytes of the copies, in aligned rows, of the operands of a large weight gradient whose rows start anywhere (0: none are worth it), and
// the copies themselves, `to` (256-byte aligned) that many bytes of the workspace.
size_t align_grad_w_bytes(const Launch &l);
heta_status align_grad_w_bf16(Launch &l, char *to);
heta_status launch_grad_w_bf16(const Launch &l, float *part);

// one type's launches from its tile shapes: large tiles (Reading: where the epilogue reads in the output's shape; Ragged: where its rows are not whole
// 16-byte pieces), small ones, and both for rows that cannot go straight into LDS
template <typename Large, typename Reading, typename Ragged, typename Small, typename StagedLarge, typename StagedSmall, typename O, bool SLOPES>
inline heta_status launch_linear(const Launch &l, size_t elt, const LinearExtra &x)
{
    constexpr bool SCALED = Large::EB == 1;
    const bool direct = l.direct(elt);
    if (!l.large()) {
        static_assert(Small::BM == 64 && Small::BN == 64 && Small::BK * sizeof(typename Small::S) == 128, "plan_split() counts such tiles");
        const SplitPlan split = plan_split(l, elt);
        if (split.n_split > 1) {
            Launch part = l;
            part.it.k_per_split = split.k_per_split;
            part.it.n_split = split.n_split;
            HETA_TRY(ensure_workspace(l.g, split.bytes));
            float *ws = static_cast<float *>(l.g->d_ws);
            const PartialEpi::Extra px{ws, l.it.N};
            HETA_TRY((direct ? part.go<Small, PartialEpi>(px) : part.go<StagedSmall, PartialEpi>(px)));
            constexpr int W = 16 / (int)sizeof(O);
            const int64_t blocks = (l.it.M * ((l.it.N + W - 1) / W) + 255) / 256;
            ProfScope prof("linear_finish_kernel", l.st, static_cast<double>(l.it.M) * l.it.N * (4.0 * part.it.n_split + sizeof(O)), 0);
            hipLaunchKernelGGL((linear_finish_kernel<O, SCALED>), dim3(static_cast<unsigned>(blocks)), dim3(256), 0, l.st, x, ws, part.it.n_split, l.it.M, l.it.N);
            HETA_LAUNCH_CHECK("linear_finish_kernel");
            return HETA_OK;
        }
        return direct ? l.go<Small, LinearEpi<O, SCALED>>(x) : l.go<StagedSmall, LinearEpi<O, SCALED>>(x);
    }
    if (!direct && !std::is_same<StagedLarge, Large>::value) return l.go<StagedLarge, LinearEpi<O, SCALED>>(x);
    if (l.it.N % (16 / (int)sizeof(O)) != 0) return l.go<Ragged, LinearEpi<O, SCALED>>(x);
    return with_act(SLOPES ? x.slope_act : x.act, [&](auto a) {
        constexpr int A = decltype(a)::value;
        if constexpr (SLOPES) return l.go<Large, LinearEpi<O, SCALED, HETA_ACT_NONE, A, A != HETA_ACT_NONE, true>>(x);
        else return x.other ? l.go<Reading, LinearEpi<O, SCALED, A, HETA_ACT_NONE, true, true>>(x) : l.go<Large, LinearEpi<O, SCALED, A, HETA_ACT_NONE, false, true>>(x);
    });
}
template <typename Large, typename Small, typename StagedLarge, typename StagedSmall> inline heta_status launch_grad_w(const Launch &l, size_t elt, float *part)
{
    const PartialEpi::Extra x{part, l.it.N};
    if (l.direct(elt)) return l.large() ? l.go<Large, PartialEpi>(x) : l.go<Small, PartialEpi>(x);
    return l.large() ? l.go<StagedLarge, PartialEpi>(x) : l.go<StagedSmall, PartialEpi>(x);
}

} // namespace heta
