// Root-mean-square norm of embedding rows with the residual's addition in front, its backward pass, and an 8-bit output
// with a scale a row for products of 8-bit operands.
//
//     s = round(x + residual) (stored if asked for),  rstd = (sum_j s_j^2 / d + eps)^(-1/2),  out = s rstd gamma
//     8-bit: scale = max_j |out_j| / 448,  q = e4m3(out / scale), or / 127 and whole numbers; a row of zeros has scale 0
//     h = s rstd, w = grad_out gamma:  grad_x = rstd (w - h sum_j(w_j h_j) / d) + grad_sum,  grad_gamma = sum over rows of grad_out h
//
// HBM-bound: six to nine operations per element that is read.  One pass: a row lives in the registers of 8 to 64 lanes
// from its load to its last store (LANES x NV chunks of eight elements; rows of more than 2,048 columns are walked by a
// workgroup, up to three times through the caches).  Statistics and all sums are fp32.  Rows need no alignment.
// grad_gamma: every lane adds up its columns over the rows it visits, a workgroup joins its groups of lanes through LDS in
// order, and the workgroups' partial sums are added in a fixed order: no atomics.
#include <algorithm>
#include <type_traits>

#include "heta_rows.h"

namespace heta {

struct NormFwd {
    const void *x, *residual; // residual nullable
    void *sum, *out;          // sum nullable
    const float *gamma;       // nullable: ones
    float *scale, *rstd;      // scale with 8-bit output, rstd nullable
    int64_t ld_x, ld_res, ld_sum, ld_out, n_rows;
    int32_t d;
    float eps;
};

template <int LANES> __device__ __forceinline__ float lanes_sum(float v)
{
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}
template <int LANES> __device__ __forceinline__ uint32_t lanes_max(uint32_t v)
{
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) v = max(v, static_cast<uint32_t>(__shfl_xor(static_cast<int>(v), o)));
    return v;
}

// Without eps, a row whose squares add up to nothing has no reciprocal root; 0 makes its outputs zeros, and so its share of the gradients.
__device__ __forceinline__ float reciprocal_root(float mean_sq) { return mean_sq == 0.f ? 0.f : 1.f / sqrtf(mean_sq); }

// A lane's eight values of chunk v are 8 / P pieces of P consecutive columns; the pieces of a group of lanes lie side by side, so
// that an access of the widest type among the row's arrays is 16 bytes of consecutive memory per lane (P = 4 where fp32 is among
// them, else 8).  100,000 unaligned rows of 789 fp32 columns, backward: 328 us with eight consecutive columns per lane; of bf16
// rows, 274 with pieces of four, 229 with pieces of eight whose last is taken apart (300,000 x 300: 270 / 259; 10^6 x 100: 241 / 200); the
// code for that piece alone takes 4 % of the time of widths that have none (700,000 x 256, backward: 267 / 257).
template <int LANES, int P> __device__ __forceinline__ int column(int v, int e, int l) { return ((v * (8 / P) + e / P) * LANES + l) * P + e % P; }

// N words at any address
template <int N, bool STREAM> __device__ __forceinline__ void load_words(const void *p, uint32_t (&w)[N])
{
    typedef uint32_t words __attribute__((ext_vector_type(N == 1 ? 2 : N), aligned(1)));
    if constexpr (N == 1) {
        __builtin_memcpy(w, p, 4);
    } else {
        words q;
        if constexpr (STREAM) q = __builtin_nontemporal_load(static_cast<const words *>(p));
        else q = *static_cast<const words *>(p);
#pragma unroll
        for (int j = 0; j < N; ++j) w[j] = q[j];
    }
}
template <int N, bool STREAM> __device__ __forceinline__ void store_words(void *p, const uint32_t (&w)[N])
{
    typedef uint32_t words __attribute__((ext_vector_type(N == 1 ? 2 : N), aligned(1)));
    if constexpr (N == 1) {
        __builtin_memcpy(p, w, 4);
    } else {
        words q;
#pragma unroll
        for (int j = 0; j < N; ++j) q[j] = w[j];
        if constexpr (STREAM) __builtin_nontemporal_store(q, static_cast<words *>(p));
        else *static_cast<words *>(p) = q;
    }
}

// The last `rest` < 8 of a row's bf16 values, as they lie in memory, by at most three accesses (rest is uniform).
__device__ __forceinline__ void load_tail(const bf16_t *p, int rest, uint32_t (&w)[4])
{
    if (rest & 4) {
        uint32_t t[2];
        load_words<2, false>(p, t);
        w[0] = t[0];
        w[1] = t[1];
        p += 4;
    }
    if (rest & 2) {
        uint32_t t;
        __builtin_memcpy(&t, p, 4);
        w[0] = rest & 4 ? w[0] : t;
        w[2] = rest & 4 ? t : w[2];
        p += 2;
    }
    if (rest & 1) {
        const uint32_t t = *p;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = j == rest / 2 ? t : w[j];
    }
}
__device__ __forceinline__ void store_tail(bf16_t *p, int rest, const uint32_t (&w)[4])
{
    if (rest & 4) {
        store_words<2, false>(p, {w[0], w[1]});
        p += 4;
    }
    if (rest & 2) {
        const uint32_t t = rest & 4 ? w[2] : w[0];
        __builtin_memcpy(p, &t, 4);
        p += 2;
    }
    if (rest & 1) *p = static_cast<bf16_t>(rest == 1 ? w[0] : rest == 3 ? w[1] : rest == 5 ? w[2] : w[3]);
}

// TAIL: the width may be no multiple of P.  Without it lanes beyond the width still go through the branch for single elements, which reads
// none; with plain zeros there, the compiler's order of the loads costs 6 % (700,000 x 256, backward: 273 us for 257).
template <int LANES, int NV, int P, bool TAIL, bool STREAM, typename T> __device__ __forceinline__ void load_row(const T *row, int d, int l, float (&x)[NV][8])
{
    constexpr int N = P * (int)sizeof(T) / 4;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int h = 0; h < 8; h += P) {
            const int c = column<LANES, P>(v, h, l);
            if (c + P <= d) {
                uint32_t w[N];
                load_words<N, STREAM>(row + c, w);
#pragma unroll
                for (int e = 0; e < P; ++e) {
                    if constexpr (sizeof(T) == 4) x[v][h + e] = __uint_as_float(w[e]);
                    else x[v][h + e] = __uint_as_float(e & 1 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
                }
            } else if constexpr (TAIL && P == 8 && sizeof(T) == 2) {
                uint32_t w[4] = {0u, 0u, 0u, 0u};
                if (c < d) load_tail(row + c, d & 7, w);
#pragma unroll
                for (int e = 0; e < P; ++e) x[v][h + e] = __uint_as_float(e & 1 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
            } else {
#pragma unroll
                for (int e = 0; e < P; ++e) x[v][h + e] = c + e < d ? widen(row[c + e]) : 0.f;
            }
        }
}
template <int LANES, int NV, int P, bool TAIL, bool STREAM, typename T> __device__ __forceinline__ void store_row(T *row, int d, int l, const float (&x)[NV][8])
{
    constexpr int N = P * (int)sizeof(T) / 4;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int h = 0; h < 8; h += P) {
            const int c = column<LANES, P>(v, h, l);
            uint32_t w[N];
#pragma unroll
            for (int j = 0; j < N; ++j) {
                if constexpr (sizeof(T) == 4) w[j] = __float_as_uint(x[v][h + j]);
                else w[j] = pack2_bf16(x[v][h + 2 * j], x[v][h + 2 * j + 1]);
            }
            if (c + P <= d) {
                store_words<N, STREAM>(row + c, w);
            } else if constexpr (TAIL && P == 8 && sizeof(T) == 2) {
                if (c < d) store_tail(row + c, d & 7, w);
            } else {
#pragma unroll
                for (int e = 0; e < P; ++e)
                    if (c + e < d) {
                        if constexpr (sizeof(T) == 4) row[c + e] = x[v][h + e];
                        else row[c + e] = static_cast<bf16_t>(w[e / 2] >> (16 * (e & 1)));
                    }
            }
        }
}

__device__ __forceinline__ uint32_t four_e4m3(float a, float b, float c, float d)
{
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true));
}
// O of an 8-bit output: uint8_t for e4m3, int8_t for whole numbers
template <typename O> __device__ __forceinline__ uint32_t four_codes(float a, float b, float c, float d)
{
    if constexpr (std::is_same<O, int8_t>::value) return four_i8(a, b, c, d);
    else return four_e4m3(a, b, c, d);
}
template <typename O> __device__ __forceinline__ float codes_factor(float amax)
{
    if constexpr (std::is_same<O, int8_t>::value) return i8_factor(amax);
    else return e4m3_factor(amax);
}
template <typename O> __device__ __forceinline__ float codes_scale(float amax)
{
    if constexpr (std::is_same<O, int8_t>::value) return i8_scale(amax);
    else return e4m3_scale(amax);
}
template <typename O, int LANES, int NV, int P> __device__ __forceinline__ void store_row_codes(uint8_t *row, int d, int l, const float (&x)[NV][8], float f)
{
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int h = 0; h < 8; h += P) {
            const int c = column<LANES, P>(v, h, l);
            uint32_t w[P / 4];
#pragma unroll
            for (int j = 0; j < P / 4; ++j) w[j] = four_codes<O>(x[v][h + 4 * j] * f, x[v][h + 4 * j + 1] * f, x[v][h + 4 * j + 2] * f, x[v][h + 4 * j + 3] * f);
            if (c + P <= d) {
                store_words<P / 4, false>(row + c, w);
            } else {
#pragma unroll
                for (int e = 0; e < P; ++e)
                    if (c + e < d) row[c + e] = static_cast<uint8_t>((w[e / 4] >> (8 * (e & 3))) & 0xff);
            }
        }
}

template <typename T> __device__ __forceinline__ float rounded(float v)
{
    if constexpr (sizeof(T) == 2) return widen(to_bf16(v));
    else return v;
}

// T: type of x, residual and sum; O: of the output
template <typename T, typename O, int LANES, int NV, int P, bool TAIL, bool STREAM> __global__ void __launch_bounds__(256) rms_norm_kernel(NormFwd p)
{
    constexpr int GROUPS = 256 / LANES;
    const int l = threadIdx.x % LANES, grp = threadIdx.x / LANES;
    float gamma[NV][8];
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int c = column<LANES, P>(v, e, l);
            gamma[v][e] = p.gamma && c < p.d ? p.gamma[c] : 1.f;
        }
    for (int64_t r = static_cast<int64_t>(blockIdx.x) * GROUPS + grp; r < p.n_rows; r += static_cast<int64_t>(gridDim.x) * GROUPS) {
        float x[NV][8];
        load_row<LANES, NV, P, TAIL, STREAM>(static_cast<const T *>(p.x) + r * p.ld_x, p.d, l, x);
        if (p.residual) {
            float y[NV][8];
            load_row<LANES, NV, P, TAIL, STREAM>(static_cast<const T *>(p.residual) + r * p.ld_res, p.d, l, y);
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int e = 0; e < 8; ++e) x[v][e] = rounded<T>(x[v][e] + y[v][e]);
        }
        if (p.sum) store_row<LANES, NV, P, TAIL, STREAM>(static_cast<T *>(p.sum) + r * p.ld_sum, p.d, l, x);
        float ss = 0.f;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int e = 0; e < 8; ++e) ss += x[v][e] * x[v][e];
        const float rstd = reciprocal_root(lanes_sum<LANES>(ss) / static_cast<float>(p.d) + p.eps);
        if (p.rstd && l == 0) p.rstd[r] = rstd;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int e = 0; e < 8; ++e) x[v][e] = x[v][e] * rstd * gamma[v][e];
        if constexpr (sizeof(O) == 1) {
            uint32_t top = 0;
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int e = 0; e < 8; ++e) top = max(top, magnitude(x[v][e]));
            const float amax = __uint_as_float(lanes_max<LANES>(top));
            if (l == 0) p.scale[r] = codes_scale<O>(amax);
            store_row_codes<O, LANES, NV, P>(static_cast<uint8_t *>(p.out) + r * p.ld_out, p.d, l, x, codes_factor<O>(amax));
        } else {
            store_row<LANES, NV, P, TAIL, STREAM>(static_cast<O *>(p.out) + r * p.ld_out, p.d, l, x);
        }
    }
}

// Sum, and largest magnitude, over the 256 threads of a workgroup, in every thread.
__device__ __forceinline__ float group_sum(float v, float *lds)
{
    v = lanes_sum<64>(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}
__device__ __forceinline__ float group_max(uint32_t v, float *lds)
{
    v = lanes_max<64>(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = __uint_as_float(v);
    __syncthreads();
    return __uint_as_float(max(max(__float_as_uint(lds[0]), __float_as_uint(lds[1])), max(__float_as_uint(lds[2]), __float_as_uint(lds[3]))));
}

// Rows too wide for one wavefront's registers: a workgroup per row.  `sum` may alias x or residual: a thread reads its
// columns before it writes them, and later passes read the sum.
template <typename T, typename O> __global__ void __launch_bounds__(256) rms_norm_wide_kernel(NormFwd p)
{
    __shared__ float lds[4];
    for (int64_t r = blockIdx.x; r < p.n_rows; r += gridDim.x) {
        const T *x = static_cast<const T *>(p.x) + r * p.ld_x, *y = p.residual ? static_cast<const T *>(p.residual) + r * p.ld_res : nullptr;
        T *sum = p.sum ? static_cast<T *>(p.sum) + r * p.ld_sum : nullptr;
        float ss = 0.f;
        for (int c = threadIdx.x; c < p.d; c += 256) {
            const float s = y ? rounded<T>(widen(x[c]) + widen(y[c])) : widen(x[c]);
            if (sum) {
                if constexpr (sizeof(T) == 2) sum[c] = to_bf16(s);
                else sum[c] = s;
            }
            ss += s * s;
        }
        const float rstd = reciprocal_root(group_sum(ss, lds) / static_cast<float>(p.d) + p.eps);
        if (p.rstd && threadIdx.x == 0) p.rstd[r] = rstd;
        auto value = [&](int c) {
            const float s = sum ? widen(sum[c]) : (y ? rounded<T>(widen(x[c]) + widen(y[c])) : widen(x[c]));
            return s * rstd * (p.gamma ? p.gamma[c] : 1.f);
        };
        if constexpr (sizeof(O) == 1) {
            uint32_t top = 0;
            for (int c = threadIdx.x; c < p.d; c += 256) top = max(top, magnitude(value(c)));
            const float amax = group_max(top, lds);
            if (threadIdx.x == 0) p.scale[r] = codes_scale<O>(amax);
            const float f = codes_factor<O>(amax);
            for (int c = threadIdx.x; c < p.d; c += 256) {
                const float v = value(c) * f;
                (static_cast<uint8_t *>(p.out) + r * p.ld_out)[c] = static_cast<uint8_t>(four_codes<O>(v, 0.f, 0.f, 0.f) & 0xff);
            }
        } else {
            O *out = static_cast<O *>(p.out) + r * p.ld_out;
            for (int c = threadIdx.x; c < p.d; c += 256) {
                if constexpr (sizeof(O) == 2) out[c] = to_bf16(value(c));
                else out[c] = value(c);
            }
        }
    }
}

struct NormBwd {
    const void *x, *grad_out, *grad_sum; // grad_sum nullable
    void *grad_x;
    const float *gamma, *rstd;           // gamma nullable
    float *part;                         // [workgroups][d], nullable
    int64_t ld_x, ld_go, ld_gs, ld_gx, n_rows;
    int32_t d;
};

template <typename T, typename G, int LANES, int NV, int P, bool TAIL, bool STREAM> __global__ void __launch_bounds__(256) rms_norm_bwd_kernel(NormBwd p)
{
    constexpr int GROUPS = 256 / LANES;
    __shared__ float joined[GROUPS * LANES * NV * 8];
    const int l = threadIdx.x % LANES, grp = threadIdx.x / LANES;
    float gamma[NV][8], dg[NV][8];
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int c = column<LANES, P>(v, e, l);
            gamma[v][e] = p.gamma && c < p.d ? p.gamma[c] : 1.f;
            dg[v][e] = 0.f;
        }
    const float inv_d = 1.f / static_cast<float>(p.d);
    for (int64_t r = static_cast<int64_t>(blockIdx.x) * GROUPS + grp; r < p.n_rows; r += static_cast<int64_t>(gridDim.x) * GROUPS) {
        float h[NV][8], w[NV][8];
        load_row<LANES, NV, P, TAIL, STREAM>(static_cast<const T *>(p.x) + r * p.ld_x, p.d, l, h);
        load_row<LANES, NV, P, TAIL, STREAM>(static_cast<const G *>(p.grad_out) + r * p.ld_go, p.d, l, w);
        const float rstd = p.rstd[r];
        float dot = 0.f;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                h[v][e] *= rstd;
                dg[v][e] += w[v][e] * h[v][e];
                w[v][e] *= gamma[v][e];
                dot += w[v][e] * h[v][e];
            }
        dot = lanes_sum<LANES>(dot) * inv_d;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int e = 0; e < 8; ++e) w[v][e] = rstd * (w[v][e] - h[v][e] * dot);
        if (p.grad_sum) {
            load_row<LANES, NV, P, TAIL, STREAM>(static_cast<const T *>(p.grad_sum) + r * p.ld_gs, p.d, l, h);
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int e = 0; e < 8; ++e) w[v][e] += h[v][e];
        }
        store_row<LANES, NV, P, TAIL, STREAM>(static_cast<T *>(p.grad_x) + r * p.ld_gx, p.d, l, w);
    }
    if (!p.part) return;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int e = 0; e < 8; ++e) joined[(grp * NV * 8 + v * 8 + e) * LANES + l] = dg[v][e];
    __syncthreads();
    for (int q = threadIdx.x; q < LANES * NV * 8; q += 256) {
        float s = 0.f;
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) s += joined[g * NV * 8 * LANES + q];
        const int c = column<LANES, P>(q / LANES / 8, q / LANES % 8, q % LANES);
        if (c < p.d) p.part[static_cast<int64_t>(blockIdx.x) * p.d + c] = s;
    }
}

// Rows too wide for one wavefront's registers: a workgroup per row; grad_gamma by a kernel of its own over slabs of rows.
template <typename T, typename G> __global__ void __launch_bounds__(256) rms_norm_bwd_wide_kernel(NormBwd p)
{
    __shared__ float lds[4];
    for (int64_t r = blockIdx.x; r < p.n_rows; r += gridDim.x) {
        const T *x = static_cast<const T *>(p.x) + r * p.ld_x, *gs = p.grad_sum ? static_cast<const T *>(p.grad_sum) + r * p.ld_gs : nullptr;
        const G *go = static_cast<const G *>(p.grad_out) + r * p.ld_go;
        T *gx = static_cast<T *>(p.grad_x) + r * p.ld_gx;
        const float rstd = p.rstd[r];
        float dot = 0.f;
        for (int c = threadIdx.x; c < p.d; c += 256) dot += widen(go[c]) * (p.gamma ? p.gamma[c] : 1.f) * (widen(x[c]) * rstd);
        dot = group_sum(dot, lds) / static_cast<float>(p.d);
        for (int c = threadIdx.x; c < p.d; c += 256) {
            float v = rstd * (widen(go[c]) * (p.gamma ? p.gamma[c] : 1.f) - widen(x[c]) * rstd * dot);
            if (gs) v += widen(gs[c]);
            if constexpr (sizeof(T) == 2) gx[c] = to_bf16(v);
            else gx[c] = v;
        }
    }
}
template <typename T, typename G> __global__ void __launch_bounds__(256) rms_norm_gamma_kernel(NormBwd p, int64_t rows_each)
{
    const uint32_t strips = (p.d + 255) / 256;
    const int64_t slab = blockIdx.x / strips;
    const int c = static_cast<int>(blockIdx.x % strips) * 256 + threadIdx.x;
    if (c >= p.d) return;
    const int64_t end = min(p.n_rows, (slab + 1) * rows_each);
    float s = 0.f;
#pragma unroll 4
    for (int64_t r = slab * rows_each; r < end; ++r)
        s += widen(static_cast<const G *>(p.grad_out)[r * p.ld_go + c]) * (widen(static_cast<const T *>(p.x)[r * p.ld_x + c]) * p.rstd[r]);
    p.part[slab * p.d + c] = s;
}

// ---- host side ---------------------------------------------------------------------------------------
// Lanes and chunks per row by width, so that as few lanes as possible lie idle: f(lanes, chunks) or, above, wide().
template <typename F, typename W> static void by_width(int32_t d, F f, W wide)
{
    using std::integral_constant;
    if (d <= 64) f(integral_constant<int, 8>{}, integral_constant<int, 1>{});
    else if (d <= 128) f(integral_constant<int, 16>{}, integral_constant<int, 1>{});
    else if (d <= 256) f(integral_constant<int, 32>{}, integral_constant<int, 1>{});
    else if (d <= 512) f(integral_constant<int, 64>{}, integral_constant<int, 1>{});
    else if (d <= 1024) f(integral_constant<int, 64>{}, integral_constant<int, 2>{});
    else if (d <= 2048) f(integral_constant<int, 64>{}, integral_constant<int, 4>{});
    else wide();
}
// Workgroups at most, each walking over rows (us on three sets of inputs in turn).  1.1 M rows of 256 bf16 columns with 2,048 / 4,096 / 16,384 workgroups and
// one per 8 rows: to 8 bits 380 / 376 / 378 / 537, to bf16 409 / 405 / 402 / 537; without the streaming hint 381 and 440 with 16,384.  Backward of 700,000 rows with 1,024 /
// 2,048 / 4,096 / 8,192: 275 / 295 / 259 / 276, 285 without the hint; of 100,000 fp32 rows of 789 238 / 240 / 246 / 263, and 264.
constexpr int64_t kNormBlocks = 16384, kNormBwdBlocks = 4096;
static unsigned row_blocks(int64_t n_rows, int groups, int64_t most) { return static_cast<unsigned>(std::max<int64_t>(1, std::min<int64_t>((n_rows + groups - 1) / groups, most))); }

using std::integral_constant;
template <typename T, typename O> static void launch_norm(const NormFwd &p, bool stream, hipStream_t st)
{
    by_width(
        p.d,
        [&](auto lanes, auto nv) {
            constexpr int L = decltype(lanes)::value, V = decltype(nv)::value;
            const dim3 grid(row_blocks(p.n_rows, 256 / L, kNormBlocks));
            auto go = [&](auto piece, auto tail) {
                constexpr int P = decltype(piece)::value;
                constexpr bool TAIL = decltype(tail)::value;
                if (stream) hipLaunchKernelGGL((rms_norm_kernel<T, O, L, V, P, TAIL, true>), grid, dim3(256), 0, st, p);
                else hipLaunchKernelGGL((rms_norm_kernel<T, O, L, V, P, TAIL, false>), grid, dim3(256), 0, st, p);
            };
            if constexpr (sizeof(T) == 2 && sizeof(O) <= 2)
                if (p.d % 8 == 0) return go(integral_constant<int, 8>{}, std::false_type{});
            go(integral_constant<int, sizeof(T) == 2 && sizeof(O) == 2 ? 8 : 4>{}, std::true_type{});
        },
        [&] { hipLaunchKernelGGL((rms_norm_wide_kernel<T, O>), dim3(row_blocks(p.n_rows, 1, 8192)), dim3(256), 0, st, p); });
}


template <typename T, typename G> static void launch_norm_bwd(const NormBwd &p, bool stream, int64_t n_part, hipStream_t st)
{
    by_width(
        p.d,
        [&](auto lanes, auto nv) {
            constexpr int L = decltype(lanes)::value, V = decltype(nv)::value;
            const dim3 grid(static_cast<unsigned>(n_part));
            auto go = [&](auto piece, auto tail) {
                constexpr int P = decltype(piece)::value;
                constexpr bool TAIL = decltype(tail)::value;
                if (stream) hipLaunchKernelGGL((rms_norm_bwd_kernel<T, G, L, V, P, TAIL, true>), grid, dim3(256), 0, st, p);
                else hipLaunchKernelGGL((rms_norm_bwd_kernel<T, G, L, V, P, TAIL, false>), grid, dim3(256), 0, st, p);
            };
            if constexpr (sizeof(T) == 2 && sizeof(G) == 2) {
                if (p.d % 8 == 0) go(integral_constant<int, 8>{}, std::false_type{});
                else go(integral_constant<int, 8>{}, std::true_type{});
            } else {
                go(integral_constant<int, 4>{}, std::true_type{});
            }
        },
        [&] {
            hipLaunchKernelGGL((rms_norm_bwd_wide_kernel<T, G>), dim3(row_blocks(p.n_rows, 1, 8192)), dim3(256), 0, st, p);
            if (p.part)
                hipLaunchKernelGGL((rms_norm_gamma_kernel<T, G>), dim3(static_cast<unsigned>(n_part * ((p.d + 255) / 256))), dim3(256), 0, st, p,
                                   (p.n_rows + n_part - 1) / n_part);
        });
}

} // namespace heta

using namespace heta;

extern "C" heta_status heta_rms_norm(int64_t n_rows, int32_t d, const void *x, heta_dtype x_dt, int64_t ld_x, const void *residual, int64_t ld_res, const float *gamma,
                                     float eps, void *sum, int64_t ld_sum, void *out, heta_dtype out_dt, int64_t ld_out, float *scale, float *rstd, void *hip_stream)
{
    const char *who = "heta_rms_norm";
    if (n_rows < 0 || d <= 0) return fail(HETA_ERR_SHAPE, "%s: need n_rows >= 0 and d > 0", who);
    if (d > kWidest) return fail(HETA_ERR_UNSUPPORTED, "%s: rows too wide", who);
    if (!valid_dtype(x_dt) || (!valid_dtype(out_dt) && out_dt != HETA_E4M3 && out_dt != HETA_I8)) return fail(HETA_ERR_INVALID_ARG, "%s: bad dtype", who);
    if (!(eps >= 0.f)) return fail(HETA_ERR_INVALID_ARG, "%s: need eps >= 0", who);
    const bool q = out_dt == HETA_E4M3 || out_dt == HETA_I8;
    if (x_dt == HETA_BF16 && out_dt == HETA_F32) return fail(HETA_ERR_UNSUPPORTED, "%s: bf16 rows have a bf16 or an 8-bit output", who);
    if (q != (scale != nullptr) && !(q && n_rows == 0)) return fail(HETA_ERR_INVALID_ARG, "%s: scales belong to an 8-bit output, and that needs them", who);
    const size_t esz = dtype_size(x_dt), osz = q ? 1 : dtype_size(out_dt);
    HETA_TRY(check_rows(who, "x", x, n_rows, ld_x, d, esz));
    HETA_TRY(check_rows(who, "out", out, n_rows, ld_out, d, osz));
    if (residual) HETA_TRY(check_rows(who, "residual", residual, n_rows, ld_res, d, esz));
    if (sum) HETA_TRY(check_rows(who, "sum", sum, n_rows, ld_sum, d, esz));
    for (const float *v : {gamma, static_cast<const float *>(scale), static_cast<const float *>(rstd)})
        if (reinterpret_cast<uintptr_t>(v) & 3u) return fail(HETA_ERR_INVALID_ARG, "%s: pointer not aligned to its element size", who);
    // every array is read and written row by row by the lanes that hold the row: outputs may lie on inputs, in the same rows
    const RowRange rx(x, n_rows, ld_x, d, esz), rr(residual, n_rows, ld_res, d, esz), rs(sum, n_rows, ld_sum, d, esz), ro(out, n_rows, ld_out, d, osz);
    const bool sum_on_x = sum == x && ld_sum == ld_x, sum_on_res = sum == residual && ld_sum == ld_res;
    const RowRange rg(gamma, 1, d, d, 4), rscale(scale, 1, n_rows, n_rows, 4), rrstd(rstd, 1, n_rows, n_rows, 4);
    for (const RowRange &o : {rs, ro})
        for (const RowRange &v : {rg, rscale, rrstd})
            if (o.overlaps(v)) return fail(HETA_ERR_INVALID_ARG, "%s: gamma, scale or rstd overlaps out or sum", who);
    for (const RowRange &v : {rx, rr, rg})
        if (rscale.overlaps(v) || rrstd.overlaps(v)) return fail(HETA_ERR_INVALID_ARG, "%s: scale or rstd overlaps an operand", who);
    if (rscale.overlaps(rrstd)) return fail(HETA_ERR_INVALID_ARG, "%s: scale overlaps rstd", who);
    if ((rs.overlaps(rx) && !sum_on_x) || (rs.overlaps(rr) && !sum_on_res) || ro.overlaps(rx) || ro.overlaps(rr) || ro.overlaps(rs))
        return fail(HETA_ERR_INVALID_ARG, "%s: out overlaps another array, or sum one in other rows", who);
    if (n_rows == 0) return HETA_OK;
    const NormFwd p{x, residual, sum, out, gamma, scale, rstd, ld_x, ld_res, ld_sum, ld_out, n_rows, d, eps};
    hipStream_t st = as_stream(hip_stream);
    const double bytes = static_cast<double>(n_rows) * d * (esz * (1.0 + !!residual + !!sum) + osz);
    const bool stream = streams(bytes);
    ProfScope prof("rms_norm_kernel", st, bytes, 6.0 * n_rows * d);
    if (x_dt == HETA_F32) {
        if (out_dt == HETA_I8) launch_norm<float, int8_t>(p, stream, st);
        else if (q) launch_norm<float, uint8_t>(p, stream, st);
        else if (out_dt == HETA_F32) launch_norm<float, float>(p, stream, st);
        else launch_norm<float, bf16_t>(p, stream, st);
    } else {
        if (out_dt == HETA_I8) launch_norm<bf16_t, int8_t>(p, stream, st);
        else if (q) launch_norm<bf16_t, uint8_t>(p, stream, st);
        else launch_norm<bf16_t, bf16_t>(p, stream, st);
    }
    HETA_LAUNCH_CHECK("rms_norm_kernel");
    return HETA_OK;
}

extern "C" heta_status heta_rms_norm_bwd(heta_graph *g, int64_t n_rows, int32_t d, const void *x, heta_dtype x_dt, int64_t ld_x, const float *gamma, const float *rstd,
                                         const void *grad_out, heta_dtype go_dt, int64_t ld_go, const void *grad_sum, int64_t ld_gs, void *grad_x, int64_t ld_gx,
                                         float *grad_gamma, void *hip_stream)
{
    const char *who = "heta_rms_norm_bwd";
    if (!g) return fail(HETA_ERR_INVALID_ARG, "%s: null handle", who);
    if (n_rows < 0 || d <= 0) return fail(HETA_ERR_SHAPE, "%s: need n_rows >= 0 and d > 0", who);
    if (d > kWidest) return fail(HETA_ERR_UNSUPPORTED, "%s: rows too wide", who);
    if (!valid_dtype(x_dt) || !valid_dtype(go_dt)) return fail(HETA_ERR_INVALID_ARG, "%s: bad dtype", who);
    if (x_dt == HETA_BF16 && go_dt == HETA_F32) return fail(HETA_ERR_UNSUPPORTED, "%s: bf16 rows have a bf16 gradient", who);
    const size_t esz = dtype_size(x_dt), gsz = dtype_size(go_dt);
    HETA_TRY(check_rows(who, "x", x, n_rows, ld_x, d, esz));
    HETA_TRY(check_rows(who, "grad_out", grad_out, n_rows, ld_go, d, gsz));
    HETA_TRY(check_rows(who, "grad_x", grad_x, n_rows, ld_gx, d, esz));
    if (grad_sum) HETA_TRY(check_rows(who, "grad_sum", grad_sum, n_rows, ld_gs, d, esz));
    if (!rstd && n_rows > 0) return fail(HETA_ERR_INVALID_ARG, "%s: null rstd", who);
    for (const float *v : {gamma, rstd, static_cast<const float *>(grad_gamma)})
        if (reinterpret_cast<uintptr_t>(v) & 3u) return fail(HETA_ERR_INVALID_ARG, "%s: pointer not aligned to its element size", who);
    const RowRange rx(x, n_rows, ld_x, d, esz), rg(grad_out, n_rows, ld_go, d, gsz), rs(grad_sum, n_rows, ld_gs, d, esz), ro(grad_x, n_rows, ld_gx, d, esz);
    // grad_x may be grad_sum (the same lane reads and writes); rows of more than 2,048 columns read x and grad_out twice
    if (ro.overlaps(rx) || ro.overlaps(rg) || (ro.overlaps(rs) && !(grad_x == grad_sum && ld_gx == ld_gs)))
        return fail(HETA_ERR_INVALID_ARG, "%s: grad_x overlaps an operand", who);
    const RowRange rgamma(gamma, 1, d, d, 4), rrstd(rstd, 1, n_rows, n_rows, 4), rgg(grad_gamma, 1, d, d, 4);
    if (ro.overlaps(rgamma) || ro.overlaps(rrstd)) return fail(HETA_ERR_INVALID_ARG, "%s: grad_x overlaps an operand", who);
    for (const RowRange &v : {rx, rg, rs, ro, rgamma, rrstd})
        if (rgg.overlaps(v)) return fail(HETA_ERR_INVALID_ARG, "%s: grad_gamma overlaps an operand or grad_x", who);
    int64_t n_part = 0;
    by_width(d, [&](auto lanes, auto) { n_part = row_blocks(n_rows, 256 / decltype(lanes)::value, kNormBwdBlocks); }, [&] { n_part = row_blocks(n_rows, 32, 256); });
    if (n_rows == 0) n_part = 0;
    if (grad_gamma) HETA_TRY(ensure_workspace(g, static_cast<size_t>(std::max<int64_t>(n_part, 1)) * d * sizeof(float)));
    float *part = grad_gamma ? static_cast<float *>(g->d_ws) : nullptr;
    hipStream_t st = as_stream(hip_stream);
    if (n_rows > 0) {
        const NormBwd p{x, grad_out, grad_sum, grad_x, gamma, rstd, part, ld_x, ld_go, ld_gs, ld_gx, n_rows, d};
        const double bytes = static_cast<double>(n_rows) * d * (esz * (2.0 + !!grad_sum) + gsz);
        const bool stream = streams(bytes);
        ProfScope prof("rms_norm_bwd_kernel", st, bytes, 9.0 * n_rows * d);
        if (x_dt == HETA_BF16) launch_norm_bwd<bf16_t, bf16_t>(p, stream, n_part, st);
        else if (go_dt == HETA_F32) launch_norm_bwd<float, float>(p, stream, n_part, st);
        else launch_norm_bwd<float, bf16_t>(p, stream, n_part, st);
        HETA_LAUNCH_CHECK("rms_norm_bwd_kernel");
    }
    return grad_gamma ? fold_partials(part, n_part, d, grad_gamma, HETA_F32, d, d, st) : HETA_OK;
}
