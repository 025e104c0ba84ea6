// Consecutive elements of a row as fp32, for kernels that read and write rows of either element type (not part of the ABI).
// Rows need no alignment beyond their elements': global memory takes 16-byte accesses at any address.
#pragma once

#include "heta_gemm.h"

namespace heta {

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(bf16_t x) { return __uint_as_float(static_cast<uint32_t>(x) << 16); }

// 16 bytes at any address; STREAM: with the hint that they will not be needed again soon
typedef uint32_t uintx4 __attribute__((ext_vector_type(4)));
typedef uint32_t uintx4_any __attribute__((ext_vector_type(4), aligned(1)));
template <bool STREAM = false> __device__ __forceinline__ uintx4 load16(const void *p)
{
    if constexpr (STREAM) return __builtin_nontemporal_load(static_cast<const uintx4_any *>(p));
    else return *static_cast<const uintx4_any *>(p);
}
template <bool STREAM = false> __device__ __forceinline__ void store16(void *p, uintx4 v)
{
    if constexpr (STREAM) __builtin_nontemporal_store(v, static_cast<uintx4_any *>(p));
    else *static_cast<uintx4_any *>(p) = v;
}

// eight elements, `valid` of which exist (others read as 0)
template <bool STREAM = false> __device__ __forceinline__ void load8(const float *p, int valid, float (&v)[8])
{
    if (valid >= 8) {
        const uintx4 a = load16<STREAM>(p), b = load16<STREAM>(p + 4);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[j] = __uint_as_float(a[j]);
            v[4 + j] = __uint_as_float(b[j]);
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < valid ? p[e] : 0.f;
}
template <bool STREAM = false> __device__ __forceinline__ void load8(const bf16_t *p, int valid, float (&v)[8])
{
    if (valid >= 8) {
        const uintx4 a = load16<STREAM>(p);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[2 * j] = __uint_as_float(a[j] << 16);
            v[2 * j + 1] = __uint_as_float(a[j] & 0xffff0000u);
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < valid ? widen(p[e]) : 0.f;
}
template <bool STREAM = false> __device__ __forceinline__ void store8(float *p, int valid, const float (&v)[8])
{
    if (valid >= 8) {
        const uintx4 a = {__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
        const uintx4 b = {__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7])};
        store16<STREAM>(p, a);
        store16<STREAM>(p + 4, b);
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (e < valid) p[e] = v[e];
}
template <bool STREAM = false> __device__ __forceinline__ void store8(bf16_t *p, int valid, const float (&v)[8])
{
    if (valid >= 8) {
        const uintx4 a = {pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3]), pack2_bf16(v[4], v[5]), pack2_bf16(v[6], v[7])};
        store16<STREAM>(p, a);
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (e < valid) p[e] = static_cast<bf16_t>(pack2_bf16(v[e], v[e]) & 0xffffu);
}

// 16 bytes of outputs (valid of their elements exist) from fp32, and as they lie in memory
template <typename O> __device__ __forceinline__ uintx4 pack16(const float (&y)[16 / sizeof(O)])
{
    if constexpr (sizeof(O) == 2) return uintx4{pack2_bf16(y[0], y[1]), pack2_bf16(y[2], y[3]), pack2_bf16(y[4], y[5]), pack2_bf16(y[6], y[7])};
    else return uintx4{__float_as_uint(y[0]), __float_as_uint(y[1]), __float_as_uint(y[2]), __float_as_uint(y[3])};
}
template <typename O> __device__ __forceinline__ void unpack16(uintx4 w, float (&y)[16 / sizeof(O)])
{
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (sizeof(O) == 2) {
            y[2 * j] = __uint_as_float(w[j] << 16);
            y[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
        } else {
            y[j] = __uint_as_float(w[j]);
        }
    }
}
template <typename O> __device__ __forceinline__ void store_piece(O *p, int valid, uintx4 w)
{
    constexpr int W = 16 / (int)sizeof(O);
    if (valid >= W) {
        store16(p, w);
        return;
    }
#pragma unroll
    for (int e = 0; e < W; ++e)
        if (e < valid) {
            if constexpr (sizeof(O) == 2) p[e] = static_cast<O>(w[e / 2] >> (16 * (e & 1)));
            else p[e] = __uint_as_float(w[e]);
        }
}
template <typename O> __device__ __forceinline__ uintx4 load_piece(const O *p, int valid)
{
    constexpr int W = 16 / (int)sizeof(O);
    if (valid >= W) return load16(p);
    uintx4 w = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int e = 0; e < W; ++e)
        if (e < valid) {
            if constexpr (sizeof(O) == 2) w[e / 2] |= static_cast<uint32_t>(p[e]) << (16 * (e & 1));
            else w[e] = __float_as_uint(p[e]);
        }
    return w;
}

// 8-bit rows.  |v| as an integer: ordered like the magnitudes, infinity above the numbers and NaN above infinity, so that the largest of a
// row with a NaN is NaN (fmaxf drops it).
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }
// What the values of a row (or column) whose largest magnitude is amax are multiplied by, and its scale, which may be subnormal.  Below 2^-119
// the factor 448 / amax leaves fp32's range: such rows count as zeros.  NaN makes scale and values NaN.
constexpr float kE4m3Least = 1.504632769052528e-36f; // 2^-119
__device__ __forceinline__ float e4m3_factor(float amax) { return amax >= kE4m3Least ? 448.f / amax : amax != amax ? amax : 0.f; }
__device__ __forceinline__ float e4m3_scale(float amax) { return amax < kE4m3Least ? 0.f : amax / 448.f; }

// Argument checks of the calls on such rows (host).  Widths stay a little below 2^31: kernels count columns in 32 bits, a workgroup's at a time.
constexpr int32_t kWidest = INT32_MAX - 1023;
inline heta_status check_rows(const char *who, const char *what, const void *p, int64_t n_rows, int64_t ld, int64_t d, size_t elt)
{
    if (!p && n_rows > 0) return fail(HETA_ERR_INVALID_ARG, "%s: null %s", who, what);
    if (ld < d) return fail(HETA_ERR_SHAPE, "%s: leading dimension of %s is below its width", who, what);
    if (reinterpret_cast<uintptr_t>(p) % elt) return fail(HETA_ERR_INVALID_ARG, "%s: %s is not aligned to its element size", who, what);
    return HETA_OK;
}

// Calls that move more than the chip's 256 MB last-level cache holds read and write with the streaming hint; below, what a
// call writes is still cached when the next one reads it.
inline bool streams(double bytes) { return bytes > 256e6; }

// out[c] (or, for rows of `width`, out[(c / width) * ld + c % width]) = sum over s < n_part of part[s * total + c], c < total,
// in a fixed order; out is fp32 or bf16.  Deterministic second half of sums over rows that many workgroups share.
constexpr int64_t kFoldMost = int64_t(256) * (max_blocks(256) - 1); // columns
heta_status fold_partials(const float *part, int64_t n_part, int64_t total, void *out, heta_dtype out_dt, int32_t width, int64_t ld, hipStream_t st);

} // namespace heta
