// Eight consecutive elements of a row as fp32, for kernels that read and write rows of either element type (not part of
// the ABI).  `vec`: the rows are 16-byte aligned; `valid`: elements of the eight that exist (others read as 0).
#pragma once

#include "heta_gemm.h"

namespace heta {

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(bf16_t x) { return __uint_as_float(static_cast<uint32_t>(x) << 16); }

__device__ __forceinline__ void load8(const float *p, int valid, bool vec, float (&v)[8])
{
    if (vec && valid >= 8) {
        const float4 a = reinterpret_cast<const float4 *>(p)[0], b = reinterpret_cast<const float4 *>(p)[1];
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < valid ? p[e] : 0.f;
}
__device__ __forceinline__ void load8(const bf16_t *p, int valid, bool vec, float (&v)[8])
{
    if (vec && valid >= 8) {
        const uint4 a = *reinterpret_cast<const uint4 *>(p);
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[2 * j] = __uint_as_float(w[j] << 16);
            v[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < valid ? widen(p[e]) : 0.f;
}
__device__ __forceinline__ void store8(float *p, int valid, bool vec, const float (&v)[8])
{
    if (vec && valid >= 8) {
        reinterpret_cast<float4 *>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
        reinterpret_cast<float4 *>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (e < valid) p[e] = v[e];
}
__device__ __forceinline__ void store8(bf16_t *p, int valid, bool vec, const float (&v)[8])
{
    if (vec && valid >= 8) {
        *reinterpret_cast<uint4 *>(p) = make_uint4(pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3]), pack2_bf16(v[4], v[5]), pack2_bf16(v[6], v[7]));
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (e < valid) p[e] = static_cast<bf16_t>(pack2_bf16(v[e], v[e]) & 0xffffu);
}

// rows of `ld` elements from p on that can be moved 16 bytes at a time (a null pointer can: it is not read)
inline bool vec_rows(const void *p, int64_t ld, size_t elt) { return !p || (aligned16(p) && (ld * static_cast<int64_t>(elt)) % 16 == 0); }

// out[c] (or, for rows of `width`, out[(c / width) * ld + c % width]) = sum over s < n_part of part[s * total + c], c < total,
// in a fixed order; out is fp32 or bf16.  Deterministic second half of sums over rows that many workgroups share.
heta_status fold_partials(const float *part, int64_t n_part, int64_t total, void *out, heta_dtype out_dt, int32_t width, int64_t ld, hipStream_t st);

} // namespace heta
