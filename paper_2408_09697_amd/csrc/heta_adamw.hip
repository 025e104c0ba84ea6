// Adam with decoupled weight decay over the tensors of a model, states in fp32 or in 8 bits.
//
//     m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,  W = (1 - lr wd) W - lr c1 m / (sqrt(v) sqrt(c2) + eps),  c = 1 / (1 - b^step)
//
// 8-bit states are m and r = sqrt(v) (half of v's range of exponents), e4m3 with a scale for each 128 columns of a row: the largest
// magnitude of the block is 448.  They are read as numbers, advanced in fp32 and rounded up or down with the probability that makes
// the mean right, by 16 bits of a hash of the element's place, the step and a seed.  Rounded to the nearest, r would stand
// still: with b2 = 0.999 a step moves it by 0.05 %, and neighbours of e4m3 are 6 to 12 % apart.  r > 0 is kept at least at the
// smallest code, so that no m is ever divided by the r = 0 of an element that has had a gradient: |m| / r stays below the ratio of the two
// scales whatever is rounded.  Every product and sum is rounded on its own (no contraction): the kernels agree bit for bit.
//
// HBM-bound: 28 bytes an element with fp32 throughout, 10.1 with bf16 weights and gradients and 8-bit states.  A lane holds eight
// consecutive columns; a block of 128 columns is 16 lanes, which join their largest magnitudes by shuffles.
#include <algorithm>
#include <cmath>

#include "heta_rows.h"

namespace heta {

struct AdamwHyper {
    float lr_c1, beta1, one_less_beta1, beta2, one_less_beta2, root_c2, eps;
};

// An update of consecutive elements with fp32 states.
struct AdamwFlat {
    void *W;
    const void *grad;
    float *m, *v;
    int64_t n;
    float keep; // 1 - lr weight_decay
    uint32_t block0;
};
constexpr int kAdamwFlat = 64;
struct AdamwFlatCall {
    AdamwFlat item[kAdamwFlat];
    AdamwHyper h;
    int n;
    uint32_t first; // first workgroup of this launch
};

// An update of rows.
struct AdamwRows {
    void *W;
    const void *grad;
    void *m, *v;
    float *m_scale, *v_scale; // 8-bit states
    const int64_t *ids;       // nullable: the first n rows
    int64_t ld_w, ld_grad, ld_state, ld_scale, n, rows;
    int32_t d, per_row;       // blocks of 128 columns of a row
    float keep;
    uint32_t key0, key1, block0;
    int32_t lanes_log;        // lanes of a block: 16, or fewer for narrower rows
};
constexpr int kAdamwRows = 24;
struct AdamwRowsCall {
    AdamwRows item[kAdamwRows];
    AdamwHyper h;
    int n;
    uint32_t first;
};
static_assert(sizeof(AdamwFlatCall) <= 3584 && sizeof(AdamwRowsCall) <= 3584, "kernel arguments are limited to 4 KB");

// The item whose workgroups `block` is among; a lane looks at an item.
template <typename Call> __device__ __forceinline__ int item_of(const Call &q, uint32_t block)
{
    const int lane = threadIdx.x & 63;
    const uint64_t before = __ballot(lane < q.n && block >= q.item[lane < q.n ? lane : 0].block0);
    return __popcll(before) - 1;
}

__device__ __forceinline__ void advance_states(const AdamwHyper &h, float g, float &m, float &v)
{
#pragma clang fp contract(off)
    m = h.beta1 * m + h.one_less_beta1 * g;
    v = h.beta2 * v + h.one_less_beta2 * g * g;
}
// r = sqrt(v).  The quotient by the hardware's reciprocal (one unit in the last place; the denominator is 0 or at least 1e-23).
__device__ __forceinline__ float advance_weight(const AdamwHyper &h, float keep, float m, float r, float w)
{
#pragma clang fp contract(off)
    return w * keep - h.lr_c1 * m * __builtin_amdgcn_rcpf(r * h.root_c2 + h.eps);
}

template <typename WT, typename GT> __global__ void __launch_bounds__(256) adamw_flat_kernel(AdamwFlatCall q)
{
    const uint32_t block = q.first + blockIdx.x;
    const AdamwFlat &p = q.item[item_of(q, block)];
    const int64_t at = (static_cast<int64_t>(block - p.block0) * 256 + threadIdx.x) * 8;
    if (at >= p.n) return;
    const int valid = static_cast<int>(min(p.n - at, static_cast<int64_t>(8)));
    float w[8], g[8], m[8], v[8];
    load8(static_cast<const WT *>(p.W) + at, valid, w);
    load8(static_cast<const GT *>(p.grad) + at, valid, g);
    load8(p.m + at, valid, m);
    load8(p.v + at, valid, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        advance_states(q.h, g[e], m[e], v[e]);
        w[e] = advance_weight(q.h, p.keep, m[e], sqrtf(v[e]), w[e]);
    }
    store8(static_cast<WT *>(p.W) + at, valid, w);
    store8(p.m + at, valid, m);
    store8(p.v + at, valid, v);
}

// 32 bits for the element that `x` stands for: two rounds of multiplication and shifts (the 32-bit finalizer of MurmurHash3, which Appleby published in 2011, a bijection in which every
// bit of the input changes about half of the output's), a key in front of each; x has the first one already.
__device__ __forceinline__ uint32_t element_bits(uint32_t x, uint32_t key1)
{
    x ^= x >> 16;
    x *= 0x85ebca6bu;
    x ^= x >> 13;
    x += key1;
    x *= 0xc2b2ae35u;
    return x ^ (x >> 16);
}

// The root of a v from 2^-100 up: y = 1 / sqrt(v) to one unit in the last place, g = v y, and Newton's step g + (v - g^2) y / 2.  It is the correctly
// rounded root for every one of the 2^24 significands of two binades, and so for all (the remainder v - g^2 is exact as long as it is no subnormal).
constexpr uint32_t kQuickLeast = 27u << 23, kQuickRange = 0x7f800000u - kQuickLeast; // 2^-100, and from there to infinity, as they are held
__device__ __forceinline__ float quick_root(float v)
{
    const float y = __builtin_amdgcn_rsqf(v), g = v * y;
    return fmaf(fmaf(-g, g, v), 0.5f * y, g);
}

// What a block's values are multiplied by, and its scale, as in the other 8-bit rows but by reciprocals.
__device__ __forceinline__ float state_factor(float amax) { return amax >= kE4m3Least ? 1.f / amax * 448.f : amax != amax ? amax : 0.f; }
__device__ __forceinline__ float state_scale(float amax) { return amax < kE4m3Least ? 0.f : amax * (1.f / 448.f); }

__device__ __forceinline__ void decode8(const Codes8 &q, float scale, float (&x)[8])
{
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(q.w[j], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(q.w[j], true);
        x[4 * j] = lo[0] * scale;
        x[4 * j + 1] = lo[1] * scale;
        x[4 * j + 2] = hi[0] * scale;
        x[4 * j + 3] = hi[1] * scale;
    }
}

template <typename WT, typename GT, bool CODES, bool STREAM> __global__ void __launch_bounds__(256) adamw_rows_kernel(AdamwRowsCall q)
{
    const uint32_t block = q.first + blockIdx.x;
    const AdamwRows &p = q.item[item_of(q, block)];
    const int lanes = 1 << p.lanes_log, l = threadIdx.x & (lanes - 1);
    const int64_t unit = static_cast<int64_t>(block - p.block0) * (256 >> p.lanes_log) + (threadIdx.x >> p.lanes_log);
    // below 2^31 units (uniform; a unit is at most 255 past them) row and block come from a 32-bit division
    const int64_t i = p.n * p.per_row <= 0x7fffffff ? static_cast<int64_t>(static_cast<uint32_t>(unit) / static_cast<uint32_t>(p.per_row)) : unit / p.per_row;
    const int b = static_cast<int>(unit - i * p.per_row);
    int c = b * 128 + l * 8;
    if (i >= p.n) return;
    const int64_t row = p.ids ? p.ids[i] : i;
    if (row < 0 || row >= p.rows) return; // a row id outside the tensor: nothing is read or written for it
    int valid = max(0, min(p.d - c, 8));
    // The last lane of a row's last block steps back to its last eight columns: it does again, bit for bit, what its neighbour does with some of them (both are in one
    // wavefront: what either reads, it reads before either writes).  Element by element, the rest of a row takes 8 accesses for each array.
    if (valid > 0 && valid < 8 && l > 0) {
        c -= 8 - valid;
        valid = 8;
    }
    float w[8], g[8], m[8], v[8], r[8];
    WT *const wp = static_cast<WT *>(p.W) + row * p.ld_w + c;
    load8<STREAM>(wp, valid, w);
    load8<STREAM>(static_cast<const GT *>(p.grad) + i * p.ld_grad + c, valid, g);
    if constexpr (!CODES) {
        float *const mp = static_cast<float *>(p.m) + row * p.ld_state + c, *const vp = static_cast<float *>(p.v) + row * p.ld_state + c;
        load8<STREAM>(mp, valid, m);
        load8<STREAM>(vp, valid, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            advance_states(q.h, g[e], m[e], v[e]);
            w[e] = advance_weight(q.h, p.keep, m[e], sqrtf(v[e]), w[e]);
        }
        store8<STREAM>(wp, valid, w);
        store8<STREAM>(mp, valid, m);
        store8<STREAM>(vp, valid, v);
    } else {
        uint8_t *const mp = static_cast<uint8_t *>(p.m) + row * p.ld_state + c, *const rp = static_cast<uint8_t *>(p.v) + row * p.ld_state + c;
        float *const ms = p.m_scale + row * p.ld_scale + b, *const rs = p.v_scale + row * p.ld_scale + b;
        Codes8 mc = load_codes(mp, valid), rc = load_codes(rp, valid);
        decode8(mc, *ms, m);
        decode8(rc, *rs, r);
        uint32_t top_m = 0, top_r = 0, range = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            v[e] = r[e] * r[e];
            advance_states(q.h, g[e], m[e], v[e]);
            range = max(range, __float_as_uint(v[e]) - kQuickLeast);
        }
        // the compiler's root takes 15 operations (a table of 1.1 M x 256, bf16 weights and gradients: 619 us for 594)
        if (__any(valid > 0 && range >= kQuickRange)) {
#pragma unroll
            for (int e = 0; e < 8; ++e) r[e] = sqrtf(v[e]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) r[e] = quick_root(v[e]);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            w[e] = advance_weight(q.h, p.keep, m[e], r[e], w[e]);
            if (e < valid) {
                top_m = max(top_m, magnitude(m[e]));
                top_r = max(top_r, magnitude(r[e]));
            }
        }
        store8<STREAM>(wp, valid, w);
        for (int o = lanes >> 1; o > 0; o >>= 1) {
            top_m = max(top_m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top_m), o)));
            top_r = max(top_r, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top_r), o)));
        }
        const float am = __uint_as_float(top_m), ar = __uint_as_float(top_r), fm = state_factor(am), fr = state_factor(ar);
        const float least = fr > 0.f ? 0.001953125f : 0.f; // the smallest code
        const uint64_t place = static_cast<uint64_t>(row) * static_cast<uint64_t>(p.d) + c;
        const uint32_t lo = static_cast<uint32_t>(place), base = lo + static_cast<uint32_t>(place >> 32) * 0x9e3779b9u + p.key0;
        uint32_t x[8];
#pragma unroll
        for (uint32_t e = 0; e < 8; ++e) x[e] = base + e;
        if (__any(lo > 0xfffffff8u)) { // a chunk across a multiple of 2^32
#pragma unroll
            for (uint32_t e = 0; e < 8; ++e) x[e] += lo + e < lo ? 0x9e3779b9u : 0u;
        }
        // The hardware's conversion adds the upper 20 of its 32 random bits below the last place that is kept, subnormal codes included, and cuts the
        // rest off; 448 is its largest result.  A block with a NaN or an infinity is NaN by its scale, whatever the codes.
        int words[4] = {0, 0, 0, 0};
        auto code = [&](auto element) {
            constexpr int e = decltype(element)::value;
            const uint32_t bits = element_bits(x[e], p.key1);
            words[e / 4] = __builtin_amdgcn_cvt_sr_fp8_f32(m[e] * fm, bits << 16, words[e / 4], e % 4);
            words[2 + e / 4] = __builtin_amdgcn_cvt_sr_fp8_f32(fmaxf(r[e] * fr, r[e] > 0.f ? least : 0.f), bits & 0xffff0000u, words[2 + e / 4], e % 4);
        };
        code(std::integral_constant<int, 0>{});
        code(std::integral_constant<int, 1>{});
        code(std::integral_constant<int, 2>{});
        code(std::integral_constant<int, 3>{});
        code(std::integral_constant<int, 4>{});
        code(std::integral_constant<int, 5>{});
        code(std::integral_constant<int, 6>{});
        code(std::integral_constant<int, 7>{});
        mc = Codes8{{static_cast<uint32_t>(words[0]), static_cast<uint32_t>(words[1])}};
        rc = Codes8{{static_cast<uint32_t>(words[2]), static_cast<uint32_t>(words[3])}};
        store_codes(mp, valid, mc);
        store_codes(rp, valid, rc);
        if (l == 0) {
            *ms = state_scale(am);
            *rs = state_scale(ar);
        }
    }
}

// ---- host side ---------------------------------------------------------------------------------------
static uint32_t mix32(uint32_t x)
{
    x ^= x >> 16;
    x *= 0x85ebca6bu;
    x ^= x >> 13;
    x *= 0xc2b2ae35u;
    return x ^ (x >> 16);
}

static heta_status check_item(const char *who, const heta_adamw_item &it)
{
    if (!valid_dtype(it.dt) || !valid_dtype(it.grad_dt) || (it.state_dt != HETA_F32 && it.state_dt != HETA_E4M3)) return fail(HETA_ERR_INVALID_ARG, "%s: bad dtype", who);
    if (it.d <= 0 || it.rows < 0 || it.n < 0) return fail(HETA_ERR_SHAPE, "%s: need d > 0 and non-negative counts", who);
    if (it.d > kWidest) return fail(HETA_ERR_UNSUPPORTED, "%s: rows too wide", who);
    if (!it.ids && it.n > it.rows) return fail(HETA_ERR_SHAPE, "%s: %lld gradient rows for a tensor of %lld rows", who, (long long)it.n, (long long)it.rows);
    const bool codes = it.state_dt == HETA_E4M3;
    if (codes != (it.m_scale != nullptr) || codes != (it.v_scale != nullptr))
        if (!(codes && it.rows == 0)) return fail(HETA_ERR_INVALID_ARG, "%s: scales belong to 8-bit states, and those need them", who);
    const size_t ssz = codes ? 1 : 4;
    HETA_TRY(check_rows(who, "W", it.W, it.rows, it.ld_w, it.d, dtype_size(it.dt)));
    HETA_TRY(check_rows(who, "grad", it.grad, it.n, it.ld_grad, it.d, dtype_size(it.grad_dt)));
    HETA_TRY(check_rows(who, "m", it.m, it.rows, it.ld_state, it.d, ssz));
    HETA_TRY(check_rows(who, "v", it.v, it.rows, it.ld_state, it.d, ssz));
    if (codes) {
        HETA_TRY(check_rows(who, "m_scale", it.m_scale, it.rows, it.ld_scale, (it.d + 127) / 128, 4));
        HETA_TRY(check_rows(who, "v_scale", it.v_scale, it.rows, it.ld_scale, (it.d + 127) / 128, 4));
    }
    if (reinterpret_cast<uintptr_t>(it.ids) & 7u) return fail(HETA_ERR_INVALID_ARG, "%s: pointer not aligned to its element size", who);
    if (!(it.weight_decay >= 0.f)) return fail(HETA_ERR_INVALID_ARG, "%s: need weight_decay >= 0", who);
    return HETA_OK;
}

// No array that is written may overlap another one, of its own item or of another.  Ranges in order of address: one that begins
// behind all before it overlaps none; where one does not, every pair of those that touch is looked at (column slices of one buffer are apart).
struct Touched {
    RowRange r;
    bool written;
};
static bool arrays_collide(std::vector<Touched> &all)
{
    std::sort(all.begin(), all.end(), [](const Touched &a, const Touched &b) { return a.r.lo < b.r.lo; });
    for (size_t i = 0; i < all.size(); ++i)
        for (size_t j = i + 1; j < all.size() && all[j].r.lo < all[i].r.hi; ++j)
            if ((all[i].written || all[j].written) && all[i].r.overlaps(all[j].r)) return true;
    return false;
}

// Flat items share launches of one pair of types, row items those of one pair of types and states.
template <typename Item, typename Call, int MOST, typename Launch>
static heta_status launch_items(const std::vector<Item> &items, const AdamwHyper &h, int64_t (*blocks_of)(const Item &), Launch launch)
{
    for (size_t i = 0; i < items.size();) {
        Call q{};
        q.h = h;
        int64_t blocks = 0;
        while (i < items.size() && q.n < MOST) {
            const int64_t b = blocks_of(items[i]);
            if (q.n > 0 && blocks + b > (int64_t(1) << 31)) break;
            q.item[q.n] = items[i++];
            q.item[q.n++].block0 = static_cast<uint32_t>(blocks);
            blocks += b;
        }
        launch_pieces(blocks, 256, [&](unsigned first, unsigned count) {
            q.first = first;
            launch(q, count);
        });
        HETA_LAUNCH_CHECK("adamw kernel");
    }
    return HETA_OK;
}
static int64_t flat_blocks(const AdamwFlat &p) { return (p.n + 2047) / 2048; }
static int64_t row_blocks(const AdamwRows &p)
{
    const int64_t each = 256 >> p.lanes_log;
    return (p.n * p.per_row + each - 1) / each;
}

// f(tag of W's type, tag of the gradient's)
template <typename F> static void with_types(int k, F f)
{
    if (k == 0) f(float{}, float{});
    else if (k == 1) f(float{}, bf16_t{});
    else if (k == 2) f(bf16_t{}, float{});
    else f(bf16_t{}, bf16_t{});
}

static heta_status adamw(int32_t n_items, const heta_adamw_item *items, float lr, float beta1, float beta2, float eps, int64_t step, hipStream_t st)
{
    const char *who = "heta_adamw_multi";
    if (n_items < 0 || (n_items > 0 && !items)) return fail(HETA_ERR_INVALID_ARG, "%s: bad item list", who);
    if (step < 1) return fail(HETA_ERR_INVALID_ARG, "%s: the step counter starts at 1", who);
    if (!(beta1 >= 0.f && beta1 < 1.f) || !(beta2 >= 0.f && beta2 < 1.f) || !(eps >= 0.f))
        return fail(HETA_ERR_INVALID_ARG, "%s: need 0 <= beta1, beta2 < 1 and eps >= 0", who);
    AdamwHyper h;
    h.beta1 = beta1;
    h.beta2 = beta2;
    h.eps = eps;
    h.one_less_beta1 = static_cast<float>(1.0 - static_cast<double>(beta1));
    h.one_less_beta2 = static_cast<float>(1.0 - static_cast<double>(beta2));
    h.lr_c1 = static_cast<float>(lr / (1.0 - std::pow(static_cast<double>(beta1), static_cast<double>(step))));
    h.root_c2 = static_cast<float>(std::sqrt(1.0 / (1.0 - std::pow(static_cast<double>(beta2), static_cast<double>(step)))));
    std::vector<AdamwFlat> flat[4];
    std::vector<AdamwRows> rows[8];
    std::vector<Touched> touched;
    touched.reserve(static_cast<size_t>(n_items) * 5);
    double flat_bytes = 0, rows_bytes = 0;
    bool listed = true; // all of the items that are updated by rows are lists
    for (int32_t i = 0; i < n_items; ++i) {
        const heta_adamw_item &it = items[i];
        HETA_TRY(check_item(who, it));
        if (it.n == 0) continue;
        const bool codes = it.state_dt == HETA_E4M3;
        const size_t wsz = dtype_size(it.dt), gsz = dtype_size(it.grad_dt), ssz = codes ? 1 : 4;
        const int64_t last = it.ids ? it.rows : it.n;
        touched.push_back({RowRange(it.W, last, it.ld_w, it.d, wsz), true});
        touched.push_back({RowRange(it.m, last, it.ld_state, it.d, ssz), true});
        touched.push_back({RowRange(it.v, last, it.ld_state, it.d, ssz), true});
        touched.push_back({RowRange(it.grad, it.n, it.ld_grad, it.d, gsz), false});
        if (it.ids) touched.push_back({RowRange(it.ids, 1, it.n, it.n, 8), false});
        if (codes) {
            touched.push_back({RowRange(it.m_scale, last, it.ld_scale, (it.d + 127) / 128, 4), true});
            touched.push_back({RowRange(it.v_scale, last, it.ld_scale, (it.d + 127) / 128, 4), true});
        }
        const int types = (it.dt == HETA_BF16 ? 2 : 0) + (it.grad_dt == HETA_BF16 ? 1 : 0);
        const float keep = static_cast<float>(1.0 - static_cast<double>(lr) * it.weight_decay);
        const double bytes = static_cast<double>(it.n) * (it.d * (2.0 * wsz + gsz + 4.0 * ssz) + (codes ? 16.0 * ((it.d + 127) / 128) : 0.0) + (it.ids ? 8.0 : 0.0));
        const bool whole = it.n == 1 || (it.ld_w == it.d && it.ld_grad == it.d && it.ld_state == it.d);
        if (!codes && !it.ids && whole) {
            flat[types].push_back({it.W, it.grad, static_cast<float *>(it.m), static_cast<float *>(it.v), it.n * it.d, keep, 0});
            flat_bytes += bytes;
            continue;
        }
        AdamwRows p{it.W, it.grad, it.m, it.v, it.m_scale, it.v_scale, it.ids, it.ld_w, it.ld_grad, it.ld_state, it.ld_scale, it.n, it.rows, it.d, (it.d + 127) / 128, keep, 0, 0, 0, 4};
        while (p.lanes_log > 0 && it.d <= 4 << p.lanes_log) --p.lanes_log;
        p.key0 = mix32(it.seed + 0x9e3779b9u * static_cast<uint32_t>(step));
        p.key1 = mix32(p.key0 + 0x7f4a7c15u);
        if (row_blocks(p) > (int64_t(1) << 31)) return fail(HETA_ERR_UNSUPPORTED, "%s: too many elements for one launch", who);
        listed = listed && it.ids;
        rows[types + (codes ? 4 : 0)].push_back(p);
        rows_bytes += bytes;
    }
    for (const auto &f : flat)
        for (const AdamwFlat &p : f)
            if (flat_blocks(p) > (int64_t(1) << 31)) return fail(HETA_ERR_UNSUPPORTED, "%s: too many elements for one launch", who);
    if (arrays_collide(touched)) return fail(HETA_ERR_INVALID_ARG, "%s: an array that is written overlaps another one", who);
    if (flat_bytes > 0) {
        ProfScope prof("adamw_flat_kernel", st, flat_bytes, 0);
        for (int k = 0; k < 4; ++k) {
            heta_status e = HETA_OK;
            with_types(k, [&](auto w, auto g) {
                e = launch_items<AdamwFlat, AdamwFlatCall, kAdamwFlat>(flat[k], h, flat_blocks, [&](const AdamwFlatCall &q, unsigned count) {
                    hipLaunchKernelGGL((adamw_flat_kernel<decltype(w), decltype(g)>), dim3(count), dim3(256), 0, st, q);
                });
            });
            if (e != HETA_OK) return e;
        }
    }
    if (rows_bytes > 0) {
        ProfScope prof("adamw_rows_kernel", st, rows_bytes, 0);
        for (int k = 0; k < 8; ++k) {
            heta_status e = HETA_OK;
            with_types(k & 3, [&](auto w, auto g) {
                e = launch_items<AdamwRows, AdamwRowsCall, kAdamwRows>(rows[k], h, row_blocks, [&](const AdamwRowsCall &q, unsigned count) {
                    auto go = [&](auto codes, auto stream) {
                        hipLaunchKernelGGL((adamw_rows_kernel<decltype(w), decltype(g), decltype(codes)::value, decltype(stream)::value>), dim3(count), dim3(256), 0, st, q);
                    };
                    // Listed rows of more than the last-level cache holds are read and written with the streaming hint (200,000 of 1 M rows, 189 columns, fp32 with 8-bit
                    // states: 191 us without, 179); whole tensors are faster without (1 M x 128: fp32 states 657 us, 695 with it; 8 bits 380, 394).
                    const bool stream = listed && streams(rows_bytes);
                    if (k >= 4) stream ? go(std::true_type{}, std::true_type{}) : go(std::true_type{}, std::false_type{});
                    else stream ? go(std::false_type{}, std::true_type{}) : go(std::false_type{}, std::false_type{});
                });
            });
            if (e != HETA_OK) return e;
        }
    }
    return HETA_OK;
}

} // namespace heta

using namespace heta;

extern "C" heta_status heta_adamw_multi(int32_t n_items, const heta_adamw_item *items, float lr, float beta1, float beta2, float eps, int64_t step, void *hip_stream)
{
    try {
        return adamw(n_items, items, lr, beta1, beta2, eps, step, as_stream(hip_stream));
    } catch (const std::exception &) {
        return fail(HETA_ERR_OOM, "heta_adamw_multi: no memory for the list of items");
    }
}
