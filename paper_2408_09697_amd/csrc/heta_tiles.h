// Tiled matrix products with an epilogue of the caller's choice, on the bf16 and the 8-bit matrix pipe (not part of the
// ABI): C[M, N] = epilogue(A[M, K] . B[K, N]) for one item or for several that share a launch.
//
// Operands.  A tile lies in LDS as 16-byte chunks, in T planes (bf16 terms of the value, one for bf16 itself, three for
// fp32: see split3_pair) and in one of two layouts:
//   k-contiguous (element (r, k) at base[r * ld + k]): LDS row r holds the tile's k range, its chunks permuted by swz;
//   r-contiguous (element (r, k) at base[k * ld + r]): LDS row k, chunks at rc_place; fragments are read with the
//   transposing LDS read, so neither operand of any product is ever transposed in memory.
// It gets there straight from memory (kDirect: 16-byte aligned rows of the image's own type, T planes side by side in
// memory) or through registers (kStaged: any storage type and alignment; fp32 is split into its three terms
// there, once per workgroup, not by every wavefront that reads the tile).  A last k-tile with fewer k-values is filled up
// with zeros in LDS: fragments and products know no ragged tile.
//
// The product is formed as (B^T A^T): a lane's accumulator registers then hold consecutive COLUMNS of C, four at a time, and go
// through a strip of LDS, one 32 x 32 block per wavefront at a time, in 128-bit accesses; read back by rows, a lane has 16
// bytes of consecutive outputs, and memory sees 64 or 128 bytes of a row at a time, also for what the epilogue reads in the
// output's shape.  Stored from the registers as they lie, 32 bytes of 32 rows, products of 700,000 x 1,024 x 256 and 700,000 x 256 x 1,024
// took 477 and 622 us, with the columns in the outer loop 593 and 738, against 435 and 564 through strips.
// Outputs carry no streaming hint: with it 8-bit products of 200,000 x 1,024 x 4,096 and 700,000 x 256 x 1,024 took 1,347 and 808 us for 1,290 and
// 702, and where the output stays in the cache (20,000 x 1,024 x 4,096: 117 for 137 us) the product that reads it next loses more (351 for 335 us, both).
#pragma once

#include <algorithm>
#include <type_traits>

#include "heta_rows.h"

namespace heta {

enum TileLoad { kDirect = 0, kStaged = 1 };

typedef int intx4 __attribute__((ext_vector_type(4)));
typedef int intx8 __attribute__((ext_vector_type(8)));
typedef int intx16 __attribute__((ext_vector_type(16)));
typedef short shortx4_tr __attribute__((ext_vector_type(4)));

// ---- LDS image of one operand tile ------------------------------------------------------------------
template <bool RC, int ROWS, int BK, int EB> struct TileImage {
    static constexpr int E = 16 / EB;                  // elements per chunk
    static constexpr int CPR = RC ? ROWS / E : BK / E; // chunks per LDS row
    static constexpr int NROW = RC ? BK : ROWS;
    static constexpr int CHUNKS = NROW * CPR;
    static constexpr int BYTES = CHUNKS * 16;
    static_assert(!RC || EB == 2, "only 16-bit values are read transposed");
    static_assert(RC || CPR == 8 || CPR == 4 || CPR == 2, "the chunk permutation knows rows of 32, 64 and 128 bytes");
    static_assert(CHUNKS % 64 == 0, "a tile is a whole number of wavefront loads");
    __device__ __forceinline__ static int place(int row, int chunk)
    {
        if constexpr (RC) return (row * CPR + rc_place<CPR>(chunk, row)) * 16;
        else return (row * CPR + (chunk ^ swz<CPR>(row))) * 16;
    }
    // the chunk that lies at LDS position q (in chunks)
    __device__ __forceinline__ static int chunk_at(int q)
    {
        if constexpr (RC) return rc_chunk<CPR>(q % CPR, q / CPR);
        else return (q % CPR) ^ swz<CPR>(q / CPR);
    }
};

// ---- memory -> LDS ----------------------------------------------------------------------------------
// Rows (k-contiguous) or chunks (r-contiguous) beyond the matrix are clamped to the last one that holds a value of it:
// what they bring only reaches outputs that are not stored.  A chunk that holds a value of the matrix is 16-byte aligned
// and so within what is allocated.
template <bool RC, int ROWS, int BK, int EB, int NW, int T> struct PlaneLoader {
    using Img = TileImage<RC, ROWS, BK, EB>;
    static constexpr int SLOTS = Img::CHUNKS / 64, NI = (SLOTS + NW - 1) / NW; // every wavefront issues the same number of loads;
    static constexpr int LOADS = NI * T;                                       // surplus slots repeat one (same bytes, same place)
    const char *tile;  // uniform: the next tile's first element, plane 0
    uint32_t off[NI];  // per lane
    int64_t step, plane; // uniform, bytes
    __device__ __forceinline__ static int slot(int i, int wave) { return (i * NW + wave) % SLOTS; }
    __device__ __forceinline__ void init(const void *base, int64_t ld, int64_t plane_bytes, int64_t r0, int64_t r_total, int64_t k0, int wave, int lane)
    {
        const uint32_t ld_bytes = static_cast<uint32_t>(ld * EB);
        step = RC ? ld * BK * EB : static_cast<int64_t>(BK) * EB;
        plane = plane_bytes;
        tile = static_cast<const char *>(base) + (RC ? k0 * ld + r0 : r0 * ld + k0) * EB;
        const int64_t room = RC ? (r_total - r0 + Img::E - 1) / Img::E : r_total - r0;
        const int last = static_cast<int>(min(room, static_cast<int64_t>(RC ? Img::CPR : ROWS))) - 1;
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int q = slot(i, wave) * 64 + lane, row = q / Img::CPR, chunk = Img::chunk_at(q);
            off[i] = RC ? static_cast<uint32_t>(row) * ld_bytes + static_cast<uint32_t>(min(chunk, last)) * 16u
                        : static_cast<uint32_t>(min(row, last)) * ld_bytes + static_cast<uint32_t>(chunk) * 16u;
        }
    }
    __device__ __forceinline__ void issue(uint32_t lds, int wave)
    {
#pragma unroll
        for (int t = 0; t < T; ++t)
#pragma unroll
            for (int i = 0; i < NI; ++i) load_chunk_to_lds(tile + t * plane, off[i], lds + t * Img::BYTES + slot(i, wave) * 1024);
        tile += step;
    }
    // the last k-tile of a contraction, with only kv of its k-values: nothing beyond them is read (chunks or rows are clamped
    // to the last that holds one), and clear_tail() has to follow when the tile is there
    __device__ __forceinline__ void issue_tail(uint32_t lds, int wave, int lane, int kv, int64_t ld, int64_t r0, int64_t r_total)
    {
        const uint32_t ld_bytes = static_cast<uint32_t>(ld * EB);
        const int64_t room = RC ? (r_total - r0 + Img::E - 1) / Img::E : r_total - r0;
        const int last = static_cast<int>(min(room, static_cast<int64_t>(RC ? Img::CPR : ROWS))) - 1;
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int q = slot(i, wave) * 64 + lane, row = q / Img::CPR, chunk = Img::chunk_at(q);
            const uint32_t o = RC ? static_cast<uint32_t>(min(row, kv - 1)) * ld_bytes + static_cast<uint32_t>(min(chunk, last)) * 16u
                                  : static_cast<uint32_t>(min(row, last)) * ld_bytes + static_cast<uint32_t>(min(chunk, (kv - 1) / Img::E)) * 16u;
#pragma unroll
            for (int t = 0; t < T; ++t) load_chunk_to_lds(tile + t * plane, o, lds + t * Img::BYTES + slot(i, wave) * 1024);
        }
    }
    // zeroes what lies in the k-values from kv on
    __device__ __forceinline__ static void clear_tail(char *lds, int tid, int kv)
    {
        for (int q = tid; q < T * Img::CHUNKS; q += 64 * NW) {
            const int in = q % Img::CHUNKS, k = RC ? in / Img::CPR : Img::chunk_at(in) * Img::E; // its (first) k-value
            uint4 *p = reinterpret_cast<uint4 *>(lds) + q;
            if (k >= kv) {
                *p = make_uint4(0u, 0u, 0u, 0u);
            } else if (!RC && k + Img::E > kv) {
                uint4 u = *p;
                uint32_t w[4] = {u.x, u.y, u.z, u.w};
                const int bytes = (kv - k) * EB; // valid bytes of the chunk
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int b = bytes - 4 * j;
                    w[j] = b >= 4 ? w[j] : b <= 0 ? 0u : w[j] & ((1u << (8 * b)) - 1u);
                }
                *p = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
    }
};

// Three terms of eight values (split3_pair), also of those beyond bf16's range, whose first term would be infinite and the others NaN:
//   from 2^128 - 2^119 on: the largest bf16 number, and what is left of the value;
//   infinity: +-1, 0, +-infinity.  A product then has an infinite term only where the factor against it is the other operand's first
//   term, which is 0 for 0 alone: infinity times 0 is NaN, times anything else infinity of their signs, infinity too.
constexpr float kBeyondBf16 = 3.3961775292304957e38f; // 2^128 - 2^119
template <bool CAREFUL> __device__ __forceinline__ void split3_chunk(const float (&x)[8], uint32_t (&h)[4], uint32_t (&m)[4], uint32_t (&l)[4])
{
#pragma unroll
    for (int j = 0; j < 4; ++j) split3_pair(x[2 * j], x[2 * j + 1], h[j], m[j], l[j]);
    if constexpr (!CAREFUL) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if (!(fabsf(x[e]) >= kBeyondBf16)) continue; // NaN has NaN terms already
        const bool inf = fabsf(x[e]) > 3.402823466e38f;
        const float first = copysignf(inf ? 1.f : 3.3895313892515355e38f, x[e]), rest = inf ? 0.f : x[e] - first;
        const bf16_t mid = to_bf16(rest);
        const uint32_t t[3] = {to_bf16(first), mid, to_bf16(inf ? x[e] : rest - widen(mid))};
        const int at = 16 * (e & 1);
        h[e / 2] = (h[e / 2] & ~(0xffffu << at)) | t[0] << at;
        m[e / 2] = (m[e / 2] & ~(0xffffu << at)) | t[1] << at;
        l[e / 2] = (l[e / 2] & ~(0xffffu << at)) | t[2] << at;
    }
}

// ---- memory -> registers -> LDS ---------------------------------------------------------------------
// An item is one 16-byte chunk of the image: E consecutive elements, converted to the planes of their type.  Elements
// beyond the matrix count as zero.
template <typename S, bool RC, int ROWS, int BK, int EB, int NT, int T> struct StagedLoader {
    using Img = TileImage<RC, ROWS, BK, EB>;
    static constexpr int E = Img::E, NI = (Img::CHUNKS + NT - 1) / NT, W = E * (int)sizeof(S) / 16; // 16-byte words per item
    static_assert(W >= 1 && (T == 1 || sizeof(S) == 4), "planes are split from fp32");
    uint4 raw[NI][W];
    __device__ __forceinline__ void load(const S *base, int64_t ld, int64_t r0, int64_t r_total, int64_t k0, int64_t k_end, int tid)
    {
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int q = tid + NT * i, row = q / Img::CPR, chunk = q % Img::CPR;
            const int64_t r = RC ? r0 + chunk * E : r0 + row, k = RC ? k0 + row : k0 + chunk * E;
            const int64_t left = RC ? r_total - r : k_end - k;
            const bool in = (Img::CHUNKS % NT == 0 || q < Img::CHUNKS) && left > 0 && (RC ? k < k_end : r < r_total);
#pragma unroll
            for (int w = 0; w < W; ++w) raw[i][w] = make_uint4(0u, 0u, 0u, 0u);
            if (!in) continue;
            const S *src = base + (RC ? k * ld + r : r * ld + k);
            if (left >= E) {
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    const uintx4 q = load16(reinterpret_cast<const char *>(src) + 16 * w);
                    raw[i][w] = make_uint4(q[0], q[1], q[2], q[3]);
                }
            } else {
                union { uint4 u[W]; S s[E]; } t;
#pragma unroll
                for (int w = 0; w < W; ++w) t.u[w] = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (e < left) t.s[e] = src[e];
#pragma unroll
                for (int w = 0; w < W; ++w) raw[i][w] = t.u[w];
            }
        }
    }
    __device__ __forceinline__ void store(char *lds, int tid) const
    {
        if constexpr (T == 1) {
            put<false>(lds, tid);
        } else {
            // a wavefront with a value beyond bf16's range takes the longer way
            float top = 0.f;
#pragma unroll
            for (int i = 0; i < NI; ++i)
#pragma unroll
                for (int w = 0; w < W; ++w)
                    top = fmaxf(fmaxf(fmaxf(top, fabsf(__uint_as_float(raw[i][w].x))), fmaxf(fabsf(__uint_as_float(raw[i][w].y)), fabsf(__uint_as_float(raw[i][w].z)))),
                                fabsf(__uint_as_float(raw[i][w].w)));
            if (__builtin_expect(__any(top >= kBeyondBf16), 0)) put<true>(lds, tid);
            else put<false>(lds, tid);
        }
    }
    template <bool CAREFUL> __device__ __forceinline__ void put(char *lds, int tid) const
    {
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int q = tid + NT * i;
            if (Img::CHUNKS % NT != 0 && q >= Img::CHUNKS) continue;
            char *to = lds + Img::place(q / Img::CPR, q % Img::CPR);
            if constexpr (T == 1) {
                *reinterpret_cast<uint4 *>(to) = raw[i][0];
            } else {
                static_assert(E == 8 && T == 3, "the splitting of a chunk");
                union { uint4 u[W]; float f[E]; } x;
#pragma unroll
                for (int w = 0; w < W; ++w) x.u[w] = raw[i][w];
                uint32_t h[4], m[4], l[4];
                split3_chunk<CAREFUL>(x.f, h, m, l);
                *reinterpret_cast<uint4 *>(to) = make_uint4(h[0], h[1], h[2], h[3]);
                *reinterpret_cast<uint4 *>(to + Img::BYTES) = make_uint4(m[0], m[1], m[2], m[3]);
                *reinterpret_cast<uint4 *>(to + 2 * Img::BYTES) = make_uint4(l[0], l[1], l[2], l[3]);
            }
        }
    }
};

// ---- LDS -> fragments -------------------------------------------------------------------------------
union Frag16 { uint4 u; bf16x8 v; intx4 i; };
union Frag8 { uint4 u[2]; intx8 v; };

// the eight k-values kk + 8 * (lane / 32) + 0..7 of row r + lane % 32 (r and kk multiples of 32 and 16)
template <bool RC, int ROWS, int BK> __device__ __forceinline__ uint4 tile_frag16(const char *plane, int r, int kk, int lane)
{
    using Img = TileImage<RC, ROWS, BK, 2>;
    if constexpr (RC) {
        // two transposing reads of four k-values: 16 lanes give the addresses of 4 rows x 4 pieces of 8 bytes and get a
        // column of those 4 x 16 values each
        const int g = lane >> 4, i = lane & 15, row = kk + 8 * (g >> 1) + (i >> 2);
        const char *p = plane + Img::place(row, r / 8 + 2 * (g & 1) + ((i & 3) >> 1)) + 8 * (i & 1);
        const char *p4 = plane + Img::place(row + 4, r / 8 + 2 * (g & 1) + ((i & 3) >> 1)) + 8 * (i & 1);
        typedef __attribute__((address_space(3))) shortx4_tr *lds4_t;
        union { shortx4_tr v; uint2 u; } a, b;
        a.v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4_t)(p));
        b.v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4_t)(p4));
        return make_uint4(a.u.x, a.u.y, b.u.x, b.u.y);
    } else {
        return *reinterpret_cast<const uint4 *>(plane + Img::place(r + (lane & 31), kk / 8 + (lane >> 5)));
    }
}

// 16 k-values kk + 16 * (lane / 32) + 0..15 of row r + lane % 32, 8 bits each
template <int ROWS, int BK> __device__ __forceinline__ uint4 tile_chunk8(const char *plane, int r, int kk, int lane)
{
    using Img = TileImage<false, ROWS, BK, 1>;
    return *reinterpret_cast<const uint4 *>(plane + Img::place(r + (lane & 31), kk / 16 + (lane >> 5)));
}

// eight e4m3 values as bf16 (exact)
__device__ __forceinline__ bf16x8 widen_e4m3(uint32_t lo, uint32_t hi)
{
    union { bf16x2_t p[4]; bf16x8 v; } f;
    f.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false);
    f.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true);
    f.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false);
    f.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true);
    return f.v;
}

template <int EB, int T, int MI, int NJ, bool INT> struct Fragments { // of one step
    using F = std::conditional_t<EB == 1 && !INT, Frag8, Frag16>;
    F a[MI][T], b[NJ][T];
};

// four columns (chunk 0..7) of a row of a 32 x 32 fp32 strip
template <int COLS = 32> __device__ __forceinline__ float4 *strip_at(float *strip, int row, int chunk) { return reinterpret_cast<float4 *>(strip + row * COLS + ((chunk ^ (row & 7)) * 4)); }

// ---- items of a launch ------------------------------------------------------------------------------
struct TileItem { // M, N, K > 0
    const void *A, *B;
    int64_t lda, ldb;          // elements
    int64_t a_plane, b_plane;  // bytes from term to term (kDirect, T > 1)
    int64_t M, N, K;
    int64_t k_per_split;       // multiple of BK; n_split * k_per_split >= K
    int32_t n_split;           // every split has k-values
    int32_t mt, nt;            // tiles
    int32_t symmetric;         // C is: the tiles below the diagonal are not formed (several items, one tile size along both sides)
    uint32_t block0, places;   // one item: its tiles, places of them (a multiple of 8); several: the tiles before it, its tiles
    int32_t group = 0;         // one item that is not split: row blocks that are walked together, column by column (0, 1: each by itself)
};

// An output tile and the part of the contraction that goes into it.
struct TilePlace {
    uint32_t at;
    int64_t m0, n0, k0;
    int kn, split;
    __device__ __forceinline__ void set(const TileItem &it, uint32_t row, uint32_t col, int s, int bm, int bn)
    {
        split = s;
        m0 = static_cast<int64_t>(row) * bm;
        n0 = static_cast<int64_t>(col) * bn;
        k0 = s * it.k_per_split;
        kn = static_cast<int>(min(it.K - k0, it.k_per_split));
    }
    // One item: the first place from `at` on, `stride` apart, that has a tile.  Place -> (XCD, position in its queue) -> tile:
    // workgroups go round-robin to the 8 XCDs, each of which takes an eighth of the tiles, consecutive ones: those that share operand rows (the
    // column tiles of a row block, all tiles of a split) follow one another, and no XCD has more than one tile above the others, however
    // few row blocks or splits there are.
    __device__ __forceinline__ bool seek(const TileItem &it, uint32_t stride, int bm, int bn)
    {
        const bool splits = it.n_split > 1;
        const uint32_t inner = splits ? static_cast<uint32_t>(it.nt) * it.mt : static_cast<uint32_t>(it.nt), each = it.places / 8;
        for (; at < it.places; at += stride) {
            const uint32_t tile = at % 8 * each + at / 8;
            if (tile >= it.block0) continue;
            const uint32_t outer = tile / inner, in = tile - outer * inner;
            if (splits) {
                set(it, in / it.nt, in % it.nt, static_cast<int>(outer), bm, bn);
            } else if (it.group > 1) {
                const uint32_t first = outer / it.group * it.group, rows = min(static_cast<uint32_t>(it.mt) - first, static_cast<uint32_t>(it.group)), place = tile - first * inner;
                set(it, first + place % rows, place / rows, 0, bm, bn);
            } else {
                set(it, outer, in, 0, bm, bn);
            }
            return true;
        }
        return false;
    }
    // Several items: tile `in` of an item, row block by row block (a symmetric one's from the diagonal on).
    __device__ __forceinline__ void pick(const TileItem &it, uint32_t in, int bm, int bn)
    {
        uint32_t row = 0;
        if (it.symmetric) {
            while (in >= static_cast<uint32_t>(it.nt) - row) in -= static_cast<uint32_t>(it.nt) - row++;
            set(it, row, row + in, 0, bm, bn);
        } else {
            set(it, in / it.nt, in % it.nt, 0, bm, bn);
        }
    }
};

// Epi: what becomes of the product; all functions are device functions.
//   kItems, Extra: items of a launch at most, and what an item's epilogue needs
//   kBlocks = true: block(x, it, strip, m, n, off_diagonal, lane) takes 32 x 32 sums at row m, column n from the strip (strip_at)
//   kBlocks = false: with W = 16 bytes of columns of Out, first(cols, row, y) makes pre-activations of W sums and second(x, y, t)
//     results, t being W elements of x.other (if kReads; zeros or nothing where it is null); x.pre (if kPre and not null) and
//     out(x, it, split) receive them, rows x.ld_pre and x.ld_out apart; kWhole: N is a multiple of W.  struct Cols, Row { void
//     load(const Extra &x, int64_t n, int64_t N); } are what a lane keeps of W columns and of a row (which may lie beyond the matrix).
//   Instead, kTile = true: begin<C>(x, it, acc, place, wave, lane) sets what the sums of a tile start from, tile<C>(x, it, acc, strip, place, wave, lane)
//     takes a wavefront's sums as they lie in the registers, and choose(x, it) may change the item's addresses by what is in memory when the kernel runs; kStrip<C>: bytes of its strip.
template <typename Epi, typename = void> struct takes_tile : std::false_type {};
template <typename Epi> struct takes_tile<Epi, std::enable_if_t<Epi::kTile>> : std::true_type {};
template <typename C, typename Epi> constexpr int strip_bytes() // a 32 x 32 block of fp32, unless the epilogue says otherwise
{
    if constexpr (takes_tile<Epi>::value) return Epi::template kStrip<C>;
    else return 4096;
}
// kBits = true: 32-bit integer sums reach a block epilogue as they are held, not rounded to fp32.
template <typename Epi, typename = void> struct takes_bits : std::false_type {};
template <typename Epi> struct takes_bits<Epi, std::enable_if_t<Epi::kBits>> : std::true_type {};
template <typename Epi> struct TileArgs {
    int n_items;
    uint32_t stride; // one item: from one tile of a workgroup to its next; several: tiles of an XCD
    uint32_t total;  // several items: tiles
    TileItem item[Epi::kItems];
    typename Epi::Extra extra[Epi::kItems];
};

// S: storage type of a value (a plane's with kDirect); EB: bytes of a value in LDS (2: bf16 terms, 1: e4m3); tile of
// (32 MI WM) x (32 NJ WN), BK k-values per stage, ST stages (kDirect; two otherwise).  WIDEN: 8-bit values become bf16 on
// their way from LDS to the bf16 matrix instruction, whose sums are exact to fp32; the 8-bit instruction takes half the time,
// but aligns its products to the largest with about 14 bits below (sums of 1,024 products of random values: 1.5e-5 off
// relative to the result, against 2e-7).
// INT: the 8-bit values are whole numbers, their products are added as 32-bit integers, at the 8-bit rate and exactly (|sum| < 2^31: fewer than 2^17
// products), and rounded to fp32 in front of the epilogue (kBits: not there).
template <typename S_, int EB_, int T_, bool A_RC_, bool B_RC_, int LOAD_, int WM_, int WN_, int MI_, int NJ_, int BK_, int ST_, int OCC_, bool WIDEN_ = false, bool INT_ = false> struct TileShape {
    using S = S_;
    static constexpr int EB = EB_, T = T_, LOAD = LOAD_, WM = WM_, WN = WN_, MI = MI_, NJ = NJ_, BK = BK_, ST = LOAD_ == kDirect ? ST_ : 2, OCC = OCC_;
    static constexpr bool A_RC = A_RC_, B_RC = B_RC_, WIDEN = WIDEN_, INT = INT_;
    using Sum = std::conditional_t<INT_, intx16, floatx16>;
    static constexpr int NW = WM * WN, NT = 64 * NW, BM = 32 * MI * WM, BN = 32 * NJ * WN;
};

// Every kernel made from this template has to stay within its registers.  Where it did not, the compiler split the ranges of values that live through the epilogue,
// the load offsets of the next tile, and put the copies that save them in front of the instruction that brings back the lanes of a branch:
// lanes that the branch had masked (columns beyond N, whose bias and scales were not loaded) got stale offsets, and the next tile was read from anywhere.  Hence tiles
// of 256 x 128 for the epilogues that hold most, and bias and scales loaded by all lanes.
template <typename C, typename Epi>
__global__ void __launch_bounds__(C::NT, C::OCC) tile_gemm_kernel(TileArgs<Epi> p)
{
    using S = typename C::S;
    constexpr int EB = C::EB, T = C::T, MI = C::MI, NJ = C::NJ, BK = C::BK, ST = C::ST, NW = C::NW, NT = C::NT, BM = C::BM, BN = C::BN;
    constexpr bool DIRECT = C::LOAD == kDirect;
    using ImgA = TileImage<C::A_RC, BM, BK, EB>;
    using ImgB = TileImage<C::B_RC, BN, BK, EB>;
    constexpr int A_STAGE = ImgA::BYTES * T, STAGE = A_STAGE + ImgB::BYTES * T;
    // epilogue strips: one 32 x 32 block of sums per wavefront, its own; behind the ring where that is filled during the epilogue
    constexpr int STRIPS = NW * strip_bytes<C, Epi>(), STRIPS_AT = DIRECT ? ST * STAGE : 0;
    __shared__ __attribute__((aligned(1024))) char ring[std::max(ST * STAGE, STRIPS_AT + STRIPS)];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = (wave / C::WN) * (32 * MI), wn = (wave % C::WN) * (32 * NJ);

    int c = 0;
    TilePlace now;
    if constexpr (Epi::kItems > 1) {
        // a workgroup per tile; an XCD's are consecutive ones, so that an item's operands meet in one or two L2s
        const uint32_t tile = blockIdx.x % 8 * p.stride + blockIdx.x / 8;
        if (tile >= p.total) return;
        while (c + 1 < p.n_items && tile >= p.item[c + 1].block0) ++c; // uniform
        now.pick(p.item[c], tile - p.item[c].block0, BM, BN);
    } else {
        now.at = blockIdx.x;
        if (!now.seek(p.item[0], p.stride, BM, BN)) return;
    }
    TileItem it = p.item[c];
    const typename Epi::Extra extra = p.extra[c];
    if constexpr (takes_tile<Epi>::value) Epi::choose(extra, it);

    auto further = [&](TilePlace &t) { // the workgroup's next tile
        if constexpr (Epi::kItems > 1) return false;
        t.at += p.stride;
        return t.seek(it, p.stride, BM, BN);
    };

    typename C::Sum acc[MI][NJ];
    auto clear = [&] {
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int jj = 0; jj < NJ; ++jj)
#pragma unroll
                for (int v = 0; v < 16; ++v) acc[i][jj][v] = 0;
    };
    auto begin = [&] {
        if constexpr (takes_tile<Epi>::value) Epi::template begin<C>(extra, it, acc, now, wave, lane);
        else clear();
    };
    auto four = [&](int i, int jj, int q) {
        const auto &a = acc[i][jj];
        if constexpr (C::INT && takes_bits<Epi>::value) return make_float4(__int_as_float(a[4 * q]), __int_as_float(a[4 * q + 1]), __int_as_float(a[4 * q + 2]), __int_as_float(a[4 * q + 3]));
        else return make_float4(a[4 * q], a[4 * q + 1], a[4 * q + 2], a[4 * q + 3]);
    };

    // One k-tile.  The fragments of a step are read before the products of the step in front of it, and scheduling barriers
    // keep them there: left to itself the compiler reads a fragment just before its first product, and every step waits for LDS.
    auto compute = [&](const char *stage) {
        const char *At = stage, *Bt = stage + A_STAGE;
        constexpr int KS = C::INT ? 32 : EB == 1 ? 64 : 16, STEPS = BK / KS;
        constexpr int SETS = EB == 1 && !C::INT ? 1 : 2; // two sets of 8-bit fragments of 64 k-values do not fit beside the accumulators
        using Step = Fragments<EB, T, MI, NJ, C::INT>;
        Step f[SETS];
        auto read = [&](Step &to, int kk) {
            if constexpr (C::INT) {
#pragma unroll
                for (int jj = 0; jj < NJ; ++jj) to.b[jj][0].u = tile_chunk8<BN, BK>(Bt, wn + 32 * jj, kk, lane);
#pragma unroll
                for (int i = 0; i < MI; ++i) to.a[i][0].u = tile_chunk8<BM, BK>(At, wm + 32 * i, kk, lane);
            } else if constexpr (EB == 1) {
                // which 32 (or 8) of the k-values a lane feeds to an instruction does not matter as long as both operands agree
#pragma unroll
                for (int h = 0; h < 2; ++h) {
#pragma unroll
                    for (int jj = 0; jj < NJ; ++jj) to.b[jj][0].u[h] = tile_chunk8<BN, BK>(Bt, wn + 32 * jj, kk + 32 * h, lane);
#pragma unroll
                    for (int i = 0; i < MI; ++i) to.a[i][0].u[h] = tile_chunk8<BM, BK>(At, wm + 32 * i, kk + 32 * h, lane);
                }
            } else {
#pragma unroll
                for (int t = 0; t < T; ++t) {
#pragma unroll
                    for (int jj = 0; jj < NJ; ++jj) to.b[jj][t].u = tile_frag16<C::B_RC, BN, BK>(Bt + t * ImgB::BYTES, wn + 32 * jj, kk, lane);
#pragma unroll
                    for (int i = 0; i < MI; ++i) to.a[i][t].u = tile_frag16<C::A_RC, BM, BK>(At + t * ImgA::BYTES, wm + 32 * i, kk, lane);
                }
            }
        };
        auto multiply = [&](const Step &x) {
            if constexpr (C::INT) {
#pragma unroll
                for (int i = 0; i < MI; ++i)
#pragma unroll
                    for (int jj = 0; jj < NJ; ++jj) acc[i][jj] = __builtin_amdgcn_mfma_i32_32x32x32_i8(x.b[jj][0].i, x.a[i][0].i, acc[i][jj], 0, 0, 0);
            } else if constexpr (EB == 1 && C::WIDEN) {
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    bf16x8 wb[NJ];
#pragma unroll
                    for (int jj = 0; jj < NJ; ++jj) wb[jj] = widen_e4m3(x.b[jj][0].v[2 * h], x.b[jj][0].v[2 * h + 1]);
#pragma unroll
                    for (int i = 0; i < MI; ++i) {
                        const bf16x8 wa = widen_e4m3(x.a[i][0].v[2 * h], x.a[i][0].v[2 * h + 1]);
#pragma unroll
                        for (int jj = 0; jj < NJ; ++jj) acc[i][jj] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wb[jj], wa, acc[i][jj], 0, 0, 0);
                    }
                }
            } else if constexpr (EB == 1) {
                constexpr int kOne = 0x7f7f7f7f; // block scales of 2^0
#pragma unroll
                for (int i = 0; i < MI; ++i)
#pragma unroll
                    for (int jj = 0; jj < NJ; ++jj)
                        acc[i][jj] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x.b[jj][0].v, x.a[i][0].v, acc[i][jj], 0, 0, 0, kOne, 0, kOne);
            } else {
                // leading terms first; those whose weights add up to less than the third term's are left out
#pragma unroll
                for (int order = 0; order < T; ++order)
#pragma unroll
                    for (int ta = 0; ta < T; ++ta)
#pragma unroll
                        for (int tb = 0; tb < T; ++tb) {
                            if ((ta > tb ? ta : tb) != order || ta + tb > T - 1) continue;
#pragma unroll
                            for (int i = 0; i < MI; ++i)
#pragma unroll
                                for (int jj = 0; jj < NJ; ++jj)
                                    acc[i][jj] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x.b[jj][tb].v, x.a[i][ta].v, acc[i][jj], 0, 0, 0);
                        }
            }
        };
        read(f[0], 0);
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            if (SETS == 2 && s + 1 < STEPS) read(f[(s + 1) % SETS], (s + 1) * KS);
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(1);
            multiply(f[s % SETS]);
            __builtin_amdgcn_s_setprio(0);
            __builtin_amdgcn_sched_barrier(0);
            if (SETS == 1 && s + 1 < STEPS) read(f[0], (s + 1) * KS);
        }
    };

    // register 4 q + e of block (i, jj) is column 8 q + 4 (lane / 32) + e of row lane % 32
    auto epilogue = [&] {
        if constexpr (takes_tile<Epi>::value) {
            Epi::template tile<C>(extra, it, acc, reinterpret_cast<float *>(ring + STRIPS_AT + wave * strip_bytes<C, Epi>()), now, wave, lane);
        } else if constexpr (Epi::kBlocks) {
            const int half = lane >> 5, l32 = lane & 31;
            float *strip = reinterpret_cast<float *>(ring + STRIPS_AT + wave * 4096);
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int jj = 0; jj < NJ; ++jj) {
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        *strip_at(strip, l32, 2 * q + half) = four(i, jj, q);
                    Epi::block(extra, it, strip, now.m0 + wm + 32 * i, now.n0 + wn + 32 * jj, now.m0 != now.n0, lane);
                }
        } else {
            using O = typename Epi::Out;
            constexpr int W = 16 / (int)sizeof(O);                        // columns of a lane: 16 bytes of the output
            constexpr int LPR = 32 / W, RPP = 64 / LPR, ROUNDS = 32 / RPP; // lanes per row of a block, rows per access, accesses
            float *strip = reinterpret_cast<float *>(ring + STRIPS_AT + wave * 4096);
            // what depends on the lane is computed here for every tile: kept from one epilogue to the next, it takes registers of the products
            int here = lane;
            asm volatile("" : "+v"(here));
            const int sr = here / LPR, sc = here % LPR, half = here >> 5, l32 = here & 31;
            const int64_t rm = now.m0 + wm + sr, rn = now.n0 + wn + sc * W;
            auto valid = [&](int64_t n) { return Epi::kWhole ? W : static_cast<int>(min(it.N - n, static_cast<int64_t>(W))); };
            // What the epilogue reads in the output's shape comes for as many rows of blocks at a time as 32 registers hold, and is
            // awaited at once, in front of their stores: a load waits for every store that was issued before it, and one
            // left to the compiler, across the branches below, for every store so far at each of its uses (700,000 x 1,024 x 256 with
            // a residual: 495 to 556 us that way, 485 this way; with 64 registers accumulators spill, 556).
            constexpr int BATCH = std::max(1, std::min(MI, 8 / (NJ * ROUNDS)));
            uintx4 other[Epi::kReads ? BATCH : 1][NJ][ROUNDS];
            auto fetch = [&](int i0) {
                if constexpr (Epi::kReads)
                    if (extra.other) {
#pragma unroll
                        for (int i = i0; i < i0 + BATCH && i < MI; ++i)
#pragma unroll
                            for (int jj = 0; jj < NJ; ++jj)
#pragma unroll
                                for (int r = 0; r < ROUNDS; ++r) {
                                    const int64_t m = rm + 32 * i + RPP * r, n = rn + 32 * jj;
                                    other[i % BATCH][jj][r] = uintx4{0u, 0u, 0u, 0u};
                                    if (m < it.M && n < it.N) other[i % BATCH][jj][r] = load_piece(static_cast<const O *>(extra.other) + m * extra.ld_other + n, valid(n));
                                }
                        wait_counters<0, false>();
                    }
            };
            typename Epi::Cols cols[NJ];
#pragma unroll
            for (int jj = 0; jj < NJ; ++jj) cols[jj].load(extra, rn + 32 * jj, it.N);
            typename Epi::Row rows[MI][ROUNDS];
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int r = 0; r < ROUNDS; ++r) rows[i][r].load(extra, rm + 32 * i + RPP * r, it.M);
            wait_counters<0, false>(); // as above (8-bit 200,000 x 1,024 x 4,096: 1,404 us without, 1,133)
            O *const out = Epi::out(extra, it, now.split);
#pragma unroll
            for (int i = 0; i < MI; ++i) {
                if (i % BATCH == 0) fetch(i);
#pragma unroll
                for (int jj = 0; jj < NJ; ++jj) {
                    const int64_t n = rn + 32 * jj;
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        *strip_at(strip, l32, 2 * q + half) = four(i, jj, q);
#pragma unroll
                    for (int r = 0; r < ROUNDS; ++r) {
                        const int64_t m = rm + 32 * i + RPP * r;
                        float y[W];
#pragma unroll
                        for (int h = 0; h < W / 4; ++h) {
                            const float4 f = *strip_at(strip, RPP * r + sr, sc * (W / 4) + h);
                            y[4 * h] = f.x; y[4 * h + 1] = f.y; y[4 * h + 2] = f.z; y[4 * h + 3] = f.w;
                        }
                        if (m >= it.M || n >= it.N) continue;
                        Epi::first(cols[jj], rows[i][r], y);
                        if constexpr (Epi::kPre)
                            if (extra.pre) store_piece(static_cast<O *>(extra.pre) + m * extra.ld_pre + n, valid(n), pack16<O>(y));
                        float t[W];
                        if constexpr (Epi::kReads) unpack16<O>(other[i % BATCH][jj][r], t);
                        Epi::second(extra, y, t);
                        store_piece(out + m * extra.ld_out + n, valid(n), pack16<O>(y));
                    }
                }
            }
        }
    };

    if constexpr (DIRECT) {
        // One stream of k-tiles through the ring over all output tiles of the workgroup: the first k-tiles of the next output
        // tile are on their way while this one's epilogue runs.
        using LA = PlaneLoader<C::A_RC, BM, BK, EB, NW, T>;
        using LB = PlaneLoader<C::B_RC, BN, BK, EB, NW, T>;
        constexpr int LOADS = LA::LOADS + LB::LOADS;
        static_assert((ST - 2) * LOADS < 64, "the wait counter has 6 bits");
        LA la;
        LB lb;
        const uint32_t lds0 = lds_address(ring);
        TilePlace ahead = now; // the output tile whose k-tiles are being loaded
        int left = 0;          // k-values of it that are still to be loaded
        bool more = true;
        int known = 0, flying = 0; // k-tiles ahead of the current one: those known to be there, those issued
        auto aim = [&] {
            la.init(it.A, it.lda, it.a_plane, ahead.m0, it.M, ahead.k0, wave, lane);
            lb.init(it.B, it.ldb, it.b_plane, ahead.n0, it.N, ahead.k0, wave, lane);
            left = ahead.kn;
        };
        auto issue = [&](int s) { // the next k-tile of the stream, if there is one, into stage s
            if (left <= 0) {
                if (!more) return;
                more = further(ahead);
                if (!more) return;
                aim();
            }
            if (left >= BK) {
                la.issue(lds0 + s * STAGE, wave);
                lb.issue(lds0 + s * STAGE + A_STAGE, wave);
            } else {
                la.issue_tail(lds0 + s * STAGE, wave, lane, left, it.lda, ahead.m0, it.M);
                lb.issue_tail(lds0 + s * STAGE + A_STAGE, wave, lane, left, it.ldb, ahead.n0, it.N);
            }
            left -= BK;
            ++flying;
        };
        aim();
#pragma unroll
        for (int s = 0; s < ST - 1; ++s) issue(s);
        int cur = 0;
        while (true) {
            begin();
            for (int kv = now.kn; kv > 0; kv -= BK) {
                // this wavefront's part of the k-tile is there, and its fragment reads of the last one are done
                if (known > 0) {
                    --known;
                    wait_counters<63, true>();
                } else if (flying >= ST - 1) {
                    wait_counters<(ST - 2) * LOADS, true>();
                } else {
                    wait_counters<0, true>();
                }
                --flying;
                barrier_no_drain();
                if (kv < BK) {
                    LA::clear_tail(ring + cur * STAGE, tid, kv);
                    LB::clear_tail(ring + cur * STAGE + A_STAGE, tid, kv);
                    wait_counters<63, true>();
                    barrier_no_drain();
                }
                issue(cur == 0 ? ST - 1 : cur - 1); // every wavefront is done with the stage of the k-tile before this one
                compute(ring + cur * STAGE);
                cur = cur + 1 == ST ? 0 : cur + 1;
            }
            // The k-tiles ahead are awaited here, not behind the epilogue's stores (the counter runs in order): they were
            // issued before the last k-tile's products.
            TilePlace next = now;
            const bool again = further(next);
            if (again) {
                wait_counters<0, false>();
                known = flying;
            }
            epilogue();
            if (!again) break;
            now = next;
        }
    } else {
        StagedLoader<S, C::A_RC, BM, BK, EB, NT, T> sa;
        StagedLoader<S, C::B_RC, BN, BK, EB, NT, T> sb;
        const S *A = static_cast<const S *>(it.A), *B = static_cast<const S *>(it.B);
        do {
            const int64_t k_end = now.k0 + now.kn;
            const int tiles = (now.kn + BK - 1) / BK;
            begin();
            sa.load(A, it.lda, now.m0, it.M, now.k0, k_end, tid);
            sb.load(B, it.ldb, now.n0, it.N, now.k0, k_end, tid);
            sa.store(ring, tid);
            sb.store(ring + A_STAGE, tid);
            wait_counters<63, true>();
            barrier_no_drain();
            for (int t = 0; t < tiles; ++t) {
                const bool more = t + 1 < tiles;
                if (more) {
                    sa.load(A, it.lda, now.m0, it.M, now.k0 + static_cast<int64_t>(t + 1) * BK, k_end, tid);
                    sb.load(B, it.ldb, now.n0, it.N, now.k0 + static_cast<int64_t>(t + 1) * BK, k_end, tid);
                }
                compute(ring + (t & 1) * STAGE);
                if (more) {
                    char *next = ring + ((t + 1) & 1) * STAGE;
                    sa.store(next, tid);
                    sb.store(next + A_STAGE, tid);
                }
                wait_counters<63, true>();
                barrier_no_drain();
            }
            epilogue();
            wait_counters<63, true>();
            barrier_no_drain(); // the next tile's first k-tile overlays the strips
        } while (further(now));
    }
}

// Tiles of the items and workgroups; false where a grid cannot hold them.
template <typename C, typename Epi> inline bool plan_tiles(TileArgs<Epi> &p, uint32_t *blocks)
{
    int64_t at = 0;
    for (int i = 0; i < p.n_items; ++i) {
        TileItem &it = p.item[i];
        const int64_t mt = (it.M + C::BM - 1) / C::BM, nt = (it.N + C::BN - 1) / C::BN;
        const int64_t outer = it.n_split > 1 ? it.n_split : mt, inner = it.n_split > 1 ? mt * nt : nt;
        if (mt >= (int64_t(1) << 31) || nt >= (int64_t(1) << 31) || inner >= (int64_t(1) << 31) || it.K >= (int64_t(1) << 31)) return false;
        if (outer > (int64_t(1) << 31) / inner - 8) return false;
        it.mt = static_cast<int32_t>(mt);
        it.nt = static_cast<int32_t>(nt);
        it.block0 = static_cast<uint32_t>(Epi::kItems > 1 ? at : outer * inner);
        if (Epi::kItems > 1) it.places = static_cast<uint32_t>(it.symmetric ? mt * (mt + 1) / 2 : mt * nt);
        else it.places = static_cast<uint32_t>((outer * inner + 7) / 8 * 8);
        at += it.places;
        if (Epi::kItems > 1 && (it.n_split > 1 || (it.symmetric && C::BM != C::BN) || at > max_blocks(C::NT) - 8)) return false;
    }
    if (Epi::kItems > 1) {
        p.total = static_cast<uint32_t>(at);
        p.stride = (p.total + 7) / 8;
        *blocks = 8 * p.stride;
    } else {
        *blocks = static_cast<uint32_t>(at);
    }
    return true;
}

// workgroups of a kernel that are resident at a time
template <typename C, typename Epi> inline uint32_t resident_tiles()
{
    static const uint32_t n = [] {
        int dev = 0, cus = 0, each = 0;
        if (hipGetDevice(&dev) != hipSuccess || hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || cus <= 0) cus = 256;
        if (hipOccupancyMaxActiveBlocksPerMultiprocessor(&each, tile_gemm_kernel<C, Epi>, C::NT, 0) != hipSuccess || each <= 0) each = 1;
        return static_cast<uint32_t>(cus / 8 * 8 * each);
    }();
    return n;
}

template <typename C, typename Epi> inline heta_status launch_tiles(const char *who, const char *name, TileArgs<Epi> &p, double bytes, double flops, hipStream_t st)
{
    static_assert(sizeof(TileArgs<Epi>) <= 3584, "kernel arguments are limited to 4 KB");
    uint32_t blocks = 0;
    if (!plan_tiles<C>(p, &blocks)) return fail(HETA_ERR_UNSUPPORTED, "%s: matrix too large for one launch", who);
    if (blocks == 0) return HETA_OK;
    if (Epi::kItems == 1) p.stride = blocks = std::min(blocks, resident_tiles<C, Epi>()); // walked by the workgroups that fit the chip
    ProfScope prof(name, st, bytes, flops);
    hipLaunchKernelGGL((tile_gemm_kernel<C, Epi>), dim3(blocks), dim3(C::NT), 0, st, p);
    HETA_LAUNCH_CHECK("tile_gemm_kernel");
    return HETA_OK;
}

} // namespace heta
