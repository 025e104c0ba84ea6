// Tiled matrix products with an epilogue of the caller's choice, on the bf16 and the 8-bit matrix pipe (not part of the
// ABI): C[M, N] = epilogue(A[M, K] . B[K, N]) for one item or for several that share a launch.
//
// Operands.  A tile lies in LDS as 16-byte chunks, in T planes (bf16 terms of the value, one for bf16 itself, three for
// fp32: see split3_pair) and in one of two layouts:
//   k-contiguous (element (r, k) at base[r * ld + k]): LDS row r holds the tile's k range, its chunks permuted by swz;
//   r-contiguous (element (r, k) at base[k * ld + r]): LDS row k, chunks at rc_place; fragments are read with the
//   transposing LDS read, so neither operand of any product is ever transposed in memory.
// It gets there straight from memory (kDirect: 16-byte aligned rows of the image's own type, T planes side by side in
// memory) or through registers (kStaged / kElements: any storage type and alignment; fp32 is split into its three terms
// there, once per workgroup, not by every wavefront that reads the tile).  A last tile with fewer k-values always takes
// the way through registers, which fills up with zeros: the loop itself knows no ragged tile.
//
// The product is formed as (B^T A^T): a lane's accumulator registers then hold consecutive COLUMNS of C, four at a time,
// and the epilogue's pass through LDS takes 128-bit stores; it reads the strip back with eight consecutive columns per
// lane, so that bias, residual and output move 16 bytes (bf16) or 32 (fp32) per lane and whole cache lines per row.
#pragma once

#include <type_traits>

#include "heta_gemm.h"

namespace heta {

enum TileLoad { kDirect = 0, kStaged = 1, kElements = 2 };

typedef int intx8 __attribute__((ext_vector_type(8)));
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
};

// ---- memory -> registers -> LDS ---------------------------------------------------------------------
// An item is one 16-byte chunk of the image: E consecutive elements, converted to the planes of their type.  Elements
// beyond the matrix count as zero.
template <typename S, bool RC, int ROWS, int BK, int EB, int NT, int T, bool VEC> struct StagedLoader {
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
            if (VEC && left >= E) {
#pragma unroll
                for (int w = 0; w < W; ++w) raw[i][w] = reinterpret_cast<const uint4 *>(src)[w];
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
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int q = tid + NT * i;
            if (Img::CHUNKS % NT != 0 && q >= Img::CHUNKS) continue;
            char *to = lds + Img::place(q / Img::CPR, q % Img::CPR);
            if constexpr (T == 1) {
                *reinterpret_cast<uint4 *>(to) = raw[i][0];
            } else {
                union { uint4 u[W]; float f[E]; } x;
#pragma unroll
                for (int w = 0; w < W; ++w) x.u[w] = raw[i][w];
                uint32_t h[4], m[4], l[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) split3_pair(x.f[2 * j], x.f[2 * j + 1], h[j], m[j], l[j]);
                *reinterpret_cast<uint4 *>(to) = make_uint4(h[0], h[1], h[2], h[3]);
                *reinterpret_cast<uint4 *>(to + Img::BYTES) = make_uint4(m[0], m[1], m[2], m[3]);
                if constexpr (T == 3) *reinterpret_cast<uint4 *>(to + 2 * Img::BYTES) = make_uint4(l[0], l[1], l[2], l[3]);
            }
        }
    }
};

// ---- LDS -> fragments -------------------------------------------------------------------------------
union Frag16 { uint4 u; bf16x8 v; };
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

// ---- items of a launch ------------------------------------------------------------------------------
struct TileItem {
    const void *A, *B;
    int64_t lda, ldb;          // elements
    int64_t a_plane, b_plane;  // bytes from term to term (kDirect, T > 1)
    int64_t M, N, K;
    int64_t k_per_split;       // multiple of BK; n_split * k_per_split >= K
    int32_t n_split;
    int32_t mt, nt;            // tiles
    uint32_t block0;           // first workgroup (multiple of 8)
};

// Epi: struct with `static constexpr int kItems`, `Extra` (what an item's epilogue needs) and
//   struct Cols { __device__ Cols(const Extra &x, int64_t n, int valid); }    what a lane keeps of its eight columns n, n + 1, ...
//   __device__ static void put(const Extra &x, const TileItem &it, const Cols &c, int64_t m, int64_t n, int valid, const float (&v)[8], int split)
// for those columns (valid: as many of them as the matrix has) of row m < M.
template <typename Epi> struct TileArgs {
    int n_items;
    TileItem item[Epi::kItems];
    typename Epi::Extra extra[Epi::kItems];
};

// S: storage type of a value (a plane's with kDirect); EB: bytes of a value in LDS (2: bf16 terms, 1: e4m3); tile of
// (32 MI WM) x (32 NJ WN), BK k-values per stage, ST stages (kDirect; two otherwise).  WIDEN: 8-bit values become bf16 on
// their way from LDS to the bf16 matrix instruction, whose sums are exact to fp32; the 8-bit instruction takes half the time,
// but aligns its products to the largest with about 14 bits below (sums of 1,024 products of random values: 1.5e-5 off
// relative to the result, against 2e-7).
template <typename S_, int EB_, int T_, bool A_RC_, bool B_RC_, int LOAD_, int WM_, int WN_, int MI_, int NJ_, int BK_, int ST_, int OCC_, bool WIDEN_ = false> struct TileShape {
    using S = S_;
    static constexpr int EB = EB_, T = T_, LOAD = LOAD_, WM = WM_, WN = WN_, MI = MI_, NJ = NJ_, BK = BK_, ST = LOAD_ == kDirect ? ST_ : 2, OCC = OCC_;
    static constexpr bool A_RC = A_RC_, B_RC = B_RC_, WIDEN = WIDEN_;
    static constexpr int NW = WM * WN, NT = 64 * NW, BM = 32 * MI * WM, BN = 32 * NJ * WN;
};

template <typename C, typename Epi>
__global__ void __launch_bounds__(C::NT, C::OCC) tile_gemm_kernel(TileArgs<Epi> p)
{
    using S = typename C::S;
    constexpr int EB = C::EB, T = C::T, MI = C::MI, NJ = C::NJ, BK = C::BK, ST = C::ST, NW = C::NW, NT = C::NT, BM = C::BM, BN = C::BN;
    constexpr bool DIRECT = C::LOAD == kDirect, VEC = C::LOAD != kElements;
    using ImgA = TileImage<C::A_RC, BM, BK, EB>;
    using ImgB = TileImage<C::B_RC, BN, BK, EB>;
    constexpr int A_STAGE = ImgA::BYTES * T, STAGE = A_STAGE + ImgB::BYTES * T;
    constexpr int EW = 32 * NJ, PITCH = EW + 4; // epilogue strip: 32 rows of a wavefront's columns; rows 16 bytes further on the banks
    constexpr int STRIPS = NW * 32 * PITCH * 4;
    __shared__ __attribute__((aligned(1024))) char ring[ST * STAGE > STRIPS ? ST * STAGE : STRIPS];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = (wave / C::WN) * (32 * MI), wn = (wave % C::WN) * (32 * NJ);

    // workgroup -> item -> (XCD, position in its queue) -> tile: workgroups go round-robin to the 8 XCDs, and the tiles that
    // share operand rows (the column tiles of a row block, all tiles of a split) follow one another on one of them
    int c = 0;
    while (c + 1 < p.n_items && blockIdx.x >= p.item[c + 1].block0) ++c; // uniform
    const TileItem &it = p.item[c];
    const uint32_t b = blockIdx.x - it.block0, xcd = b % 8, j = b / 8;
    const uint32_t inner = it.n_split > 1 ? static_cast<uint32_t>(it.nt) * it.mt : static_cast<uint32_t>(it.nt);
    const uint32_t in = j % inner, outer = j / inner * 8 + xcd;
    if (outer >= static_cast<uint32_t>(it.n_split > 1 ? it.n_split : it.mt)) return;
    const int split = it.n_split > 1 ? static_cast<int>(outer) : 0;
    const int64_t m0 = static_cast<int64_t>(it.n_split > 1 ? in / it.nt : outer) * BM, n0 = static_cast<int64_t>(it.n_split > 1 ? in % it.nt : in) * BN;
    const int64_t k0 = split * it.k_per_split, k_end = min(it.K, k0 + it.k_per_split);
    const int kn = static_cast<int>(max(k_end - k0, static_cast<int64_t>(0)));

    floatx16 acc[MI][NJ];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int jj = 0; jj < NJ; ++jj)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][jj][v] = 0.f;

    auto compute = [&](const char *stage) {
        const char *At = stage, *Bt = stage + A_STAGE;
        if constexpr (EB == 1) {
#pragma unroll
            for (int kk = 0; kk < BK; kk += 64) {
                // which 32 (or 8) of the k-values a lane feeds to an instruction does not matter as long as both operands agree
                Frag8 fa[MI], fb[NJ];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
#pragma unroll
                    for (int jj = 0; jj < NJ; ++jj) fb[jj].u[h] = tile_chunk8<BN, BK>(Bt, wn + 32 * jj, kk + 32 * h, lane);
#pragma unroll
                    for (int i = 0; i < MI; ++i) fa[i].u[h] = tile_chunk8<BM, BK>(At, wm + 32 * i, kk + 32 * h, lane);
                }
                if constexpr (C::WIDEN) {
#pragma unroll
                    for (int h = 0; h < 4; ++h) {
                        bf16x8 wb[NJ];
#pragma unroll
                        for (int jj = 0; jj < NJ; ++jj) wb[jj] = widen_e4m3(fb[jj].v[2 * h], fb[jj].v[2 * h + 1]);
#pragma unroll
                        for (int i = 0; i < MI; ++i) {
                            const bf16x8 wa = widen_e4m3(fa[i].v[2 * h], fa[i].v[2 * h + 1]);
#pragma unroll
                            for (int jj = 0; jj < NJ; ++jj) acc[i][jj] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wb[jj], wa, acc[i][jj], 0, 0, 0);
                        }
                    }
                } else {
                    constexpr int kOne = 0x7f7f7f7f; // block scales of 2^0
#pragma unroll
                    for (int i = 0; i < MI; ++i)
#pragma unroll
                        for (int jj = 0; jj < NJ; ++jj)
                            acc[i][jj] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fb[jj].v, fa[i].v, acc[i][jj], 0, 0, 0, kOne, 0, kOne);
                }
            }
        } else {
#pragma unroll
            for (int kk = 0; kk < BK; kk += 16) {
                Frag16 fa[MI][T], fb[NJ][T];
#pragma unroll
                for (int t = 0; t < T; ++t) {
#pragma unroll
                    for (int jj = 0; jj < NJ; ++jj) fb[jj][t].u = tile_frag16<C::B_RC, BN, BK>(Bt + t * ImgB::BYTES, wn + 32 * jj, kk, lane);
#pragma unroll
                    for (int i = 0; i < MI; ++i) fa[i][t].u = tile_frag16<C::A_RC, BM, BK>(At + t * ImgA::BYTES, wm + 32 * i, kk, lane);
                }
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
                                    acc[i][jj] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[jj][tb].v, fa[i][ta].v, acc[i][jj], 0, 0, 0);
                        }
            }
        }
    };

    if constexpr (DIRECT) {
        using LA = PlaneLoader<C::A_RC, BM, BK, EB, NW, T>;
        using LB = PlaneLoader<C::B_RC, BN, BK, EB, NW, T>;
        constexpr int LOADS = LA::LOADS + LB::LOADS;
        static_assert((ST - 2) * LOADS < 64, "the wait counter has 6 bits");
        LA la;
        LB lb;
        la.init(it.A, it.lda, it.a_plane, m0, it.M, k0, wave, lane);
        lb.init(it.B, it.ldb, it.b_plane, n0, it.N, k0, wave, lane);
        const int full = kn / BK, tail = kn % BK, tiles = full + (tail ? 1 : 0);
        const uint32_t lds0 = lds_address(ring);
#pragma unroll
        for (int s = 0; s < ST - 1; ++s)
            if (s < full) {
                la.issue(lds0 + s * STAGE, wave);
                lb.issue(lds0 + s * STAGE + A_STAGE, wave);
            }
        int cur = 0;
        for (int t = 0; t < tiles; ++t) {
            if (t + ST - 2 < full) wait_counters<(ST - 2) * LOADS, true>(); // tile t is there; this wavefront's reads of tile t - 1 too
            else wait_counters<0, true>();
            if (t >= full) { // the last, shorter tile
                StagedLoader<S, C::A_RC, BM, BK, EB, NT, 1, true> sa;
                StagedLoader<S, C::B_RC, BN, BK, EB, NT, 1, true> sb;
#pragma unroll
                for (int q = 0; q < T; ++q) {
                    sa.load(reinterpret_cast<const S *>(static_cast<const char *>(it.A) + q * it.a_plane), it.lda, m0, it.M, k0 + full * BK, k_end, tid);
                    sb.load(reinterpret_cast<const S *>(static_cast<const char *>(it.B) + q * it.b_plane), it.ldb, n0, it.N, k0 + full * BK, k_end, tid);
                    sa.store(ring + cur * STAGE + q * ImgA::BYTES, tid);
                    sb.store(ring + cur * STAGE + A_STAGE + q * ImgB::BYTES, tid);
                }
                wait_counters<0, true>();
            }
            barrier_no_drain();
            if (t + ST - 1 < full) {
                const int s = cur == 0 ? ST - 1 : cur - 1; // (t + ST - 1) % ST
                la.issue(lds0 + s * STAGE, wave);
                lb.issue(lds0 + s * STAGE + A_STAGE, wave);
            }
            compute(ring + cur * STAGE);
            cur = cur + 1 == ST ? 0 : cur + 1;
        }
    } else {
        StagedLoader<S, C::A_RC, BM, BK, EB, NT, T, VEC> sa;
        StagedLoader<S, C::B_RC, BN, BK, EB, NT, T, VEC> sb;
        const S *A = static_cast<const S *>(it.A), *B = static_cast<const S *>(it.B);
        const int tiles = (kn + BK - 1) / BK;
        if (tiles > 0) {
            sa.load(A, it.lda, m0, it.M, k0, k_end, tid);
            sb.load(B, it.ldb, n0, it.N, k0, k_end, tid);
            sa.store(ring, tid);
            sb.store(ring + A_STAGE, tid);
        }
        wait_counters<0, true>();
        barrier_no_drain();
        for (int t = 0; t < tiles; ++t) {
            const bool more = t + 1 < tiles;
            if (more) {
                sa.load(A, it.lda, m0, it.M, k0 + static_cast<int64_t>(t + 1) * BK, k_end, tid);
                sb.load(B, it.ldb, n0, it.N, k0 + static_cast<int64_t>(t + 1) * BK, k_end, tid);
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
    }
    wait_counters<0, true>();
    barrier_no_drain(); // every wavefront's last fragment reads are done: the strips overlay the ring

    // epilogue: register 4 q + e of a lane is column 8 q + 4 (lane / 32) + e of row lane % 32
    float *strip = reinterpret_cast<float *>(ring) + wave * 32 * PITCH;
    const int half = lane >> 5, l32 = lane & 31;
    constexpr int LPR = EW / 8, RPP = 64 / LPR; // lanes per row, rows per pass
    const int lr = lane / LPR, lc = (lane % LPR) * 8;
    const int64_t n = n0 + wn + lc;
    const int valid = static_cast<int>(min(it.N - n, static_cast<int64_t>(8)));
    const typename Epi::Cols cols(p.extra[c], n, valid);
#pragma unroll
    for (int i = 0; i < MI; ++i) {
#pragma unroll
        for (int jj = 0; jj < NJ; ++jj)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *reinterpret_cast<float4 *>(strip + l32 * PITCH + 32 * jj + 8 * q + 4 * half) =
                    make_float4(acc[i][jj][4 * q], acc[i][jj][4 * q + 1], acc[i][jj][4 * q + 2], acc[i][jj][4 * q + 3]);
        // the strip is the wavefront's own, and LDS operations of one wavefront complete in order: what keeps the compiler
        // from moving the reads up is that they alias
#pragma unroll
        for (int r = 0; r < 32; r += RPP) {
            const float4 lo = *reinterpret_cast<const float4 *>(strip + (r + lr) * PITCH + lc);
            const float4 hi = *reinterpret_cast<const float4 *>(strip + (r + lr) * PITCH + lc + 4);
            const int64_t m = m0 + wm + 32 * i + r + lr;
            if (m < it.M && valid > 0) {
                const float v[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
                Epi::put(p.extra[c], it, cols, m, n, valid, v, split);
            }
        }
    }
}

// Tile counts and workgroups of the items; false where a grid cannot hold them.
template <typename C, typename Epi> inline bool plan_tiles(TileArgs<Epi> &p, uint32_t *blocks)
{
    int64_t at = 0;
    for (int i = 0; i < p.n_items; ++i) {
        TileItem &it = p.item[i];
        const int64_t mt = (it.M + C::BM - 1) / C::BM, nt = (it.N + C::BN - 1) / C::BN;
        const int64_t outer = it.n_split > 1 ? it.n_split : mt, inner = it.n_split > 1 ? mt * nt : nt;
        if (mt >= (int64_t(1) << 31) || nt >= (int64_t(1) << 31) || inner >= (int64_t(1) << 31) || it.K >= (int64_t(1) << 31)) return false;
        it.mt = static_cast<int32_t>(mt);
        it.nt = static_cast<int32_t>(nt);
        it.block0 = static_cast<uint32_t>(at);
        if (inner > 0 && outer > max_blocks(C::NT) / inner) return false;
        at += (outer + 7) / 8 * 8 * inner;
        if (at > max_blocks(C::NT)) return false;
    }
    *blocks = static_cast<uint32_t>(at);
    return true;
}

template <typename C, typename Epi> inline heta_status launch_tiles(const char *who, const char *name, TileArgs<Epi> &p, double bytes, double flops, hipStream_t st)
{
    static_assert(sizeof(TileArgs<Epi>) <= 3584, "kernel arguments are limited to 4 KB");
    uint32_t blocks = 0;
    if (!plan_tiles<C>(p, &blocks)) return fail(HETA_ERR_UNSUPPORTED, "%s: matrix too large for one launch", who);
    if (blocks == 0) return HETA_OK;
    ProfScope prof(name, st, bytes, flops);
    hipLaunchKernelGGL((tile_gemm_kernel<C, Epi>), dim3(blocks), dim3(C::NT), 0, st, p);
    HETA_LAUNCH_CHECK("tile_gemm_kernel");
    return HETA_OK;
}

} // namespace heta
