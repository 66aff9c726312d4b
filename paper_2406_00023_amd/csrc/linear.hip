// The experts' products on rows sorted by expert, with bias, activation and residual in the epilogue, and their gradients.
//   forward  y[r][n] = act(sum_k x[r][k] w[e][n][k] + bias[e][n]) + residual[r][n]       rows of expert e: offsets[e] ... offsets[e+1] - 1
//   dx[r][k] = sum_n da[r][n] w[e][n][k] (+ the same of db, w_up);  dw[e][n][k] = sum_r da[r][n] x[r][k];  dbias[e][n] = sum_r da[r][n]
//   da = dy act'(a), SwiGLU: da = dy up SiLU'(a), db = dy SiLU(a)                          (an element-wise pass, none for act = none)
// Every product is C[m][n] = sum_k A(m, k) B(n, k) with operands that are read as they lie: contraction contiguous ("rows") or
// contraction slow ("columns": w in dx, both in dw).  Both kinds go straight into LDS in 16-byte pieces; rows are read back as
// MFMA fragments, columns by transposing LDS reads (bf16) or single words (fp32), so nothing is transposed in memory.  What lies
// past the end of a contraction (a ragged K, the rows of the next expert) is zero-filled by the copy.
//
// Bound by the matrix pipe where an expert has a few hundred rows (there: by the power that it draws), by the weights' bytes where it has a
// few, by latency in between.  Measured, 16 experts: SwiGLU of 2048 x 5632, 16 384 uneven rows 690 us (1.1 PFLOP/s; a library product of
// 8192 cubed reaches 1.1), 64 rows 122 us (6.0 TB/s of weights); 5632 x 2048, 16 384 rows: forward 417 us, dx 350, dw 414; fp32, 8 experts of 281
// rows, 520 x 1048: 40, and dx and dw together 68.
#include <algorithm>
#include <cmath>

#include "activation.h"
#include "row_ops.h"

namespace etr {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((address_space(3))) void* lds_ptr;

enum Product { FORWARD = 0, INPUT = 1, WEIGHT = 2 };     // y, dx, dw

struct LinearParams {
    const void* A[2]; const void* B[2];                  // second: SwiGLU (FORWARD: B; INPUT: both; WEIGHT: A)
    void* C[2];                                          // second: WEIGHT with SwiGLU
    const int32_t* offsets;
    const float* bias[2];
    const void* residual;
    void* pre[2];
    int rows, E;
    int M, N, K;                                         // WEIGHT: output rows; output columns; contraction (of each half)
    int lda, ldb;
    int act, glu;
    int NT;                                              // column tiles
};

// Buffer descriptors that bound nothing that exists, and an offset past any of them: such a lane copies zeros.
constexpr uint32_t kRange = 0xFFFFFF00u, kPast = 0xFFFFFF80u;

__device__ __forceinline__ void copy_piece(uint64_t base, uint32_t off, void* dst) {
    const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(base));
    const uint32_t hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(base >> 32));
    void* at = reinterpret_cast<void*>((static_cast<uint64_t>(hi) << 32) | lo);
    const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(at, 0, static_cast<int>(kRange), 0x00027000);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_ptr)dst, 16, static_cast<int>(off), 0, 0, 0);
}

constexpr int kPatch = 4096;                             // LDS of a wave's epilogue (large tiles)

// s_waitcnt: at most n vector memory operations outstanding, the others as they are
template <int N> __device__ __forceinline__ void wait_copies() { __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | 0x0F70); }

// Rows of the groups, one group per lane (E <= 64): first row, number, and the row tiles before it.
struct Groups {
    int first, count, tiles_incl, tiles;
    __device__ __forceinline__ void load(const LinearParams& p, int BM) {
        const int lane = threadIdx.x & 63;
        first = 0; count = 0;
        if (lane < p.E) {
            first = p.offsets ? min(max(p.offsets[lane], 0), p.rows) : 0;
            const int end = p.offsets ? min(max(p.offsets[lane + 1], first), p.rows) : p.rows;
            count = end - first;
        }
        tiles = (count + BM - 1) / BM;
        tiles_incl = wave_scan_incl(tiles);
    }
};

// count: rows of the group; limit: the tile stores rows below it; half: WEIGHT with SwiGLU, which of the two outputs
struct Tile { int e, first, m0, n0, count, limit, half; };

// The tile list: groups one after the other; inside a group bands of 8 row tiles, in a band the row tiles of a column tile next to
// each other.  Each XCD (workgroups go round them) has an equal contiguous part of the list, so its 32 CUs work on some 8 x 4 tiles at
// once and share 8 + 4 operand slabs in its L2.
// SPLIT (large tiles, one workgroup to a CU): where the last round over an XCD's CUs would keep half of them or fewer busy, its tiles go in
// halves or quarters of their rows to as many workgroups.
template <int MODE, bool SPLIT>
__device__ __forceinline__ bool find_tile(const LinearParams& p, const Groups& g, int BM, int BN, int bid, int grid, int j, Tile& t) {
    int total, MTw = 0;
    if (MODE == WEIGHT) {
        MTw = (p.M + BM - 1) / BM;
        total = p.E * MTw * (p.glu ? 2 : 1) * p.NT;
    } else {
        total = __builtin_amdgcn_readlane(g.tiles_incl, 63) * p.NT;
    }
    const int share = (total + 7) >> 3;
    int part = 0, parts_log = 0;
    if constexpr (SPLIT) {
        const int W = grid >> 3, full = share / W * W, rest = share - full;
        if (j >= full) {
            parts_log = rest * 4 <= W ? 2 : rest * 2 <= W ? 1 : 0;
            part = (j - full) & ((1 << parts_log) - 1);
            j = full + ((j - full) >> parts_log);
        }
    }
    const int q = (bid & 7) * share + j;
    if (j >= share || q >= total) return false;
    int in, rows;
    if (MODE == WEIGHT) {
        rows = MTw * (p.glu ? 2 : 1);
        t.e = q / (rows * p.NT);
        in = q - t.e * (rows * p.NT);
    } else {
        t.e = __builtin_ctzll(__ballot(g.tiles_incl * p.NT > q));
        rows = __builtin_amdgcn_readlane(g.tiles, t.e);
        in = q - (__builtin_amdgcn_readlane(g.tiles_incl, t.e) - rows) * p.NT;
    }
    const int band = in / (8 * p.NT), in_band = in - band * 8 * p.NT, height = min(8, rows - band * 8);
    const int nt = in_band / height, mt = band * 8 + in_band - nt * height;
    t.first = __builtin_amdgcn_readlane(g.first, t.e);
    t.count = __builtin_amdgcn_readlane(g.count, t.e);
    t.half = MODE == WEIGHT && mt >= MTw ? 1 : 0;
    t.m0 = (mt - t.half * MTw) * BM;
    t.n0 = nt * BN;
    t.limit = MODE == WEIGHT ? p.M : t.count;
    if (SPLIT && parts_log) {                            // (a part past the last row stores nothing: it stays at the tile's start)
        const int height = BM >> parts_log, m0 = t.m0 + part * height;
        t.limit = m0 < t.limit ? min(t.limit, m0 + height) : t.m0;
        t.m0 = t.limit > t.m0 ? m0 : t.m0;
    }
    return true;
}

// ---- epilogue --------------------------------------------------------------------------------------------------------

template <bool BF16>
__device__ __forceinline__ void load4(const void* p, uint32_t at, float (&f)[4]) {
    if constexpr (BF16) {
        const uint2 v = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(p) + at);
        f[0] = __uint_as_float(v.x << 16); f[1] = __uint_as_float(v.x & 0xFFFF0000u);
        f[2] = __uint_as_float(v.y << 16); f[3] = __uint_as_float(v.y & 0xFFFF0000u);
    } else {
        const float4 v = *reinterpret_cast<const float4*>(static_cast<const float*>(p) + at);
        f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w;
    }
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {           // round to nearest even (v_cvt_pk_bf16_f32)
    typedef __attribute__((ext_vector_type(2))) float f32x2;
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
}
template <bool BF16>
__device__ __forceinline__ void store4(void* p, uint32_t at, const float (&f)[4]) {
    if constexpr (BF16) {
        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p) + at) = make_uint2(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]));
    } else {
        *reinterpret_cast<float4*>(static_cast<float*>(p) + at) = make_float4(f[0], f[1], f[2], f[3]);
    }
}

// acc[i][j]: 16 x 16 block i of the wave's rows, j of its columns; a lane has row l16 of a block and four columns from 4 kq on.
// GLU: blocks j < NB / 2 are gate columns, the others the up columns of the same outputs.  What is optional goes over the
// accumulators in a pass of its own, so that a call pays for what it asks for and the code stays small.
// patch: 4 KiB of LDS of this wave's own, through which bf16 values leave as whole 16-byte pieces, 8 (GLU: 4) of a row beside each
// other, or null: 8 bytes a lane as they lie.
template <bool BF16, int MODE, bool GLU, int MB, int NB, bool PATCH>
__device__ __forceinline__ void store_tile(const LinearParams& p, const Tile& t, f32x4 (&acc)[MB][NB], int m_wave, int n_wave, unsigned char* patch) {
    constexpr int NO = GLU ? NB / 2 : NB;
    static_assert(!PATCH || (BF16 && MB % 2 == 0), "");
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));                       // (what depends on it is not worth registers of the loop over k-tiles)
    const int l16 = lane & 15, kq = lane >> 4;
    const int limit = t.limit - t.m0, n_first = t.n0 + n_wave + 4 * kq;
    // uniform start of the tile, 32-bit offsets in it (one register, made anew in each pass: the passes' common addresses kept across them
    // would not fit)
    const size_t tile = ((MODE == WEIGHT ? static_cast<size_t>(t.e) * p.M : static_cast<size_t>(t.first)) + t.m0) * p.N;
    auto each = [&](auto&& f) {
        int m = m_wave + l16;
        asm volatile("" : "+v"(m));
#pragma unroll
        for (int i = 0; i < MB; ++i, m += 16) {
            const uint32_t row = static_cast<uint32_t>(m) * p.N + n_first;
#pragma unroll
            for (int j = 0; j < NO; ++j)
                if (m < limit && n_first + j * 16 < p.N) f(i, j, row + j * 16);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    auto put = [&](void* to, auto&& of) {
        char* base = static_cast<char*>(to) + tile * (BF16 ? 2 : 4);
        if constexpr (PATCH) {
            constexpr int PR = 2 * NO, RP = 64 / PR;     // pieces of a row of the wave's columns; rows that 64 lanes have a piece each of
            const int row_in = lane / PR, piece = lane % PR, n = t.n0 + n_wave + piece * 8;
            const bool full = m_wave + MB * 16 <= limit && t.n0 + n_wave + NO * 16 <= p.N;      // (uniform)
#pragma unroll
            for (int ib = 0; ib < MB / 2; ++ib) {
#pragma unroll
                for (int bi = 0; bi < 2; ++bi)
#pragma unroll
                    for (int j = 0; j < NO; ++j) {
                        const f32x4& v = of(2 * ib + bi, j);
                        const int row = bi * 16 + l16;
                        typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
                        *reinterpret_cast<u32x2*>(patch + row * PR * 16 + (((2 * j + (kq >> 1)) ^ (row & (PR - 1))) * 16) + (kq & 1) * 8) =
                            u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
                    }
                wave_sync();
                piece_t out[32 / RP];
#pragma unroll
                for (int u = 0; u < 32 / RP; ++u) {
                    const int row = u * RP + row_in;
                    out[u] = *reinterpret_cast<const piece_t*>(patch + row * PR * 16 + ((piece ^ (row & (PR - 1))) * 16));
                }
                wave_sync();
#pragma unroll
                for (int u = 0; u < 32 / RP; ++u) {
                    const int m = m_wave + ib * 32 + u * RP + row_in;
                    if (full || (m < limit && n < p.N)) *reinterpret_cast<piece_t*>(base + (static_cast<uint32_t>(m) * p.N + n) * 2u) = out[u];
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            return;
        }
        each([&](int i, int j, uint32_t at) {
            const f32x4& v = of(i, j);
            const float f[4] = {v[0], v[1], v[2], v[3]};
            store4<BF16>(base, at, f);
        });
    };
    if constexpr (MODE == FORWARD) {
#pragma unroll
        for (int h = 0; h < (GLU ? 2 : 1); ++h) {
            // (added without a branch, zeros where there is none: around one, the accumulators of both ways would be kept)
#pragma unroll
            for (int j = 0; j < NO; ++j) {
                float b[4] = {0.f, 0.f, 0.f, 0.f};
                if (p.bias[h] && n_first + j * 16 < p.N) load4<false>(p.bias[h] + static_cast<size_t>(t.e) * p.N, n_first + j * 16, b);
#pragma unroll
                for (int i = 0; i < MB; ++i)
#pragma unroll
                    for (int v = 0; v < 4; ++v) acc[i][h * NO + j][v] += b[v];
            }
            if (p.pre[h]) put(p.pre[h], [&](int i, int j) -> const f32x4& { return acc[i][h * NO + j]; });
        }
        auto map = [&](auto&& f) {
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int j = 0; j < NO; ++j) {
#pragma unroll
                    for (int v = 0; v < 4; ++v) acc[i][j][v] = f(acc[i][j][v], GLU ? acc[i][(GLU ? NO : 0) + j][v] : 1.0f);
                    __builtin_amdgcn_sched_barrier(0);   // one block at a time: keeps the live set small
                }
        };
        if constexpr (GLU) {
            map([](float a, float u) { return a * sigmoid<BF16>(a) * u; });
        } else {
            if (p.act == ETR_ACT_SILU) map([](float a, float) { return a * sigmoid<BF16>(a); });
            // (the empty statements keep the compiler from making one pass of the two, with both results of every value alive)
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int j = 0; j < NO; ++j) asm volatile("" : "+v"(acc[i][j]));
            if (p.act == ETR_ACT_GELU) map([](float a, float) { return a * normal_cdf<BF16>(a); });
        }
        if (p.residual) {                                // two rows of blocks at a time; past the ends the last row or columns again, not stored
            const char* base = static_cast<const char*>(p.residual) + tile * (BF16 ? 2 : 4);
            constexpr int U = MB >= 2 ? 2 : 1;
#pragma unroll
            for (int ib = 0; ib < MB; ib += U) {
                float r[U][NO][4];
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int j = 0; j < NO; ++j)
                        load4<BF16>(base, static_cast<uint32_t>(max(min(m_wave + (ib + u) * 16 + l16, limit - 1), 0)) * p.N + min(n_first + j * 16, p.N - 4), r[u][j]);
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int j = 0; j < NO; ++j)
#pragma unroll
                        for (int v = 0; v < 4; ++v) acc[ib + u][j][v] += r[u][j][v];
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    }
    put(p.C[MODE == WEIGHT ? t.half : 0], [&](int i, int j) -> const f32x4& { return acc[i][j]; });
}

// ---- the products ----------------------------------------------------------------------------------------------------
//
// A k-tile is 128 bytes of contraction (64 bf16, 32 fp32).  LDS, one operand of one k-tile:
//   rows kind     [row][8 pieces]; the piece at place s of a row is s ^ (row / 2 % 8), so that the 16 rows of a fragment spread over
//                 the banks
//   columns kind  bf16: [group of 64 columns][k][64 columns], the 16-column blocks of a k row in the order o ^ f(k), f(k) = bit 1 of
//                 k and twice bit 3, for the transposing reads; fp32: [k][columns], the piece at place s of a k row is s ^ 4 (k / 4 % 4)
// A workgroup of WM x WN waves has a BM x BN tile at a time; NBUF buffers, of which all but one are on their way.
// The MFMAs take the columns' fragment first, so that a lane ends up with four neighbouring columns of one row.
// KS > 1: as many such groups of waves to a workgroup, which has one tile: group g takes the k-tiles g, g + KS, ... into buffers of its
// own, and the first one adds the others' sums to its own, in their order.  For products with fewer tiles than CUs.
// bid, grid: the workgroup's number among those of this product, and theirs (a multiple of 8).
template <bool BF16, int BM, int BN, int WM, int WN, int NBUF, int KS, int MODE, bool GLU>
__device__ __forceinline__ void linear_tiles(const LinearParams& p, int bid, int grid) {
    constexpr bool AT = MODE == WEIGHT, BT = MODE != FORWARD;
    static_assert(!GLU || MODE == FORWARD, "two weights side by side: the forward product only");
    constexpr int ES = BF16 ? 2 : 4, KE = 128 / ES, PE = 16 / ES;        // bytes of an element; elements of a k-tile, of a piece
    constexpr int NW = WM * WN, MB = BM / WM / 16, NB = BN / WN / 16;
    constexpr bool DEEP = BF16 && MB == 8 && NB == 4 && NBUF == 2;       // one workgroup to a CU, which walks the tiles
    constexpr int CA = BM / 8 / NW, CB = BN / 8 / NW;    // copies of 64 pieces per wave, operand and k-tile
    constexpr int A_BYTES = BM * 128, STAGE = (BM + BN) * 128;
    static_assert(CA * NW * 8 == BM && CB * NW * 8 == BN, "whole copies for every wave");
    static_assert((!AT || BM % 64 == 0) && (!BT || BN % 64 == 0), "columns come in groups of 64");
    static_assert(KS == 1 || (!DEEP && BM * BN * 4 <= NBUF * STAGE), "a group's sums fit its buffers");
    static_assert(DEEP || !BF16 || ((!AT || MB == 2 || MB == 4) && (!BT || NB == 2 || NB == 4)), "see column_fragments");
    constexpr int OUT_N = GLU ? BN / 2 : BN;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds_all[];
    const int lane = threadIdx.x & 63, l16 = lane & 15, kq = lane >> 4;
    const int wave_all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = wave_all % NW, group = wave_all / NW, wm = wave / WN, wn = wave % WN;
    unsigned char* lds = lds_all + group * NBUF * STAGE;

    Groups groups;
    groups.load(p, BM);
    Tile t;
    int j = bid >> 3;
    if (!find_tile<MODE, DEEP>(p, groups, BM, OUT_N, bid, grid, j, t)) return;

    // k-tiles of a tile, of each half of a contraction in two halves (INPUT of SwiGLU)
    const int two = MODE == INPUT && p.glu ? 2 : 1;
    auto half_tiles = [&](const Tile& x) { return MODE == WEIGHT ? max((x.count + KE - 1) / KE, 1) : (p.K + KE - 1) / KE; };
    auto steps = [&](const Tile& x) { return (half_tiles(x) * two + KS - 1) / KS; };         // of each group

    // ---- the copy side: a tile and a k-tile of its own, ahead of the products
    // copy c of an operand: 64 pieces, lane after lane; the k (columns kind) or first k (rows kind) of a lane's piece in its k-tile, and
    // its first column
    auto columns_k = [&](int c, int width) { return BF16 ? 8 * (c & 7) + (lane >> 3) : (c * 64 + lane) / (width / 4); };
    auto columns_at = [&](int c, int width) {
        const int k = columns_k(c, width);
        if constexpr (BF16) return 64 * (c >> 3) + 16 * (((lane & 7) >> 1) ^ (((k >> 1) & 1) | ((k >> 2) & 2))) + 8 * (lane & 1);
        else return 4 * ((lane % (width / 4)) ^ (4 * ((k >> 2) & 3)));
    };
    auto rows_piece = [&](int c) { return (lane & 7) ^ (((8 * c + (lane >> 3)) >> 1) & 7); };
    struct Source { uint64_t A, B[2]; uint32_t a[CA], b[CB]; int KTh, length, kt; };
    Source s;
    bool more = true;                                    // s is a tile that is still to be copied
    auto aim = [&](const Tile& x) {
        s.KTh = half_tiles(x);
        s.length = MODE == WEIGHT ? x.count : p.K;
        s.kt = group;
        if constexpr (AT) s.A = reinterpret_cast<uint64_t>(p.A[x.half]) + static_cast<uint64_t>(x.first) * p.lda * ES;
        else s.A = static_cast<uint64_t>(x.first + x.m0) * p.lda * ES;                                   // + the half's array
        const uint64_t base = MODE == WEIGHT ? static_cast<uint64_t>(x.first) * p.ldb * ES
                                              : static_cast<uint64_t>(x.e) * (MODE == FORWARD ? p.N : p.K) * p.ldb * ES;
        s.B[0] = reinterpret_cast<uint64_t>(p.B[0]) + base;
        s.B[1] = GLU || two == 2 ? reinterpret_cast<uint64_t>(p.B[1]) + base : 0;
#pragma unroll
        for (int i = 0; i < CA; ++i) {
            const int c = wave * CA + i;
            if constexpr (AT) s.a[i] = (static_cast<uint32_t>(columns_k(c, BM)) * p.lda + min(x.m0 + columns_at(c, BM), p.M - PE)) * ES;
            else s.a[i] = static_cast<uint32_t>(min(8 * c + (lane >> 3), x.count - 1 - x.m0)) * p.lda * ES + rows_piece(c) * 16u;
        }
#pragma unroll
        for (int i = 0; i < CB; ++i) {
            const int c = wave * CB + i;
            if constexpr (BT) {
                s.b[i] = (static_cast<uint32_t>(columns_k(c, BN)) * p.ldb + min(x.n0 + columns_at(c, BN), p.N - PE)) * ES;
            } else {
                const int r = 8 * c + (lane >> 3), n = x.n0 + (GLU && r >= BN / 2 ? r - BN / 2 : r);
                s.b[i] = static_cast<uint32_t>(min(n, p.N - 1)) * p.ldb * ES + rows_piece(c) * 16u;
            }
        }
    };
    auto issue = [&](int buf) {
        const int h = s.kt >= s.KTh ? 1 : 0, kt = s.kt - h * s.KTh;
        const int left = KS > 1 && s.kt >= s.KTh * two ? 0 : s.length - kt * KE;             // of the contraction, from this k-tile on
        const uint64_t a = AT ? s.A + static_cast<uint64_t>(kt) * KE * ES * p.lda
                              : s.A + reinterpret_cast<uint64_t>(p.A[h]) + static_cast<uint64_t>(kt) * 128;
        unsigned char* dst = lds + buf * STAGE;
#pragma unroll
        for (int i = 0; i < CA; ++i) {
            const int c = wave * CA + i, k = AT ? columns_k(c, BM) : PE * rows_piece(c);
            copy_piece(a, k < left ? s.a[i] : kPast, dst + c * 1024);
        }
#pragma unroll
        for (int i = 0; i < CB; ++i) {
            const int c = wave * CB + i, k = BT ? columns_k(c, BN) : PE * rows_piece(c);
            const uint64_t b = s.B[GLU ? (c >= BN / 16 ? 1 : 0) : h] + static_cast<uint64_t>(kt) * (BT ? static_cast<uint64_t>(KE) * ES * p.ldb : 128);
            copy_piece(b, k < left ? s.b[i] : kPast, dst + A_BYTES + c * 1024);
        }
    };
    int jn = j;
    auto advance = [&]() {                               // (a source past the last tile goes on copying its last k-tile)
        if (!more) return;
        if (s.kt - group + KS < s.KTh * two) { s.kt += KS; return; }
        jn += grid >> 3;
        Tile n;
        if (find_tile<MODE, DEEP>(p, groups, BM, OUT_N, bid, grid, jn, n)) aim(n);
        else more = false;
    };

    // ---- the product side
    struct Fragment { float f[4]; };                     // bf16: 8 values of k; fp32: 4
    auto fragment = [&](const unsigned char* op, bool columns, int width, int block, int ks) -> Fragment {
        Fragment r;
        if (!columns) {
            const int row = block * 16 + l16;
            const f32x4 v = *reinterpret_cast<const f32x4*>(op + row * 128 + ((4 * ks + kq) ^ ((row >> 1) & 7)) * 16);
            r.f[0] = v[0]; r.f[1] = v[1]; r.f[2] = v[2]; r.f[3] = v[3];
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int k = 16 * ks + 4 * kq + i, col = block * 16 + l16;
                r.f[i] = *reinterpret_cast<const float*>(op + k * width * 4 + (((col >> 2) ^ (4 * kq)) * 16) + (col & 3) * 4);
            }
        }
        return r;
    };
    auto multiply = [&](const Fragment& b, const Fragment& a, f32x4 c) -> f32x4 {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, b), __builtin_bit_cast(bf16x8, a), c, 0, 0, 0);
    };
    // bf16, columns kind: all of a wave's fragments of a k-step (2 or 4: neighbouring blocks of one group of 64 columns) in one statement with
    // its own wait; through the builtin a transposing read waits for all copies on their way, because it is taken to alias what they write
    typedef int v2i __attribute__((ext_vector_type(2)));
    auto join = [](v2i lo, v2i hi) -> bf16x8 {
        typedef int v4i __attribute__((ext_vector_type(4)));
        return __builtin_bit_cast(bf16x8, v4i{lo[0], lo[1], hi[0], hi[1]});
    };
    const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_ptr)lds));
    // LDS address, in the operand's first k-step, of this lane's part of a 16-column block
    auto columns_address = [&](int block) -> uint32_t {
        const int jj = l16 >> 2, f = ((jj >> 1) & 1) | ((kq & 1) << 1);
        return (block >> 2) * 8192 + (8 * kq + jj) * 128 + (((block & 3) ^ f) * 32) + (l16 & 3) * 8;
    };
    auto column_fragments = [&](auto n_, uint32_t at, int first, Fragment* out) {
        constexpr int N = decltype(n_)::value;
        v2i x[4], y[4];
        if constexpr (N == 2)
            asm volatile("ds_read_b64_tr_b16 %0, %4\n\tds_read_b64_tr_b16 %1, %4 offset:512\n\tds_read_b64_tr_b16 %2, %5\n\t"
                         "ds_read_b64_tr_b16 %3, %5 offset:512\n\ts_waitcnt lgkmcnt(0)"
                         : "=&v"(x[0]), "=&v"(y[0]), "=&v"(x[1]), "=&v"(y[1])
                         : "v"(at + columns_address(first)), "v"(at + columns_address(first + 1)) : "memory");
        else
            asm volatile("ds_read_b64_tr_b16 %0, %8\n\tds_read_b64_tr_b16 %1, %8 offset:512\n\tds_read_b64_tr_b16 %2, %9\n\t"
                         "ds_read_b64_tr_b16 %3, %9 offset:512\n\tds_read_b64_tr_b16 %4, %10\n\tds_read_b64_tr_b16 %5, %10 offset:512\n\t"
                         "ds_read_b64_tr_b16 %6, %11\n\tds_read_b64_tr_b16 %7, %11 offset:512\n\ts_waitcnt lgkmcnt(0)"
                         : "=&v"(x[0]), "=&v"(y[0]), "=&v"(x[1]), "=&v"(y[1]), "=&v"(x[2]), "=&v"(y[2]), "=&v"(x[3]), "=&v"(y[3])
                         : "v"(at + columns_address(first)), "v"(at + columns_address(first + 1)), "v"(at + columns_address(first + 2)),
                           "v"(at + columns_address(first + 3)) : "memory");
#pragma unroll
        for (int i = 0; i < N; ++i) out[i] = __builtin_bit_cast(Fragment, join(x[i], y[i]));
    };
    // GLU: the first half of the staged weight rows are gate rows, the second the up rows of the same outputs
    auto b_block = [&](int jb) { return GLU ? (jb >= NB / 2 ? BN / 32 : 0) + wn * (NB / 2) + (jb >= NB / 2 ? jb - NB / 2 : jb) : wn * NB + jb; };

    f32x4 acc[MB][NB];
    auto clear = [&]() {
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
            for (int jb = 0; jb < NB; ++jb) acc[i][jb] = f32x4{0.f, 0.f, 0.f, 0.f};
    };
    auto store = [&]() {
        store_tile<BF16, MODE, GLU, MB, NB, DEEP>(p, t, acc, wm * MB * 16, GLU ? wn * (NB / 2) * 16 : wn * NB * 16, lds + NBUF * STAGE + wave * kPatch);
    };
    auto next_tile = [&]() {
        j += grid >> 3;
        return find_tile<MODE, DEEP>(p, groups, BM, OUT_N, bid, grid, j, t);
    };
    auto barrier = [&]() {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    aim(t);
    if constexpr (DEEP) {
        // 128 rows x 64 columns to a wave, one workgroup to a CU: nothing else covers a wait, so the loop is written out.  A k-tile is four
        // substeps of 16 MFMAs: k-step 0 and 1 of row blocks 0 - 3 and 4 - 7.  Fragments are read a substep ahead; the barrier stands
        // before the last substep, when all reads of the buffer are done: behind it go the next k-tile's first reads (that it has landed is
        // what was waited for), and the copies of the one after that into the buffer just left.
        // MFMAs and the fragment reads beside them are assembly: a transposing read through the builtin waits for all copies on their way,
        // because it is taken to alias what they write.  A statement holds 8 MFMAs (two row blocks, four column blocks), behind the first of
        // them the reads of up to four fragments, and its own wait at the end, so that they land under the other MFMAs and its outputs are
        // ordinary registers.  What the compiler cannot see in it: two wait states between an ordinary write of an operand and the
        // MFMA (the s_nop in front), and that an accumulator is not to be touched right behind (the s_nops at the end of the
        // loop; inside it nothing else uses one).
        bf16x8 fa[2][4], fb[2][4];
        // LDS addresses (buffer 0) of this lane's part of a fragment; columns: of the four 16-column blocks of the wave's first group, + 512: the
        // k four further on, + 4096: the second k-step, + 8192: the next group; rows: of the two k-steps of the wave's first block, + 2048:
        // the next block
        uint32_t at_a[4], at_b[4];
#pragma unroll
        for (int o = 0; o < 4; ++o) {
            const uint32_t columns = columns_address(o), rows = l16 * 128 + ((4 * (o & 1) + kq) ^ ((l16 >> 1) & 7)) * 16;
            at_a[o] = lds0 + wm * 16384 + (AT ? columns : rows);
            at_b[o] = lds0 + A_BYTES + (BT ? wn * 8192 + columns : wn * (GLU ? 4096 : 8192) + rows);
        }
#define ETR_MF(C, B, A) "v_mfma_f32_16x16x32_bf16 %[c" #C "], %[b" #B "], %[a" #A "], %[c" #C "]\n\t"
#define ETR_REST ETR_MF(1, 0, 1) ETR_MF(3, 1, 1) ETR_MF(2, 1, 0) ETR_MF(4, 2, 0) ETR_MF(5, 2, 1) ETR_MF(7, 3, 1) ETR_MF(6, 3, 0)
#define ETR_TR(N) "ds_read_b64_tr_b16 %[x" #N "], %[p" #N "] offset:%c[o" #N "]\n\tds_read_b64_tr_b16 %[y" #N "], %[p" #N "] offset:%c[q" #N "]\n\t"
#define ETR_RD(N) "ds_read_b128 %[r" #N "], %[p" #N "] offset:%c[o" #N "]\n\t"
#define ETR_ACC [c0] "+v"(acc[I][0]), [c1] "+v"(acc[I + 1][0]), [c2] "+v"(acc[I][1]), [c3] "+v"(acc[I + 1][1]), [c4] "+v"(acc[I][2]), \
                [c5] "+v"(acc[I + 1][2]), [c6] "+v"(acc[I][3]), [c7] "+v"(acc[I + 1][3])
#define ETR_FRAGMENTS [a0] "v"(a[0]), [a1] "v"(a[1]), [b0] "v"(b[0]), [b1] "v"(b[1]), [b2] "v"(b[2]), [b3] "v"(b[3])
#define ETR_OUT(N) [x##N] "=&v"(x[N]), [y##N] "=&v"(y[N])
#define ETR_ROW(N) [r##N] "=&v"(out[N])
#define ETR_AT(N) [p##N] "v"(COLUMNS ? at[(F + N) & 3] + slot : at[KSTEP] + slot), [o##N] "n"(offset(N)), [q##N] "n"(offset(N) + 512)
        // acc[I], acc[I + 1] += a[0..1] x b[0..3] (I < 0: no products); R fragments of k-step KSTEP from block F of half H of an operand (its
        // kind, its addresses and whether it is B) on into `out`
        auto step8 = [&](auto block, const bf16x8* a, const bf16x8* b, auto reads, auto columns_, auto is_b, const uint32_t* at, uint32_t slot, auto ks_, auto half,
                         auto from, bf16x8* out) {
            constexpr int I = decltype(block)::value < 0 ? 0 : decltype(block)::value, R = decltype(reads)::value, KSTEP = decltype(ks_)::value,
                          H = decltype(half)::value, F = decltype(from)::value;
            constexpr bool NONE = decltype(block)::value < 0, COLUMNS = decltype(columns_)::value, OF_B = decltype(is_b)::value;
            auto offset = [](int n) constexpr {
                if (COLUMNS) return KSTEP * 4096 + H * 8192;
                if (OF_B && GLU) return ((F + n) >> 1) * 16384 + ((F + n) & 1) * 2048;       // the up rows lie 128 rows behind the gate rows
                return (4 * H + F + n) * 2048;
            };
            v2i x[4], y[4];
            if constexpr (NONE && COLUMNS)
                asm volatile(ETR_TR(0) ETR_TR(1) ETR_TR(2) ETR_TR(3) "s_waitcnt lgkmcnt(0)"
                             : ETR_OUT(0), ETR_OUT(1), ETR_OUT(2), ETR_OUT(3) : ETR_AT(0), ETR_AT(1), ETR_AT(2), ETR_AT(3) : "memory");
            else if constexpr (NONE)
                asm volatile(ETR_RD(0) ETR_RD(1) ETR_RD(2) ETR_RD(3) "s_waitcnt lgkmcnt(0)"
                             : ETR_ROW(0), ETR_ROW(1), ETR_ROW(2), ETR_ROW(3) : ETR_AT(0), ETR_AT(1), ETR_AT(2), ETR_AT(3) : "memory");
            else if constexpr (R == 2 && COLUMNS)
                asm volatile("s_nop 1\n\t" ETR_MF(0, 0, 0) ETR_TR(0) ETR_TR(1) ETR_REST "s_waitcnt lgkmcnt(0)"
                             : ETR_ACC, ETR_OUT(0), ETR_OUT(1) : ETR_FRAGMENTS, ETR_AT(0), ETR_AT(1) : "memory");
            else if constexpr (R == 2)
                asm volatile("s_nop 1\n\t" ETR_MF(0, 0, 0) ETR_RD(0) ETR_RD(1) ETR_REST "s_waitcnt lgkmcnt(0)"
                             : ETR_ACC, ETR_ROW(0), ETR_ROW(1) : ETR_FRAGMENTS, ETR_AT(0), ETR_AT(1) : "memory");
            else if constexpr (COLUMNS)
                asm volatile("s_nop 1\n\t" ETR_MF(0, 0, 0) ETR_TR(0) ETR_TR(1) ETR_TR(2) ETR_TR(3) ETR_REST "s_waitcnt lgkmcnt(0)"
                             : ETR_ACC, ETR_OUT(0), ETR_OUT(1), ETR_OUT(2), ETR_OUT(3)
                             : ETR_FRAGMENTS, ETR_AT(0), ETR_AT(1), ETR_AT(2), ETR_AT(3) : "memory");
            else
                asm volatile("s_nop 1\n\t" ETR_MF(0, 0, 0) ETR_RD(0) ETR_RD(1) ETR_RD(2) ETR_RD(3) ETR_REST "s_waitcnt lgkmcnt(0)"
                             : ETR_ACC, ETR_ROW(0), ETR_ROW(1), ETR_ROW(2), ETR_ROW(3)
                             : ETR_FRAGMENTS, ETR_AT(0), ETR_AT(1), ETR_AT(2), ETR_AT(3) : "memory");
            if constexpr (COLUMNS) {
#pragma unroll
                for (int i = 0; i < (NONE ? 4 : R); ++i) out[i] = join(x[i], y[i]);
            }
        };
#undef ETR_MF
#undef ETR_REST
#undef ETR_TR
#undef ETR_RD
#undef ETR_ACC
#undef ETR_FRAGMENTS
#undef ETR_OUT
#undef ETR_ROW
#undef ETR_AT
#define ETR_INT(V) std::integral_constant<int, (V)>{}
        // 64-row halves of this wave's 128 that have a row to store at all, none if its columns lie past the last: tiles at the end of an
        // expert's rows multiply what they have, and the wave beside them on the SIMD has the matrix pipe for itself meanwhile
        int live = 2;
        auto count_live = [&]() {
            const int rows_left = t.limit - t.m0 - wm * 128;
            live = t.n0 + (GLU ? wn * 32 : wn * 64) < p.N ? min(max((rows_left + 63) >> 6, 0), 2) : 0;
        };
        // Substep (ks, h); then the next fragments: of A (half nh, k-step nks) and, with nbks >= 0, of B, from buffer b.
        auto substep = [&](auto live_, auto ks_, auto h_, int b, auto nh_, auto nks_, auto nbks_, auto&& behind) {
            constexpr int ks = decltype(ks_)::value, h = decltype(h_)::value, nh = decltype(nh_)::value, nks = decltype(nks_)::value,
                          nbks = decltype(nbks_)::value, first = h >= decltype(live_)::value ? -1 : 4 * h, second = first < 0 ? -1 : first + 2;
            const uint32_t slot = static_cast<uint32_t>(b) * STAGE;
            // first statement: the fragments of B (all four), or the first two of A; second: those of A that are left.  Without products
            // (nothing of these 64 rows is stored): four at a time
            if constexpr (nbks >= 0)
                step8(ETR_INT(first), fa[h], fb[ks], ETR_INT(4), ETR_INT(BT), ETR_INT(1), at_b, slot, ETR_INT(nbks < 0 ? 0 : nbks), ETR_INT(0), ETR_INT(0), fb[nbks < 0 ? 0 : nbks]);
            else if constexpr (first >= 0)
                step8(ETR_INT(first), fa[h], fb[ks], ETR_INT(2), ETR_INT(AT), ETR_INT(0), at_a, slot, ETR_INT(nks), ETR_INT(nh), ETR_INT(0), fa[nh]);
            __builtin_amdgcn_sched_barrier(0);
            behind();
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (nbks >= 0 || first < 0)
                step8(ETR_INT(second), fa[h] + 2, fb[ks], ETR_INT(4), ETR_INT(AT), ETR_INT(0), at_a, slot, ETR_INT(nks), ETR_INT(nh), ETR_INT(0), fa[nh]);
            else
                step8(ETR_INT(second), fa[h] + 2, fb[ks], ETR_INT(2), ETR_INT(AT), ETR_INT(0), at_a, slot, ETR_INT(nks), ETR_INT(nh), ETR_INT(2), fa[nh] + 2);
            __builtin_amdgcn_sched_barrier(0);
        };
        issue(0); advance();
        issue(1); advance();
        wait_copies<CA + CB>();
        barrier();
        step8(ETR_INT(-1), nullptr, nullptr, ETR_INT(4), ETR_INT(AT), ETR_INT(0), at_a, 0u, ETR_INT(0), ETR_INT(0), ETR_INT(0), fa[0]);
        step8(ETR_INT(-1), nullptr, nullptr, ETR_INT(4), ETR_INT(BT), ETR_INT(1), at_b, 0u, ETR_INT(0), ETR_INT(0), ETR_INT(0), fb[0]);
        int buf = 0;
        do {
            clear();
            count_live();
            const int KT = half_tiles(t) * two;
            auto k_loop = [&](auto n) {
                for (int kt = 0; kt < KT; ++kt) {
                    substep(n, ETR_INT(0), ETR_INT(0), buf, ETR_INT(1), ETR_INT(0), ETR_INT(1), [&]() {});
                    substep(n, ETR_INT(0), ETR_INT(1), buf, ETR_INT(0), ETR_INT(1), ETR_INT(-1), [&]() {});
                    substep(n, ETR_INT(1), ETR_INT(0), buf, ETR_INT(1), ETR_INT(1), ETR_INT(-1), [&]() {});
                    __builtin_amdgcn_s_waitcnt(0x0070);  // vmcnt(0), lgkmcnt(0): the next k-tile is here, this wave's reads are done
                    barrier();
                    __builtin_amdgcn_sched_barrier(0);
                    substep(n, ETR_INT(1), ETR_INT(1), buf ^ 1, ETR_INT(0), ETR_INT(0), ETR_INT(0), [&]() { issue(buf); });
                    advance();
                    buf ^= 1;
                }
                asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");         // the last products are written before anything reads them
            };
            // (the empty statements: what the three ways leave behind is one set of registers, not merged by copies)
            auto pin = [&]() {
#pragma unroll
                for (int i = 0; i < MB; ++i)
#pragma unroll
                    for (int jb = 0; jb < NB; ++jb) asm volatile("" : "+v"(acc[i][jb]));
#pragma unroll
                for (int i = 0; i < 4; ++i) asm volatile("" : "+v"(fa[0][i]), "+v"(fb[0][i]));
            };
            if (live == 2) k_loop(ETR_INT(2));
            pin();
            if (live == 1) k_loop(ETR_INT(1));
            pin();
            if (live == 0) k_loop(ETR_INT(0));
            pin();
            store();
        } while (next_tile());
#undef ETR_INT
    } else {
#pragma unroll
        for (int b = 0; b < NBUF - 1; ++b) { issue(b); advance(); }
        int buf = 0;
        for (;;) {
            clear();
            const int KT = steps(t);
            for (int kt = 0; kt < KT; ++kt) {
                wait_copies<(NBUF - 2) * (CA + CB)>();   // this wave's part of the k-tile has landed
                barrier();                               // ... and everybody's; and everybody is done with the buffer before it
                issue(buf == 0 ? NBUF - 1 : buf - 1);
                advance();
                const unsigned char* op = lds + buf * STAGE;
#pragma unroll
                for (int ks = 0; ks < 2; ++ks) {
                    const uint32_t at = lds0 + buf * STAGE + ks * 4096;
                    Fragment fa[MB], fb[NB];
                    if constexpr (BF16 && BT) {
                        column_fragments(std::integral_constant<int, NB>{}, at + A_BYTES, wn * NB, fb);
                    } else {
#pragma unroll
                        for (int jb = 0; jb < NB; ++jb) fb[jb] = fragment(op + A_BYTES, BT, BN, b_block(jb), ks);
                    }
                    if constexpr (BF16 && AT) {
                        column_fragments(std::integral_constant<int, MB>{}, at, wm * MB, fa);
                    } else {
#pragma unroll
                        for (int i = 0; i < MB; ++i) fa[i] = fragment(op, AT, BM, wm * MB + i, ks);
                    }
                    if constexpr (BF16) {
#pragma unroll
                        for (int i = 0; i < MB; ++i)
#pragma unroll
                            for (int jb = 0; jb < NB; ++jb) acc[i][jb] = multiply(fb[jb], fa[i], acc[i][jb]);
                    } else {                             // four MFMAs to a pair of fragments: not one behind the other
#pragma unroll
                        for (int v = 0; v < 4; ++v)
#pragma unroll
                            for (int i = 0; i < MB; ++i)
#pragma unroll
                                for (int jb = 0; jb < NB; ++jb)
                                    acc[i][jb] = __builtin_amdgcn_mfma_f32_16x16x4f32(fb[jb].f[v], fa[i].f[v], acc[i][jb], 0, 0, 0);
                    }
                }
                buf = buf + 1 == NBUF ? 0 : buf + 1;
            }
            if constexpr (KS > 1) {
                wait_copies<0>();                        // nothing is on its way into the buffers any more
                barrier();
                f32x4* sums = reinterpret_cast<f32x4*>(lds) + (threadIdx.x % (NW * 64));
                if (group > 0) {
#pragma unroll
                    for (int i = 0; i < MB; ++i)
#pragma unroll
                        for (int jb = 0; jb < NB; ++jb) sums[(i * NB + jb) * NW * 64] = acc[i][jb];
                }
                __syncthreads();
                if (group > 0) return;
#pragma unroll
                for (int g = 1; g < KS; ++g)
#pragma unroll
                    for (int i = 0; i < MB; ++i)
#pragma unroll
                        for (int jb = 0; jb < NB; ++jb) acc[i][jb] += sums[g * (NBUF * STAGE / 16) + (i * NB + jb) * NW * 64];
                store();
                return;
            }
            store();
            if (!next_tile()) break;
            wait_copies<0>();                            // (the stores too: the counted waits are for copies alone)
        }
    }
    wait_copies<0>();                                    // the copies that nobody needed
}

template <bool BF16, int BM, int BN, int WM, int WN, int NBUF, int KS, int MODE, bool GLU>
__global__ __launch_bounds__(WM* WN * KS * 64, WM * WN * KS > 8 ? 4 : 2) void linear_kernel(LinearParams p) {
    linear_tiles<BF16, BM, BN, WM, WN, NBUF, KS, MODE, GLU>(p, blockIdx.x, gridDim.x);
}
// dx and dw in one launch, where both take the small tiles: the first `n_input` workgroups (a multiple of 8) are dx's
template <bool BF16, int BM, int BN, int WM, int WN, int NBUF, int KS>
__global__ __launch_bounds__(WM* WN * KS * 64, KS > 1 ? 4 : 2) void linear_backward_kernel(LinearParams input, LinearParams weight, int n_input) {
    if (static_cast<int>(blockIdx.x) < n_input) linear_tiles<BF16, BM, BN, WM, WN, NBUF, KS, INPUT, false>(input, blockIdx.x, n_input);
    else linear_tiles<BF16, BM, BN, WM, WN, NBUF, KS, WEIGHT, false>(weight, blockIdx.x - n_input, gridDim.x - n_input);
}

// ---- the element-wise middle of the backward ----------------------------------------------------------------------------
//
// da = dy act'(a) (db = dy SiLU(a)) and the column sums of both over 32 rows of an expert, before they are rounded.  A workgroup has such
// a chunk of rows and 64 pieces of columns; a wave every fourth row of it.  Bound by memory: one or two rows of pre-activations and
// one of dy in, one or two out: 16 384 x 2048 bf16, sums alone, 22 us (3 TB/s; a third of it the launch and the last chunks); 2250 x 1048 fp32 with
// GELU 11 us, where chunks of 128 rows took 33.
constexpr int kChunk = 32;
struct MiddleParams {
    const piece_t* pre; const piece_t* pre_up; const piece_t* dy; piece_t* da; piece_t* db;
    float* part;            // [2 with SwiGLU][chunks][N], optional
    float* dbias[2];        // [E][N]; where no expert has more than a chunk of rows: the sums go here at once (a workgroup per expert)
    const int32_t* offsets;
    int rows, E, N, pieces, act, chunks;
};
template <bool BF16>
__global__ __launch_bounds__(256) void linear_middle_kernel(MiddleParams p) {
    using R = Piece<BF16>;
    constexpr int V = R::kN;
    __shared__ float sums[3][64][2 * V];
    LinearParams q{};
    q.offsets = p.offsets; q.rows = p.rows; q.E = p.E;
    Groups g;
    g.load(q, kChunk);
    const int chunk = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const bool direct = p.dbias[0] != nullptr;
    if (!direct && chunk >= __builtin_amdgcn_readlane(g.tiles_incl, 63)) return;
    const int e = direct ? chunk : __builtin_ctzll(__ballot(g.tiles_incl > chunk));
    const int in_group = direct ? 0 : chunk - (__builtin_amdgcn_readlane(g.tiles_incl, e) - __builtin_amdgcn_readlane(g.tiles, e));
    const int first = __builtin_amdgcn_readlane(g.first, e) + in_group * kChunk;
    const int n_rows = min(kChunk, __builtin_amdgcn_readlane(g.count, e) - in_group * kChunk);
    const int c = blockIdx.y * 64 + lane;
    const bool in = c < p.pieces, glu = p.act == ETR_ACT_SWIGLU;
    float sa[V], sb[V];
#pragma unroll
    for (int i = 0; i < V; ++i) sa[i] = sb[i] = 0.f;
    // four rows of a wave at a time, all of them requested before the first is used
    for (int r0 = wave; in && r0 < n_rows; r0 += 16) {
        piece_t dv[4], av[4], bv[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (r0 + 4 * u >= n_rows) continue;
            const size_t at = static_cast<size_t>(first + r0 + 4 * u) * p.pieces + c;
            dv[u] = p.dy[at];
            if (p.act != ETR_ACT_NONE) av[u] = p.pre[at];
            if (glu) bv[u] = p.pre_up[at];
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (r0 + 4 * u >= n_rows) continue;
            const size_t at = static_cast<size_t>(first + r0 + 4 * u) * p.pieces + c;
            float d[V], a[V], b[V];
            R::unpack(dv[u], d);
            if (p.act != ETR_ACT_NONE) R::unpack(av[u], a);
            if (glu) R::unpack(bv[u], b);
            if (p.act == ETR_ACT_GELU) {
#pragma unroll
                for (int i = 0; i < V; ++i)
                    a[i] = d[i] * (normal_cdf<BF16>(a[i]) + a[i] * 0.39894228040143268f * (BF16 ? __expf(-0.5f * a[i] * a[i]) : gaussian_f32(a[i])));
            } else if (p.act != ETR_ACT_NONE) {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float sg = sigmoid<BF16>(a[i]), grad = sg * (1.0f + a[i] * (1.0f - sg));
                    const float up = glu ? b[i] : 1.0f;
                    b[i] = d[i] * a[i] * sg;
                    a[i] = d[i] * up * grad;
                }
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i) a[i] = d[i];
            }
            if (p.da) p.da[at] = R::pack(a);
            if (glu && p.db) p.db[at] = R::pack(b);
#pragma unroll
            for (int i = 0; i < V; ++i) { sa[i] += a[i]; sb[i] += glu ? b[i] : 0.f; }
        }
    }
    if (!p.part && !direct) return;
    if (wave > 0) {
#pragma unroll
        for (int i = 0; i < V; ++i) { sums[wave - 1][lane][i] = sa[i]; sums[wave - 1][lane][V + i] = sb[i]; }
    }
    __syncthreads();
    if (wave > 0 || !in) return;
    const size_t at = static_cast<size_t>(chunk) * p.N + static_cast<size_t>(c) * V;
    float* out = (direct ? p.dbias[0] : p.part) + at;
    float* out_up = direct ? p.dbias[1] + at : out + static_cast<size_t>(p.chunks) * p.N;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        out[i] = ((sa[i] + sums[0][lane][i]) + sums[1][lane][i]) + sums[2][lane][i];
        if (glu) out_up[i] = ((sb[i] + sums[0][lane][V + i]) + sums[1][lane][V + i]) + sums[2][lane][V + i];
    }
}

// dbias[e][n]: the chunks of expert e, sixteen groups of them side by side, in a fixed order
__global__ __launch_bounds__(1024) void linear_bias_kernel(MiddleParams p, float* dbias, float* dbias_up) {
    __shared__ float sums[16][64];
    LinearParams q{};
    q.offsets = p.offsets; q.rows = p.rows; q.E = p.E;
    Groups g;
    g.load(q, kChunk);
    const int e = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = blockIdx.x * 64 + lane;
    // (offsets that are no ascending ones may name more chunks than there are)
    const int begin = min(__builtin_amdgcn_readlane(g.tiles_incl, e) - __builtin_amdgcn_readlane(g.tiles, e), p.chunks);
    const int tiles = min(__builtin_amdgcn_readlane(g.tiles, e), p.chunks - begin);
    const float* part = p.part + static_cast<size_t>(blockIdx.z) * p.chunks * p.N;
    float s = 0.f;
    if (n < p.N) {
#pragma unroll 4
        for (int i = wave; i < tiles; i += 16) s += part[static_cast<size_t>(begin + i) * p.N + n];
    }
    sums[wave][lane] = s;
    __syncthreads();
    if (wave > 0 || n >= p.N) return;
    s = 0.f;
#pragma unroll
    for (int w = 0; w < 16; ++w) s += sums[w][lane];
    (blockIdx.z ? dbias_up : dbias)[static_cast<size_t>(e) * p.N + n] = s;
}

// ---- host ------------------------------------------------------------------------------------------------------------

long long tiles_at_most(const LinearParams& p, int mode, int BM, int out_n) {
    const long long columns = (p.N + out_n - 1) / out_n;
    if (mode == WEIGHT) return columns * ((p.M + BM - 1) / BM) * p.E * (p.glu ? 2 : 1);
    // full tiles of all rows together, and one more in part for each group
    return columns * (p.rows / BM + std::min(p.E, p.rows));
}

template <int BM, int BN, bool GLU> long long plan_tiles(LinearParams& p, int mode) {          // fills NT; the tiles at most
    p.NT = (p.N + (GLU ? BN / 2 : BN) - 1) / (GLU ? BN / 2 : BN);
    return tiles_at_most(p, mode, BM, GLU ? BN / 2 : BN);
}
template <bool BF16, int BM, int BN, int WM, int WN, int NBUF, int KS, int MODE, bool GLU>
hipError_t launch_tiles(LinearParams p, hipStream_t st) {
    constexpr bool large = BM * BN >= 256 * 256;
    constexpr size_t lds = static_cast<size_t>(BM + BN) * 128 * NBUF * KS + (large ? WM * WN * kPatch : 0);
    auto kern = linear_kernel<BF16, BM, BN, WM, WN, NBUF, KS, MODE, GLU>;
    const hipError_t err = ensure_dynamic_lds(reinterpret_cast<const void*>(kern), lds);
    if (err != hipSuccess) return err;
    const long long tiles = plan_tiles<BM, BN, GLU>(p, MODE);
    // one workgroup on each CU that walks the tiles (up to four parts of one), or (small tiles) one for each of them
    const long long most = large ? cu_count() / 8 : 1 << 17, wanted = (tiles + 7) / 8 * (large ? 4 : 1);
    if (KS > 1 && wanted > most) return hipErrorInvalidValue;
    const long long blocks = std::min(wanted, most) * 8;
    hipLaunchKernelGGL(kern, dim3(static_cast<unsigned>(blocks)), dim3(WM * WN * KS * 64), lds, st, p);
    return hipGetLastError();
}
template <bool BF16, int NBUF, int KS>
hipError_t launch_small_backward(LinearParams input, LinearParams weight, hipStream_t st) {
    constexpr size_t lds = 128 * 128 * NBUF * KS;
    auto kern = linear_backward_kernel<BF16, 64, 64, 2, 2, NBUF, KS>;
    const hipError_t err = ensure_dynamic_lds(reinterpret_cast<const void*>(kern), lds);
    if (err != hipSuccess) return err;
    const long long most = 1 << 17, tiles_input = plan_tiles<64, 64, false>(input, INPUT), tiles_weight = plan_tiles<64, 64, false>(weight, WEIGHT);
    const long long n_input = std::min((tiles_input + 7) / 8, most) * 8, n_weight = std::min((tiles_weight + 7) / 8, most) * 8;
    if (KS > 1 && std::max(tiles_input, tiles_weight) > 8 * most) return hipErrorInvalidValue;
    hipLaunchKernelGGL(kern, dim3(static_cast<unsigned>(n_input + n_weight)), dim3(256 * KS), lds, st, input, weight, static_cast<int>(n_input));
    return hipGetLastError();
}

// The tiles of a product, by estimate.  THIN: 16 rows x 16 columns (SwiGLU 32 weight rows, dx 64 columns), every wave a group of its own, 16
// (8) to share the contraction; ROWS32: 32 rows x 64 weight rows (128 for SwiGLU and dx); deep: four groups of waves share a tile's contraction.
enum class Tiles { THIN, ROWS32, T64, T128, T256 };
struct Choice { Tiles tiles; bool deep; double us; };
// Estimated microseconds: rounds of tiles over the places that they have on the chip, each a time per k-tile (alone ... chip full) and a time
// besides.  In microseconds per 64-deep bf16 k-tile, fitted to 130 products (1 to 16384 rows in 1 to 64 groups, widths of 128 to 8192; each
// forward, with SwiGLU, dx and dw, by all the tiles); on 130 others the choice takes 1.4 % more than the best of the tiles, on average:
//   T256    one to a CU    0.94 ... 1.69 (the power limit), 5.5 besides; a last round of half the CUs or fewer goes in parts
//   T128    two to a CU    0.67 ... 1.2, 4.2
//   T64     two to a CU    0.33 ... 0.55, 2.8; deep: one to a CU, 1.05 per four k-tiles, 3
//   ROWS32  three (of 64 columns) or two to a CU, 0.25 ... 0.45 or 0.38 ... 0.6, 2; deep: one to a CU, 0.65 or 1.6 per four, 3
//   THIN    one to a CU, 0.45 (SwiGLU 0.85, dx 0.8) per 16 (8) k-tiles, 3.2, and 1.8 for them all; fp32 0.7 (0.85, 1.45)
// Few rows, THIN and the best of the others: 18 rows, 3840 x 1472 6.0 and 12.0 us, fp32 9.8 and 39.2; 64 rows, 4096 x 4096 24.9 and 12.7, fp32
// 38.4 and 41.6; dx of 64 rows, 8192 x 256 16.2 and 27.8, fp32 50 and 143.
// 2048 rows in 16 groups, 2048 x 2048: T256 46, T128 33, T64 40 us; 4096 rows: 48, 57, 68; 512 rows dense, 4096 x 4096: 61, 43, 29.
// fp32, per 32-deep k-tile, where the CU's matrix pipes set the time as soon as two 64 x 64 tiles share it: T64 0.7 alone or 0.47 per tile on the
// CU, and 0.5 for its epilogue, ROWS32 0.45 or 0.25 and 0.4 (of 128 columns: T64's); deep: a quarter of the k-tiles, 4.5 times the work in
// each.  (A tile of 128 x 128: 2.1 and 2.4, more than the four 64 x 64 tiles in its place, and 2.0 alone: not built.)
double estimate_us(Choice c, double tiles, double k_tiles, bool wide, bool transposed, bool bf16) {
    const double cus = cu_count();
    if (c.tiles == Tiles::THIN) {
        const double step = bf16 ? (transposed ? 0.8 : wide ? 0.85 : 0.45) : transposed ? 1.45 : wide ? 0.85 : 0.7;
        return 1.8 + std::ceil(std::max(1.0, tiles / cus) - 0.1) * (3.2 + step * std::ceil(k_tiles / (wide ? 8 : 16)));
    }
    const double steps = c.deep ? std::ceil(k_tiles / 4) : k_tiles;
    if (!bf16) {
        const bool t64 = c.tiles == Tiles::T64 || wide;
        const double alone = t64 ? 0.7 : 0.45, each = t64 ? 0.47 : 0.25, epilogue = t64 ? 0.5 : 0.4;
        return std::max(steps * (c.deep ? 1.7 * alone : alone), std::max(1.0, tiles / cus) * (steps * each * (c.deep ? 4.5 : 1.0) + epilogue)) + (c.deep ? 5.0 : 4.0);
    }
    double places = 2, alone = 0, full = 0, besides = 0;
    switch (c.tiles) {
        case Tiles::THIN: break;
        case Tiles::T256: places = 1; alone = 0.94; full = 1.69; besides = 5.5; break;
        case Tiles::T128: alone = 0.67; full = 1.2; besides = 4.2; break;
        case Tiles::T64: alone = 0.33; full = 0.55; besides = 2.8; break;
        case Tiles::ROWS32: places = wide ? 2 : 3; alone = wide ? 0.38 : 0.25; full = wide ? 0.6 : 0.45; besides = 2.0; break;
    }
    if (c.deep) { places = 1; alone = full = c.tiles == Tiles::T64 ? 1.05 : wide ? 1.6 : 0.65; besides = 3.0; }
    const double r = tiles / (places * cus), rest = r - std::floor(r);
    double rounds = r <= 1 ? 1.0 : c.deep ? std::ceil(r - 0.1) : c.tiles == Tiles::T256 ? std::ceil(r) : r < 4 ? std::ceil(2 * r) / 2 : r + 0.25;
    if (c.tiles == Tiles::T256 && r > 1 && rest > 0) rounds = std::floor(r) + (rest <= 0.25 ? 0.55 : rest <= 0.5 ? 0.7 : 1.0);
    double crowd = std::min(1.0, r);                     // half of it the chip's, half from where tiles share a CU
    if (places > 1) crowd = 0.5 * crowd + 0.5 * std::max(0.0, std::min(1.0, (r * places - 1) / (places - 1)));
    return rounds * (steps * (alone + (full - alone) * crowd) + besides);
}
// small: only T64 is to be had, deep or not
template <int MODE, bool GLU>
Choice choose_tiles(const LinearParams& p, bool bf16, bool small = false, bool small_deep = false) {
    const double rows_each = MODE == WEIGHT ? p.M : static_cast<double>(p.rows) / p.E;           // rows of a group, on average
    const double groups = MODE == WEIGHT ? p.E * (p.glu ? 2 : 1) : std::min(p.E, p.rows);
    const int halves = MODE == INPUT && p.glu ? 2 : 1, depth = bf16 ? 64 : 32;
    const double k_tiles = halves * std::ceil((MODE == WEIGHT ? static_cast<double>(p.rows) / p.E : p.K) / depth);
    // row tiles of a group: half a tile more than its rows fill, on average, where they are the batch's
    auto tiles = [&](int BM, int BN) {
        const double whole = std::ceil(rows_each / BM), mean = MODE == WEIGHT || rows_each < 1 ? whole : std::max(whole, rows_each / BM + (p.E > 1 ? 0.5 : 0.0));
        return groups * mean * std::ceil(static_cast<double>(p.N) / (GLU ? BN / 2 : BN));
    };
    Choice best{Tiles::T64, false, 1e30};
    auto offer = [&](Tiles kind, bool deep, int BM, int BN) {
        const double n = tiles(BM, BN);
        if (deep && ((k_tiles < 8 && kind != Tiles::THIN) || n > 4.0 * cu_count())) return;           // (one tile to a workgroup)
        double us = estimate_us({kind, deep, 0}, n, k_tiles, kind == Tiles::THIN ? BN > 16 : BN == 128, MODE != FORWARD, bf16);
        // dx in bf16 by THIN reads the weights, 128 bytes of a row at a time, at 3.5 TB/s at most; ROWS32 at 5.5 (64 experts of 512 x 6784, 907
        // rows: 105 and 81 us)
        if (MODE == INPUT && bf16 && kind == Tiles::THIN) us = std::max(us, groups * p.N * halves * p.K * 2 / 3.5e6);
        if (us < best.us) best = {kind, deep, us};
    };
    const int columns32 = GLU || MODE == INPUT ? 128 : 64;
    if (small) {
        offer(Tiles::T64, small_deep, 64, 64);
        return best;
    }
    if (bf16) {
        offer(Tiles::T256, false, 256, 256);
        offer(Tiles::T128, false, 128, 128);
    }
    offer(Tiles::T64, false, 64, 64);
    offer(Tiles::T64, true, 64, 64);
    if (MODE != WEIGHT && rows_each <= 256) {
        offer(Tiles::ROWS32, false, 32, columns32);
        offer(Tiles::ROWS32, true, 32, columns32);
    }
    if (MODE != WEIGHT) offer(Tiles::THIN, true, 16, MODE == INPUT ? 64 : GLU ? 32 : 16);
    return best;
}
template <bool BF16, int MODE, bool GLU>
hipError_t launch_typed(const LinearParams& p, hipStream_t st) {
    const Choice c = choose_tiles<MODE, GLU>(p, BF16);
    if constexpr (MODE != WEIGHT) {
        constexpr int columns = MODE == INPUT ? 64 : GLU ? 32 : 16;
        if (c.tiles == Tiles::THIN) return launch_tiles<BF16, 16, columns, 1, 1, 2, (columns > 16 ? 8 : 16), MODE, GLU>(p, st);
    }
    if constexpr (MODE != WEIGHT) {
        if (c.tiles == Tiles::ROWS32) {
            if constexpr (GLU || MODE == INPUT)
                return c.deep ? launch_tiles<BF16, 32, 128, 1, 4, 2, 4, MODE, GLU>(p, st) : launch_tiles<BF16, 32, 128, 1, 4, 4, 1, MODE, GLU>(p, st);
            else
                return c.deep ? launch_tiles<BF16, 32, 64, 1, 4, 3, 4, MODE, GLU>(p, st) : launch_tiles<BF16, 32, 64, 1, 4, 4, 1, MODE, GLU>(p, st);
        }
    }
    if constexpr (BF16) {
        if (c.tiles == Tiles::T256) return launch_tiles<true, 256, 256, 2, 4, 2, 1, MODE, GLU>(p, st);
        if (c.tiles == Tiles::T128) return launch_tiles<true, 128, 128, 2, 2, 2, 1, MODE, GLU>(p, st);
    }
    return c.deep ? launch_tiles<BF16, 64, 64, 2, 2, 2, 4, MODE, GLU>(p, st) : launch_tiles<BF16, 64, 64, 2, 2, BF16 ? 4 : 2, 1, MODE, GLU>(p, st);
}
template <int MODE, bool GLU>
hipError_t launch_product(const LinearParams& p, bool bf16, hipStream_t st) {
    return bf16 ? launch_typed<true, MODE, GLU>(p, st) : launch_typed<false, MODE, GLU>(p, st);
}

// dx and dw in one launch of 64 x 64 tiles, unless each by its own takes less: the longer of the two while they fit on the chip together, else
// their sum less what a launch costs.  Together and apart: 500 rows, 512 x 512 in fp32 14.0 and 19.9 us; 2500 in 8 groups, 1048 x 520 in fp32
// 92.0 and 97.4; 112 in 4, 384 x 1664 21.4 and 25.3 (with the forward); 18 rows, 3840 x 1472 in fp32 87.9 and 37.6
enum class Joint { NONE, PLAIN, DEEP };
Joint choose_joint(const LinearParams& p, const LinearParams& q, bool bf16) {
    const Choice ci = choose_tiles<INPUT, false>(p, bf16), cw = choose_tiles<WEIGHT, false>(q, bf16);
    const double apart = ci.us + cw.us, weight_us = choose_tiles<WEIGHT, false>(q, bf16, true).us;
    const long long tiles = tiles_at_most(p, INPUT, 64, 64) + tiles_at_most(q, WEIGHT, 64, 64);
    auto together = [&](bool deep) {
        const double input_us = choose_tiles<INPUT, false>(p, bf16, true, deep).us;
        return tiles <= (deep ? 1 : 2) * cu_count() ? std::max(input_us, weight_us) : input_us + weight_us - 3.0;
    };
    if (tiles_at_most(q, WEIGHT, 64, 64) <= cu_count() && together(true) <= apart) return Joint::DEEP;
    return together(false) <= apart ? Joint::PLAIN : Joint::NONE;
}

// sizes of the three products
LinearParams forward_sizes(const etr_linear_config& c) {
    LinearParams p{};
    p.rows = c.rows; p.E = c.E; p.N = c.N; p.K = c.K; p.lda = p.ldb = c.K; p.act = c.act; p.glu = c.act == ETR_ACT_SWIGLU;
    return p;
}
LinearParams input_sizes(const etr_linear_config& c) {
    LinearParams p{};
    p.rows = c.rows; p.E = c.E; p.N = c.K; p.K = c.N; p.lda = c.N; p.ldb = c.K; p.glu = c.act == ETR_ACT_SWIGLU;
    return p;
}
LinearParams weight_sizes(const etr_linear_config& c) {
    LinearParams p{};
    p.rows = c.rows; p.E = c.E; p.M = c.N; p.N = c.K; p.K = c.rows; p.lda = c.N; p.ldb = c.K; p.glu = c.act == ETR_ACT_SWIGLU;
    return p;
}

int chunks_at_most(const etr_linear_config& c) { return c.rows / kChunk + std::min(c.E, c.rows); }
size_t middle_bytes(const etr_linear_config& c) {
    return c.act == ETR_ACT_NONE ? 0 : align_up(static_cast<size_t>(c.rows) * c.N * elt_bytes(c.dtype));
}

}  // namespace

size_t linear_ws_bytes(const etr_linear_config& c) {
    const int n = c.act == ETR_ACT_SWIGLU ? 2 : 1;
    return n * middle_bytes(c) + align_up(static_cast<size_t>(n) * chunks_at_most(c) * c.N * 4);
}

hipError_t launch_expert_linear(const etr_linear_config& c, const void* x, const int32_t* offsets, const void* w, const void* w_up, const float* bias,
                                const float* bias_up, const void* residual, void* y, void* pre, void* pre_up, hipStream_t st) {
    LinearParams p = forward_sizes(c);
    p.A[0] = x; p.B[0] = w; p.B[1] = w_up; p.C[0] = y;
    p.offsets = offsets; p.bias[0] = bias; p.bias[1] = bias_up; p.residual = residual; p.pre[0] = pre; p.pre[1] = pre_up;
    return p.glu ? launch_product<FORWARD, true>(p, c.dtype == ETR_BF16, st) : launch_product<FORWARD, false>(p, c.dtype == ETR_BF16, st);
}

hipError_t launch_expert_linear_backward(const etr_linear_config& c, const void* x, const int32_t* offsets, const void* w, const void* w_up,
                                         const void* pre, const void* pre_up, const void* dy, void* dx, void* dw, void* dw_up, float* dbias,
                                         float* dbias_up, void* ws, hipStream_t st) {
    const bool glu = c.act == ETR_ACT_SWIGLU, bf16 = c.dtype == ETR_BF16;
    char* at = static_cast<char*>(ws);
    const size_t middle = middle_bytes(c);
    void* da = c.act == ETR_ACT_NONE ? nullptr : at;
    void* db = glu ? at + middle : nullptr;
    const bool direct = dbias && c.rows <= kChunk;
    const MiddleParams m{static_cast<const piece_t*>(pre), static_cast<const piece_t*>(pre_up), static_cast<const piece_t*>(dy), static_cast<piece_t*>(da),
                         static_cast<piece_t*>(db), dbias && !direct ? reinterpret_cast<float*>(at + (glu ? 2 : 1) * middle) : nullptr,
                         {direct ? dbias : nullptr, direct ? dbias_up : nullptr}, offsets, c.rows, c.E, c.N,
                         static_cast<int>(static_cast<size_t>(c.N) * elt_bytes(c.dtype) / 16), c.act, chunks_at_most(c)};
    hipError_t err;
    if (da || dbias) {
        const dim3 grid(direct ? c.E : m.chunks, (m.pieces + 63) / 64);
        if (bf16) hipLaunchKernelGGL(linear_middle_kernel<true>, grid, dim3(256), 0, st, m);
        else hipLaunchKernelGGL(linear_middle_kernel<false>, grid, dim3(256), 0, st, m);
        if ((err = hipGetLastError()) != hipSuccess) return err;
    }
    if (dbias && !direct) {
        hipLaunchKernelGGL(linear_bias_kernel, dim3((c.N + 63) / 64, c.E, glu ? 2 : 1), dim3(1024), 0, st, m, dbias, dbias_up);
        if ((err = hipGetLastError()) != hipSuccess) return err;
    }
    LinearParams p = input_sizes(c), q = weight_sizes(c);
    p.offsets = q.offsets = offsets;
    p.A[0] = q.A[0] = da ? da : dy; p.A[1] = q.A[1] = db;
    p.B[0] = w; p.B[1] = w_up; p.C[0] = dx;
    q.B[0] = x; q.C[0] = dw; q.C[1] = dw_up;
    if (dx && dw) {
        const Joint joint = choose_joint(p, q, bf16);
        if (joint == Joint::DEEP) return bf16 ? launch_small_backward<true, 2, 4>(p, q, st) : launch_small_backward<false, 2, 4>(p, q, st);
        if (joint == Joint::PLAIN) return bf16 ? launch_small_backward<true, 4, 1>(p, q, st) : launch_small_backward<false, 2, 1>(p, q, st);
    }
    if (dx && (err = launch_product<INPUT, false>(p, bf16, st)) != hipSuccess) return err;
    return dw ? launch_product<WEIGHT, false>(q, bf16, st) : hipSuccess;
}

}  // namespace etr

extern "C" int etr_linear_plan(const etr_linear_config* c, int product) {
    using namespace etr;
    const bool bf16 = c->dtype == ETR_BF16;
    auto form = [](Choice t) { return static_cast<int>(t.tiles) + (t.deep ? 8 : 0); };
    const LinearParams p = forward_sizes(*c), i = input_sizes(*c), w = weight_sizes(*c);
    if (product == 0) return form(p.glu ? choose_tiles<FORWARD, true>(p, bf16) : choose_tiles<FORWARD, false>(p, bf16));
    if (product == 1) return form(choose_tiles<INPUT, false>(i, bf16));
    if (product == 2) return form(choose_tiles<WEIGHT, false>(w, bf16));
    return static_cast<int>(choose_joint(i, w, bf16));
}
