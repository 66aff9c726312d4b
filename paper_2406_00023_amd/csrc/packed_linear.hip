// The experts' products of packed operands (e4m3 values, a power of two per block of 128 along the contraction), with bias, activation,
// residual and packing of the results in the epilogue, and the gradient of their weights.
//   forward  y[r][n] = act(sum_k x[r][k] w[e][n][k] + bias[e][n]) + residual[r][n]       (dx is this product too, of weights along columns)
//   weights  dw[e][n][k] = sum_r da[r][n] x[r][k]                                        both operands along columns
// Every operand is rows of whole 128-byte blocks, padded with zeros, so that every product is C[m][n] = sum_k A(m, k) B(n, k) with both
// contractions contiguous, and a k-tile is one block: 128 bytes and one scale for each row of a tile.
// Results in bf16: the scaled MFMA, 32 x 32 x 64 8-bit values, takes the bytes and the scales as they are.  It cuts products off 2^-13 below the
// largest of some 16 neighbours, which is less than sums in fp32 keep (measured: 1.5e-5 of a result's size on normal data; 1.6e-4, all to one side, where one
// value of every block is 100 times the others).  A rounding to bf16 (2^-8) covers it.  Packed results are not rounded to bf16: of theirs 1 in 600 to 1200
// lies so near a tie that it goes to the other side, 1e-3 off in norm from what is nearest (sums in fp32: 1e-4), and as far from the unrounded
// results as those (2.65e-2).  Chosen for the rate: 32768 x 4096 x 1408 SwiGLU with everything kept packed 455 us, with sums in fp32 691.
// Results in fp32 go without it: the values are converted to bf16, which holds them and their scale exactly, and multiplied there, with
// sums in fp32 (6e-8); so do packed results by themselves where the type says fp32.
//
// Bound by the matrix pipe where an expert has a few hundred rows (there: by the power that it draws), by the weights' bytes where it has a
// few, by latency in between.  Measured, bf16: 8192 cubed 440 us (2.5 PFLOP/s; a library product 2.6); 16 experts, SwiGLU of 2048 x 5632, 16 384 uneven rows 395 us
// (1.9), 64 rows 65 us (5.7 TB/s of weights); 11264 x 2048 of the same rows 425 us, of even ones 340; weights' gradient of 11264 x 2048 over them 510.
#include <algorithm>
#include <cmath>

#include "activation.h"
#include "packed.h"

namespace etr {
namespace {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) void* lds_ptr;

struct PackedParams {
    const uint8_t* A; const uint8_t* As;                 // x, or da (and db) along columns
    const uint8_t* B[2]; const uint8_t* Bs[2];           // the weights (second: up), or x along columns
    void* C[2];                                          // y (optional), or dw and dw_up
    uint8_t* P[3]; uint8_t* Ps[3];                       // packed results, optional: y, a, the up product
    const int32_t* offsets;
    const float* bias[2];
    const void* residual;
    int rows, E;
    int M, N;                                            // WEIGHT: output rows of each half; output columns
    int blocks;                                          // FORWARD: k-tiles
    int act, glu;
    int NT;                                              // column tiles
};

enum Product { FORWARD = 0, WEIGHT = 1 };                // y (or dx), dw

// count: rows of the group; limit: the tile stores rows below it; half: WEIGHT with SwiGLU, which of the two outputs
struct Tile { int e, first, m0, n0, count, limit, half; };

// The tile list: experts one after the other; inside one bands of 8 row tiles, in a band the row tiles of a column tile next to
// each other.  Each XCD (workgroups go round them) has a contiguous part of the list, so its 32 CUs work on some 8 x 4 tiles at once and share
// 8 + 4 operand slabs in its L2.
// SPLIT (one workgroup to a CU): the parts are equal in work, where a tile of WEIGHT takes as long as its expert has rows (16 experts of
// 600 to 1700 rows, 2048 x 11264: 547 us with equal numbers of tiles, 498 so); and where the last round over an XCD's CUs would keep
// half of them or fewer busy, its tiles go in halves or quarters of their rows to as many workgroups.
template <int MODE, bool SPLIT>
struct TileList {
    int tiles, tiles_incl;                               // of a lane's expert; WEIGHT: of every expert the same, and not used
    int start, end, per_xcd;                             // this XCD's part of the list; workgroups that share it
    __device__ __forceinline__ void load(const PackedParams& p, const Segments& seg, int BM, int bid, int grid) {
        const int xcd = bid & 7;
        per_xcd = grid >> 3;
        tiles = tiles_incl = 0;
        if (MODE == WEIGHT && SPLIT) {
            const int each = (p.M + BM - 1) / BM * (p.glu ? 2 : 1) * p.NT, lane = threadIdx.x & 63;
            const long long weight = lane < p.E ? seg.blocks + 4 : 0, incl = wave_scan_incl(weight * each);
            auto at = [](long long v, int e) {
                return static_cast<long long>(static_cast<uint64_t>(static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(v), e))) |
                                              static_cast<uint64_t>(static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(v >> 32), e))) << 32);
            };
            const long long all = at(incl, 63);
            auto border = [&](int x) {                   // first tile of XCD x
                if (x == 8) return p.E * each;
                const long long target = all / 8 * x;
                const int e = __builtin_ctzll(__ballot(incl > target));
                const long long w = at(weight, e), in = target - (at(incl, e) - w * each);
                return e * each + min(static_cast<int>(static_cast<double>(in + w - 1) / static_cast<double>(w)), each);
            };
            start = border(xcd);
            end = border(xcd + 1);
        } else {
            int all = p.E * ((p.M + BM - 1) / BM) * (p.glu ? 2 : 1) * p.NT;
            if (MODE != WEIGHT) {
                tiles = (seg.count + BM - 1) / BM;
                tiles_incl = wave_scan_incl(tiles);
                all = __builtin_amdgcn_readlane(tiles_incl, 63) * p.NT;
            }
            const int share = (all + 7) >> 3;
            start = xcd * share;
            end = min(start + share, all);
        }
    }
    __device__ __forceinline__ bool find(const PackedParams& p, const Segments& seg, int BM, int BN, int j, Tile& t) const {
        const int share = end - start;
        int part = 0, parts_log = 0;
        if constexpr (SPLIT) {
            const int full = share / per_xcd * per_xcd, rest = share - full;
            if (j >= full) {
                parts_log = rest * 4 <= per_xcd ? 2 : rest * 2 <= per_xcd ? 1 : 0;
                part = (j - full) & ((1 << parts_log) - 1);
                j = full + ((j - full) >> parts_log);
            }
        }
        if (j >= share) return false;
        const int q = start + j;
        int in, rows, MTw = 0;
        if (MODE == WEIGHT) {
            MTw = (p.M + BM - 1) / BM;
            rows = MTw * (p.glu ? 2 : 1);
            t.e = q / (rows * p.NT);
            in = q - t.e * (rows * p.NT);
        } else {
            t.e = __builtin_ctzll(__ballot(tiles_incl * p.NT > q));
            rows = __builtin_amdgcn_readlane(tiles, t.e);
            in = q - (__builtin_amdgcn_readlane(tiles_incl, t.e) - rows) * p.NT;
        }
        const int band = in / (8 * p.NT), in_band = in - band * 8 * p.NT, height = min(8, rows - band * 8);
        const int nt = in_band / height, mt = band * 8 + in_band - nt * height;
        t.first = __builtin_amdgcn_readlane(seg.first, t.e);
        t.count = __builtin_amdgcn_readlane(seg.count, t.e);
        t.half = MODE == WEIGHT && mt >= MTw ? 1 : 0;
        t.m0 = (mt - t.half * MTw) * BM;
        t.n0 = nt * BN;
        t.limit = MODE == WEIGHT ? p.M : t.count;
        if (SPLIT && parts_log) {                        // (a part past the last row stores nothing: it stays at the tile's start)
            const int of_part = BM >> parts_log, m0 = t.m0 + part * of_part;
            t.limit = m0 < t.limit ? min(t.limit, m0 + of_part) : t.m0;
            t.m0 = t.limit > t.m0 ? m0 : t.m0;
        }
        return true;
    }
};

// What the copies of one operand need: 64-bit base of a tile's first row in this k-tile, and the buffer bound.
constexpr uint32_t kRange = 0xFFFFFF00u, kPast = 0xFFFFFF80u;         // an offset past any buffer: such a lane copies zeros

__device__ __forceinline__ v4i descriptor(uint64_t base) {
    const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(base));
    const uint32_t hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(base >> 32));
    return v4i{static_cast<int>(lo), static_cast<int>(hi & 0xFFFFu), static_cast<int>(kRange), 0x00027000};
}
// Copies into LDS, 16 or 4 bytes a lane, lane after lane from `at`; N of them, 1 KiB apart there.  In assembly, without an output: the compiler would
// otherwise take every later read of LDS to wait for them; they are waited for by hand.  What the compiler does not see in it either: five wait
// states between a vector instruction's write of a scalar register (a spilled one comes back that way) and a memory operation that
// reads it, and one behind M0's.
template <int N> __device__ __forceinline__ void copy16(v4i from, const uint32_t* off, uint32_t at) {
    if constexpr (N >= 4) {
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %5, 0 offen lds\n\t"
                     "s_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %5, 0 offen lds\n\t"
                     "s_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tbuffer_load_dwordx4 %3, %5, 0 offen lds\n\t"
                     "s_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tbuffer_load_dwordx4 %4, %5, 0 offen lds"
                     ::"s"(at), "v"(off[0]), "v"(off[1]), "v"(off[2]), "v"(off[3]), "s"(from) : "memory", "m0", "scc");
        copy16<N - 4>(from, off + 4, at + 4096);
    } else if constexpr (N > 0) {
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(at), "v"(off[0]), "s"(from) : "memory", "m0");
        copy16<N - 1>(from, off + 1, at + 1024);
    }
}
__device__ __forceinline__ void copy4(v4i from, uint32_t off, uint32_t at) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(at), "v"(off), "s"(from) : "memory", "m0");
}
// at most N of this wave's vector memory operations are outstanding
template <int N> __device__ __forceinline__ void wait_copies() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | 0x0F70);
    asm volatile("" ::: "memory");
}
// this wave's reads of LDS are done
__device__ __forceinline__ void wait_reads() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xC07F);
    asm volatile("" ::: "memory");
}
__device__ __forceinline__ void barrier() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// LDS of a wave's own, through which its results leave.  (Four waves of a SwiGLU have half as much, so that two workgroups of them fit a CU.)
constexpr int patch_bytes(bool glu, int waves) { return glu && waves == 4 ? 1024 : 2048; }

// eight values of a block as bf16, exactly
__device__ __forceinline__ bf16x8 widen(int lo, int hi, float scale) {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// ---- epilogue --------------------------------------------------------------------------------------------------------

template <bool WIDE>
__device__ __forceinline__ float activate(int act, float a, float up, bool glu) {
    if (glu) return a * sigmoid<!WIDE>(a) * up;
    if (act == ETR_ACT_SILU) return a * sigmoid<!WIDE>(a);
    if (act == ETR_ACT_GELU) return a * normal_cdf<!WIDE>(a);
    return a;
}
template <bool WIDE>
__device__ __forceinline__ void store4(void* p, size_t at, const float (&f)[4]) {
    if constexpr (WIDE) {
        *reinterpret_cast<float4*>(static_cast<float*>(p) + at) = make_float4(f[0], f[1], f[2], f[3]);
    } else {
        typedef __attribute__((ext_vector_type(2))) float f32x2;
        const uint32_t lo = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{f[0], f[1]}, bf16x2));
        const uint32_t hi = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{f[2], f[3]}, bf16x2));
        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p) + at) = make_uint2(lo, hi);
    }
}
template <bool WIDE>
__device__ __forceinline__ void load4(const void* p, size_t at, float (&f)[4]) {
    if constexpr (WIDE) {
        const float4 v = *reinterpret_cast<const float4*>(static_cast<const float*>(p) + at);
        f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w;
    } else {
        const uint2 v = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(p) + at);
        f[0] = __uint_as_float(v.x << 16); f[1] = __uint_as_float(v.x & 0xFFFF0000u);
        f[2] = __uint_as_float(v.y << 16); f[3] = __uint_as_float(v.y & 0xFFFF0000u);
    }
}

// ---- tiles of 32 x 32 blocks -------------------------------------------------------------------------------------------
//
// LDS, an operand of a k-tile: [row][8 pieces of 16 bytes]; the piece at place s of a row is s ^ (row / 2 % 8), so that the rows of a fragment
// spread over the banks.  Behind both operands their scales, a dword (four k-tiles) for each row.  A fragment's lane has row lane % 32 of its
// block and 32 of the 64 bytes of half a k-tile; which ones does not matter as long as it is the same for both operands.
// A workgroup of WM x WN waves has a BM x BN tile at a time, and two buffers: while one is multiplied the next k-tile is copied into the other.
// The MFMAs take the columns' fragment first, so that a lane ends up with runs of four neighbouring columns of one row.
// WIDE: results in fp32.
template <bool WIDE, int BM, int BN, int WM, int WN, int MODE, bool GLU, bool WALK>
__global__ __launch_bounds__(WM* WN * 64, 2) void packed_tiles_kernel(PackedParams p) {
    constexpr int NW = WM * WN, MB = BM / WM / 32, NB = BN / WN / 32, NO = GLU ? NB / 2 : NB;
    constexpr int OUT_N = GLU ? BN / 2 : BN;
    constexpr int CA = BM / 8, CB = BN / 8;              // copies of 64 pieces per operand and k-tile
    constexpr int SA = (BM + 63) / 64, SB = BN / 64;     // copies of 64 scales
    constexpr int SW = (SA + SB + NW - 1) / NW;
    constexpr int A_BYTES = BM * kBlock, TILE_BYTES = (BM + BN) * kBlock, STAGE = TILE_BYTES + (SA + SB) * 256;
    constexpr int kColumnWaves = kBlock / (NO * 32);     // waves that share a block of 128 output columns
    static_assert(CA % NW == 0 && CB % NW == 0 && BN % 64 == 0 && OUT_N % kBlock == 0 && kBlock % (NO * 32) == 0 && (!GLU || NB % 2 == 0), "");
    constexpr int TOPS = WN * BM * 4;                    // bytes of tops
    // of what is stored: bytes of a value; blocks side by side in a patch; its row's bytes and pieces; rows to a store
    constexpr bool PATCH = !WIDE;
    constexpr int ES = WIDE ? 4 : 2, JC = PATCH || NW * 32 * NO * 32 * ES > TILE_BYTES ? 1 : NO, RB = JC * 32 * ES, PR = RB / 16, RP = 64 / PR;
    constexpr int STORES = MB * NO / JC * (32 / RP);
    constexpr int kPatch = patch_bytes(GLU, NW), PROWS = PATCH ? std::min(32, kPatch / RB) : 32;         // rows of a patch
    static_assert(NO % JC == 0 && NW * 32 * RB <= TILE_BYTES && PROWS % RP == 0, "");
    auto spread = [](int row) { return PR == 4 ? (row >> 2) & 3 : row & (PR - 1); };         // rows of a patch over the banks
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    float (*tops)[BM] = reinterpret_cast<float (*)[BM]>(lds + 2 * STAGE);                 // [WN][BM]
    const int lane = threadIdx.x & 63, l32 = lane & 31, kh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave / WN, wn = wave % WN;
    const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_ptr)lds));

    Segments seg;
    seg.load(p.offsets, p.rows, p.E, false);
    Tile t;
    const int bid = blockIdx.x, grid = gridDim.x;
    TileList<MODE, WALK> list;
    list.load(p, seg, BM, bid, grid);
    int j = bid >> 3;
    if (!list.find(p, seg, BM, OUT_N, j, t)) return;

    // ---- the copy side: a tile and a k-tile of its own, ahead of the products.  A wave copies CA / NW and CB / NW times 64 pieces, of B rows that
    // belong to one of the two weights, and 64 scales (or twice that).
    constexpr int WA = CA / NW, WB = CB / NW;
    struct Source { uint64_t a, b, scales[SW], stride[SW]; uint32_t at_a[WA], at_b[WB], at_s[SW]; int KT, kt; };
    Source s;
    bool more = true;                                    // s is a tile that is still to be copied
    auto copy_row = [&](int c) { return 8 * c + (lane >> 3); };
    auto copy_piece = [&](int c) { return (lane & 7) ^ ((copy_row(c) >> 1) & 7); };
    auto aim = [&](const Tile& x) {
        uint64_t row_a, row_b, group_a, group_b;         // rows, and dwords of scales, before the tile's
        uint32_t pitch;
        uint64_t rows_a;                                 // of the packed matrix
        if constexpr (MODE == WEIGHT) {
            const int blocks = __builtin_amdgcn_readlane(seg.blocks, x.e), before = __builtin_amdgcn_readlane(seg.blocks_incl, x.e) - blocks;
            const uint64_t groups_before = __builtin_amdgcn_readlane(seg.groups_incl, x.e) - __builtin_amdgcn_readlane(seg.groups, x.e);
            rows_a = static_cast<uint64_t>(p.M) * (p.glu ? 2 : 1);
            s.KT = blocks;
            pitch = static_cast<uint32_t>(blocks) * kBlock;
            row_a = static_cast<uint64_t>(x.half) * p.M + x.m0;
            group_a = groups_before * rows_a + row_a;
            group_b = groups_before * p.N + x.n0;
            s.a = reinterpret_cast<uint64_t>(p.A) + static_cast<uint64_t>(before) * kBlock * rows_a + row_a * pitch;
            s.b = reinterpret_cast<uint64_t>(p.B[0]) + static_cast<uint64_t>(before) * kBlock * p.N + static_cast<uint64_t>(x.n0) * pitch;
        } else {
            const int which = GLU && wave >= NW / 2 ? 1 : 0;
            rows_a = static_cast<uint64_t>(p.rows);
            s.KT = p.blocks;
            pitch = static_cast<uint32_t>(p.blocks) * kBlock;
            row_a = static_cast<uint64_t>(x.first) + x.m0;
            row_b = static_cast<uint64_t>(x.e) * p.N + x.n0;
            group_a = row_a;
            group_b = static_cast<uint64_t>(x.e) * ((p.blocks + 3) / 4) * p.N + x.n0;
            s.a = reinterpret_cast<uint64_t>(p.A) + row_a * pitch;
            s.b = reinterpret_cast<uint64_t>(p.B[which]) + row_b * pitch;
        }
        s.kt = 0;
        // rows that are not stored are not read, nor is a contraction without a block: zeros
        const int rows_in = s.KT ? x.limit - x.m0 : 0, columns_in = s.KT ? p.N - x.n0 : 0;
#pragma unroll
        for (int i = 0; i < WA; ++i) {
            const int c = wave * WA + i, r = copy_row(c);
            s.at_a[i] = r < rows_in ? static_cast<uint32_t>(r) * pitch + copy_piece(c) * 16u : kPast;
        }
#pragma unroll
        for (int i = 0; i < WB; ++i) {
            const int c = wave * WB + i, r = copy_row(c), n = GLU && r >= BN / 2 ? r - BN / 2 : r;
            s.at_b[i] = n < columns_in ? static_cast<uint32_t>(n) * pitch + copy_piece(c) * 16u : kPast;
        }
#pragma unroll
        for (int i = 0; i < SW; ++i) {                   // (waves without one of their own copy the last again)
            const int c = min(wave + i * NW, SA + SB - 1), r = 64 * (c < SA ? c : c - SA) + lane, n = GLU && c >= SA && r >= BN / 2 ? r - BN / 2 : r;
            s.scales[i] = c < SA ? reinterpret_cast<uint64_t>(p.As) + group_a * 4 : reinterpret_cast<uint64_t>(p.Bs[GLU && c >= SA + SB / 2 ? 1 : 0]) + group_b * 4;
            s.stride[i] = (c < SA ? rows_a : static_cast<uint64_t>(p.N)) * 4;
            s.at_s[i] = n < (c < SA ? rows_in : columns_in) ? static_cast<uint32_t>(n) * 4 : kPast;
        }
        s.KT = max(s.KT, 1);
    };
    auto issue = [&](int buf) {
        const uint32_t dst = lds0 + buf * STAGE;
        const v4i a = descriptor(s.a), b = descriptor(s.b);
        copy16<WA>(a, s.at_a, dst + wave * WA * 1024);
        copy16<WB>(b, s.at_b, dst + A_BYTES + wave * WB * 1024);
#pragma unroll
        for (int i = 0; i < SW; ++i) copy4(descriptor(s.scales[i]), s.at_s[i], dst + TILE_BYTES + min(wave + i * NW, SA + SB - 1) * 256);
    };
    int jn = j;
    auto advance = [&]() {                               // (a source past the last tile goes on copying its last k-tile)
        if (!more) return;
        if (s.kt + 1 < s.KT) {
            s.kt += 1;
            s.a += kBlock;
            s.b += kBlock;
            if ((s.kt & 3) == 0) {
#pragma unroll
                for (int i = 0; i < SW; ++i) s.scales[i] += s.stride[i];
            }
            return;
        }
        jn += grid >> 3;
        Tile n;
        if (list.find(p, seg, BM, OUT_N, jn, n)) aim(n);
        else more = false;
    };

    // ---- the product side
    auto b_block = [&](int jb) { return GLU ? (jb >= NO ? BN / 64 : 0) + wn * NO + (jb >= NO ? jb - NO : jb) : wn * NB + jb; };
    auto fragment = [&](const unsigned char* op, int block, int half) -> v8i {
        const int row = block * 32 + l32, x = (row >> 1) & 7;
        const v4i lo = *reinterpret_cast<const v4i*>(op + row * kBlock + ((4 * half + 2 * kh) ^ x) * 16);
        const v4i hi = *reinterpret_cast<const v4i*>(op + row * kBlock + ((4 * half + 2 * kh + 1) ^ x) * 16);
        return v8i{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    };
    // first: the sums begin here
    auto multiply = [&](const v8i (&fa)[MB], const v8i (&fb)[NB], const int (&sa)[MB], const int (&sb)[NB], f32x16 (&c)[MB][NB], auto first) {
        constexpr f32x16 none{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        constexpr bool FIRST = decltype(first)::value;
        if constexpr (!WIDE) {
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int jb = 0; jb < NB; ++jb)
                    c[i][jb] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fb[jb], fa[i], FIRST ? none : c[i][jb], 0, 0, 0, sb[jb], 0, sa[i]);
        } else {                                         // every fragment is converted once
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                bf16x8 wa[MB], wb[NB];
#pragma unroll
                for (int i = 0; i < MB; ++i) wa[i] = widen(fa[i][2 * q], fa[i][2 * q + 1], scale_value(sa[i]));
#pragma unroll
                for (int jb = 0; jb < NB; ++jb) wb[jb] = widen(fb[jb][2 * q], fb[jb][2 * q + 1], scale_value(sb[jb]));
#pragma unroll
                for (int i = 0; i < MB; ++i)
#pragma unroll
                    for (int jb = 0; jb < NB; ++jb)
                        c[i][jb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wb[jb], wa[i], FIRST && q == 0 ? none : c[i][jb], 0, 0, 0);
            }
        }
    };
    f32x16 acc[MB][NB];
    aim(t);
    issue(0);
    advance();
    wait_copies<0>();
    int buf = 0;
    bool ahead = false;                                  // the tile's second k-tile is on its way, and behind it
    bool behind = false;                                 // exactly STORES stores of this wave
    for (;;) {
        const int KT = MODE == WEIGHT ? max(__builtin_amdgcn_readlane(seg.blocks, t.e), 1) : p.blocks;
        // a wave none of whose rows is stored multiplies nothing (tiles at the end of an expert's rows), and the wave beside it on the SIMD has the
        // matrix pipe for itself meanwhile
        const bool live = t.n0 + wn * NO * 32 < p.N && t.limit - t.m0 > wm * MB * 32;
        for (int kt = 0; kt < KT; ++kt) {
            barrier();                                   // everybody's part of the k-tile has landed, and everybody is done with the other buffer
            if (kt > 0 || !ahead) {
                issue(buf ^ 1);
                advance();
            }
            if (live) {
                const unsigned char* op = lds + buf * STAGE;
                const uint32_t* sc = reinterpret_cast<const uint32_t*>(op + TILE_BYTES);
                const int shift = 8 * (kt & 3);
                int sa[MB], sb[NB];
#pragma unroll
                for (int i = 0; i < MB; ++i) sa[i] = static_cast<int>(sc[(wm * MB + i) * 32 + l32] >> shift) & 255;
#pragma unroll
                for (int jb = 0; jb < NB; ++jb) sb[jb] = static_cast<int>(sc[SA * 64 + b_block(jb) * 32 + l32] >> shift) & 255;
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    v8i fa[MB], fb[NB];
#pragma unroll
                    for (int jb = 0; jb < NB; ++jb) fb[jb] = fragment(op + A_BYTES, b_block(jb), half);
#pragma unroll
                    for (int i = 0; i < MB; ++i) fa[i] = fragment(op, wm * MB + i, half);
                    if (half == 0 && kt == 0) multiply(fa, fb, sa, sb, acc, std::true_type{});
                    else multiply(fa, fb, sa, sb, acc, std::false_type{});
                }
            }
            // this wave's part of the next k-tile has landed, of the next tile's first one too; stores behind it may still be on their way
            if (kt == 0 && behind) wait_copies<STORES>();
            else wait_copies<0>();
            wait_reads();
            buf ^= 1;
        }

        // ---- the results: lane: row l of a block, columns 8 q + 4 h ... + 3 of it for q = 0 ... 3
        // They leave through the buffer that was multiplied last, which nobody copies into before the next k-tile's barrier.  What is optional
        // goes over the accumulators in a pass of its own, a row block at a time (the barriers to the scheduler), so that few values live
        // beside them; what depends on `lane_now` is made anew in each pass and takes no registers of the loop over k-tiles.
        const int limit = t.limit - t.m0;
        const int n_wave = t.n0 + wn * NO * 32;          // first output column of the wave
        const size_t first = (MODE == WEIGHT ? static_cast<size_t>(t.e) * p.M : static_cast<size_t>(t.first)) + t.m0;
        unsigned char* room = lds + (buf ^ 1) * STAGE;
        auto lane_now = [&]() { int l = lane; asm volatile("" : "+v"(l)); return l; };
        auto pin = [&]() {
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int jb = 0; jb < NB; ++jb) asm volatile("" : "+v"(acc[i][jb]));
        };
        pin();
        barrier();                                       // everybody has read it
        // without packed results only the waves' own patches are written, and the next tile's second k-tile can be on its way meanwhile
        ahead = PATCH && !(MODE == FORWARD && (p.P[0] || p.P[1] || p.P[2]));
        if (ahead) {
            issue(buf ^ 1);
            advance();
        }
        // packs blocks j0 ... j0 + NO - 1 of the accumulators, as many row blocks of each wave at a time as there is room for.
        // room: [row][OUT_N bytes], the pieces of a row in an order of its own
        auto pack = [&](uint8_t* to, uint8_t* scales, auto j0_) {
            constexpr int PR = OUT_N / 16, j0 = decltype(j0_)::value;    // pieces of a row
            constexpr int CI = MB * WM * 32 * OUT_N <= TILE_BYTES ? MB : MB / 2, ROWS = CI * WM * 32;
            static_assert(MB % CI == 0 && ROWS * OUT_N <= TILE_BYTES && ROWS * PR % (NW * 64) == 0 && NW * 64 % PR == 0, "");
            auto place = [](int row, int piece) { return row * OUT_N + ((piece ^ (OUT_N == 128 ? row >> 1 : row)) & (PR - 1)) * 16; };
            const int Np = blocks_of(p.N) * kBlock, w0 = wn / kColumnWaves * kColumnWaves, block = n_wave / kBlock;
            const bool ragged = n_wave + NO * 32 > p.N;                  // (uniform)
            {
                const int l = lane_now(), h = l >> 5;
#pragma unroll
                for (int i = 0; i < MB; ++i) {
                    float top = 0.f;
#pragma unroll
                    for (int jb = 0; jb < NO; ++jb)
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const float four = top_of<4>([&](int v) { return acc[i][j0 + jb][4 * q + v]; });
                            top = ragged && n_wave + jb * 32 + 8 * q + 4 * h >= p.N ? top : fmaxf(top, four);
                        }
                    top = fmaxf(top, __shfl_xor(top, 32));
                    if (h == 0) tops[wn][(wm * MB + i) * 32 + (l & 31)] = top;
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
#pragma unroll
            for (int i0 = 0; i0 < MB; i0 += CI) {
                __syncthreads();
                const int l = lane_now(), h = l >> 5;
#pragma unroll
                for (int i = i0; i < i0 + CI; ++i) {
                    const int m = (wm * MB + i) * 32 + (l & 31), row = (wm * CI + i - i0) * 32 + (l & 31);
                    float top = tops[w0][m];
#pragma unroll
                    for (int w = 1; w < kColumnWaves; ++w) top = fmaxf(top, tops[w0 + w][m]);
                    const uint32_t byte = scale_byte(top);
                    const float scale = scale_value(byte);
#pragma unroll
                    for (int jb = 0; jb < NO; ++jb)
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const int c = wn * NO * 32 + jb * 32 + 8 * q + 4 * h;
                            const f32x16& a = acc[i][j0 + jb];
                            uint32_t four = to_e4m3(a[4 * q], a[4 * q + 1], a[4 * q + 2], a[4 * q + 3], scale);
                            if (ragged && t.n0 + c >= p.N) four = 0u;
                            *reinterpret_cast<uint32_t*>(room + place(row, c >> 4) + (c & 15)) = four;
                        }
                    if (m < limit && wn == w0 && h == 0 && n_wave < p.N) {
                        uint8_t* at = scales + (static_cast<size_t>(block >> 2) * p.rows + first + m) * 4;
                        at[block & 3] = static_cast<uint8_t>(byte);
                        if (block == blocks_of(p.N) - 1)
                            for (int b = (block & 3) + 1; b < 4; ++b) at[b] = 127;
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                __syncthreads();
                int tid = threadIdx.x;
                asm volatile("" : "+v"(tid));
                const int c = tid % PR;
                uint8_t* base = to + first * Np + t.n0;
#pragma unroll 4
                for (int u = 0; u < ROWS * PR / (NW * 64); ++u) {
                    const int row = u * (NW * 64 / PR) + tid / PR, m = (row / (CI * 32) * MB + i0) * 32 + row % (CI * 32);
                    const piece_t v = *reinterpret_cast<const piece_t*>(room + place(row, c));
                    if (m < limit && t.n0 + c * 16 < Np) *reinterpret_cast<piece_t*>(base + static_cast<size_t>(m) * Np + c * 16) = v;
                }
            }
            __syncthreads();                             // (before the next ones are written)
        };
        if constexpr (MODE == FORWARD) {
            auto map = [&](auto&& f) {
#pragma unroll
                for (int i = 0; i < MB; ++i)
#pragma unroll
                    for (int jb = 0; jb < NO; ++jb)
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
#pragma unroll
                            for (int v = 4 * q; v < 4 * q + 4; ++v) acc[i][jb][v] = f(acc[i][jb][v], GLU ? acc[i][(GLU ? NO : 0) + jb][v] : 1.0f);
                            __builtin_amdgcn_sched_barrier(0);
                        }
                pin();
            };
            auto half = [&](auto h_) {
                constexpr int h = decltype(h_)::value;
                if (p.bias[h]) {
                    const int l = lane_now(), kq = 4 * (l >> 5);
#pragma unroll
                    for (int jb = 0; jb < NO; ++jb)
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const int n = n_wave + jb * 32 + 8 * q + kq;
                            float b[4] = {0.f, 0.f, 0.f, 0.f};
                            if (n < p.N) load4<true>(p.bias[h] + static_cast<size_t>(t.e) * p.N, n, b);
#pragma unroll
                            for (int i = 0; i < MB; ++i)
#pragma unroll
                                for (int v = 0; v < 4; ++v) acc[i][h * NO + jb][4 * q + v] += b[v];
                            __builtin_amdgcn_sched_barrier(0);
                        }
                    pin();
                }
                if (p.P[1 + h]) {
                    pack(p.P[1 + h], p.Ps[1 + h], std::integral_constant<int, h * NO>{});
                    pin();
                }
            };
            half(std::integral_constant<int, 0>{});
            if constexpr (GLU) {
                half(std::integral_constant<int, 1>{});
                map([](float a, float u) { return a * sigmoid<!WIDE>(a) * u; });
            } else {
                if (p.act == ETR_ACT_SILU) map([](float a, float) { return a * sigmoid<!WIDE>(a); });
                pin();                                   // (or one pass is made of the two, with both results of every value alive)
                if (p.act == ETR_ACT_GELU) map([](float a, float) { return a * normal_cdf<!WIDE>(a); });
            }
            if (p.residual) {
                const int l = lane_now(), kq = 4 * (l >> 5);
                const char* base = static_cast<const char*>(p.residual) + first * p.N * (WIDE ? 4 : 2);
#pragma unroll
                for (int i = 0; i < MB; ++i) {
                    // (past the ends the last row or columns again, not stored)
                    const size_t row = static_cast<size_t>(max(min((wm * MB + i) * 32 + (l & 31), limit - 1), 0)) * p.N;
                    float r[NO][4][4];
#pragma unroll
                    for (int jb = 0; jb < NO; ++jb)
#pragma unroll
                        for (int q = 0; q < 4; ++q) load4<WIDE>(base, row + min(n_wave + jb * 32 + 8 * q + kq, p.N - 4), r[jb][q]);
#pragma unroll
                    for (int jb = 0; jb < NO; ++jb)
#pragma unroll
                        for (int q = 0; q < 4; ++q)
#pragma unroll
                            for (int v = 0; v < 4; ++v) acc[i][jb][4 * q + v] += r[jb][q][v];
                    __builtin_amdgcn_sched_barrier(0);
                }
                pin();
            }
            if (p.P[0]) {
                pack(p.P[0], p.Ps[0], std::integral_constant<int, 0>{});
                pin();
            }
        }
        void* C = p.C[MODE == WEIGHT ? t.half : 0];
        if (C) {
            // 32 rows of the wave's columns (JC blocks of them) at a time through its patch, or through its part of the room, so that they leave as
            // whole pieces side by side
            const int l = lane_now(), h = l >> 5;
            unsigned char* patch = PATCH ? lds + 2 * STAGE + TOPS + wave * kPatch : room + wave * 32 * RB;
            const int row_in = l / PR, piece = l % PR;
            char* base = static_cast<char*>(C) + first * p.N * ES;
            const bool full = (wm + 1) * MB * 32 <= limit && n_wave + NO * 32 <= p.N;        // (uniform over the wave)
            behind = PATCH && ahead && full;
#pragma unroll
            for (int i = 0; i < MB; ++i) {
                if ((wm * MB + i) * 32 < limit) {        // (uniform)
#pragma unroll
                    for (int j0 = 0; j0 < NO; j0 += JC) {
                        const int n = n_wave + j0 * 32 + piece * (16 / ES);
#pragma unroll
                        for (int r0 = 0; r0 < 32; r0 += PROWS) {
                            const int row = (l & 31) - r0;
                            if (PROWS == 32 || (row >= 0 && row < PROWS)) {
#pragma unroll
                                for (int jb = 0; jb < JC; ++jb)
#pragma unroll
                                    for (int q = 0; q < 4; ++q) {
                                        const int at = (jb * 32 + 8 * q + 4 * h) * ES;
                                        const f32x16& a = acc[i][j0 + jb];
                                        const float f[4] = {a[4 * q], a[4 * q + 1], a[4 * q + 2], a[4 * q + 3]};
                                        store4<WIDE>(patch + row * RB + ((at >> 4) ^ spread(row)) * 16 + (at & 15), 0, f);
                                    }
                            }
                            wave_sync();
                            piece_t out[PROWS / RP];
#pragma unroll
                            for (int u = 0; u < PROWS / RP; ++u) {
                                const int from = u * RP + row_in;
                                out[u] = *reinterpret_cast<const piece_t*>(patch + from * RB + (piece ^ spread(from)) * 16);
                            }
                            wave_sync();
                            const int m = (wm * MB + i) * 32 + r0 + row_in;
                            char* at = base + (static_cast<size_t>(m) * p.N + n) * ES;
                            if (full) {
#pragma unroll
                                for (int u = 0; u < PROWS / RP; ++u) *reinterpret_cast<piece_t*>(at + static_cast<size_t>(u * RP) * p.N * ES) = out[u];
                            } else {
#pragma unroll
                                for (int u = 0; u < PROWS / RP; ++u)
                                    if (m + u * RP < limit && n < p.N) *reinterpret_cast<piece_t*>(at + static_cast<size_t>(u * RP) * p.N * ES) = out[u];
                            }
                        }
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        } else {
            behind = false;
        }
        j += grid >> 3;
        if (!list.find(p, seg, BM, OUT_N, j, t)) break;
        wait_reads();
    }
    wait_copies<0>();                                    // the copies that nobody needed
}

// ---- few rows ----------------------------------------------------------------------------------------------------------
//
// 16 rows x 16 NW output columns to a workgroup: waves with 16 columns each (SwiGLU: 16 gate and 16 up), KS of them to share a
// contraction, stream their weight rows straight into registers, a 16 x 16 x 128 MFMA to a k-tile.  A lane has row
// lane % 16 of a block and 16 bytes out of each half of the k-tile, so that a load takes 64 bytes of a row.
// Bound by the weights' bytes where a CU has waves enough (64 rows in 16 groups, 2048 x 5632 SwiGLU 65 us, 5.7 TB/s).  Else by latency: the branch at the
// contraction's end lets the compiler move each k-tile's loads down to their MFMA, so that a wave has one k-tile on its way, not the four that are
// written beside each other (32 rows in 8 groups, 4096 x 1408 SwiGLU, packed results: 39 us; tiles of 32 rows, which take it, 30).
// PACK: results are packed too, which takes a workgroup with all 128 columns of a block.
template <bool WIDE, int NW, int KS, bool GLU, bool PACK>
__global__ __launch_bounds__(64 * NW * KS, NW * KS > 8 ? 4 : 2) void packed_rows_kernel(PackedParams p) {
    constexpr int BM = 16, NG = GLU ? 2 : 1;
    static_assert(!PACK || NW == 8, "");
    __shared__ float tops[NW][BM];
    __shared__ f32x4 sums[KS > 1 ? KS - 1 : 1][NG][KS > 1 ? NW * 64 : 1];
    const int lane = threadIdx.x & 63, l16 = lane & 15, kq = lane >> 4;
    const int wave_all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = wave_all % NW, group = wave_all / NW;
    Segments seg;
    seg.load(p.offsets, p.rows, p.E, false);
    TileList<FORWARD, false> list;
    list.load(p, seg, BM, blockIdx.x, gridDim.x);
    Tile t;
    for (int j = blockIdx.x >> 3; list.find(p, seg, BM, 16 * NW, j, t); j += gridDim.x >> 3) {
        const size_t pitch = static_cast<size_t>(p.blocks) * kBlock, first = static_cast<size_t>(t.first) + t.m0;
        const int rows_left = t.count - t.m0, n0 = t.n0 + wave * 16, G = (p.blocks + 3) / 4;
        const size_t row_a = first + min(l16, rows_left - 1), row_b = min(n0 + l16, p.N - 1);
        const uint8_t* a = p.A + row_a * pitch + kq * 16;
        const uint32_t* as = reinterpret_cast<const uint32_t*>(p.As) + row_a;
        const uint8_t* b[NG];
        const uint32_t* bs[NG];
#pragma unroll
        for (int h = 0; h < NG; ++h) {
            b[h] = p.B[h] + (static_cast<size_t>(t.e) * p.N + row_b) * pitch + kq * 16;
            bs[h] = reinterpret_cast<const uint32_t*>(p.Bs[h]) + static_cast<size_t>(t.e) * G * p.N + row_b;
        }
        f32x4 acc[NG];
#pragma unroll
        for (int h = 0; h < NG; ++h) acc[h] = f32x4{0.f, 0.f, 0.f, 0.f};
        // four k-tiles, whose scales are a dword, in turn; a group of waves takes every KS-th four
        for (int g = group; g < G; g += KS) {
            const uint32_t sa = as[static_cast<size_t>(g) * p.rows];
            uint32_t sb[NG];
#pragma unroll
            for (int h = 0; h < NG; ++h) sb[h] = bs[h][static_cast<size_t>(g) * p.N];
            v4i fa[4][2], fb[NG][4][2];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                // (past the last k-tile the last again, with nothing added for it)
                const size_t at = static_cast<size_t>(min(4 * g + u, p.blocks - 1)) * kBlock;
#pragma unroll
                for (int s = 0; s < 2; ++s) {
#pragma unroll
                    for (int h = 0; h < NG; ++h) fb[h][u][s] = *reinterpret_cast<const v4i*>(b[h] + at + s * 64);
                    fa[u][s] = *reinterpret_cast<const v4i*>(a + at + s * 64);
                }
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                if (4 * g + u >= p.blocks) break;        // (uniform; this k-tile's loads end up behind it)
                const uint32_t xa = (sa >> (8 * u)) & 255u;
                if constexpr (!WIDE) {
                    const v8i x{fa[u][0][0], fa[u][0][1], fa[u][0][2], fa[u][0][3], fa[u][1][0], fa[u][1][1], fa[u][1][2], fa[u][1][3]};
#pragma unroll
                    for (int h = 0; h < NG; ++h) {
                        const v4i lo = fb[h][u][0], hi = fb[h][u][1];
                        const v8i w{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
                        acc[h] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, acc[h], 0, 0, 0, static_cast<int>((sb[h] >> (8 * u)) & 255u), 0, static_cast<int>(xa));
                    }
                } else {
#pragma unroll
                    for (int s = 0; s < 2; ++s)
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
                            const bf16x8 x = widen(fa[u][s][2 * q], fa[u][s][2 * q + 1], scale_value(xa));
#pragma unroll
                            for (int h = 0; h < NG; ++h)
                                acc[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(fb[h][u][s][2 * q], fb[h][u][s][2 * q + 1], scale_value((sb[h] >> (8 * u)) & 255u)), x,
                                                                                acc[h], 0, 0, 0);
                        }
                }
            }
        }
        if constexpr (KS > 1) {
            if (group > 0) {
#pragma unroll
                for (int h = 0; h < NG; ++h) sums[group - 1][h][threadIdx.x % (NW * 64)] = acc[h];
            }
            __syncthreads();
            if (group == 0) {
#pragma unroll
                for (int s = 0; s < KS - 1; ++s)
#pragma unroll
                    for (int h = 0; h < NG; ++h) acc[h] += sums[s][h][threadIdx.x];
            }
            __syncthreads();
        }
        // lane: row l16, columns 4 kq ... + 3 of the wave's 16
        const int n = n0 + 4 * kq, Np = blocks_of(p.N) * kBlock;
        const bool mine = group == 0, row_in = mine && l16 < rows_left;
        auto pack = [&](uint8_t* to, uint8_t* scales, const f32x4& v) {
            float top = 0.f;
            if (n < p.N) top = fmaxf(fmaxf(finite_abs(v[0]), finite_abs(v[1])), fmaxf(finite_abs(v[2]), finite_abs(v[3])));
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            if (mine && kq == 0) tops[wave][l16] = top;
            __syncthreads();
            top = tops[0][l16];
#pragma unroll
            for (int w = 1; w < NW; ++w) top = fmaxf(top, tops[w][l16]);
            const uint32_t byte = scale_byte(top);
            const float scale = scale_value(byte);
            if (row_in && n < Np)
                *reinterpret_cast<uint32_t*>(to + (first + l16) * Np + n) = n < p.N ? to_e4m3(v[0], v[1], v[2], v[3], scale) : 0u;
            if (row_in && wave == 0 && kq == 0) {
                const int block = t.n0 / kBlock;
                uint8_t* at = scales + (static_cast<size_t>(block >> 2) * p.rows + first + l16) * 4;
                at[block & 3] = static_cast<uint8_t>(byte);
                if (block == blocks_of(p.N) - 1)
                    for (int x = (block & 3) + 1; x < 4; ++x) at[x] = 127;
            }
            __syncthreads();
        };
#pragma unroll
        for (int h = 0; h < NG; ++h) {
            if (p.bias[h] && n < p.N) {
                float f[4];
                load4<true>(p.bias[h] + static_cast<size_t>(t.e) * p.N, n, f);
#pragma unroll
                for (int v = 0; v < 4; ++v) acc[h][v] += f[v];
            }
            if (PACK && p.P[1 + h]) pack(p.P[1 + h], p.Ps[1 + h], acc[h]);
        }
        float r[4] = {0.f, 0.f, 0.f, 0.f};
        if (p.residual && row_in && n < p.N) load4<WIDE>(p.residual, (first + l16) * p.N + n, r);
#pragma unroll
        for (int v = 0; v < 4; ++v) acc[0][v] = activate<WIDE>(p.act, acc[0][v], acc[NG - 1][v], GLU) + r[v];
        if (PACK && p.P[0]) pack(p.P[0], p.Ps[0], acc[0]);
        if (p.C[0] && row_in && n < p.N) {
            const float f[4] = {acc[0][0], acc[0][1], acc[0][2], acc[0][3]};
            store4<WIDE>(p.C[0], (first + l16) * p.N + n, f);
        }
    }
}

// ---- host ------------------------------------------------------------------------------------------------------------

long long tiles_at_most(const PackedParams& p, int mode, int BM, int out_n) {
    const long long columns = (p.N + out_n - 1) / out_n;
    if (mode == WEIGHT) return columns * ((p.M + BM - 1) / BM) * p.E * (p.glu ? 2 : 1);
    // full tiles of all rows together, and one more in part for each group
    return columns * (p.rows / BM + std::min(p.E, p.rows));
}

template <bool WIDE, int BM, int BN, int WM, int WN, int MODE, bool GLU, bool WALK>
hipError_t launch_tiles(PackedParams p, hipStream_t st) {
    constexpr int out_n = GLU ? BN / 2 : BN;
    constexpr size_t lds = 2 * static_cast<size_t>((BM + BN) * kBlock + ((BM + 63) / 64 + BN / 64) * 256) + WN * BM * 4 + (WIDE ? 0 : WM * WN * patch_bytes(GLU, WM * WN));
    auto kern = packed_tiles_kernel<WIDE, BM, BN, WM, WN, MODE, GLU, WALK>;
    const hipError_t err = ensure_dynamic_lds(reinterpret_cast<const void*>(kern), lds);
    if (err != hipSuccess) return err;
    p.NT = (p.N + out_n - 1) / out_n;
    const long long tiles = tiles_at_most(p, MODE, BM, out_n);
    // one workgroup on each CU that walks the tiles (up to four parts of one), or one for each of them
    const long long blocks = std::min<long long>((tiles + 7) / 8 * (WALK ? 4 : 1), WALK ? cu_count() / 8 : 1 << 17) * 8;
    hipLaunchKernelGGL(kern, dim3(static_cast<unsigned>(blocks)), dim3(WM * WN * 64), lds, st, p);
    return hipGetLastError();
}
template <bool WIDE, int NW, int KS, bool GLU, bool PACK>
hipError_t launch_rows(PackedParams p, hipStream_t st) {
    p.NT = (p.N + 16 * NW - 1) / (16 * NW);
    const long long tiles = tiles_at_most(p, FORWARD, 16, 16 * NW);
    const long long blocks = std::min<long long>((tiles + 7) / 8, 1 << 17) * 8;
    hipLaunchKernelGGL((packed_rows_kernel<WIDE, NW, KS, GLU, PACK>), dim3(static_cast<unsigned>(blocks)), dim3(64 * NW * KS), 0, st, p);
    return hipGetLastError();
}

// The form of a product, by estimate.  ROWS16: 16 rows x 16 columns, eight waves to share the contraction; ROWS32: x 32, four of them; ROWS128: x 128,
// a wave for 16 columns each, where results are packed; T32 ... T256: tiles of that many rows, x 128 columns, T256 x 256 (weight rows of a SwiGLU: twice
// as many for T32 and T64, and no T128).
enum class Form { ROWS16, ROWS32, ROWS128, T32, T64, T128, T256 };
struct Choice { Form form; double us; };
// Microseconds: rounds of tiles over the places that they have on the chip, each a time per k-tile (alone ... chip full) and a time besides; and the
// weights' bytes at 5 TB/s at least.  ROWS: the weights' bytes for every 16 rows, at 5.5 TB/s.  (bf16; fp32 takes longer with all of them.)
// What it leaves out: the rows' bytes and a workgroup's own time in ROWS, so that many rows of few columns go there (2^20 rows, K = 128: N = 32
// 181 us, N = 64, in tiles, 77); how uneven the groups are, since it goes by the average; and a contraction is never shared between
// workgroups, so that the weights' gradient of few tiles takes as long as its rows (32768 rows, 128 x 128 131 us, 1024 x 1024 136).  Measured, us, in this order:
// ROWS16 / 32, T32, T64, T128, T256 (SwiGLU without T128):
//   18 rows dense, 3840 x 1472          6.3  9.5                       2048 in 16 groups, 5632 x 2048         59   57   42   48
//   96 in 4, 2816 x 1024               10.3 12.6  12.0 14.6 18.2 24.8  4096 in 16, 2048 x 2048                44   37   34   30
//   64 in 16, 5632 x 2048              32.5 32.3  29.0 29.6 32.6 44.7  300 dense, 4096 x 4096                 20.1 19.7 25.1 33.9
//   64 in 16, 2048 x 5632 SwiGLU       92   65    74   77        82    1024 dense, 4096 x 4096                42   25   27   35
//   32 in 8, 4096 x 1408 SwiGLU        18.5 21                         512 in 8, 2048 x 1408 SwiGLU           16.8 18.1      21.2
//   1 in 64, 2048 x 1408 SwiGLU         5.9  7.3  14.5 17.3      20.9  32768 in 8, 2816 x 4096                775  574  428  369
double estimate_us(Form f, double tiles, double k_tiles, bool glu) {
    double places = 1, alone = 0, full = 0, besides = 0;
    switch (f) {
        case Form::T256: alone = 0.87; full = 1.75; besides = 6.0; break;
        case Form::T128: places = 2; alone = 0.6; full = 1.1; besides = 4.5; break;
        case Form::T64: places = glu ? 1 : 3; alone = glu ? 0.85 : 0.45; full = glu ? 1.2 : 1.15; besides = glu ? 4.0 : 3.5; break;
        case Form::T32: places = glu ? 2 : 3; alone = glu ? 0.7 : 0.33; full = glu ? 1.2 : 0.78; besides = glu ? 4.0 : 3.0; break;
        default: break;
    }
    const double r = tiles / (places * cu_count()), rest = r - std::floor(r);
    double rounds = r <= 1 ? 1.0 : f == Form::T256 ? std::ceil(r) : r < 4 ? std::ceil(2 * r) / 2 : r + 0.25;
    if (f == Form::T256 && r > 1 && rest > 0) rounds = std::floor(r) + (rest <= 0.25 ? 0.55 : rest <= 0.5 ? 0.7 : 1.0);
    double crowd = std::min(1.0, r);                     // half of it the chip's, half from where tiles share a CU
    if (places > 1) crowd = 0.5 * crowd + 0.5 * std::max(0.0, std::min(1.0, (r * places - 1) / (places - 1)));
    return rounds * (k_tiles * (alone + (full - alone) * crowd) + besides);
}
template <int MODE, bool GLU>
Choice choose_form(const PackedParams& p, bool packs) {
    const double rows_each = MODE == WEIGHT ? p.M : static_cast<double>(p.rows) / p.E;               // rows of a group, on average
    const double groups = MODE == WEIGHT ? p.E * (p.glu ? 2 : 1) : std::min(p.E, p.rows);
    const double k_tiles = MODE == WEIGHT ? std::ceil(static_cast<double>(p.rows) / p.E / kBlock) : p.blocks;
    const double weights = MODE == WEIGHT ? 0 : groups * p.N * p.blocks * kBlock * (GLU ? 2 : 1);    // bytes
    // row tiles of a group: half a tile more than its rows fill, on average, where they are the batch's
    auto row_tiles = [&](int BM) {
        const double whole = std::ceil(rows_each / BM);
        return MODE == WEIGHT || rows_each < 1 ? whole : std::max(whole, rows_each / BM + (p.E > 1 ? 0.5 : 0.0));
    };
    Choice best{Form::T256, 1e30};
    auto offer = [&](Form f, double us) { if (us < best.us) best = {f, us}; };
    auto offer_tiles = [&](Form f, int BM, int out_n) {
        const double us = estimate_us(f, groups * row_tiles(BM) * ((p.N + out_n - 1) / out_n), k_tiles, GLU);
        offer(f, std::max(us, 3.0 + weights / 5.0e6));
    };
    offer_tiles(Form::T256, 256, GLU ? 128 : 256);
    if (!GLU) offer_tiles(Form::T128, 128, 128);
    offer_tiles(Form::T64, 64, 128);
    offer_tiles(Form::T32, 32, 128);
    if (MODE != WEIGHT) {
        const double bytes = weights * row_tiles(16), us = 3.5 + bytes / 5.5e6;
        // (a CU takes in 27 KB a microsecond in that loop, one k-tile of each wave on its way)
        if (packs) offer(Form::ROWS128, std::max(us, 3.5 + std::ceil(groups * row_tiles(16) * blocks_of(p.N) / cu_count()) * kBlock * p.blocks * kBlock * (GLU ? 2 : 1) / 27e3));
        else offer(groups * row_tiles(16) * p.N / 16 < 2048 ? Form::ROWS16 : Form::ROWS32, us);
    }
    return best;
}

template <bool WIDE, bool GLU>
hipError_t launch_forward(const PackedParams& p, hipStream_t st) {
    const bool packs = p.P[0] || p.P[1] || p.P[2];
    switch (choose_form<FORWARD, GLU>(p, packs).form) {
        case Form::ROWS16: return launch_rows<WIDE, 1, 8, GLU, false>(p, st);
        case Form::ROWS32: return launch_rows<WIDE, 2, 4, GLU, false>(p, st);
        case Form::ROWS128: return launch_rows<WIDE, 8, 1, GLU, true>(p, st);
        case Form::T32: return launch_tiles<WIDE, 32, GLU ? 256 : 128, 1, 4, FORWARD, GLU, false>(p, st);
        case Form::T64: return launch_tiles<WIDE, 64, GLU ? 256 : 128, 1, 4, FORWARD, GLU, false>(p, st);
        case Form::T128:
            if constexpr (!GLU) return launch_tiles<WIDE, 128, 128, 2, 2, FORWARD, false, false>(p, st);
            break;
        case Form::T256: return launch_tiles<WIDE, 256, 256, 2, 4, FORWARD, GLU, true>(p, st);
    }
    return hipErrorInvalidValue;
}
template <bool WIDE>
hipError_t launch_weight(const PackedParams& p, hipStream_t st) {
    switch (choose_form<WEIGHT, false>(p, false).form) {
        case Form::T32: return launch_tiles<WIDE, 32, 128, 1, 4, WEIGHT, false, false>(p, st);
        case Form::T64: return launch_tiles<WIDE, 64, 128, 1, 4, WEIGHT, false, false>(p, st);
        case Form::T128: return launch_tiles<WIDE, 128, 128, 2, 2, WEIGHT, false, false>(p, st);
        case Form::T256: return launch_tiles<WIDE, 256, 256, 2, 4, WEIGHT, false, true>(p, st);
        default: return hipErrorInvalidValue;
    }
}

// sizes of the products
PackedParams forward_sizes(const etr_linear_config& c) {
    PackedParams p{};
    p.rows = c.rows; p.E = c.E; p.N = c.N; p.blocks = blocks_of(c.K); p.act = c.act; p.glu = c.act == ETR_ACT_SWIGLU;
    return p;
}
PackedParams weight_sizes(const etr_linear_config& c) {
    PackedParams p{};
    p.rows = c.rows; p.E = c.E; p.M = c.N; p.N = c.K; p.glu = c.act == ETR_ACT_SWIGLU;
    return p;
}

}  // namespace

hipError_t launch_packed_linear(const etr_linear_config& c, const etr_packed& x, const int32_t* offsets, const etr_packed* const w[2], const float* bias,
                                 const float* bias_up, const void* residual, void* y, const etr_packed* const kept[3], hipStream_t st) {
    PackedParams p = forward_sizes(c);
    p.A = static_cast<const uint8_t*>(x.values); p.As = static_cast<const uint8_t*>(x.scales);
    for (int i = 0; i < 2; ++i)
        if (w[i]) { p.B[i] = static_cast<const uint8_t*>(w[i]->values); p.Bs[i] = static_cast<const uint8_t*>(w[i]->scales); }
    for (int i = 0; i < 3; ++i)
        if (kept[i]) { p.P[i] = static_cast<uint8_t*>(kept[i]->values); p.Ps[i] = static_cast<uint8_t*>(kept[i]->scales); }
    p.C[0] = y; p.offsets = offsets; p.bias[0] = bias; p.bias[1] = bias_up; p.residual = residual;
    if (c.dtype == ETR_BF16) return p.glu ? launch_forward<false, true>(p, st) : launch_forward<false, false>(p, st);
    return p.glu ? launch_forward<true, true>(p, st) : launch_forward<true, false>(p, st);
}

hipError_t launch_packed_weight_gradient(const etr_linear_config& c, const etr_packed& dt, const etr_packed& xt, const int32_t* offsets, void* dw, void* dw_up,
                                   hipStream_t st) {
    PackedParams p = weight_sizes(c);
    p.A = static_cast<const uint8_t*>(dt.values); p.As = static_cast<const uint8_t*>(dt.scales);
    p.B[0] = static_cast<const uint8_t*>(xt.values); p.Bs[0] = static_cast<const uint8_t*>(xt.scales);
    p.C[0] = dw; p.C[1] = dw_up; p.offsets = offsets;
    return c.dtype == ETR_BF16 ? launch_weight<false>(p, st) : launch_weight<true>(p, st);
}

}  // namespace etr

extern "C" int etr_packed_plan(const etr_linear_config* c, int product) {
    using namespace etr;
    if (product == 2) return static_cast<int>(choose_form<WEIGHT, false>(weight_sizes(*c), false).form);
    const PackedParams p = forward_sizes(*c);
    return static_cast<int>(p.glu ? choose_form<FORWARD, true>(p, product == 1).form : choose_form<FORWARD, false>(p, product == 1).form);
}
