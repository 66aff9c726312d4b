// Packing into 8 bits and back: rows, tokens through the tables of the sorted rows, columns (from either form), and the element-wise
// part of the products' backward, which packs its results both ways.
//   scale = the smallest power of two by which the largest finite magnitude of a block of 128 comes to 448 or less; q = e4m3(x / scale)
// All of it is bound by memory.  The division is by a power of two, so that it is exact, and the result the same in any arithmetic.
// Measured: 32768 tokens x 4096 bf16, top-2, packed 112 us (4.9 TB/s), back 138 (5.8); 16 matrices of 5632 x 2048 bf16 along rows 120 us (4.6), along
// columns 100 (5.5); 16384 x 5632 SwiGLU gradients from packed pre-activations, both ways, 176 us (4.2); packed rows of 16384 x 2048 along columns 19.
#include <algorithm>

#include "activation.h"
#include "packed.h"

namespace etr {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;

// ---- along rows ------------------------------------------------------------------------------------------------------
//
// A wave takes 512 columns at a time, 8 to a lane: sixteen lanes hold a block, and the four blocks' scales are one dword.
struct RowsParams {
    const void* x; uint8_t* q; uint32_t* s;             // unpack: q, s in, y out
    void* y;
    const int32_t* row_of;
    int rows, k;            // rows in; pack of tokens: rows of x, and k rows of the result for each
    int out_rows;           // rows of the packed matrix (the stride of its scales)
    int K, blocks, groups;
    int walkers;            // rows that are under way at once
};
// Steps of 512 columns of a wave: 4, or 1 where that leaves CUs without a wave (32 tokens x 2048, top-2: packed in 4.4 and 2.9 us, back in 3.2 and 2.4).
// All four are on their way at once but in packing from bf16, whose conversion stands behind the bound of its load, with a wait for it: there a CU's
// other waves are what hides the latency (4.6 TB/s).  A row's parts go to neighbouring waves, which walk the rows together.

template <bool BF16>
__device__ __forceinline__ void load8(const void* x, size_t at, float (&f)[8]) {
    if constexpr (BF16) {
        Piece<true>::unpack(*reinterpret_cast<const piece_t*>(static_cast<const uint16_t*>(x) + at), f);
    } else {
        Piece<false>::unpack(*reinterpret_cast<const piece_t*>(static_cast<const float*>(x) + at), f);
        Piece<false>::unpack(*reinterpret_cast<const piece_t*>(static_cast<const float*>(x) + at + 4), f + 4);
    }
}
template <bool BF16>
__device__ __forceinline__ void store8(void* y, size_t at, const float (&f)[8]) {
    if constexpr (BF16) {
        *reinterpret_cast<piece_t*>(static_cast<uint16_t*>(y) + at) = Piece<true>::pack(f);
    } else {
        *reinterpret_cast<piece_t*>(static_cast<float*>(y) + at) = Piece<false>::pack(f);
        *reinterpret_cast<piece_t*>(static_cast<float*>(y) + at + 4) = Piece<false>::pack(f + 4);
    }
}

template <bool BF16, bool TOKENS, int kSteps>
__global__ __launch_bounds__(kThreads) void pack_rows_kernel(RowsParams p, int matrices) {
    const int lane = threadIdx.x & 63, wave = blockIdx.x * kWaves + (threadIdx.x >> 6), parts = (p.groups + kSteps - 1) / kSteps, g0 = wave % parts * kSteps;
    if (wave >= p.walkers * parts) return;
    for (long long row = wave / parts; row < static_cast<long long>(p.rows) * matrices; row += p.walkers) {
        float f[kSteps][8];
#pragma unroll
        for (int u = 0; u < kSteps; ++u) {
            const int c = (g0 + u) * 512 + lane * 8;
#pragma unroll
            for (int i = 0; i < 8; ++i) f[u][i] = 0.f;
            if (c < p.K) load8<BF16>(p.x, static_cast<size_t>(row) * p.K + c, f[u]);
        }
        int mine = -1;
        if constexpr (TOKENS) {
            mine = lane < p.k ? p.row_of[static_cast<size_t>(row) * p.k + lane] : -1;
            if (mine >= p.out_rows) mine = -1;
        }
        uint2 q[kSteps];
        uint32_t s[kSteps];
#pragma unroll
        for (int u = 0; u < kSteps; ++u) {
            const uint32_t byte = scale_byte(row16_max(top_of<8>([&](int i) { return f[u][i]; })));
            const float scale = scale_value(byte);
            q[u].x = to_e4m3(f[u][0], f[u][1], f[u][2], f[u][3], scale);
            q[u].y = to_e4m3(f[u][4], f[u][5], f[u][6], f[u][7], scale);
            s[u] = 0;
#pragma unroll
            for (int b = 0; b < 4; ++b)
                s[u] |= ((g0 + u) * 4 + b < p.blocks ? static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(byte), 16 * b)) : 127u) << (8 * b);
        }
        auto put = [&](size_t values, size_t scales, size_t stride) {
#pragma unroll
            for (int u = 0; u < kSteps; ++u) {
                const int c = (g0 + u) * 512 + lane * 8;
                if (c < p.blocks * kBlock) *reinterpret_cast<uint2*>(p.q + values + c) = q[u];
                if (g0 + u < p.groups && lane == 0) p.s[scales + static_cast<size_t>(g0 + u) * stride] = s[u];
            }
        };
        if constexpr (TOKENS) {
            for (int j = 0; j < p.k; ++j) {
                const int r = __builtin_amdgcn_readlane(mine, j);
                if (r >= 0) put(static_cast<size_t>(r) * p.blocks * kBlock, r, p.out_rows);
            }
        } else {
            const int matrix = matrices > 1 ? static_cast<int>(row) / p.rows : 0, r = static_cast<int>(row) - matrix * p.rows;
            put(static_cast<size_t>(row) * p.blocks * kBlock, static_cast<size_t>(matrix) * p.groups * p.rows + r, p.rows);
        }
    }
}

template <bool BF16, int kSteps>
__global__ __launch_bounds__(kThreads) void unpack_rows_kernel(RowsParams p, int matrices) {
    const int lane = threadIdx.x & 63, wave = blockIdx.x * kWaves + (threadIdx.x >> 6), parts = (p.groups + kSteps - 1) / kSteps, g0 = wave % parts * kSteps;
    if (wave >= p.walkers * parts) return;
    for (long long row = wave / parts; row < static_cast<long long>(p.rows) * matrices; row += p.walkers) {
        const int matrix = matrices > 1 ? static_cast<int>(row) / p.rows : 0, r = static_cast<int>(row) - matrix * p.rows;
        uint2 q[kSteps];
        uint32_t s[kSteps];
#pragma unroll
        for (int u = 0; u < kSteps; ++u) {
            const int c = (g0 + u) * 512 + lane * 8;
            q[u] = make_uint2(0u, 0u);
            s[u] = 0;
            if (c < p.K) {
                q[u] = *reinterpret_cast<const uint2*>(p.q + static_cast<size_t>(row) * p.blocks * kBlock + c);
                s[u] = p.s[(static_cast<size_t>(matrix) * p.groups + g0 + u) * p.rows + r];
            }
        }
#pragma unroll
        for (int u = 0; u < kSteps; ++u) {
            const int c = (g0 + u) * 512 + lane * 8;
            const float scale = scale_value((s[u] >> (8 * (lane >> 4))) & 255u);
            float f[8];
            from_e4m3(q[u].x, scale, f);
            from_e4m3(q[u].y, scale, f + 4);
            if (c < p.K) store8<BF16>(p.y, static_cast<size_t>(row) * p.K + c, f);
        }
    }
}

// ---- tiles of 128 rows and 128 columns: along columns, and both ways ----------------------------------------------------
//
// (Twice the threads with half the rows each: 32768 x 4096 packed again along columns 84 us instead of 58.)
// A thread has eight neighbouring columns of eight neighbouring rows.  A row's largest is found in the sixteen lanes that have it, a
// column's over a wave's 32 rows and then, through LDS, over the four waves.  Values along columns go through LDS too, 8 rows of a
// column at a time, so that they leave as 128 bytes of a column.
enum Source { FROM_F32 = 0, FROM_BF16 = 1, FROM_PACKED = 2 };

struct TileParams {
    const void* x;                                       // the matrix, or dy
    const uint8_t* q[2]; const uint32_t* s[2];           // a matrix packed along rows; or the packed pre-activations
    const int32_t* offsets;
    int rows, E, K, stacked;                             // rows: of each matrix of a stack, or of all
    uint8_t* row_q; uint8_t* row_s; int row_pitch;       // along rows: out, optional
    uint8_t* column_q; uint8_t* column_s; int column_rows;   // along columns: out, optional; rows of a segment's matrix
    int half_blocks;                                     // > 0: a pair of stacks beside each other: blocks of 128 rows to a half
    int half;                                            // which of the two
    float* part; int chunks;                             // column sums of every chunk, optional
    float* sums[2];                                      // where no expert has more than a chunk: the sums of an expert
};

struct TileLds {
    float top[kWaves][kBlock];
    uint2 column[kBlock][16];                            // [column][8 rows each], the eights of a column in the order o ^ (column / 8)
};

// Packs a tile v[row][column] (rows 8 rg + i, columns 8 cg + j of it) along columns.
// block: the block of rows, `last` if its matrix has no more; values: the matrix's first byte; pitch: bytes of its rows;
// scales: its first byte of scales; c0: the tile's first column, limit: its columns; matrix_rows: rows of the packed matrix;
// base: row of the packed matrix that column 0 is
__device__ __forceinline__ void pack_tile_columns(const float (&v)[8][8], TileLds& lds, uint8_t* values, size_t pitch, uint8_t* scales, int block, bool last,
                                                  int c0, int limit, int matrix_rows, int base) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, cg = lane & 15, rg = tid >> 4;
    float top[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        top[j] = top_of<8>([&](int i) { return v[i][j]; });
        top[j] = fmaxf(top[j], __shfl_xor(top[j], 16));
        top[j] = fmaxf(top[j], __shfl_xor(top[j], 32));
    }
    __syncthreads();                                     // (an earlier tile's reads are done)
    if (lane < 16) {
#pragma unroll
        for (int j = 0; j < 8; ++j) lds.top[wave][cg * 8 + j] = top[j];
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int c = cg * 8 + j;
        float t = lds.top[0][c];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) t = fmaxf(t, lds.top[w][c]);
        const uint32_t byte = scale_byte(t);
        const float scale = scale_value(byte);
        const uint2 q = make_uint2(to_e4m3(v[0][j], v[1][j], v[2][j], v[3][j], scale), to_e4m3(v[4][j], v[5][j], v[6][j], v[7][j], scale));
        lds.column[c][rg ^ cg] = q;
        if (rg == 0 && c0 + c < limit) {
            uint8_t* at = scales + (static_cast<size_t>(block >> 2) * matrix_rows + base + c0 + c) * 4;
            at[block & 3] = static_cast<uint8_t>(byte);
            if (last)
                for (int b = (block & 3) + 1; b < 4; ++b) at[b] = 127;
        }
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int c = u * 32 + (tid >> 3), piece = tid & 7;
        const uint2 lo = lds.column[c][(2 * piece) ^ (c >> 3)], hi = lds.column[c][(2 * piece + 1) ^ (c >> 3)];
        if (c0 + c < limit)
            *reinterpret_cast<piece_t*>(values + static_cast<size_t>(base + c0 + c) * pitch + static_cast<size_t>(block) * kBlock + piece * 16) = piece_t{lo.x, lo.y, hi.x, hi.y};
    }
}

// Packs the same tile along rows.  first: the tile's first row of the packed matrix; n_rows: its rows; block: its block of columns
__device__ __forceinline__ void pack_tile_rows(const float (&v)[8][8], uint8_t* values, size_t pitch, uint8_t* scales, int block, bool last, size_t first, int n_rows,
                                               int matrix_rows) {
    const int cg = threadIdx.x & 15, rg = threadIdx.x >> 4;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t byte = scale_byte(row16_max(top_of<8>([&](int j) { return v[i][j]; })));
        const float scale = scale_value(byte);
        if (rg * 8 + i < n_rows) {
            const size_t row = first + rg * 8 + i;
            *reinterpret_cast<uint2*>(values + row * pitch + static_cast<size_t>(block) * kBlock + cg * 8) =
                make_uint2(to_e4m3(v[i][0], v[i][1], v[i][2], v[i][3], scale), to_e4m3(v[i][4], v[i][5], v[i][6], v[i][7], scale));
            if (cg == 0) {
                uint8_t* at = scales + (static_cast<size_t>(block >> 2) * matrix_rows + row) * 4;
                at[block & 3] = static_cast<uint8_t>(byte);
                if (last)
                    for (int b = (block & 3) + 1; b < 4; ++b) at[b] = 127;
            }
        }
    }
}

// Column sums of a tile, in a fixed order: a thread's rows, the wave's, the waves'.
__device__ __forceinline__ void tile_sums(const float (&v)[8][8], TileLds& lds, float* out, int c0, int limit) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, cg = lane & 15;
    float sum[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        sum[j] = ((v[0][j] + v[1][j]) + (v[2][j] + v[3][j])) + ((v[4][j] + v[5][j]) + (v[6][j] + v[7][j]));
        sum[j] += __shfl_xor(sum[j], 16);
        sum[j] += __shfl_xor(sum[j], 32);
    }
    __syncthreads();
    if (lane < 16) {
#pragma unroll
        for (int j = 0; j < 8; ++j) lds.top[wave][cg * 8 + j] = sum[j];
    }
    __syncthreads();
    if (tid < kBlock && c0 + tid < limit) out[c0 + tid] = (lds.top[0][tid] + lds.top[1][tid]) + (lds.top[2][tid] + lds.top[3][tid]);
}

// Eight neighbouring values of a row as they lie in memory.
template <int SOURCE> struct Eight {
    piece_t v[SOURCE == FROM_F32 ? 2 : 1];
    __device__ __forceinline__ void load(const TileParams& p, size_t row, int c) {
        const size_t at = row * p.K + c;
        if constexpr (SOURCE == FROM_BF16) {
            v[0] = *reinterpret_cast<const piece_t*>(static_cast<const uint16_t*>(p.x) + at);
        } else {
            v[0] = *reinterpret_cast<const piece_t*>(static_cast<const float*>(p.x) + at);
            v[1] = *reinterpret_cast<const piece_t*>(static_cast<const float*>(p.x) + at + 4);
        }
    }
    __device__ __forceinline__ void unpack(float (&f)[8]) const {
        if constexpr (SOURCE == FROM_BF16) {
            Piece<true>::unpack(v[0], f);
        } else {
            Piece<false>::unpack(v[0], f);
            Piece<false>::unpack(v[1], f + 4);
        }
    }
};
struct EightPacked {
    uint2 q; uint32_t s;
    // matrix_scales: first dword of the matrix's scales; scale_row, of scale_rows: the row there
    __device__ __forceinline__ void load(const uint8_t* values, const uint32_t* scales, int pitch, size_t row, int c, size_t matrix_scales, size_t scale_row, int scale_rows) {
        q = *reinterpret_cast<const uint2*>(values + row * pitch + c);
        s = scales[matrix_scales + static_cast<size_t>(c >> 9) * scale_rows + scale_row];
    }
    __device__ __forceinline__ void unpack(int c, float (&f)[8]) const {
        const float scale = scale_value((s >> (8 * ((c >> 7) & 3))) & 255u);
        from_e4m3(q.x, scale, f);
        from_e4m3(q.y, scale, f + 4);
    }
};
template <> struct Eight<FROM_PACKED> : EightPacked {};

// ACT (an etr_act): dy in `x`, the packed pre-activations in q and s
// SPLIT: few tiles, whose latency counts: workgroups of their own (blockIdx.y) for each direction and, with SwiGLU, for each half.
template <int SOURCE, int ACT, bool SPLIT>
__global__ __launch_bounds__(kThreads, 2) void pack_tiles_kernel(TileParams p) {
    __shared__ TileLds lds;
    const int tid = threadIdx.x, cg = tid & 15, rg = tid >> 4;
    Segments g;
    g.load(p.offsets, p.rows, p.E, p.stacked);
    const bool direct = p.sums[0] != nullptr;            // a workgroup to an expert, which has 128 rows at most
    const int per_half = blocks_of(p.K), nb = blockIdx.x % per_half, chunk = blockIdx.x / per_half, c0 = nb * kBlock, c = c0 + cg * 8;
    if (!direct && chunk >= __builtin_amdgcn_readlane(g.blocks_incl, 63)) return;
    const int e = direct ? chunk : __builtin_ctzll(__ballot(g.blocks_incl > chunk));
    const int blocks = __builtin_amdgcn_readlane(g.blocks, e), blocks_before = __builtin_amdgcn_readlane(g.blocks_incl, e) - blocks;
    const int groups_before = __builtin_amdgcn_readlane(g.groups_incl, e) - __builtin_amdgcn_readlane(g.groups, e);
    const int block = direct ? 0 : chunk - blocks_before;
    const int n_rows = min(kBlock, __builtin_amdgcn_readlane(g.count, e) - block * kBlock);
    const size_t first = static_cast<size_t>(__builtin_amdgcn_readlane(g.first, e)) + static_cast<size_t>(block) * kBlock;
    const bool nothing = direct && n_rows <= 0;          // an expert without rows: zeros for its sums, and no block
    // FAST: the exponential's exponent without its lower part, a term off by some (|a| + 4) 2^-24 of its size.  Far below what dy's own rounding to
    // bf16 (2^-8) has left open, for the packed results and for the sums over rows alike; the sums have these terms' errors, beside their own in fp32.
    constexpr bool FAST = SOURCE == FROM_BF16;
    constexpr bool GLU = ACT == ETR_ACT_SWIGLU;
    constexpr int n_halves = GLU ? 2 : 1, parts = SPLIT ? 1 : n_halves;                     // parts: halves at a time
    const int half = SPLIT ? blockIdx.y % n_halves : 0;
    const bool along_rows = !SPLIT || static_cast<int>(blockIdx.y) < n_halves, along_columns = !SPLIT || !along_rows;
    if (SPLIT && !(along_rows ? p.row_q || p.part || direct : p.column_q != nullptr)) return;

    // everything is requested before the first is used; past the ends the last row or columns again, which count as zeros
    Eight<SOURCE> from[8];
    EightPacked pre[ACT != ETR_ACT_NONE ? 8 : 1], up[GLU ? 8 : 1];
    const int pitch = blocks_of(p.K) * kBlock, cc = min(c, p.K - 8);
    if (!nothing) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const size_t row = first + min(rg * 8 + i, n_rows - 1);
            if constexpr (SOURCE == FROM_PACKED) {
                // a stack's matrices have scales of their own
                from[i].load(p.q[0], p.s[0], pitch, row, cc, p.stacked ? static_cast<size_t>(e) * scale_groups_of(p.K) * p.rows : 0,
                             p.stacked ? row - static_cast<size_t>(e) * p.rows : row, p.rows);
            } else {
                from[i].load(p, row, cc);
            }
            if constexpr (ACT != ETR_ACT_NONE) pre[i].load(p.q[0], p.s[0], pitch, row, cc, 0, row, p.rows);
            if constexpr (GLU) up[i].load(p.q[1], p.s[1], pitch, row, cc, 0, row, p.rows);
        }
    }
    float v[parts][8][8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float (&d)[8] = v[0][i];
        if constexpr (SOURCE == FROM_PACKED) from[i].unpack(cc, d);
        else from[i].unpack(d);
        if constexpr (ACT != ETR_ACT_NONE) {
            float a[8], b[8];
            pre[i].unpack(cc, a);
            if constexpr (GLU) up[i].unpack(cc, b);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if constexpr (ACT == ETR_ACT_GELU) {
                    d[j] *= normal_cdf<FAST>(a[j]) + a[j] * 0.39894228040143268f * (FAST ? __expf(-0.5f * a[j] * a[j]) : gaussian_f32(a[j]));
                } else {
                    const float sg = sigmoid<FAST>(a[j]), slope = sg * (1.0f + a[j] * (1.0f - sg));
                    if constexpr (GLU && SPLIT) {        // (compiled to uniform branches, 16 to a row of eight)
                        d[j] *= half ? a[j] * sg : b[j] * slope;
                    } else if constexpr (GLU) {
                        v[parts - 1][i][j] = d[j] * (a[j] * sg);
                        d[j] *= b[j] * slope;
                    } else {
                        d[j] *= slope;
                    }
                }
            }
        }
        if (rg * 8 + i >= n_rows || c >= p.K) {
#pragma unroll
            for (int u = 0; u < parts; ++u)
#pragma unroll
                for (int j = 0; j < 8; ++j) v[u][i][j] = 0.f;
        }
        __builtin_amdgcn_sched_barrier(0);               // one row at a time: keeps the live set small
    }
#pragma unroll
    for (int u = 0; u < parts; ++u) {
        const int h = half + u;
        if (p.row_q && along_rows && !nothing) pack_tile_rows(v[u], p.row_q, p.row_pitch, p.row_s, h * per_half + nb, h == n_halves - 1 && nb == per_half - 1, first, n_rows, p.rows);
        if (along_rows && (p.part || direct)) {
            float* out = direct ? p.sums[h] + static_cast<size_t>(e) * p.K : p.part + (static_cast<size_t>(h) * p.chunks + chunk) * p.K;
            tile_sums(v[u], lds, out, c0, p.K);
        }
        if (p.column_q && along_columns && !nothing) {
            if (p.half_blocks) {                         // a pair of stacks: the matrix has 2 half_blocks blocks
                const int all = 2 * p.half_blocks, at = p.half * p.half_blocks + block;
                pack_tile_columns(v[u], lds, p.column_q + static_cast<size_t>(e) * p.K * all * kBlock, static_cast<size_t>(all) * kBlock,
                                  p.column_s + static_cast<size_t>(e) * ((all + 3) / 4) * p.K * 4, at, at == all - 1, c0, p.K, p.K, 0);
            } else {
                pack_tile_columns(v[u], lds, p.column_q + static_cast<size_t>(blocks_before) * kBlock * p.column_rows, static_cast<size_t>(blocks) * kBlock,
                                  p.column_s + static_cast<size_t>(groups_before) * 4 * p.column_rows, block, block == blocks - 1, c0, p.K, p.column_rows,
                                  h * p.K);
            }
        }
    }
}

// dbias[e][n]: the chunks of expert e, sixteen groups of them side by side, in a fixed order
__global__ __launch_bounds__(1024) void join_sums_kernel(TileParams p, float* dbias, float* dbias_up) {
    __shared__ float sums[16][64];
    Segments g;
    g.load(p.offsets, p.rows, p.E, false);
    const int e = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = blockIdx.x * 64 + lane;
    const int blocks = __builtin_amdgcn_readlane(g.blocks, e), begin = __builtin_amdgcn_readlane(g.blocks_incl, e) - blocks;
    const float* part = p.part + static_cast<size_t>(blockIdx.z) * p.chunks * p.K;
    float s = 0.f;
    if (n < p.K) {
#pragma unroll 4
        for (int i = wave; i < blocks; i += 16) s += part[static_cast<size_t>(begin + i) * p.K + n];
    }
    sums[wave][lane] = s;
    __syncthreads();
    if (wave > 0 || n >= p.K) return;
    s = 0.f;
#pragma unroll
    for (int w = 0; w < 16; ++w) s += sums[w][lane];
    (blockIdx.z ? dbias_up : dbias)[static_cast<size_t>(e) * p.K + n] = s;
}

// ---- host ------------------------------------------------------------------------------------------------------------

RowsParams rows_params(int rows, int K) {
    RowsParams p{};
    p.rows = p.out_rows = rows;
    p.K = K; p.blocks = blocks_of(K); p.groups = scale_groups_of(K);
    return p;
}
template <class F4, class F1>
hipError_t launch_rows(F4 four, F1 one, RowsParams p, int matrices, hipStream_t st) {
    const long long rows = static_cast<long long>(p.rows) * matrices;                        // (2^30 at most)
    const bool few = rows * p.groups <= 16ll * cu_count();
    const int parts = few ? p.groups : (p.groups + 3) / 4;
    p.walkers = static_cast<int>(std::min<long long>(rows, std::max(1, (1 << 22) / parts)));
    const dim3 grid(static_cast<unsigned>((static_cast<long long>(p.walkers) * parts + kWaves - 1) / kWaves));
    if (few) hipLaunchKernelGGL(one, grid, dim3(kThreads), 0, st, p, matrices);
    else hipLaunchKernelGGL(four, grid, dim3(kThreads), 0, st, p, matrices);
    return hipGetLastError();
}
template <bool BF16, bool TOKENS>
hipError_t launch_pack(const RowsParams& p, int matrices, hipStream_t st) {
    return launch_rows(pack_rows_kernel<BF16, TOKENS, 4>, pack_rows_kernel<BF16, TOKENS, 1>, p, matrices, st);
}
template <bool BF16>
hipError_t launch_unpack(const RowsParams& p, int matrices, hipStream_t st) {
    return launch_rows(unpack_rows_kernel<BF16, 4>, unpack_rows_kernel<BF16, 1>, p, matrices, st);
}
int chunks_at_most(int rows, int E, bool stacked) { return stacked ? E * blocks_of(rows) : rows / kBlock + std::min(E, rows); }

template <int SOURCE, int ACT>
hipError_t launch_tiles(const TileParams& p, int chunks, hipStream_t st) {
    const unsigned tiles = static_cast<unsigned>(blocks_of(p.K)) * chunks;
    // A tile for each direction and half once a tile of all leaves half of the CUs idle; chip filled, what they compute twice costs more.  us, of all / split:
    // SwiGLU bf16 44 tiles 13.9 / 9.1, 130 14.4 / 11.2, 304 15.5 / 17.5; SiLU 44 8.9 / 7.4, 165 9.3 / 9.5; GELU fp32 110 11.6 / 10.1, 165 11.8 / 13.6.
    // One border for all, where SiLU and GELU have theirs; SwiGLU's lies between 130 and 304 tiles, and from 129 up to there it takes longer than split.
    if constexpr (SOURCE != FROM_PACKED) {
        const bool both = (p.row_q || p.part || p.sums[0]) && p.column_q;
        if (2ll * tiles <= cu_count() && (ACT == ETR_ACT_SWIGLU || both)) {
            hipLaunchKernelGGL((pack_tiles_kernel<SOURCE, ACT, true>), dim3(tiles, ACT == ETR_ACT_SWIGLU ? 4 : 2), dim3(kThreads), 0, st, p);
            return hipGetLastError();
        }
    }
    hipLaunchKernelGGL((pack_tiles_kernel<SOURCE, ACT, false>), dim3(tiles), dim3(kThreads), 0, st, p);
    return hipGetLastError();
}

}  // namespace

size_t packed_columns_bytes(const etr_pack_config& c) {
    if (!c.sorted) return packed_bytes(static_cast<size_t>(c.E) * c.K, c.rows);
    return static_cast<size_t>(c.K) * kBlock * (c.rows / kBlock + std::min(c.E, c.rows));
}
size_t packed_columns_scale_bytes(const etr_pack_config& c) {
    if (!c.sorted) return scale_bytes(static_cast<size_t>(c.E) * c.K, c.rows);
    return static_cast<size_t>(c.K) * 4 * (c.rows / (4 * kBlock) + std::min(c.E, c.rows));
}

hipError_t launch_pack_rows(const etr_pack_config& c, const void* x, void* values, void* scales, hipStream_t st) {
    RowsParams p = rows_params(c.rows, c.K);
    const int matrices = c.sorted ? 1 : c.E;
    p.x = x; p.q = static_cast<uint8_t*>(values); p.s = static_cast<uint32_t*>(scales);
    return c.dtype == ETR_BF16 ? launch_pack<true, false>(p, matrices, st) : launch_pack<false, false>(p, matrices, st);
}

hipError_t launch_pack_sorted_rows(const etr_sort_config& c, const void* x, const int32_t* row_of, void* values, void* scales, hipStream_t st) {
    RowsParams p = rows_params(c.T, c.d);
    p.k = c.k; p.out_rows = c.T * c.k; p.row_of = row_of;
    p.x = x; p.q = static_cast<uint8_t*>(values); p.s = static_cast<uint32_t*>(scales);
    return c.dtype == ETR_BF16 ? launch_pack<true, true>(p, 1, st) : launch_pack<false, true>(p, 1, st);
}

hipError_t launch_unpack_rows(const etr_pack_config& c, const void* values, const void* scales, void* y, hipStream_t st) {
    RowsParams p = rows_params(c.rows, c.K);
    const int matrices = c.sorted ? 1 : c.E;
    p.q = static_cast<uint8_t*>(const_cast<void*>(values)); p.s = static_cast<uint32_t*>(const_cast<void*>(scales)); p.y = y;
    return c.dtype == ETR_BF16 ? launch_unpack<true>(p, matrices, st) : launch_unpack<false>(p, matrices, st);
}

hipError_t launch_pack_columns(const etr_pack_config& c, const void* x, const etr_packed* packed, const int32_t* offsets, int half, void* values, void* scales,
                               hipStream_t st) {
    TileParams p{};
    p.x = x;
    if (packed) { p.q[0] = static_cast<const uint8_t*>(packed->values); p.s[0] = static_cast<const uint32_t*>(packed->scales); }
    p.offsets = offsets; p.rows = c.rows; p.E = c.E; p.K = c.K; p.stacked = !c.sorted;
    p.column_q = static_cast<uint8_t*>(values); p.column_s = static_cast<uint8_t*>(scales); p.column_rows = c.K;
    if (half >= 0) { p.half_blocks = blocks_of(c.rows); p.half = half; }
    const int chunks = chunks_at_most(c.rows, c.E, p.stacked);
    if (packed) return launch_tiles<FROM_PACKED, ETR_ACT_NONE>(p, chunks, st);
    return c.dtype == ETR_BF16 ? launch_tiles<FROM_BF16, ETR_ACT_NONE>(p, chunks, st) : launch_tiles<FROM_F32, ETR_ACT_NONE>(p, chunks, st);
}

size_t packed_act_ws_bytes(const etr_linear_config& c) {
    return align_up(static_cast<size_t>(c.act == ETR_ACT_SWIGLU ? 2 : 1) * chunks_at_most(c.rows, c.E, false) * c.N * 4);
}

hipError_t launch_packed_act_backward(const etr_linear_config& c, const void* dy, const int32_t* offsets, const etr_packed* pre8, const etr_packed* pre_up8,
                                const etr_packed* d8, const etr_packed* dt8, float* dbias, float* dbias_up, void* ws, hipStream_t st) {
    const bool glu = c.act == ETR_ACT_SWIGLU, direct = dbias && c.rows <= kBlock;
    TileParams p{};
    p.x = dy; p.offsets = offsets; p.rows = c.rows; p.E = c.E; p.K = c.N;
    const etr_packed* pre[2] = {pre8, pre_up8};
    for (int i = 0; i < 2; ++i)
        if (pre[i]) { p.q[i] = static_cast<const uint8_t*>(pre[i]->values); p.s[i] = static_cast<const uint32_t*>(pre[i]->scales); }
    if (d8) {
        p.row_q = static_cast<uint8_t*>(d8->values); p.row_s = static_cast<uint8_t*>(d8->scales);
        p.row_pitch = (glu ? 2 : 1) * blocks_of(c.N) * kBlock;
    }
    if (dt8) { p.column_q = static_cast<uint8_t*>(dt8->values); p.column_s = static_cast<uint8_t*>(dt8->scales); p.column_rows = (glu ? 2 : 1) * c.N; }
    p.chunks = chunks_at_most(c.rows, c.E, false);
    if (direct) { p.sums[0] = dbias; p.sums[1] = dbias_up; }
    else if (dbias) p.part = static_cast<float*>(ws);
    const int chunks = direct ? c.E : p.chunks;
    const bool bf16 = c.dtype == ETR_BF16;
    hipError_t err = hipErrorInvalidValue;
    switch (c.act) {
        case ETR_ACT_NONE: err = bf16 ? launch_tiles<FROM_BF16, ETR_ACT_NONE>(p, chunks, st) : launch_tiles<FROM_F32, ETR_ACT_NONE>(p, chunks, st); break;
        case ETR_ACT_SILU: err = bf16 ? launch_tiles<FROM_BF16, ETR_ACT_SILU>(p, chunks, st) : launch_tiles<FROM_F32, ETR_ACT_SILU>(p, chunks, st); break;
        case ETR_ACT_GELU: err = bf16 ? launch_tiles<FROM_BF16, ETR_ACT_GELU>(p, chunks, st) : launch_tiles<FROM_F32, ETR_ACT_GELU>(p, chunks, st); break;
        case ETR_ACT_SWIGLU: err = bf16 ? launch_tiles<FROM_BF16, ETR_ACT_SWIGLU>(p, chunks, st) : launch_tiles<FROM_F32, ETR_ACT_SWIGLU>(p, chunks, st); break;
    }
    if (err != hipSuccess || !p.part) return err;
    hipLaunchKernelGGL(join_sums_kernel, dim3((c.N + 63) / 64, c.E, glu ? 2 : 1), dim3(1024), 0, st, p, dbias, dbias_up);
    return hipGetLastError();
}

}  // namespace etr
