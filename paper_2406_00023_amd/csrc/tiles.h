// The tiles of a product on rows sorted by expert: which rows an expert has, and which tile is a workgroup's next.  P: a product's
// parameters, with offsets (device, [E+1], or null), rows, E, M, glu and NT.
#pragma once

#include "etr_internal.h"

namespace etr {
namespace {

enum Product { FORWARD = 0, INPUT = 1, WEIGHT = 2 };     // y, dx, dw

// Rows of the groups, one group per lane (E <= 64): first row, number, and the row tiles before it.
struct Groups {
    int first, count, tiles_incl, tiles;
    template <class P> __device__ __forceinline__ void load(const P& p, int BM) {
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
template <int MODE, bool SPLIT, class P>
__device__ __forceinline__ bool find_tile(const P& p, const Groups& g, int BM, int BN, int bid, int grid, int j, Tile& t) {
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

}  // namespace
}  // namespace etr
