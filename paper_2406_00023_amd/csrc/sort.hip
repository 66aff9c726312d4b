// Rows sorted by expert without padding: the tables (a stable counting sort of the pairs (token, place) by expert), the rows
// taken there and brought back with their weights, and both gradients.
//   xs[row] = x[t];   out[t] = sum_j w_tj ys[row_tj];   dx[t] = sum_j dxs[row_tj];   dys[row_tj] = w_tj dout[t]
//   with g' the gradient of the weights, g'_tj = <dout[t], ys[row_tj]>:  dgate[t][e] = sum of g'_tj over the places that list e,
//   or, where the weights are divided by their sum S over the token:  (g'_tj - sum_i g'_ti w_ti) / S
// The tables are bound by latency (two launches, or one for few pairs), the row movers by memory.  All row movers
// walk the tokens, not the rows: a token's row is read or written once while its k copies are streamed, no atomics are
// needed for the sums over a token's rows, and their order is that of the places.
// Measured: 32768 tokens x 4096 bf16, top-2 of 32: tables 9 us, rows taken 142 us and brought back 138 (5.7 TB/s), their gradients 137 and 247 (5.4);
// 32 x 2048, top-2 of 16: 2.4, 2.6 and 3.1.
#include <algorithm>

#include "row_ops.h"

namespace etr {
namespace {

constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / kWave;
// One launch for up to 4096 pairs (64 pairs 2.4 us), two for more (9003 pairs 2.3 + 3.8 us; one workgroup took 18, about a microsecond per
// 1024 pairs).  One workgroup for up to kOnePairs pairs; else kMinPairs or more to a workgroup, and at most 256 workgroups.
constexpr int kMaxSortBlocks = 256, kMinPairs = 1024, kOnePairs = 4096;
constexpr int kHeld = kOnePairs / kSortThreads;            // pairs of a thread that stay in registers between counting and placing
constexpr int kMaxExperts = 64;

struct SortParams {
    const int32_t* topk; const int32_t* slot_of;
    int32_t* offsets; int32_t* row_of; int32_t* pair_of;
    int32_t* hist;          // [workgroups][E]
    int k, E, bits;         // bits: 2^bits >= E + 1
    int pairs, per_block;   // per_block: whole rounds of kSortThreads
};

// expert of pair q, or E where it is not in use (and for q past the end)
__device__ __forceinline__ int pair_expert(const SortParams& p, int q, int end) {
    if (q >= end) return p.E;
    const int e = p.topk[q];
    if (e < 0 || e >= p.E) return p.E;
    if (p.slot_of && p.slot_of[static_cast<size_t>(q / p.k) * p.E + e] < 0) return p.E;
    return e;
}
// lanes of the wave whose e is this lane's
__device__ __forceinline__ uint64_t same_expert(int e, int bits) {
    uint64_t same = ~0ull;
    for (int b = 0; b < bits; ++b) {
        const uint64_t set = __ballot((e >> b) & 1);
        same &= (e >> b) & 1 ? set : ~set;
    }
    return same;
}

// Experts of N groups of 64 pairs from q on, all requested before the first is used.
template <int N>
__device__ __forceinline__ void load_experts(const SortParams& p, int q, int end, int (&e)[N]) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < N; ++i) e[i] = p.E;
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (q + i * 64 < end) e[i] = pair_expert(p, q + i * 64 + lane, end);
}
// Pairs of each expert in each wave's part of the workgroup's share: the wave's own row of LDS, so no atomics.  e: the experts of its last
// N groups of 64 pairs (all of them where it has no more).
template <int N>
__device__ __forceinline__ void count_pairs(const SortParams& p, int first, int end, int (*cnt)[kMaxExperts + 1], int (&e)[N]) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    for (int i = lane; i <= kMaxExperts; i += 64) cnt[wave][i] = 0;
    wave_sync();
    for (int q = first; q < end; q += 64 * N) {              // (uniform over the wave)
        load_experts(p, q, end, e);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (q + i * 64 >= end) continue;
            const uint64_t same = same_expert(e[i], p.bits);
            if (__builtin_ctzll(same) == lane) cnt[wave][e[i]] += __popcll(same);
            wave_sync();
        }
    }
}

// this wave's part of the workgroup's share of the pairs
__device__ __forceinline__ void wave_part(const SortParams& p, int& first, int& end) {
    const int begin = min(static_cast<int>(blockIdx.x) * p.per_block, p.pairs), stop = min(begin + p.per_block, p.pairs), part = p.per_block / kSortWaves;
    first = min(begin + static_cast<int>(threadIdx.x >> 6) * part, stop);
    end = min(first + part, stop);
}

__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(SortParams p) {
    __shared__ int cnt[kSortWaves][kMaxExperts + 1];
    int first, end;
    wave_part(p, first, end);
    int e[4];
    count_pairs(p, first, end, cnt, e);
    __syncthreads();
    if (static_cast<int>(threadIdx.x) < p.E) {
        int s = 0;
        for (int w = 0; w < kSortWaves; ++w) s += cnt[w][threadIdx.x];
        p.hist[blockIdx.x * p.E + threadIdx.x] = s;
    }
}

// Every workgroup adds up the counts of all of them itself (at most 256 x 64 numbers out of the L2) instead of waiting for
// a launch between that does; ONE: it is the only workgroup, and its own counts are all there are.
template <bool ONE>
__global__ __launch_bounds__(kSortThreads) void sort_rank_kernel(SortParams p) {
    __shared__ int cnt[kSortWaves][kMaxExperts + 1];
    __shared__ int before[kMaxExperts], total[kMaxExperts], base[kMaxExperts + 1];
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    int first, end;
    wave_part(p, first, end);
    if (tid < kMaxExperts) before[tid] = total[tid] = 0;
    __syncthreads();
    if constexpr (!ONE) {
        const int per = kSortThreads / p.E, e = tid % p.E, part = tid / p.E;       // `per` threads to an expert
        if (part < per) {
            int sum_before = 0, sum = 0;
            for (int b = part; b < static_cast<int>(gridDim.x); b += per) {
                const int n = p.hist[b * p.E + e];
                sum += n;
                sum_before += b < static_cast<int>(blockIdx.x) ? n : 0;
            }
            atomicAdd(&before[e], sum_before);               // whole numbers: any order gives the same
            atomicAdd(&total[e], sum);
        }
    }
    constexpr int N = ONE ? kHeld : 4;
    int e[N];
    count_pairs(p, first, end, cnt, e);
    __syncthreads();
    if (wave == 0) {                                         // lane = expert: rows before each expert, then before each wave
        int all = 0;
        if (lane < p.E) {
            if constexpr (ONE) {
                for (int w = 0; w < kSortWaves; ++w) all += cnt[w][lane];
            } else {
                all = total[lane];
            }
        }
        const int incl = wave_scan_incl(all);
        int at = incl - all + (ONE ? 0 : before[lane]);
        for (int w = 0; w < kSortWaves; ++w) {
            const int n = cnt[w][lane];
            cnt[w][lane] = at;
            at += n;
        }
        if (lane == 63) base[0] = incl;                      // rows in use
        if (blockIdx.x == 0) {
            if (lane == 0) p.offsets[0] = 0;
            if (lane < p.E) p.offsets[lane + 1] = incl;
        }
    }
    __syncthreads();
    const int used = base[0];
    for (int q0 = first; q0 < end; q0 += 64 * N) {
        if (end - first > 64 * N) load_experts(p, q0, end, e);              // (else they are still there)
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int q = q0 + i * 64;
            if (q >= end) continue;
            const uint64_t same = same_expert(e[i], p.bits);
            const int rank = __popcll(same & ((1ull << lane) - 1ull));
            const bool in = e[i] < p.E;
            const int row = in ? cnt[wave][e[i]] + rank : -1;
            wave_sync();
            if (in && rank == 0) cnt[wave][e[i]] += __popcll(same);
            wave_sync();
            if (q + lane < end) {
                p.row_of[q + lane] = row;
                if (in) p.pair_of[row] = q + lane;
                if (q + lane >= used) p.pair_of[q + lane] = -1;             // (no pair's row lies there)
            }
        }
    }
}

// ---- rows ----------------------------------------------------------------------------------------------------------

struct RowsParams {
    const piece_t* in;      // x, ys, dxs
    piece_t* out;           // xs, out, dx
    const float* gate; const int32_t* topk; const int32_t* row_of;
    int T, k, E, pieces, rows, gate_norm;
    int segments;           // parts of a row, each a wave's
};

// Lane j < k: row of the token's j-th pair, -1 if not in use
__device__ __forceinline__ int lane_row(const int32_t* row_of, size_t t, int k, int rows, int lane) {
    const int r = lane < k ? row_of[t * k + lane] : -1;
    return r < rows ? r : -1;
}
// The inverse of a token's sum of weights, 0 without one, in two factors: that of a sum below 2^-128 is no fp32 number.
struct Inverse {
    float lift = 1.0f, value = 1.0f;
    __device__ __forceinline__ void set(float sum) {
        lift = sum < 0x1p-100f ? 0x1p100f : 1.0f;
        value = sum > 0.f ? 1.0f / (sum * lift) : 0.f;
    }
    __device__ __forceinline__ float of(float v) const { return v * lift * value; }
};
// Lane j < k: weight of the token's j-th pair (0 if not in use); with `norm` divided by the token's sum, whose inverse is handed back
__device__ __forceinline__ float lane_weight(const float* gate, const int32_t* topk, size_t t, int k, int E, int row, int norm, int lane,
                                             int& expert, Inverse& inverse) {
    expert = -1;
    float w = 0.f;
    if (row >= 0) {                                          // (only in lanes below k)
        expert = topk[t * k + lane];
        if (expert >= 0 && expert < E) w = gate[t * E + expert];
    }
    if (norm) {
        inverse.set(wave_sum(w));
        w = inverse.of(w);
    }
    return w;
}

constexpr int kRowsThreads = 256, kRowsWaves = kRowsThreads / kWave;
constexpr int kSegment = 4;                                  // 16-byte pieces per lane and segment

// xs[row_of[t][j]] = x[t]: a wave has a segment of a token's row, read once and stored k times.
__global__ __launch_bounds__(kRowsThreads) void sort_rows_kernel(RowsParams p) {
    const int lane = threadIdx.x & 63;
    for (long long unit = static_cast<long long>(blockIdx.x) * kRowsWaves + (threadIdx.x >> 6); unit < p.T * static_cast<long long>(p.segments);
         unit += static_cast<long long>(gridDim.x) * kRowsWaves) {
        const long long t = unit / p.segments;
        const int c0 = static_cast<int>(unit - t * p.segments) * kSegment * kWave + lane;
        piece_t v[kSegment];
#pragma unroll
        for (int u = 0; u < kSegment; ++u)
            if (c0 + u * kWave < p.pieces) v[u] = p.in[static_cast<size_t>(t) * p.pieces + c0 + u * kWave];
        const int mine = lane_row(p.row_of, t, p.k, p.rows, lane);
        for (int j = 0; j < p.k; ++j) {
            const int row = __builtin_amdgcn_readlane(mine, j);
            if (row < 0) continue;
            piece_t* dst = p.out + static_cast<size_t>(row) * p.pieces;
#pragma unroll
            for (int u = 0; u < kSegment; ++u)
                if (c0 + u * kWave < p.pieces) __builtin_nontemporal_store(v[u], dst + c0 + u * kWave);
        }
    }
}

// out[t] = sum_j w_tj in[row_of[t][j]] (WEIGHTED) or the plain sum, in the order of the places
template <bool BF16, bool WEIGHTED>
__global__ __launch_bounds__(kRowsThreads) void gather_sum_kernel(RowsParams p) {
    using R = Piece<BF16>;
    constexpr int V = R::kN;
    const int lane = threadIdx.x & 63;
    for (long long unit = static_cast<long long>(blockIdx.x) * kRowsWaves + (threadIdx.x >> 6); unit < p.T * static_cast<long long>(p.segments);
         unit += static_cast<long long>(gridDim.x) * kRowsWaves) {
        const long long t = unit / p.segments;
        const int c0 = static_cast<int>(unit - t * p.segments) * kSegment * kWave + lane;
        const int mine = lane_row(p.row_of, t, p.k, p.rows, lane);
        float weight = 1.0f;
        int expert;
        Inverse inverse;
        if constexpr (WEIGHTED) weight = lane_weight(p.gate, p.topk, t, p.k, p.E, mine, p.gate_norm, lane, expert, inverse);
        float acc[kSegment][V];
#pragma unroll
        for (int u = 0; u < kSegment; ++u)
#pragma unroll
            for (int i = 0; i < V; ++i) acc[u][i] = 0.f;
        uint64_t left = __ballot(mine >= 0);
        while (left) {                                           // two rows at a time: both are requested before the first is used
            piece_t v[2][kSegment];
            float w[2];
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const int j = left ? __builtin_ctzll(left) : -1;
                left &= left - 1;                                // (0 stays 0: 0 & ~0)
                const int row = __builtin_amdgcn_readlane(mine, j < 0 ? 0 : j);
                w[s] = j < 0 ? 0.f : lane_value(weight, j);
#pragma unroll
                for (int u = 0; u < kSegment; ++u)
                    v[s][u] = j >= 0 && c0 + u * kWave < p.pieces ? p.in[static_cast<size_t>(row) * p.pieces + c0 + u * kWave] : piece_t{0u, 0u, 0u, 0u};
            }
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int u = 0; u < kSegment; ++u) {
                    float f[V];
                    R::unpack(v[s][u], f);
#pragma unroll
                    for (int i = 0; i < V; ++i) acc[u][i] = WEIGHTED ? fmaf(w[s], f[i], acc[u][i]) : acc[u][i] + f[i];
                }
        }
#pragma unroll
        for (int u = 0; u < kSegment; ++u)
            if (c0 + u * kWave < p.pieces)
                __builtin_nontemporal_store(R::pack(acc[u]), p.out + static_cast<size_t>(t) * p.pieces + c0 + u * kWave);
    }
}

struct UnsortBackwardParams {
    const piece_t* dout; const piece_t* ys; piece_t* dys; float* dgate;
    const float* gate; const int32_t* topk; const int32_t* row_of;
    int T, k, E, pieces, rows, gate_norm;
};

// A team (a wave, or a workgroup where a row is too wide for one) has a token: its row of dout in registers, its rows of ys one
// after the other, the next one requested while the sum of the present one is folded.
template <bool BF16, int TEAM, int NV>
__global__ __launch_bounds__(TEAM < 256 ? 256 : TEAM) void unsort_backward_kernel(UnsortBackwardParams p) {
    using R = Piece<BF16>;
    constexpr int V = R::kN;
    __shared__ TeamLds lds;
    int half = 0;
    const int l = threadIdx.x % TEAM, lane = threadIdx.x & 63, per_block = blockDim.x / TEAM;
    for (long long t = static_cast<long long>(blockIdx.x) * per_block + threadIdx.x / TEAM; t < p.T;
         t += static_cast<long long>(gridDim.x) * per_block) {
        const piece_t zero = {0u, 0u, 0u, 0u};
        const int mine = lane_row(p.row_of, t, p.k, p.rows, lane);
        piece_t up[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) up[i] = l + i * TEAM < p.pieces ? p.dout[static_cast<size_t>(t) * p.pieces + l + i * TEAM] : zero;
        uint64_t left = __ballot(mine >= 0);
        piece_t y[NV];
        auto request = [&](int j) {
            const int row = __builtin_amdgcn_readlane(mine, j);
#pragma unroll
            for (int i = 0; i < NV; ++i) y[i] = l + i * TEAM < p.pieces ? p.ys[static_cast<size_t>(row) * p.pieces + l + i * TEAM] : zero;
        };
        int j = left ? __builtin_ctzll(left) : -1;
        if (j >= 0) request(j);
        int expert;
        Inverse inverse;
        const float weight = lane_weight(p.gate, p.topk, t, p.k, p.E, mine, p.gate_norm, lane, expert, inverse);
        float dweight = 0.f;                                     // lane j: <dout[t], ys[row_tj]>
        while (j >= 0) {
            left &= left - 1;
            const int next = left ? __builtin_ctzll(left) : -1;
            float dot[1] = {0.f};
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                float f[V], g[V];
                R::unpack(up[i], f);
                R::unpack(y[i], g);
#pragma unroll
                for (int q = 0; q < V; ++q) dot[0] = fmaf(f[q], g[q], dot[0]);
            }
            if (next >= 0) request(next);
            const int row = __builtin_amdgcn_readlane(mine, j);
            const float w = lane_value(weight, j);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                if (l + i * TEAM >= p.pieces) continue;
                float f[V];
                R::unpack(up[i], f);
#pragma unroll
                for (int q = 0; q < V; ++q) f[q] *= w;
                __builtin_nontemporal_store(R::pack(f), p.dys + static_cast<size_t>(row) * p.pieces + l + i * TEAM);
            }
            team_sum<TEAM>(dot, lds, half);
            if (lane == j) dweight = dot[0];
            j = next;
        }
        if (TEAM > 64 && threadIdx.x >= 64) continue;            // the first wave has all that is left to do
        if (p.gate_norm) {                                       // w = g / S: d / d g_j = (dw_j - sum_i dw_i w_i) / S
            const float mix = wave_sum(dweight * weight);
            dweight = inverse.of(dweight - mix);
        }
        float dg = 0.f;                                          // lane e
        for (uint64_t m = __ballot(mine >= 0 && expert >= 0); m; m &= m - 1) {
            const int i = __builtin_ctzll(m);
            const float dw = lane_value(dweight, i);
            dg += __builtin_amdgcn_readlane(expert, i) == lane ? dw : 0.f;
        }
        if (lane < p.E) p.dgate[static_cast<size_t>(t) * p.E + lane] = dg;
    }
}

int pieces_of(const etr_sort_config& c) { return static_cast<int>(static_cast<size_t>(c.d) * elt_bytes(c.dtype) / 16); }

int pairs_per_block(const etr_sort_config& c) {
    const int pairs = c.T * c.k;
    if (pairs <= kOnePairs) return kOnePairs;
    const int even = (pairs + kMaxSortBlocks - 1) / kMaxSortBlocks;
    return (std::max(even, kMinPairs) + kSortThreads - 1) / kSortThreads * kSortThreads;
}
int sort_blocks(const etr_sort_config& c) { const int per = pairs_per_block(c); return static_cast<int>((static_cast<long long>(c.T) * c.k + per - 1) / per); }

RowsParams rows_params(const etr_sort_config& c, const void* in, const float* gate, const int32_t* topk, const int32_t* row_of, void* out) {
    RowsParams p{static_cast<const piece_t*>(in), static_cast<piece_t*>(out), gate, topk, row_of, c.T, c.k, c.E, pieces_of(c), c.T * c.k, c.gate_norm, 0};
    p.segments = (p.pieces + kSegment * kWave - 1) / (kSegment * kWave);
    return p;
}
constexpr long long kMostBlocks = 1 << 20;                   // (2^32 threads to a launch)
unsigned row_blocks(const RowsParams& p) {
    return static_cast<unsigned>(std::min((static_cast<long long>(p.T) * p.segments + kRowsWaves - 1) / kRowsWaves, kMostBlocks));
}

template <bool BF16, int TEAM, int NV>
hipError_t launch_unsort_backward_form(const UnsortBackwardParams& p, hipStream_t st) {
    constexpr int threads = TEAM < 256 ? 256 : TEAM, per_block = threads / TEAM;
    hipLaunchKernelGGL((unsort_backward_kernel<BF16, TEAM, NV>), dim3(static_cast<unsigned>(std::min<long long>((p.T + per_block - 1) / per_block, kMostBlocks))), dim3(threads), 0, st, p);
    return hipGetLastError();
}
template <bool BF16>
hipError_t unsort_backward_by_width(const UnsortBackwardParams& p, hipStream_t st) {
    if (p.pieces <= 64) return launch_unsort_backward_form<BF16, 64, 1>(p, st);
    if (p.T <= 2048 && p.pieces > 64 && p.pieces <= 256) return launch_unsort_backward_form<BF16, 256, 1>(p, st);
    if (p.pieces <= 128) return launch_unsort_backward_form<BF16, 64, 2>(p, st);
    if (p.pieces <= 256) return launch_unsort_backward_form<BF16, 64, 4>(p, st);
    if (p.T <= 2048 && p.pieces <= 512) return launch_unsort_backward_form<BF16, 256, 2>(p, st);
    if (p.pieces <= 512) return launch_unsort_backward_form<BF16, 64, 8>(p, st);
    if (p.pieces <= 1024) return launch_unsort_backward_form<BF16, 256, 4>(p, st);
    if (p.pieces <= 2048) return launch_unsort_backward_form<BF16, 256, 8>(p, st);
    return launch_unsort_backward_form<BF16, 1024, 8>(p, st);
}

}  // namespace

size_t sort_ws_bytes(const etr_sort_config& c) { return align_up(static_cast<size_t>(sort_blocks(c)) * c.E * 4); }

hipError_t launch_sort_tokens(const etr_sort_config& c, const int32_t* topk, const int32_t* slot_of, int32_t* offsets, int32_t* row_of,
                              int32_t* pair_of, void* ws, hipStream_t st) {
    SortParams p{topk, slot_of, offsets, row_of, pair_of, static_cast<int32_t*>(ws), c.k, c.E, 0, c.T * c.k, pairs_per_block(c)};
    while ((1 << p.bits) < c.E + 1) ++p.bits;
    const int blocks = sort_blocks(c);
    if (blocks == 1) {
        // the workgroup's waves share what there is in whole rounds of 64 pairs
        p.per_block = (p.pairs + kSortThreads - 1) / kSortThreads * kSortThreads;
        hipLaunchKernelGGL(sort_rank_kernel<true>, dim3(1), dim3(kSortThreads), 0, st, p);
        return hipGetLastError();
    }
    hipLaunchKernelGGL(sort_count_kernel, dim3(blocks), dim3(kSortThreads), 0, st, p);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
    hipLaunchKernelGGL(sort_rank_kernel<false>, dim3(blocks), dim3(kSortThreads), 0, st, p);
    return hipGetLastError();
}

hipError_t launch_sort_rows(const etr_sort_config& c, const void* x, const int32_t* row_of, void* xs, hipStream_t st) {
    const RowsParams p = rows_params(c, x, nullptr, nullptr, row_of, xs);
    hipLaunchKernelGGL(sort_rows_kernel, dim3(row_blocks(p)), dim3(kRowsThreads), 0, st, p);
    return hipGetLastError();
}

hipError_t launch_sort_rows_backward(const etr_sort_config& c, const void* dxs, const int32_t* row_of, void* dx, hipStream_t st) {
    const RowsParams p = rows_params(c, dxs, nullptr, nullptr, row_of, dx);
    auto kern = c.dtype == ETR_BF16 ? gather_sum_kernel<true, false> : gather_sum_kernel<false, false>;
    hipLaunchKernelGGL(kern, dim3(row_blocks(p)), dim3(kRowsThreads), 0, st, p);
    return hipGetLastError();
}

hipError_t launch_unsort_rows(const etr_sort_config& c, const void* ys, const float* gate, const int32_t* topk, const int32_t* row_of,
                              void* out, hipStream_t st) {
    const RowsParams p = rows_params(c, ys, gate, topk, row_of, out);
    auto kern = c.dtype == ETR_BF16 ? gather_sum_kernel<true, true> : gather_sum_kernel<false, true>;
    hipLaunchKernelGGL(kern, dim3(row_blocks(p)), dim3(kRowsThreads), 0, st, p);
    return hipGetLastError();
}

hipError_t launch_unsort_rows_backward(const etr_sort_config& c, const void* dout, const void* ys, const float* gate, const int32_t* topk,
                                       const int32_t* row_of, void* dys, float* dgate, hipStream_t st) {
    const UnsortBackwardParams p{static_cast<const piece_t*>(dout), static_cast<const piece_t*>(ys), static_cast<piece_t*>(dys), dgate, gate,
                                 topk, row_of, c.T, c.k, c.E, pieces_of(c), c.T * c.k, c.gate_norm};
    return c.dtype == ETR_BF16 ? unsort_backward_by_width<true>(p, st) : unsort_backward_by_width<false>(p, st);
}

}  // namespace etr
