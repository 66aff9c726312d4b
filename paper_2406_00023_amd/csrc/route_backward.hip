// Gradient of the routing (pooled affinities, cosine, softmax) with respect to the tokens, by itself:
//   ds[e] = gate[e] (dgate[e] - <dgate, gate>),  b = sum_e ds[e] score[e],  u[p] = sum_e ds[e] w_e[p] / |w_e|
//   FULL:   dx_j = u[p(j)] / (sqrt(D) |x|) - b x_j / |x|^2
//   POOLED: dx_j = (u[p(j)] / |g| - b g[p(j)] / |g|^2) / D,  g = means over the groups
// and dx_add joined to it.  Bound by memory (two rows in, one out), so a wave holds its token's row in registers between
// its norm and its use; the embeddings, divided by their norms, lie in LDS for all waves of a workgroup, and u passes through
// LDS from the lanes that have the groups to those that have their 16-byte pieces.  Measured: 65536 x 4096 bf16, 64 experts of 64 pooled
// features 319 us (5.2 TB/s), pooled 329; 32768 x 2048 fp32, 32 experts of 64, 155 and pooled 162 (5.2); 213 x 5120 fp32, 64 experts of 80, whose
// rows come twice, 21 us (element by element 58); 512 x 256 fp32, 8 experts, 3.2 us.  Element by element: 32768 x 1536 bf16 in groups of 12, 208
// us for 63 of bytes, pooled in groups of 24 434.
#include <algorithm>
#include <cmath>

#include "row_ops.h"

namespace etr {
namespace {

struct RouteBackwardParams {
    const void* x; const float* w_emb; const float* score; const float* gate; const float* dgate; const void* dx_add; void* dx;
    int T, d, E, D, P, pieces, full;
};

// unit[e][p] = w_e[p] / |w_e| (0 for a zero embedding): one wave per embedding
__device__ __forceinline__ void stage_units(const RouteBackwardParams& p, float* unit) {
    const int lane = threadIdx.x & 63, waves = blockDim.x >> 6;
    for (int e = threadIdx.x >> 6; e < p.E; e += waves) {
        float s = 0.f;
        for (int q = lane; q < p.P; q += 64) {
            const float f = p.w_emb[static_cast<size_t>(e) * p.P + q];
            unit[e * p.P + q] = f;
            s = fmaf(f, f, s);
        }
        s = wave_sum(s);
        const float inv = s > 0.f ? 1.0f / sqrtf(s) : 0.f;
        for (int q = lane; q < p.P; q += 64) unit[e * p.P + q] *= inv;       // (the lane's own words)
    }
    __syncthreads();
}

// softmax backward of one token, lane = expert: ds, and b in all lanes
__device__ __forceinline__ float score_gradient(const RouteBackwardParams& p, size_t t, int lane, float& b) {
    float dg = 0.f, g = 0.f, sc = 0.f;
    if (lane < p.E) {
        dg = p.dgate[t * p.E + lane];
        g = p.gate[t * p.E + lane];
        sc = p.score[t * p.E + lane];
    }
    const float ds = g * (dg - wave_sum(dg * g));
    b = wave_sum(ds * sc);
    return ds;
}

// Groups of whole 16-byte pieces (D a multiple of a piece; POOLED: as many pieces to a group as a power of two).  A row of up to 64 NV
// pieces stays in registers; with WIDE it comes in parts of that size, twice.
template <bool BF16, int NV, bool WIDE>
__global__ __launch_bounds__(1024) void route_backward_kernel(RouteBackwardParams p) {
    using R = Piece<BF16>;
    constexpr int V = R::kN;
    extern __shared__ float sm[];
    float* unit = sm;                                        // [E][P]
    float* u = sm + p.E * p.P + (threadIdx.x >> 6) * p.P;    // [P] per wave
    const int lane = threadIdx.x & 63, per_group = p.D / V;
    stage_units(p, unit);
    const piece_t* x = static_cast<const piece_t*>(p.x);
    const piece_t* add = static_cast<const piece_t*>(p.dx_add);
    const piece_t zero = {0u, 0u, 0u, 0u};
    const int waves = blockDim.x >> 6;
    auto group_sum = [&](float s) {                          // over the lanes that share a group
        for (int o = 1; o < per_group; o <<= 1) s += __shfl_xor(s, o, 64);
        return s;
    };
    for (long long t = static_cast<long long>(blockIdx.x) * waves + (threadIdx.x >> 6); t < p.T; t += static_cast<long long>(gridDim.x) * waves) {
        const size_t row = static_cast<size_t>(t) * p.pieces;
        piece_t xv[NV], av[NV];
        auto load = [&](piece_t (&v)[NV], const piece_t* from, int c0) {
#pragma unroll
            for (int i = 0; i < NV; ++i) v[i] = from && c0 + lane + i * 64 < p.pieces ? from[row + c0 + lane + i * 64] : zero;
        };
        load(xv, x, 0);
        if (!WIDE) load(av, add, 0);
        float b;
        const float ds = score_gradient(p, t, lane, b);
        for (int q = lane; q < p.P; q += 64) {
            float s = 0.f;
#pragma unroll 4
            for (int e = 0; e < p.E; ++e) s = fmaf(lane_value(ds, e), unit[e * p.P + q], s);
            u[q] = s;
        }
        float square = 0.f, mean[NV];
        for (int c0 = 0; c0 < (WIDE ? p.pieces : 1); c0 += 64 * NV) {
            if (WIDE && c0) load(xv, x, c0);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                float f[V], s = 0.f;
                R::unpack(xv[i], f);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    if (p.full) square = fmaf(f[j], f[j], square);
                    else s += f[j];
                }
                if (!p.full) {
                    mean[i] = group_sum(s) / p.D;
                    square = fmaf(mean[i], mean[i], square);                 // (counted by each of the group's lanes)
                }
            }
        }
        square = wave_sum(square);
        if (!p.full) square /= per_group;
        const float inv = square > 0.f ? 1.0f / sqrtf(square) : 0.f;
        const float cu = p.full ? inv / sqrtf(static_cast<float>(p.D)) : inv / p.D;
        const float cx = square > 0.f ? b / square * (p.full ? 1.0f : 1.0f / p.D) : 0.f;
        wave_sync();
        for (int c0 = 0; c0 < (WIDE ? p.pieces : 1); c0 += 64 * NV) {
            if (WIDE) {
                load(xv, x, c0);
                load(av, add, c0);
            }
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = c0 + lane + i * 64;
                float f[V], a[V];
                R::unpack(xv[i], f);
                R::unpack(av[i], a);
                if (WIDE && !p.full) {
                    float s = 0.f;
#pragma unroll
                    for (int j = 0; j < V; ++j) s += f[j];
                    mean[i] = group_sum(s) / p.D;
                }
                if (c >= p.pieces) continue;
                const float uc = u[c / per_group] * cu;
#pragma unroll
                for (int j = 0; j < V; ++j) a[j] += uc - cx * (p.full ? f[j] : mean[i]);
                __builtin_nontemporal_store(R::pack(a), static_cast<piece_t*>(p.dx) + row + c);
            }
        }
        wave_sync();                                         // u is written again by the next token
    }
}

// Any group size and width: a lane has whole groups, element by element.
template <bool BF16>
__global__ __launch_bounds__(256) void route_backward_groups_kernel(RouteBackwardParams p) {
    extern __shared__ float unit[];                          // [E][P]
    const int lane = threadIdx.x & 63, waves = blockDim.x >> 6;
    stage_units(p, unit);
    auto load = [&](const void* v, size_t i) -> float {
        if constexpr (BF16) return __uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t*>(v)[i]) << 16);
        else return static_cast<const float*>(v)[i];
    };
    for (long long t = static_cast<long long>(blockIdx.x) * waves + (threadIdx.x >> 6); t < p.T; t += static_cast<long long>(gridDim.x) * waves) {
        const size_t row = static_cast<size_t>(t) * p.d;
        float b;
        const float ds = score_gradient(p, t, lane, b);
        auto group_mean = [&](int q) {
            float s = 0.f;
            for (int j = 0; j < p.D; ++j) s += load(p.x, row + static_cast<size_t>(q) * p.D + j);
            return s / p.D;
        };
        float square = 0.f;
        for (int q = lane; q < p.P; q += 64) {
            if (p.full) {
                for (int j = 0; j < p.D; ++j) { const float f = load(p.x, row + static_cast<size_t>(q) * p.D + j); square = fmaf(f, f, square); }
            } else {
                const float m = group_mean(q);
                square = fmaf(m, m, square);
            }
        }
        square = wave_sum(square);
        const float inv = square > 0.f ? 1.0f / sqrtf(square) : 0.f;
        const float cu = p.full ? inv / sqrtf(static_cast<float>(p.D)) : inv / p.D;
        const float cx = square > 0.f ? b / square * (p.full ? 1.0f : 1.0f / p.D) : 0.f;
        for (int q0 = 0; q0 < p.P; q0 += 64) {               // (all lanes stay active for lane_value)
            const int q = q0 + lane;
            float s = 0.f;
            for (int e = 0; e < p.E; ++e) {
                const float v = lane_value(ds, e);
                s = fmaf(v, q < p.P ? unit[e * p.P + q] : 0.f, s);
            }
            if (q >= p.P) continue;
            const float uc = s * cu, m = p.full ? 0.f : group_mean(q);
            for (int j = 0; j < p.D; ++j) {
                const size_t at = row + static_cast<size_t>(q) * p.D + j;
                const float v = (p.dx_add ? load(p.dx_add, at) : 0.f) + (uc - cx * (p.full ? load(p.x, at) : m));
                if constexpr (BF16) static_cast<__bf16*>(p.dx)[at] = static_cast<__bf16>(v);
                else static_cast<float*>(p.dx)[at] = v;
            }
        }
    }
}

template <bool BF16, int NV, bool WIDE = false>
hipError_t launch_pieces(const RouteBackwardParams& p, int waves, size_t lds, hipStream_t st) {
    const void* kern = reinterpret_cast<const void*>(route_backward_kernel<BF16, NV, WIDE>);
    const hipError_t err = ensure_dynamic_lds(kern, lds);
    if (err != hipSuccess) return err;
    // as many workgroups as are resident together (16 waves to a CU at this kernel's registers, or what the LDS holds)
    const long long resident = static_cast<long long>(cu_count()) * std::max<long long>(1, std::min<long long>(16 / waves, (160 * 1024) / static_cast<long long>(lds)));
    const long long blocks = std::min(resident, (static_cast<long long>(p.T) + waves - 1) / waves);
    hipLaunchKernelGGL((route_backward_kernel<BF16, NV, WIDE>), dim3(static_cast<unsigned>(blocks)), dim3(waves * 64), lds, st, p);
    return hipGetLastError();
}
template <bool BF16>
hipError_t launch_typed(const RouteBackwardParams& p, hipStream_t st) {
    constexpr int V = Piece<BF16>::kN;
    const int per_group = p.D / V;
    const size_t embeddings = static_cast<size_t>(p.E) * p.P * 4, row = static_cast<size_t>(p.P) * 4;
    // four waves share a copy of the embeddings, more where fewer copies fit a CU
    int waves = embeddings > 64 * 1024 ? 16 : embeddings > 32 * 1024 ? 8 : 4;
    while (waves > 1 && embeddings + waves * row > 160 * 1024) waves /= 2;
    const bool whole = p.D % V == 0 && (p.full || (per_group <= 64 && (per_group & (per_group - 1)) == 0));
    if (whole && embeddings + waves * row <= 160 * 1024) {
        const size_t lds = embeddings + waves * row;
        if (p.pieces <= 64) return launch_pieces<BF16, 1>(p, waves, lds, st);
        if (p.pieces <= 128) return launch_pieces<BF16, 2>(p, waves, lds, st);
        if (p.pieces <= 256) return launch_pieces<BF16, 4>(p, waves, lds, st);
        if (p.pieces <= 512) return launch_pieces<BF16, 8>(p, waves, lds, st);
        return launch_pieces<BF16, 8, true>(p, waves, lds, st);
    }
    const hipError_t err = ensure_dynamic_lds(reinterpret_cast<const void*>(route_backward_groups_kernel<BF16>), embeddings);
    if (err != hipSuccess) return err;
    const long long blocks = std::min<long long>(static_cast<long long>(cu_count()) * 4, (static_cast<long long>(p.T) + 3) / 4);
    hipLaunchKernelGGL(route_backward_groups_kernel<BF16>, dim3(static_cast<unsigned>(blocks)), dim3(256), embeddings, st, p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_route_backward(const etr_config& c, const void* x, const float* w_emb, const float* score, const float* gate,
                                 const float* dgate, const void* dx_add, void* dx, hipStream_t st) {
    const RouteBackwardParams p{x, w_emb, score, gate, dgate, dx_add, dx, c.T, c.d, c.E, c.D, c.d / c.D,
                                static_cast<int>(static_cast<size_t>(c.d) * elt_bytes(c.dtype) / 16), c.cos == ETR_COS_FULL};
    return c.dtype == ETR_BF16 ? launch_typed<true>(p, st) : launch_typed<false>(p, st);
}

}  // namespace etr
