// The join of a block's output with the residual stream and the RMS norm in front of the next block, forward and backward:
//   x' = rs x + bs gate[t] N(y) w_post,   h = N(x') w_pre,   N(v) = v inv(v),  inv(v) = 1 / sqrt(mean v^2 + eps)
// and, with r = dx' + dN(x')^T (dh w_pre),
//   dN(v)^T u = inv (u - v inv^2 mean(u v))
//   dx = rs r;  dgate = bs <r, N(y) w_post>;  dy = dN(y)^T (bs gate r w_post);  dw_post = sum_t bs gate r N(y);  dw_pre = sum_t dh N(x')
// Bound by memory: two rows in and two out per token forward, four in and two out backward.  So every row crosses once: a
// team of threads (a wave, or a workgroup) holds a token's rows in registers between the sums and their use, all loads of a
// token are requested before the first is waited for, and nothing is kept from the forward: the backward has the rows in
// its hands anyway and takes their sums of squares again.  Measured: 32768 x 4096 bf16, everything at once, forward 207 us (5.2 TB/s),
// backward 333 (4.8; a large copy 4.9) and the weights' sums 8; 3001 x 1080 fp32 without the norm behind the block 10, 21 and 4; 32768 x 2048
// fp32 forward 209 (5.1 TB/s).  Rows of more than 8192 values spill in the backward (bf16 from 16392 on 138 registers: 2048 x 32768, both ways,
// 615 us for 247 of bytes).
#include <algorithm>

#include "row_ops.h"

namespace etr {
namespace {

struct NormParams {
    const piece_t* x; const piece_t* y; const float* gate; const float* w_post; const float* w_pre;
    piece_t* x_out; piece_t* h;
    int T, pieces;
    float inv_d, eps, rs, bs;
};

template <int N>
__device__ __forceinline__ void load_weights(const float* w, int c, float (&f)[N]) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
        const float4 v = *reinterpret_cast<const float4*>(w + static_cast<size_t>(c) * N + i);
        f[i] = v.x; f[i + 1] = v.y; f[i + 2] = v.z; f[i + 3] = v.w;
    }
}

template <bool BF16, int TEAM, int NV>
__global__ __launch_bounds__(TEAM < 256 ? 256 : TEAM) void block_norm_kernel(NormParams p) {
    using R = Piece<BF16>;
    constexpr int V = R::kN;
    __shared__ TeamLds lds;
    int half = 0;
    const int l = threadIdx.x % TEAM, per_block = blockDim.x / TEAM;
    for (long long t = static_cast<long long>(blockIdx.x) * per_block + threadIdx.x / TEAM; t < p.T; t += static_cast<long long>(gridDim.x) * per_block) {
        const size_t row = static_cast<size_t>(t) * p.pieces;
        piece_t s[NV], y[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = l + i * TEAM;
            s[i] = c < p.pieces ? p.x[row + c] : piece_t{0u, 0u, 0u, 0u};
            if (p.y) y[i] = c < p.pieces ? p.y[row + c] : piece_t{0u, 0u, 0u, 0u};
        }
        if (p.y) {
            float w = p.bs * (p.gate ? p.gate[t] : 1.0f);
            if (p.w_post) {
                float sum[1] = {0.f};
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    float f[V];
                    R::unpack(y[i], f);
#pragma unroll
                    for (int j = 0; j < V; ++j) sum[0] = fmaf(f[j], f[j], sum[0]);
                }
                team_sum<TEAM>(sum, lds, half);
                w *= 1.0f / sqrtf(sum[0] * p.inv_d + p.eps);
            }
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = l + i * TEAM;
                if (c >= p.pieces) continue;
                float f[V], g[V], o[V];
                R::unpack(y[i], f);
                R::unpack(s[i], o);
                if (p.w_post) load_weights(p.w_post, c, g);
#pragma unroll
                for (int j = 0; j < V; ++j) o[j] = fmaf(p.rs, o[j], w * (p.w_post ? f[j] * g[j] : f[j]));
                s[i] = R::pack(o);                       // the stream as it is stored is what the norm below reads
                p.x_out[row + c] = s[i];
            }
        }
        if (p.w_pre) {
            float sum[1] = {0.f};
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                float f[V];
                R::unpack(s[i], f);
#pragma unroll
                for (int j = 0; j < V; ++j) sum[0] = fmaf(f[j], f[j], sum[0]);
            }
            team_sum<TEAM>(sum, lds, half);
            const float inv = 1.0f / sqrtf(sum[0] * p.inv_d + p.eps);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = l + i * TEAM;
                if (c >= p.pieces) continue;
                float f[V], g[V];
                R::unpack(s[i], f);
                load_weights(p.w_pre, c, g);
#pragma unroll
                for (int j = 0; j < V; ++j) f[j] = f[j] * inv * g[j];
                p.h[row + c] = R::pack(f);
            }
        }
    }
}

struct NormBackwardParams {
    const piece_t* s; const piece_t* y; const float* gate; const float* w_post; const float* w_pre;
    const piece_t* dx_out; const piece_t* dh;
    piece_t* dx; piece_t* dy; float* dgate;
    float* part_post; float* part_pre;       // [workgroups][d] `stride` apart, each optional: partial sums of dw_post and dw_pre
    size_t stride;
    int T, pieces;
    float inv_d, eps, rs, bs;
};

// Backward: one workgroup per token at a time, walking on in steps of the grid; the weights' gradients stay in its registers until the end.
template <bool BF16, int TEAM, int NV>
__global__ __launch_bounds__(TEAM) void block_norm_backward_kernel(NormBackwardParams p) {
    using R = Piece<BF16>;
    constexpr int V = R::kN;
    __shared__ TeamLds lds;
    int half = 0;
    const int l = threadIdx.x;
    const piece_t zero = {0u, 0u, 0u, 0u};
    float acc_post[NV][V], acc_pre[NV][V];
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) acc_post[i][j] = acc_pre[i][j] = 0.f;
    for (long long t = blockIdx.x; t < p.T; t += gridDim.x) {
        const size_t row = static_cast<size_t>(t) * p.pieces;
        piece_t s[NV], y[NV], up[NV], dh[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = l + i * TEAM;
            const bool in = c < p.pieces;
            up[i] = in && p.dx_out ? p.dx_out[row + c] : zero;
            y[i] = in && p.y ? p.y[row + c] : zero;
            s[i] = in && p.w_pre ? p.s[row + c] : zero;
            dh[i] = in && p.w_pre ? p.dh[row + c] : zero;
        }
        // sums over the row: s^2 and <dh w_pre, s> of the norm behind the join, y^2 of the one before it
        float sum[3] = {0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = l + i * TEAM;
            float f[V];
            if (p.w_pre && c < p.pieces) {
                float u[V], g[V];
                R::unpack(s[i], f);
                R::unpack(dh[i], u);
                load_weights(p.w_pre, c, g);
#pragma unroll
                for (int j = 0; j < V; ++j) { sum[0] = fmaf(f[j], f[j], sum[0]); sum[1] = fmaf(u[j] * g[j], f[j], sum[1]); }
            }
            if (p.w_post) {
                R::unpack(y[i], f);
#pragma unroll
                for (int j = 0; j < V; ++j) sum[2] = fmaf(f[j], f[j], sum[2]);
            }
        }
        team_sum<TEAM>(sum, lds, half);
        const float inv = 1.0f / sqrtf(sum[0] * p.inv_d + p.eps), mean = sum[1] * p.inv_d * inv * inv;
        const float inv_y = p.w_post ? 1.0f / sqrtf(sum[2] * p.inv_d + p.eps) : 1.0f;
        const float w = p.bs * (p.gate ? p.gate[t] : 1.0f);
        float dot[1] = {0.f};                            // <r, y w_post>
        float r[NV][V];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = l + i * TEAM;
            R::unpack(up[i], r[i]);
            if (c >= p.pieces) continue;
            float f[V], u[V], g[V];
            if (p.w_pre) {
                R::unpack(s[i], f);
                R::unpack(dh[i], u);
                load_weights(p.w_pre, c, g);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    r[i][j] += inv * (u[j] * g[j] - f[j] * mean);
                    acc_pre[i][j] = fmaf(u[j], f[j] * inv, acc_pre[i][j]);
                }
            }
#pragma unroll
            for (int j = 0; j < V; ++j) f[j] = (p.y ? p.rs : 1.0f) * r[i][j];
            p.dx[row + c] = R::pack(f);
            if (!p.y) continue;
            R::unpack(y[i], f);
            if (p.w_post) load_weights(p.w_post, c, g);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float rg = p.w_post ? r[i][j] * g[j] : r[i][j];
                dot[0] = fmaf(rg, f[j], dot[0]);
                acc_post[i][j] = fmaf(w * r[i][j], f[j] * inv_y, acc_post[i][j]);
            }
        }
        if (!p.y) continue;                              // (uniform)
        if (p.w_post || p.dgate) team_sum<TEAM>(dot, lds, half);
        if (p.dgate && l == 0) p.dgate[t] = p.bs * inv_y * dot[0];
        const float mean_y = dot[0] * p.inv_d * inv_y * inv_y;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = l + i * TEAM;
            if (c >= p.pieces) continue;
            float f[V], g[V];
            R::unpack(y[i], f);
            if (p.w_post) load_weights(p.w_post, c, g);
#pragma unroll
            for (int j = 0; j < V; ++j) f[j] = p.w_post ? w * inv_y * (r[i][j] * g[j] - f[j] * mean_y) : w * r[i][j];
            p.dy[row + c] = R::pack(f);
        }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = l + i * TEAM;
        if (c >= p.pieces) continue;
        const size_t at = blockIdx.x * p.stride + static_cast<size_t>(c) * V;
#pragma unroll
        for (int j = 0; j < V; j += 4) {
            if (p.part_post) *reinterpret_cast<float4*>(p.part_post + at + j) = make_float4(acc_post[i][j], acc_post[i][j + 1], acc_post[i][j + 2], acc_post[i][j + 3]);
            if (p.part_pre) *reinterpret_cast<float4*>(p.part_pre + at + j) = make_float4(acc_pre[i][j], acc_pre[i][j + 1], acc_pre[i][j + 2], acc_pre[i][j + 3]);
        }
    }
}

// Column sums of the workgroups' partial sums: 8 float4 columns by 128 row groups, joined in LDS in a fixed order.
constexpr int kSumCols = 8, kSumGroups = 128;
__global__ __launch_bounds__(kSumCols* kSumGroups) void norm_weight_sum_kernel(const float* __restrict__ part, int n_part, int width, int d,
                                                                               float* __restrict__ first, float* __restrict__ second) {
    __shared__ float4 lds[kSumGroups][kSumCols];
    const int col = threadIdx.x % kSumCols, group = threadIdx.x / kSumCols, c4 = blockIdx.x * kSumCols + col;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (c4 * 4 < width)
        for (int i = group; i < n_part; i += kSumGroups) {
            const float4 v = *reinterpret_cast<const float4*>(part + static_cast<size_t>(i) * width + c4 * 4);
            s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
        }
    lds[group][col] = s;
    for (int n = kSumGroups / 2; n >= 1; n >>= 1) {
        __syncthreads();
        if (group < n) {
            const float4 v = lds[group + n][col];
            s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
            lds[group][col] = s;
        }
    }
    if (group == 0 && c4 * 4 < width) {
        float* out = c4 * 4 < d && first ? first + c4 * 4 : second + c4 * 4 - (first ? d : 0);
        *reinterpret_cast<float4*>(out) = s;
    }
}

int pieces_of(const etr_norm_config& c) { return static_cast<int>(static_cast<size_t>(c.d) * elt_bytes(c.dtype) / 16); }

// Workgroups of the backward: whole rounds of the chip, at least four tokens to a workgroup where there are enough, so
// that the partial sums stay small beside the rows.
int backward_groups(const etr_norm_config& c) {
    const int most = 256 * 4;
    const int groups = c.T / 4 + (c.T % 4 != 0);         // (T + 3 may not fit 32 bits)
    return groups < most ? groups : most;
}

template <bool BF16, int TEAM, int NV>
hipError_t launch_forward(const NormParams& p, hipStream_t st) {
    constexpr int threads = TEAM < 256 ? 256 : TEAM;
    const long long rows_per = threads / TEAM;
    const long long blocks = std::min<long long>((p.T + rows_per - 1) / rows_per, 1 << 20);     // (2^32 threads to a launch)
    hipLaunchKernelGGL((block_norm_kernel<BF16, TEAM, NV>), dim3(static_cast<unsigned>(blocks)), dim3(threads), 0, st, p);
    return hipGetLastError();
}
template <bool BF16, int TEAM>
hipError_t forward_by_width(const NormParams& p, hipStream_t st) {
    if (p.pieces <= TEAM) return launch_forward<BF16, TEAM, 1>(p, st);
    if (p.pieces <= 2 * TEAM) return launch_forward<BF16, TEAM, 2>(p, st);
    if (p.pieces <= 4 * TEAM) return launch_forward<BF16, TEAM, 4>(p, st);
    return launch_forward<BF16, TEAM, 8>(p, st);
}
// A wave holds a row of up to 512 pieces (4096 bf16) without a barrier for its sums; a workgroup holds wider ones, and narrower ones where the
// tokens are too few to fill the chip with waves (32 x 2048: 3.0 us).
template <bool BF16>
hipError_t forward_by_team(const NormParams& p, hipStream_t st) {
    if (p.pieces <= 64 || (p.pieces <= 64 * 8 && p.T > 2048)) return forward_by_width<BF16, 64>(p, st);
    if (p.pieces <= 256 * 8) return forward_by_width<BF16, 256>(p, st);
    return launch_forward<BF16, 1024, 4>(p, st);
}

template <bool BF16, int TEAM, int NV>
hipError_t launch_backward(const NormBackwardParams& p, int groups, hipStream_t st) {
    hipLaunchKernelGGL((block_norm_backward_kernel<BF16, TEAM, NV>), dim3(groups), dim3(TEAM), 0, st, p);
    return hipGetLastError();
}
template <bool BF16>
hipError_t backward_by_width(const NormBackwardParams& p, int groups, hipStream_t st) {
    if (p.pieces <= 64) return launch_backward<BF16, 64, 1>(p, groups, st);
    if (p.pieces <= 256) return launch_backward<BF16, 256, 1>(p, groups, st);
    if (p.pieces <= 512) return launch_backward<BF16, 256, 2>(p, groups, st);
    if (p.pieces <= 1024) return launch_backward<BF16, 256, 4>(p, groups, st);
    if (p.pieces <= 2048) return launch_backward<BF16, 1024, 2>(p, groups, st);
    return launch_backward<BF16, 1024, 4>(p, groups, st);
}

}  // namespace

size_t norm_ws_bytes(const etr_norm_config& c) { return align_up(static_cast<size_t>(backward_groups(c)) * 2 * c.d * 4); }

hipError_t launch_block_norm(const etr_norm_config& c, const void* x, const void* y, const float* gate, const float* w_post,
                             const float* w_pre, void* x_out, void* h, hipStream_t st) {
    const NormParams p{static_cast<const piece_t*>(x), static_cast<const piece_t*>(y), gate, w_post, w_pre,
                       static_cast<piece_t*>(x_out), static_cast<piece_t*>(h), c.T, pieces_of(c), 1.0f / c.d, c.eps,
                       c.residual_scale, c.block_scale};
    return c.dtype == ETR_BF16 ? forward_by_team<true>(p, st) : forward_by_team<false>(p, st);
}

hipError_t launch_block_norm_backward(const etr_norm_config& c, const void* x_out, const void* y, const float* gate,
                                      const float* w_post, const float* w_pre, const void* dx_out, const void* dh, void* dx,
                                      void* dy, float* dgate, float* dw_post, float* dw_pre, void* ws, hipStream_t st) {
    const int groups = backward_groups(c), want = (dw_post != nullptr) + (dw_pre != nullptr);
    float* part = static_cast<float*>(ws);
    const bool one = groups == 1;                        // its sums are the results
    const NormBackwardParams p{static_cast<const piece_t*>(x_out), static_cast<const piece_t*>(y), gate, w_post, w_pre,
                               static_cast<const piece_t*>(dx_out), static_cast<const piece_t*>(dh), static_cast<piece_t*>(dx),
                               static_cast<piece_t*>(dy), dgate, one || !dw_post ? dw_post : part, one || !dw_pre ? dw_pre : part + (dw_post ? c.d : 0),
                               static_cast<size_t>(want) * c.d,
                               c.T, pieces_of(c), 1.0f / c.d, c.eps, c.residual_scale, c.block_scale};
    const hipError_t err = c.dtype == ETR_BF16 ? backward_by_width<true>(p, groups, st) : backward_by_width<false>(p, groups, st);
    if (err != hipSuccess || want == 0 || one) return err;
    const int width = want * c.d;
    hipLaunchKernelGGL(norm_weight_sum_kernel, dim3((width / 4 + kSumCols - 1) / kSumCols), dim3(kSumCols * kSumGroups), 0, st,
                       static_cast<const float*>(ws), groups, width, c.d, dw_post, dw_pre);
    return hipGetLastError();
}

}  // namespace etr
