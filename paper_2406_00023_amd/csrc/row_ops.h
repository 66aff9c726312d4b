// Device helpers of the row kernels (block norm, sorted rows, router gradient): 16-byte pieces of a row in either storage
// type, and sums over the team of threads that holds a row.
#pragma once

#include <type_traits>

#include "etr_internal.h"

namespace etr {

typedef unsigned int piece_t __attribute__((ext_vector_type(4)));       // 16 bytes of a row

template <bool BF16> struct Piece;
template <> struct Piece<false> {
    static constexpr int kN = 4;            // elements of a piece
    __device__ static void unpack(const piece_t& v, float* f) {
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(v[i]);
    }
    __device__ static piece_t pack(const float* f) {
        return piece_t{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
    }
};
template <> struct Piece<true> {
    static constexpr int kN = 8;
    __device__ static void unpack(const piece_t& v, float* f) {
#pragma unroll
        for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(v[i] << 16); f[2 * i + 1] = __uint_as_float(v[i] & 0xFFFF0000u); }
    }
    __device__ static piece_t pack(const float* f) {                     // round to nearest even (v_cvt_pk_bf16_f32)
        typedef __attribute__((ext_vector_type(2))) float f32x2;
        typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
        piece_t v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{f[2 * i], f[2 * i + 1]}, bf16x2));
        return v;
    }
};

// LDS that the lanes of one wave pass to each other: what was written before is seen behind it (no instruction of its own).
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}
__device__ __forceinline__ float lane_value(float v, int lane) {          // lane: uniform
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
}

// Sum over the 64 lanes of a wave, the same in all of them; fixed order.  All lanes active.
__device__ __forceinline__ float wave_sum(float v) {
    auto dpp = [](float x, auto ctrl) {
        return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), decltype(ctrl)::value, 0xF, 0xF, true));
    };
    v += dpp(v, std::integral_constant<int, 0xB1>{});        // quad swap 1
    v += dpp(v, std::integral_constant<int, 0x4E>{});        // quad swap 2
    v += dpp(v, std::integral_constant<int, 0x141>{});       // half-row mirror
    v += dpp(v, std::integral_constant<int, 0x140>{});       // row mirror: sums of 16 lanes
    return (lane_value(v, 0) + lane_value(v, 16)) + (lane_value(v, 32) + lane_value(v, 48));
}

// The same over a team of TEAM threads: a wave, or a whole workgroup.  `half` says which half of the LDS room is next: a half is
// written again only two sums later, behind the barrier of the other one, so one barrier per sum is enough.
constexpr int kTeamSums = 4;
struct TeamLds { float part[2][kTeamSums][16]; };
template <int TEAM, int N>
__device__ __forceinline__ void team_sum(float (&v)[N], TeamLds& lds, int& half) {
    static_assert(N <= kTeamSums, "");
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = wave_sum(v[i]);
    if constexpr (TEAM > 64) {
        constexpr int W = TEAM / 64;
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) lds.part[half][i][threadIdx.x >> 6] = v[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float s = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w) s += lds.part[half][i][w];
            v[i] = s;
        }
        half ^= 1;
    }
}

}  // namespace etr
