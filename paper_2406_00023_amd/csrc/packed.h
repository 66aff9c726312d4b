// Packed matrices: e4m3 values with a power of two for each block of 128 along the contraction.  Sizes, and the device side of
// packing one block.
#pragma once

#include "row_ops.h"

namespace etr {

constexpr int kBlock = 128;                              // values that share a scale
inline __host__ __device__ int blocks_of(int n) { return (n + kBlock - 1) / kBlock; }
inline __host__ __device__ int scale_groups_of(int n) { return (n + 4 * kBlock - 1) / (4 * kBlock); }   // dwords of scales to a row

// Bytes of matrices of `count` x [rows][K], along rows
inline size_t packed_bytes(size_t count, int K) { return count * static_cast<size_t>(blocks_of(K)) * kBlock; }
inline size_t scale_bytes(size_t count, int K) { return count * 4 * static_cast<size_t>(scale_groups_of(K)); }

namespace {

// The byte of the smallest power of two, 2^-127 at least, by which a magnitude comes to 448 = 1.75 x 2^8 or less.
// (448 has the mantissa 0x600000: what is added carries into the exponent exactly where the mantissa is larger.)
__device__ __forceinline__ uint32_t scale_byte(float top) { return max((__float_as_uint(top) + 0x1FFFFFu) >> 23, 8u) - 8u; }
// 2^(byte - 127); byte 0 is below the normal numbers
__device__ __forceinline__ float scale_value(uint32_t byte) { return __uint_as_float(max(byte << 23, 0x400000u)); }
// magnitude that takes part in a block's largest: NaN and infinities have none
__device__ __forceinline__ float finite_abs(float v) { return fabsf(v) < __builtin_inff() ? fabsf(v) : 0.f; }
// Largest magnitude of what is finite among n values: NaN is no operand to a maximum, and infinities are looked at only where there are any.
template <int N, class F>
__device__ __forceinline__ float top_of(F&& value) {
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) top = fmaxf(top, fabsf(value(i)));
    if (__builtin_expect(__any(top == __builtin_inff()), 0)) {
        top = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) top = fmaxf(top, finite_abs(value(i)));
    }
    return top;
}
// four values divided by their power of two, lowest byte first.  (An infinity stays one under any power, and is converted to NaN, as NaN is;
// what is finite is 448 at most.)
__device__ __forceinline__ uint32_t to_e4m3(float a, float b, float c, float d, float scale) {
    typedef short i16x2 __attribute__((ext_vector_type(2)));
    const i16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(i16x2{0, 0}, a, b, scale, false);
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(lo, c, d, scale, true));
}
// four packed values, times their power of two
__device__ __forceinline__ void from_e4m3(uint32_t v, float scale, float* f) {
    const auto lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(v, scale, false), hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(v, scale, true);
    f[0] = lo[0]; f[1] = lo[1]; f[2] = hi[0]; f[3] = hi[1];
}

// Largest over the 16 lanes of a row of lanes, in all of them.  All lanes active.
__device__ __forceinline__ float row16_max(float v) {
    auto dpp = [](float x, auto ctrl) {
        return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), decltype(ctrl)::value, 0xF, 0xF, true));
    };
    v = fmaxf(v, dpp(v, std::integral_constant<int, 0xB1>{}));       // quad swap 1
    v = fmaxf(v, dpp(v, std::integral_constant<int, 0x4E>{}));       // quad swap 2
    v = fmaxf(v, dpp(v, std::integral_constant<int, 0x141>{}));      // half-row mirror
    return fmaxf(v, dpp(v, std::integral_constant<int, 0x140>{}));   // row mirror
}

// Inclusive running maximum over the 64 lanes of numbers from 0 up, by the moves of wave_scan_incl.  All lanes active.
__device__ __forceinline__ int wave_max_incl(int v) {
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false));   // row_shr:1
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false));   // row_shr:2
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false));   // row_shr:4
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false));   // row_shr:8
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false));   // row_bcast:15 -> rows 1, 3
    return max(v, __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false));   // row_bcast:31 -> rows 2, 3
}

// Rows of the groups, one group per lane, for operands whose groups lie one behind the other: the offsets' running maximum, so that
// the groups' rows are `rows` in all whatever the offsets say.  blocks: of 128 rows, a last one in part; groups: of four blocks, whose scales
// are a dword; _incl: those of the groups before and of this one.
struct Segments {
    int first, count, blocks, blocks_incl, groups, groups_incl;
    __device__ __forceinline__ void load(const int32_t* offsets, int rows, int E, bool stacked) {
        const int lane = threadIdx.x & 63;
        int end = 0;
        if (stacked) {
            first = lane < E ? lane * rows : 0;
            count = lane < E ? rows : 0;
        } else {
            int begin = lane < E && offsets ? min(max(offsets[lane], 0), rows) : 0;
            end = lane < E ? (offsets ? min(max(offsets[lane + 1], 0), rows) : rows) : 0;
            begin = wave_max_incl(begin);
            end = max(begin, wave_max_incl(end));
            first = begin;
            count = lane < E ? end - begin : 0;
        }
        blocks = (count + kBlock - 1) / kBlock;
        groups = (blocks + 3) / 4;
        blocks_incl = wave_scan_incl(blocks);
        groups_incl = wave_scan_incl(groups);
    }
};

}  // namespace
}  // namespace etr
