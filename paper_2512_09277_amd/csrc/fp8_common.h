// e4m3 with a scale for each block of 128: how a block is quantized.
//   m = max(largest magnitude of the block, 1e-30)    scale = m / 448    q = e4m3(x * (448 / m))
// The divisions and the product are rounded to fp32, so every kernel that quantizes a block gives the same bits.  The floor keeps
// 448 / m finite; a block of zeros has q = 0.  Magnitudes are compared as integers, where NaN is the largest: a block with a NaN has
// scale NaN and q NaN, one with an infinity scale infinity and q NaN in its place.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "mfma_common.h"

namespace metro {
namespace {

constexpr int kBlock = 128;                 // values of a row that share a scale, and rows of a weight block
constexpr float kE4m3Max = 448.f;
constexpr float kSmallest = 1e-30f;

__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

struct BlockScale { float scale, inverse; };
__device__ __forceinline__ BlockScale block_scale(uint32_t largest) {
    const float m = __uint_as_float(max(largest, __float_as_uint(kSmallest)));
    return BlockScale{m / kE4m3Max, kE4m3Max / m};
}

// Four values, |v| <= 448 (1 + 2^-23) or NaN, as e4m3, round to nearest even: nothing rounds past 448, so the conversion's own
// handling of larger values does not matter.
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
    int v = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    v = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, v, true);
    return (uint32_t)v;
}

// Largest over aligned groups of 8 or 16 lanes, in every lane of the group; registers only.
template <int kLanes>
__device__ __forceinline__ uint32_t group_max(uint32_t v) {
    static_assert(kLanes == 8 || kLanes == 16, "");
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xb1, 0xf, 0xf, true));        // quad_perm: lane ^ 1
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4e, 0xf, 0xf, true));        // quad_perm: lane ^ 2
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xf, 0xf, true));       // row_half_mirror: the other quad of 8
    if (kLanes == 16) v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xf, 0xf, true));   // row_mirror: the other 8
    return v;
}

inline __device__ __host__ int64_t up16(int64_t n) { return (n + 15) & ~(int64_t)15; }
inline __device__ __host__ int blocks_of(int n) { return (n + kBlock - 1) / kBlock; }

}  // namespace
}  // namespace metro
