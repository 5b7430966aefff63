// A vector of kN columns of one row, 16 bytes or a single element: bf16 or fp32 in memory, fp32 in registers.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace metro {
namespace {

__device__ __forceinline__ float bf16_bits_to_f32(uint32_t bits16) { return __uint_as_float(bits16 << 16); }
__device__ __forceinline__ uint32_t f32_to_bf16_bits(float v) {
    uint32_t u = __float_as_uint(v);
    if (v != v) return (u >> 16) | 0x0040u;   // NaN stays a (quiet) NaN: the rounding add could carry it into Inf or -0
    u += 0x7fffu + ((u >> 16) & 1u);          // round to nearest even
    return u >> 16;
}

template <bool kBf16, int kN>
struct RowVec {
    static_assert(kN == 1 || kN == (kBf16 ? 8 : 4), "an element or 16 bytes");
    using Raw = std::conditional_t<kN == 1, std::conditional_t<kBf16, uint16_t, uint32_t>, uint4>;

    static __device__ __forceinline__ Raw load(const void* p, size_t i) { return reinterpret_cast<const Raw*>(p)[i]; }
    static __device__ __forceinline__ void store(void* p, size_t i, const Raw& v) { reinterpret_cast<Raw*>(p)[i] = v; }
    static __device__ __forceinline__ void widen(const Raw& v, float (&f)[kN]) {
        if constexpr (kN == 1) {
            f[0] = kBf16 ? bf16_bits_to_f32(v) : __uint_as_float(v);
        } else {
            const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (kBf16) {
                    f[2 * i] = bf16_bits_to_f32(u[i] & 0xffffu);
                    f[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
                } else {
                    f[i] = __uint_as_float(u[i]);
                }
            }
        }
    }
    static __device__ __forceinline__ Raw narrow(const float (&f)[kN]) {
        if constexpr (kN == 1) {
            return (Raw)(kBf16 ? f32_to_bf16_bits(f[0]) : __float_as_uint(f[0]));
        } else {
            uint32_t o[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (kBf16) o[i] = f32_to_bf16_bits(f[2 * i]) | (f32_to_bf16_bits(f[2 * i + 1]) << 16);
                else o[i] = __float_as_uint(f[i]);
            }
            return make_uint4(o[0], o[1], o[2], o[3]);
        }
    }
};

}  // namespace
}  // namespace metro
