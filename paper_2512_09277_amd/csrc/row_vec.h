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

// Memory at any element alignment; the hardware takes unaligned 128-bit global accesses.
typedef uint32_t u32x4_vec __attribute__((ext_vector_type(4)));
typedef u32x4_vec u32x4_any __attribute__((aligned(2)));

// kN: 16 bytes of elements, or 1.  kAny: vectors start at any element.
template <bool kBf16, int kN, bool kAny = false>
struct RowVec {
    static_assert(kN == 1 || kN == (kBf16 ? 8 : 4), "an element or 16 bytes");
    using Raw = std::conditional_t<kN == 1, std::conditional_t<kBf16, uint16_t, uint32_t>, u32x4_vec>;
    using Memory = std::conditional_t<kN != 1 && kAny, u32x4_any, Raw>;

    // i: an element, the vector's first
    static __device__ __forceinline__ Raw load(const void* p, size_t i) {
        return *reinterpret_cast<const Memory*>(reinterpret_cast<const char*>(p) + i * (kBf16 ? 2 : 4));
    }
    static __device__ __forceinline__ void store(void* p, size_t i, const Raw& v) {
        *reinterpret_cast<Memory*>(reinterpret_cast<char*>(p) + i * (kBf16 ? 2 : 4)) = v;
    }
    static __device__ __forceinline__ void widen(const Raw& v, float (&f)[kN]) {
        if constexpr (kN == 1) {
            f[0] = kBf16 ? bf16_bits_to_f32(v) : __uint_as_float(v);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (kBf16) {
                    f[2 * i] = bf16_bits_to_f32(v[i] & 0xffffu);
                    f[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
                } else {
                    f[i] = __uint_as_float(v[i]);
                }
            }
        }
    }
    static __device__ __forceinline__ Raw narrow(const float (&f)[kN]) {
        if constexpr (kN == 1) {
            return (Raw)(kBf16 ? f32_to_bf16_bits(f[0]) : __float_as_uint(f[0]));
        } else {
            Raw o;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (kBf16) o[i] = f32_to_bf16_bits(f[2 * i]) | (f32_to_bf16_bits(f[2 * i + 1]) << 16);
                else o[i] = __float_as_uint(f[i]);
            }
            return o;
        }
    }
};

}  // namespace
}  // namespace metro
