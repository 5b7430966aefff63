// moe_quantize_fp8 and moe_quantize_weights_fp8: rows to e4m3 with a scale for each 128 values of a row, weights to e4m3 with a scale for
// each 128 x 128.  One pass: a block stays in registers between its maximum and its rounding, so every byte is read and written once,
// and HBM bounds both: 16384 rows of 7168 in bf16, 352 MB, 63 us, 5.6 TB/s (67 us with at most 4096 workgroups); weights of 18 x 1536 x
// 2048 in bf16, 170 MB, 34.6 us, 4.9 TB/s (39.5 with the values widened to fp32 in registers), 1.06 GB of them 197 us.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "fp8_common.h"
#include "metro.h"

namespace metro {
namespace {

constexpr int kThreads = 256;
constexpr int kPer = 8;                     // values of a lane: 16 lanes are a block of a row

// Memory at any element alignment; the hardware takes unaligned 128-bit global loads.
typedef u32x4 u32x4_any __attribute__((aligned(2)));

// kPer values from column `c` of a row, as they are in memory.  kVec: rows are whole, aligned groups of kPer; else any rows, with zeros
// past the end.  A lane of quantize_weights_kernel holds 64 values from its maximum to its rounding: in 16 bits half the registers.
template <bool kBf16, bool kVec>
struct Values {
    static constexpr int kLoads = kBf16 ? 1 : 2;
    u32x4 raw[kLoads];

    __device__ __forceinline__ void load(const void* row, int c, int K) {
        const char* p = reinterpret_cast<const char*>(row) + (size_t)c * (kBf16 ? 2 : 4);
        if (kVec || c + kPer <= K) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                if constexpr (kVec) raw[i] = reinterpret_cast<const u32x4*>(p)[i];
                else raw[i] = reinterpret_cast<const u32x4_any*>(p)[i];
            }
        } else {                                            // the last values of a row
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
                if (c + e >= K) continue;
                if constexpr (kBf16) raw[0][e >> 1] |= (uint32_t)reinterpret_cast<const uint16_t*>(p)[e] << (16 * (e & 1));
                else raw[e >> 2][e & 3] = reinterpret_cast<const uint32_t*>(p)[e];
            }
        }
    }
    __device__ __forceinline__ void widen(float (&f)[kPer]) const {
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            if constexpr (kBf16) f[e] = __uint_as_float(e & 1 ? raw[0][e >> 1] & 0xffff0000u : raw[0][e >> 1] << 16);
            else f[e] = __uint_as_float(raw[e >> 2][e & 3]);
        }
    }
};

// q rows are 16-byte aligned, so a lane's eight bytes are too.
__device__ __forceinline__ void store_values(uint8_t* row, int c, int K, const float (&f)[kPer], float inverse) {
    const u32x2 v = {pack_e4m3(f[0] * inverse, f[1] * inverse, f[2] * inverse, f[3] * inverse),
                     pack_e4m3(f[4] * inverse, f[5] * inverse, f[6] * inverse, f[7] * inverse)};
    if (c + kPer <= K) {
        *reinterpret_cast<u32x2*>(row + c) = v;
    } else {
#pragma unroll
        for (int e = 0; e < kPer; ++e)
            if (c + e < K) row[c + e] = (uint8_t)(v[e >> 2] >> (8 * (e & 3)));
    }
}

__device__ __forceinline__ uint32_t largest_of(const float (&f)[kPer]) {
    uint32_t m = magnitude(f[0]);
#pragma unroll
    for (int e = 1; e < kPer; ++e) m = max(m, magnitude(f[e]));
    return m;
}

// A block of a row per 16 lanes; workgroups take runs of kTurns * 16 blocks, whose loads go out together.
template <bool kBf16, bool kVec, int kTurns>
__global__ __launch_bounds__(kThreads) void quantize_rows_kernel(const void* __restrict__ x, int64_t row_bytes, int R, int K,
                                                                 const int32_t* __restrict__ n_rows, uint8_t* __restrict__ q, int ldq,
                                                                 float* __restrict__ scale) {
    const int nb = blocks_of(K);
    const int rows = n_rows ? min(max(n_rows[0], 0), R) : R;
    const int64_t n = (int64_t)rows * nb, stride = (int64_t)gridDim.x * (kTurns * kThreads / 16);
    const int c16 = (threadIdx.x & 15) * kPer;
    for (int64_t first = (int64_t)blockIdx.x * (kTurns * kThreads / 16) + threadIdx.x / 16; first < n; first += stride) {
        Values<kBf16, kVec> f[kTurns];
        int row[kTurns], col[kTurns];
#pragma unroll
        for (int u = 0; u < kTurns; ++u) {
            const int64_t i = min(first + u * (kThreads / 16), n - 1);          // past the end: the last block again
            row[u] = (int)(n >> 32 ? i / nb : (int64_t)((uint32_t)i / (uint32_t)nb));
            col[u] = (int)(i - (int64_t)row[u] * nb);
            const int c = col[u] * kBlock + c16;
            f[u] = {};
            if (c < K) f[u].load(reinterpret_cast<const char*>(x) + row[u] * row_bytes, c, K);      // else: a short last block
        }
#pragma unroll
        for (int u = 0; u < kTurns; ++u) {
            float v[kPer];
            f[u].widen(v);
            const BlockScale s = block_scale(group_max<16>(largest_of(v)));
            if (first + u * (kThreads / 16) >= n) continue;
            store_values(q + (size_t)row[u] * ldq, col[u] * kBlock + c16, K, v, s.inverse);
            if ((threadIdx.x & 15) == 0) scale[(size_t)row[u] * nb + col[u]] = s.scale;
        }
    }
}

// A workgroup per block of 128 x 128: thread (r, c) holds columns 8 c .. 8 c + 7 of rows r, r + 16, ...
template <bool kBf16, bool kVec>
__global__ __launch_bounds__(kThreads) void quantize_weights_kernel(const void* __restrict__ w, int64_t row_bytes, int rows, int K,
                                                                    uint8_t* __restrict__ q, int ldq, float* __restrict__ scale) {
    constexpr int kTurns = kBlock / 16;
    __shared__ uint32_t part[kThreads / 64];
    const int nb = blocks_of(K), nr = blocks_of(rows);
    const int64_t id = blockIdx.x;
    const int64_t at = id / nb;                                                 // (slot, row block)
    const int cb = (int)(id - at * nb), slot = (int)(at / nr), rb = (int)(at - (int64_t)slot * nr);
    const int r0 = rb * kBlock + threadIdx.x / 16, c = cb * kBlock + (threadIdx.x & 15) * kPer;
    const int64_t base = (int64_t)slot * rows;
    Values<kBf16, kVec> f[kTurns];
#pragma unroll
    for (int u = 0; u < kTurns; ++u) {
        const int r = r0 + u * 16;
        f[u] = {};
        if (r < rows && c < K) f[u].load(reinterpret_cast<const char*>(w) + (base + r) * row_bytes, c, K);
    }
    uint32_t m = 0;
#pragma unroll
    for (int u = 0; u < kTurns; ++u) {
        float v[kPer];
        f[u].widen(v);
        m = max(m, largest_of(v));
    }
    m = group_max<16>(m);
    m = max(m, (uint32_t)__shfl_xor((int)m, 16));
    m = max(m, (uint32_t)__shfl_xor((int)m, 32));
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = m;
    __syncthreads();
#pragma unroll
    for (int o = 0; o < kThreads / 64; ++o) m = max(m, part[o]);
    const BlockScale s = block_scale(m);
    if (threadIdx.x == 0) scale[id] = s.scale;
    if (c >= K) return;
#pragma unroll
    for (int u = 0; u < kTurns; ++u) {
        const int r = r0 + u * 16;
        if (r >= rows) continue;
        float v[kPer];
        f[u].widen(v);
        store_values(q + (base + r) * (int64_t)ldq, c, K, v, s.inverse);
    }
}

bool whole_vectors(const void* p, int64_t ld, int K, int dtype) {
    const int per = dtype == METRO_DTYPE_BF16 ? 8 : 4;
    return ((uintptr_t)p & 15) == 0 && ld % per == 0 && K % 8 == 0;
}

constexpr int kMaxSide = 1 << 30;           // rows, K: block counts stay inside 32 bits

int check_types(int ld, int K, int dtype, const void* q, int ldq) {
    if (K > kMaxSide) return METRO_ERR_UNSUPPORTED;
    if (K < 1 || ld < K || ldq < K || ldq % 16 != 0 || ((uintptr_t)q & 15) != 0) return METRO_ERR_INVALID_ARG;
    if (dtype != METRO_DTYPE_BF16 && dtype != METRO_DTYPE_F32) return METRO_ERR_UNSUPPORTED;
    return METRO_OK;
}

}  // namespace
}  // namespace metro

extern "C" int moe_quantize_fp8(const void* x, int ldx, int R, int K, int dtype, const int32_t* n_rows, void* q, int ldq, float* scale,
                                void* stream) {
    using namespace metro;
    if (R < 0) return METRO_ERR_INVALID_ARG;
    const int rc = check_types(ldx, K, dtype, q, ldq);
    if (rc != METRO_OK) return rc;
    if (R == 0) return METRO_OK;
    if (!x || !q || !scale) return METRO_ERR_INVALID_ARG;
    const bool bf16 = dtype == METRO_DTYPE_BF16, vec = whole_vectors(x, ldx, K, dtype);
    const int64_t n = (int64_t)R * blocks_of(K);
    auto go = [&](auto kernel, int turns) {
        const int64_t per = turns * (kThreads / 16);
        const uint32_t grid = (uint32_t)std::min<int64_t>((n + per - 1) / per, 1 << 20);
        hipLaunchKernelGGL(kernel, dim3(grid), dim3(kThreads), 0, (hipStream_t)stream, x, (int64_t)ldx * (bf16 ? 2 : 4), R, K, n_rows,
                           (uint8_t*)q, ldq, scale);
    };
    if (bf16 && vec) go(quantize_rows_kernel<true, true, 2>, 2);
    else if (bf16) go(quantize_rows_kernel<true, false, 1>, 1);
    else if (vec) go(quantize_rows_kernel<false, true, 2>, 2);
    else go(quantize_rows_kernel<false, false, 1>, 1);
    return hipGetLastError() == hipSuccess ? METRO_OK : METRO_ERR_HIP;
}

extern "C" int moe_quantize_weights_fp8(const void* w, int ldw, int slots, int rows, int K, int dtype, void* q, int ldq, float* scale,
                                        void* stream) {
    using namespace metro;
    if (slots < 0 || rows < 1) return METRO_ERR_INVALID_ARG;
    const int rc = check_types(ldw, K, dtype, q, ldq);
    if (rc != METRO_OK) return rc;
    if (slots == 0) return METRO_OK;
    if (!w || !q || !scale) return METRO_ERR_INVALID_ARG;
    const int64_t n = rows > kMaxSide ? 0 : (int64_t)slots * blocks_of(rows) * blocks_of(K);
    if (rows > kMaxSide || n >= (1 << 24)) return METRO_ERR_UNSUPPORTED;                           // a launch has fewer than 2^32 threads
    const bool bf16 = dtype == METRO_DTYPE_BF16, vec = whole_vectors(w, ldw, K, dtype);
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((uint32_t)n), dim3(kThreads), 0, (hipStream_t)stream, w, (int64_t)ldw * (bf16 ? 2 : 4), rows, K,
                           (uint8_t*)q, ldq, scale);
    };
    if (bf16 && vec) go(quantize_weights_kernel<true, true>);
    else if (bf16) go(quantize_weights_kernel<true, false>);
    else if (vec) go(quantize_weights_kernel<false, true>);
    else go(quantize_weights_kernel<false, false>);
    return hipGetLastError() == hipSuccess ? METRO_OK : METRO_ERR_HIP;
}
