// moe_permute_rows and moe_unpermute_backward: tokens sorted by expert, and the gradient of the weighted sum that brings them back.
// Both walk the tokens, not the sorted rows: a token's row is then read once for all its pairs here, and the dot products of the
// weights' gradient stay inside one workgroup.  Bound by HBM: every byte is read or written once.  Gradient of the combine, 8192 tokens x
// 2048 in bf16, k = 8, all pairs here: 571 MB in 117 us, 4.9 TB/s, what a large copy reaches.  Sort of 4096 tokens x 7168 in bf16, batches
// of 70, 71 and 171 MB: 20 us on average, 5.2 TB/s (22 us with one vector of a lane on its way at a time).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "metro.h"
#include "row_vec.h"

namespace metro {
namespace {

constexpr int kThreads = 256;
constexpr int kPairs = 8;                   // pairs of a token that are in registers at a time
constexpr int kAhead = 4;                   // vectors of a row that a lane loads before it stores the first

// Sum over the lanes of a wave, in every lane; fixed order.
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

// Lanes of a token: a wave (kWave64), four tokens to a workgroup, or the workgroup.
template <bool kBf16, int kN, bool kWaveToken>
__global__ __launch_bounds__(kThreads) void permute_rows_kernel(const void* __restrict__ x, const int32_t* __restrict__ pair_row,
                                                                int T, int k, int n_vec, void* __restrict__ x_perm) {
    using V = RowVec<kBf16, kN>;
    constexpr int kLanes = kWaveToken ? 64 : kThreads;
    const int lane = threadIdx.x % kLanes;
    const int t = kWaveToken ? (int)blockIdx.x * (kThreads / 64) + (int)(threadIdx.x >> 6) : (int)blockIdx.x;
    if (t >= T) return;
    const int cap = T * k;
    for (int j0 = 0; j0 < k; j0 += kPairs) {
        int row[kPairs];
        bool any = false;
#pragma unroll
        for (int j = 0; j < kPairs; ++j) {
            row[j] = j0 + j < k ? pair_row[(size_t)t * k + j0 + j] : -1;
            if (row[j] >= cap) row[j] = -1;
            any |= row[j] >= 0;
        }
        if (!any) continue;
        for (int c0 = lane; c0 < n_vec; c0 += kLanes * kAhead) {
            typename V::Raw v[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
                if (c0 + u * kLanes < n_vec) v[u] = V::load(x, (size_t)t * n_vec + c0 + u * kLanes);
#pragma unroll
            for (int j = 0; j < kPairs; ++j) {
                if (row[j] < 0) continue;                 // uniform per token
#pragma unroll
                for (int u = 0; u < kAhead; ++u)
                    if (c0 + u * kLanes < n_vec) V::store(x_perm, (size_t)row[j] * n_vec + c0 + u * kLanes, v[u]);
            }
        }
    }
}

template <bool kBf16, int kN, bool kWaveToken>
__global__ __launch_bounds__(kThreads) void unpermute_backward_kernel(const void* __restrict__ dout, const void* __restrict__ y_perm,
                                                                      const int32_t* __restrict__ pair_row,
                                                                      const float* __restrict__ topk_w, int T, int k, int n_vec,
                                                                      void* __restrict__ dy_perm, float* __restrict__ dtopk_w) {
    using V = RowVec<kBf16, kN>;
    constexpr int kLanes = kWaveToken ? 64 : kThreads;
    __shared__ float part[kWaveToken ? 1 : kThreads / 64][kPairs];
    const int lane = threadIdx.x % kLanes;
    const int t = kWaveToken ? (int)blockIdx.x * (kThreads / 64) + (int)(threadIdx.x >> 6) : (int)blockIdx.x;
    if (t >= T) return;                                   // whole waves; with workgroups per token, never
    const int cap = T * k;
    for (int j0 = 0; j0 < k; j0 += kPairs) {
        int row[kPairs];
        float w[kPairs], dot[kPairs];
        bool any = false;
#pragma unroll
        for (int j = 0; j < kPairs; ++j) {
            const bool in = j0 + j < k;
            row[j] = in ? pair_row[(size_t)t * k + j0 + j] : -1;
            if (row[j] >= cap) row[j] = -1;
            w[j] = in ? topk_w[(size_t)t * k + j0 + j] : 0.f;
            dot[j] = 0.f;
            any |= row[j] >= 0;
        }
        if (any) {
            for (int c = lane; c < n_vec; c += kLanes) {
                const auto g = V::load(dout, (size_t)t * n_vec + c);
                typename V::Raw y[kPairs];
#pragma unroll
                for (int j = 0; j < kPairs; ++j)
                    if (row[j] >= 0) y[j] = V::load(y_perm, (size_t)row[j] * n_vec + c);     // uniform per token
                float gf[kN];
                V::widen(g, gf);
#pragma unroll
                for (int j = 0; j < kPairs; ++j) {
                    if (row[j] < 0) continue;
                    float yf[kN], out[kN];
                    V::widen(y[j], yf);
#pragma unroll
                    for (int e = 0; e < kN; ++e) {
                        dot[j] = fmaf(gf[e], yf[e], dot[j]);
                        out[e] = w[j] * gf[e];
                    }
                    V::store(dy_perm, (size_t)row[j] * n_vec + c, V::narrow(out));
                }
            }
#pragma unroll
            for (int j = 0; j < kPairs; ++j)
                if (row[j] >= 0) dot[j] = wave_sum(dot[j]);
        }
        if (kWaveToken) {
#pragma unroll
            for (int j = 0; j < kPairs; ++j)
                if (j0 + j < k && lane == j) dtopk_w[(size_t)t * k + j0 + j] = dot[j];
        } else {
            if (j0) __syncthreads();                      // the last round's sums have been read
            if ((threadIdx.x & 63) == 0) {
#pragma unroll
                for (int j = 0; j < kPairs; ++j) part[threadIdx.x >> 6][j] = dot[j];
            }
            __syncthreads();
            const int j = threadIdx.x;
            if (j < kPairs && j0 + j < k) {
                float s = part[0][j];
#pragma unroll
                for (int o = 1; o < kThreads / 64; ++o) s += part[o][j];
                dtopk_w[(size_t)t * k + j0 + j] = s;
            }
        }
    }
}

// f(kBf16, kN, kWaveToken, vectors of a row, workgroups): 16-byte vectors where rows are whole ones, else element by element; a
// wave per token up to 2 vectors a lane.  Measured for the gradient of the combine, us, a wave / a workgroup per token: 256 vectors,
// 8192 and 512 tokens (bf16, k = 8, all pairs here) 133 / 117 and 16.8 / 11.4.
template <typename F>
int by_shape(int T, int H, int dtype, bool aligned, F&& f) {
    const int per = dtype == METRO_DTYPE_BF16 ? 8 : 4;
    const bool vec = aligned && H % per == 0;
    const int n_vec = vec ? H / per : H;
    const bool wave = n_vec <= 128;
    const int grid = wave ? (T + kThreads / 64 - 1) / (kThreads / 64) : T;
    auto pick = [&](auto Bf16, auto N) {
        if (wave) f(Bf16, N, std::true_type{}, n_vec, grid);
        else f(Bf16, N, std::false_type{}, n_vec, grid);
    };
    using Four = std::integral_constant<int, 4>;
    using Eight = std::integral_constant<int, 8>;
    using One = std::integral_constant<int, 1>;
    if (dtype == METRO_DTYPE_BF16) {
        if (vec) pick(std::true_type{}, Eight{});
        else pick(std::true_type{}, One{});
    } else {
        if (vec) pick(std::false_type{}, Four{});
        else pick(std::false_type{}, One{});
    }
    return hipGetLastError() == hipSuccess ? METRO_OK : METRO_ERR_HIP;
}

int check_rows(int T, int k, int H, int dtype) {
    if (T < 0 || k < 1 || H < 1) return METRO_ERR_INVALID_ARG;
    if (dtype != METRO_DTYPE_BF16 && dtype != METRO_DTYPE_F32) return METRO_ERR_UNSUPPORTED;
    return (int64_t)T * k >= (1 << 24) ? METRO_ERR_UNSUPPORTED : METRO_OK;
}

}  // namespace
}  // namespace metro

extern "C" int moe_permute_rows(const void* x, const int32_t* pair_row, int T, int k, int H, int dtype, void* x_perm, void* stream) {
    using namespace metro;
    const int rc = check_rows(T, k, H, dtype);
    if (rc != METRO_OK || T == 0) return rc;
    if (!x || !pair_row || !x_perm) return METRO_ERR_INVALID_ARG;
    const bool aligned = (((uintptr_t)x | (uintptr_t)x_perm) & 15) == 0;
    return by_shape(T, H, dtype, aligned, [&](auto Bf16, auto N, auto Wave, int n_vec, int grid) {
        hipLaunchKernelGGL((permute_rows_kernel<decltype(Bf16)::value, decltype(N)::value, decltype(Wave)::value>), dim3(grid), dim3(kThreads),
                           0, (hipStream_t)stream, x, pair_row, T, k, n_vec, x_perm);
    });
}

extern "C" int moe_unpermute_backward(const void* dout, const void* y_perm, const int32_t* pair_row, const float* topk_w, int T, int k,
                                      int H, int dtype, void* dy_perm, float* dtopk_w, void* stream) {
    using namespace metro;
    const int rc = check_rows(T, k, H, dtype);
    if (rc != METRO_OK || T == 0) return rc;
    if (!dout || !y_perm || !pair_row || !topk_w || !dy_perm || !dtopk_w) return METRO_ERR_INVALID_ARG;
    const bool aligned = (((uintptr_t)dout | (uintptr_t)y_perm | (uintptr_t)dy_perm) & 15) == 0;
    return by_shape(T, H, dtype, aligned, [&](auto Bf16, auto N, auto Wave, int n_vec, int grid) {
        hipLaunchKernelGGL((unpermute_backward_kernel<decltype(Bf16)::value, decltype(N)::value, decltype(Wave)::value>), dim3(grid),
                           dim3(kThreads), 0, (hipStream_t)stream, dout, y_perm, pair_row, topk_w, T, k, n_vec, dy_perm, dtopk_w);
    });
}
