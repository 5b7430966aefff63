// moe_permute_rows, its gradient, and moe_unpermute_backward: tokens sorted by expert, and the gradient of the weighted sum that brings
// them back.  All walk the tokens, not the sorted rows: a token's row is then read once for all its pairs here, and the dot products of the
// weights' gradient stay inside one workgroup.  Bound by HBM: every byte is read or written once.  Gradient of the combine, 8192 tokens x
// 2048 in bf16, k = 8, all pairs here: 571 MB in 117 us, 4.9 TB/s, what a large copy reaches.  Sort of 4096 tokens x 7168 in bf16, batches
// of 70, 71 and 171 MB: 20 us on average, 5.2 TB/s (22 us with one vector of a lane on its way at a time).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "metro.h"
#include "row_vec.h"

namespace metro {

// unpermute.hip: the sums of moe_permute_rows_backward over rows of whole, aligned vectors
int sum_whole_rows(const void* dx_perm, const int32_t* pair_row, int T, int k, int H, int dtype, void* dx, void* stream);

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

// The kernels take whole vectors of a row, then the elements that are left, lane < H - n_vec * kN: with H next to 2^31 the sum
// n_vec * kN + lane passes it.  kAny: rows that are no whole vectors, or not 16-byte aligned;
// their vectors start anywhere (2048 tokens x 2001 in bf16, k = 6, all pairs here, us, against element by element: sort 12.7 -> 11.5,
// its gradient 21.9 -> 11.8, gradient of the combine 63 -> 30).
// Lanes of a token: a wave (kWaveToken), four tokens to a workgroup, or the workgroup.
template <bool kWaveToken>
struct TokenLanes {
    static constexpr int kLanes = kWaveToken ? 64 : kThreads;
    static __device__ __forceinline__ int lane() { return threadIdx.x % kLanes; }
    static __device__ __forceinline__ int token() {
        return kWaveToken ? (int)blockIdx.x * (kThreads / 64) + (int)(threadIdx.x >> 6) : (int)blockIdx.x;
    }
};

// The rows of pairs j0 .. j0 + kPairs - 1 of a token, -1 for those of other ranks; whether there is one.
__device__ __forceinline__ bool rows_of(const int32_t* __restrict__ pair_row, int t, int k, int j0, int cap, int (&row)[kPairs]) {
    bool any = false;
#pragma unroll
    for (int j = 0; j < kPairs; ++j) {
        row[j] = j0 + j < k ? pair_row[(size_t)t * k + j0 + j] : -1;
        if (row[j] >= cap) row[j] = -1;
        any |= row[j] >= 0;
    }
    return any;
}

template <bool kBf16, bool kAny, bool kWaveToken>
__global__ __launch_bounds__(kThreads) void permute_rows_kernel(const void* __restrict__ x, const int32_t* __restrict__ pair_row,
                                                                int T, int k, int H, void* __restrict__ x_perm) {
    constexpr int kN = kBf16 ? 8 : 4, kLanes = TokenLanes<kWaveToken>::kLanes;
    using V = RowVec<kBf16, kN, kAny>;
    using E = RowVec<kBf16, 1>;
    const int lane = TokenLanes<kWaveToken>::lane(), t = TokenLanes<kWaveToken>::token(), n_vec = H / kN;
    if (t >= T) return;
    for (int j0 = 0; j0 < k; j0 += kPairs) {
        int row[kPairs];
        if (!rows_of(pair_row, t, k, j0, T * k, row)) continue;
        for (int c0 = lane; c0 < n_vec; c0 += kLanes * kAhead) {
            typename V::Raw v[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
                if (c0 + u * kLanes < n_vec) v[u] = V::load(x, (size_t)t * H + (c0 + u * kLanes) * kN);
#pragma unroll
            for (int j = 0; j < kPairs; ++j) {
                if (row[j] < 0) continue;                 // uniform per token
#pragma unroll
                for (int u = 0; u < kAhead; ++u)
                    if (c0 + u * kLanes < n_vec) V::store(x_perm, (size_t)row[j] * H + (c0 + u * kLanes) * kN, v[u]);
            }
        }
        if (kAny && lane < H - n_vec * kN) {
            const auto v = E::load(x, (size_t)t * H + n_vec * kN + lane);
#pragma unroll
            for (int j = 0; j < kPairs; ++j)
                if (row[j] >= 0) E::store(x_perm, (size_t)row[j] * H + n_vec * kN + lane, v);
        }
    }
}

template <bool kBf16, bool kAny, bool kWaveToken>
__global__ __launch_bounds__(kThreads) void unpermute_backward_kernel(const void* __restrict__ dout, const void* __restrict__ y_perm,
                                                                      const int32_t* __restrict__ pair_row,
                                                                      const float* __restrict__ topk_w, int T, int k, int H,
                                                                      void* __restrict__ dy_perm, float* __restrict__ dtopk_w) {
    constexpr int kN = kBf16 ? 8 : 4, kLanes = TokenLanes<kWaveToken>::kLanes;
    __shared__ float part[kWaveToken ? 1 : kThreads / 64][kPairs];
    const int lane = TokenLanes<kWaveToken>::lane(), t = TokenLanes<kWaveToken>::token(), n_vec = H / kN;
    if (t >= T) return;                                   // whole waves; with workgroups per token, never
    for (int j0 = 0; j0 < k; j0 += kPairs) {
        int row[kPairs];
        float w[kPairs], dot[kPairs] = {};
        const bool any = rows_of(pair_row, t, k, j0, T * k, row);
#pragma unroll
        for (int j = 0; j < kPairs; ++j) w[j] = j0 + j < k ? topk_w[(size_t)t * k + j0 + j] : 0.f;
        // the columns from `at` on that a vector (or an element) holds
        auto columns = [&](auto vec, int at) {
            using V = decltype(vec);
            constexpr int n = sizeof(typename V::Raw) == 16 ? kN : 1;
            const auto g = V::load(dout, (size_t)t * H + at);
            typename V::Raw y[kPairs];
#pragma unroll
            for (int j = 0; j < kPairs; ++j)
                if (row[j] >= 0) y[j] = V::load(y_perm, (size_t)row[j] * H + at);     // uniform per token
            float gf[n];
            V::widen(g, gf);
#pragma unroll
            for (int j = 0; j < kPairs; ++j) {
                if (row[j] < 0) continue;
                float yf[n], out[n];
                V::widen(y[j], yf);
#pragma unroll
                for (int e = 0; e < n; ++e) {
                    dot[j] = fmaf(gf[e], yf[e], dot[j]);
                    out[e] = w[j] * gf[e];
                }
                V::store(dy_perm, (size_t)row[j] * H + at, V::narrow(out));
            }
        };
        if (any) {
            for (int c = lane; c < n_vec; c += kLanes) columns(RowVec<kBf16, kN, kAny>{}, c * kN);
            if (kAny && lane < H - n_vec * kN) columns(RowVec<kBf16, 1>{}, n_vec * kN + lane);
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

// The gradient of the sort where rows are no whole vectors (the others: unpermute.hip): the same sums in the same order.
template <bool kBf16, bool kWaveToken>
__global__ __launch_bounds__(kThreads) void sum_rows_kernel(const void* __restrict__ dx_perm, const int32_t* __restrict__ pair_row, int T,
                                                            int k, int H, void* __restrict__ dx) {
    constexpr int kN = kBf16 ? 8 : 4, kLanes = TokenLanes<kWaveToken>::kLanes;
    const int lane = TokenLanes<kWaveToken>::lane(), t = TokenLanes<kWaveToken>::token(), n_vec = H / kN;
    if (t >= T) return;
    auto columns = [&](auto vec, int at) {
        using V = decltype(vec);
        constexpr int n = sizeof(typename V::Raw) == 16 ? kN : 1;
        float sum[n] = {};
        for (int j0 = 0; j0 < k; j0 += kPairs) {
            int row[kPairs];
            if (!rows_of(pair_row, t, k, j0, T * k, row)) continue;
            typename V::Raw y[kPairs];
#pragma unroll
            for (int j = 0; j < kPairs; ++j)
                if (row[j] >= 0) y[j] = V::load(dx_perm, (size_t)row[j] * H + at);
#pragma unroll
            for (int j = 0; j < kPairs; ++j) {
                if (row[j] < 0) continue;
                float f[n];
                V::widen(y[j], f);
#pragma unroll
                for (int e = 0; e < n; ++e) sum[e] += f[e];
            }
        }
        V::store(dx, (size_t)t * H + at, V::narrow(sum));
    };
    for (int c = lane; c < n_vec; c += kLanes) columns(RowVec<kBf16, kN, true>{}, c * kN);
    if (lane < H - n_vec * kN) columns(RowVec<kBf16, 1>{}, n_vec * kN + lane);
}

// f(kBf16, kAny, kWaveToken, workgroups): a wave per token up to 2 vectors a lane.  Measured for the gradient of the combine, us, a
// wave / a workgroup per token: 256 vectors, 8192 and 512 tokens (bf16, k = 8, all pairs here) 133 / 117 and 16.8 / 11.4.
template <typename F>
int by_shape(int T, int H, int dtype, bool aligned, F&& f) {
    const int per = dtype == METRO_DTYPE_BF16 ? 8 : 4;
    const bool any = !aligned || H % per != 0, wave = H / per <= 128;
    const int grid = wave ? (T + kThreads / 64 - 1) / (kThreads / 64) : T;
    auto pick = [&](auto Bf16, auto Any) {
        if (wave) f(Bf16, Any, std::true_type{}, grid);
        else f(Bf16, Any, std::false_type{}, grid);
    };
    if (dtype == METRO_DTYPE_BF16) {
        if (any) pick(std::true_type{}, std::true_type{});
        else pick(std::true_type{}, std::false_type{});
    } else {
        if (any) pick(std::false_type{}, std::true_type{});
        else pick(std::false_type{}, std::false_type{});
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
    return by_shape(T, H, dtype, aligned, [&](auto Bf16, auto Any, auto Wave, int grid) {
        hipLaunchKernelGGL((permute_rows_kernel<decltype(Bf16)::value, decltype(Any)::value, decltype(Wave)::value>), dim3(grid), dim3(kThreads),
                           0, (hipStream_t)stream, x, pair_row, T, k, H, x_perm);
    });
}

extern "C" int moe_permute_rows_backward(const void* dx_perm, const int32_t* pair_row, int T, int k, int H, int dtype, void* dx,
                                         void* stream) {
    using namespace metro;
    const int rc = check_rows(T, k, H, dtype);
    if (rc != METRO_OK || T == 0) return rc;
    if (!dx_perm || !pair_row || !dx) return METRO_ERR_INVALID_ARG;
    if (H % (dtype == METRO_DTYPE_BF16 ? 8 : 4) == 0 && (((uintptr_t)dx_perm | (uintptr_t)dx) & 15) == 0)
        return sum_whole_rows(dx_perm, pair_row, T, k, H, dtype, dx, stream);
    return by_shape(T, H, dtype, false, [&](auto Bf16, auto, auto Wave, int grid) {
        hipLaunchKernelGGL((sum_rows_kernel<decltype(Bf16)::value, decltype(Wave)::value>), dim3(grid), dim3(kThreads), 0,
                           (hipStream_t)stream, dx_perm, pair_row, T, k, H, dx);
    });
}

extern "C" int moe_unpermute_backward(const void* dout, const void* y_perm, const int32_t* pair_row, const float* topk_w, int T, int k,
                                      int H, int dtype, void* dy_perm, float* dtopk_w, void* stream) {
    using namespace metro;
    const int rc = check_rows(T, k, H, dtype);
    if (rc != METRO_OK || T == 0) return rc;
    if (!dout || !y_perm || !pair_row || !topk_w || !dy_perm || !dtopk_w) return METRO_ERR_INVALID_ARG;
    const bool aligned = (((uintptr_t)dout | (uintptr_t)y_perm | (uintptr_t)dy_perm) & 15) == 0;
    return by_shape(T, H, dtype, aligned, [&](auto Bf16, auto Any, auto Wave, int grid) {
        hipLaunchKernelGGL((unpermute_backward_kernel<decltype(Bf16)::value, decltype(Any)::value, decltype(Wave)::value>), dim3(grid),
                           dim3(kThreads), 0, (hipStream_t)stream, dout, y_perm, pair_row, topk_w, T, k, H, dy_perm, dtopk_w);
    });
}
