// moe_grouped_mm_fp8 and moe_grouped_ffn_fp8: rows sorted by expert times their expert's e4m3 weights, rows and weights with an fp32
// scale for each block of 128 (fp8_common.h).
//
// Values are widened to bf16, so products are exact and sums fp32 in both forms; a result depends on the form by the order of its sums only.
// Few rows a group (fp8_split.h): bound by the weights' bytes, half of bf16's, every activated weight row streamed once per tile of at most
// 32 rows.  The FFN's activation between the products stays fp32 in memory and is quantized by the tiles that read it, which saves a launch.
// Many rows a group (fp8_ring.h): tiles of 128 or 64 rows x 256 weight rows, the activation quantized where it is made.
// Measured, us: FFN, a rank of eight, 8 tokens at 2048 x 768 13.2 (kernels of 7.0 + 5.2; the weights alone 3.8 at 6.2 TB/s), 97 tokens at 7168 x
// 2048 193 (5.9 TB/s of weights), 1024 tokens 360 (bf16 experts: 606), 4000 tokens at 2048 x 768 63; product of 16384 rows in 16 groups,
// 4096 x 4096, 527 (1.04 PFLOP/s under sustained load).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "fp8_common.h"
#include "fp8_ring.h"
#include "fp8_split.h"
#include "metro.h"

namespace metro {
namespace {

constexpr int kNarrowRows32 = 32;           // of a K-split tile
constexpr int kNarrowGrid = 2560;           // five rounds of the 512 resident workgroups, the rest in turns

// Against 1536: 97 and 512 tokens at 7168 x 2048 196 -> 193 and 303 -> 299 us.  One step of loads in flight a wave does as well as two (8
// tokens at 2048 x 768 13.0, 13.6; elsewhere equal): two workgroups of four waves on a CU have enough.  Slower: two workgroups per CU that
// take items in turn, the next item's loads issued by the last steps (8 tokens 15.3, 97 tokens at 7168 x 2048 204); three workgroups
// per CU (registers spill).
template <bool kGateUp, bool kQuantX, typename OT, bool kRagged>
__global__ __launch_bounds__(kFp8Threads, 2) void fp8_narrow_kernel(Fp8Args a, int64_t n_items) {
    __shared__ __attribute__((aligned(16))) char mem[65536];
    __shared__ float scale[4 * 64];
    const Fp8Lds lds{mem, scale};
    for (int64_t id = blockIdx.x; id < n_items; id += gridDim.x) {
        const Item it = locate_in_order(a.group_offsets, a.groups, a.T * a.k, kNarrowRows32, a.ntn, id);
        if (!it.valid) return;                                       // uniform; items are consecutive
        if (it.tile.rows <= 16) fp8_tile<kGateUp, kQuantX, OT, 1, 1, kRagged>(a, it.tile, lds);
        else fp8_tile<kGateUp, kQuantX, OT, 2, 1, kRagged>(a, it.tile, lds);
        __syncthreads();                                             // the next item's sums reuse the LDS
    }
}

// A workgroup per CU; each takes every n-th item of its XCD's list, big ones first.
constexpr int kRingGrid = 256;
template <bool kGateUp, typename OT>
__global__ __launch_bounds__(kRingThreads, 2) void fp8_ring_kernel(RingArgs a) {
    RingList list;
    int n[2];
    list.read(a.group_offsets, a.groups, a.T * a.k, blockIdx.x & 7, a.ntn, n);
    const int step = gridDim.x >> 3, id = blockIdx.x >> 3;
    fp8_ring_items<kGateUp, OT, 0>(a, list, id, n[0], step);
    __syncthreads();                                                 // the other class has other places in LDS
    fp8_ring_items<kGateUp, OT, 1>(a, list, (id + step - n[0] % step) % step, n[1], step);       // in turn behind them
}

inline int launched() { return hipGetLastError() == hipSuccess ? METRO_OK : METRO_ERR_HIP; }

// dtype: of dst
template <bool kGateUp, bool kQuantX>
int launch(Fp8Args a, int dtype, hipStream_t st) {
    const int cols = kFp8Blocks * (kGateUp ? 8 : 16);
    a.ntn = (a.n_out + cols - 1) / cols;
    const int64_t n_items = (int64_t)max_tiles(a.T * a.k, a.groups, kNarrowRows32) * a.ntn;
    const uint32_t grid = (uint32_t)std::min<int64_t>(n_items, kNarrowGrid);
    const bool whole = a.K % kBlock == 0 && a.n_out % kBlock == 0;
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(grid), dim3(kFp8Threads), 0, st, a, n_items); };
    if (kGateUp || dtype == METRO_DTYPE_F32) {
        if (whole) go(fp8_narrow_kernel<kGateUp, kQuantX, float, false>);
        else go(fp8_narrow_kernel<kGateUp, kQuantX, float, true>);
    } else if constexpr (!kGateUp) {
        if (whole) go(fp8_narrow_kernel<kGateUp, kQuantX, __bf16, false>);
        else go(fp8_narrow_kernel<kGateUp, kQuantX, __bf16, true>);
    }
    return launched();
}

// Ring tiles address rows and a slot's weights in 32 bits.
bool ring_fits(const Fp8Args& a, bool gate_up) {
    const uint64_t rows = a.perm_pair ? a.T : (uint64_t)a.T * a.k;
    return a.K % kBlock == 0 && a.n_out % kBlock == 0 && rows * a.ldx < (1ull << 32) && (uint64_t)a.n_out * (gate_up ? 2 : 1) * a.ldw < (1ull << 32);
}

template <bool kGateUp, typename OT>
int launch_ring(RingArgs a, hipStream_t st) {
    const int cols = kGateUp ? 128 : 256;
    a.ntn = (a.n_out + cols - 1) / cols;
    const int cap = a.T * a.k;
    const int64_t tiles = std::min<int64_t>(cap, max_tiles(cap, a.groups, kRingTileRows));
    const int64_t per_xcd = a.ntn < 8 ? (tiles * a.ntn + 7) / 8 : tiles * ((a.ntn + 7) / 8);
    const uint32_t grid = (uint32_t)std::min<int64_t>(8 * per_xcd, kRingGrid);
    hipLaunchKernelGGL((fp8_ring_kernel<kGateUp, OT>), dim3(grid), dim3(kRingThreads), 0, st, a);
    return launched();
}

// Ring tiles for batches of many rows.  With token lists the host knows T * k, of which a rank of eight has an eighth: more than 4096.
// Measured, the FFN of such a rank, K-split / ring tiles, us: 512 tokens (k = 8) 36 / 40 at 2048 x 768, 105 / 98 at 4096 x 1536, 298 / 319 at
// 7168 x 2048; 256 tokens 30 / 39, 85 / 89, 270 / 295; 768, 640 and 640 tokens 43 / 40, 104 / 102, 320 / 320 (1024 of the last: 462 / 365).
constexpr int kRingPairs = 4096;
// Rows in order are all there.  More than one K-split tile a group, and 2048 items of these, four for every workgroup that can be
// resident.  Measured, K-split / ring tiles, us, bf16: one group of 4096 x 4096, 512, 1024 and 2048 rows 32 / 56, 59 / 58 and 110 / 69; of
// 2048 x 7168, 1024 rows 52 / 90; of 512 x 1024, 4096 rows 15 / 20; 4 groups of 4096 x 4096, 512 and 1024 rows 35 / 55 and 61 / 58; 16
// groups, 1024, 2048 and 16384 rows 92 / 71, 149 / 117 and 938 / 541; 16 groups of 2048 x 1024, 1024 and 2048 rows 17.0 / 16.6 and 26.8 /
// 23.1; 32 groups of 4096 x 4096, 1024 and 2048 rows 122 / 110 and 180 / 143.  fp32: one group of 4096 x 4096, 512, 1024 and 2048 rows
// 33 / 58, 60 / 63 and 113 / 77; 16 groups, 1024 and 2048 rows 92 / 75 and 152 / 128.
constexpr int64_t kRingProducts = 1 << 22;  // rows x columns
bool many_rows(const Fp8Args& a) {
    const int64_t cap = (int64_t)a.T * a.k;
    return a.perm_pair ? cap > kRingPairs : cap > kNarrowRows32 * a.groups && cap * a.n_out >= kRingProducts;
}

constexpr int kMaxSide = 1 << 20;           // K, columns
constexpr int kMaxPitch = 1 << 28;          // eight rows are addressed in 32 bits

bool misaligned(const void* p) { return ((uintptr_t)p & 15) != 0; }

int check_sizes(const int32_t* group_offsets, int T, int k, int groups, int H, int I, int dtype) {
    if (T < 0 || k < 1 || groups < 1 || H < 1 || I < 1 || !group_offsets) return METRO_ERR_INVALID_ARG;
    if (dtype != METRO_DTYPE_BF16 && dtype != METRO_DTYPE_F32) return METRO_ERR_UNSUPPORTED;
    if (groups > kMaxSpr || (int64_t)T * k >= (1 << 24) || H > kMaxSide || I > kMaxSide) return METRO_ERR_UNSUPPORTED;
    return METRO_OK;
}

int check_matrix(const void* p, int ld, int K, const float* scale) {
    return !p || !scale || misaligned(p) || ld < K || ld % 16 != 0 || ld > kMaxPitch ? METRO_ERR_INVALID_ARG : METRO_OK;
}

inline size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }

// Between the two products: fp32, or (ring tiles) e4m3 and scales, which is less.
inline size_t act_bytes(int T, int k, int I) { return align256((size_t)T * k * up16(I) * 4); }

}  // namespace
}  // namespace metro

extern "C" int moe_grouped_mm_fp8(const void* x, int ldx, const float* xs, const int32_t* perm_pair, const int32_t* group_offsets, int T,
                                  int k, int groups, int K, int N, const void* w, int ldw, const float* ws, int dtype, void* y,
                                  void* stream) {
    using namespace metro;
    const int rc = check_sizes(group_offsets, T, k, groups, K, N, dtype);
    if (rc != METRO_OK) return rc;
    if (T == 0) return METRO_OK;
    if (check_matrix(x, ldx, K, xs) != METRO_OK || check_matrix(w, ldw, K, ws) != METRO_OK || !y || misaligned(y)) return METRO_ERR_INVALID_ARG;
    const Fp8Args a{x, xs, perm_pair, group_offsets, (const uint8_t*)w, ws, y, ldx, T, k, groups, K, N, ldw, N, 0};
    if (many_rows(a) && ring_fits(a, false)) {
        RingArgs r{};
        (Fp8Args&)r = a;
        return dtype == METRO_DTYPE_BF16 ? launch_ring<false, __bf16>(r, (hipStream_t)stream)
                                         : launch_ring<false, float>(r, (hipStream_t)stream);
    }
    return launch<false, false>(a, dtype, (hipStream_t)stream);
}

extern "C" size_t moe_grouped_ffn_fp8_workspace_bytes(int T, int k, int spr, int H, int I) {
    using namespace metro;
    if (T < 0 || k < 1 || spr < 1 || H < 1 || I < 1) return 0;
    return act_bytes(T, k, I) + 256;
}

extern "C" int moe_grouped_ffn_fp8(const void* x, int ldx, const float* xs, const int32_t* perm_pair, const int32_t* group_offsets, int T,
                                   int k, int spr, int H, int I, const void* w13, int ldw13, const float* s13, const void* w2, int ldw2,
                                   const float* s2, int dtype, void* y_perm, void* ws, size_t ws_bytes, void* stream) {
    using namespace metro;
    int rc = check_sizes(group_offsets, T, k, spr, H, I, dtype);
    if (rc != METRO_OK) return rc;
    if (T == 0) return METRO_OK;
    if (check_matrix(x, ldx, H, xs) != METRO_OK || check_matrix(w13, ldw13, H, s13) != METRO_OK || check_matrix(w2, ldw2, I, s2) != METRO_OK ||
        !perm_pair || !y_perm || misaligned(y_perm) || !ws || ((uintptr_t)ws & 255) != 0)
        return METRO_ERR_INVALID_ARG;
    if (ws_bytes < moe_grouped_ffn_fp8_workspace_bytes(T, k, spr, H, I)) return METRO_ERR_WORKSPACE;
    const int ld_act = (int)up16(I);
    const int cap = T * k;
    if (cap > kRingPairs && H % kBlock == 0 && I % kBlock == 0 && dtype == METRO_DTYPE_BF16) {
        uint8_t* act = (uint8_t*)ws;
        float* act_scale = (float*)((char*)ws + align256((size_t)cap * I));
        RingArgs up{}, down{};
        (Fp8Args&)up = Fp8Args{x, xs, perm_pair, group_offsets, (const uint8_t*)w13, s13, nullptr, ldx, T, k, spr, H, I, ldw13, I, 0};
        up.act = act, up.act_scale = act_scale;
        (Fp8Args&)down = Fp8Args{act, act_scale, nullptr, group_offsets, (const uint8_t*)w2, s2, y_perm, I, T, k, spr, I, H, ldw2, H, 0};
        if (ring_fits(up, true) && ring_fits(down, false)) {
            rc = launch_ring<true, float>(up, (hipStream_t)stream);
            return rc != METRO_OK ? rc : launch_ring<false, __bf16>(down, (hipStream_t)stream);
        }
    }
    const Fp8Args up{x, xs, perm_pair, group_offsets, (const uint8_t*)w13, s13, ws, ldx, T, k, spr, H, I, ldw13, ld_act, 0};
    rc = launch<true, false>(up, METRO_DTYPE_F32, (hipStream_t)stream);
    if (rc != METRO_OK) return rc;
    const Fp8Args down{ws, nullptr, nullptr, group_offsets, (const uint8_t*)w2, s2, y_perm, ld_act, T, k, spr, I, H, ldw2, H, 0};
    return launch<false, true>(down, dtype, (hipStream_t)stream);
}
