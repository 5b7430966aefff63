// Tile of a product of e4m3 rows with e4m3 weights for many rows: 256 weight rows (128 gate and 128 up, or 256 columns) x 16 MT rows by
// one workgroup of eight waves (4 across the weights x 2 across the rows), both operands from memory straight to an LDS ring of D
// stages.  A stage is a block of 128 k of every row, so its sum is scaled and added to the running one once per stage.
//
// LDS is cut into units of 64 rows x 128 bytes (of up to 32, for the last two), which one load instruction of every thread fills; a row's 16-byte piece p is at
// place p ^ (row & 7), so that the 16 rows of a fragment read spread over the banks.  A direct load puts lane i's 16 bytes at place i
// behind a common base, so the lane that fills place i reads piece i ^ (row & 7) of the row: still whole lines.  Every unit is an LDS
// variable of its own: that is how the compiler knows that a fragment read does not depend on the loads in flight to other units.
//
// One barrier per step.  When step s begins its fragments are in registers; behind the barrier -- every wave has read all of stage s,
// and stage s + 1 has arrived -- the stage is refilled with step s + D, the fragments of s + 1 are read, and s is multiplied.
// The wait before the barrier is a count of newer loads, so these are unconditional: past the end every lane takes the same bytes.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>
#include <utility>

#include "fp8_split.h"

namespace metro {
namespace {

constexpr int kRingThreads = 512;
constexpr int kRingTileRows = 128;
constexpr int kBand = 8;                    // tiles of a slot that are taken through all columns of an XCD together

// LDS: 18 units of 8 KB, two of 4 KB, the scales of four stages.
template <int I>
__device__ __forceinline__ char* ring_unit() {
    static_assert(I < 20, "");
    __shared__ __attribute__((aligned(1024))) char unit[I < 18 ? 8192 : 4096];
    return unit;
}
template <int I>
__device__ __forceinline__ float* ring_scale() {            // of 128 rows, then of the weights: gate's, up's
    static_assert(I < 4, "");
    __shared__ __attribute__((aligned(1024))) float scale[256];
    return scale;
}

template <int n>
__device__ __forceinline__ void wait_all_but() {        // outstanding vector loads at most n, no LDS access outstanding
    static_assert(n < 64, "");
    __builtin_amdgcn_s_waitcnt((n & 15) | (7 << 4) | ((n >> 4) << 14));
}

struct RingArgs : Fp8Args {
    uint8_t* act;               // gate/up: the activation in e4m3 [cap, ldd], and its scales [cap, blocks of n_out]
    float* act_scale;
};

// Unit of 64 rows (at most) of a stage's activations.
template <int MT>
constexpr int x_unit(int stage, int p) { return MT == 2 ? 16 + stage : 12 + stage * (MT / 4) + p; }

template <bool kGateUp, typename OT, int MT>
__device__ __forceinline__ void fp8_ring_tile(const RingArgs& a, const Tile t) {
    constexpr int M2 = MT / 2, D = MT == 2 ? 4 : 3, kXUnits = MT == 8 ? 2 : 1;
    constexpr int kUnitLoads = 4 + kXUnits, kLoads = kUnitLoads + 1;    // of a stage, per lane
    static_assert(MT == 2 || MT == 4 || MT == 8, "");
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r16 = lane & 15, q = lane >> 4, tx = wv & 3, ty = wv >> 2;
    const int nb = a.K / kBlock, col0 = t.col * (kGateUp ? 128 : 256);
    const int piece = ((tid & 7) ^ ((tid >> 3) & 7)) * 16;

    // unit p of a stage: weight rows w_row(p) ..+ 63; gate/up: two of gate, two of up.  Past the last column: the tile's first again
    auto w_row = [&](int p) { return kGateUp ? (p >> 1) * a.n_out + col0 + (p & 1) * 64 : col0 + p * 64 < a.n_out ? col0 + p * 64 : col0; };
    const uint8_t* wslot = a.w + (size_t)t.slot * (size_t)(kGateUp ? 2 * (int64_t)a.n_out : a.n_out) * a.ldw;
    const __amdgpu_buffer_rsrc_t w_rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)wslot, 0, -1, 0x00027000);
    const __amdgpu_buffer_rsrc_t x_rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)a.x, 0, -1, 0x00027000);
    uint32_t w_at[4];
#pragma unroll
    for (int p = 0; p < 4; ++p) w_at[p] = (uint32_t)w_row(p) * (uint32_t)a.ldw;
    const uint32_t w_lane = (uint32_t)(tid >> 3) * (uint32_t)a.ldw + piece;
    auto source = [&](int r) {                              // past the tile: its last row
        const int row = t.row0 + min(r, t.rows - 1);
        return (uint32_t)(a.perm_pair ? min(max(a.perm_pair[row] / a.k, 0), a.T - 1) : row);
    };
    uint32_t x_lane[kXUnits];
#pragma unroll
    for (int p = 0; p < kXUnits; ++p) x_lane[p] = source(p * 64 + (MT == 2 ? (tid >> 3) & 31 : tid >> 3)) * (uint32_t)a.ldx + piece;
    // Scales: two waves load those of 64 rows each, the others those of the weights: gate's and up's, or of columns 0..127 and
    // 128..255 (if there are any).  Six waves load the same, which costs less than a branch in the loop.
    const int row_blocks = blocks_of(a.n_out) * (kGateUp ? 2 : 1), second = kGateUp ? blocks_of(a.n_out) : col0 + 128 < a.n_out ? 1 : 0;
    const size_t ws_slot = (size_t)t.slot * row_blocks + col0 / kBlock;
    const __amdgpu_buffer_rsrc_t s_rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)(wv < 2 ? a.xs : a.ws + ws_slot * nb), 0, -1, 0x00027000);
    const uint32_t s_lane = (wv < 2 ? source(wv * 64 + lane) : (uint32_t)((lane & 1) * second)) * (uint32_t)(nb * 4);
    const int s_at = min(wv, 2) * 64;

    // piece p of a stage's loads: scales first, then the units
    auto load = [&](auto U, auto P, int s) {
        constexpr int set = decltype(U)::value % D, p = decltype(P)::value;
        const bool real = s < nb;
        const int step = min(s, nb - 1);
        if constexpr (p < 4) {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(w_rsrc, (__attribute__((address_space(3))) void*)(ring_unit<set * 4 + p>() + wv * 1024), 16,
                                                     (int)(real ? w_lane : 0u), (int)(w_at[p] + step * kBlock), 0, 0);
        } else {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                x_rsrc, (__attribute__((address_space(3))) void*)(ring_unit<x_unit<MT>(set, p - 4)>() + (MT == 2 ? wv & 3 : wv) * 1024), 16,
                (int)(real ? x_lane[p - 4] : 0u), step * kBlock, 0, 0);
        }
    };
    auto load_scale = [&](auto U, int s) {
        constexpr int set = decltype(U)::value % D;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(s_rsrc, (__attribute__((address_space(3))) void*)(ring_scale<set>() + s_at), 4, (int)s_lane,
                                                 min(s, nb - 1) * 4, 0, 0);
    };
    const int rd = r16 * 128 + ((q ^ (r16 & 7)) * 16);
    i32x8 fw[4], fx[M2];                                    // each is replaced once it has been multiplied
    auto fragment = [&](const char* p) {
        const u32x4 lo = *reinterpret_cast<const u32x4*>(p + rd), hi = *reinterpret_cast<const u32x4*>(p + (rd ^ 64));
        i32x8 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = (int)lo[e], v[4 + e] = (int)hi[e];
        return v;
    };
    auto read_w = [&](auto U, auto B) {
        constexpr int set = decltype(U)::value % D, b = decltype(B)::value;
        fw[b] = fragment(ring_unit<set * 4 + b>() + tx * 2048);
    };
    auto read_x = [&](auto U, auto B) {
        constexpr int set = decltype(U)::value % D, mt = decltype(B)::value;
        fx[mt] = fragment(ring_unit<x_unit<MT>(set, mt >> 1)>() + ((mt & 1) * 2 + ty) * 2048);
    };
    floatx4 acc[4][M2];
    auto multiply = [&](auto B, auto M, float scale) {
        constexpr int b = decltype(B)::value, mt = decltype(M)::value;
        const floatx4 p = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fw[b], fx[mt], floatx4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);
#pragma unroll
        for (int v = 0; v < 4; ++v) acc[b][mt][v] = fmaf(p[v], scale, acc[b][mt][v]);
    };
    auto arrive = [&](auto Left) {
        __builtin_amdgcn_sched_barrier(0);
        wait_all_but<decltype(Left)::value>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    float xscale[M2], wscale[2];
    auto read_scale = [&](auto U) {
        constexpr int set = decltype(U)::value % D;
#pragma unroll
        for (int mt = 0; mt < M2; ++mt) xscale[mt] = ring_scale<set>()[mt * 32 + ty * 16 + r16];
        wscale[0] = ring_scale<set>()[128];
        wscale[1] = ring_scale<set>()[129];
    };
    // The loads of step s + D go out between the products: a burst of them in front would hold the products back.
    auto step = [&](auto U, int s) {
        constexpr int u = decltype(U)::value;
        constexpr std::integral_constant<int, u + 1> next{};
        float scale[2][M2];
#pragma unroll
        for (int mt = 0; mt < M2; ++mt) scale[0][mt] = xscale[mt] * wscale[0], scale[1][mt] = xscale[mt] * wscale[1];
        arrive(std::integral_constant<int, (D - 2) * kLoads>{});
        read_scale(next);
        load_scale(U, s + D);
        run_steps(std::make_integer_sequence<int, 4>{}, [&](auto B, int) {
            constexpr int b = decltype(B)::value;
            run_steps(std::make_integer_sequence<int, M2>{}, [&](auto M, int) {
                constexpr int mt = decltype(M)::value, at = b * M2 + mt;
                multiply(B, M, scale[b >> 1][mt]);
                if constexpr (b == 3) read_x(next, M);
                constexpr int from = at * kUnitLoads / (4 * M2), to = (at + 1) * kUnitLoads / (4 * M2);
                if constexpr (to > from) load(U, std::integral_constant<int, from>{}, s + D);
                if constexpr (to > from + 1) load(U, std::integral_constant<int, from + 1>{}, s + D);
            }, 0);
            read_w(next, B);
            __builtin_amdgcn_sched_barrier(0);
        }, 0);
    };
    asm volatile("; ring of %0 stages, %1 loads each" ::"i"(D), "i"(kLoads));      // a comment in the assembly, no instruction
    run_steps(std::make_integer_sequence<int, D>{}, [&](auto U, int s) {
        load_scale(U, s);
        run_steps(std::make_integer_sequence<int, kUnitLoads>{}, [&](auto P, int) { load(U, P, s); }, 0);
        __builtin_amdgcn_sched_barrier(0);                  // the waits count on this order
    }, 0);
#pragma unroll
    for (int b = 0; b < 4; ++b)
#pragma unroll
        for (int mt = 0; mt < M2; ++mt) acc[b][mt] = floatx4{0.f, 0.f, 0.f, 0.f};
    constexpr std::integral_constant<int, 0> first{};
    arrive(std::integral_constant<int, (D - 1) * kLoads>{});
    read_scale(first);
    run_steps(std::make_integer_sequence<int, M2>{}, [&](auto M, int) { read_x(first, M); }, 0);
    run_steps(std::make_integer_sequence<int, 4>{}, [&](auto B, int) { read_w(first, B); }, 0);
    constexpr int kPeriod = D % 2 ? 2 * D : D;
    int s = 0;
    for (; s + kPeriod <= nb; s += kPeriod) run_steps(std::make_integer_sequence<int, kPeriod>{}, step, s);
    run_steps_tail(std::make_integer_sequence<int, kPeriod - 1>{}, step, s, nb);
    wait_all_but<0>();                                      // nothing is on its way to LDS when the workgroup ends or goes on
    asm volatile("; ring done");

    if constexpr (kGateUp) {
        // Columns col0 .. col0 + 127 are one block of the activation: its maximum over the lanes of a row, then over four waves.
        float o[2][M2][4];
        __syncthreads();
        uint32_t* part = reinterpret_cast<uint32_t*>(ring_unit<0>());       // [row][wave]
#pragma unroll
        for (int mt = 0; mt < M2; ++mt) {
            uint32_t m = 0;
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const float g = acc[b][mt][v];
                    o[b][mt][v] = g / (1.0f + expf(-g)) * acc[b + 2][mt][v];
                    m = max(m, magnitude(o[b][mt][v]));
                }
            m = max(m, (uint32_t)__shfl_xor((int)m, 16));
            m = max(m, (uint32_t)__shfl_xor((int)m, 32));
            if (q == 0) part[(mt * 32 + ty * 16 + r16) * 4 + tx] = m;
        }
        __syncthreads();
#pragma unroll
        for (int mt = 0; mt < M2; ++mt) {
            const int row = mt * 32 + ty * 16 + r16;
            const u32x4 m = reinterpret_cast<const u32x4*>(part)[row];
            const BlockScale sc = block_scale(max(max(m[0], m[1]), max(m[2], m[3])));
            if (row >= t.rows) continue;
            const size_t out = (size_t)(t.row0 + row);
#pragma unroll
            for (int b = 0; b < 2; ++b)
                *reinterpret_cast<uint32_t*>(a.act + out * a.ldd + col0 + b * 64 + tx * 16 + q * 4) =
                    pack_e4m3(o[b][mt][0] * sc.inverse, o[b][mt][1] * sc.inverse, o[b][mt][2] * sc.inverse, o[b][mt][3] * sc.inverse);
            if (tx == 0 && q == 0) a.act_scale[out * (a.n_out / kBlock) + t.col] = sc.scale;
        }
        __syncthreads();                                    // the next tile's loads take the LDS
    } else {
#pragma unroll
        for (int mt = 0; mt < M2; ++mt) {
            const int row = mt * 32 + ty * 16 + r16;
            if (row >= t.rows) continue;
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const int col = col0 + b * 64 + tx * 16 + q * 4;
                const float o[4] = {acc[b][mt][0], acc[b][mt][1], acc[b][mt][2], acc[b][mt][3]};
                if (col < a.n_out) store_columns(reinterpret_cast<OT*>(a.dst) + (size_t)(t.row0 + row) * a.ldd + col, 4, true, o);
            }
        }
        __syncthreads();
    }
}

// All tiles of 128 rows (the last of a slot shorter) x column tiles.  Workgroup i runs on XCD i mod 8, each with an L2 of its own: the
// tiles of a column of one slot read the same weights, so they are neighbours in the list of one XCD, and the columns of a slot go
// round the XCDs.  With fewer columns than XCDs the items themselves go round.  Lane = slot.
struct RingList {
    int begin, rows, tiles, first, mine, incl, stride;

    __device__ __forceinline__ int read(const int32_t* __restrict__ group_offsets, int groups, int cap, int xcd, int n_cols) {
        const int l = lane_id();
        int m = 0;
        begin = 0;
        if (l < groups) {                       // offsets that are not a partition of [0, cap] are clamped
            begin = min(max(group_offsets[l], 0), cap);
            m = min(max(group_offsets[l + 1], begin), cap) - begin;
        }
        rows = m;
        tiles = (m + kRingTileRows - 1) / kRingTileRows;
        stride = n_cols < 8 ? 1 : 8;
        first = n_cols < 8 ? 0 : (xcd - l * n_cols) & 7;
        mine = tiles * (n_cols < 8 ? n_cols : (n_cols - first + 7) >> 3);
        incl = wave_inclusive_sum(mine);
        const int n = __builtin_amdgcn_readlane(incl, kWave - 1);
        return n_cols < 8 ? (n - xcd + 7) >> 3 : n;
    }
    __device__ __forceinline__ Tile tile(int nth, int xcd) const {
        const int i = stride == 1 ? nth * 8 + xcd : nth;
        const uint64_t owner = __ballot(incl - mine <= i && i < incl);             // exactly one lane
        const int o = __ffsll((unsigned long long)owner) - 1;
        const int n = __builtin_amdgcn_readlane(tiles, o), at = i - __builtin_amdgcn_readlane(incl - mine, o);
        const int cols = (uint32_t)__builtin_amdgcn_readlane(mine, o) / (uint32_t)n;
        const int band = (uint32_t)at / (uint32_t)(kBand * cols), height = min(kBand, n - band * kBand), in = at - band * kBand * cols;
        const int c = (uint32_t)in / (uint32_t)height, row = (band * kBand + in - c * height) * kRingTileRows;
        Tile t;
        t.slot = o;
        t.col = __builtin_amdgcn_readlane(first, o) + c * stride;
        t.row0 = __builtin_amdgcn_readlane(begin, o) + row;
        t.rows = min(kRingTileRows, __builtin_amdgcn_readlane(rows, o) - row);
        return t;
    }
};

}  // namespace
}  // namespace metro
