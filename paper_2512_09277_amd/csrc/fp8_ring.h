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
//
// A workgroup has a CU for itself, so nothing else runs while a tile begins or ends: the last D steps of a tile therefore load the first
// D of the workgroup's next one.  Step j of it goes where step j of any tile is expected, stage j % D, which is free in that of the
// last steps that has the same remainder.
//
// The values are widened to bf16 as in fp8_split.h: products are exact, sums fp32.  The matrix cores' own e4m3 products
// (v_mfma_f32_16x16x128_f8f6f4) are faster, 337 us for 16384 rows x 4096 x 4096 in 16 groups instead of 530, but they align the products of
// a block to the largest and drop what is more than 13 binary places below it: of 448 * 448 - 448 * 448 + 126 nothing is left.
//
// A step's activations are widened once, in front, and 16 weight rows at a time once per step and wave: 128 conversions for 64 products.
//
// Measured on 16384 rows x 4096 columns in one group: 1.08 PFLOP/s at K = 4096, 1.17 at 7168, 1.84 us a step of a tile of 128 rows.  Vector
// instructions bound it: 277 of a wave and step (the conversions 4.5 cycles each, the scaled additions, addresses) beside 64 matrix
// instructions of 17.6 cycles, two waves to a SIMD.
// Before that, with e4m3 products: scales through LDS instead of registers (16 lines a load, 8 waves) and loads between the products
// 437 -> 329 us; the next tile's loads 365 -> 350 and results in whole lines with products added two later 350 -> 332 (16 groups).  No
// difference: the order of tiles in bands of 4, 8 or 16; now, the matrix instructions of two products in turn.
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

template <int I>
__device__ __forceinline__ uint32_t* ring_part() {          // a row's maximum in each of four waves
    __shared__ __attribute__((aligned(16))) uint32_t part[kRingTileRows * 4];
    return part;
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
constexpr int x_unit(int stage, int p) { return MT == 2 ? 16 + stage : 12 + stage * 2 + p; }

// Where the loads of a tile come from.
template <bool kGateUp, int kXUnits>
struct RingSource {
    const uint8_t* w;           // the slot's weights
    const float* scale;         // rows' scales (two waves) or the weights'
    uint32_t w_lane, w_at[4];   // of unit p, this lane's row of the tile's weights
    uint32_t x_lane[kXUnits], s_lane;

    static __device__ __forceinline__ int row_of(int p) {           // of the tile, whose 16 bytes this lane loads to unit p
        return p * 64 + (kXUnits == 1 ? (threadIdx.x >> 3) & 31 : threadIdx.x >> 3);
    }
    // Rows are loaded a tile ahead of their use (`raw`), for they may hang on a load of their own.
    struct Raw { int row[kXUnits], scale_row; };
    static __device__ __forceinline__ Raw raw(const RingArgs& a, const Tile& t) {
        auto source = [&](int r) {                                  // past the tile: its last row
            const int row = t.row0 + min(r, t.rows - 1);
            return a.perm_pair ? a.perm_pair[row] : row;
        };
        Raw r;
#pragma unroll
        for (int p = 0; p < kXUnits; ++p) r.row[p] = source(row_of(p));
        r.scale_row = source((int)(threadIdx.x & 127));
        return r;
    }
    __device__ __forceinline__ void set(const RingArgs& a, const Tile& t, const Raw& raw, int wv) {
        const int nb = a.K / kBlock, col0 = t.col * (kGateUp ? 128 : 256), piece = ((threadIdx.x & 7) ^ ((threadIdx.x >> 3) & 7)) * 16;
        auto token = [&](int r) { return (uint32_t)(a.perm_pair ? min(max(r / a.k, 0), a.T - 1) : r); };
        const int second = kGateUp ? blocks_of(a.n_out) : col0 + 128 < a.n_out ? 1 : 0;
        w = a.w + (size_t)t.slot * (size_t)(kGateUp ? 2 * (int64_t)a.n_out : a.n_out) * a.ldw;
        // Row i of wave tx's 16 rows in unit p is column 64 tx + 16 (i / 4) + 4 p + i % 4 of the tile; gate/up: units 0, 1 gate, 2, 3 up,
        // column 32 tx + 8 (i / 4) + 4 (p % 2) + i % 4 of either.  A lane then ends up with 16 (8) neighbouring columns of a row, and the
        // lanes of a wave with whole lines.  Past the last column: the tile's first half again.
        const int i = (threadIdx.x >> 3) & 15, tx = threadIdx.x >> 7, in = kGateUp ? tx : second ? tx : tx & 1;
        w_lane = (uint32_t)(kGateUp ? in * 32 + (i >> 2) * 8 + (i & 3) : in * 64 + (i >> 2) * 16 + (i & 3)) * (uint32_t)a.ldw + piece;
#pragma unroll
        for (int p = 0; p < 4; ++p) w_at[p] = (uint32_t)(kGateUp ? (p >> 1) * a.n_out + col0 + (p & 1) * 4 : col0 + p * 4) * (uint32_t)a.ldw;
#pragma unroll
        for (int p = 0; p < kXUnits; ++p) x_lane[p] = token(raw.row[p]) * (uint32_t)a.ldx + piece;
        // Two waves load the scales of 64 rows each, the others those of the weights: gate's and up's, or of columns 0..127 and
        // 128..255 (if there are any).  Six waves load the same, which costs less than a branch in the loop.
        const int row_blocks = blocks_of(a.n_out) * (kGateUp ? 2 : 1);
        scale = wv < 2 ? a.xs : a.ws + ((size_t)t.slot * row_blocks + col0 / kBlock) * nb;
        s_lane = (wv < 2 ? token(raw.scale_row) : (uint32_t)((threadIdx.x & 1) * second)) * (uint32_t)(nb * 4);
    }
};

// ready: the first D stages are in LDS or on their way.  has_next: the last steps load those of `then`.
template <bool kGateUp, typename OT, int MT, typename Source>
__device__ __forceinline__ void fp8_ring_tile(const RingArgs& a, const Tile t, const Source& now, const Source& then, bool ready, bool has_next) {
    constexpr bool kBig = MT > 2;
    constexpr int M2 = MT / 2, D = kBig ? 3 : 4, kXUnits = kBig ? 2 : 1;
    constexpr int kUnitLoads = 4 + kXUnits, kLoads = kUnitLoads + 1;    // of a stage, per lane
    static_assert(MT == 2 || MT == 4 || MT == 8, "");
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r16 = lane & 15, q = lane >> 4, tx = wv & 3, ty = wv >> 2;
    const int nb = a.K / kBlock, col0 = t.col * (kGateUp ? 128 : 256);
    const int s_at = min(wv, 2) * 64;

    // A load of step s: of this tile, of the next one's step `first` (s % D), or of nothing new.
    struct From { __amdgpu_buffer_rsrc_t w, scale; int at; bool own, real; };
    const __amdgpu_buffer_rsrc_t x_rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)a.x, 0, -1, 0x00027000);
    auto from = [&](int s, int first) {
        const bool own = s < nb;
        return From{__builtin_amdgcn_make_buffer_rsrc((void*)(own ? now.w : then.w), 0, -1, 0x00027000),
                    __builtin_amdgcn_make_buffer_rsrc((void*)(own ? now.scale : then.scale), 0, -1, 0x00027000), own ? s : min(first, nb - 1), own,
                    own || has_next};
    };
    auto load = [&](auto U, auto P, const From& f) {
        constexpr int set = decltype(U)::value % D, p = decltype(P)::value;
        if constexpr (p < 4) {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(f.w, (__attribute__((address_space(3))) void*)(ring_unit<set * 4 + p>() + wv * 1024), 16,
                                                     (int)(!f.real ? 0u : f.own ? now.w_lane : then.w_lane), (int)((f.own ? now.w_at[p] : then.w_at[p]) + f.at * kBlock), 0, 0);
        } else {
            const uint32_t lane_at = f.own ? now.x_lane[p - 4] : then.x_lane[p - 4];
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                x_rsrc, (__attribute__((address_space(3))) void*)(ring_unit<x_unit<MT>(set, p - 4)>() + (kBig ? wv : wv & 3) * 1024), 16,
                (int)(f.real ? lane_at : 0u), f.at * kBlock, 0, 0);
        }
    };
    auto load_scale = [&](auto U, const From& f) {
        constexpr int set = decltype(U)::value % D;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(f.scale, (__attribute__((address_space(3))) void*)(ring_scale<set>() + s_at), 4,
                                                 (int)(f.own ? now.s_lane : then.s_lane), f.at * 4, 0, 0);
    };
    int rd = r16 * 128 + ((q ^ (r16 & 7)) * 16);
    struct Bytes { u32x4 lo, hi; };
    struct Wide { bf16x8 part[4]; };
    Bytes fw[4], fx[M2];                                    // of the next step once they have been widened
    Wide xw[M2];
    auto fragment = [&](const char* p) { return Bytes{*reinterpret_cast<const u32x4*>(p + rd), *reinterpret_cast<const u32x4*>(p + (rd ^ 64))}; };
    auto widen = [](const Bytes& f) {
        return Wide{{widen_e4m3(f.lo[0], f.lo[1]), widen_e4m3(f.lo[2], f.lo[3]), widen_e4m3(f.hi[0], f.hi[1]), widen_e4m3(f.hi[2], f.hi[3])}};
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
    // A product is added two products later: its result takes longer than the next one to be issued.
    constexpr int kProducts = 4 * M2, kLate = 2;
    floatx4 late[kLate] = {};
    float late_scale[kLate] = {};
    auto add_late = [&](auto I) {                                   // product I (of this step, or counted back into the last one)
        constexpr int i = (decltype(I)::value + kProducts) % kProducts, slot = (decltype(I)::value + kProducts) % kLate;
#pragma unroll
        for (int v = 0; v < 4; ++v) acc[i / M2][i % M2][v] = fmaf(late[slot][v], late_scale[slot], acc[i / M2][i % M2][v]);
    };
    auto multiply = [&](auto I, const Wide& w, const Wide& x, float scale) {
        constexpr int i = decltype(I)::value, slot = i % kLate;
        floatx4 p = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < 4; ++c) p = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w.part[c], x.part[c], p, 0, 0, 0);
        add_late(std::integral_constant<int, i - kLate>{});
        late[slot] = p;
        late_scale[slot] = scale;
        __builtin_amdgcn_sched_barrier(0);
    };
    auto arrive = [&](auto Left) {
        __builtin_amdgcn_sched_barrier(0);
        wait_all_but<decltype(Left)::value>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    float xscale[M2], wscale[kGateUp ? 2 : 1];
    auto read_scale = [&](auto U) {
        constexpr int set = decltype(U)::value % D;
#pragma unroll
        for (int mt = 0; mt < M2; ++mt) xscale[mt] = ring_scale<set>()[mt * 32 + ty * 16 + r16];
        wscale[0] = ring_scale<set>()[kGateUp ? 128 : 128 + (tx >> 1)];
        if constexpr (kGateUp) wscale[1] = ring_scale<set>()[129];
    };
    // The loads of step s + D go out between the products: a burst of them in front would hold the products back.
    auto step = [&](auto U, int s) {
        constexpr int u = decltype(U)::value;
        constexpr std::integral_constant<int, u + 1> next{};
        float scale[kGateUp ? 2 : 1][M2];
#pragma unroll
        for (int mt = 0; mt < M2; ++mt) {
            scale[0][mt] = xscale[mt] * wscale[0];
            if constexpr (kGateUp) scale[1][mt] = xscale[mt] * wscale[1];
        }
        const From f = from(s + D, u % D);
        asm volatile("" : "+v"(rd));                        // or the addresses of all units, computed ahead, spill registers
#pragma unroll
        for (int mt = 0; mt < M2; ++mt) xw[mt] = widen(fx[mt]);
        arrive(std::integral_constant<int, (D - 2) * kLoads>{});
        read_scale(next);
        load_scale(U, f);
        run_steps(std::make_integer_sequence<int, 4>{}, [&](auto B, int) {
            constexpr int b = decltype(B)::value;
            const Wide ww = widen(fw[b]);
            run_steps(std::make_integer_sequence<int, M2>{}, [&](auto M, int) {
                constexpr int mt = decltype(M)::value, at = b * M2 + mt;
                multiply(std::integral_constant<int, at>{}, ww, xw[mt], scale[kGateUp ? b >> 1 : 0][mt]);
                if constexpr (b == 3) read_x(next, M);
                constexpr int begin = at * kUnitLoads / (4 * M2), end = (at + 1) * kUnitLoads / (4 * M2);
                if constexpr (end > begin) load(U, std::integral_constant<int, begin>{}, f);
                if constexpr (end > begin + 1) load(U, std::integral_constant<int, begin + 1>{}, f);
            }, 0);
            read_w(next, B);
            __builtin_amdgcn_sched_barrier(0);
        }, 0);
    };
    asm volatile("; ring of %0 stages, %1 loads each" ::"i"(D), "i"(kLoads));      // a comment in the assembly, no instruction
    if (!ready) {
        run_steps(std::make_integer_sequence<int, D>{}, [&](auto U, int s) {
            const From f{__builtin_amdgcn_make_buffer_rsrc((void*)now.w, 0, -1, 0x00027000),
                         __builtin_amdgcn_make_buffer_rsrc((void*)now.scale, 0, -1, 0x00027000), min(s, nb - 1), true, true};
            load_scale(U, f);
            run_steps(std::make_integer_sequence<int, kUnitLoads>{}, [&](auto P, int) { load(U, P, f); }, 0);
            __builtin_amdgcn_sched_barrier(0);              // the waits count on this order
        }, 0);
        wait_all_but<(D - 1) * kLoads>();
    }
#pragma unroll
    for (int b = 0; b < 4; ++b)
#pragma unroll
        for (int mt = 0; mt < M2; ++mt) acc[b][mt] = floatx4{0.f, 0.f, 0.f, 0.f};
    constexpr std::integral_constant<int, 0> first{};
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    read_scale(first);
    run_steps(std::make_integer_sequence<int, M2>{}, [&](auto M, int) { read_x(first, M); }, 0);
    run_steps(std::make_integer_sequence<int, 4>{}, [&](auto B, int) { read_w(first, B); }, 0);
    constexpr int kPeriod = D % 2 ? 2 * D : D;
    int s = 0;
    for (; s + kPeriod <= nb; s += kPeriod) run_steps(std::make_integer_sequence<int, kPeriod>{}, step, s);
    run_steps_tail(std::make_integer_sequence<int, kPeriod - 1>{}, step, s, nb);
    add_late(std::integral_constant<int, -2>{});
    add_late(std::integral_constant<int, -1>{});
    // The next tile's stages have arrived before anything else is issued, so that it need not wait for this one's results to be
    // stored; without one, nothing is on its way to LDS when the workgroup ends.
    __builtin_amdgcn_sched_barrier(0);
    wait_all_but<0>();
    asm volatile("; ring done" ::: "memory");

    if constexpr (kGateUp) {
        // Columns col0 .. col0 + 127 are one block of the activation: its maximum over the lanes of a row, then over four waves.
        float o[2][M2][4];
        uint32_t* const part = ring_part<0>();
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
            u32x2 v;
#pragma unroll
            for (int b = 0; b < 2; ++b)
                v[b] = pack_e4m3(o[b][mt][0] * sc.inverse, o[b][mt][1] * sc.inverse, o[b][mt][2] * sc.inverse, o[b][mt][3] * sc.inverse);
            *reinterpret_cast<u32x2*>(a.act + out * a.ldd + col0 + tx * 32 + q * 8) = v;
            if (tx == 0 && q == 0) a.act_scale[out * (a.n_out / kBlock) + t.col] = sc.scale;
        }
    } else {
#pragma unroll
        for (int mt = 0; mt < M2; ++mt) {
            const int row = mt * 32 + ty * 16 + r16;
            if (row >= t.rows) continue;
            const int col = col0 + tx * 64 + q * 16;
            if (col >= a.n_out) continue;
            OT* out = reinterpret_cast<OT*>(a.dst) + (size_t)(t.row0 + row) * a.ldd + col;
            if constexpr (sizeof(OT) == 4) {
#pragma unroll
                for (int b = 0; b < 4; ++b) *reinterpret_cast<floatx4*>(out + b * 4) = acc[b][mt];
            } else {
#pragma unroll
                for (int b = 0; b < 4; b += 2)
                    *reinterpret_cast<u32x4*>(out + b * 4) =
                        u32x4{pack_bf16x2(acc[b][mt][0], acc[b][mt][1]), pack_bf16x2(acc[b][mt][2], acc[b][mt][3]),
                              pack_bf16x2(acc[b + 1][mt][0], acc[b + 1][mt][1]), pack_bf16x2(acc[b + 1][mt][2], acc[b + 1][mt][3])};
            }
        }
    }
}

// A slot's rows make tiles of 128 (or 64) rows and one for the remainder: big ones (more than 32 rows) and at most one small one.  Workgroup i runs
// on XCD i mod 8, each with an L2 of its own: the tiles of a column of one slot read the same weights, so they are neighbours in the
// list of one XCD, and the columns of a slot go round the XCDs.  With fewer columns than XCDs the items themselves go round.
// Lane = slot.
constexpr int kSmallRows = 32;
struct RingList {
    int begin, rows, first, stride, xcd, size;     // size: rows of a tile
    int tiles[2], incl[2];                      // of big ones, small ones: tiles of the slot, items of the slots up to it

    __device__ __forceinline__ void read(const int32_t* __restrict__ group_offsets, int groups, int cap, int xcd_, int n_cols, int (&n)[2]) {
        const int l = lane_id();
        int m = 0;
        begin = 0;
        if (l < groups) {                       // offsets that are not a partition of [0, cap] are clamped
            begin = min(max(group_offsets[l], 0), cap);
            m = min(max(group_offsets[l + 1], begin), cap) - begin;
        }
        rows = m;
        xcd = xcd_;
        // Rounds of the launch's workgroups with tiles of 128 and of 64 rows, of which one takes about three quarters of the time (0.59
        // where the weights are not what it waits for).  Measured, the FFN, us, 128 rows always / by this rule: 640, 1024, 2048 and 4000 tokens
        // at 2048 x 768 52.7 / 39.4, 53.2 / 41.0, 54.6 / 46.1, 64.4 / 65.2; 640 and 1024 at 4096 x 1536 105.5 / 101.8, 118.9 / 109.4; at
        // 7168 x 2048 326.6 / 320.4, 358.2 / 364.8 (383.9 where two thirds are assumed).
        auto rounds = [&](int r) {
            const int n = __builtin_amdgcn_readlane(wave_inclusive_sum((m + r - 1) / r), kWave - 1);
            return (int)(((int64_t)n * n_cols + gridDim.x - 1) / gridDim.x);
        };
        size = 3 * (int64_t)rounds(kRingTileRows / 2) < 4 * (int64_t)rounds(kRingTileRows) ? kRingTileRows / 2 : kRingTileRows;
        const int part = m & (size - 1), full = m / size;
        tiles[0] = full + (part > kSmallRows);
        tiles[1] = part > 0 && part <= kSmallRows;
        stride = n_cols < 8 ? 1 : 8;
        first = n_cols < 8 ? 0 : (xcd - l * n_cols) & 7;
        const int cols = n_cols < 8 ? n_cols : (n_cols - first + 7) >> 3;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            incl[c] = wave_inclusive_sum(tiles[c] * cols);
            n[c] = __builtin_amdgcn_readlane(incl[c], kWave - 1);
            if (n_cols < 8) n[c] = (n[c] - xcd + 7) >> 3;
        }
    }
    template <int kClass>
    __device__ __forceinline__ Tile tile(int nth) const {
        const int i = stride == 1 ? nth * 8 + xcd : nth, before = __shfl_up(incl[kClass], 1), from = lane_id() ? before : 0;
        const uint64_t owner = __ballot(from <= i && i < incl[kClass]);            // exactly one lane
        const int o = __ffsll((unsigned long long)owner) - 1;
        const int n = __builtin_amdgcn_readlane(tiles[kClass], o), at = i - __builtin_amdgcn_readlane(from, o), m = __builtin_amdgcn_readlane(rows, o);
        const int c = (uint32_t)at / (uint32_t)n, row = kClass ? m & ~(size - 1) : (at - c * n) * size;
        Tile t;
        t.slot = o;
        t.col = __builtin_amdgcn_readlane(first, o) + c * stride;
        t.row0 = __builtin_amdgcn_readlane(begin, o) + row;
        t.rows = min(size, m - row);
        return t;
    }
};

// The items id, id + step, ... of a class.
template <bool kGateUp, typename OT, int kClass>
__device__ __forceinline__ void fp8_ring_items(const RingArgs& a, const RingList& list, int id, int n, int step) {
    using Source = RingSource<kGateUp, kClass ? 1 : 2>;
    if (id >= n) return;
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Tile t = list.tile<kClass>(id), t1 = id + step < n ? list.tile<kClass>(id + step) : t;
    Source now, then;
    now.set(a, t, Source::raw(a, t), wv);
    typename Source::Raw raw = Source::raw(a, t1);
    for (bool ready = false;; ready = true) {
        const bool more = id + step < n;
        then.set(a, t1, raw, wv);
        const Tile t2 = id + 2 * step < n ? list.tile<kClass>(id + 2 * step) : t1;
        raw = Source::raw(a, t2);
        if constexpr (kClass == 1) fp8_ring_tile<kGateUp, OT, 2>(a, t, now, then, ready, more);
        else if (t.rows <= 64) fp8_ring_tile<kGateUp, OT, 4>(a, t, now, then, ready, more);
        else fp8_ring_tile<kGateUp, OT, 8>(a, t, now, then, ready, more);
        if (!more) return;
        id += step;
        t = t1, t1 = t2;
        now = then;
    }
}

}  // namespace
}  // namespace metro
