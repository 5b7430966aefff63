// One tile of a product of e4m3 rows with e4m3 weights, K split over the four waves of a workgroup:
//     y[r][n] = sum over blocks b of  xs[r][b] * ws[n / 128][b] * sum over k in b of x[r][k] * w[n][k]
// A step is a block: 128 bytes of every row, a cache line.  Loads take whole lines (8 rows x 128 bytes), and a step passes through
// the wave's own LDS to get operand layout: 128 bytes per row, its 16-byte piece p at place p ^ (row & 7).  Lane (r16, q) supplies
// pieces q and q + 4 of weight row r16 and of row r16; which k sits in which operand slot does not matter as long as both sides
// agree.  Four v_mfma_f32_16x16x32_bf16 sum a block, and the sum is added to the running one times the block's two scales.  The waves
// take steps w, w + 4, ... and add their sums up through LDS in a fixed order.
// The values are widened to bf16, which is exact, instead of using the matrix cores' e4m3 products: those align the products of a
// block to the largest and drop what is below about 2^-13 of it (sums of 128 products of normal values off by 1.5e-5 rms; 1e-8 with
// bf16 operands).  At 4.5 cycles a pair and wave, widening the operands of a step and its products are some 640 cycles for 8 KB of
// weights, a fifth of the time in which HBM delivers those to the four SIMDs of a CU.
//
// kQuantX: the rows are fp32 and are quantized on the way to LDS, a block of a row by 8 lanes; that saves a launch between the
// two products of the FFN where few rows are read by few column tiles.
// kRagged: any K and number of columns.  Rows are read in whole 16-byte pieces; bytes past K are zeroed in both operands, pieces past
// the row's last one are not read.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>
#include <utility>

#include "ffn_common.h"
#include "fp8_common.h"

namespace metro {
namespace {

constexpr int kFp8Threads = 256;
constexpr int kFp8Blocks = 4;               // 16-row weight blocks of a tile: 64 columns, or 32 gate and 32 up columns

struct Fp8Args {
    const void* x;              // e4m3 rows, or fp32 rows to be quantized (kQuantX)
    const float* xs;            // [rows of x, blocks of K]; not with kQuantX
    const int32_t* perm_pair;   // row r is that of token perm_pair[r] / k; null: row r itself
    const int32_t* group_offsets;
    const uint8_t* w;           // [groups, n_out (gate/up: 2 n_out), K], rows ldw bytes apart
    const float* ws;            // [groups, blocks of n_out (gate/up: twice), blocks of K]
    void* dst;                  // [cap, n_out], rows ldd elements apart
    int64_t ldx;                // elements
    int T, k, groups, K, n_out, ldw, ldd;
    int ntn;                    // column tiles
};

struct Fp8Lds {
    char* mem;                  // per wave 8 KB for a step of weights, 8 KB for a step of rows; then the partial sums
    float* scale;               // per wave 64 row scales (kQuantX)
    __device__ __forceinline__ char* wave_w(int wave) const { return mem + wave * 16384; }
    __device__ __forceinline__ char* wave_x(int wave) const { return mem + wave * 16384 + 8192; }
    __device__ __forceinline__ float* wave_scale(int wave) const { return scale + wave * 64; }
    __device__ __forceinline__ floatx4* part(int u) const { return reinterpret_cast<floatx4*>(mem) + u * 256; }
};

// x * mask of the `valid` first bytes of a 16-byte piece (any int)
__device__ __forceinline__ u32x4 keep_bytes(u32x4 v, int valid) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int n = min(max(valid - 4 * e, 0), 4);
        v[e] = n == 0 ? 0u : v[e] & (0xffffffffu >> (8 * (4 - n)));
    }
    return v;
}

// Eight values as bf16, exactly.
__device__ __forceinline__ bf16x8 widen_e4m3(uint32_t lo, uint32_t hi) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    bf16x8 r;
    const uint32_t word[2] = {lo, hi};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(word[i], 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(word[i], 1.f, true);
        r[4 * i] = a[0], r[4 * i + 1] = a[1], r[4 * i + 2] = b[0], r[4 * i + 3] = b[1];
    }
    return r;
}

template <typename OT>
__device__ __forceinline__ void store_columns(OT* out, int left, bool vec, const float (&o)[4]) {
    if (vec) {
        if (left > 0) {
            if constexpr (sizeof(OT) == 4) *reinterpret_cast<floatx4*>(out) = floatx4{o[0], o[1], o[2], o[3]};
            else *reinterpret_cast<u32x2*>(out) = u32x2{pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3])};
        }
    } else {
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            if (v >= left) continue;
            if constexpr (sizeof(OT) == 4) out[v] = o[v];
            else out[v] = __builtin_bit_cast(OT, (uint16_t)(pack_bf16x2(o[v], 0.f) & 0xffffu));
        }
    }
}

template <bool kGateUp, bool kQuantX, typename OT, int MT, int DEPTH, bool kRagged>
__device__ __forceinline__ void fp8_tile(const Fp8Args& a, const Tile t, const Fp8Lds lds) {
    constexpr int NB = kFp8Blocks, kUnits = kGateUp ? NB / 2 : NB;
    constexpr int kXLoads = kQuantX ? MT * 8 : MT * 2;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r16 = lane & 15, q = lane >> 4, r8 = lane >> 3, c8 = lane & 7;
    const int nb = blocks_of(a.K), n_steps = nb, mine = (n_steps - wv + 3) >> 2;
    const int mt_count = (t.rows + 15) >> 4, col0 = t.col * kUnits * 16;
    const int row_blocks = blocks_of(a.n_out) * (kGateUp ? 2 : 1);
    const int k_end = kRagged ? (int)up16(a.K) : a.K;          // bytes of a row that are read
    char* const lds_w = lds.wave_w(wv);
    char* const lds_x = lds.wave_x(wv);
    float* const lds_s = lds.wave_scale(wv);

    auto w_row0 = [&](int b) { return (kGateUp && b >= kUnits ? a.n_out : 0) + col0 + (b % kUnits) * 16; };
    auto x_row = [&](int r) {                                       // past the tile: its last row
        const int row = t.row0 + min(r, t.rows - 1);
        return a.perm_pair ? min(max(a.perm_pair[row] / a.k, 0), a.T - 1) : row;
    };
    const uint8_t* wslot = a.w + (size_t)t.slot * (size_t)(kGateUp ? 2 * (int64_t)a.n_out : a.n_out) * a.ldw;
    // the scale that this lane loads: gate by the lower half of the wave, up by the upper; a lane-dependent address keeps the load a
    // vector load, in order with the others
    const float* ws = a.ws + ((size_t)t.slot * row_blocks + col0 / kBlock + (kGateUp && lane >= 32 ? blocks_of(a.n_out) : 0)) * nb;

    uint32_t xr[kQuantX ? MT * 2 : kXLoads], sr[kQuantX ? 1 : MT];
#pragma unroll
    for (int i = 0; i < MT * 2; ++i) xr[i] = (uint32_t)x_row(i * 8 + r8);
    if constexpr (!kQuantX) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) sr[mt] = (uint32_t)x_row(mt * 16 + r16);
    }
    int wr[kRagged ? NB : 1][2];
    if constexpr (kRagged) {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int h = 0; h < 2; ++h) {                           // past the last column: that one
                const int c = (b % kUnits) * 16 + h * 8 + r8;
                wr[b][h] = (kGateUp && b >= kUnits ? a.n_out : 0) + min(col0 + c, a.n_out - 1);
            }
    }

    u32x4 w[DEPTH][NB][2], x[DEPTH][kXLoads];
    float wsc[DEPTH], xsc[DEPTH][kQuantX ? 1 : MT];
    const uint32_t w_lane = (uint32_t)r8 * (uint32_t)a.ldw + c8 * 16;
    auto step_of = [&](int s) { return wv + 4 * min(s, mine - 1); };
    // Past the wave's last step every lane takes the same bytes of a line that is there already.
    auto load = [&](auto U, int s) {
        constexpr int buf = decltype(U)::value % DEPTH;
        const int step = step_of(s);
        const bool real = s < mine;
        const int k = step * kBlock + c8 * 16;
#pragma unroll
        for (int i = 0; i < MT * 2; ++i) {
            if constexpr (kQuantX) {
                const float* p = reinterpret_cast<const float*>(a.x) + (size_t)xr[i] * a.ldx;
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const int f = step * kBlock + v * 32 + c8 * 4;
                    x[buf][i * 4 + v] = *reinterpret_cast<const u32x4*>(p + (real ? kRagged ? min(f, k_end - 4) : f : 0));
                }
            } else {
                const uint8_t* p = reinterpret_cast<const uint8_t*>(a.x) + (size_t)xr[i] * a.ldx;
                x[buf][i] = *reinterpret_cast<const u32x4*>(p + (real ? kRagged ? min(k, k_end - 16) : k : 0));
            }
        }
        if constexpr (!kQuantX) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) xsc[buf][mt] = a.xs[(size_t)sr[mt] * nb + step];
        }
        wsc[buf] = ws[step];
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if constexpr (kRagged)
                    w[buf][b][h] = *reinterpret_cast<const u32x4*>(wslot + (size_t)(uint32_t)wr[b][h] * (uint32_t)a.ldw + min(k, k_end - 16));
                else
                    w[buf][b][h] = *reinterpret_cast<const u32x4*>(wslot + (size_t)(w_row0(b) + h * 8) * a.ldw + (size_t)step * kBlock + (real ? w_lane : 0u));
            }
    };
    auto place = [](int r, int p) { return r * 128 + ((p ^ (r & 7)) * 16); };
    auto store = [&](auto U, int s) {
        constexpr int buf = decltype(U)::value % DEPTH;
        const int step = step_of(s), k = step * kBlock + c8 * 16;
        const bool last = kRagged && step == n_steps - 1;           // uniform
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                u32x4 v = w[buf][b][h];
                if (last) v = keep_bytes(v, a.K - k);
                *reinterpret_cast<u32x4*>(lds_w + b * 2048 + h * 1024 + place(r8, c8)) = v;
            }
#pragma unroll
        for (int i = 0; i < MT * 2; ++i) {
            if constexpr (kQuantX) {
                float f[16];
#pragma unroll
                for (int v = 0; v < 4; ++v)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        f[v * 4 + e] = __uint_as_float(x[buf][i * 4 + v][e]);
                        if (last && step * kBlock + v * 32 + c8 * 4 + e >= a.K) f[v * 4 + e] = 0.f;
                    }
                uint32_t m = 0;
#pragma unroll
                for (int e = 0; e < 16; ++e) m = max(m, magnitude(f[e]));
                const BlockScale sc = block_scale(group_max<8>(m));
                if (c8 == 0) lds_s[i * 8 + r8] = sc.scale;
#pragma unroll
                for (int v = 0; v < 4; ++v)                         // k = v * 32 + 4 c8 ..: piece 2 v + c8 / 4, word c8 % 4
                    *reinterpret_cast<uint32_t*>(lds_x + i * 1024 + place(r8, 2 * v + (c8 >> 2)) + (c8 & 3) * 4) =
                        pack_e4m3(f[v * 4] * sc.inverse, f[v * 4 + 1] * sc.inverse, f[v * 4 + 2] * sc.inverse, f[v * 4 + 3] * sc.inverse);
            } else {
                u32x4 v = x[buf][i];
                if (last) v = keep_bytes(v, a.K - k);
                *reinterpret_cast<u32x4*>(lds_x + i * 1024 + place(r8, c8)) = v;
            }
        }
    };
    floatx4 acc[NB][MT];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) acc[b][mt] = floatx4{0.f, 0.f, 0.f, 0.f};
    struct Fragment { bf16x8 part[4]; };
    auto fragment = [&](const char* p) {
        Fragment f;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const u32x4 v = *reinterpret_cast<const u32x4*>(p + place(r16, j * 4 + q));
            f.part[2 * j] = widen_e4m3(v[0], v[1]);
            f.part[2 * j + 1] = widen_e4m3(v[2], v[3]);
        }
        return f;
    };
    auto consume = [&](float wscale, const float (&xscale)[kQuantX ? 1 : MT]) {
        const float g = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(wscale), 0));
        const float u = kGateUp ? __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(wscale), 32)) : g;
        Fragment xf[MT];
        float sx[MT];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            xf[mt] = fragment(lds_x + mt * 2048);
            sx[mt] = kQuantX ? lds_s[mt * 16 + r16] : xscale[kQuantX ? 0 : mt];
        }
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const Fragment wf = fragment(lds_w + b * 2048);
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                floatx4 p = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < 4; ++c) p = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf.part[c], xf[mt].part[c], p, 0, 0, 0);
                const float f = sx[mt] * (b < kUnits ? g : u);
#pragma unroll
                for (int v = 0; v < 4; ++v) acc[b][mt][v] = fmaf(p[v], f, acc[b][mt][v]);
            }
        }
    };
    auto wave_fence = [] { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); };

    if (mine > 0) {
        run_steps(std::make_integer_sequence<int, DEPTH>{}, load, 0);
        auto step = [&](auto U, int s) {
            constexpr int buf = decltype(U)::value % DEPTH;
            const float wscale = wsc[buf];
            float xscale[kQuantX ? 1 : MT] = {};
            if constexpr (!kQuantX) {
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) xscale[mt] = xsc[buf][mt];
            }
            wave_fence();
            store(U, s);
            wave_fence();
            __builtin_amdgcn_sched_barrier(0);              // the loads refill the registers just stored, none earlier
            load(U, s + DEPTH);
            __builtin_amdgcn_sched_barrier(0);
            consume(wscale, xscale);
        };
        auto final_step = [&](auto U, int s) {
            constexpr int buf = decltype(U)::value % DEPTH;
            wave_fence();
            store(U, s);
            wave_fence();
            consume(wsc[buf], xsc[buf]);
        };
        int s = 0;
        for (; s + DEPTH < mine; s += DEPTH) run_steps(std::make_integer_sequence<int, DEPTH>{}, step, s);
        run_steps_tail(std::make_integer_sequence<int, DEPTH>{}, final_step, s, mine);
    }
    __syncthreads();                                        // the partial sums take the LDS of all waves

#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
            if (mt < mt_count) lds.part(b * MT + mt)[wv * 64 + lane] = acc[b][mt];
    __syncthreads();
    auto total = [&](int u) {
        const floatx4* p = lds.part(u) + lane;
        floatx4 s = p[0];
#pragma unroll
        for (int o = 1; o < 4; ++o) s += p[o * 64];
        return s;
    };
    const bool vec = !kRagged || a.n_out % 4 == 0;          // uniform; dst and its rows are then 4-element aligned
#pragma unroll
    for (int u0 = 0; u0 < kUnits * MT; u0 += 4) {
        const int u = u0 + wv, b = u / MT, mt = u % MT;     // (output block, row sub-tile) of this wave
        if (u >= kUnits * MT || mt >= mt_count) continue;
        const int row = mt * 16 + r16, col = col0 + b * 16 + q * 4;
        float o[4];
        const floatx4 g = total(u);
        if (kGateUp) {
            const floatx4 h = total(u + kUnits * MT);
#pragma unroll
            for (int v = 0; v < 4; ++v) o[v] = g[v] / (1.0f + expf(-g[v])) * h[v];
        } else {
#pragma unroll
            for (int v = 0; v < 4; ++v) o[v] = g[v];
        }
        if (row < t.rows) store_columns(reinterpret_cast<OT*>(a.dst) + (size_t)(t.row0 + row) * a.ldd + col, a.n_out - col, vec, o);
    }
}

}  // namespace
}  // namespace metro
