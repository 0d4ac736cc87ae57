// Products of a few token rows with 16-row tiles of packed codes where every
// wave has one piece of work (gfx950): the few-token form of the linear with
// adapters (lora_linear.hip) and the experts of a whole MoE layer
// (moe_layer.hip).
//
// Split.  A workgroup owns RT tiles of 16 weight rows (of one matrix, or of
// gate and up); its waves split K, wave w takes the steps w, w + KW, .. of 128
// bytes per row.  A wave issues the loads of its activations and then all its
// weights at once, converts the activations while the weights are under way,
// multiplies and leaves its sums in LDS, where they meet behind one barrier.
// There is no loop over tiles: the launch has a workgroup for each, and the
// hardware starts the next one where one ends.  Reading 92 MB in 8 KB pieces,
// one per wave, took 15.3 us on this card against 17.3 to 21 with persistent
// waves that prefetch, and 16 MB 4.1 against 5.2 to 9.6 (loads only, whole
// 128-byte lines of 8 rows per instruction, launch included): a persistent
// wave ramps its stream up once and waits for its slowest piece at the end.
#pragma once

#include "tile_step.h"

namespace qmlp {
namespace {

// Sums of this wave's steps: acc[m][t] of matrix m and the 16 rows from
// row0 + 16 t on (rows past N give zeros).  The tokens are the operand's rows:
// lane j = lane & 15 supplies row `xrow` of rx (ldx elements apart; zeros
// where it is not `live`).  K % 64 == 0.  Not yet scaled by kTileUnscale.
template <int B, int G, int NM, int RT>
__device__ __forceinline__ void oneshot_products(f32x4_t (&acc)[NM][RT], const Rsrc (&rc)[NM], const Rsrc (&rm)[NM],
                                                 Rsrc rx, int xrow, bool live, int ldx, int K, int N, int row0,
                                                 int first, int ns, int kw, int lane) {
    typedef Lay<B, G> Y;
    const int rb = K * B / 8, ng = K / G;
#pragma unroll
    for (int m = 0; m < NM; ++m)
#pragma unroll
        for (int t = 0; t < RT; ++t) acc[m][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
    for (int gs = first; gs < ns; gs += kw) {
        AOps<B, G> a;
        act_load<B, G>(a, rx, gs, live ? xrow : 0, 1 << 30, ldx, live, lane);
        const int u = gs * 8 + lane_unit<Y::QW == 4>(lane);
        const uint32_t ol = 16 * u < rb ? (uint32_t)((lane & 7) * rb + 16 * u) : kPastEnd;
        const uint32_t ml = (uint32_t)((lane & 15) * ng + gs * Y::GSU + meta_first<Y::GSU>(lane >> 4)) * 4u;
        TileW<B, G> w[NM][RT];
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int m = 0; m < NM; ++m) {
                const int row = row0 + 16 * t;
                w_load<B, G>(w[m][t], rc[m], rm[m], ol, ml, 8u * (uint32_t)rb,
                             row < N ? (uint32_t)row * (uint32_t)rb : kPastEnd,
                             row < N ? (uint32_t)row * (uint32_t)ng * 4u : kPastEnd);
            }
        Corr<B, G> cr;
        act_mask<B, G>(a, gs, K, lane);
        act_convert<B, G>(a);
        group_sums<B, G>(a, cr, lane);
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int m = 0; m < NM; ++m) tile_step<B, G>(w[m][t], a, cr, acc[m][t], ng - gs * Y::GSU, lane);
    }
}

// Steps of a row, and the waves that share them evenly (at most `most`).
inline int oneshot_steps(int K, int bits) { return (K * bits + 1023) / 1024; }
inline int oneshot_waves(int ns, int most) {
    const int per = (ns + most - 1) / most;
    return (ns + per - 1) / per;
}

// Eight values of the activation type (binary16, or bfloat16 where bf) as fp32.
__device__ __forceinline__ void act8(const uint4& v, bool bf, float (&f)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = bf ? __uint_as_float(w[i] << 16) : h2f(w[i] & 0xFFFFu);
        f[2 * i + 1] = bf ? __uint_as_float(w[i] & 0xFFFF0000u) : h2f(w[i] >> 16);
    }
}

// fp32 to the activation type, nearest even.
__device__ __forceinline__ uint16_t act_bits(float v, bool bf) {
    if (!bf)
        return (uint16_t)f2h(v);
    return __builtin_bit_cast(uint16_t, (__bf16)v);
}

}  // namespace
}  // namespace qmlp
