// The choice of a token's experts from its logits, by one wave (gfx950): for the
// router alone (moe_route.hip) and the whole layer (moe_layer.hip).
#pragma once

#include "decode_common.h"
#include "moe_layer.h"

#include <float.h>

namespace qmlp {
namespace {

// v of the lane that DPP control CTRL names, or v itself where it names none.
template <int CTRL, int ROWS>
__device__ __forceinline__ double dpp_f64(double v) {
    const uint2 u = __builtin_bit_cast(uint2, v);
    return __builtin_bit_cast(double, make_uint2((uint32_t)__builtin_amdgcn_update_dpp((int)u.x, (int)u.x, CTRL, ROWS, 0xF, false),
                                                 (uint32_t)__builtin_amdgcn_update_dpp((int)u.y, (int)u.y, CTRL, ROWS, 0xF, false)));
}
__device__ __forceinline__ double lane_f64(double v, int lane) {
    const uint2 u = __builtin_bit_cast(uint2, v);
    return __builtin_bit_cast(double, make_uint2((uint32_t)__builtin_amdgcn_readlane((int)u.x, lane),
                                                 (uint32_t)__builtin_amdgcn_readlane((int)u.y, lane)));
}
// Over the wave: the largest v (none NaN), and the sum.
__device__ __forceinline__ double wave_max(double v) {
    v = fmax(v, dpp_f64<0xB1, 0xF>(v));                    // quad_perm: lanes 1 and 2 away
    v = fmax(v, dpp_f64<0x4E, 0xF>(v));
    v = fmax(v, dpp_f64<0x141, 0xF>(v));                   // row_half_mirror, row_mirror
    v = fmax(v, dpp_f64<0x140, 0xF>(v));
    v = fmax(v, dpp_f64<0x142, 0xF>(v));                   // row_bcast 15 and 31: into the rows that follow
    v = fmax(v, dpp_f64<0x143, 0xF>(v));
    return lane_f64(v, 63);
}
__device__ __forceinline__ double wave_sum(double v) {
    v += dpp_f64<0xB1, 0xF>(v);
    v += dpp_f64<0x4E, 0xF>(v);
    v += dpp_f64<0x141, 0xF>(v);
    v += dpp_f64<0x140, 0xF>(v);
    return (lane_f64(v, 0) + lane_f64(v, 16)) + (lane_f64(v, 32) + lane_f64(v, 48));
}

// Lane j < k: the j-th chosen expert and its weight; -1 and 0 where there is none.
struct Chosen {
    int e;
    float w;
};
// The k largest of the logits l[0 .. E): expert e in lane e & 63; ties to the
// lower expert; NaN and -inf are never chosen, +inf counts as the largest fp32.
__device__ __forceinline__ Chosen route_select(const double* l, int E, int k, int score, int lane) {
    constexpr int N = kMoeExperts / 64;
    const double none = -__builtin_inf();
    double v[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int e = lane + 64 * i;
        v[i] = none;
        if (64 * i < E)                                    // (the same for every lane: no turns are spent past E)
            v[i] = e < E ? l[e] : none;
    }
    double top = none;
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (64 * i < E) {
            v[i] = v[i] != v[i] ? none : fmin(v[i], (double)FLT_MAX);
            top = fmax(top, v[i]);
        }
    float all = 0.0f;
    if (score == QMLP_SCORE_SOFTMAX) {
        const double first = wave_max(top);
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (64 * i < E)
                all += v[i] == none ? 0.0f : expf((float)(v[i] - first));
        all = group_sum<64>(all);
    }
    double mine = none, best = none;                       // lane j: the j-th chosen
    int me = -1;
    for (int j = 0; j < k; ++j) {
        const double b = wave_max(top);
        if (b == none)
            break;
        if (j == 0)
            best = b;
        int e = -1;
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (64 * i < E && e < 0) {
                const uint64_t at = __ballot(v[i] == b);
                if (at) {
                    e = 64 * i + __builtin_ctzll(at);
                    if (lane == (e & 63))
                        v[i] = none;
                }
            }
        if (lane == (e & 63)) {
            top = none;
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (64 * i < E)
                    top = fmax(top, v[i]);
        }
        if (lane == j) {
            mine = b;
            me = e;
        }
    }
    // weights: a softmax of z over the chosen ones, z the logit or log sigmoid(logit), both largest for the
    // first; or a softmax over all experts
    if (score == QMLP_SCORE_SOFTMAX)
        return {me, me >= 0 ? expf((float)(mine - best)) / all : 0.0f};
    auto z = [&](double t) {
        return score == QMLP_SCORE_SIGMOID ? fmin(t, 0.0) - (double)log1pf(expf(-(float)fabs(t))) : t;
    };
    const float g = me >= 0 ? expf((float)(z(mine) - z(best))) : 0.0f, sum = group_sum<64>(g);
    return {me, me >= 0 ? g / sum : 0.0f};
}

}  // namespace
}  // namespace qmlp
