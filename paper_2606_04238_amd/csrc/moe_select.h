// The choice of a token's experts from its logits, by one wave (gfx950): for the
// router alone (moe_route.hip) and the whole layer (moe_layer.hip).
#pragma once

#include "decode_common.h"
#include "moe_layer.h"

#include <float.h>

namespace qmlp {
namespace {

template <int CTRL>
__device__ __forceinline__ double dpp_f64(double v) {
    const uint2 u = __builtin_bit_cast(uint2, v);
    return __builtin_bit_cast(double, make_uint2(dpp_u32<CTRL>(u.x), dpp_u32<CTRL>(u.y)));
}
__device__ __forceinline__ double lane_f64(double v, int lane) {
    const uint2 u = __builtin_bit_cast(uint2, v);
    return __builtin_bit_cast(double, make_uint2((uint32_t)__builtin_amdgcn_readlane((int)u.x, lane),
                                                 (uint32_t)__builtin_amdgcn_readlane((int)u.y, lane)));
}
// Over the wave, the same in every lane: the sum of v.
__device__ __forceinline__ double wave_sum(double v) {
    v += dpp_f64<DPP_QUAD_XOR1>(v);
    v += dpp_f64<DPP_QUAD_XOR2>(v);
    v += dpp_f64<DPP_HALF_MIRROR>(v);
    v += dpp_f64<DPP_MIRROR>(v);
    return (lane_f64(v, 0) + lane_f64(v, 16)) + (lane_f64(v, 32) + lane_f64(v, 48));
}

// Logits as 64-bit keys in their order, in two halves; 0 for what is never chosen,
// NaN and -inf.  +inf counts as the largest fp32.
struct Key {
    uint32_t hi, lo;
};
__device__ __forceinline__ Key key_of(double v) {
    const uint2 u = __builtin_bit_cast(uint2, fmin(v, (double)FLT_MAX));
    const bool neg = (int)u.y < 0, any = v > -__builtin_inf();
    return {any ? (neg ? ~u.y : u.y | 0x80000000u) : 0u, any ? (neg ? ~u.x : u.x) : 0u};
}
__device__ __forceinline__ double value_of(uint32_t hi, uint32_t lo) {
    const bool neg = (int)hi >= 0;
    return __builtin_bit_cast(double, neg ? make_uint2(~lo, ~hi) : make_uint2(lo, hi & 0x7FFFFFFFu));
}

// Lane j < k: the j-th chosen expert and its weight; -1 and 0 where there is none.
struct Chosen {
    int e;
    float w;
};
// The largest of the keys (expert e in lane e & 63, place e / 64, N places), taken out: its
// expert, lower ones first among equals, and its halves; -1 where none is left.
// The high halves decide, the low ones only between equal high ones.
template <int N>
__device__ __forceinline__ int take_largest(Key (&key)[N], int lane, uint32_t& hi, uint32_t& lo) {
    uint32_t t = 0;
#pragma unroll
    for (int i = 0; i < N; ++i)
        t = max(t, key[i].hi);
    hi = wave_max(t);
    lo = 0;
    if (hi == 0)
        return -1;
    int e = -1, some = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const uint64_t at = __ballot(key[i].hi == hi);
        if (at && e < 0) {
            e = 64 * i + __builtin_ctzll(at);
            lo = (uint32_t)__builtin_amdgcn_readlane((int)key[i].lo, e & 63);
        }
        some += __builtin_popcountll(at);
    }
    if (some > 1) {
        t = 0;
#pragma unroll
        for (int i = 0; i < N; ++i)
            t = max(t, key[i].hi == hi ? key[i].lo : 0u);
        lo = wave_max(t);
        e = -1;
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (e < 0) {
                const uint64_t at = __ballot(key[i].hi == hi && key[i].lo == lo);
                if (at)
                    e = 64 * i + __builtin_ctzll(at);
            }
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (e == 64 * i + lane)
            key[i].hi = key[i].lo = 0;
    return e;
}

// The k largest of the logits v (expert e in lane e & 63, place e / 64; anything past
// E).  Where SURE is false the logits may be off by `off`, and where that could change
// the choice or its order, the experts in question (all, where off is not finite)
// are written to list (E entries, this wave's), from which exact(n, put) forms their
// logits and hands each to put(expert, logit).
template <bool SURE, int N, typename EXACT>
__device__ __forceinline__ Chosen route_select(double (&v)[N], int E, int k, int score, int lane, double off, int16_t* list,
                                               EXACT exact) {
    const double none = -__builtin_inf();
    Key key[N];
    double mine = none, first = none;                      // lane j: the j-th chosen
    int me = -1;
    bool sure = SURE || off == 0.0;
    uint32_t in = ~0u;                                     // bit i: expert lane + 64 i may be chosen
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (lane + 64 * i >= E)
            v[i] = none;
    for (;;) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            key[i] = key_of(SURE || (in >> i & 1) ? v[i] : none);
        mine = first = none;
        me = -1;
        for (int j = 0; j < (sure ? k : k + 1); ++j) {
            uint32_t hi, lo;
            const int e = take_largest(key, lane, hi, lo);
            if (e < 0)
                break;
            const double b = value_of(hi, lo);
            if (j == 0)
                first = b;
            if (lane == j) {
                mine = b;
                me = e;
            }
        }
        if constexpr (SURE)
            break;
        // pairs that are too close: chosen experts beside one are in question, and, where it is the k-th and the
        // next, every expert down to 2 off below the k-th
        const bool all = !(off < __builtin_inf());
        const double above = __shfl_up(mine, 1, 64), edge = lane_f64(mine, k - 1), from = edge - 2.0 * off;
        const uint64_t pairs = __ballot(lane > 0 && lane <= k && me >= 0 && above - mine <= 2.0 * off);
        if (sure || (!all && pairs == 0))
            break;
        sure = true;
        uint32_t redo = 0;
        for (uint64_t at = (pairs | pairs >> 1) & ((1ull << k) - 1); at; at &= at - 1) {
            const int e = __builtin_amdgcn_readlane(me, __builtin_ctzll(at));
            redo |= lane == (e & 63) ? 1u << (e >> 6) : 0u;
        }
        int n = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const double u = fmin(v[i], (double)FLT_MAX);
            const bool near = u >= from;
            const bool q = lane + 64 * i < E && (all || (redo >> i & 1) || ((pairs >> k & 1) && near && u <= edge));
            const uint64_t at = __ballot(q);
            if (q)
                list[n + __builtin_amdgcn_mbcnt_hi((uint32_t)(at >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)at, 0))] = (int16_t)(lane + 64 * i);
            n += __builtin_popcountll(at);
            in = all || near ? in : in & ~(1u << i);
        }
        __asm__ volatile("s_waitcnt lgkmcnt(0)" ::: "memory");         // (the list is this wave's own)
        exact(n, [&](int e, double s) {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (e == lane + 64 * i)
                    v[i] = s;
        });
    }
    me = lane < k ? me : -1;
    // weights: a softmax over all experts, or of z over the chosen ones, z the logit or log sigmoid(logit);
    // both are largest for the first
    if (score == QMLP_SCORE_SOFTMAX) {
        float all = 0.0f;
#pragma unroll
        for (int i = 0; i < N; ++i)
            all += v[i] > none ? expf((float)(fmin(v[i], (double)FLT_MAX) - first)) : 0.0f;
        all = group_sum<64>(all);
        return {me, me >= 0 ? expf((float)(mine - first)) / all : 0.0f};
    }
    auto z = [&](double t) {
        return score == QMLP_SCORE_SIGMOID ? fmin(t, 0.0) - (double)log1pf(expf(-(float)fabs(t))) : t;
    };
    const float g = me >= 0 ? expf((float)(z(mine) - z(first))) : 0.0f, sum = group_sum<64>(g);
    return {me, me >= 0 ? g / sum : 0.0f};
}
// Of right logits l[0 .. E).
template <int N>
__device__ __forceinline__ Chosen route_select(const double* l, int E, int k, int score, int lane) {
    double v[N];
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = l[min(lane + 64 * i, E - 1)];
    return route_select<true>(v, E, k, score, lane, 0.0, nullptr, [](int, auto) {});
}
// (Places past the last expert cost turns all the same: 64 tokens of 32 experts in one
// workgroup 17.8 us with eight places, 10.7 with one.)
__device__ __forceinline__ Chosen route_select(const double* l, int E, int k, int score, int lane) {
    return E <= 64 ? route_select<1>(l, E, k, score, lane) : E <= 128 ? route_select<2>(l, E, k, score, lane)
                   : route_select<kMoeExperts / 64>(l, E, k, score, lane);
}

}  // namespace
}  // namespace qmlp
