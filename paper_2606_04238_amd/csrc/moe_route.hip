// The router of a mixture-of-experts layer (gfx950; Sec. 5, the MoE decoder's
// routing): l = x Wr^T + b, the k largest of each token, their weights.
//
// The sums are fp64: which expert comes first must not depend on how a sum was
// split, and binary16 or bfloat16 products are exact in fp64, so two experts
// trade places only where their logits agree to about 2^-50 of sum |x w|.
#include "moe_layer.h"
#include "decode_launch.h"
#include "oneshot.h"

#include <float.h>

namespace qmlp {
namespace {

constexpr int kRouteTok = 8;

// A wave: one expert, eight tokens; lanes split d.
__global__ void __launch_bounds__(256) route_logits_kernel(RouteArgs a) {
    const int lane = threadIdx.x & 63, e = blockIdx.x * 4 + (threadIdx.x >> 6), m0 = blockIdx.y * kRouteTok;
    if (e >= a.E)
        return;
    double s[kRouteTok] = {};
    for (int c = lane * 8; c < a.d; c += 512) {
        float w[8];
        act8(*reinterpret_cast<const uint4*>(a.router + (long)e * a.d + c), a.bf, w);
#pragma unroll
        for (int t = 0; t < kRouteTok; ++t) {
            if (m0 + t < a.M) {
                float x[8];
                act8(*reinterpret_cast<const uint4*>(a.x + (long)(m0 + t) * a.d + c), a.bf, x);
#pragma unroll
                for (int i = 0; i < 8; ++i) s[t] = __builtin_fma((double)x[i], (double)w[i], s[t]);
            }
        }
    }
#pragma unroll
    for (int t = 0; t < kRouteTok; ++t) {
        double v = s[t];
#pragma unroll
        for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o, 64);
        if (lane == 0 && m0 + t < a.M)
            a.logits[(long)(m0 + t) * a.E + e] = v + (a.bias ? (double)a.bias[e] : 0.0);
    }
}

// The k largest of a token's logits by one wave, expert e in lane e & 63: ties
// to the lower expert; NaN and -inf are never chosen, +inf counts as the
// largest fp32.  Slots that find nothing: expert -1, weight 0.
__device__ __forceinline__ void route_select(const double* l, int E, int k, int score, int32_t* idx, float* w, int lane) {
    constexpr int N = kMoeExperts / 64;
    const double none = -__builtin_inf();
    double v[N];
    double top = none;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int e = lane + 64 * i;
        v[i] = e < E ? l[e] : none;
        v[i] = v[i] != v[i] ? none : fmin(v[i], (double)FLT_MAX);
        top = fmax(top, v[i]);
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) top = fmax(top, __shfl_xor(top, o, 64));
    float all = 0.0f;
    if (score == QMLP_SCORE_SOFTMAX) {
#pragma unroll
        for (int i = 0; i < N; ++i) all += v[i] == none ? 0.0f : expf((float)(v[i] - top));
#pragma unroll
        for (int o = 32; o; o >>= 1) all += __shfl_xor(all, o, 64);
    }
    double mine = none;                                    // lane j: the j-th chosen
    int me = -1;
    for (int j = 0; j < k; ++j) {
        double b = none;
        int be = kMoeExperts;
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (v[i] > b) {
                b = v[i];
                be = lane + 64 * i;
            }
#pragma unroll
        for (int o = 32; o; o >>= 1) {
            const double ob = __shfl_xor(b, o, 64);
            const int oe = __shfl_xor(be, o, 64);
            if (ob > b || (ob == b && oe < be)) {
                b = ob;
                be = oe;
            }
        }
        if (b == none)
            break;
        if (lane == j) {
            mine = b;
            me = be;
        }
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (be == lane + 64 * i)
                v[i] = none;
    }
    // weights: a softmax of z over the chosen ones, z the logit or log sigmoid(logit); or over all experts
    float g = 0.0f;
    if (score == QMLP_SCORE_SOFTMAX) {
        g = me >= 0 ? expf((float)(mine - top)) / all : 0.0f;
    } else {
        double z = mine;
        if (score == QMLP_SCORE_SIGMOID && me >= 0)
            z = fmin(mine, 0.0) - (double)log1pf(expf(-(float)fabs(mine)));
        double zt = me >= 0 ? z : none;
#pragma unroll
        for (int o = 32; o; o >>= 1) zt = fmax(zt, __shfl_xor(zt, o, 64));
        g = me >= 0 ? expf((float)(z - zt)) : 0.0f;
        float sum = g;
#pragma unroll
        for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o, 64);
        g = me >= 0 ? g / sum : 0.0f;
    }
    if (lane < k) {
        idx[lane] = me;
        w[lane] = g;
    }
}

__global__ void __launch_bounds__(256) route_select_kernel(RouteArgs a) {
    const int m = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (m < a.M)
        route_select(a.logits + (long)m * a.E, a.E, a.k, a.score, a.idx + (long)m * a.k, a.w + (long)m * a.k, threadIdx.x & 63);
}

}  // namespace

hipError_t launch_route(const RouteArgs& a, hipStream_t st) {
    route_logits_kernel<<<dim3((unsigned)(a.E + 3) / 4, (unsigned)(a.M + kRouteTok - 1) / kRouteTok), 256, 0, st>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess)
        return e;
    route_select_kernel<<<(unsigned)(a.M + 3) / 4, 256, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace qmlp
