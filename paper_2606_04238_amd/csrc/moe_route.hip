// The router of a mixture-of-experts layer (gfx950; Sec. 5, the MoE decoder's
// routing): l = x Wr^T + b, the k largest of each token, their weights.
//
// The sums are fp64: which expert comes first must not depend on how a sum was
// split, and binary16 or bfloat16 products are exact in fp64, so two experts
// trade places only where their logits agree to about 2^-50 of sum |x w|.
#include "moe_layer.h"
#include "moe_select.h"
#include "oneshot.h"

namespace qmlp {
namespace {

typedef double f64x4_t __attribute__((ext_vector_type(4)));

constexpr int kRouteTok = 8, kRouteWaves = 4;

// Few tokens: a workgroup owns an expert and eight tokens and issues all its loads,
// 16 bytes a lane, before the first product.
__global__ void __launch_bounds__(kRouteWaves * 64) route_few_kernel(RouteArgs a) {
    constexpr int N = 2, step = kRouteWaves * 64 * 8;
    __shared__ double red[kRouteWaves][kRouteTok];
    const int tid = threadIdx.x, e = blockIdx.x, m0 = blockIdx.y * kRouteTok, nt = min(kRouteTok, a.M - m0);
    const uint16_t *wr = a.router + (long)e * a.d, *xr = a.x + (long)m0 * a.d;
    const double bias = a.bias ? (double)a.bias[e] : 0.0;
    double s[kRouteTok] = {};
    for (int c = tid * 8; c < a.d; c += N * step) {
        uint4 wv[N], xv[N][kRouteTok];
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (c + i * step < a.d) {
                wv[i] = ld16(wr + c + i * step);
#pragma unroll
                for (int t = 0; t < kRouteTok; ++t)
                    if (t < nt)
                        xv[i][t] = ld16(xr + (long)t * a.d + c + i * step);
            }
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (c + i * step < a.d) {
                float w[8];
                act8(wv[i], a.bf, w);
#pragma unroll
                for (int t = 0; t < kRouteTok; ++t)
                    if (t < nt) {
                        float x[8];
                        act8(xv[i][t], a.bf, x);
#pragma unroll
                        for (int k = 0; k < 8; ++k) s[t] = __builtin_fma((double)x[k], (double)w[k], s[t]);
                    }
            }
    }
#pragma unroll
    for (int t = 0; t < kRouteTok; ++t)
        if (t < nt) {
            const double v = wave_sum(s[t]);
            if ((tid & 63) == 0)
                red[tid >> 6][t] = v;
        }
    __syncthreads();
    if (tid < nt) {
        double v = red[0][tid];
#pragma unroll
        for (int w = 1; w < kRouteWaves; ++w) v += red[w][tid];
        a.logits[(long)(m0 + tid) * a.E + e] = v + bias;
    }
}

// Many tokens: a workgroup owns 32 tokens and 32 experts, its waves split d, and
// each step of 32 elements is 8 k-steps of v_mfma_f64_16x16x4_f64: lane 16 q + j
// loads 8 elements of row j from 8 q on and gives them one after another (the
// same order on both sides, so which k-step an element lands in does not matter).
constexpr int kManyWaves = 8;
__global__ void __launch_bounds__(kManyWaves * 64) route_many_kernel(RouteArgs a) {
    __shared__ double red[kManyWaves][4][64][4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, j = lane & 15, q = lane >> 4;
    const int m0 = blockIdx.y * 32, e0 = blockIdx.x * 32;
    const uint16_t *xr[2], *wr[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        xr[i] = a.x + (long)min(m0 + 16 * i + j, a.M - 1) * a.d;
        wr[i] = a.router + (long)min(e0 + 16 * i + j, a.E - 1) * a.d;
    }
    f64x4_t acc[2][2] = {};
    uint4 xv[2], wv[2];
    auto load = [&](int k) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            xv[i] = k < a.d ? ld16(xr[i] + k) : make_uint4(0, 0, 0, 0);
            wv[i] = k < a.d ? ld16(wr[i] + k) : make_uint4(0, 0, 0, 0);
        }
    };
    load(wave * 32 + 8 * q);
    for (int k = wave * 32; k < a.d; k += kManyWaves * 32) {
        float x[2][8], w[2][8];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            act8(xv[i], a.bf, x[i]);
            act8(wv[i], a.bf, w[i]);
        }
        load(k + kManyWaves * 32 + 8 * q);
#pragma unroll
        for (int s = 0; s < 8; ++s)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int n = 0; n < 2; ++n)
                    acc[i][n] = __builtin_amdgcn_mfma_f64_16x16x4f64((double)x[i][s], (double)w[n][s], acc[i][n], 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int v = 0; v < 4; ++v) red[wave][2 * i + n][lane][v] = acc[i][n][v];
    __syncthreads();
    // item: token 16 i + 4 v + q, expert 16 n + j
    for (int it = tid; it < 1024; it += kManyWaves * 64) {
        const int c = it >> 8, l = it & 63, v = (it >> 6) & 3;
        double s = red[0][c][l][v];
#pragma unroll
        for (int w = 1; w < kManyWaves; ++w) s += red[w][c][l][v];
        const int m = m0 + 16 * (c >> 1) + 4 * v + (l >> 4), e = e0 + 16 * (c & 1) + (l & 15);
        if (m < a.M && e < a.E)
            a.logits[(long)m * a.E + e] = s + (a.bias ? (double)a.bias[e] : 0.0);
    }
}

__global__ void __launch_bounds__(256) route_select_kernel(RouteArgs a) {
    const int m = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (m >= a.M)
        return;
    const Chosen c = route_select(a.logits + (long)m * a.E, a.E, a.k, a.score, lane);
    if (lane < a.k) {
        a.idx[(long)m * a.k + lane] = c.e;
        a.w[(long)m * a.k + lane] = c.w;
    }
}

}  // namespace

hipError_t launch_route_logits(const RouteArgs& a, hipStream_t st) {
    // (us, few and many: d = 4096, E = 128: M = 64 14.9 and 48.4, 256 42.6 and 48.4, 2048 262 and 50.8; d = 2880,
    // E = 32: M = 256 13.6 and 36.1, 2048 66.1 and 36.2)
    if (a.M < 512)
        route_few_kernel<<<dim3((unsigned)a.E, (unsigned)(a.M + kRouteTok - 1) / kRouteTok), kRouteWaves * 64, 0, st>>>(a);
    else
        route_many_kernel<<<dim3((unsigned)(a.E + 31) / 32, (unsigned)(a.M + 31) / 32), kManyWaves * 64, 0, st>>>(a);
    return hipGetLastError();
}
hipError_t launch_route(const RouteArgs& a, hipStream_t st) {
    const hipError_t e = launch_route_logits(a, st);
    if (e != hipSuccess)
        return e;
    route_select_kernel<<<(unsigned)(a.M + 3) / 4, 256, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace qmlp
