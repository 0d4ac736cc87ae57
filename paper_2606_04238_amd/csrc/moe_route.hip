// The router of a mixture-of-experts layer (gfx950; Sec. 5, the MoE decoder's
// routing): l = x Wr^T + b, the k largest of each token, their weights.
//
// Which expert comes first must not depend on how a sum was split.  Binary16 and
// bfloat16 products are exact in fp64, so two experts of fp64 sums trade places
// only where their logits agree to about 2^-50 of sum |x w|: few tokens are summed
// so.  Many tokens are multiplied by the 16-bit matrix instructions, their sums of
// 32 products added in fp64; the choice (moe_select.h) forms in fp64 again the
// logits that could change places by what those sums may be off.
#include "moe_layer.h"
#include "moe_select.h"
#include "oneshot.h"

namespace qmlp {
namespace {

constexpr int kRouteTok = 4, kRouteWaves = 4;

// Few tokens: a workgroup owns an expert and four tokens and issues all its loads,
// 16 bytes a lane, before the first product.  Its time is that of one trip to memory:
// one token of 2880 and 32 experts 3.6 us, eight 5.6 (8.9 with eight tokens a
// workgroup), 64 of 4096 and 128 experts 13.9.
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

// Many tokens: a workgroup owns 32 tokens and 32 experts, its waves split d in steps
// of 32, kManyAhead of them loaded at once: lane 16 q + j takes 8 elements of row j from
// 8 q on.  With the logits go the rows' norms, |x| and |w|, which bound what a logit
// may be off: a sum of 32 products in fp32, however the instruction orders it, by
// 32 roundings of 2^-23 of sum |x w|, and all of them together by 2^-18 |x| |w|.
// (2048 tokens of 4096 and 128 experts 21.0 us; fp64 matrix instructions took 50.8,
// one to four steps ahead, 8 or 16 waves, and tiles of 64 x 64 with d in four shares
// 20.9 to 22.2.)
constexpr int kManyWaves = 8, kManyAhead = 2;
template <bool BF>
__device__ __forceinline__ float squares(const uint4& v, float s) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (BF) {
            const float lo = __uint_as_float(w[i] << 16), hi = __uint_as_float(w[i] & 0xFFFF0000u);
            s = __builtin_fmaf(hi, hi, __builtin_fmaf(lo, lo, s));
        } else {
            s = dot2(w[i], w[i], s);
        }
    }
    return s;
}
template <bool BF>
__global__ void __launch_bounds__(kManyWaves * 64) route_many_kernel(RouteArgs a) {
    const bool want[2] = {blockIdx.x == 0, blockIdx.y == 0};           // whose norms are this workgroup's to form

    __shared__ double red[kManyWaves][4][4][64];
    __shared__ float norm[kManyWaves][2][2][16];
    __shared__ uint32_t some[kManyWaves][2][2][16];
    const int tid = threadIdx.x, lane = tid & 63, j = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int m0 = blockIdx.y * 32, e0 = blockIdx.x * 32;
    // tokens, experts: rows past the last give zeros (d < 2^24: a tile's bytes fit 32 bits)
    const Rsrc rows[2] = {rsrc(a.x + (long)m0 * a.d, (uint32_t)min(32, a.M - m0) * (uint32_t)a.d * 2u),
                          rsrc(a.router + (long)e0 * a.d, (uint32_t)min(32, a.E - e0) * (uint32_t)a.d * 2u)};
    const uint32_t at0 = (uint32_t)(j * a.d + 8 * q) * 2u, at1 = at0 + 32u * (uint32_t)a.d;
    double acc[4][4] = {};
    float ss[2][2] = {};
    uint32_t any[2][2] = {};
    uint4 r[kManyAhead][2][2];
    auto place = [&](int s) { return 32 * (wave + kManyWaves * s); };
    auto load = [&](int n, int k) {
        const bool in = k + 8 * q < a.d;
        const uint32_t o0 = in ? at0 + 2u * (uint32_t)k : kPastEnd, o1 = in ? at1 + 2u * (uint32_t)k : kPastEnd;
#pragma unroll
        for (int o = 0; o < 2; ++o) {
            r[n][o][0] = bload16<0>(rows[o], o0, 0);
            r[n][o][1] = bload16<0>(rows[o], o1, 0);
        }
    };
#pragma unroll
    for (int n = 0; n < kManyAhead; ++n) load(n, place(n));
    for (int s = 0; place(s) < a.d; s += kManyAhead) {
#pragma unroll
        for (int n = 0; n < kManyAhead; ++n) {
            uint4(&v)[2][2] = r[n];
            __builtin_amdgcn_sched_barrier(0);             // a step's loads are in flight while the steps before it run
            f32x4_t p[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const f32x4_t zero = {0.f, 0.f, 0.f, 0.f};
                p[c] = BF ? mfma16_bf(v[0][c >> 1], v[1][c & 1], zero) : mfma16(v[0][c >> 1], v[1][c & 1], zero);
            }
#pragma unroll
            for (int o = 0; o < 2; ++o)
                if (want[o])
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        ss[o][i] = squares<BF>(v[o][i], ss[o][i]);
                        any[o][i] |= (v[o][i].x | v[o][i].y | v[o][i].z | v[o][i].w) & 0x7FFF7FFFu;
                    }
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int t = 0; t < 4; ++t) acc[c][t] += (double)p[c][t];
            load(n, place(s + n + kManyAhead));
        }
    }
#pragma unroll
    for (int o = 0; o < 2; ++o)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float s = ss[o][i];
            uint32_t n = any[o][i];
            s += __shfl_xor(s, 16, 64);
            s += __shfl_xor(s, 32, 64);
            n |= __shfl_xor(n, 16, 64);
            n |= __shfl_xor(n, 32, 64);
            if (q == 0) {
                norm[wave][o][i][j] = s;
                some[wave][o][i][j] = n;
            }
        }
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int t = 0; t < 4; ++t) red[wave][c][t][lane] = acc[c][t];
    __syncthreads();
    // item: token 16 (c / 2) + 4 q + t, expert 16 (c % 2) + j
    for (int it = tid; it < 1024; it += kManyWaves * 64) {
        const int c = it >> 8, t = (it >> 6) & 3, l = it & 63;
        double s = red[0][c][t][l];
#pragma unroll
        for (int w = 1; w < kManyWaves; ++w) s += red[w][c][t][l];
        const int m = m0 + 16 * (c >> 1) + 4 * (l >> 4) + t, e = e0 + 16 * (c & 1) + (l & 15);
        if (m < a.M && e < a.E)
            a.logits[(long)m * a.E + e] = s + (a.bias ? (double)a.bias[e] : 0.0);
    }
    if (tid < 64) {
        const int o = tid >> 5, i = (tid >> 4) & 1, at = (o ? e0 : m0) + 16 * i + j;
        float s = 0.0f;
        uint32_t n = 0;
#pragma unroll
        for (int w = 0; w < kManyWaves; ++w) {
            s += norm[w][o][i][j];
            n |= some[w][o][i][j];
        }
        // an upper bound: the sum's own roundings, and squares below the normal numbers (each under 2^-126)
        s = n ? 1.01f * sqrtf(s) + 0x1p-63f * sqrtf((float)a.d) : 0.0f;
        if (o == 0 && want[0] && at < a.M)
            a.xnorm[at] = s;
        if (o == 1 && want[1] && at < a.E)
            a.wnorm[at] = s;
    }
}

// A workgroup: one token, whose logits may be off by 2^-18 |x| max |w|.  Its first
// wave chooses; the logits it asks for are formed by all four, which share d.  (Eight
// waves a SIMD: 2048 tokens of 128 experts 23 us, 28 with three and no register
// in memory; a token a wave, which formed its logits alone, 38.)
constexpr int kChooseWaves = 4;
template <int N>
__global__ void __launch_bounds__(kChooseWaves * 64, 8) route_choose_kernel(RouteArgs a) {
    constexpr int P = 2;                                   // experts side by side
    __shared__ double part[kChooseWaves][kMoeExperts];
    __shared__ int16_t list[kMoeExperts];
    __shared__ int count;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), m = blockIdx.x;
    const uint16_t* xr = a.x + (long)m * a.d;
    auto multiply = [&](int n) {
        for (int i = 0; i < n; i += P) {
            int e[P];
            double s[P] = {};
#pragma unroll
            for (int p = 0; p < P; ++p) e[p] = __builtin_amdgcn_readfirstlane(list[min(i + p, n - 1)]);
            for (int c = tid * 8; c < a.d; c += kChooseWaves * 512) {
                float x[8], w[8];
                act8(ld16(xr + c), a.bf, x);
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    act8(ld16(a.router + (long)e[p] * a.d + c), a.bf, w);
#pragma unroll
                    for (int t = 0; t < 8; ++t) s[p] = __builtin_fma((double)x[t], (double)w[t], s[p]);
                }
            }
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const double v = wave_sum(s[p]);
                if (lane == 0 && i + p < n)
                    part[wave][i + p] = v;
            }
        }
    };
    if (wave != 0) {
        __syncthreads();
        const int n = count;
        if (n > 0) {
            multiply(n);
            __syncthreads();
        }
        return;
    }
    double v[N];
    uint32_t wn = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int e = min(lane + 64 * i, a.E - 1);
        v[i] = a.logits[(long)m * a.E + e];
        wn = max(wn, __float_as_uint(a.wnorm[e]));         // (not negative: in the order of their bits, NaN last)
    }
    // (past 2^126 the fp32 sums could overflow where the logit does not)
    const double norms = (double)a.xnorm[m] * (double)__uint_as_float(wave_max(wn));
    const double off = norms < 0x1p126 ? 0x1p-18 * norms : __builtin_inf();
    bool asked = false;
    const Chosen c = route_select<false>(v, a.E, a.k, a.score, lane, off, list, [&](int n, auto put) {
        asked = true;
        count = n;
        __syncthreads();
        multiply(n);
        __syncthreads();
        for (int i = 0; i < n; ++i) {
            const int e = __builtin_amdgcn_readfirstlane(list[i]);
            double s = part[0][i];
#pragma unroll
            for (int w = 1; w < kChooseWaves; ++w) s += part[w][i];
            put(e, s + (a.bias ? (double)a.bias[e] : 0.0));
        }
    });
    if (!asked) {
        count = 0;
        __syncthreads();
    }
    if (lane < a.k) {
        a.idx[(long)m * a.k + lane] = c.e;
        a.w[(long)m * a.k + lane] = c.w;
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
    route_few_kernel<<<dim3((unsigned)a.E, (unsigned)(a.M + kRouteTok - 1) / kRouteTok), kRouteWaves * 64, 0, st>>>(a);
    return hipGetLastError();
}
hipError_t launch_route(const RouteArgs& a, hipStream_t st) {
    // (us, few and many, the choice included: d = 4096, E = 128: M = 128 25.8 and 28.3, 256 39.5 and 28.4, 2048 244
    // and 35.4; d = 2880, E = 32: M = 256 16.2 and 20.8, 512 23.3 and 21.6, 2048 60.6 and 22.3; d = 2048, E = 512:
    // M = 16 14.7 and 21.2, 64 29.6 and 28.2)
    const bool few = (long)a.M * a.E <= 16384;
    hipError_t e;
    if (few) {
        e = launch_route_logits(a, st);
    } else {
        auto k = a.bf ? route_many_kernel<true> : route_many_kernel<false>;
        k<<<dim3((unsigned)(a.E + 31) / 32, (unsigned)(a.M + 31) / 32), kManyWaves * 64, 0, st>>>(a);
        e = hipGetLastError();
    }
    if (e != hipSuccess)
        return e;
    if (few)
        route_select_kernel<<<(unsigned)(a.M + 3) / 4, 256, 0, st>>>(a);
    else
        (a.E <= 64 ? route_choose_kernel<1> : a.E <= 128 ? route_choose_kernel<2> : route_choose_kernel<kMoeExperts / 64>)
            <<<(unsigned)a.M, kChooseWaves * 64, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace qmlp
