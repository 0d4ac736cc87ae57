// Causal attention over the 4-bit cache (gfx950): the simple form, a workgroup a row and head.
//
// scores s_j = scale q . K_j (log2 units), w_j = 2^(s_j - max), y = sum w_j V_j / (sum w_j + sink),
// with the maximum and the sum carried along (one pass over the tokens).
#include "kv_cache.h"
#include "qmlp_device.h"

namespace qmlp {
namespace {

template <int D>
__global__ void __launch_bounds__(64) simple_kernel(AttnArgs a) {
    __shared__ float qs[D], ws[64], os[D];
    const int t = blockIdx.x, g = blockIdx.y, lane = threadIdx.x, lg = a.cache.page_log2;
    // the request of row t
    int b = -1;
    if (a.starts) {
        for (int i = 0; i < a.B && b < 0; ++i)
            if (t >= a.starts[i] && t < a.starts[i + 1])
                b = i;
    } else {
        b = t;
    }
    if (b < 0)
        return;
    const int len = min(max(a.lens[b], 0), a.W << lg);
    const int s0 = a.starts ? a.starts[b] : t, n = a.starts ? a.starts[b + 1] - s0 : 1;
    const int pos = len - n + t - s0, first = a.window ? max(0, pos - a.window + 1) : 0;
    for (int i = lane; i < D; i += 64) {
        const uint32_t v = a.q[t * a.ldq + (long)g * D + i];
        qs[i] = a.bf ? __uint_as_float(v << 16) : h2f(v);
        os[i] = 0.0f;
    }
    __syncthreads();
    float m = -1e30f, l = 0.0f, o[D / 64] = {};
    for (int j0 = first; j0 <= pos; j0 += 64) {
        const int j = j0 + lane;
        float s = -INFINITY;
        int p = -1;
        if (j <= pos) {
            p = a.table[(long)b * a.W + (j >> lg)];
            if (p >= 0 && p < a.cache.pages) {
                const int in = j & ((1 << lg) - 1);
                const uint32_t* kw = reinterpret_cast<const uint32_t*>(a.cache.at(D, p, g / a.G));
                const uint32_t mt = kw[((D / 8) << lg) + in];
                const float z = h2f(mt >> 16);
                float acc = 0.0f;
                for (int w = 0; w < D / 8; ++w) {
                    const uint32_t c = kw[in * (D / 8) + w];
                    for (int i = 0; i < 8; ++i)
                        acc += qs[8 * w + i] * ((float)((c >> (4 * ((i >> 1) + 4 * (i & 1)))) & 15u) - z);
                }
                s = acc * h2f(mt & 0xFFFFu) * a.scale;
            } else {
                p = -1;
            }
        }
        float top = s;
        for (int d = 1; d < 64; d <<= 1)
            top = fmaxf(top, __shfl_xor(top, d, 64));
        const float mn = fmaxf(m, top), al = exp2f(m - mn), e = exp2f(s - mn);
        m = mn;
        l = l * al + e;
        ws[lane] = p >= 0 ? e : 0.0f;
        for (int k = 0; k < D / 64; ++k) {
            o[k] *= al;
            __syncthreads();
            for (int i = 0; i < 64 && j0 + i <= pos; ++i) {
                const int pi = a.table[(long)b * a.W + ((j0 + i) >> lg)];
                if (pi < 0 || pi >= a.cache.pages)
                    continue;
                const int in = (j0 + i) & ((1 << lg) - 1), d = lane + 64 * k;
                const uint32_t* vw = reinterpret_cast<const uint32_t*>(a.cache.at(D, pi, g / a.G) + a.cache.side(D));
                const uint32_t mt = vw[((D / 8) << lg) + in], c = vw[((in >> 2) * (D / 8) + d / 8) * 4 + (in & 3)];
                o[k] += ws[i] * (h2f(mt & 0xFFFFu) * ((float)((c >> (4 * (((d & 7) >> 1) + 4 * (d & 1)))) & 15u) - h2f(mt >> 16)));
            }
            __syncthreads();
        }
    }
    for (int d = 1; d < 64; d <<= 1)
        l += __shfl_xor(l, d, 64);
    const float den = l + (a.sinks ? exp2f(a.sinks[g] * 1.4426950408889634f - m) : 0.0f);
    for (int k = 0; k < D / 64; ++k) {
        const float y = l > 0.0f || l != l ? o[k] / den : 0.0f;
        a.y[t * a.ldy + (long)g * D + lane + 64 * k] = a.bf ? __builtin_bit_cast(uint16_t, (__bf16)y) : (uint16_t)f2h(y);
    }
}

}  // namespace

size_t kv_attention_bytes(int, int, int) { return 256; }

hipError_t launch_kv_attention(const AttnArgs& a, int, hipStream_t st) {
    const dim3 grid(a.T, a.Hq);
    if (a.D == 128)
        simple_kernel<128><<<grid, 64, 0, st>>>(a);
    else
        simple_kernel<64><<<grid, 64, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace qmlp
