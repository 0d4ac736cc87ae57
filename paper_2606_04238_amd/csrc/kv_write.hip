// Norm and rotation of query and key heads with the write of keys and values
// into the 4-bit cache, and the read of tokens back (gfx950).
//
// What bounds the first is reading q, k, v and writing q (the cache takes a
// quarter of k and v), so every element is loaded once, 16 bytes a lane: a head is
// D/8 lanes of a wave and the 8 numbers of a lane are one word of codes.  Sums,
// ranges and the partner of a rotated dim come from other lanes of the head.  One token of 32 + 8 + 8 heads of 128 takes
// 4.5 us; 4096 tokens 37 us (2.4 TB/s, half of what a large copy reaches).  By counters the vector units are then busy 59 % of the
// time, and waves, three a SIMD, wait 54 % of theirs: the fp64 of keys and angles is work, and the chain of a head (load, sums over its
// lanes) is not hidden.  Four tokens a workgroup 62 us, a workgroup for every 16 heads 50 us, the next head's load ahead 50 to 64 us.
#include <type_traits>

#include "kv_cache.h"
#include "qmlp_device.h"
#include "quant_device.h"

#pragma clang fp contract(off)

namespace qmlp {
namespace {

// 16-bit activation <-> fp32
template <bool BF>
__device__ __forceinline__ float up16(uint32_t bits) { return BF ? __uint_as_float(bits << 16) : h2f(bits); }
template <bool BF>
__device__ __forceinline__ uint32_t down16(float v) {
    return BF ? (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v) : f2h(v);
}
__device__ __forceinline__ uint32_t word_at(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

template <int LPH, typename T, typename F>
__device__ __forceinline__ T over_head(T v, F f) {
#pragma unroll
    for (int d = 1; d < LPH; d <<= 1)
        v = f(v, __shfl_xor(v, d, 64));
    return v;
}

// The codes of a lane's 8 numbers as one word, dims 0..7 at nibbles 0 4 1 5 2 6 3 7, and the head's (scale, zero):
// the quantizer of pack.hip with a head as the group.
template <int LPH>
__device__ __forceinline__ uint32_t quantize(const float (&x)[8], uint32_t& meta) {
    float lo = 0.0f, hi = 0.0f;
    int bad = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const bool fin = (__float_as_uint(x[i]) & 0x7F800000u) != 0x7F800000u;
        lo = __builtin_fminf(lo, fin ? x[i] : 0.0f);
        hi = __builtin_fmaxf(hi, fin ? x[i] : 0.0f);
        bad |= !fin;
    }
    lo = over_head<LPH>(lo, [](float a, float b) { return __builtin_fminf(a, b); });
    hi = over_head<LPH>(hi, [](float a, float b) { return __builtin_fmaxf(a, b); });
    bad = over_head<LPH>(bad, [](int a, int b) { return a | b; });
    uint32_t s16 = f64_to_f16_bits(((double)hi - (double)lo) / 15.0);
    if (s16 == 0)
        s16 = 0x3C00u;
    if (bad || s16 == 0x7C00u) {
        meta = 0x00007E00u;                               // scale NaN, zero 0
        return 0;
    }
    const float s = h2f(s16), r = 1.0f / s;
    const float z = __builtin_fminf(div_rint(-lo, s, r), 15.0f);
    meta = s16 | (f2h(z + 0.0f) << 16);                   // (+ 0: never -0)
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float c = __builtin_fminf(__builtin_fmaxf(div_rint(x[i], s, r) + z, 0.0f), 15.0f);
        w |= (uint32_t)c << (4 * ((i >> 1) + 4 * (i & 1)));
    }
    return w;
}

template <int D>
__device__ __forceinline__ void store_codes(const KvView& c, int slot, int head, int side, int lane, uint32_t w, uint32_t meta) {
    const int lg = c.page_log2, o = slot & ((1 << lg) - 1);
    uint8_t* base = c.at(D, slot >> lg, head) + (side ? c.side(D) : 0u);
    uint32_t* words = reinterpret_cast<uint32_t*>(base);
    words[side ? ((o >> 2) * (D / 8) + lane) * 4 + (o & 3) : o * (D / 8) + lane] = w;
    if (lane == 0)
        reinterpret_cast<uint32_t*>(base + ((size_t)(D / 2) << lg))[o] = meta;
}

// One head: norm and rotation of a lane's 8 numbers in F, rounded to fp32 and then to the activation type (in fp32, once).
// `turn`: (cos, sin) of each pair, scaled.  `far` (fp32): the squares
// pass fp32 on either side (bfloat16 numbers of 2^60, or with eps 0 of 2^-50), and the result does not count.
template <int D, bool BF, typename F, typename P>
__device__ __forceinline__ uint4 turned(const HeadsArgs& a, const uint4 raw, const uint16_t* weight, const P* turn, int lane, bool& far) {
    constexpr int LPH = D / 8;
    F x[8], p[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
        x[i] = (F)up16<BF>(i & 1 ? word_at(raw, i >> 1) >> 16 : word_at(raw, i >> 1) & 0xFFFFu);
    F inv = (F)1;
    if (weight) {
        F s = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            s += x[i] * x[i];
        s = over_head<LPH>(s, [](F u, F v) { return u + v; });
        const F m = s / (F)D + (F)a.eps;
        if constexpr (std::is_same<F, double>::value) {
            inv = 1.0 / __builtin_sqrt(m);
        } else {
            inv = 1.0f / __builtin_sqrtf(m);
            far = !(m >= 0x1p-100f && m <= 0x1p120f);
        }
        const uint4 w = reinterpret_cast<const uint4*>(weight)[lane];
#pragma unroll
        for (int i = 0; i < 8; ++i)
            x[i] = x[i] * inv * (F)up16<BF>(i & 1 ? word_at(w, i >> 1) >> 16 : word_at(w, i >> 1) & 0xFFFFu);
    }
    if (a.inv) {
        const int half = a.rot / 2, hl = half / 8;        // lanes to the partner where halves turn
        const bool on = 8 * lane < a.rot;
        if (a.next) {
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                const auto cs = turn[on ? i / 2 * (a.rot / 8) + lane : 0];
                const F c = cs.x, s = cs.y;
                p[i] = x[i] * c - x[i + 1] * s;
                p[i + 1] = x[i + 1] * c + x[i] * s;
            }
        } else {
            const bool first = lane < hl;
            const int me = threadIdx.x & 63, from = on ? (first ? me + hl : me - hl) : me;
            const int at = on ? (first ? lane : lane - hl) : 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const auto cs = turn[i * hl + at];
                const F o = __shfl(x[i], from, 64), c = cs.x, s = cs.y;
                p[i] = first ? x[i] * c - o * s : x[i] * c + o * s;
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
            x[i] = on ? p[i] : x[i];
    }
    uint32_t h[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
        h[i] = down16<BF>((float)x[i]);
    return make_uint4(h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16);
}

template <bool BF>
__device__ __forceinline__ void unpacked(const uint4& v, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
        x[i] = up16<BF>(i & 1 ? word_at(v, i >> 1) >> 16 : word_at(v, i >> 1) & 0xFFFFu);
}

// A workgroup takes one token's heads g, g + step, ... (q, then k, then v), D/8 lanes each; the token's
// angles are reduced once, a thread a pair: positions times frequencies as a product of fp64 (far positions
// lose nothing that a 16-bit result or a code shows), in turns, then cos and sin of what is left of a turn.
template <int D, bool BF>
__global__ void __launch_bounds__(256, 5) qk_kernel(HeadsArgs a) {
    constexpr int LPH = D / 8, HPW = 256 / LPH;           // heads at a time
    __shared__ double2 turn64[D / 2];
    __shared__ float2 turn32[D / 2];
    const int t = blockIdx.x, tid = threadIdx.x, lane = tid % LPH;
    if (a.inv) {
        if (tid < a.rot / 2) {
            // pairs as the lanes take them, neighbouring lanes side by side
            const int n = a.next ? (tid & 3) * (a.rot / 8) + tid / 4 : (tid & 7) * (a.rot / 16) + tid / 8;
            double turns = (double)a.pos[t] * (double)a.inv[tid] * 0.15915494309189533577;    // 1 / (2 pi)
            turns -= __builtin_rint(turns);
            double s, c;
            sincospi(2.0 * turns, &s, &c);
            turn64[n] = {c * (double)a.mul, s * (double)a.mul};
            turn32[n] = {(float)turn64[n].x, (float)turn64[n].y};
        }
        __syncthreads();
    }
    const int kv = a.k ? a.Hk : 0, all = a.Hq + kv * (a.cache.data ? 2 : 1);
    int slot = -1;
    if (a.cache.data) {
        slot = a.slots[t];
        if ((slot >> a.cache.page_log2) >= a.cache.pages)
            slot = -1;
    }
    for (int g0 = blockIdx.y * HPW; g0 < all; g0 += gridDim.y * HPW) {
        // (shuffles reach only lanes of the same head, which leave the loop body together)
        const int g = g0 + tid / LPH;
        if (g >= all)
            continue;
        const int side = g < a.Hq ? 0 : g < a.Hq + kv ? 1 : 2, h = g - (side == 0 ? 0 : side == 1 ? a.Hq : a.Hq + kv);
        const uint16_t* src = side == 0 ? a.q + t * a.ldq : side == 1 ? a.k + t * a.ldk : a.v + t * a.ldv;
        uint4 v = reinterpret_cast<const uint4*>(src + (long)h * D)[lane];
        bool far = false;
        uint4 u = v;
        if (side == 0)
            u = turned<D, BF, float>(a, v, a.qw, turn32, lane, far);
        if (side == 1 || far)
            u = turned<D, BF, double>(a, v, side == 0 ? a.qw : a.kw, turn64, lane, far);
        if (side == 0) {
            reinterpret_cast<uint4*>(a.q_out + t * a.ldqo + (long)h * D)[lane] = u;
            continue;
        }
        v = u;
        if (side == 1 && a.k_out)
            reinterpret_cast<uint4*>(a.k_out + t * a.ldko + (long)h * D)[lane] = v;
        if (slot >= 0) {
            float x[8];
            unpacked<BF>(v, x);
            uint32_t meta;
            const uint32_t w = quantize<LPH>(x, meta);
            store_codes<D>(a.cache, slot, h, side - 1, lane, w, meta);
        }
    }
}

// A lane a word of codes: 16 bytes out.
template <int D, bool BF>
__global__ void __launch_bounds__(256) read_kernel(KvView c, const int32_t* slots, int T, uint16_t* k, uint16_t* v) {
    constexpr int WPH = D / 8;
    const long i = (long)blockIdx.x * 256 + threadIdx.x;
    const int w = (int)(i % WPH);
    const long th = i / WPH;
    if (th >= (long)T * c.heads)
        return;
    const int t = (int)(th / c.heads), h = (int)(th % c.heads), lg = c.page_log2;
    const int slot = slots[t];
    const bool in = slot >= 0 && (slot >> lg) < c.pages;
    const int o = slot & ((1 << lg) - 1);
    const uint8_t* base = c.at(D, in ? slot >> lg : 0, h);
#pragma unroll
    for (int side = 0; side < 2; ++side) {
        uint16_t* out = side ? v : k;
        if (!out)
            continue;
        uint32_t word = 0, m = 0;
        if (in) {
            const uint32_t* words = reinterpret_cast<const uint32_t*>(base + side * c.side(D));
            word = words[side ? ((o >> 2) * WPH + w) * 4 + (o & 3) : o * WPH + w];
            m = words[((D / 8) << lg) + o];
        }
        const float s = h2f(m & 0xFFFFu), z = h2f(m >> 16);
        uint32_t r[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            r[j] = in ? down16<BF>(s * ((float)((word >> (4 * ((j >> 1) + 4 * (j & 1)))) & 15u) - z)) : 0u;
        reinterpret_cast<uint4*>(out + th * D)[w] = make_uint4(r[0] | r[1] << 16, r[2] | r[3] << 16, r[4] | r[5] << 16, r[6] | r[7] << 16);
    }
}

}  // namespace

hipError_t launch_qk_norm_rope(const HeadsArgs& a, hipStream_t st) {
    const int all = a.Hq + (a.k ? a.Hk : 0) * (a.cache.data ? 2 : 1), hpw = 256 / (a.D / 8);
    // few tokens: every set of heads a workgroup of its own; many: one workgroup, which forms the angles once (us, 32 + 8 + 8 heads of
    // 128, sets and one: 32 tokens 4.4 and 6.1, 384 6.7 and 7.6, 512 7.8 and 7.8, 1024 11.5 and 10.1, 4096 35 and 29)
    const int sets = (all + hpw - 1) / hpw, split = a.T >= 512 ? 1 : sets;
    const dim3 grid(a.T, split);
    if (a.D == 128)
        a.bf ? qk_kernel<128, true><<<grid, 256, 0, st>>>(a) : qk_kernel<128, false><<<grid, 256, 0, st>>>(a);
    else
        a.bf ? qk_kernel<64, true><<<grid, 256, 0, st>>>(a) : qk_kernel<64, false><<<grid, 256, 0, st>>>(a);
    return hipGetLastError();
}

hipError_t launch_kv_read(const KvView& c, int D, const int32_t* slots, int T, int bf, uint16_t* k, uint16_t* v, hipStream_t st) {
    const long lanes = (long)T * c.heads * (D / 8);
    const unsigned grid = (unsigned)((lanes + 255) / 256);
    if (D == 128)
        bf ? read_kernel<128, true><<<grid, 256, 0, st>>>(c, slots, T, k, v) : read_kernel<128, false><<<grid, 256, 0, st>>>(c, slots, T, k, v);
    else
        bf ? read_kernel<64, true><<<grid, 256, 0, st>>>(c, slots, T, k, v) : read_kernel<64, false><<<grid, 256, 0, st>>>(c, slots, T, k, v);
    return hipGetLastError();
}

}  // namespace qmlp
