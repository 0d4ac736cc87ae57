// Device helpers of the attention kernels over the 4-bit cache: codes as exact
// binary16 integers, rows of queries as matrix operands, partial results in the
// workspace.
#pragma once

#include <type_traits>

#include "kv_cache.h"
#include "qmlp_device.h"

namespace qmlp {
namespace {

typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef __amdgpu_buffer_rsrc_t Rsrc;

constexpr float kNone = -3.4028235e38f;                   // a maximum before any score: none is lower
constexpr float kTop = 32768.0f, kReset = 8.0f;           // weights in binary16: at most 2^15, 2^8 where the maximum is taken anew
constexpr float kLeast = 16777216.0f;                     // 1 / the least scale (a scale of 0, as in an empty cache, counts as that for the maximum)
constexpr float kFar = 1048576.0f;                        // scores past 2^20: see shifted()
constexpr int kDevice = 16;                               // device-coherent (sc1): read or written by other compute units

__device__ __forceinline__ f32x4_t mfma16(const uint4& a, const uint4& b, f32x4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x16_t mfma32(const uint4& a, const uint4& b, f32x16_t c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c, 0, 0, 0);
}
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
__device__ __forceinline__ f32x4_t mfma16_bf(const uint4& a, const uint4& b, f32x4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}
__device__ __forceinline__ Rsrc rsrc(const void* p, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), (short)0, (int)bytes, 0x00020000);
}
__device__ __forceinline__ float exp2_(float v) { return __builtin_amdgcn_exp2f(v); }
__device__ __forceinline__ float finite(float v) {            // an infinity as the largest number, NaN as it is
    return __builtin_fabsf(v) == INFINITY ? __builtin_copysignf(3.4028235e38f, v) : v;
}
__device__ __forceinline__ float log2_(float v) { return __builtin_amdgcn_logf(v); }

// The low (high) half of w times v, and c added: the conversion is the instruction's.
__device__ __forceinline__ float fma_lo(uint32_t w, float v, float c) { return __builtin_fmaf(h2f(w & 0xFFFFu), v, c); }
__device__ __forceinline__ float fma_hi(uint32_t w, float v, float c) { return __builtin_fmaf(h2f(w >> 16), v, c); }

// Two fp32 to two binary16, each rounded to nearest even.
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t){a, b}, half2_t));
}

// 64 in binary16 has its unit place at bit 4, so a code there reads 64 + code exactly: one and-or gives two.
constexpr uint32_t kMask = 0x00F000F0u;
__device__ __forceinline__ uint32_t magic64() {
    uint32_t v;
    __asm__ volatile("v_mov_b32 %0, 0x54005400" : "=v"(v));
    return v;
}
// The codes of a word (or of the same half of two words) as pairs: bits 4f of both halves.
__device__ __forceinline__ void pairs64(uint32_t w, uint32_t mv, uint32_t (&e)[4]) {
    e[0] = ((w << 4) & kMask) | mv;
    e[1] = (w & kMask) | mv;
    e[2] = ((w >> 4) & kMask) | mv;
    e[3] = ((w >> 8) & kMask) | mv;
}
__device__ __forceinline__ uint32_t lows(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t highs(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }
__device__ __forceinline__ uint32_t add2(uint32_t a, uint32_t b) {
    return __builtin_bit_cast(uint32_t, (half2_t)(__builtin_bit_cast(half2_t, a) + __builtin_bit_cast(half2_t, b)));
}
// The larger halves: of binary16 numbers that are not negative, the larger numbers.
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
    typedef uint16_t u16x2_t __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2_t, a), __builtin_bit_cast(u16x2_t, b)));
}
__device__ __forceinline__ uint32_t comp(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// fp32 as the sum of three bfloat16 numbers (24 bits): what the matrix cores multiply by small integers exactly.
__device__ __forceinline__ void three_bf16(float v, uint32_t (&p)[3]) {
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        p[i] = (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v);
        v -= __uint_as_float(p[i] << 16);
    }
}

// The maximum taken anew from a row's scores (rounded to fp32): most, the largest, and best, the largest with its value's scale
// added as a power of two.  It leaves 2^kReset to the best; past 2^20 an fp32 number cannot carry that difference (its
// neighbours are up to 2^104 away), so there the largest score itself weighs 1, and no weight times a scale passes 65504.
__device__ __forceinline__ float shifted(float m, float most, float best) {
    return fmaxf(m, __builtin_fabsf(most) > kFar ? most : best - kReset);
}

// A product is rounded here: not joined with the sum it goes into.
__device__ __forceinline__ float rounded(float v) {
    __asm__ volatile("" : "+v"(v));
    return v;
}

// One request of a call.
struct Request {
    int len, n, row0;                                     // cached tokens, rows of this step, the first of them
};
__device__ __forceinline__ Request request(const AttnArgs& a, int b) {
    Request r;
    r.len = min(max(a.lens[b], 0), (int)min((long)a.W << a.cache.page_log2, (long)INT32_MAX));
    if (a.starts) {
        // rows outside [0, T) do not exist, whatever starts says
        const int s = min(max(a.starts[b], 0), a.T);
        r.row0 = s;
        r.n = min(max(a.starts[b + 1], s), a.T) - s;
    } else {
        r.row0 = b;
        r.n = 1;
    }
    return r;
}

// A wave's rows of q as operands: `n` 16-byte pieces a lane, all of a lane's from one row, whose other pieces are
// with the lanes that `over_row` and `or_row` join.  bfloat16 is rewritten as binary16 times a power of two which puts the number
// that `largest` makes of the lane's largest (of its row, or of several rows) into [2^14, 2^15): 8 significant bits fit the 11,
// and what that cannot hold is below 2^-31 of that number.  A row with an infinity or NaN becomes zeros, and its sum NaN.
// Returns the power's inverse; sum: of the row as it is now.
template <int N, typename Over, typename OverOr, typename Largest>
__device__ __forceinline__ float operand_rows(uint4 (&v)[N], bool bf, float& sum, Over over_row, OverOr or_row, Largest largest) {
    const uint32_t ebits = bf ? 0x7F80u : 0x7C00u;
    uint32_t bad = 0, top = 0;
#pragma unroll
    for (int p = 0; p < N; ++p)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t w = comp(v[p], i), lo = w & 0x7FFFu, hi = (w >> 16) & 0x7FFFu;
            bad |= (lo >= ebits) | (hi >= ebits);
            top = max(top, max(lo, hi));
        }
    bad = or_row(bad);
    if (bad) {
        top = 0;
#pragma unroll
        for (int p = 0; p < N; ++p)
            v[p] = make_uint4(0, 0, 0, 0);
    }
    float back = 1.0f;
    if (bf) {
        top = largest(top);
        const int e = (int)(top >> 7);                    // biased by 127
        const int k = top == 0 ? 0 : min(14 + 127 - max(e, 1), 126);
        const float up = __uint_as_float((uint32_t)(k + 127) << 23);
        back = __builtin_ldexpf(1.0f, -k);
#pragma unroll
        for (int p = 0; p < N; ++p) {
            uint32_t o[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t w = comp(v[p], i);
                o[i] = pack2(__uint_as_float(w << 16) * up, __uint_as_float(w & 0xFFFF0000u) * up);
            }
            v[p] = make_uint4(o[0], o[1], o[2], o[3]);
        }
    }
    sum = 0.0f;
#pragma unroll
    for (int p = 0; p < N; ++p)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            sum += h2f(comp(v[p], i) & 0xFFFFu) + h2f(comp(v[p], i) >> 16);
    sum = over_row(sum);
    if (bad)
        sum = NAN;
    return back;
}

__device__ __forceinline__ uint32_t out16(float v, int bf) {
    return bf ? (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v) : f2h(v);
}
// Four numbers of a row of y.
__device__ __forceinline__ void store4(uint16_t* p, const float (&o)[4], int bf) {
    *reinterpret_cast<uint2*>(p) = make_uint2(out16(o[0], bf) | out16(o[1], bf) << 16, out16(o[2], bf) | out16(o[3], bf) << 16);
}

// Rows of partial results are o[0..D) relative to 2^m, m and the sum l.  Joined: 2^(m_i - m) weighs each part; a sink
// adds its own weight to the sum.  A row that saw nothing has l = 0 (and m = kNone) and gives zeros.
__device__ __forceinline__ float row_factor(const AttnArgs& a, int head, float m, float l) {
    const float d = a.sinks ? l + exp2_(a.sinks[head] * 1.4426950408889634f - m) : l;
    return l == 0.0f ? 0.0f : 1.0f / d;
}

// A request as LDS holds it, with the units of work of those before it.
template <typename I>
struct Known {
    I before;
    Request q;
    __device__ __forceinline__ Request uniform() const {
        return Request{__builtin_amdgcn_readfirstlane(q.len), __builtin_amdgcn_readfirstlane(q.n), __builtin_amdgcn_readfirstlane(q.row0)};
    }
};

// The work of a call is cut evenly over the workgroups: request b stands for `work` units of it. Every workgroup
// forms the sums itself (the lengths are on the device only).  Returns the total.
template <int NT, typename I, typename F>
__device__ __forceinline__ I prefix_work(const AttnArgs& a, Known<I>* known, F work) {
    __shared__ I wave_sum[NT / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    I total = 0;
    for (int b0 = 0; b0 < a.B; b0 += NT) {
        const int b = b0 + tid;
        Request q{0, 0, 0};
        I v = 0;
        if (b < a.B) {
            q = request(a, b);
            v = work(q);
        }
        I inc = v;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const I o = __shfl_up(inc, d, 64);
            inc += lane >= d ? o : 0;
        }
        if (lane == 63)
            wave_sum[wave] = inc;
        __syncthreads();
        I before = total;
#pragma unroll
        for (int w = 0; w < NT / 64; ++w) {
            before += w < wave ? wave_sum[w] : 0;
            total += wave_sum[w];
        }
        if (b < a.B)
            known[b] = Known<I>{before + inc - v, q};
        __syncthreads();
    }
    return total;
}
// The last b in [0, B) with at most i units before it: the request with unit i.
template <typename I>
__device__ __forceinline__ int request_of(const Known<I>* known, int B, I i) {
    int lo = 0, hi = B;
    while (hi - lo > 1) {
        const int m = (lo + hi) >> 1;
        if (known[m].before <= i)
            lo = m;
        else
            hi = m;
    }
    return lo;
}

}  // namespace
}  // namespace qmlp
