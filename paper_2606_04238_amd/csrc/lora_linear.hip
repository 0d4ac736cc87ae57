// A quantized linear with low-rank adapters of many requests (gfx950):
//   y[m] = W x[m] + s_a B_a (A_a x[m]),   a = ids[m]
// (Sec. 3.1 Eq. (1) with an adapter per row; Sec. 4.2, the adapters stay
// separate from the quantized base, which is what lets requests share it).
// This file: the preparation launch (t = s_a A_a x, and bfloat16 rows as
// binary16) and the linear of up to 16 rows; lora_gemm.hip has more rows.
//
// bfloat16 rows.  The matrix-core arithmetic on packed codes is binary16
// (tile_step.h), so a bfloat16 row enters as x 2^e with the largest |x| in
// [2^14, 2^15) and its finished sums leave times 2^-e.  Both are exact for
// every element down to 2^-28 of the row's largest (binary16 keeps 11 bits of
// a bfloat16's 8 down to 2^-14); what is lost below that is under 2^-39 of the
// largest element.
#include "lora_linear.h"
#include "decode_launch.h"
#include "oneshot.h"

namespace qmlp {
namespace {

constexpr int kPrepWaves = 8;

__device__ __forceinline__ float wave_sum(float v) { return group_sum<64>(v); }

// blockIdx.x: token, blockIdx.y: eight ranks of t, or (the last one, where
// bfloat16) the row's conversion.  t: the waves split k, a lane takes eight
// elements of x and of eight rows of A at a time, fp32 throughout.  It is one
// trip to memory of 9 KB a wave; the launch's time is its latency.
__global__ void __launch_bounds__(kPrepWaves * 64) lora_prep_kernel(LoraArgs a) {
    const int m = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint16_t* xr = a.x + (long)m * a.ldx;
    const int ny = a.T > 0 ? a.R / 8 : 0;
    if ((int)blockIdx.y >= ny) {
        __shared__ float best[kPrepWaves];
        float top = 0.0f;
        for (int k = tid * 8; k < a.k; k += kPrepWaves * 64 * 8) {
            float f[8];
            act8(*reinterpret_cast<const uint4*>(xr + k), true, f);
#pragma unroll
            for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(f[i]));
        }
#pragma unroll
        for (int s = 1; s < 64; s *= 2) top = fmaxf(top, __shfl_xor(top, s, 64));
        if (lane == 0)
            best[wave] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kPrepWaves; ++w) top = fmaxf(top, best[w]);
        // top = f 2^E with 1 <= f < 2: e = 14 - E (2^e a normal number: rows whose largest is below 2^-112, or not
        // finite, keep e = 126 or -113)
        const int E = (int)(__float_as_uint(top) >> 23) - 127;
        const int e = min(14 - E, 126);
        const float up = __uint_as_float((uint32_t)(127 + e) << 23);
        for (int k = tid * 8; k < a.k; k += kPrepWaves * 64 * 8) {
            float f[8];
            act8(*reinterpret_cast<const uint4*>(xr + k), true, f);
            uint32_t o[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = f2h(f[2 * i] * up) | (f2h(f[2 * i + 1] * up) << 16);
            *reinterpret_cast<uint4*>(a.x16 + (long)m * a.k + k) = make_uint4(o[0], o[1], o[2], o[3]);
        }
        if (tid == 0)
            a.xf[m] = __uint_as_float((uint32_t)(127 - e) << 23);
        return;
    }
    const int id = a.ids[m], r0 = blockIdx.y * 8;
    if (id < 0 || id >= a.T) {
        if (tid < 8)
            a.t[(long)m * a.R + r0 + tid] = 0.0f;
        return;
    }
    const uint16_t* ar = a.A + ((long)id * a.R + r0) * a.k;
    float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int k = tid * 8; k < a.k; k += kPrepWaves * 64 * 8) {
        const uint4 xv = *reinterpret_cast<const uint4*>(xr + k);
        uint4 av[8];
#pragma unroll
        for (int r = 0; r < 8; ++r) av[r] = *reinterpret_cast<const uint4*>(ar + (long)r * a.k + k);
        float x[8];
        act8(xv, a.bf, x);
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            float v[8];
            act8(av[r], a.bf, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) s[r] = __builtin_fmaf(x[i], v[i], s[r]);
        }
    }
    __shared__ float red[kPrepWaves][8];
#pragma unroll
    for (int r = 0; r < 8; ++r) {
        const float v = wave_sum(s[r]);
        if (lane == 0)
            red[wave][r] = v;
    }
    __syncthreads();
    if (tid < 8) {
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < kPrepWaves; ++w) v += red[w][tid];
        a.t[(long)m * a.R + r0 + tid] = (a.scale ? a.scale[id] : 1.0f) * v;
    }
}

// Adds B_a[o][8 c .. 8 c + 7] . t[token][8 c ..] for the lane's row o and its
// tokens 4 q + v.  A row with no adapter adds nothing (not 0 B: an adapter
// that holds infinities belongs to its own rows only).
__device__ __forceinline__ void lora_rank8(f32x4_t& acc, const LoraArgs& a, int o, int c, int lane) {
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        const int tok = 4 * (lane >> 4) + v;
        const int id = tok < a.M ? a.ids[tok] : -1;
        if (id >= 0 && id < a.T && o < a.n) {
            float b[8];
            act8(*reinterpret_cast<const uint4*>(a.B + ((long)id * a.n + o) * a.R + 8 * c), a.bf, b);
            const float* t = a.t + (long)tok * a.R + 8 * c;
            float s = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) s = __builtin_fmaf(b[i], t[i], s);
            acc[v] += s;
        }
    }
}

// Up to 16 rows of x: a workgroup owns RT tiles of 16 outputs (oneshot.h), the
// waves share its LoRA terms by eight ranks.
template <int B, int G, int RT>
__global__ void __launch_bounds__(1024) lora_few_kernel(LoraArgs a, int ns, int kw) {
    extern __shared__ uint4 smem[];
    f32x4_t* red = reinterpret_cast<f32x4_t*>(smem);       // [kw][RT][64]
    const int lane = threadIdx.x & 63, j = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row0 = blockIdx.x * 16 * RT;
    const int rb = a.k * B / 8, ng = a.k / G;
    const Rsrc rc[1] = {rsrc(a.codes, (uint32_t)a.n * (uint32_t)rb)};
    const Rsrc rm[1] = {rsrc(a.meta, (uint32_t)a.n * (uint32_t)ng * 4u)};
    const int ldx = a.x16 ? a.k : (int)a.ldx;
    const Rsrc rx = rsrc(a.x16 ? a.x16 : a.x, (uint32_t)((a.M - 1) * ldx + a.k) * 2u);
    f32x4_t acc[1][RT];
    oneshot_products<B, G, 1, RT>(acc, rc, rm, rx, j, j < a.M, ldx, a.k, a.n, row0, wave, ns, kw, lane);
    // the factor of bfloat16 rows, before terms that do not have it
    float f[4];
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        const int tok = 4 * (lane >> 4) + v;
        f[v] = kTileUnscale * (a.x16 && tok < a.M ? a.xf[tok] : 1.0f);
    }
#pragma unroll
    for (int t = 0; t < RT; ++t) {
#pragma unroll
        for (int v = 0; v < 4; ++v) acc[0][t][v] *= f[v];
        if (a.T > 0)
            for (int c = wave; c < a.R / 8; c += kw) lora_rank8(acc[0][t], a, row0 + 16 * t + j, c, lane);
        red[(wave * RT + t) * 64 + lane] = acc[0][t];
    }
    __syncthreads();
    for (int t = wave; t < RT; t += kw) {
        f32x4_t s = red[t * 64 + lane];
        for (int w = 1; w < kw; ++w) s += red[(w * RT + t) * 64 + lane];
        const int o = row0 + 16 * t + j;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int tok = 4 * (lane >> 4) + v;
            if (tok < a.M && o < a.n)
                a.y[(long)tok * a.ldy + o] = act_bits(s[v], a.bf);
        }
    }
}

}  // namespace

hipError_t launch_lora_prep(const LoraArgs& a, hipStream_t st) {
    const unsigned ny = (a.T > 0 ? a.R / 8 : 0) + (a.bf ? 1 : 0);
    if (ny == 0)
        return hipSuccess;
    lora_prep_kernel<<<dim3((unsigned)a.M, ny), kPrepWaves * 64, 0, st>>>(a);
    return hipGetLastError();
}

hipError_t launch_lora_few(const LoraArgs& a, hipStream_t st) {
    if (a.M < 1 || a.M > kLoraFewTokens)
        return hipErrorInvalidValue;
    constexpr int RT = 1;
    const int ns = oneshot_steps(a.k, a.bits), kw = oneshot_waves(ns, 16);
    const unsigned grid = (unsigned)((a.n + 16 * RT - 1) / (16 * RT));
    const size_t lds = (size_t)kw * RT * 1024;
#define QMLP_LF(B_, G_)                                                              \
    if (a.bits == B_ && a.g == G_) {                                                 \
        lora_few_kernel<B_, G_, RT><<<grid, (unsigned)kw * 64, lds, st>>>(a, ns, kw); \
        return hipGetLastError();                                                    \
    }
    QMLP_LF(2, 32) QMLP_LF(2, 64) QMLP_LF(2, 128) QMLP_LF(4, 32) QMLP_LF(4, 64) QMLP_LF(4, 128)
    return hipErrorInvalidValue;
}

}  // namespace qmlp
