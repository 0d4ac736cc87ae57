// The experts of a whole mixture-of-experts layer for a few tokens (gfx950;
// Sec. 5, Sec. 3.3, Sec. 4.2): every (token, slot) pair the router chose is an
// instance; the instances of an expert run side by side, up to 16 of them as
// the rows of a matrix operand, so an expert is read once per 16.
//
// Launches: LoRA-A of every instance together with the grouping of the
// instances by expert; gate/up with SiLU(G) * U; down; the routing-weighted
// sum.  Gate/up and down have a workgroup per block of instances and few weight
// rows, each wave one piece of K (oneshot.h).
#include "moe_layer.h"
#include "decode_launch.h"
#include "oneshot.h"

namespace qmlp {
namespace {

constexpr int kGroupWaves = 8;
constexpr int kMaxInst = kMoeTokens * kMoeTopk;

// Workgroup 0: the blocks, experts ascending, instances ascending.
__device__ __forceinline__ void moe_group(const MoeArgs& a, int tid) {
    __shared__ int16_t ids[kMaxInst];
    __shared__ int sum[kMoeExperts];
    static_assert(kGroupWaves * 64 >= kMoeExperts, "a thread per expert");
    const int n = a.M * a.k;
    for (int i = tid; i < n; i += kGroupWaves * 64) ids[i] = (int16_t)a.idx[i];
    __syncthreads();
    int c = 0;
    if (tid < a.E)
        for (int i = 0; i < n; ++i) c += ids[i] == tid;
    const int nb = (c + 15) >> 4;
    if (tid < kMoeExperts)
        sum[tid] = nb;
    __syncthreads();
    for (int o = 1; o < kMoeExperts; o *= 2) {             // inclusive sums
        const int v = tid < kMoeExperts && tid >= o ? sum[tid - o] : 0;
        __syncthreads();
        if (tid < kMoeExperts)
            sum[tid] += v;
        __syncthreads();
    }
    if (tid == 0)
        a.blocks[0] = sum[kMoeExperts - 1];
    if (tid < a.E && c > 0) {
        int* b = a.blocks + kBlkInts * (1 + sum[tid] - nb);
        int at = 0;
        for (int i = 0; i < n; ++i)
            if (ids[i] == tid) {
                int* blk = b + (at >> 4) * kBlkInts;
                blk[kBlkInst + (at & 15)] = i;
                blk[kBlkTok + (at & 15)] = i / a.k;
                ++at;
            }
        for (int s = 0; s < nb; ++s) {
            b[s * kBlkInts] = tid;
            b[s * kBlkInts + 1] = min(16, c - 16 * s);
        }
    }
}

// Workgroup 0 groups; workgroup 1 + (instance, eight rows of [A_g; A_u]): t.
__global__ void __launch_bounds__(kGroupWaves * 64) moe_prep_kernel(MoeArgs a) {
    const int tid = threadIdx.x, lane = tid & 63;
    if (blockIdx.x == 0) {
        moe_group(a, tid);
        return;
    }
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int nc = 2 * a.r / 8, i = (blockIdx.x - 1) / nc, c = (blockIdx.x - 1) - i * nc;
    const int e = a.idx[i];
    if (e < 0)
        return;
    const uint16_t* ar = 8 * c < a.r ? a.Ag + ((long)e * a.r + 8 * c) * a.d : a.Au + ((long)e * a.r + 8 * c - a.r) * a.d;
    const uint16_t* xr = a.x + (long)(i / a.k) * a.d;
    float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int k = tid * 8; k < a.d; k += kGroupWaves * 64 * 8) {
        const uint4 xv = *reinterpret_cast<const uint4*>(xr + k);
        uint4 av[8];
#pragma unroll
        for (int r = 0; r < 8; ++r) av[r] = *reinterpret_cast<const uint4*>(ar + (long)r * a.d + k);
#pragma unroll
        for (int r = 0; r < 8; ++r)
            s[r] = dot2(xv.w, av[r].w, dot2(xv.z, av[r].z, dot2(xv.y, av[r].y, dot2(xv.x, av[r].x, s[r]))));
    }
    __shared__ float red[kGroupWaves][8];
#pragma unroll
    for (int r = 0; r < 8; ++r) {
        const float v = group_sum<64>(s[r]);
        if (lane == 0)
            red[wave][r] = v;
    }
    __syncthreads();
    if (tid < 8) {
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < kGroupWaves; ++w) v += red[w][tid];
        a.t[(long)i * 2 * a.r + 8 * c + tid] = a.lora_scale * v;
    }
}

// Gate and up rows of one block of instances -> h.
template <int B, int G, int RT>
__global__ void __launch_bounds__(1024) moe_gateup_kernel(MoeArgs a, int ns, int kw) {
    if ((int)blockIdx.y >= a.blocks[0])
        return;
    extern __shared__ uint4 smem[];
    f32x4_t* red = reinterpret_cast<f32x4_t*>(smem);       // [kw][2][RT][64]
    const int lane = threadIdx.x & 63, j = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int* blk = a.blocks + kBlkInts * (1 + blockIdx.y);
    const int e = blk[0], n = blk[1], row0 = blockIdx.x * 16 * RT;
    const int rb = a.d * B / 8, ng = a.d / G;
    const long wb = (long)a.f * rb, mb = (long)a.f * ng * 4;
    const char *cg = reinterpret_cast<const char*>(a.cg), *cu = reinterpret_cast<const char*>(a.cu);
    const char *mg = reinterpret_cast<const char*>(a.mg), *mu = reinterpret_cast<const char*>(a.mu);
    const Rsrc rc[2] = {rsrc(cg + e * wb, (uint32_t)wb), rsrc(cu + e * wb, (uint32_t)wb)};
    const Rsrc rm[2] = {rsrc(mg + e * mb, (uint32_t)mb), rsrc(mu + e * mb, (uint32_t)mb)};
    const Rsrc rx = rsrc(a.x, (uint32_t)(a.M * a.d) * 2u);
    f32x4_t acc[2][RT];
    oneshot_products<B, G, 2, RT>(acc, rc, rm, rx, j < n ? blk[kBlkTok + j] : 0, j < n, a.d, a.d, a.f, row0, wave, ns, kw, lane);
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            f32x4_t v = acc[m][t] * kTileUnscale;
            const int o = row0 + 16 * t + j;
            for (int c = wave; c < a.r / 8; c += kw)
                if (o < a.f) {
                    float b[8];
                    act8(*reinterpret_cast<const uint4*>((m ? a.Bu : a.Bg) + ((long)e * a.f + o) * a.r + 8 * c), false, b);
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        const int i = 4 * (lane >> 4) + u;
                        if (i < n) {
                            const float* tt = a.t + (long)blk[kBlkInst + i] * 2 * a.r + m * a.r + 8 * c;
#pragma unroll
                            for (int z = 0; z < 8; ++z) v[u] = __builtin_fmaf(b[z], tt[z], v[u]);
                        }
                    }
                }
            red[((wave * 2 + m) * RT + t) * 64 + lane] = v;
        }
    __syncthreads();
    for (int t = wave; t < RT; t += kw) {
        f32x4_t g = red[t * 64 + lane], u = red[(RT + t) * 64 + lane];
        for (int w = 1; w < kw; ++w) {
            g += red[(w * 2 * RT + t) * 64 + lane];
            u += red[((w * 2 + 1) * RT + t) * 64 + lane];
        }
        const int o = row0 + 16 * t + j;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int i = 4 * (lane >> 4) + v;
            if (i < n && o < a.f)
                a.h[(long)blk[kBlkInst + i] * a.f + o] = (uint16_t)f2h(g[v] / (1.0f + __expf(-g[v])) * u[v]);
        }
    }
}

// Down rows of one block of instances -> fp32 outputs of each instance.
template <int B, int G, int RT>
__global__ void __launch_bounds__(1024) moe_down_kernel(MoeArgs a, int ns, int kw) {
    if ((int)blockIdx.y >= a.blocks[0])
        return;
    extern __shared__ uint4 smem[];
    f32x4_t* red = reinterpret_cast<f32x4_t*>(smem);       // [kw][RT][64]
    const int lane = threadIdx.x & 63, j = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int* blk = a.blocks + kBlkInts * (1 + blockIdx.y);
    const int e = blk[0], n = blk[1], row0 = blockIdx.x * 16 * RT;
    const int rb = a.f * B / 8, ng = a.f / G;
    const long wb = (long)a.d * rb, mb = (long)a.d * ng * 4;
    const Rsrc rc[1] = {rsrc(reinterpret_cast<const char*>(a.cd) + e * wb, (uint32_t)wb)};
    const Rsrc rm[1] = {rsrc(reinterpret_cast<const char*>(a.md) + e * mb, (uint32_t)mb)};
    const Rsrc rx = rsrc(a.h, (uint32_t)(a.M * a.k * a.f) * 2u);
    f32x4_t acc[1][RT];
    oneshot_products<B, G, 1, RT>(acc, rc, rm, rx, j < n ? blk[kBlkInst + j] : 0, j < n, a.f, a.f, a.d, row0, wave, ns, kw, lane);
#pragma unroll
    for (int t = 0; t < RT; ++t) red[(wave * RT + t) * 64 + lane] = acc[0][t] * kTileUnscale;
    __syncthreads();
    for (int t = wave; t < RT; t += kw) {
        f32x4_t s = red[t * 64 + lane];
        for (int w = 1; w < kw; ++w) s += red[(w * RT + t) * 64 + lane];
        const int o = row0 + 16 * t + j;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int i = 4 * (lane >> 4) + v;
            if (i < n && o < a.d)
                a.part[(long)blk[kBlkInst + i] * a.d + o] = s[v];
        }
    }
}

// y[m] = sum of w[m][j] part[m k + j], j ascending; slots without an expert add nothing.
__global__ void __launch_bounds__(256) moe_combine_kernel(MoeArgs a) {
    const int m = blockIdx.y, c = (blockIdx.x * 256 + threadIdx.x) * 4;
    if (c >= a.d)
        return;
    f32x4_t s = {0.f, 0.f, 0.f, 0.f};
    for (int j = 0; j < a.k; ++j) {
        const int i = m * a.k + j;
        if (a.idx[i] >= 0)
            s += a.w[i] * *reinterpret_cast<const f32x4_t*>(a.part + (long)i * a.d + c);
    }
    *reinterpret_cast<uint2*>(a.y + (long)m * a.d + c) = make_uint2(f2h(s[0]) | f2h(s[1]) << 16, f2h(s[2]) | f2h(s[3]) << 16);
}

}  // namespace

hipError_t launch_moe_experts(const MoeArgs& a, hipStream_t st) {
    const int n = a.M * a.k, nb = moe_blocks_most(n, a.E);
    moe_prep_kernel<<<(unsigned)(1 + n * (2 * a.r / 8)), kGroupWaves * 64, 0, st>>>(a);
    hipError_t err = hipGetLastError();
    if (err != hipSuccess)
        return err;
    auto run = [&](auto k, int K, int rows, int bits, int nm, int rt) {
        const int ns = oneshot_steps(K, bits), kw = oneshot_waves(ns, 16);
        const size_t lds = (size_t)kw * nm * rt * 1024;
        hipError_t e = set_lds(k, lds);
        if (e != hipSuccess)
            return e;
        k<<<dim3((unsigned)(rows + 16 * rt - 1) / (16 * rt), (unsigned)nb), (unsigned)kw * 64, lds, st>>>(a, ns, kw);
        return hipGetLastError();
    };
    constexpr int RT = 1;
    err = hipErrorInvalidValue;
#define QMLP_MG(B_, G_) \
    if (a.gb == B_ && a.gg == G_) err = run(moe_gateup_kernel<B_, G_, RT>, a.d, a.f, B_, 2, RT);
    QMLP_MG(2, 32) QMLP_MG(2, 64) QMLP_MG(2, 128) QMLP_MG(4, 32) QMLP_MG(4, 64) QMLP_MG(4, 128)
    if (err != hipSuccess)
        return err;
    err = hipErrorInvalidValue;
#define QMLP_MD(B_, G_) \
    if (a.db == B_ && a.dg == G_) err = run(moe_down_kernel<B_, G_, RT>, a.f, a.d, B_, 1, RT);
    QMLP_MD(2, 32) QMLP_MD(2, 64) QMLP_MD(2, 128) QMLP_MD(4, 32) QMLP_MD(4, 64) QMLP_MD(4, 128)
    if (err != hipSuccess)
        return err;
    moe_combine_kernel<<<dim3((unsigned)(a.d + 1023) / 1024, (unsigned)a.M), 256, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace qmlp
