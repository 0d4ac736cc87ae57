// The experts of a whole mixture-of-experts layer for a few tokens (gfx950;
// Sec. 5, Sec. 3.3, Sec. 4.2): every (token, slot) pair the router chose is an
// instance; the instances of an expert run side by side, up to 16 of them as
// the rows of a matrix operand, so an expert is read once per 16.
//
// Launches: the router's logits (moe_route.hip); the choice, the grouping of the
// instances by expert and x in operand order; LoRA-A of each block of
// instances; gate/up with SiLU(G) * U; down; the routing-weighted sum.  Gate/up
// and down have a workgroup per block of instances and few weight rows
// (oneshot.h).
#include "moe_layer.h"
#include "decode_launch.h"
#include "moe_select.h"
#include "oneshot.h"

namespace qmlp {
namespace {

constexpr int kChooseWaves = 16;

// Workgroup 0: every token's experts, and the blocks, experts ascending, tokens
// ascending.  A token chooses an expert at most once, so a 64-bit mask of tokens is
// an expert's list, and an instance's place the number of bits below its own.
__device__ __forceinline__ void moe_group(const MoeArgs& a, int tid) {
    __shared__ uint32_t list[kMoeExperts][2];
    __shared__ int16_t ids[kMoeTokens * kMoeTopk], start[kMoeExperts];
    __shared__ int sums[kMoeExperts / 64];
    static_assert(kChooseWaves * 64 >= kMoeExperts && kChooseWaves * 64 >= kMoeTokens * kMoeTopk, "a thread per expert, and per instance");
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = a.M * a.k;
    if (tid < kMoeExperts)
        list[tid][0] = list[tid][1] = 0;
    __syncthreads();
    for (int m = wave; m < a.M; m += kChooseWaves) {
        const Chosen c = route_select(a.logits + (long)m * a.E, a.E, a.k, a.score, lane);
        if (lane < a.k) {
            const int i = m * a.k + lane;
            a.idx[i] = c.e;
            a.w[i] = c.w;
            ids[i] = (int16_t)c.e;
            if (c.e >= 0)
                atomicOr(&list[c.e][m >> 5], 1u << (m & 31));
        }
    }
    __syncthreads();
    int c = 0, nb = 0, at = 0;                             // of expert tid: instances, blocks; both of those up to it
    if (tid < kMoeExperts) {
        c = __popc(list[tid][0]) + __popc(list[tid][1]);
        nb = (c + 15) >> 4;
        at = c << 16 | nb;
#pragma unroll
        for (int o = 1; o < 64; o *= 2) {
            const int v = __shfl_up(at, o, 64);
            at += lane >= o ? v : 0;
        }
        if (lane == 63)
            sums[wave] = at;
    }
    __syncthreads();
    int all = 0;
#pragma unroll
    for (int w = 0; w < kMoeExperts / 64; ++w) {
        if (w < wave)
            at += sums[w];
        all += sums[w];
    }
    if (tid < kMoeExperts) {
        const int first = (at & 0xFFFF) - nb, place = (at >> 16) - c;
        start[tid] = (int16_t)first;
        for (int s = 0; s < nb; ++s) {
            int* b = a.blocks + (first + s) * kBlkInts;
            b[0] = tid;
            b[1] = min(16, c - 16 * s);
            b[2] = place + 16 * s;
        }
    }
    for (int b = (all & 0xFFFF) + tid; b < moe_blocks_most(n, a.E); b += kChooseWaves * 64) a.blocks[b * kBlkInts + 1] = 0;
    __syncthreads();
    if (tid < n && ids[tid] >= 0) {
        const int e = ids[tid], m = tid / a.k;
        const uint64_t before = ((uint64_t)list[e][1] << 32 | list[e][0]) & ((1ull << m) - 1);
        const int p = __popcll(before);
        int* b = a.blocks + (start[e] + (p >> 4)) * kBlkInts + (p & 15);
        b[kBlkInst] = tid;
        b[kBlkTok] = m;
    }
}

// Workgroup 0 chooses and groups; the others bring a row of x into operand order
// each.  (Side by side with the others' a token's row would bring their lines along:
// a block's tokens are any of them, and few.  Gate and up of 21 experts of 2880,
// eight tokens 37.4 us and 41.4, 64 68.6 and 77.5.)
__global__ void __launch_bounds__(kChooseWaves * 64) moe_choose_kernel(MoeArgs a) {
    const int tid = threadIdx.x;
    if (blockIdx.x == 0) {
        moe_group(a, tid);
        return;
    }
    const int m = blockIdx.x - 1;
    operands_of_row<kChooseWaves>(a.x + (long)m * a.d, a.d, false, a.gb, a.gg,
                                  reinterpret_cast<uint4*>(a.xo) + (long)m * (operand_row(a.d, a.gb) / 8),
                                  reinterpret_cast<float2*>(a.xs) + (long)m * (operand_sums(a.d, a.gb, a.gg) / 2), 1, nullptr, tid);
}

// A block of the table in registers: expert and instances are uniform (scalar
// loads), the lane's own instance and token come with one vector load each.
struct Block {
    int e, n, at, inst, tok;
};
__device__ __forceinline__ Block block_of(const MoeArgs& a, int b, int lane) {
    const int* p = a.blocks + kBlkInts * b;
    const int n = p[1], l = (lane & 15) < n ? lane & 15 : 0;
    return {p[0], n, p[2], p[kBlkInst + l], p[kBlkTok + l]};
}

// t of one block of instances: 16 rows of the expert's [A_g; A_u], whose 2 r rows
// are a multiple of 16, by x as they lie in memory; the waves split d.  (An instance
// and eight rows a workgroup, A read once per instance: 31 us for 256 instances, now
// 9.1.)
constexpr int kShrinkWaves = 8;
__global__ void __launch_bounds__(kShrinkWaves * 64) moe_shrink_kernel(MoeArgs a) {
    constexpr int N = 4;
    __shared__ f32x4_t red[kShrinkWaves][64];
    const int lane = threadIdx.x & 63, j = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Block bl = block_of(a, blockIdx.y, lane);
    if (bl.n == 0)
        return;
    const int row = blockIdx.x * 16 + j;
    const uint16_t* ar = (row < a.r ? a.Ag + ((long)bl.e * a.r + row) * a.d : a.Au + ((long)bl.e * a.r + row - a.r) * a.d) + 8 * q;
    const uint16_t* xr = a.x + (long)bl.tok * a.d + 8 * q;
    f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
    for (int k = wave * 32; k < a.d; k += N * kShrinkWaves * 32) {
        uint4 xv[N], av[N];
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (k + i * kShrinkWaves * 32 < a.d) {
                xv[i] = ld16(xr + k + i * kShrinkWaves * 32);
                av[i] = ld16(ar + k + i * kShrinkWaves * 32);
            }
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (k + i * kShrinkWaves * 32 < a.d)
                acc = mfma16(xv[i], av[i], acc);
    }
    red[wave][lane] = acc;
    __syncthreads();
    if (wave == 0) {
#pragma unroll
        for (int w = 1; w < kShrinkWaves; ++w) acc += red[w][lane];
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int i = __shfl(bl.inst, 4 * q + v, 64);
            if (4 * q + v < bl.n)
                a.t[(long)i * 2 * a.r + row] = a.lora_scale * acc[v];
        }
    }
}

// Gate and up rows of one block of instances -> h.  Eight ranks of one matrix's
// LoRA-B are two v_mfma_f32_16x16x4_f32 with t as the other operand, ranks 2 q and
// 2 q + 1 of them in lane quarter q.  Measured (2 bits in groups of 64, d = f = 2880,
// rank 16, 4 of 32 experts): one token 9.6 us, eight 37.6 (21 experts, 109 MB, 2.9
// TB/s), 64 67.0 (166 MB); vector instructions 38 % and tag lookups 54 % of the
// cycles at eight.
template <int B, int G, int RT>
__global__ void __launch_bounds__(512) moe_gateup_kernel(MoeArgs a, int ns, int kw) {
    extern __shared__ uint4 smem[];
    f32x4_t* red = reinterpret_cast<f32x4_t*>(smem);       // [kw][2][RT][64]
    const int lane = threadIdx.x & 63, j = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Block bl = block_of(a, blockIdx.y, lane);
    if (bl.n == 0)
        return;
    const int rb = a.d * B / 8, ng = a.d / G;
    const long wb = (long)a.f * rb, mb = (long)a.f * ng * 4;
    const char *cg = reinterpret_cast<const char*>(a.cg), *cu = reinterpret_cast<const char*>(a.cu);
    const char *mg = reinterpret_cast<const char*>(a.mg), *mu = reinterpret_cast<const char*>(a.mu);
    OneWork<2> o;
    one_magic(o);
    o.rc[0] = rsrc(cg + bl.e * wb, (uint32_t)wb);
    o.rc[1] = rsrc(cu + bl.e * wb, (uint32_t)wb);
    o.rm[0] = rsrc(mg + bl.e * mb, (uint32_t)mb);
    o.rm[1] = rsrc(mu + bl.e * mb, (uint32_t)mb);
    const bool live = j < bl.n;
    const uint32_t xb = operand_row(a.d, B) * 2u, sb = operand_sums(a.d, B, G) * 4u;
    o.rows = 1;
    o.rx = rsrc(a.xo, (uint32_t)a.M * xb);
    o.rs = rsrc(a.xs, (uint32_t)a.M * sb);
    place<B, G>(o, (uint32_t)bl.tok * xb, (uint32_t)bl.tok * sb, live, q);
    o.K = a.d;
    o.N = a.f;
    o.row0 = blockIdx.x * 16 * RT;
    // rank chunk c of matrix m: item 2 c + m
    const int items = a.r / 4;
    struct {
        float t[2];
        uint32_t b[RT];
    } k8;
    auto rank_load = [&](int it) {
        const int m = it & 1, at = 8 * (it >> 1) + 2 * q;
        const float* tp = a.t + (long)(live ? bl.inst : 0) * 2 * a.r + m * a.r + at;
        k8.t[0] = tp[0];
        k8.t[1] = tp[1];
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            const int n = o.row0 + 16 * t + j < a.f ? o.row0 + 16 * t + j : a.f - 1;
            k8.b[t] = *reinterpret_cast<const uint32_t*>((m ? a.Bu : a.Bg) + ((long)bl.e * a.f + n) * a.r + at);
        }
    };
    f32x4_t acc[2][RT];
    auto rank_add = [&](int it) {
        const float t0 = live ? k8.t[0] : 0.0f, t1 = live ? k8.t[1] : 0.0f;
#pragma unroll
        for (int m = 0; m < 2; ++m)
            if (m == (it & 1))
#pragma unroll
                for (int t = 0; t < RT; ++t)
                    acc[m][t] = mfma4(t1, h2f(k8.b[t] >> 16), mfma4(t0, h2f(k8.b[t] & 0xFFFFu), acc[m][t]));
    };
    oneshot_products<B, G, 2, RT, false>(acc, o, wave, ns, kw, lane, [&] {
        if (wave < items)
            rank_load(wave);
    });
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int t = 0; t < RT; ++t) acc[m][t] *= kTileUnscale;
    if (wave < items)
        rank_add(wave);
    for (int it = wave + kw; it < items; it += kw) {       // few waves: short rows
        rank_load(it);
        rank_add(it);
    }
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int t = 0; t < RT; ++t) red[((wave * 2 + m) * RT + t) * 64 + lane] = acc[m][t];
    __syncthreads();
    const int hrow = operand_row(a.f, a.db);
    uint16_t* h = a.h + (long)bl.at * hrow;                // the block's rows, side by side
    if (blockIdx.x == 0)                                   // and what pads them to whole steps
        for (int i = threadIdx.x; i < (hrow - a.f) * bl.n; i += kw * 64) h[a.f * bl.n + i] = 0;
    for (int t = wave; t < RT; t += kw) {
        f32x4_t g = red[t * 64 + lane], u = red[(RT + t) * 64 + lane];
        for (int w = 1; w < kw; ++w) {
            g += red[(w * 2 * RT + t) * 64 + lane];
            u += red[((w * 2 + 1) * RT + t) * 64 + lane];
        }
        const int n = o.row0 + 16 * t + j, at = operand_at(n, a.db, a.dg);
        // h is rounded to binary16, which down's matrix instructions take: half a step of each element, as the
        // output's own rounding (the layer is 2.9e-4 off 64 bits with it, the output's rounding alone 2.1e-4)
#pragma unroll
        for (int v = 0; v < 4; ++v)
            if (4 * q + v < bl.n && n < a.f)
                h[((at >> 3) * bl.n + 4 * q + v) * 8 + (at & 7)] = (uint16_t)f2h(g[v] / (1.0f + __expf(-g[v])) * u[v]);
    }
}

// Down rows of one block of instances -> fp32 outputs of each instance.  Measured (4
// bits in groups of 64, as above): 7.7 us, 25.1 (98 MB, 3.9 TB/s), 44.6 (149 MB).
template <int B, int G, int RT>
__global__ void __launch_bounds__(512) moe_down_kernel(MoeArgs a, int ns, int kw) {
    extern __shared__ uint4 smem[];
    f32x4_t* red = reinterpret_cast<f32x4_t*>(smem);       // [kw][RT][64]
    const int lane = threadIdx.x & 63, j = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Block bl = block_of(a, blockIdx.y, lane);
    if (bl.n == 0)
        return;
    const int rb = a.f * B / 8, ng = a.f / G;
    const long wb = (long)a.d * rb, mb = (long)a.d * ng * 4;
    OneWork<1> o;
    one_magic(o);
    o.rc[0] = rsrc(reinterpret_cast<const char*>(a.cd) + bl.e * wb, (uint32_t)wb);
    o.rm[0] = rsrc(reinterpret_cast<const char*>(a.md) + bl.e * mb, (uint32_t)mb);
    const int hrow = operand_row(a.f, B);
    o.rows = (uint32_t)bl.n;
    o.rx = rsrc(a.h + (long)bl.at * hrow, o.rows * (uint32_t)hrow * 2u);
    place<B, G>(o, 16u * j, 0u, j < bl.n, q);
    o.K = a.f;
    o.N = a.d;
    o.row0 = blockIdx.x * 16 * RT;
    f32x4_t acc[1][RT];
    oneshot_products<B, G, 1, RT, true>(acc, o, wave, ns, kw, lane, [] {});
#pragma unroll
    for (int t = 0; t < RT; ++t) red[(wave * RT + t) * 64 + lane] = acc[0][t] * kTileUnscale;
    __syncthreads();
    for (int t = wave; t < RT; t += kw) {
        f32x4_t s = red[t * 64 + lane];
        for (int w = 1; w < kw; ++w) s += red[(w * RT + t) * 64 + lane];
        const int n = o.row0 + 16 * t + j;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int i = __shfl(bl.inst, 4 * q + v, 64);
            if (4 * q + v < bl.n && n < a.d)
                a.part[(long)i * a.d + n] = s[v];
        }
    }
}

// y[m] = sum of w[m][j] part[m k + j], j ascending; slots without an expert add
// nothing (their parts, which no launch wrote, are loaded all the same: a load
// behind a load of the slot's expert would wait for it: 2.2 to 4.7 us, a launch).
__global__ void __launch_bounds__(256) moe_combine_kernel(MoeArgs a) {
    constexpr int N = 8;
    const int m = blockIdx.y, c = (blockIdx.x * 256 + threadIdx.x) * 4;
    if (c >= a.d)
        return;
    f32x4_t s = {0.f, 0.f, 0.f, 0.f};
    for (int j0 = 0; j0 < a.k; j0 += N) {
        f32x4_t p[N];
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (j0 + j < a.k)
                p[j] = *reinterpret_cast<const f32x4_t*>(a.part + (long)(m * a.k + j0 + j) * a.d + c);
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (j0 + j < a.k && a.idx[m * a.k + j0 + j] >= 0)
                s += a.w[m * a.k + j0 + j] * p[j];
    }
    *reinterpret_cast<uint2*>(a.y + (long)m * a.d + c) = make_uint2(f2h(s[0]) | f2h(s[1]) << 16, f2h(s[2]) | f2h(s[3]) << 16);
}

}  // namespace

hipError_t launch_moe_experts(const MoeArgs& a, hipStream_t st) {
    const int n = a.M * a.k, nb = moe_blocks_most(n, a.E);
    moe_choose_kernel<<<1u + (unsigned)a.M, kChooseWaves * 64, 0, st>>>(a);
    hipError_t err = hipGetLastError();
    if (err != hipSuccess)
        return err;
    if (a.r > 0) {
        moe_shrink_kernel<<<dim3((unsigned)a.r / 8, (unsigned)nb), kShrinkWaves * 64, 0, st>>>(a);
        if ((err = hipGetLastError()) != hipSuccess)
            return err;
    }
    auto run = [&](auto k, int K, int bits, int rows, int nm, int rt) {
        const int ns = oneshot_steps(K, bits), kw = oneshot_waves(ns);
        k<<<dim3((unsigned)(rows + 16 * rt - 1) / (16 * rt), (unsigned)nb), (unsigned)kw * 64, (size_t)kw * nm * rt * 1024, st>>>(a, ns, kw);
        return hipGetLastError();
    };
    // Down takes two tiles (us, d = f = 2880, 4 of 32 experts, one tile and two: M = 1 7.2 and 8.3, 8 29.6 and 25.5, 64
    // 59.2 and 47.9).
    const bool two = moe_two_tiles(n, a.E, a.f, a.gb, plan_cus());
    err = hipErrorInvalidValue;
#define QMLP_MG(B_, G_)                                                                             \
    if (a.gb == B_ && a.gg == G_)                                                                   \
        err = two ? run(moe_gateup_kernel<B_, G_, 2>, a.d, B_, a.f, 2, 2) : run(moe_gateup_kernel<B_, G_, 1>, a.d, B_, a.f, 2, 1);
    QMLP_MG(2, 32) QMLP_MG(2, 64) QMLP_MG(2, 128) QMLP_MG(4, 32) QMLP_MG(4, 64) QMLP_MG(4, 128)
    if (err != hipSuccess)
        return err;
    err = hipErrorInvalidValue;
#define QMLP_MD(B_, G_)           \
    if (a.db == B_ && a.dg == G_) \
        err = run(moe_down_kernel<B_, G_, 2>, a.f, B_, a.d, 1, 2);
    QMLP_MD(2, 32) QMLP_MD(2, 64) QMLP_MD(2, 128) QMLP_MD(4, 32) QMLP_MD(4, 64) QMLP_MD(4, 128)
    if (err != hipSuccess)
        return err;
    moe_combine_kernel<<<dim3((unsigned)(a.d + 1023) / 1024, (unsigned)a.M), 256, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace qmlp
