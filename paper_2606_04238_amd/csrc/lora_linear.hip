// A quantized linear with low-rank adapters of many requests (gfx950):
//   y[m] = W x[m] + s_a B_a (A_a x[m]),   a = ids[m]
// (Sec. 3.1 Eq. (1) with an adapter per row; Sec. 4.2, the adapters stay
// separate from the quantized base, which is what lets requests share it).
// This file: the preparation launch (t = s_a A_a x, and bfloat16 rows as
// binary16) and the linear of up to 16 rows; lora_gemm.hip has more rows.
//
// bfloat16 rows.  The matrix-core arithmetic on packed codes is binary16
// (oneshot.h, lora_gemm.hip), so a bfloat16 row enters as x 2^e with the largest |x| in
// [2^14, 2^15) and its finished sums leave times 2^-e.  Both are exact for
// every element down to 2^-28 of the row's largest (binary16 keeps 11 bits of
// a bfloat16's 8 down to 2^-14); what is lost below that is under 2^-39 of the
// largest element.
#include "lora_linear.h"
#include "decode_launch.h"
#include "oneshot.h"

namespace qmlp {
namespace {

constexpr int kPrepWaves = 8, kPrepRowGroups = 256;
constexpr int kLoraPrepRows = 256;       // more rows: lora_prep_many_kernel

// s[r] += x[k .. k + 7] . (row r of A)[k .. k + 7], eight rows a.k apart.
template <int NR>
__device__ __forceinline__ void ranks_dot(float (&s)[NR], const LoraArgs& a, const uint16_t* xr, const uint16_t* ar, int k) {
    const uint4 xv = *reinterpret_cast<const uint4*>(xr + k);
    uint4 av[NR];
#pragma unroll
    for (int r = 0; r < NR; ++r) av[r] = *reinterpret_cast<const uint4*>(ar + (long)r * a.k + k);
    float x[8];
    act8(xv, a.bf, x);
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        float v[8];
        act8(av[r], a.bf, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) s[r] = __builtin_fmaf(x[i], v[i], s[r]);
    }
}

// Row m as binary16 x 2^e, and 2^-e, by one wave: rows of up to 4096 elements stay
// in its registers between the two passes.
__device__ __forceinline__ void convert_row(const LoraArgs& a, int m, int lane) {
    constexpr int N = 8;
    const uint16_t* xr = a.x + (long)m * a.ldx;
    uint16_t* o = a.x16 + (long)m * a.k;
    uint4 v[N];
    float top = 0.0f;
    for (int k0 = 0; k0 < a.k; k0 += N * 512) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int k = k0 + i * 512 + lane * 8;
            v[i] = k < a.k ? *reinterpret_cast<const uint4*>(xr + k) : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float f[8];
            act8(v[i], true, f);
#pragma unroll
            for (int u = 0; u < 8; ++u) top = fmaxf(top, fabsf(f[u]));
        }
    }
#pragma unroll
    for (int s = 1; s < 64; s *= 2) top = fmaxf(top, __shfl_xor(top, s, 64));
    const int e = row_shift(top);
    const float up = __uint_as_float((uint32_t)(127 + e) << 23);
    for (int k0 = 0; k0 < a.k; k0 += N * 512) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int k = k0 + i * 512 + lane * 8;
            if (k >= a.k)
                continue;
            if (a.k > N * 512)
                v[i] = *reinterpret_cast<const uint4*>(xr + k);
            float f[8];
            act8(v[i], true, f);
            uint32_t w[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) w[u] = f2h(f[2 * u] * up) | (f2h(f[2 * u + 1] * up) << 16);
            *reinterpret_cast<uint4*>(o + k) = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
    if (lane == 0)
        a.xf[m] = __uint_as_float((uint32_t)(127 - e) << 23);
}

// t[m][r] as the linear's launch reads it: fp32, or two bfloat16 terms.
__device__ __forceinline__ void put_t(const LoraArgs& a, int m, int r, float t) {
    const long at = (long)m * a.R + r;
    if (a.tb) {
        const uint32_t hi = act_bits(t, true);
        a.tb[at] = (uint16_t)hi;
        a.tb[(long)a.M * a.R + at] = act_bits(t - __uint_as_float(hi << 16), true);
    } else {
        a.t[at] = t;
    }
}

// slots[s] of every set of 32 rows: its number among those with more than
// kMixedFrom adapters (none counts as one), -1 past kMixedSets and for the others;
// where a set has a number, its place at [sets + number].  One workgroup.
__device__ __forceinline__ void lora_find_mixed(const LoraArgs& a, int tid) {
    __shared__ int count[kPrepWaves * 64];
    constexpr int N = kPrepWaves * 64;
    const int sets = (a.M + 31) / 32, per = (sets + N - 1) / N;           // at most 64: M <= 2^20
    unsigned long long mine = 0;
    for (int i = 0; i < per && tid * per + i < sets; ++i) {
        const int s = tid * per + i, n = min(32, a.M - 32 * s);
        int v[32];
#pragma unroll
        for (int u = 0; u < 32; ++u) v[u] = a.ids[32 * (long)s + (u < n ? u : 0)];
        // distinct ones, up to kMixedFrom + 1
        int seen[kMixedFrom], d = 0;
#pragma unroll
        for (int u = 0; u < 32; ++u) {
            const int id = v[u] >= 0 && v[u] < a.T ? v[u] : -1;
            bool is = false;
#pragma unroll
            for (int k = 0; k < kMixedFrom; ++k) is = is || (k < d && seen[k] == id);
            if (!is) {
#pragma unroll
                for (int k = 0; k < kMixedFrom; ++k) seen[k] = k == d ? id : seen[k];
                ++d;
            }
        }
        mine |= (unsigned long long)(d > kMixedFrom) << i;
    }
    const int c = __popcll(mine);
    count[tid] = c;
    __syncthreads();
    for (int o = 1; o < N; o *= 2) {
        const int v = tid >= o ? count[tid - o] : 0;
        __syncthreads();
        count[tid] += v;
        __syncthreads();
    }
    int at = count[tid] - c;
    for (int i = 0; i < per && tid * per + i < sets; ++i) {
        const bool m = mine >> i & 1;
        a.slots[tid * per + i] = m && at < kMixedSets ? at : -1;
        if (m && at < kMixedSets)
            a.slots[sets + at] = tid * per + i;
        at += m;
    }
    if (tid >= count[N - 1] && tid < kMixedSets)
        a.slots[sets + tid] = -1;
}

// Adapter terms B_a t of four rows and 256 outputs by a workgroup, past 16 rows: RC
// neighbouring lanes take a row of B (8 RC ranks), so that its lines are read whole,
// and everything is loaded before the first product.  (A lane a row of B, 64 ranks,
// 48 rows of 4096, n = 6144: 19.5 us instead of 13.8.)
constexpr int kTermRows = 4;
template <int RC>
struct Terms {
    static constexpr int PC = 256 / RC;                    // columns of a pass, RC passes
    int ad[kTermRows];
    uint4 b[kTermRows][RC], t0[kTermRows], t1[kTermRows];
    __device__ __forceinline__ void load(const LoraArgs& a, int m0, int c0, int tid) {
        const int k = 8 * (tid % RC);
#pragma unroll
        for (int r = 0; r < kTermRows; ++r) {
            const int m = min(m0 + r, a.M - 1), v = a.ids[m];
            ad[r] = m0 + r < a.M && v >= 0 && v < a.T ? v : -1;
            t0[r] = ld16(a.tb + (long)m * a.R + k);
            t1[r] = ld16(a.tb + ((long)a.M + m) * a.R + k);
        }
#pragma unroll
        for (int r = 0; r < kTermRows; ++r)
#pragma unroll
            for (int p = 0; p < RC; ++p)
                b[r][p] = ld16(a.B + ((long)max(ad[r], 0) * a.n + min(c0 + p * PC + tid / RC, a.n - 1)) * a.R + k);
    }
    // s[r] += row r's term of column c0 + tid (not 0 B where there is no adapter: one's infinities are its own rows')
    __device__ __forceinline__ void add(float (&s)[kTermRows], float (&at)[kTermRows][256], bool bf, int tid) const {
#pragma unroll
        for (int r = 0; r < kTermRows; ++r) {
            float t[8], lo[8];
            act8(t0[r], true, t);
            act8(t1[r], true, lo);
#pragma unroll
            for (int i = 0; i < 8; ++i) t[i] += lo[i];
#pragma unroll
            for (int p = 0; p < RC; ++p) {
                float w[8], u = 0.0f;
                act8(b[r][p], bf, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) u = __builtin_fmaf(t[i], w[i], u);
                if constexpr (RC > 1)
                    u = group_sum<RC>(u);
                if (tid % RC == 0)
                    at[r][p * PC + tid / RC] = u;
            }
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kTermRows; ++r)
            if (ad[r] >= 0)
                s[r] += at[r][tid];
    }
};

// The terms of the rows of the mixed sets, a workgroup's slots kMixedStride apart (most
// calls have few).  (In the product's launch itself these rows' adapters, one after
// another, held their workgroups back: 4096 rows of which 48 decode, rank 64, 391 us
// instead of 344 with one adapter; 600 rows of 64 adapters, rank 64, three of 19
// sets there, 1024 x 1024: 115 us, 16.3 without.)
constexpr int kMixedStride = 16;
template <int RC>
__global__ void __launch_bounds__(256) lora_mixed_kernel(LoraArgs a, int most) {
    __shared__ float at[kTermRows][256];
    const int tid = threadIdx.x, c = blockIdx.x * 256 + tid, r0 = kTermRows * (blockIdx.y & 7);
    for (int slot = blockIdx.y >> 3; slot < most; slot += kMixedStride) {
        const int set = a.slots[(a.M + 31) / 32 + slot];
        if (set < 0)
            return;
        Terms<RC> x;
        x.load(a, 32 * set + r0, blockIdx.x * 256, tid);
        float s[kTermRows] = {};
        x.add(s, at, a.bf, tid);
        if (c < a.n)
#pragma unroll
            for (int u = 0; u < kTermRows; ++u) a.mixed[((long)slot * 32 + r0 + u) * a.n + c] = s[u];
        __syncthreads();                                   // (at is free again)
    }
}

// y = the sum of the shares of k, in their order, and the adapters' terms.
template <int RC>
__global__ void __launch_bounds__(256) lora_join_kernel(LoraArgs a) {
    constexpr bool ADS = RC > 0;                           // (0: no adapters)
    constexpr int P = 8;                                   // shares loaded at once
    __shared__ float at[kTermRows][256];
    const int tid = threadIdx.x, m0 = blockIdx.y * kTermRows, c = blockIdx.x * 256 + tid;
    Terms<ADS ? RC : 1> x;
    if constexpr (ADS)
        x.load(a, m0, blockIdx.x * 256, tid);
    float s[kTermRows] = {};
    for (int i0 = 0; i0 < a.shares; i0 += P) {
        float p[P][kTermRows];
#pragma unroll
        for (int i = 0; i < P; ++i)
#pragma unroll
            for (int r = 0; r < kTermRows; ++r)
                p[i][r] = a.parts[((long)min(i0 + i, a.shares - 1) * a.M + min(m0 + r, a.M - 1)) * a.n + min(c, a.n - 1)];
#pragma unroll
        for (int i = 0; i < P; ++i)
#pragma unroll
            for (int r = 0; r < kTermRows; ++r) s[r] += i0 + i < a.shares ? p[i][r] : 0.0f;
    }
    if constexpr (ADS)
        x.add(s, at, a.bf, tid);
#pragma unroll
    for (int r = 0; r < kTermRows; ++r)
        if (m0 + r < a.M && c < a.n)
            a.y[(long)(m0 + r) * a.ldy + c] = act_bits(s[r], a.bf);
}

// blockIdx.x: token, blockIdx.y: NR ranks of t, or (the last one) the row's conversion
// to operands, past 16 rows of bfloat16 to binary16.  t: the waves split k, a lane
// takes eight elements of x and of NR rows of A at a time, fp32 throughout.  Eight
// ranks share a read of x; two where that leaves few workgroups, each of
// which reads no more than one compute unit can (us: one row of 17408, rank 16 7.8
// with two, 14.0 with eight; of 9728, rank 64 6.0 and 9.9).
template <int NR>
__global__ void __launch_bounds__(kPrepWaves * 64) lora_prep_kernel(LoraArgs a) {
    const int m = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int ny = a.T > 0 ? a.R / NR : 0;
    if (m >= a.M) {
        if (blockIdx.y == 0)
            lora_find_mixed(a, tid);
        return;
    }
    if ((int)blockIdx.y >= ny) {
        if (a.xo)
            operands_of_row<kPrepWaves>(a.x + (long)m * a.ldx, a.k, a.bf, a.bits, a.g, reinterpret_cast<uint4*>(a.xo) + m,
                                        reinterpret_cast<float2*>(a.xs) + m, a.M, a.xf + m, tid);
        else if (wave == 0)
            convert_row(a, m, lane);
        return;
    }
    const uint16_t* xr = a.x + (long)m * a.ldx;
    const int id = a.ids[m], r0 = blockIdx.y * NR;
    if (a.t && blockIdx.y == 0 && tid < 16) {
        if (tid == m)
            a.known[m] = id >= 0 && id < a.T ? id : -1;
        else if (m == 0 && tid >= a.M)
            a.known[tid] = -1;
    }
    if (id < 0 || id >= a.T) {
        if (tid < NR)
            put_t(a, m, r0 + tid, 0.0f);
        return;
    }
    const uint16_t* ar = a.A + ((long)id * a.R + r0) * a.k;
    float s[NR] = {};
    for (int k = tid * 8; k < a.k; k += kPrepWaves * 64 * 8) ranks_dot<NR>(s, a, xr, ar, k);
    __shared__ float red[kPrepWaves][NR];
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        const float v = group_sum<64>(s[r]);
        if (lane == 0)
            red[wave][r] = v;
    }
    __syncthreads();
    if (tid < NR) {
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < kPrepWaves; ++w) v += red[w][tid];
        put_t(a, m, r0 + tid, (a.scale ? a.scale[id] : 1.0f) * v);
    }
}

// t of row m by one workgroup: R / 8 sets of waves take eight ranks each and split k.
__device__ __forceinline__ void lora_row(const LoraArgs& a, int m, int id, float* rs, int tid) {
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int per = kPrepWaves * 8 / a.R, r0 = 8 * (wave / per);
    float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (id >= 0) {
        const uint16_t* xr = a.x + (long)m * a.ldx;
        const uint16_t* ar = a.A + ((long)id * a.R + r0) * a.k;
        for (int k = ((wave % per) * 64 + lane) * 8; k < a.k; k += per * 64 * 8) ranks_dot<8>(s, a, xr, ar, k);
    }
#pragma unroll
    for (int r = 0; r < 8; ++r) {
        const float v = group_sum<64>(s[r]);
        if (lane == 0)
            rs[wave * 8 + r] = v;
    }
    __syncthreads();
    if (tid < a.R) {
        float v = 0.0f;
        for (int w = 0; w < per; ++w) v += rs[((tid >> 3) * per + w) * 8 + (tid & 7)];
        put_t(a, m, tid, id < 0 ? 0.0f : (a.scale ? a.scale[id] : 1.0f) * v);
    }
    __syncthreads();
}

// The adapters of the 16 rows of a tile (lane j: row j): the first, the first that
// differs, and whether there are more.
struct TileAds {
    int id, id0, id1;
    bool more;
};
__device__ __forceinline__ TileAds tile_adapters(const LoraArgs& a, int m0, int j) {
    const int v = m0 + j < a.M ? a.ids[m0 + j] : -1;
    TileAds t;
    t.id = v >= 0 && v < a.T ? v : -1;
    const uint32_t any = (uint32_t)__ballot(t.id >= 0) & 0xFFFFu;
    t.id0 = any ? __builtin_amdgcn_readlane(t.id, __builtin_ctz(any)) : -1;
    const uint32_t rest = any & ~((uint32_t)__ballot(t.id == t.id0) & 0xFFFFu);
    t.id1 = rest ? __builtin_amdgcn_readlane(t.id, __builtin_ctz(rest)) : -1;
    t.more = (rest & ~((uint32_t)__ballot(t.id == t.id1) & 0xFFFFu)) != 0;
    return t;
}

// The same for many rows, one workgroup after another: one that finds the mixed
// sets; one per 16 rows, which multiplies them on the matrix cores where they
// have at most two adapters between them (a prompt); kPrepRowGroups that share
// the rows of the other tiles, a row at a time; and those that convert.  (A
// workgroup per row and eight ranks would read x and A R / 8 and M times: at 4096
// rows of rank 64 200 us.  16 per tile of which most have nothing to do: 115.)
__global__ void __launch_bounds__(kPrepWaves * 64) lora_prep_many_kernel(LoraArgs a, int tiles, int rowgroups) {
    __shared__ f32x4_t red[kPrepWaves][4][64];
    const int tid = threadIdx.x, lane = tid & 63, j = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int block = blockIdx.x;
    if (block == 0) {
        if (tiles > 0)
            lora_find_mixed(a, tid);
        return;
    }
    block -= 1;
    if (block < rowgroups) {
        // sets of kPrepWaves * 4 tiles: a wave looks at four of them, 16 rows each
        __shared__ unsigned long long flags;
        int seen = 0;                                      // rows of earlier tiles
        for (int t0 = 0; t0 < tiles; t0 += 64) {
            if (tid == 0)
                flags = 0;
            __syncthreads();
            unsigned long long f = 0;
            for (int u = wave; u < 64 && t0 + u < tiles; u += kPrepWaves)
                if (tile_adapters(a, 16 * (t0 + u), j).more)
                    f |= 1ull << u;
            if (lane == 0 && f)
                atomicOr(&flags, f);
            __syncthreads();
            f = flags;
            __syncthreads();
            for (; f; f &= f - 1) {
                const int m0 = 16 * (t0 + __builtin_ctzll(f));
                // this workgroup's rows of the 16: numbers block, block + rowgroups, ..
                for (int p = (block - seen % rowgroups + rowgroups) % rowgroups; p < 16; p += rowgroups) {
                    const int m = m0 + p;
                    if (m < a.M) {
                        const int v = a.ids[m];
                        lora_row(a, m, v >= 0 && v < a.T ? v : -1, reinterpret_cast<float*>(red), tid);
                    }
                }
                seen += 16;
            }
        }
        return;
    }
    block -= rowgroups;
    if (block >= tiles) {
        const int m = (block - tiles) * kPrepWaves + wave;
        if (m < a.M)
            convert_row(a, m, lane);
        return;
    }
    const int m0 = block * 16;
    const TileAds t = tile_adapters(a, m0, j);
    if (t.more)
        return;
    const uint16_t* xr = a.x + (long)(m0 + j < a.M ? m0 + j : a.M - 1) * a.ldx + 8 * q;
    const int rt = (a.R + 15) / 16, n = a.k / 32;
    f32x4_t out = {0.f, 0.f, 0.f, 0.f};                    // wave w < rt: ranks 16 w ..
    for (int u = 0; u < 2; ++u) {
        const int ad = u ? t.id1 : t.id0;
        if (ad < 0)
            break;
        const uint16_t* ar = a.A + (long)ad * a.R * a.k + 8 * q;
        f32x4_t acc[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[c] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll 2
        for (int s = wave; s < n; s += kPrepWaves) {
            const uint4 xv = *reinterpret_cast<const uint4*>(xr + 32 * s);
            uint4 av[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const int rk = 16 * c + j < a.R ? 16 * c + j : a.R - 1;
                if (c < rt)
                    av[c] = *reinterpret_cast<const uint4*>(ar + (long)rk * a.k + 32 * s);
            }
#pragma unroll
            for (int c = 0; c < 4; ++c)
                if (c < rt)
                    acc[c] = a.bf ? mfma16_bf(xv, av[c], acc[c]) : mfma16(xv, av[c], acc[c]);
        }
        __syncthreads();
#pragma unroll
        for (int c = 0; c < 4; ++c)
            if (c < rt)
                red[wave][c][lane] = acc[c];
        __syncthreads();
        if (wave < rt) {
            f32x4_t v = red[0][wave][lane];
#pragma unroll
            for (int w = 1; w < kPrepWaves; ++w) v += red[w][wave][lane];
            const float sc = a.scale ? a.scale[ad] : 1.0f;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (__builtin_amdgcn_ds_bpermute(4 * (4 * q + i), t.id) == ad)
                    out[i] = sc * v[i];
        }
    }
    if (wave < rt && 16 * wave + j < a.R)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (m0 + 4 * q + i < a.M)
                put_t(a, m0 + 4 * q + i, 16 * wave + j, out[i]);
}

// An item of the adapters' share of RT tiles, it = 4 c + v: eight ranks, 8 c .., for
// the tokens 4 q + v; B_a[o][8 c ..] of the lane's row o = row0 + 16 t + j.  A row
// with no adapter adds nothing (not 0 B: an adapter that holds infinities belongs
// to its own rows only).
template <int RT>
struct Rank8 {
    int id;
    uint4 b[RT];
    f32x4_t t[2];
};
template <int RT>
__device__ __forceinline__ void rank8_load(Rank8<RT>& k, const LoraArgs& a, int row0, int it, int lane) {
    const int q = lane >> 4, j = lane & 15, v = it & 3, c = it >> 2;
    // uniform addresses: scalar loads, which do not queue behind the weights
    const int i0 = a.known[v], i1 = a.known[4 + v], i2 = a.known[8 + v], i3 = a.known[12 + v];
    k.id = q < 2 ? (q == 0 ? i0 : i1) : (q == 2 ? i2 : i3);
    if (k.id >= 0) {
        const f32x4_t* tp = reinterpret_cast<const f32x4_t*>(a.t + (long)(4 * q + v) * a.R + 8 * c);
        k.t[0] = tp[0];
        k.t[1] = tp[1];
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            const int o = row0 + 16 * t + j < a.n ? row0 + 16 * t + j : a.n - 1;
            k.b[t] = *reinterpret_cast<const uint4*>(a.B + ((long)k.id * a.n + o) * a.R + 8 * c);
        }
    }
}
template <int RT>
__device__ __forceinline__ void rank8_add(f32x4_t (&acc)[1][RT], const Rank8<RT>& k, int it, bool bf) {
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        float b[8], s = 0.0f;
        act8(k.b[t], bf, b);
#pragma unroll
        for (int i = 0; i < 8; ++i) s = __builtin_fmaf(b[i], k.t[i >> 2][i & 3], s);
        s = k.id >= 0 ? s : 0.0f;
#pragma unroll
        for (int v = 0; v < 4; ++v)
            if (v == (it & 3))
                acc[0][t][v] += s;
    }
}

// Up to 16 rows of x: a workgroup owns RT tiles of 16 outputs (oneshot.h), the
// waves share its adapters' terms by eight ranks.  Measured (us, 4 bits): one row of
// 2560 x 4096 6.6, 16 of 6144 x 4096 with rank 32 11.0, 7 of 5120 x 17408 25.6 (1.9
// TB/s; its codes alone in the same pieces 16.8).
template <int B, int G, int RT>
__global__ void __launch_bounds__(512) lora_few_kernel(LoraArgs a, int ns, int kw) {
    extern __shared__ uint4 smem[];
    f32x4_t* red = reinterpret_cast<f32x4_t*>(smem);       // [kw][RT][64]
    const int lane = threadIdx.x & 63, j = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int rb = a.k * B / 8, ng = a.k / G;
    OneWork<1> o;
    one_magic(o);
    o.rc[0] = rsrc(a.codes, (uint32_t)a.n * (uint32_t)rb);
    o.rm[0] = rsrc(a.meta, (uint32_t)a.n * (uint32_t)ng * 4u);
    o.rows = (uint32_t)a.M;
    o.rx = rsrc(a.xo, (uint32_t)a.M * operand_row(a.k, B) * 2u);
    o.rs = rsrc(a.xs, (uint32_t)a.M * operand_sums(a.k, B, G) * 4u);
    place<B, G>(o, 16u * j, 8u * j, j < a.M, lane >> 4);
    o.K = a.k;
    o.N = a.n;
    o.row0 = blockIdx.x * 16 * RT;
    const int items = a.T > 0 ? a.R / 2 : 0;
    f32x4_t acc[1][RT];
    Rank8<RT> k8;
    float f[4] = {1.f, 1.f, 1.f, 1.f};
    oneshot_products<B, G, 1, RT, false>(acc, o, wave, ns, kw, lane, [&] {
        if (wave < items)
            rank8_load<RT>(k8, a, o.row0, wave, lane);
        if (a.bf)
#pragma unroll
            for (int v = 0; v < 4; ++v) f[v] = a.xf[4 * (lane >> 4) + v < a.M ? 4 * (lane >> 4) + v : 0];
    });
    // the factor of bfloat16 rows, before terms that do not have it
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int v = 0; v < 4; ++v) acc[0][t][v] *= kTileUnscale * f[v];
    if (wave < items)
        rank8_add<RT>(acc, k8, wave, a.bf);
    for (int it = wave + kw; it < items; it += kw) {
        rank8_load<RT>(k8, a, o.row0, it, lane);
        rank8_add<RT>(acc, k8, it, a.bf);
    }
#pragma unroll
    for (int t = 0; t < RT; ++t) red[(wave * RT + t) * 64 + lane] = acc[0][t];
    __syncthreads();
    for (int t = wave; t < RT; t += kw) {
        f32x4_t s = red[t * 64 + lane];
        for (int w = 1; w < kw; ++w) s += red[(w * RT + t) * 64 + lane];
        const int n = o.row0 + 16 * t + j;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int tok = 4 * (lane >> 4) + v;
            if (tok < a.M && n < a.n)
                a.y[(long)tok * a.ldy + n] = act_bits(s[v], a.bf);
        }
    }
}

}  // namespace

hipError_t launch_lora_prep(const LoraArgs& a, hipStream_t st) {
    const int nr = (long)a.M * a.R / 8 < 128 ? 2 : 8;
    const unsigned ny = (a.T > 0 ? a.R / nr : 0) + (a.bf || a.xo ? 1 : 0);
    if (ny == 0)
        return hipSuccess;
    if (a.M > kLoraPrepRows) {
        const int tiles = a.T > 0 ? (a.M + 15) / 16 : 0;
        const int rowgroups = tiles == 0 ? 0 : 16 * tiles < kPrepRowGroups ? 16 * tiles : kPrepRowGroups;
        const unsigned convert = a.bf ? (unsigned)(a.M + kPrepWaves - 1) / kPrepWaves : 0u;
        lora_prep_many_kernel<<<1u + rowgroups + tiles + convert, kPrepWaves * 64, 0, st>>>(a, tiles, rowgroups);
        return hipGetLastError();
    }
    const bool find = a.T > 0 && a.tb && !a.parts;                     // one more column of workgroups looks for the mixed sets
    (nr == 2 ? lora_prep_kernel<2> : lora_prep_kernel<8>)<<<dim3((unsigned)a.M + (find ? 1u : 0u), ny), kPrepWaves * 64, 0, st>>>(a);
    return hipGetLastError();
}

hipError_t launch_lora_mixed(const LoraArgs& a, hipStream_t st) {
    auto k = a.R == 8 ? lora_mixed_kernel<1> : a.R == 16 ? lora_mixed_kernel<2> : a.R == 32 ? lora_mixed_kernel<4> : lora_mixed_kernel<8>;
    const int most = lora_mixed_most(a.M);
    k<<<dim3((unsigned)(a.n + 255) / 256, 8u * (unsigned)(most < kMixedStride ? most : kMixedStride)), 256, 0, st>>>(a, most);
    return hipGetLastError();
}

hipError_t launch_lora_join(const LoraArgs& a, hipStream_t st) {
    auto k = a.T == 0 ? lora_join_kernel<0> : a.R == 8 ? lora_join_kernel<1> : a.R == 16 ? lora_join_kernel<2> : a.R == 32 ? lora_join_kernel<4> : lora_join_kernel<8>;
    k<<<dim3((unsigned)(a.n + 255) / 256, (unsigned)(a.M + kTermRows - 1) / kTermRows), 256, 0, st>>>(a);
    return hipGetLastError();
}

hipError_t launch_lora_few(const LoraArgs& a, hipStream_t st) {
    if (a.M < 1 || a.M > kLoraFewTokens)
        return hipErrorInvalidValue;
    const int rt = lora_few_tiles(a.n, a.cus), ns = oneshot_steps(a.k, a.bits), kw = oneshot_waves(ns);
    const unsigned grid = (unsigned)((a.n + 16 * rt - 1) / (16 * rt));
    auto run = [&](auto k) {
        k<<<grid, (unsigned)kw * 64, (size_t)kw * rt * 1024, st>>>(a, ns, kw);
        return hipGetLastError();
    };
#define QMLP_LF(B_, G_)            \
    if (a.bits == B_ && a.g == G_) \
        return rt == 1 ? run(lora_few_kernel<B_, G_, 1>) : run(lora_few_kernel<B_, G_, 2>);
    QMLP_LF(2, 32) QMLP_LF(2, 64) QMLP_LF(2, 128) QMLP_LF(4, 32) QMLP_LF(4, 64) QMLP_LF(4, 128)
    return hipErrorInvalidValue;
}

}  // namespace qmlp
