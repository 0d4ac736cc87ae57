// The linear with adapters of many requests at more than 16 rows (gfx950),
// y = x W^T + s_a (x A_a^T) B_a^T, a dense product on the matrix cores:
// weights are unpacked to binary16 in LDS, scale * (q - zero) rounded once (the
// value qmlp_dequant gives; 2^-12 relative at most, as much as one rounding of
// the output, and independent from group to group) and multiplied with
// v_mfma_f32_32x32x16_f16.  bfloat16 rows come as binary16 times a power of two
// (lora_linear.hip), so both types run the same products.
//
// Adapters first: the accumulators start as s_a B_a t of each row.  The
// distinct adapters of a workgroup's rows are found in LDS, and for each of
// them t and B_a are multiplied for all rows, of which only its own take the
// sums (a select, not a product with zero: an adapter that holds infinities
// stays with its own rows).  Binary16: t is rounded to it after a power of two
// per row that brings its largest into [2^14, 2^15), 2^-12 of the adapter's
// term.  bfloat16: t enters as two bfloat16 terms (2^-17) beside B_a as it is,
// whose range is that of fp32.  The sums take the row's powers of two before the
// weights' products are added.
//
// Tile engine: BM rows x BN outputs per workgroup, K in steps of 64 staged in
// LDS, chunk c of row r at c ^ ((r >> 1) & 7), two buffers, the next step's
// loads in registers while a step runs (prefill.hip's scheme).
#include "lora_linear.h"
#include "decode_launch.h"
#include "oneshot.h"

namespace qmlp {
namespace {

typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

__device__ __forceinline__ f32x16_t mfma32(const uint4& a, const uint4& b, const f32x16_t& c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c, 0,
                                                  0, 0);
}
__device__ __forceinline__ f32x16_t mfma32_bf(const uint4& a, const uint4& b, const f32x16_t& c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c,
                                                   0, 0, 0);
}
__device__ __forceinline__ uint4 ld16(const void* p) {
    const u32x4 v = *reinterpret_cast<const u32x4*>(p);
    return make_uint4(v.x, v.y, v.z, v.w);
}
__device__ __forceinline__ void st16(uint4* p, const uint4& v) { *reinterpret_cast<u32x4*>(p) = u32x4{v.x, v.y, v.z, v.w}; }
__device__ __forceinline__ int swz(int r, int c) { return r * 8 + (c ^ ((r >> 1) & 7)); }
// Row of accumulator element v of a 32 x 32 tile (the column is lane & 31).
__device__ __forceinline__ int acc_row(int v, int lane) { return 8 * (v >> 2) + 4 * (lane >> 5) + (v & 3); }

__device__ __forceinline__ uint32_t pk_add(uint32_t a, uint32_t b) {
    return __builtin_bit_cast(uint32_t, __builtin_bit_cast(half2_t, a) + __builtin_bit_cast(half2_t, b));
}

// CPT codes of one row to binary16 scale * (q - zero), CPT / 8 chunks: a pair
// of codes as 1024 + q (one and-or), minus 1024 + zero (exact), times scale.
template <int BITS, int CPT>
__device__ __forceinline__ void dequant_store(uint4* lds, const uint32_t (&w)[BITS * CPT / 32], uint32_t meta, int row,
                                              int part) {
    const uint32_t s2 = __builtin_amdgcn_perm(0u, meta, 0x01000100u);
    const uint32_t off = pk_add(0xE400E400u, __builtin_amdgcn_perm(0u, meta, 0x03020302u) ^ 0x80008000u);   // -1024 - z
    constexpr int C0 = CPT / 8, PW = 16 / BITS;            // pairs (c_i, c_{PW + i}) of a word
#pragma unroll
    for (int i = 0; i < BITS * CPT / 32; ++i) {
        uint32_t v[PW];
        constexpr uint32_t mask = BITS == 2 ? 0x00030003u : 0x000F000Fu;
#pragma unroll
        for (int p = 0; p < PW; ++p) v[p] = pk_mul(pk_add(((w[i] >> (BITS * p)) & mask) | 0x64006400u, off), s2);
        if constexpr (BITS == 2) {
            st16(&lds[swz(row, part * C0 + 2 * i)], make_uint4(pair_lo(v[0], v[1]), pair_lo(v[2], v[3]),
                                                               pair_lo(v[4], v[5]), pair_lo(v[6], v[7])));
            st16(&lds[swz(row, part * C0 + 2 * i + 1)], make_uint4(pair_hi(v[0], v[1]), pair_hi(v[2], v[3]),
                                                                   pair_hi(v[4], v[5]), pair_hi(v[6], v[7])));
        } else {
            st16(&lds[swz(row, part * C0 + i)],
                 make_uint4(pair_lo(v[0], v[1]), pair_lo(v[2], v[3]), pair_hi(v[0], v[1]), pair_hi(v[2], v[3])));
        }
    }
}

// Eight values of t as matrix operands: binary16 t f in t0, or the bfloat16
// t and what that leaves in t0 and t1.
__device__ __forceinline__ void adapter_operand(const float (&t)[8], float f, bool bf, uint4& t0, uint4& t1) {
    uint32_t a[4], b[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (bf) {
            const uint32_t l = act_bits(t[2 * i], true), h = act_bits(t[2 * i + 1], true);
            a[i] = l | h << 16;
            b[i] = act_bits(t[2 * i] - __uint_as_float(l << 16), true) |
                   (uint32_t)act_bits(t[2 * i + 1] - __uint_as_float(h << 16), true) << 16;
        } else {
            a[i] = f2h(t[2 * i] * f) | f2h(t[2 * i + 1] * f) << 16;
            b[i] = 0;
        }
    }
    t0 = make_uint4(a[0], a[1], a[2], a[3]);
    t1 = make_uint4(b[0], b[1], b[2], b[3]);
}

template <int BITS, int BM, int BN, int WM, int WN>
__global__ void __launch_bounds__(BM / (32 * WM) * (BN / (32 * WN)) * 64) lora_gemm_kernel(LoraArgs a) {
    constexpr int WMW = BM / (32 * WM), NT = WMW * (BN / (32 * WN)) * 64;
    constexpr int CA = BM * 8 / NT, P = NT / BN, CPT = 64 / P, NW = BITS * CPT / 32;
    static_assert(CA * NT == BM * 8 && P * BN == NT && CPT >= 16 && CPT <= 32 && NW >= 1, "staging shares");
    extern __shared__ uint4 smem[];
    int* rid = reinterpret_cast<int*>(smem + 2 * (BM + BN) * 8);      // [BM] adapter of a row, or -1
    float* rf = reinterpret_cast<float*>(rid + BM);                   // [BM] factor of the adapter's sums
    float* ro = rf + BM;                                              // [BM] factor of the finished row
    int* list = reinterpret_cast<int*>(ro + BM);                      // [BM] distinct adapters
    int* nlist = list + BM;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave % WMW, wn = wave / WMW;
    const int mtiles = (a.M + BM - 1) / BM;
    const int m0 = blockIdx.x % mtiles * BM, n0 = blockIdx.x / mtiles * BN;
    const uint16_t* x = a.x16 ? a.x16 : a.x;
    const long ldx = a.x16 ? a.k : a.ldx;

    // staging: rows past M (n) repeat the last one and are dropped at the end
    const uint16_t* xp[CA];
#pragma unroll
    for (int i = 0; i < CA; ++i) {
        const int id = tid + NT * i, row = m0 + (id >> 3);
        xp[i] = x + (long)(row < a.M ? row : a.M - 1) * ldx + (id & 7) * 8;
    }
    const int trow = tid / P, part = tid % P, wrow = n0 + trow < a.n ? n0 + trow : a.n - 1;
    const uint32_t* crow = a.codes + (long)wrow * (a.k * BITS / 32) + part * NW;
    const uint32_t* mrow = a.meta + (long)wrow * (a.k / a.g);
    uint4 xv[CA];
    uint32_t qw[NW], qm;
    auto load = [&](int k0) {
#pragma unroll
        for (int i = 0; i < CA; ++i) xv[i] = ld16(xp[i] + k0);
        const uint32_t* p = crow + k0 * BITS / 32;
        if constexpr (NW == 4) {
            const uint4 v = ld16(p);
            qw[0] = v.x; qw[1] = v.y; qw[2] = v.z; qw[3] = v.w;
        } else if constexpr (NW == 2) {
            const uint2 v = *reinterpret_cast<const uint2*>(p);
            qw[0] = v.x; qw[1] = v.y;
        } else {
            qw[0] = *p;
        }
        qm = mrow[(k0 + part * CPT) / a.g];
    };
    auto store = [&](uint4* buf) {
#pragma unroll
        for (int i = 0; i < CA; ++i) {
            const int id = tid + NT * i;
            st16(&buf[swz(id >> 3, id & 7)], xv[i]);
        }
        dequant_store<BITS, CPT>(buf + BM * 8, qw, qm, trow, part);
    };
    load(0);

    f32x16_t acc[WM][WN];
#pragma unroll
    for (int i = 0; i < WM; ++i)
#pragma unroll
        for (int j = 0; j < WN; ++j) acc[i][j] = f32x16_t{};
    // adapters of the rows and their distinct ones
    if (tid == 0)
        *nlist = 0;
    for (int i = tid; i < BM; i += NT) {
        const int m = m0 + i;
        int id = m < a.M && a.T > 0 ? a.ids[m] : -1;
        id = id < a.T ? id : -1;
        float top = 0.0f;
        if (id >= 0)
            for (int r = 0; r < a.R; r += 4) {
                const f32x4_t v = *reinterpret_cast<const f32x4_t*>(a.t + (long)m * a.R + r);
                top = fmaxf(fmaxf(top, fmaxf(fabsf(v[0]), fabsf(v[1]))), fmaxf(fabsf(v[2]), fabsf(v[3])));
            }
        const int e = min(14 - ((int)(__float_as_uint(top) >> 23) - 127), 100);
        const float out = a.x16 && m < a.M ? a.xf[m] : 1.0f;
        rid[i] = id;
        rf[i] = a.bf ? 1.0f : __uint_as_float((uint32_t)(127 + e) << 23);
        ro[i] = out;
    }
    __syncthreads();
    for (int i = tid; i < BM; i += NT) {
        const int id = rid[i];
        bool first = id >= 0;
        for (int k = 0; k < i && first; ++k) first = rid[k] != id;
        if (first)
            list[atomicAdd(nlist, 1)] = id;                // the order of the list changes nothing: one adapter per row
    }
    __syncthreads();
    const int r = lane & 31, hk = lane >> 5;
    for (int l = 0; l < *nlist; ++l) {
        const int id = list[l];
#pragma unroll
        for (int i = 0; i < WM; ++i) {
            const int row = wm * 32 * WM + i * 32;
            const int m = m0 + row + r < a.M ? m0 + row + r : a.M - 1;
            if (!__any(rid[row + r] == id))
                continue;
#pragma unroll
            for (int j = 0; j < WN; ++j) {
                const int col = n0 + wn * 32 * WN + j * 32 + r;
                f32x16_t s{};
                for (int k = 0; k < a.R; k += 16) {
                    const int kk = k + 8 * hk;
                    uint4 t0 = make_uint4(0, 0, 0, 0), t1 = t0, bv = t0;
                    if (kk < a.R) {
                        float t[8];
                        const float* tp = a.t + (long)m * a.R + kk;
#pragma unroll
                        for (int u = 0; u < 8; ++u) t[u] = tp[u];
                        adapter_operand(t, rf[row + r], a.bf, t0, t1);
                        bv = ld16(a.B + ((long)id * a.n + (col < a.n ? col : a.n - 1)) * a.R + kk);
                    }
                    s = a.bf ? mfma32_bf(t1, bv, mfma32_bf(t0, bv, s)) : mfma32(t0, bv, s);
                }
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    const int at = row + acc_row(v, lane);
                    acc[i][j][v] = rid[at] == id ? s[v] / rf[at] / ro[at] : acc[i][j][v];
                }
            }
        }
    }

    const int nk = a.k / 64;
    store(smem);
    load(nk > 1 ? 64 : 0);
    for (int kt = 0; kt < nk; ++kt) {
        __syncthreads();
        const uint4* xs = smem + (kt & 1) * (BM + BN) * 8;
        const uint4* ws = xs + BM * 8;
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            uint4 av[WM], bv[WN];
#pragma unroll
            for (int i = 0; i < WM; ++i) av[i] = ld16(&xs[swz(wm * 32 * WM + i * 32 + r, 2 * s + hk)]);
#pragma unroll
            for (int j = 0; j < WN; ++j) bv[j] = ld16(&ws[swz(wn * 32 * WN + j * 32 + r, 2 * s + hk)]);
#pragma unroll
            for (int i = 0; i < WM; ++i)
#pragma unroll
                for (int j = 0; j < WN; ++j) acc[i][j] = mfma32(av[i], bv[j], acc[i][j]);
        }
        store(smem + ((kt + 1) & 1) * (BM + BN) * 8);
        load((kt + 2 < nk ? kt + 2 : nk - 1) * 64);
    }
#pragma unroll
    for (int j = 0; j < WN; ++j) {
        const int col = n0 + wn * 32 * WN + j * 32 + r;
#pragma unroll
        for (int i = 0; i < WM; ++i)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const int at = wm * 32 * WM + i * 32 + acc_row(v, lane), m = m0 + at;
                if (m < a.M && col < a.n)
                    a.y[(long)m * a.ldy + col] = act_bits(acc[i][j][v] * ro[at], a.bf);
            }
    }
}

}  // namespace

hipError_t launch_lora_gemm(const LoraArgs& a, hipStream_t st) {
    auto run = [&](auto k, int BM, int BN, int nt) {
        const size_t lds = (size_t)2 * (BM + BN) * 128 + (size_t)BM * 16 + 16;
        const hipError_t e = set_lds(k, lds);
        if (e != hipSuccess)
            return e;
        const unsigned grid = (unsigned)(((a.M + BM - 1) / BM) * ((a.n + BN - 1) / BN));
        k<<<grid, (unsigned)nt, lds, st>>>(a);
        return hipGetLastError();
    };
    if (a.bits == 2)
        return run(lora_gemm_kernel<2, 128, 128, 2, 2>, 128, 128, 256);
    return run(lora_gemm_kernel<4, 128, 128, 2, 2>, 128, 128, 256);
}

}  // namespace qmlp
