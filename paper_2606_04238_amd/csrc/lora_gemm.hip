// The linear with adapters of many requests at more than 16 rows (gfx950),
// y = x W^T + s_a (x A_a^T) B_a^T, a dense product on the matrix cores:
// weights are unpacked to binary16 in LDS, scale * (q - zero) rounded once (the
// value qmlp_dequant gives; 2^-11 relative at most, as much as one rounding of
// the output, and independent from weight to weight: 4-bit weights take a binary16
// output from 2.1e-4 off 64 bits to 2.7e-4, and 2-bit ones, whose products with an
// 11-bit scale mostly fit, leave it) and multiplied with
// v_mfma_f32_32x32x16_f16.  bfloat16 rows come as binary16 times a power of two
// (lora_linear.hip), so both types run the same products.
//
// Few tiles: k is split into shares, which leave their sums in memory;
// lora_join_kernel adds them and the adapters' terms.
//
// Otherwise adapters first: the accumulators start as B_a t of each row.  Where a wave's rows
// all have one adapter (a prompt), its products go there directly.  Sets of 32 rows
// with many (decoding sequences) find their terms ready in memory
// (lora_mixed_kernel; kMixedSets of them, the first in the call); for the others,
// for each adapter of the 32 rows, t and B_a are multiplied for all of them, and its own rows
// take the sums (a select, not a product with zero: an adapter that holds
// infinities stays with its own rows).  t enters as two bfloat16 terms (2^-17 of
// it), whose range is that of fp32, beside B_a as it is, or as the two bfloat16
// terms that a binary16 value is exactly.
//
// Tile engine: BM rows x BN outputs per workgroup, K in steps of 64 staged in
// LDS, chunk c of row r at c ^ ((r >> 1) & 7).  x is copied to LDS by the memory
// system (ST slots, ST - 1 steps ahead); codes are in registers QA + 1 steps ahead
// and unpacked into two buffers, one step ahead; one barrier per step.  Measured:
// bfloat16 4096 x 6144 x 4096 with rank 64 252 to 262 us from run to run (788 to 818
// TFLOP/s; matrix units busy 39 % of the cycles, 41 % of the waves' time waits), 2-bit
// 333 x 9728 x 2560 37 us in 228 tiles (1.3 waves a SIMD).
#include "lora_linear.h"
#include "decode_launch.h"
#include "oneshot.h"

namespace qmlp {
namespace {

typedef float f32x16_t __attribute__((ext_vector_type(16)));

__device__ __forceinline__ f32x16_t mfma32(const uint4& a, const uint4& b, const f32x16_t& c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c, 0,
                                                  0, 0);
}
__device__ __forceinline__ f32x16_t mfma32_bf(const uint4& a, const uint4& b, const f32x16_t& c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c,
                                                   0, 0, 0);
}
__device__ __forceinline__ void st16(uint4* p, const uint4& v) { *reinterpret_cast<u32x4*>(p) = u32x4{v.x, v.y, v.z, v.w}; }
// 16 bytes per lane from memory to LDS, lane l to lds + l.  (The host's pass knows no such builtin.)
__device__ __forceinline__ void load_to_lds(Rsrc r, uint4* lds, uint32_t voff, uint32_t soff) {
#ifdef __HIP_DEVICE_COMPILE__
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)lds, 16, voff, soff, 0, 0);
#endif
}
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

// The two bfloat16 terms of eight binary16 values (exact: eight bits and the other three).
__device__ __forceinline__ void split_f16(const uint4& v, uint4& hi, uint4& lo) {
    float f[8];
    act8(v, false, f);
    uint32_t h[4], l[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t a = act_bits(f[2 * i], true), b = act_bits(f[2 * i + 1], true);
        h[i] = a | b << 16;
        l[i] = act_bits(f[2 * i] - __uint_as_float(a << 16), true) |
               (uint32_t)act_bits(f[2 * i + 1] - __uint_as_float(b << 16), true) << 16;
    }
    hi = make_uint4(h[0], h[1], h[2], h[3]);
    lo = make_uint4(l[0], l[1], l[2], l[3]);
}

template <int BITS, int BM, int BN, int WM, int WN, int ST, bool SPLIT>
__global__ void __launch_bounds__(BM / (32 * WM) * (BN / (32 * WN)) * 64) lora_gemm_kernel(LoraArgs a, int lg) {
    constexpr int WMW = BM / (32 * WM), NW_ = WMW * (BN / (32 * WN)), NT = NW_ * 64;
    constexpr int CA = BM / (8 * NW_);                     // x loads of a wave and step, eight rows each
    constexpr int P = NT / BN >= 4 ? 4 : NT / BN >= 2 ? 2 : 1, CPT = 64 / P, NW = BITS * CPT / 32;
    static_assert(CA >= 1 && BM % (8 * NW_) == 0 && NT >= BN && CPT <= 32 && NW >= 1, "staging shares");
    constexpr int QA = ST > 3 ? 4 : 2;                     // steps whose codes are in registers or under way
    constexpr int XB = BM * 8, WB = BN * 8;                // 16-byte chunks of a stage
    extern __shared__ uint4 smem[];                        // x [ST][BM][8], weights [2][BN][8], then the rows' 2^-e
    uint4* wsm = smem + ST * XB;
    float* ro = reinterpret_cast<float*>(wsm + 2 * WB);
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave % WMW, wn = wave / WMW;
    // the row tiles' columns one after another: rows of many adapters (usually the first) take longer and start first
    const int ntiles = (a.n + BN - 1) / BN;
    const int m0 = (int)blockIdx.x / ntiles * BM, n0 = (int)blockIdx.x % ntiles * BN;
    // the steps of 64 this workgroup multiplies: all, or its share of k (lora_join_kernel adds shares and adapters)
    const int steps = a.k / 64, share = blockIdx.y, kb = SPLIT ? share * steps / (int)gridDim.y : 0;
    const int nk = SPLIT ? (share + 1) * steps / (int)gridDim.y - kb : steps;
    const long ldx = a.x16 ? a.k : a.ldx;

    // x goes from memory to LDS without registers, eight rows (1 KB) per load: lane l writes chunk l & 7 of row l >> 3,
    // so it reads the chunk that belongs there.  Buffer loads: rows past M (n) read zeros, and are dropped at the end.
    // (Loads to LDS in their global form count as flat ones, and every wait for a register becomes one for all.)
    const int mrows = min(BM, a.M - m0), nrows = min(BN, a.n - n0), rb = a.k * BITS / 8, ng = a.k >> lg;
    const Rsrc rx = rsrc((a.x16 ? a.x16 : a.x) + (long)m0 * ldx, (uint32_t)((mrows - 1) * (int)ldx + a.k) * 2u);
    const Rsrc rc = rsrc(reinterpret_cast<const char*>(a.codes) + (long)n0 * rb, (uint32_t)(nrows * rb));
    const Rsrc rm = rsrc(a.meta + (long)n0 * ng, (uint32_t)(nrows * ng) * 4u);
    uint32_t xo[CA];
#pragma unroll
    for (int i = 0; i < CA; ++i) {
        const int lr = (wave * CA + i) * 8 + (lane >> 3);
        xo[i] = (uint32_t)lr * (uint32_t)ldx * 2u + (uint32_t)((lane & 7) ^ ((lr >> 1) & 7)) * 16u;
    }
    const int trow = tid / P, part = tid % P;
    const bool stager = NT == BN * P || tid < BN * P;
    const uint32_t co = (uint32_t)(trow * rb + part * NW * 4), mo = (uint32_t)(trow * ng + (lg == 5 ? part * CPT >> 5 : 0)) * 4u;
    struct Q {
        uint32_t w[NW], m;
    };
    auto load_x = [&](int kt, int slot) {
#pragma unroll
        for (int i = 0; i < CA; ++i)
            load_to_lds(rx, smem + slot * XB + (wave * CA + i) * 64, xo[i], (uint32_t)(kb + kt) * 128u);
    };
    auto load_w = [&](Q& q, int kt) {
        const uint32_t so = (uint32_t)(kb + kt) * 8u * BITS;
        if constexpr (NW == 4) {
            const auto v = __builtin_amdgcn_raw_buffer_load_b128(rc, co, so, 0);
            q.w[0] = v[0]; q.w[1] = v[1]; q.w[2] = v[2]; q.w[3] = v[3];
        } else if constexpr (NW == 2) {
            const auto v = __builtin_amdgcn_raw_buffer_load_b64(rc, co, so, 0);
            q.w[0] = v[0]; q.w[1] = v[1];
        } else {
            q.w[0] = __builtin_amdgcn_raw_buffer_load_b32(rc, co, so, 0);
        }
        q.m = __builtin_amdgcn_raw_buffer_load_b32(rm, mo, (uint32_t)(((kb + kt) * 64) >> lg) * 4u, 0);
    };
    Q q[QA];
#pragma unroll
    for (int s = 0; s < ST - 1; ++s) load_x(s < nk ? s : nk - 1, s);
    __asm__ volatile("" ::: "memory");                     // (the steps' windows below count on this order)
#pragma unroll
    for (int s = 0; s < QA; ++s) load_w(q[s], s < nk ? s : nk - 1);

    f32x16_t acc[WM][WN];
#pragma unroll
    for (int i = 0; i < WM; ++i)
#pragma unroll
        for (int j = 0; j < WN; ++j) acc[i][j] = f32x16_t{};
    const int r = lane & 31, hk = lane >> 5;
    for (int i = tid; i < BM; i += NT) ro[i] = a.x16 && m0 + i < a.M ? a.xf[m0 + i] : 1.0f;
    __syncthreads();
    // the factor 2^e that takes an adapter's sums to the scale of a bfloat16 row's products
    auto up = [&](int at) { return __uint_as_float(0x7F000000u - __float_as_uint(ro[at])); };
    if (!SPLIT && a.T > 0) {
        int id[WM];
        bool same = true;                                  // this wave's rows have one adapter, or none (or lie past M)
        const int mf = m0 + wm * 32 * WM;
        int ad0 = a.ids[mf < a.M ? mf : a.M - 1];
        ad0 = ad0 >= 0 && ad0 < a.T ? ad0 : -1;
#pragma unroll
        for (int i = 0; i < WM; ++i) {
            const int m = mf + i * 32 + r;
            const int v = a.ids[m < a.M ? m : a.M - 1];
            id[i] = v >= 0 && v < a.T && m < a.M ? v : -1;
            same = same && __all(id[i] == ad0 || m >= a.M);
        }
        const uint16_t* tp = a.tb + 8 * hk;
        const uint16_t* bp = a.B + 8 * hk;
        const long tlo = (long)a.M * a.R;
        auto load_b = [&](uint4 (&b)[WN], int ad, int k) {
#pragma unroll
            for (int j = 0; j < WN; ++j) {
                const int col = n0 + wn * 32 * WN + j * 32 + r;
                b[j] = k + 8 * hk < a.R ? ld16(bp + ((long)ad * a.n + (col < a.n ? col : a.n - 1)) * a.R + k) : make_uint4(0, 0, 0, 0);
            }
        };
        auto load_t = [&](uint4& t0, uint4& t1, int i, int k) {
            const int m = mf + i * 32 + r;
            const uint16_t* p = tp + (long)(m < a.M ? m : a.M - 1) * a.R + k;
            const bool live = k + 8 * hk < a.R;
            t0 = live ? ld16(p) : make_uint4(0, 0, 0, 0);
            t1 = live ? ld16(p + tlo) : make_uint4(0, 0, 0, 0);
        };
        if (same) {
            if (ad0 >= 0) {
#pragma unroll 1
                for (int k = 0; k < a.R; k += 32) {        // all loads of 32 ranks, then the products
                    uint4 t0[2][WM], t1[2][WM], b0[2][WN], b1;
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        load_b(b0[c], ad0, k + 16 * c);
#pragma unroll
                        for (int i = 0; i < WM; ++i) load_t(t0[c][i], t1[c][i], i, k + 16 * c);
                    }
#pragma unroll
                    for (int c = 0; c < 2; ++c)
#pragma unroll
                        for (int j = 0; j < WN; ++j) {
                            if (!a.bf)
                                split_f16(b0[c][j], b0[c][j], b1);
#pragma unroll
                            for (int i = 0; i < WM; ++i) {
                                acc[i][j] = mfma32_bf(t1[c][i], b0[c][j], mfma32_bf(t0[c][i], b0[c][j], acc[i][j]));
                                if (!a.bf)
                                    acc[i][j] = mfma32_bf(t0[c][i], b1, acc[i][j]);
                            }
                        }
                }
                if (a.bf)
#pragma unroll
                    for (int i = 0; i < WM; ++i)
#pragma unroll
                        for (int v = 0; v < 16; ++v) {
                            const float f = up(wm * 32 * WM + i * 32 + acc_row(v, lane));
#pragma unroll
                            for (int j = 0; j < WN; ++j) acc[i][j][v] *= f;
                        }
            }
        } else {
#pragma unroll
            for (int i = 0; i < WM; ++i) {
                const int row = wm * 32 * WM + i * 32, slot = m0 + row < a.M ? a.slots[(m0 + row) / 32] : -1;
                uint32_t todo = (uint32_t)__ballot(id[i] >= 0);
                if (slot >= 0) {                           // lora_mixed_kernel has formed these rows' terms
#pragma unroll
                    for (int j = 0; j < WN; ++j) {
                        const int col = n0 + wn * 32 * WN + j * 32 + r;
#pragma unroll
                        for (int v = 0; v < 16; ++v) {
                            const int at = acc_row(v, lane);
                            acc[i][j][v] = a.mixed[((long)slot * 32 + at) * a.n + (col < a.n ? col : a.n - 1)] * up(row + at);
                        }
                    }
                    continue;
                }
#pragma unroll 1
                while (todo) {
                    const int ad = __builtin_amdgcn_readlane(id[i], __builtin_ctz(todo));
                    const uint32_t own = (uint32_t)__ballot(id[i] == ad);
                    todo &= ~own;
                    f32x16_t s[WN];
#pragma unroll
                    for (int j = 0; j < WN; ++j) s[j] = f32x16_t{};
#pragma unroll 1
                    for (int k = 0; k < a.R; k += 32) {
                        uint4 t0[2], t1[2], b0[2][WN], b1;
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            load_b(b0[c], ad, k + 16 * c);
                            load_t(t0[c], t1[c], i, k + 16 * c);
                        }
#pragma unroll
                        for (int c = 0; c < 2; ++c)
#pragma unroll
                            for (int j = 0; j < WN; ++j) {
                                if (!a.bf)
                                    split_f16(b0[c][j], b0[c][j], b1);
                                s[j] = mfma32_bf(t1[c], b0[c][j], mfma32_bf(t0[c], b0[c][j], s[j]));
                                if (!a.bf)
                                    s[j] = mfma32_bf(t0[c], b1, s[j]);
                            }
                    }
#pragma unroll
                    for (int j = 0; j < WN; ++j)
#pragma unroll
                        for (int v = 0; v < 16; ++v) {
                            const int at = acc_row(v, lane);
                            acc[i][j][v] = own >> at & 1 ? s[j][v] * up(row + at) : acc[i][j][v];
                        }
                }
            }
        }
    }

    // Step kt multiplies slot kt % ST of x and kt & 1 of the weights, while x of the steps up to kt + ST - 1 and codes up
    // to kt + 1 + QA are under way and the weights of kt + 1 are unpacked.
    if (stager)
        dequant_store<BITS, CPT>(wsm, q[0].w, q[0].m, trow, part);
    load_w(q[0], nk > QA ? QA : nk - 1);
    int slot = 0;
    auto step = [&](int kt, Q& qn) {
        lds_barrier();
        const uint4* xs = smem + slot * XB;
        const uint4* ws = wsm + (kt & 1) * WB;
        {
            const int far = slot == 0 ? ST - 1 : slot - 1;
            load_x(kt + ST - 1 < nk ? kt + ST - 1 : nk - 1, far);
        }
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
        if (stager)
            dequant_store<BITS, CPT>(wsm + ((kt + 1) & 1) * WB, qn.w, qn.m, trow, part);
        __asm__ volatile("" ::: "memory");                 // the codes' registers are free now, not before
        load_w(qn, kt + 1 + QA < nk ? kt + 1 + QA : nk - 1);
        slot = slot + 1 == ST ? 0 : slot + 1;
    };
    // x of a step has arrived where only what was issued after it is under way: ST - 2 steps' x, and in the loop as many
    // steps' two loads of codes (in the last steps no codes: the compiler drops loads that no later step uses)
    int kt = 0;
    for (; kt + QA <= nk; kt += QA)
#pragma unroll
        for (int i = 0; i < QA; ++i) {
            vm_window<(ST - 2) * (CA + 2)>();
            step(kt + i, q[(i + 1) % QA]);
        }
#pragma unroll
    for (int i = 0; i < QA - 1; ++i)
        if (kt + i < nk) {
            vm_window<(ST - 2) * CA>();
            step(kt + i, q[(i + 1) % QA]);
        }
    __asm__ volatile("s_waitcnt vmcnt(0)" ::: "memory");   // no copy into LDS outlives the workgroup
#pragma unroll
    for (int j = 0; j < WN; ++j) {
        const int col = n0 + wn * 32 * WN + j * 32 + r;
#pragma unroll
        for (int i = 0; i < WM; ++i)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const int at = wm * 32 * WM + i * 32 + acc_row(v, lane), m = m0 + at;
                if (m < a.M && col < a.n) {
                    if (SPLIT)
                        a.parts[((long)share * a.M + m) * a.n + col] = acc[i][j][v] * ro[at];
                    else
                        a.y[(long)m * a.ldy + col] = act_bits(acc[i][j][v] * ro[at], a.bf);
                }
            }
    }
}

// 17 to 64 rows: a workgroup owns 32 WM rows and 128 outputs, a wave all of the rows
// and 32 outputs, whose weights go from memory to its registers and are unpacked
// there: in a step of 64 lane 32 h + r takes the 32 codes of row r from 32 h on, and
// multiplies them with chunk 4 h + s of x in product s.  Only x is staged; the codes
// are kMidAhead steps ahead.  (us, and by the tiles of lora_gemm_kernel: 17 x 6144 x
// 4096 11.2 and 14.0, 32 x 28672 x 4096 35 and 50; at 67 rows 17.2 and 16.4, at 333 x
// 9728 x 2560 40 and 38: rows are staged again for every 128 outputs.  Eight steps
// ahead, of x or the codes, took 3 to 10 % more.)
constexpr int kMidSlots = 4, kMidAhead = 4;
template <int BITS, int WM>
__global__ void __launch_bounds__(256) lora_mid_kernel(LoraArgs a, int lg) {
    constexpr int BM = 32 * WM, XB = BM * 8, ST = kMidSlots, QA = kMidAhead, NW = BITS;
    extern __shared__ uint4 smem[];                        // x [ST][BM][8], then the rows' 2^-e
    float* ro = reinterpret_cast<float*>(smem + ST * XB);
    const int tid = threadIdx.x, lane = tid & 63, r = lane & 31, hk = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int ntiles = (a.n + 127) / 128, m0 = (int)blockIdx.x / ntiles * BM, n0 = (int)blockIdx.x % ntiles * 128 + 32 * wave;
    // this workgroup's share of k, in steps of 64
    const int steps = a.k / 64, share = blockIdx.y, kb = share * steps / (int)gridDim.y, nk = (share + 1) * steps / (int)gridDim.y - kb;
    const long ldx = a.x16 ? a.k : a.ldx;
    const int mrows = min(BM, a.M - m0), nrows = max(0, min(32, a.n - n0)), rb = a.k * BITS / 8, ng = a.k >> lg;
    const Rsrc rx = rsrc((a.x16 ? a.x16 : a.x) + (long)m0 * ldx, (uint32_t)((mrows - 1) * (int)ldx + a.k) * 2u);
    const Rsrc rc = rsrc(reinterpret_cast<const char*>(a.codes) + (long)n0 * rb, (uint32_t)(nrows * rb));
    const Rsrc rm = rsrc(a.meta + (long)n0 * ng, (uint32_t)(nrows * ng) * 4u);
    uint32_t xo[WM];
#pragma unroll
    for (int i = 0; i < WM; ++i) {
        const int lr = (wave * WM + i) * 8 + (lane >> 3);
        xo[i] = (uint32_t)lr * (uint32_t)ldx * 2u + (uint32_t)((lane & 7) ^ ((lr >> 1) & 7)) * 16u;
    }
    const uint32_t co = (uint32_t)(r * rb + hk * 4 * BITS), mo = (uint32_t)(r * ng) * 4u;
    struct Q {
        uint32_t w[NW], m;
    };
    auto load_x = [&](int kt, int slot) {
#pragma unroll
        for (int i = 0; i < WM; ++i)
            load_to_lds(rx, smem + slot * XB + (wave * WM + i) * 64, xo[i], (uint32_t)(kb + kt) * 128u);
    };
    auto load_w = [&](Q& q, int kt) {
        const uint32_t so = (uint32_t)(kb + kt) * 8u * BITS;
        if constexpr (NW == 4) {
            const auto v = __builtin_amdgcn_raw_buffer_load_b128(rc, co, so, 0);
            q.w[0] = v[0]; q.w[1] = v[1]; q.w[2] = v[2]; q.w[3] = v[3];
        } else {
            const auto v = __builtin_amdgcn_raw_buffer_load_b64(rc, co, so, 0);
            q.w[0] = v[0]; q.w[1] = v[1];
        }
        q.m = __builtin_amdgcn_raw_buffer_load_b32(rm, mo + (uint32_t)(((kb + kt) * 64 + 32 * hk) >> lg) * 4u, 0, 0);
    };
    // eight codes of product s as binary16 scale * (q - zero), rounded once
    auto unpack = [&](const Q& q, uint32_t s2, uint32_t off, int s) {
        constexpr int PW = 16 / BITS;                      // pairs (c_i, c_{PW + i}) of a word
        constexpr uint32_t mask = BITS == 2 ? 0x00030003u : 0x000F000Fu;
        const uint32_t w = q.w[BITS == 2 ? s >> 1 : s];
        uint32_t v[PW];
#pragma unroll
        for (int p = 0; p < PW; ++p) v[p] = pk_mul(pk_add(((w >> (BITS * p)) & mask) | 0x64006400u, off), s2);
        if constexpr (BITS == 2)
            return (s & 1) ? make_uint4(pair_hi(v[0], v[1]), pair_hi(v[2], v[3]), pair_hi(v[4], v[5]), pair_hi(v[6], v[7]))
                           : make_uint4(pair_lo(v[0], v[1]), pair_lo(v[2], v[3]), pair_lo(v[4], v[5]), pair_lo(v[6], v[7]));
        else
            return make_uint4(pair_lo(v[0], v[1]), pair_lo(v[2], v[3]), pair_hi(v[0], v[1]), pair_hi(v[2], v[3]));
    };
    Q q[QA];
#pragma unroll
    for (int s = 0; s < ST - 1; ++s) load_x(s < nk ? s : nk - 1, s);
    __asm__ volatile("" ::: "memory");
#pragma unroll
    for (int s = 0; s < QA; ++s) load_w(q[s], s < nk ? s : nk - 1);
    f32x16_t acc[WM];
#pragma unroll
    for (int i = 0; i < WM; ++i) acc[i] = f32x16_t{};
    for (int i = tid; i < BM; i += 256) ro[i] = a.x16 && m0 + i < a.M ? a.xf[m0 + i] : 1.0f;
    int slot = 0;
    // Step kt multiplies slot kt % ST of x, while x of step kt + ST - 1 and the codes up to kt + QA are under way.
    auto step = [&](int kt, Q& c) {
        lds_barrier();
        const uint4* xs = smem + slot * XB;
        load_x(kt + ST - 1 < nk ? kt + ST - 1 : nk - 1, slot == 0 ? ST - 1 : slot - 1);
        const uint32_t s2 = __builtin_amdgcn_perm(0u, c.m, 0x01000100u);
        const uint32_t off = pk_add(0xE400E400u, __builtin_amdgcn_perm(0u, c.m, 0x03020302u) ^ 0x80008000u);   // -1024 - z
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const uint4 wv = unpack(c, s2, off, s);
#pragma unroll
            for (int i = 0; i < WM; ++i) acc[i] = mfma32(ld16(&xs[swz(i * 32 + r, 4 * hk + s)]), wv, acc[i]);
        }
        __asm__ volatile("" ::: "memory");                 // the codes' registers are free now, not before
        load_w(c, kt + QA < nk ? kt + QA : nk - 1);
        slot = slot + 1 == ST ? 0 : slot + 1;
    };
    int kt = 0;                                            // (windows as in lora_gemm_kernel)
    for (; kt + QA <= nk; kt += QA)
#pragma unroll
        for (int i = 0; i < QA; ++i) {
            vm_window<(ST - 2) * (WM + 2)>();
            step(kt + i, q[i]);
        }
#pragma unroll
    for (int i = 0; i < QA - 1; ++i)
        if (kt + i < nk) {
            vm_window<(ST - 2) * WM>();
            step(kt + i, q[i]);
        }
    __asm__ volatile("s_waitcnt vmcnt(0)" ::: "memory");   // no copy into LDS outlives the workgroup
    const int col = n0 + r;
#pragma unroll
    for (int i = 0; i < WM; ++i)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
            const int at = i * 32 + acc_row(v, lane), m = m0 + at;
            if (m < a.M && col < a.n) {
                if (a.parts)
                    a.parts[((long)share * a.M + m) * a.n + col] = acc[i][v] * ro[at];
                else
                    a.y[(long)m * a.ldy + col] = act_bits(acc[i][v] * ro[at], a.bf);
            }
        }
}

}  // namespace

hipError_t launch_lora_gemm(const LoraArgs& a, hipStream_t st) {
    const int lg = a.g == 32 ? 5 : a.g == 64 ? 6 : 7;
    const unsigned shares = (unsigned)a.shares;
    if (a.M <= kLoraMidRows) {
        const int wm = (a.M + 31) / 32;
        const unsigned grid = (unsigned)(a.n + 127) / 128;
        const size_t lds = (size_t)kMidSlots * wm * 4096 + wm * 128;
        auto k = a.bits == 2 ? (wm == 1 ? lora_mid_kernel<2, 1> : lora_mid_kernel<2, 2>) : (wm == 1 ? lora_mid_kernel<4, 1> : lora_mid_kernel<4, 2>);
        k<<<dim3(grid, shares), 256, lds, st>>>(a, lg);
        return hipGetLastError();
    }
    auto run = [&](auto k, int BM, int BN, int nt, int stages) {
        const size_t lds = (size_t)(stages * BM + 2 * BN) * 128 + (size_t)BM * 4;
        const hipError_t e = set_lds(k, lds);
        if (e != hipSuccess)
            return e;
        const unsigned grid = (unsigned)(((a.M + BM - 1) / BM) * ((a.n + BN - 1) / BN));
        k<<<dim3(grid, shares), (unsigned)nt, lds, st>>>(a, lg);
        return hipGetLastError();
    };
    if (shares > 1)
        return a.bits == 2 ? run(lora_gemm_kernel<2, 128, 128, 2, 1, 4, true>, 128, 128, 512, 4)
                           : run(lora_gemm_kernel<4, 128, 128, 2, 1, 4, true>, 128, 128, 512, 4);
    if (lora_large_tiles(a.M, a.n, a.cus))
        return a.bits == 2 ? run(lora_gemm_kernel<2, 256, 192, 2, 3, 3, false>, 256, 192, 512, 3)
                           : run(lora_gemm_kernel<4, 256, 192, 2, 3, 3, false>, 256, 192, 512, 3);
    return a.bits == 2 ? run(lora_gemm_kernel<2, 128, 128, 2, 1, 4, false>, 128, 128, 512, 4)
                       : run(lora_gemm_kernel<4, 128, 128, 2, 1, 4, false>, 128, 128, 512, 4);
}

}  // namespace qmlp
