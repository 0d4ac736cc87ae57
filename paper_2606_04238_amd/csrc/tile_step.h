// One step of a 16-row tile of 2- or 4-bit codes on the matrix cores
// (decode_tile.hip, and in half steps oneshot.h): the layout of a step, its
// activations as matrix operands with their group sums, the weight loads and
// the products.  The arithmetic is described at the top of decode_tile.hip.
#pragma once

#include "decode_common.h"
#include "mfma_tile.h"

namespace qmlp {
namespace {

// The same value, opaque to the compiler: addresses formed from it where they
// are used now and then (once per block or tile) are not kept across the main
// loop, which has no register to spare.
__device__ __forceinline__ int fresh(int v) {
    __asm__ volatile("" : "+v"(v));
    return v;
}

__device__ __forceinline__ f32x4_t mfma4(float a, float b, f32x4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}

// Layout of one step (32 code words of each of 16 rows) of B-bit codes in
// groups of G.
template <int B, int G>
struct Lay {
    static constexpr int CPS = 1024 / B;                   // codes per row and step
    static constexpr int WPG = G * B / 32;                 // words per group
    static constexpr bool HALF = WPG == 2;                 // 2-bit, group 32
    static constexpr int QW = HALF ? 1 : WPG / 4;          // words per quarter and group
    static constexpr int GSU = 32 / WPG;                   // groups per step
    static constexpr int MPG = HALF ? 1 : B == 2 ? 2 * QW : QW;   // matrix instructions per group
    static constexpr int NA = MPG * GSU;                   // A operands per step
};

template <int B, int G>
using AOps = uint4[Lay<B, G>::NA];

// The (scale | zero) words of a step's groups of lane row j: quarter q loads
// its quarter of them, groups q GSU/4 .. (both where there are only two), and
// meta_spread hands them to the other quarters.
template <int GSU>
struct TileMeta {
    static constexpr int NW = GSU == 2 ? 2 : GSU / 4;
    uint32_t w[NW];
};
template <int GSU>
__device__ __forceinline__ int meta_first(int q) { return GSU == 2 ? 0 : q * (GSU / 4); }
template <int GSU>
__device__ __forceinline__ void meta_load(TileMeta<GSU>& m, Rsrc r, uint32_t voff) {
    if constexpr (GSU == 16) {
        const uint4 v = bload16<0>(r, voff, 0);
        m.w[0] = v.x;
        m.w[1] = v.y;
        m.w[2] = v.z;
        m.w[3] = v.w;
    } else if constexpr (GSU == 4) {
        m.w[0] = __builtin_amdgcn_raw_buffer_load_b32(r, voff, 0, 0);
    } else {
        const uint2 v = bload8(r, voff, 0);
        m.w[0] = v.x;
        m.w[1] = v.y;
    }
}
// Word e of every quarter, in all quarters: sc[k] is the scale of group
// k GSU/4 + e (with equal operands a swap leaves one side's value on both).
__device__ __forceinline__ void meta_spread(uint32_t w, float (&sc)[4]) {
    uint32_t x = w, y = w;
    swap16(x, y);                                          // x: quarters 0 0 2 2, y: 1 1 3 3
    uint32_t x2 = x, y2 = y;
    swap32(x, x2);                                         // x: 0 everywhere, x2: 2
    swap32(y, y2);
    sc[0] = h2f(x & 0xFFFFu);
    sc[1] = h2f(y & 0xFFFFu);
    sc[2] = h2f(x2 & 0xFFFFu);
    sc[3] = h2f(y2 & 0xFFFFu);
}

// ---- activations
// Raw activations of (this lane's) step gs: token j (zeros past M) and the
// words of its quarter (zeros past K; `live` false: all zeros).  rx covers
// the block's M rows of K.
template <int B, int G>
__device__ __forceinline__ void act_load(AOps<B, G>& a, Rsrc rx, int gs, int j, int M, int K, bool live, int lane) {
    typedef Lay<B, G> Y;
    constexpr int CW = 32 / B;                             // codes per word
    const int q = lane >> 4;
    const bool tok = live && j < M;
    const int W0 = gs * 32 + (Y::HALF ? q >> 1 : quarter_word<Y::QW>(q));
    const uint32_t o = tok ? (uint32_t)(j * K + CW * W0 + (Y::HALF ? 8 * (q & 1) : 0)) * 2u : kPastEnd;
    constexpr int NWD = Y::HALF ? Y::GSU : Y::GSU * Y::QW;
#pragma unroll
    for (int i = 0; i < NWD; ++i) {
        const uint32_t oi = o + 2u * CW * (Y::HALF ? 2 * i : (i / Y::QW) * Y::WPG + i % Y::QW);
        if constexpr (B == 2 && !Y::HALF) {
            a[2 * i] = bload16<0>(rx, oi, 0);
            a[2 * i + 1] = bload16<0>(rx, oi + 16, 0);
        } else {
            a[i] = bload16<0>(rx, oi, 0);
        }
    }
}
// Words past the row's end (the next token's) become zeros.
template <int B, int G>
__device__ __forceinline__ void act_mask(AOps<B, G>& a, int gs, int K, int lane) {
    typedef Lay<B, G> Y;
    constexpr int CW = 32 / B, PER = Y::HALF || B == 4 ? 1 : 2;
    if (__all((gs + 1) * Y::CPS <= K))
        return;
    const int q = lane >> 4, W0 = gs * 32 + (Y::HALF ? q >> 1 : quarter_word<Y::QW>(q));
#pragma unroll
    for (int i = 0; i < Y::NA; ++i) {
        const int k = i / PER;
        if (CW * (W0 + (Y::HALF ? 2 * k : (k / Y::QW) * Y::WPG + k % Y::QW)) >= K)
            a[i] = make_uint4(0u, 0u, 0u, 0u);
    }
}

// (a.lo, b.lo) and (a.hi, b.hi) of two words of halves.
__device__ __forceinline__ uint32_t pair_lo(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t pair_hi(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }
__device__ __forceinline__ uint32_t pk_mul(uint32_t a, uint32_t b) {
    return __builtin_bit_cast(uint32_t, __builtin_bit_cast(half2_t, a) * __builtin_bit_cast(half2_t, b));
}
__device__ __forceinline__ constexpr uint32_t pow2_pair(int e) {      // binary16 2^e in both halves
    return (uint32_t)((15 + e) << 10) * 0x00010001u;
}
// Fraction position j of pair p (0..3) of the matrix operand of half h, and
// the smallest of them: x' = x 2^(kPosMin - j).
constexpr int kPosMin = 4;
constexpr float kTileUnscale = 1.0f / 16.0f;               // 2^-kPosMin, of a finished sum
template <int B, bool HALF>
__device__ __forceinline__ constexpr int pair_pos(int h, int p) {
    if (B == 4) return p < 2 ? 4 : 6;
    if (HALF || h == 0) return (p & 1) ? 6 : 4;
    return p == 1 ? 4 : p == 2 ? 6 : 8;
}
template <int B, bool HALF>
__device__ __forceinline__ uint4 scale_pairs(uint4 v, int h) {
    return make_uint4(pk_mul(v.x, pow2_pair(kPosMin - pair_pos<B, HALF>(h, 0))),
                      pk_mul(v.y, pow2_pair(kPosMin - pair_pos<B, HALF>(h, 1))),
                      pk_mul(v.z, pow2_pair(kPosMin - pair_pos<B, HALF>(h, 2))),
                      pk_mul(v.w, pow2_pair(kPosMin - pair_pos<B, HALF>(h, 3))));
}
template <int B, bool HALF>
__device__ __forceinline__ uint4 unscale_pairs(int h) {
    return make_uint4(pow2_pair(pair_pos<B, HALF>(h, 0)), pow2_pair(pair_pos<B, HALF>(h, 1)),
                      pow2_pair(pair_pos<B, HALF>(h, 2)), pow2_pair(pair_pos<B, HALF>(h, 3)));
}
// Raw words to matrix operands x' in the pair order of the codes.
template <int B, int G>
__device__ __forceinline__ void act_convert(AOps<B, G>& a) {
    typedef Lay<B, G> Y;
    if constexpr (B == 2 && !Y::HALF) {
#pragma unroll
        for (int i = 0; i < Y::NA / 2; ++i) {
            const uint4 l = a[2 * i], h = a[2 * i + 1];
            a[2 * i] = scale_pairs<B, false>(make_uint4(pair_lo(l.x, h.x), pair_hi(l.x, h.x), pair_lo(l.y, h.y),
                                                        pair_hi(l.y, h.y)), 0);
            a[2 * i + 1] = scale_pairs<B, false>(make_uint4(pair_lo(l.z, h.z), pair_hi(l.z, h.z), pair_lo(l.w, h.w),
                                                            pair_hi(l.w, h.w)), 1);
        }
    } else {
#pragma unroll
        for (int i = 0; i < Y::NA; ++i) {                  // eight codes, pairs p and 4 + p
            const uint4 r = a[i];
            a[i] = scale_pairs<B, Y::HALF>(make_uint4(pair_lo(r.x, r.z), pair_hi(r.x, r.z), pair_lo(r.y, r.w),
                                                    pair_hi(r.y, r.w)), 0);
        }
    }
}
// The A operands of a step's offset and zero-point terms.  With C = sum x'
// and X = sum 2^j x' (16 sum x) of a token and group, the group's codes add
// s (p - 1024 C - z X), p their plain product with x'.  The second and third
// terms of all groups are one fp32 contraction over groups, rows (s, s z)
// against tokens (-1024 C, -X): v_mfma_f32_16x16x4_f32, where instruction m
// takes the m-th group of every quarter of the lanes, whose words that quarter
// loaded (two groups per step: quarters 0, 1 the C and 2, 3 the X of groups
// 0, 1).  C and X come from the matrix cores with the activations as the B
// operand, so every lane gets its own token's.
template <int B, int G>
struct Corr {
    static constexpr int NC = Lay<B, G>::GSU == 2 ? 1 : Lay<B, G>::GSU / 4;
    float c[NC], x[NC];
};
template <int B, int G>
__device__ __forceinline__ void group_sums(const AOps<B, G>& a, Corr<B, G>& k, int lane) {
    typedef Lay<B, G> Y;
    const uint4 one = make_uint4(0x3C003C00u, 0x3C003C00u, 0x3C003C00u, 0x3C003C00u);
    const int q = lane >> 4;
#pragma unroll
    for (int i = 0; i < Y::GSU; ++i) {
        f32x4_t c = {0.f, 0.f, 0.f, 0.f}, x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int m = 0; m < Y::MPG; ++m) {
            c = mfma16(one, a[i * Y::MPG + m], c);
            x = mfma16(unscale_pairs<B, Y::HALF>(B == 2 && !Y::HALF ? m & 1 : 0), a[i * Y::MPG + m], x);
        }
        if constexpr (Y::GSU == 2) {
            if (i == 0 || (q & 1)) k.c[0] = q < 2 ? -1024.0f * c[0] : -x[0];
        } else {
            constexpr int NC = Corr<B, G>::NC;
            if (i < NC || q == i / NC) {
                k.c[i % NC] = -1024.0f * c[0];
                k.x[i % NC] = -x[0];
            }
            // settled one group at a time: every group's sums at once would not fit the registers
            __asm__ volatile("" : "+v"(k.c[i % NC]), "+v"(k.x[i % NC]));
        }
    }
}

// ---- weights
// A step's code loads of one matrix and its groups' (scale | zero) words.
template <int B, int G>
struct TileW {
    uint4 c[2];
    TileMeta<Lay<B, G>::GSU> m;
};

// Loads of one step of the 16 rows that start at byte offsets co / mo of the
// code and metadata arrays: ol / ml are the lane's offsets for the step, rb8
// the bytes of eight rows.  co and mo of kPastEnd (no such tile), or ol (no
// such step or unit), load zeros; both together wrap to the first lines of
// the array, in range, for a tile whose sums nobody adds.
template <int B, int G>
__device__ __forceinline__ void w_load(TileW<B, G>& w, Rsrc rc, Rsrc rm, uint32_t ol, uint32_t ml, uint32_t rb8,
                                       uint32_t co, uint32_t mo) {
    w.c[0] = bload16<kAuxNt>(rc, ol + co, 0);
    w.c[1] = bload16<kAuxNt>(rc, ol + co + rb8, 0);
    meta_load(w.m, rm, ml + mo);
}

// acc += the step's product with the A operands a.  `tail`: the number of
// groups of this step inside the row (GSU on all but the last step of a
// ragged row).
template <int B, int G>
__device__ __forceinline__ void tile_step(TileW<B, G>& w, const AOps<B, G>& a, const Corr<B, G>& k, f32x4_t& acc,
                                          int tail, int lane) {
    typedef Lay<B, G> Y;
    const uint32_t mv = magic_vgpr();
    const int q = lane >> 4;
    pin4(w.c[0]);
    pin4(w.c[1]);
    arrange<Y::QW != 4, Y::QW == 1>(w.c);
    typedef TileMeta<Y::GSU> Meta;
    if (tail < Y::GSU) {
#pragma unroll
        for (int e = 0; e < Meta::NW; ++e)
            if (meta_first<Y::GSU>(q) + e >= tail)
                w.m.w[e] = 0;
    }
    // the offset and zero-point terms
    if constexpr (Y::GSU == 2) {
        const uint32_t mw = (q & 1) ? w.m.w[1] : w.m.w[0];
        const float sc = h2f(mw & 0xFFFFu);
        acc = mfma4(k.c[0], q < 2 ? sc : sc * h2f(mw >> 16), acc);
    } else {
#pragma unroll
        for (int m = 0; m < Y::GSU / 4; ++m) {
            const float sc = h2f(w.m.w[m] & 0xFFFFu);
            acc = mfma4(k.c[m], sc, acc);
            acc = mfma4(k.x[m], sc * h2f(w.m.w[m] >> 16), acc);
        }
    }
    const f32x4_t zero = {0.f, 0.f, 0.f, 0.f};
    if constexpr (Y::HALF) {
        // codes 0..7 or 8..15 of a word as pairs (p, 4 + p) at bits 2 p of both halves
        const uint32_t sel = (q & 1) ? 0x0C030C02u : 0x0C010C00u;
#pragma unroll
        for (int eh = 0; eh < 2; ++eh) {
            float sc[2][4];
            meta_spread(w.m.w[2 * eh], sc[0]);
            meta_spread(w.m.w[2 * eh + 1], sc[1]);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                // this lane's codes of unit 2 k + eh: groups 4 k + 2 eh and the next
                uint32_t x = word_of(w.c[k >> 1], 2 * (k & 1) + eh), y = x;
                swap16(x, y);
                const uint32_t wd[2] = {__builtin_amdgcn_perm(0u, x, sel), __builtin_amdgcn_perm(0u, y, sel)};
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    const uint32_t v = wd[s], v4 = v << 4;
                    const f32x4_t p = mfma16(a[4 * k + 2 * eh + s],
                                             make_uint4(magic(v4, 0x00300030u, mv), magic(v4, 0x00C000C0u, mv),
                                                        magic(v, 0x00300030u, mv), magic(v, 0x00C000C0u, mv)), zero);
                    acc += sc[s][k] * p;
                }
            }
        }
    } else {
        constexpr int NE = Y::GSU == 2 ? 1 : Y::GSU / 4;
#pragma unroll
        for (int e = 0; e < NE; ++e) {
            float sc[4];
            if constexpr (Y::GSU == 2) {
                sc[0] = h2f(w.m.w[0] & 0xFFFFu);
                sc[1] = h2f(w.m.w[1] & 0xFFFFu);
            } else {
                meta_spread(w.m.w[e], sc);
            }
#pragma unroll
            for (int k = 0; k < Y::GSU / NE; ++k) {
                const int i = k * NE + e;                  // group of the step
                f32x4_t p = zero;
#pragma unroll
                for (int ww = 0; ww < Y::QW; ++ww) {
                    const uint32_t v = Y::QW == 1   ? word_of(w.c[i >> 2], i & 3)
                                       : Y::QW == 2 ? word_of(w.c[i >> 1], 2 * (i & 1) + ww)
                                                    : word_of(w.c[i & 1], ww);
                    if constexpr (B == 2) {
                        uint32_t x[8];
                        extract_w2(v, x, mv);
                        p = mfma16(a[i * Y::MPG + 2 * ww], make_uint4(x[0], x[1], x[2], x[3]), p);
                        p = mfma16(a[i * Y::MPG + 2 * ww + 1], make_uint4(x[4], x[5], x[6], x[7]), p);
                    } else {
                        uint32_t x[4];
                        extract_w4(v, x, mv);
                        p = mfma16(a[i * Y::MPG + ww], make_uint4(x[0], x[1], x[2], x[3]), p);
                    }
                }
                acc += sc[k] * p;
            }
        }
    }
}

}  // namespace
}  // namespace qmlp
