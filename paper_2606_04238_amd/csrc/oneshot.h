// Products of a few token rows with 16-row tiles of packed codes where every
// wave has one piece of work (gfx950): the few-token form of the linear with
// adapters (lora_linear.hip) and the experts of a whole MoE layer
// (moe_layer.hip).
//
// Split.  A workgroup owns RT tiles of 16 weight rows (of one matrix, or of gate
// and up); its waves split K, wave w takes the steps w, w + KW, .. of 64 bytes per
// row.  A wave has the next step's weights and the next operands under way while
// it multiplies, and leaves its sums in LDS, where they meet behind one barrier.
// There is no loop over tiles: the launch has a workgroup for each, and the
// hardware starts the next one where one ends.  Reading 92 MB in 8 KB pieces,
// one per wave, took 15.3 us on this card against 17.3 to 21 with persistent
// waves that prefetch, and 16 MB 4.1 against 5.2 to 9.6 (loads only, launch
// included): a persistent wave ramps its stream up once and waits for its
// slowest piece at the end.
//
// Activations.  What bounded these kernels were the vector caches' tag lookups: with
// a row after the other in memory an operand's 64 lanes read 64 places (a
// bfloat16 7 x 5120 x 17408 product: 459 lookups a step, 62 400 a compute unit in
// 70 000 cycles).  So the launch before lays the rows side by side: 16 bytes of
// every row, then the next 16; an operand is four runs of up to 256 bytes.  (us, rows
// one after the other and side by side: that product 30.0 and 25.6, 16 x 6144 x
// 4096 13.9 and 10.9, 16 x 5120 x 17408 40.6 and 30.4, one row 8.7 and 8.7; down of 32
// experts, 8 rows each, 47.8 and 44.4.)  Copying codes and (scale | zero) words to
// LDS in whole lines first did not pay: 42 against 41 for gate and up.
//
// Arithmetic.  That of decode_tile.hip but for the powers of two: a code at fraction
// bits j.. of a binary16 2^(14 - j) reads 2^(14 - j) + 16 q, whatever j is, so the
// activations are operands as they are.  (Beside 1024 + q 2^j they would be multiplied
// by 2^(4 - j), j up to 8, and rounded to binary16 again: 16 rows of 1e-4, k = 1024,
// were 3.4e-3 off 64 bits at 2 bits and 1.3e-3 at 4, where the output's own rounding,
// all that is left now, is 2.1e-4.)  The offsets' sum is C = sum of 2^(14 - j) x, that
// of the zero points X = 16 sum of x.
#pragma once

#include "oneshot_plan.h"
#include "tile_step.h"

namespace qmlp {
namespace {

// A step is 64 bytes of each of a tile's 16 rows.  Lane l = 16 q + j loads unit
// perm(q) (16 bytes) of row j, and E4 and E5 (mfma_tile.h) bring quarter q its words
// of every group, as in the first half of a tile kernel's step.  Activations come in
// the operands' order (operand16 below): an operand is one 16-byte load, and lanes
// without a row read past the end, zeros.  Their group sums come with them
// (SUMS = false) or are formed here.
template <int B, int G>
struct OneLay {
    typedef Lay<B, G> Y;
    static constexpr int CPS = 512 / B;                    // codes per row and step
    static constexpr int GS = Y::GSU / 2;                  // groups per step: 1, 2, 4 or 8
    static constexpr int NA = Y::NA / 2;                   // operands per step
    static constexpr int NW = GS == 2 || GS == 8 ? 2 : 1;  // (scale | zero) words of a lane
    static constexpr int NC = GS == 8 ? 2 : 1;             // pairs of group sums of a lane
};
template <int B, int G, int NM, int RT>
struct OneStep {
    float kc[OneLay<B, G>::NC], kx[OneLay<B, G>::NC];
    uint4 w[NM * RT];
    uint32_t m[NM * RT][OneLay<B, G>::NW];
};
// What a wave multiplies: rows row0 .. of NM matrices [N][K] with the rows of the
// activations (a lane's row: place() of it).  K % 64 == 0; weight rows past N give
// zeros.
template <int NM>
struct OneWork {
    Rsrc rc[NM], rm[NM];
    Rsrc rx, rs;                                           // operands, group sums
    uint32_t xv, sv;                                       // this lane's place in them at step 0, or kPastEnd
    uint32_t rows;                                         // rows side by side there
    int K, N, row0;
    uint32_t magic[3];                                     // pairs of 2^(14 - j), j = 4, 6 and 8, made at the kernel's start
};
// (Those constants are made at the start, and kept: an instruction written by hand
// gets no distance from matrix instructions, and one among them that shared a
// register with an unused part of a running one's result was overwritten by it.)
template <int NM>
__device__ __forceinline__ void one_magic(OneWork<NM>& o) {
    o.magic[0] = magic_vgpr();
    o.magic[1] = o.magic[0] - 0x08000800u;
    o.magic[2] = o.magic[0] - 0x10001000u;
}
// The code pairs of extract_w4 and extract_w2 (qmlp_device.h), each above its own power of two.
__device__ __forceinline__ void one_extract_w4(uint32_t w, uint32_t (&e)[4], const uint32_t (&m)[3]) {
    e[0] = magic(w << 4, 0x00F000F0u, m[0]);
    e[1] = magic(w, 0x00F000F0u, m[0]);
    e[2] = magic(w >> 2, 0x03C003C0u, m[1]);
    e[3] = magic(w >> 6, 0x03C003C0u, m[1]);
}
__device__ __forceinline__ void one_extract_w2(uint32_t w, uint32_t (&e)[8], const uint32_t (&m)[3]) {
    const uint32_t l = w << 4, r = w >> 6;
    e[0] = magic(l, 0x00300030u, m[0]);
    e[1] = magic(l, 0x00C000C0u, m[1]);
    e[2] = magic(w, 0x00300030u, m[0]);
    e[3] = magic(w, 0x00C000C0u, m[1]);
    e[4] = magic(w, 0x03000300u, m[2]);
    e[5] = magic(r, 0x00300030u, m[0]);
    e[6] = magic(r, 0x00C000C0u, m[1]);
    e[7] = magic(r, 0x03000300u, m[2]);
}
// 2^(4 - j) of the pairs of an operand: 2^-10 of the codes' offsets.
template <int B, bool HALF>
__device__ __forceinline__ uint4 offset_pairs(int h) {
    return make_uint4(pow2_pair(kPosMin - pair_pos<B, HALF>(h, 0)), pow2_pair(kPosMin - pair_pos<B, HALF>(h, 1)),
                      pow2_pair(kPosMin - pair_pos<B, HALF>(h, 2)), pow2_pair(kPosMin - pair_pos<B, HALF>(h, 3)));
}

// The operands of a step are loaded while the step before is multiplied, each into
// the register of the one it follows: loads come back in order, and one behind the
// next step's weights would wait for them (2 bits, four of eight operands so: gate
// and up of one token 10.3 us instead of 9.7; groups of 32 keep four, whose scales
// take the registers).
template <int B, int G>
constexpr int one_ahead() {
    return Lay<B, G>::HALF ? 4 : OneLay<B, G>::NA;
}
// A lane's place in the operands and the group sums of a row that begins there at
// bytes x and sums.
template <int B, int G, int NM>
__device__ __forceinline__ void place(OneWork<NM>& o, uint32_t x, uint32_t sums, bool live, int q) {
    typedef Lay<B, G> Y;
    typedef OneLay<B, G> L;
    const uint32_t chunk = Y::HALF ? 4 / B * (q >> 1) + (q & 1) : 4 / B * quarter_word<Y::QW>(q);
    const uint32_t group = L::GS == 1 ? 0 : L::GS == 2 ? q & 1 : q * L::NC, part = L::GS == 1 ? q & 1 : L::GS == 2 ? q >> 1 : 0;
    o.xv = live ? x + chunk * o.rows * 16u : kPastEnd;
    o.sv = live ? sums + group * o.rows * 8u + 4u * part : kPastEnd;
}
template <int B, int G, int NM>
__device__ __forceinline__ void one_operand(uint4& a, const OneWork<NM>& o, int gs, int i) {
    typedef Lay<B, G> Y;
    constexpr int CW = 32 / B, PER = Y::HALF || B == 4 ? 1 : 2;           // codes and operands per word
    const int w = i / PER, at = Y::HALF ? 2 * w : (w / Y::QW) * Y::WPG + w % Y::QW;
    a = bload16<0>(o.rx, o.xv, (uint32_t)(CW / 8 * (gs * 16 + at) + i % PER) * o.rows * 16u);
}

template <int B, int G, int NM, int RT, bool SUMS>
__device__ __forceinline__ void one_load(OneStep<B, G, NM, RT>& s, const OneWork<NM>& o, int gs, int lane) {
    typedef Lay<B, G> Y;
    typedef OneLay<B, G> L;
    const int rb = o.K * B / 8, ng = o.K / G, q = lane >> 4, j = lane & 15;
    if constexpr (!SUMS) {
        const uint32_t at = (uint32_t)(gs * L::GS) * o.rows * 8u;
        if constexpr (L::GS <= 2) {
            s.kc[0] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(o.rs, o.sv, at, 0));
        } else {
#pragma unroll
            for (int i = 0; i < L::NC; ++i) {
                const uint2 v = bload8(o.rs, o.sv, at + 8u * o.rows * i);
                s.kc[i] = __uint_as_float(v.x);
                s.kx[i] = __uint_as_float(v.y);
            }
        }
    }
    const int b4 = q & 1, b5 = q >> 1, u = gs * 4 + (Y::QW == 4 ? 2 * b5 + b4 : 2 * b4 + b5);
    const int g0 = gs * L::GS + (L::GS <= 2 ? 0 : q * (L::GS / 4));
    const bool in = 16 * u < rb, gin = g0 < ng;
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int m = 0; m < NM; ++m) {
            const int row = o.row0 + 16 * t + j;
            const bool real = row < o.N;
            s.w[t * NM + m] = bload16<0>(o.rc[m], real && in ? (uint32_t)row * (uint32_t)rb + 16u * (uint32_t)u : kPastEnd, 0);
            const uint32_t mo = real && gin ? ((uint32_t)row * (uint32_t)ng + (uint32_t)g0) * 4u : kPastEnd;
            uint32_t(&mw)[L::NW] = s.m[t * NM + m];
            if constexpr (L::NW == 2) {
                const uint2 v = bload8(o.rm[m], mo, 0);
                mw[0] = v.x;
                mw[1] = v.y;
            } else {
                mw[0] = __builtin_amdgcn_raw_buffer_load_b32(o.rm[m], mo, 0, 0);
            }
        }
}

// acc[m][t] += the step's products: the arithmetic of tile_step.h, with the tiles
// side by side and a group's products added one group later, so that a matrix
// instruction is not waited for at once.
template <int B, int G, int NM, int RT, bool SUMS, typename NEXT>
__device__ __forceinline__ void one_multiply(f32x4_t (&acc)[NM][RT], OneStep<B, G, NM, RT>& s, const OneWork<NM>& o,
                                             int gs, int lane, NEXT next) {
    typedef Lay<B, G> Y;
    typedef OneLay<B, G> L;
    constexpr int N = NM * RT;
    const int q = lane >> 4, left = o.K / G - gs * L::GS;  // groups of the row from this step on
    const f32x4_t zero = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < N; ++c) {
        if constexpr (Y::QW != 4) {                        // E4, E5
            swap16(s.w[c].x, s.w[c].z);
            swap16(s.w[c].y, s.w[c].w);
        }
        if constexpr (Y::QW == 1) {
            swap32(s.w[c].x, s.w[c].y);
            swap32(s.w[c].z, s.w[c].w);
        }
        if (left < L::GS) {
#pragma unroll
            for (int e = 0; e < L::NW; ++e)
                if ((L::GS <= 2 ? 0 : q * (L::GS / 4)) + e >= left)
                    s.m[c][e] = 0;
        }
    }
    // a group's sums from its operands, kept where its offset and zero-point terms want them
    constexpr uint32_t k16 = pow2_pair(kPosMin);
    const uint4 sixteen = make_uint4(k16, k16, k16, k16);
    f32x4_t gc = zero, gx = zero;
    auto sum_up = [&](int i, int m, const uint4& a) {
        if constexpr (SUMS) {
            gc = mfma16(offset_pairs<B, Y::HALF>(B == 2 && !Y::HALF ? m & 1 : 0), a, m == 0 ? zero : gc);
            gx = mfma16(sixteen, a, m == 0 ? zero : gx);
            if (m + 1 < Y::MPG)
                return;
            if constexpr (L::GS == 1) {
                s.kc[0] = (q & 1) ? -gx[0] : -1024.0f * gc[0];
            } else if constexpr (L::GS == 2) {
                if (i == 0 || (q & 1)) s.kc[0] = q < 2 ? -1024.0f * gc[0] : -gx[0];
            } else if (i < L::NC || q == i / L::NC) {
                s.kc[i % L::NC] = -1024.0f * gc[0];
                s.kx[i % L::NC] = -gx[0];
            }
        }
    };
    f32x4_t before[N];
    float by[N];
    bool some = false;
    auto add = [&] {
        if (some)
#pragma unroll
            for (int c = 0; c < N; ++c) acc[c % NM][c / NM] += by[c] * before[c];
        some = true;
    };
    float sc[N][L::NW][4];
    if constexpr (L::GS == 1 || L::GS == 2) {
#pragma unroll
        for (int c = 0; c < N; ++c)
#pragma unroll
            for (int e = 0; e < L::NW; ++e) sc[c][0][e] = h2f(s.m[c][e] & 0xFFFFu);
    } else {
#pragma unroll
        for (int c = 0; c < N; ++c)
#pragma unroll
            for (int e = 0; e < L::NW; ++e) meta_spread(s.m[c][e], sc[c][e]);
    }
    if constexpr (Y::HALF) {                               // eight groups: unit u holds groups 2 u and 2 u + 1
        const uint32_t sel = (q & 1) ? 0x0C030C02u : 0x0C010C00u;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            uint32_t wd[N][2];
#pragma unroll
            for (int c = 0; c < N; ++c) {
                uint32_t x = word_of(s.w[c], u), y = x;
                swap16(x, y);
                wd[c][0] = __builtin_amdgcn_perm(0u, x, sel);
                wd[c][1] = __builtin_amdgcn_perm(0u, y, sel);
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                f32x4_t p[N];
                const uint4 av = next(2 * u + h);
                sum_up(2 * u + h, 0, av);
#pragma unroll
                for (int c = 0; c < N; ++c) {
                    const uint32_t v = wd[c][h], v4 = v << 4;
                    p[c] = mfma16(av, make_uint4(magic(v4, 0x00300030u, o.magic[0]), magic(v4, 0x00C000C0u, o.magic[1]),
                                                 magic(v, 0x00300030u, o.magic[0]), magic(v, 0x00C000C0u, o.magic[1])), zero);
                }
                add();
#pragma unroll
                for (int c = 0; c < N; ++c) {
                    before[c] = p[c];
                    by[c] = sc[c][h][u];
                }
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < L::GS; ++i) {
            f32x4_t p[N];
#pragma unroll
            for (int c = 0; c < N; ++c) p[c] = zero;
#pragma unroll
            for (int ww = 0; ww < Y::QW; ++ww) {
                const uint4 a0 = next(B == 2 ? i * Y::MPG + 2 * ww : i * Y::MPG + ww);
                sum_up(i, B == 2 ? 2 * ww : ww, a0);
                uint4 a1 = a0;
                if constexpr (B == 2) {
                    a1 = next(i * Y::MPG + 2 * ww + 1);
                    sum_up(i, 2 * ww + 1, a1);
                }
#pragma unroll
                for (int c = 0; c < N; ++c) {
                    const uint32_t v = word_of(s.w[c], i * Y::QW + ww);
                    if constexpr (B == 2) {
                        uint32_t x[8];
                        one_extract_w2(v, x, o.magic);
                        p[c] = mfma16(a0, make_uint4(x[0], x[1], x[2], x[3]), p[c]);
                        p[c] = mfma16(a1, make_uint4(x[4], x[5], x[6], x[7]), p[c]);
                    } else {
                        uint32_t x[4];
                        one_extract_w4(v, x, o.magic);
                        p[c] = mfma16(a0, make_uint4(x[0], x[1], x[2], x[3]), p[c]);
                    }
                }
            }
            add();
#pragma unroll
            for (int c = 0; c < N; ++c) {
                before[c] = p[c];
                by[c] = sc[c][0][i];
            }
        }
    }
    add();
    // the offset and zero-point terms
#pragma unroll
    for (int e = 0; e < L::NC; ++e)
#pragma unroll
        for (int c = 0; c < N; ++c) {
            f32x4_t& ac = acc[c % NM][c / NM];
            const uint32_t mw = L::GS == 2 && (q & 1) ? s.m[c][L::NW - 1] : s.m[c][e];
            const float sc = h2f(mw & 0xFFFFu), sz = sc * h2f(mw >> 16);
            if constexpr (L::GS == 1) {
                ac = mfma4(s.kc[0], q == 0 ? sc : q == 1 ? sz : 0.0f, ac);
            } else if constexpr (L::GS == 2) {
                ac = mfma4(s.kc[0], q < 2 ? sc : sz, ac);
            } else {
                ac = mfma4(s.kc[e], sc, ac);
                ac = mfma4(s.kx[e], sz, ac);
            }
        }
}
// Sums of the wave's steps first, first + kw, .. below ns: acc[m][t] of matrix m and
// the 16 rows from row0 + 16 t on, not yet scaled by kTileUnscale.  The first step's
// loads go out at once, and `more` issues what else the wave will need behind its
// weights; then a step's weights are under way while the one before is multiplied.
template <int B, int G, int NM, int RT, bool SUMS, typename MORE>
__device__ __forceinline__ void oneshot_products(f32x4_t (&acc)[NM][RT], const OneWork<NM>& o, int first, int ns, int kw,
                                                 int lane, MORE more) {
#pragma unroll
    for (int m = 0; m < NM; ++m)
#pragma unroll
        for (int t = 0; t < RT; ++t) acc[m][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    constexpr int NA = OneLay<B, G>::NA;
    constexpr int AH = one_ahead<B, G>();
    static_assert(NA % AH == 0, "a ring slot is known at compile time");
    OneStep<B, G, NM, RT> s;
    uint4 r[AH];
    int gs = first;                                        // < ns
    one_load<B, G, NM, RT, SUMS>(s, o, gs, lane);
    more();
#pragma unroll
    for (int n = 0; n < AH; ++n) one_operand<B, G, NM>(r[n], o, gs, n);
    __builtin_amdgcn_sched_barrier(0);                     // every load above is issued before the first is waited for
    auto multiply = [&](bool last) {
        one_multiply<B, G, NM, RT, SUMS>(acc, s, o, gs, lane, [&](int n) {
            const int f = n + AH;
            const uint4 a = r[n % AH];
            if (!last || f < NA)
                one_operand<B, G, NM>(r[n % AH], o, f < NA ? gs : gs + kw, f % NA);
            return a;
        });
    };
    for (; gs + kw < ns; gs += kw) {
        OneStep<B, G, NM, RT> n;
        one_load<B, G, NM, RT, SUMS>(n, o, gs + kw, lane);
        __builtin_amdgcn_sched_barrier(0);
        multiply(false);
        s = n;
    }
    multiply(true);
}

// ---- activations in the operands' order, for the launch before
// Where element e of a row goes (within its block of 16), and 2^-10 of the offset of
// the codes that it meets.
__device__ __forceinline__ int operand_at(int e, int bits, int g) {
    return bits == 2 && g != 32 ? (e & ~15) + 2 * (e & 7) + ((e >> 3) & 1) : (e & ~7) + 2 * (e & 3) + ((e >> 2) & 1);
}
__device__ __forceinline__ float operand_offset(int e, int bits, int g) {
    int p;                                                 // fraction position of the element's pair
    if (bits == 4)
        p = (e & 3) < 2 ? 4 : 6;
    else if (g == 32 || (e & 7) < 4)
        p = (e & 1) ? 6 : 4;
    else
        p = (e & 3) == 1 ? 4 : (e & 3) == 2 ? 6 : 8;
    return __uint_as_float((uint32_t)(127 + kPosMin - p) << 23);
}
// Sixteen elements of a row (fp32, already binary16 values) as two operands, and the
// sums -C and -X of the group they are in: lanes whose blocks share a group lie side
// by side, and each gets the sums.
__device__ __forceinline__ void operand16(const float (&f)[16], int bits, int g, uint4 (&o)[2], float& c, float& x) {
    uint32_t w[8];
    c = x = 0.0f;
    const bool across = bits == 2 && g != 32;              // pairs (e, 8 + e) of 16, or (e, 4 + e) of 8
#pragma unroll
    for (int p = 0; p < 8; ++p) {
        const int e0 = across ? p : (p & 3) + 8 * (p >> 2), e1 = across ? 8 + p : e0 + 4;
        const float f0 = across ? f[p] : f[(p & 3) + 8 * (p >> 2)], f1 = across ? f[8 + p] : f[(p & 3) + 8 * (p >> 2) + 4];
        w[p] = f2h(f0) | f2h(f1) << 16;
        c += f0 * operand_offset(e0, bits, g) + f1 * operand_offset(e1, bits, g);
        x += f0 + f1;
    }
    c = -1024.0f * c;
    x = -16.0f * x;
    if (g == 32) {
        c = group_sum<2>(c);
        x = group_sum<2>(x);
    } else if (g == 64) {
        c = group_sum<4>(c);
        x = group_sum<4>(x);
    } else {
        c = group_sum<8>(c);
        x = group_sum<8>(x);
    }
    o[0] = make_uint4(w[0], w[1], w[2], w[3]);
    o[1] = make_uint4(w[4], w[5], w[6], w[7]);
}

// The e of a bfloat16 row whose largest element is top = f 2^E, 1 <= f < 2: 14 - E,
// with 2^e a normal number (a row whose largest is below 2^-112, or not finite,
// keeps 126 or -114).
__device__ __forceinline__ int row_shift(float top) { return min(14 - ((int)(__float_as_uint(top) >> 23) - 127), 126); }

__device__ __forceinline__ uint4 ld16(const void* p) {
    const u32x4 v = *reinterpret_cast<const u32x4*>(p);
    return make_uint4(v.x, v.y, v.z, v.w);
}

// Eight values of the activation type (binary16, or bfloat16 where bf) as fp32.
__device__ __forceinline__ void act8(const uint4& v, bool bf, float (&f)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = bf ? __uint_as_float(w[i] << 16) : h2f(w[i] & 0xFFFFu);
        f[2 * i + 1] = bf ? __uint_as_float(w[i] & 0xFFFF0000u) : h2f(w[i] >> 16);
    }
}

// fp32 to the activation type, nearest even.
__device__ __forceinline__ uint16_t act_bits(float v, bool bf) {
    if (!bf)
        return (uint16_t)f2h(v);
    return __builtin_bit_cast(uint16_t, (__bf16)v);
}

// A row of K binary16 or (bf) bfloat16 elements in operand order, padded with zeros,
// and its group sums, by a workgroup of W waves, at o and sums among `rows` rows
// side by side; bfloat16 times 2^e, 2^-e to *back.  16 elements per lane; the first N
// pieces of a wave stay in its registers between the two passes that bfloat16 takes.
template <int W>
__device__ __forceinline__ void operands_of_row(const uint16_t* x, int K, bool bf, int bits, int g, uint4* o, float2* sums,
                                                int rows, float* back, int tid) {
    constexpr int N = 3;
    __shared__ uint32_t best[W];
    const int lane = tid & 63, wave = tid >> 6, len = operand_row(K, bits);
    uint4 v[N][2];
    auto load = [&](uint4 (&r)[2], int e) {
        const uint4 z = make_uint4(0, 0, 0, 0);
        r[0] = e < K ? *reinterpret_cast<const uint4*>(x + e) : z;
        r[1] = e < K ? *reinterpret_cast<const uint4*>(x + e + 8) : z;
    };
    auto widen = [&](const uint4 (&r)[2], float (&f)[16]) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float t[8];
            act8(r[h], bf, t);
#pragma unroll
            for (int i = 0; i < 8; ++i) f[8 * h + i] = t[i];
        }
    };
    const int first = (wave * 64 + lane) * 16, step = W * 1024;
#pragma unroll
    for (int i = 0; i < N; ++i) load(v[i], first + i * step);
    float up = 1.0f;
    if (bf) {
        // the largest magnitude by its bits, two at a time (a NaN is the largest: its row is lost in any case)
        typedef uint16_t u16x2_t __attribute__((ext_vector_type(2)));
        u16x2_t mag = {0, 0};
        auto most = [&](const uint4 (&r)[2]) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t w[4] = {r[h].x, r[h].y, r[h].z, r[h].w};
#pragma unroll
                for (int u = 0; u < 4; ++u) mag = __builtin_elementwise_max(mag, __builtin_bit_cast(u16x2_t, w[u] & 0x7FFF7FFFu));
            }
        };
#pragma unroll
        for (int i = 0; i < N; ++i) most(v[i]);
        for (int e = first + N * step; e < K; e += step) {
            uint4 r[2];
            load(r, e);
            most(r);
        }
        uint32_t top = wave_max(max((uint32_t)mag.x, (uint32_t)mag.y));
        if (lane == 0)
            best[wave] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < W; ++w) top = max(top, best[w]);
        const int e = row_shift(__uint_as_float(top << 16));
        up = __uint_as_float((uint32_t)(127 + e) << 23);
        if (tid == 0)
            *back = __uint_as_float((uint32_t)(127 - e) << 23);
    }
    auto put = [&](const uint4 (&r)[2], int e) {
        float f[16], c, xs;
        uint4 w[2];
        widen(r, f);
        if (bf)
#pragma unroll
            for (int u = 0; u < 16; ++u) f[u] = h2f(f2h(f[u] * up));
        operand16(f, bits, g, w, c, xs);
        if (e < len) {
            o[(long)(e / 8) * rows] = w[0];
            o[(long)(e / 8 + 1) * rows] = w[1];
            if (e % g == 0)
                sums[(long)(e / g) * rows] = make_float2(c, xs);
        }
    };
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (wave * 1024 + i * step < len)                  // (waves past the row's end have nothing to write)
            put(v[i], first + i * step);
    for (int e0 = N * step; e0 < len; e0 += step) {
        const int e = first + e0;
        uint4 r[2];
        load(r, e);
        put(r, e);
    }
}

}  // namespace
}  // namespace qmlp
