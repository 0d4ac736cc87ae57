// Causal attention over the 4-bit cache for many rows a request (prompts and their chunks), gfx950.
//
// The mathematics of kv_attention.hip.  With rows to spare what bounds it is arithmetic: the matrix products, and beside
// them the weights (an exponential and five more operations for each of rows x tokens).  So a workgroup takes 256 rows
// (of all heads that share a K/V head), unpacks 64 tokens (128 where heads are 64 wide) once for all of them into LDS, as
// exact binary16 integers code - zero, and the scales go on the scores and the weights, which are touched anyway.  A
// wave owns 32 rows; its products are transposed (tokens or dims down, rows across), so that weights go from one
// product to the other in registers.  Three stages of LDS (see the loop).
//
// LDS: K [tokens][D], 16-byte pieces (8 dims) at place p ^ (token & 7); V [D dims][tokens], a piece being the eight
// tokens a lane multiplies at once (16 s + 4 h + {0..3, 8..11}), at place p ^ (dim & 7) ^ (dim / 8 & 7), so that
// eight neighbouring lanes read different banks.  (Not all: at D = 128 a row of K has 16 pieces and a read stays in half of them.
// By counters 21 % of the cycles of LDS are conflicts.)
//
// Prompts of 2501, 2058 and 1341 tokens of 32 heads of 128 on 8 K/V heads: 179 us (563 TFLOP/s); 1000 tokens after 15000
// beside 15 decoding requests: 337 us (754 TFLOP/s, where a large product of the library reaches 1160).  On the way:
// 128 rows a workgroup 195 and 438 us; 256 rows 205 and 397; tiles handed out by their length 200; weights and products in turns
// with operands from LDS two turns ahead 187 and 359; a third stage, so that every tile has both neighbours' products
// beside it, 181 and 356; pieces of V without turned halves 177 and 348.  By counters (the mixed step) the
// vector units are busy 54 % of the time and the matrix cores 33 %, waves wait for data or each other 35 %; steps of 128 tokens
// at D = 128 spilled registers (398 us).
#include "qmlp_internal.h"

#include "decode_launch.h"
#include "kv_device.h"
#include "kv_window.h"

namespace qmlp {
namespace {

constexpr int kWaves = 8, kTileRows = 32 * kWaves, kThreads = 64 * kWaves, kMostShares = 16;
constexpr uint32_t kApart = 12;                           // powers of two
constexpr int kJoin = 8;                                  // parts under way where they are joined

template <int D>
struct __attribute__((aligned(256))) Stage {
    static constexpr int tokens = 8192 / D;               // of a step: 64 or 128
    uint16_t k[tokens * D];
    uint16_t v[D * tokens];
    float sk[tokens], sv[tokens];
    uint32_t away[kWaves];                                // nonzero: a wave met tokens that are not there
};

template <int D>
__global__ void __launch_bounds__(kThreads, 2) rows_kernel(AttnArgs a, int limit, int target) {
    constexpr int KS = D / 16, DT = D / 32, kTokens = Stage<D>::tokens, TJ = kTokens / 32;
    using St = Stage<D>;
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    __shared__ uint32_t arrived, tops[kWaves], leasts[kWaves];
    __shared__ float backs[kTileRows];                    // of each row, where they differ: its power's inverse
    Stage<D>* stage = reinterpret_cast<Stage<D>*>(smem);
    Known<int32_t>* known = reinterpret_cast<Known<int32_t>*>(smem + 3 * sizeof(Stage<D>));
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5, col = lane & 31;
    const int lg = a.cache.page_log2, Hk = a.cache.heads;

    auto tiles_of = [&](const Request& q) {
        const long rows = (long)q.n * a.G;
        return rows <= limit ? 0 : (int)((rows + kTileRows - 1) / kTileRows);
    };
    const int tiles = prefix_work<kThreads, int32_t>(a, known, [&](const Request& q) { return tiles_of(q); });
    const int items = tiles * Hk;
    // few items: the tokens of each are shared by several workgroups
    const int shares = items ? min(max(target / items, 1), kMostShares) : 1;
    if ((int)blockIdx.x >= items * shares)
        return;
    // neighbouring workgroups (on different XCDs) take different K/V heads; tiles go by the tokens before their end,
    // most first, so that the last to be handed out are short (ties: by request)
    const int head = (int)blockIdx.x % Hk, rest = (int)blockIdx.x / Hk, part = rest % shares, nth = rest / shares;
    // tiles of a request with at least s steps before their end
    auto longer = [&](const Request& q, int s) {
        const int x = (s - 1) * kTokens - (q.len - q.n), nt = tiles_of(q);
        return nt == 0 || x > q.n - 1 ? 0 : x <= 0 ? nt : nt - (int)((long)x * a.G / kTileRows);
    };
    auto count = [&](int s) {
        int c = 0;
        for (int i = lane; i < a.B; i += 64)
            c += longer(known[i].q, s);
#pragma unroll
        for (int d = 1; d < 64; d <<= 1)
            c += __shfl_xor(c, d, 64);
        return __builtin_amdgcn_readfirstlane(c);
    };
    // the most steps that more than nth tiles have, and which of the tiles with just that many
    // (a request with fewer tokens than rows begins before 0)
    int lo = -(a.T / kTokens) - 2, hi = (a.W << lg) / kTokens + 2;          // count(lo) > nth >= count(hi)
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (count(mid) > nth)
            lo = mid;
        else
            hi = mid;
    }
    int left = nth - count(hi), b = 0, tile = 0;
    for (int b0 = 0; b0 < a.B; b0 += 64) {
        int c = 0, c1 = 0;
        if (b0 + lane < a.B) {
            c1 = longer(known[b0 + lane].q, hi);
            c = longer(known[b0 + lane].q, lo) - c1;
        }
        int before = c;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(before, d, 64);
            before += lane >= d ? o : 0;
        }
        const int all = __builtin_amdgcn_readlane(before, 63);
        before -= c;
        if (left < all) {
            const int src = __builtin_ctzll(__ballot(left >= before && left < before + c));
            b = b0 + src;
            tile = __builtin_amdgcn_readlane(c1, src) + left - __builtin_amdgcn_readlane(before, src);      // from the last
            break;
        }
        left -= all;
    }
    b = __builtin_amdgcn_readfirstlane(b);
    const Request q = known[b].uniform();
    tile = tiles_of(q) - 1 - tile;
    const int rows = min((int)((long)q.n * a.G - (long)tile * kTileRows), kTileRows);
    const int first = q.len - q.n + tile * kTileRows / a.G, last = q.len - q.n + (tile * kTileRows + rows - 1) / a.G;   // positions
    const int low0 = first_seen(first, a.window) / kTokens;
    const int all = max(0, last / kTokens + 1 - low0);    // steps of the tile (last < 0: none)
    // (at least four steps a share: joining costs about as much)
    const int own = min(shares, max(1, all / 4));
    if (part >= own)
        return;
    const int i0 = low0 + (int)((long)all * part / own), i1 = low0 + (last < 0 ? 0 : (int)((long)all * (part + 1) / own));

    // the wave's rows' positions, and this lane's row
    const int wrows = min(rows - wave * 32, 32);
    const int wfirst = q.len - q.n + (tile * kTileRows + wave * 32) / a.G;
    const int wlast = wrows > 0 ? q.len - q.n + (tile * kTileRows + wave * 32 + wrows - 1) / a.G : -1;
    const int r = wave * 32 + col, row = tile * kTileRows + r, tok = row / a.G;
    const int pos = r < rows ? q.len - q.n + tok : -1;
    const int low = first_seen(pos, a.window);
    uint4 qv[KS];
    {
        const uint16_t* src = a.q + (long)(q.row0 + tok) * a.ldq + ((long)head * a.G + row % a.G) * D + h * 8;
#pragma unroll
        for (int i = 0; i < KS; ++i)
            qv[i] = r < rows ? *reinterpret_cast<const uint4*>(src + 16 * i) : make_uint4(0, 0, 0, 0);
    }

    // staging: a thread of the lower four waves takes 4 words of a token of K, one of the upper four a word of 4 tokens of V
    const bool takes_k = wave < 4;
    const int sid = tid & 255;
    const int ktok = D == 128 ? sid >> 2 : sid >> 1, kc = D == 128 ? sid & 3 : sid & 1;
    // (16 neighbouring threads of V: eight words of the two quads that share pieces)
    const int vword = (sid & 7) | (D == 128 ? (sid >> 1) & 8 : 0);
    const int vquad = D == 128 ? ((sid >> 2) & 2) | ((sid >> 5) & 1) | ((sid >> 4) & 12) : ((sid >> 2) & 2) | ((sid >> 4) & 1) | ((sid >> 3) & 28);
    const int mine0 = takes_k ? ktok : 4 * vquad;         // the first token of it
    int page = 0;                                         // page number of the step to be loaded next
    auto load_pages = [&](int i) { page = a.table[(long)b * a.W + min((i * kTokens + mine0) >> lg, a.W - 1)]; };
    uint4 codes, meta;                                    // (meta of K: one token's, in x)
    int there = 0;                                        // how many of its tokens are there
    auto load = [&](int i) {
        const int t = i * kTokens + mine0;
        const bool known_page = (uint32_t)page < (uint32_t)a.cache.pages;
        there = known_page ? min(max(q.len - t, 0), takes_k ? 1 : 4) : 0;
        const uint8_t* base = a.cache.at(D, known_page ? page : 0, head) + (takes_k ? 0u : a.cache.side(D));
        const uint32_t o = (uint32_t)t & ((1u << lg) - 1u);
        codes = *reinterpret_cast<const uint4*>(base + o * (D / 2) + (takes_k ? kc : vword) * 16);
        base += ((uint32_t)(D / 2) << lg) + o * 4u;
        if (takes_k)
            meta.x = *reinterpret_cast<const uint32_t*>(base);
        else
            meta = *reinterpret_cast<const uint4*>(base);
    };
    float scale = 0.0f;                                   // of a raw score, with the power of two of q
    const uint32_t mv = magic64();
    auto put = [&](Stage<D>& s) {
        if (takes_k) {
            const uint32_t m = there ? meta.x : 0x3C00u;
            const uint32_t z = (m >> 16) | (m & 0xFFFF0000u), off = add2(z, mv) ^ 0x80008000u;        // -(64 + zero), twice
            // (threads of the upper half of a row begin with its second pair of words: see the banks above)
            const bool turn = D == 128 && (kc & 2);
            const uint32_t w[4] = {turn ? codes.z : codes.x, turn ? codes.w : codes.y, turn ? codes.x : codes.z, turn ? codes.y : codes.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t e[4];
                pairs64(w[i], mv, e);
                const int piece = 4 * kc + (i ^ (turn ? 2 : 0));
                *reinterpret_cast<uint4*>(s.k + ktok * D + ((piece ^ (ktok & 7)) << 3)) =
                    make_uint4(add2(e[0], off), add2(e[1], off), add2(e[2], off), add2(e[3], off));
            }
            if (kc == 0)
                s.sk[ktok] = there ? finite(h2f(m & 0xFFFFu) * scale) : INFINITY;       // (a scale is never infinite: not there)
        } else {
            uint32_t m[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                m[i] = i < there ? comp(meta, i) : 0x3C00u;
            const uint32_t off[2] = {add2(highs(m[0], m[1]), mv) ^ 0x80008000u, add2(highs(m[2], m[3]), mv) ^ 0x80008000u};
            uint32_t out[8][2];
#pragma unroll
            for (int pr = 0; pr < 2; ++pr) {
                uint32_t e[4], f[4];
                pairs64(lows(comp(codes, 2 * pr), comp(codes, 2 * pr + 1)), mv, e);
                pairs64(highs(comp(codes, 2 * pr), comp(codes, 2 * pr + 1)), mv, f);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    out[2 * i][pr] = add2(e[i], off[pr]);
                    out[2 * i + 1][pr] = add2(f[i], off[pr]);
                }
            }
            const int piece = 2 * (vquad >> 2) + (vquad & 1), half = (vquad >> 1) & 1;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                *reinterpret_cast<uint2*>(s.v + (8 * vword + j) * kTokens + ((piece ^ j ^ (vword & 7)) << 3) + 4 * half) =
                    make_uint2(out[j][0], out[j][1]);
            if (vword == 0)
                *reinterpret_cast<float4*>(s.sv + 4 * vquad) =
                    make_float4(h2f(m[0] & 0xFFFFu), h2f(m[1] & 0xFFFFu), h2f(m[2] & 0xFFFFu), h2f(m[3] & 0xFFFFu));
        }
        const uint64_t gone = __ballot(there < (takes_k ? 1 : 4));
        if (lane == 0)
            s.away[wave] = gone != 0;
    };

    f32x16_t o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i)
            o[d][i] = 0.0f;
    float m = kNone, l = 0.0f;
    if (i0 < i1) {
        load_pages(i0);
        load(i0);
        if (i0 + 1 < i1)
            load_pages(i0 + 1);
    }
    float qsum;
    // One power of two for the workgroup's rows, which the scales of keys take along, unless a row's largest number is below 2^-kApart
    // of the others'.  Then each row has its own, and every step goes the way of partly seen ones, which multiplies by it: what a
    // row shares loses below 2^-(39 - kApart) of its largest number, less than an fp32 sum does.
    bool apart = false;
    const float back = operand_rows(qv, a.bf, qsum, [](float v) { return v + __shfl_xor(v, 32, 64); },
                                    [](uint32_t v) { return v | (uint32_t)__shfl_xor((int)v, 32, 64); },
                                    [&](uint32_t top) {
                                        top = max(top, (uint32_t)__shfl_xor((int)top, 32, 64));
                                        uint32_t most = wave_max(top), least = ~wave_max(top ? ~top : 0u);      // (no row of zeros)
                                        if (lane == 0) {
                                            tops[wave] = most;
                                            leasts[wave] = least;
                                        }
                                        __syncthreads();
#pragma unroll
                                        for (int w = 0; w < kWaves; ++w) {
                                            most = max(most, tops[w]);
                                            least = min(least, leasts[w]);
                                        }
                                        apart = __builtin_amdgcn_readfirstlane(least < most && (most >> 7) - (least >> 7) > kApart);
                                        return apart ? top : most;
                                    });
    if (apart && h == 0)
        backs[r] = back;                                  // (read by this wave alone)
    scale = apart ? a.scale : a.scale * back;
    const bool bad = qsum != qsum;                        // an infinity or NaN in the row

    // Three stages: at step i the matrix cores read stages i and i + 1 and, in the step's first turns, i - 1, whose
    // place stage i + 2 then takes.  One meeting of the waves a step, after those turns.
    if (i0 < i1) {
        put(stage[0]);
        if (i0 + 1 < i1) {
            load(i0 + 1);
            put(stage[1]);
            if (i0 + 2 < i1) {
                load_pages(i0 + 2);
                load(i0 + 2);
                if (i0 + 3 < i1)
                    load_pages(i0 + 3);
            }
        }
    }
    __syncthreads();

    // Tiles of 32 tokens.  While a tile's weights are formed on the vector units, the matrix cores have the next
    // tile's scores and the last one's output: a wave issues in order, so their instructions alternate.  Their first
    // operands come from LDS two turns ahead, the scales half a tile.
    f32x16_t x[2];                                        // scores, tokens 32 j + 8 (e / 4) + 4 h + e % 4 of row `col`
    uint32_t pk[2][8] = {};                               // weights times scales
    uint4 kf[3], vf[3];
    float4 sk[2], sv[2];
    const uint32_t kplace = (uint32_t)(col * D * 2 + ((h ^ (col & 7)) << 4));
    const uint32_t vplace = (uint32_t)(offsetof(Stage<D>, v) + col * kTokens * 2 + ((h ^ (col & 7) ^ (col >> 3)) << 4));
    const uint32_t splace = (uint32_t)offsetof(Stage<D>, sk) + 16u * h;
    uint32_t before = 0, now = 0, next = (uint32_t)sizeof(Stage<D>);        // where the stages are (of the first step: no output yet, weights 0)
    // (places in LDS are formed anew from one number each: kept apart they would take the registers)
    uint32_t kat = 0, vat = 0, sat = 0;
    // turn n = 0 .. KS - 1 of tile j: step n of the scores of tile j + 1, and of the output of tile j - 1 (piece 2 (j - 1) + u + h of
    // dim 32 d + col)
    auto fetch = [&](int j, int n) {
        const int jk = (j + 1) % TJ, jv = (j + TJ - 1) % TJ, u = n / DT, d = n % DT;
        kf[n % 3] = *reinterpret_cast<const uint4*>(smem + (kat ^ (uint32_t)(n << 5)) + jk * 64 * D);
        vf[n % 3] = *reinterpret_cast<const uint4*>(smem + (vat ^ (uint32_t)(jv << 6 ^ u << 5 ^ (d & 1) << 6)) + d * 64 * kTokens);
    };
    auto scales = [&](int j, int g) {                     // of tokens 32 j + 8 g + 4 h ..
        sk[g & 1] = *reinterpret_cast<const float4*>(smem + sat + 128 * j + 32 * g);
        sv[g & 1] = *reinterpret_cast<const float4*>(smem + sat + 128 * j + 32 * g + 4 * kTokens);
    };
    auto begin = [&](int j, bool of_next) {               // of tile j of this step, or of the next one's first
        kat = (j + 1 < TJ && !of_next ? now : next) + kplace;
        vat = (j > 0 || of_next ? now : before) + vplace;
        sat = (of_next ? next : now) + splace;
        pin(kat);
        pin(vat);
        pin(sat);
        fetch(j, 0);
        fetch(j, 1);
        scales(j, 0);
    };
    auto output = [&](int j, int n) {
        const int u = n / DT, d = n % DT;
        const uint32_t(&w)[8] = pk[(j + 1) & 1];
        o[d] = mfma32(vf[n % 3], make_uint4(w[4 * u], w[4 * u + 1], w[4 * u + 2], w[4 * u + 3]), o[d]);
    };
    auto zero = [](f32x16_t& y) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
            y[e] = 0.0f;
    };
    auto section = [&](auto tile_of_step, int t, bool full) {
        constexpr int j = decltype(tile_of_step)::value;
        f32x16_t &xj = x[j & 1], &y = x[(j + 1) & 1];
        uint32_t(&pj)[8] = pk[j & 1];
        const St& s = *reinterpret_cast<const St*>(smem + now);
        float sum = 0.0f;
        uint32_t top = 0;                                 // of the rounded weights, two by two
        // weights of two tokens, scores times their scales (or, where they have been seen to, as they are)
        auto weigh2 = [&](int e, const float4& ks, const float4& vs, auto raw) {
            const float ka = e & 2 ? ks.z : ks.x, kb = e & 2 ? ks.w : ks.y, va = e & 2 ? vs.z : vs.x, vb = e & 2 ? vs.w : vs.y;
            float ea, eb, wa, wb;
            if constexpr (decltype(raw)::value) {
                ea = exp2_(__builtin_fmaf(xj[e], ka, -m));
                eb = exp2_(__builtin_fmaf(xj[e + 1], kb, -m));
                wa = ea * va;
                wb = eb * vb;
            } else {
                ea = exp2_(xj[e] - m);
                eb = exp2_(xj[e + 1] - m);
                wa = xj[e] == -INFINITY ? 0.0f : ea * va;                    // (the scale may be NaN)
                wb = xj[e + 1] == -INFINITY ? 0.0f : eb * vb;
            }
            sum += ea + eb;
            pj[e >> 1] = pack2(wa, wb);
            top = max2(top, pj[e >> 1]);
        };
        auto weigh = [&] {                                // all of them, as they are
            sum = 0.0f;
            top = 0;
#pragma unroll
            for (int e = 0; e < 16; e += 2)
                weigh2(e, float4{}, *reinterpret_cast<const float4*>(s.sv + 32 * j + 8 * (e >> 2) + 4 * h), std::false_type{});
        };
        zero(y);
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            constexpr int per = 16 / KS;                  // weights of a turn
            if (k + 2 < KS)
                fetch(j, k + 2);
            y = mfma32(kf[k % 3], qv[k], y);
            output(j, k);
            if (per * k % 4 == 0 && per * k / 4 + 1 < 4)
                scales(j, per * k / 4 + 1);
#pragma unroll
            for (int e = per * k; e < per * (k + 1); e += 2)
                weigh2(e, sk[(e >> 2) & 1], sv[(e >> 2) & 1], std::true_type{});
            // (they stay here, and are not put off to where it is known that every token is seen)
            pin(top);
            __asm__ volatile("" : "+v"(sum));
            __builtin_amdgcn_sched_barrier(0);
        }
        if (j > 0)
            begin((j + 1) % TJ, j + 1 == TJ);
        if (!full) {
            // what a row does not see weighs nothing, whatever lies there
            const float back = apart ? backs[r] : 1.0f;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int at = 32 * j + 8 * (e >> 2) + 4 * h + (e & 3), n = t + at;
                const float k1 = s.sk[at];
                xj[e] = n <= pos && n >= low && k1 != INFINITY ? rounded(xj[e] * k1 * back) : -INFINITY;
            }
            weigh();
        }
        // (a weight that passes binary16 is infinite there)
        if (__ballot(h2f(top & 0xFFFFu) > kTop || h2f(top >> 16) > kTop || sum > 16.0f * kTop * kLeast)) {
            float best = kNone, most = kNone;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int at = 32 * j + 8 * (e >> 2) + 4 * h + (e & 3);
                if (full)
                    xj[e] = rounded(xj[e] * s.sk[at]);
                most = fmaxf(most, xj[e]);
                best = fmaxf(best, xj[e] + log2_(fmaxf(s.sv[at], 1.0f / kLeast)));
            }
            most = fmaxf(most, __shfl_xor(most, 32, 64));
            best = fmaxf(best, __shfl_xor(best, 32, 64));
            const float mn = shifted(m, most, best), f = exp2_(m - mn);
            m = mn;
            l *= f;
#pragma unroll
            for (int d = 0; d < DT; ++d)
                o[d] *= f;
            weigh();
        }
        l += sum;
    };

    if (i0 < i1) {                                        // the first tile's scores
        kat = now + kplace;
        pin(kat);
        zero(x[0]);
#pragma unroll
        for (int k = 0; k < KS; ++k)
            x[0] = mfma32(*reinterpret_cast<const uint4*>(smem + (kat ^ (uint32_t)(k << 5))), qv[k], x[0]);
        begin(0, false);
    }
    auto last_output = [&] {
        vat = before + vplace;
        pin(vat);
#pragma unroll
        for (int n = 0; n < KS; ++n) {
            const int u = n / DT, d = n % DT;
            vf[n % 3] = *reinterpret_cast<const uint4*>(smem + (vat ^ (uint32_t)((TJ - 1) << 6 ^ u << 5 ^ (d & 1) << 6)) + d * 64 * kTokens);
            output(0, n);
        }
    };
    for (int i = i0; i < i1; ++i) {
        const int t = i * kTokens;
        const St& s = *reinterpret_cast<const St*>(smem + now);
        const uint4 aw = *reinterpret_cast<const uint4*>(s.away), aw2 = *reinterpret_cast<const uint4*>(s.away + 4);
        const bool full = !apart && __builtin_amdgcn_readfirstlane((aw.x | aw.y | aw.z | aw.w | aw2.x | aw2.y | aw2.z | aw2.w) == 0 &&
                                                         t + kTokens - 1 <= wfirst && t >= first_seen(wlast, a.window));
        section(std::integral_constant<int, 0>{}, t, full);
        __syncthreads();
        begin(1, false);
        if (i + 2 < i1) {
            put(*reinterpret_cast<St*>(smem + (i == i0 ? 2 * (uint32_t)sizeof(St) : before)));
            if (i + 3 < i1) {
                load(i + 3);
                if (i + 4 < i1)
                    load_pages(i + 4);
            }
        }
        section(std::integral_constant<int, 1>{}, t, full);
        if constexpr (TJ > 2) {
            section(std::integral_constant<int, 2>{}, t, full);
            section(std::integral_constant<int, 3>{}, t, full);
        }
        const uint32_t free = i == i0 ? 2 * (uint32_t)sizeof(St) : before;
        before = now;
        now = next;
        next = free;
    }
    if (i0 < i1)
        last_output();
    l += __shfl_xor(l, 32, 64);
    if (bad && l != 0.0f)
        l = NAN;

    const int g = head * a.G + row % a.G;
    uint16_t* y = a.y + (long)(q.row0 + tok) * a.ldy + (long)g * D;
    if (own == 1) {
        const float f = row_factor(a, g, m, l);
        if (r < rows)
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float v[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        v[k] = l == 0.0f ? 0.0f : o[d][4 * e + k] * f;
                    store4(y + 32 * d + 8 * e + 4 * h, v, a.bf);
                }
        return;
    }
    // parts of an item: [rows][D], then m and l of the rows; the last to come joins them
    typedef uint32_t w4 __attribute__((ext_vector_type(4)));
    const int item = nth * Hk + head;
    const size_t place = (size_t)kTileRows * (D + 2) * 4;
    uint8_t* parts = reinterpret_cast<uint8_t*>(a.part) + (size_t)item * shares * place;
    const Rsrc rp = rsrc(parts, (uint32_t)(place * own));
    const uint32_t mine = (uint32_t)(part * place);
    if (r < rows) {
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const w4 u = {__float_as_uint(o[d][4 * e]), __float_as_uint(o[d][4 * e + 1]), __float_as_uint(o[d][4 * e + 2]),
                              __float_as_uint(o[d][4 * e + 3])};
                __builtin_amdgcn_raw_buffer_store_b128(u, rp, mine + (uint32_t)(r * D + 32 * d + 8 * e + 4 * h) * 4u, 0, kDevice);
            }
        if (h == 0) {
            __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(m), rp, mine + (uint32_t)(kTileRows * D + r) * 4u, 0, kDevice);
            __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(l), rp, mine + (uint32_t)(kTileRows * (D + 1) + r) * 4u, 0, kDevice);
        }
    }
    __asm__ volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (tid == 0)
        arrived = __hip_atomic_fetch_add(a.done + item, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    if (arrived != (uint32_t)own - 1u)
        return;
    if (tid == 0)
        __hip_atomic_store(a.done + item, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    for (int c = tid; c < rows * (D / 4); c += kThreads) {
        const int jr = c / (D / 4), d = 4 * (c % (D / 4)), rr = tile * kTileRows + jr, gg = head * a.G + rr % a.G;
        float mm = kNone, ls = 0.0f, v[4] = {0, 0, 0, 0};
        for (int p0 = 0; p0 < own; p0 += kJoin) {
            w4 u[kJoin];
            float pm[kJoin], pl[kJoin];
#pragma unroll
            for (int k = 0; k < kJoin; ++k) {
                if (p0 + k >= own)
                    break;
                const uint32_t at = (uint32_t)((p0 + k) * place);
                u[k] = __builtin_amdgcn_raw_buffer_load_b128(rp, at + (uint32_t)(jr * D + d) * 4u, 0, kDevice);
                pm[k] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rp, at + (uint32_t)(kTileRows * D + jr) * 4u, 0, kDevice));
                pl[k] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rp, at + (uint32_t)(kTileRows * (D + 1) + jr) * 4u, 0, kDevice));
            }
#pragma unroll
            for (int k = 0; k < kJoin; ++k)
                if (p0 + k < own) {
                    const float mn = fmaxf(mm, pm[k]), f0 = exp2_(mm - mn), f1 = exp2_(pm[k] - mn);
                    mm = mn;
                    ls = ls * f0 + pl[k] * f1;
#pragma unroll
                    for (int x = 0; x < 4; ++x)
                        v[x] = v[x] * f0 + __uint_as_float(u[k][x]) * f1;
                }
        }
        const float f = row_factor(a, gg, mm, ls);
#pragma unroll
        for (int k = 0; k < 4; ++k)
            v[k] = ls == 0.0f ? 0.0f : v[k] * f;
        store4(a.y + (long)(q.row0 + rr / a.G) * a.ldy + (long)gg * D + d, v, a.bf);
    }
}

int rows_target() { return plan_cus(); }

template <int D>
hipError_t launch(const AttnArgs& a, int limit, hipStream_t st) {
    const size_t lds = 3 * sizeof(Stage<D>) + (size_t)a.B * sizeof(Known<int32_t>);
    const hipError_t e = set_lds(rows_kernel<D>, lds + 1024);
    if (e != hipSuccess)
        return e;
    // tiles of the requests at most: each may have one that is not full
    const int most = ((int)((long)a.T * a.G / kTileRows) + (a.B < a.T ? a.B : a.T)) * a.cache.heads;
    rows_kernel<D><<<most > rows_target() ? most : rows_target(), kThreads, lds, st>>>(a, limit, rows_target());
    return hipGetLastError();
}

}  // namespace

size_t kv_rows_bytes(int D) { return (size_t)rows_target() * kTileRows * (D + 2) * 4; }

hipError_t launch_kv_rows(const AttnArgs& a, int limit, hipStream_t st) {
    return a.D == 128 ? launch<128>(a, limit, st) : launch<64>(a, limit, st);
}

}  // namespace qmlp
