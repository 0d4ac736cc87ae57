// Causal attention over the 4-bit cache for a few rows a request (decoding), gfx950.
//
//   s_j = scale q . K_j,  w_j = 2^(s_j log2(e) - m),  y = sum_j w_j V_j / (sum_j w_j + sink)
//
// One pass over the tokens, the maximum m and the sum carried along.  What bounds it is reading the cache
// (D + 8 bytes a token and head), so all heads that share a K/V head, and the rows of a request, are one
// operand of up to 16 rows, and codes go from the loads to the matrix cores in registers: the cache's layout
// is the operands'.  K: a lane's D/4 dims of one token, codes as 64 + code; with u = sum q the offset comes off as
// s = scale_K (sum q (64 + c) - (64 + zero) u).  The product is transposed (tokens down, rows
// across), so that a lane's eight weights are those of one row and go on as the second product's operand without
// moving.  V: a lane's words are 4 tokens' same 8 dims; halves of two tokens' words side by side give the pairs.
// Weights times the values' scales are rounded to binary16 (fp32 sums of exact products after that), and the zeros come
// off through one more product of the same weights with 64 + zero.
//
// The rounding to binary16 is made where weights are at most 2^15 and, when the maximum is taken anew, 2^8: normal
// numbers down to 2^-22 of the largest.  m moves only when a weight would pass 2^15.
//
// 131072 tokens of 8 K/V heads of 128 (143 MB) take 38.9 us, of which the pass over the cache is 24 us (5.8 TB/s, by clocks in the
// kernel), 3 us go before it (lengths, pages, the first loads: three trips to memory) and the rest to joining 64 parts.  One
// sequence of 2001 tokens, 16 parts an item, takes 11.6 us.  One step of a wave under way instead of two: 59 us and 13.9 us.
#include "qmlp_internal.h"

#include "decode_launch.h"
#include "kv_device.h"
#include "kv_window.h"

namespace qmlp {
namespace {

typedef uint32_t w4 __attribute__((ext_vector_type(4)));
constexpr int kMostParts = 64;
constexpr int kAhead = 8;                                 // parts under way where they are joined
constexpr int kRows = 16, kStep = 128;                    // rows of a tile; tokens of a workgroup's step, 32 a wave

// One tile of 16 tokens as its lanes hold it.
template <int D>
struct Tile {
    uint32_t k[D / 32];                                   // D/4 dims of token lane & 15
    uint4 v;                                              // 8 dims of 4 tokens
    uint4 km, vm;                                         // (scale, zero) of 4 tokens
    uint32_t kz;                                          // and of token lane & 15
};

template <int D>
struct Step {
    Tile<D> tile[2];
    bool hidden[2];                                       // its page is not one of the cache's
};

template <int D>
__device__ __forceinline__ void load_tile(Tile<D>& t, const AttnArgs& a, int pid, int head, int in_page) {
    const uint32_t lane = threadIdx.x & 63, h = lane >> 4, r = lane & 15, side = a.cache.side(D);
    const uint8_t* base = a.cache.at(D, pid, head);
    const uint8_t* codes = base + (uint32_t)in_page * (D / 2);
    const uint8_t* meta = base + ((uint32_t)(D / 2) << a.cache.page_log2) + (uint32_t)in_page * 4u;
    if constexpr (D == 128) {
        const u32x4 k = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(codes + r * 64u + h * 16u));
        t.k[0] = k.x;
        t.k[1] = k.y;
        t.k[2] = k.z;
        t.k[3] = k.w;
    } else {
        const uint2 k = *reinterpret_cast<const uint2*>(codes + r * 32u + h * 8u);
        t.k[0] = k.x;
        t.k[1] = k.y;
    }
    t.v = load_stream(reinterpret_cast<const uint4*>(codes + side + h * (2u * D) + (r & (D / 8 - 1)) * 16u));
    t.km = *reinterpret_cast<const uint4*>(meta + h * 16u);
    t.vm = *reinterpret_cast<const uint4*>(meta + side + h * 16u);
    t.kz = *reinterpret_cast<const uint32_t*>(meta + r * 4u);
}

// (Two workgroups a compute unit: three steps of 32 tokens in registers leave two waves a SIMD.)
// Work is cut evenly over the workgroups (see prefix_work): a unit is one step of one item, an item a tile
// of rows of one K/V head.  A workgroup's range can begin and end inside items; what it has of those goes to the
// workspace, two places a workgroup, and the last to come to an item (a counter at the item's first workgroup) joins
// its parts.
template <int D, typename I>
__global__ void __launch_bounds__(256, 2) few_kernel(AttnArgs a, int limit) {
    constexpr int NT = D / 16, LD = D + 4;                // tiles of outputs; row of LDS
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    float* lo = reinterpret_cast<float*>(smem);           // [4][16][LD]
    __shared__ float lm[4][kRows], ll[4][kRows];
    __shared__ uint32_t arrived;
    __shared__ int longest;
    Known<I>* known = reinterpret_cast<Known<I>*>(smem + 4 * kRows * LD * 4);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 4, col = lane & 15;
    const int lg = a.cache.page_log2, Hk = a.cache.heads;

    auto first_step = [&](const Request& q) { return first_seen(q.len - q.n, a.window) / kStep; };      // of the first row, in steps
    auto tiles_of = [&](const Request& q) {
        const long rows = (long)q.n * a.G;
        return rows > limit ? 0 : (int)((rows + kRows - 1) / kRows);
    };
    auto steps_of = [&](const Request& q) { return max(1, (q.len + kStep - 1) / kStep - first_step(q)); };
    if (tid == 0)
        longest = 0;
    __syncthreads();
    const I total = prefix_work<256, I>(a, known, [&](const Request& q) {
        const int tiles = tiles_of(q), steps = steps_of(q);
        if (tiles && steps > kMostParts)
            atomicMax(&longest, steps);
        return (I)tiles * Hk * steps;
    });
    // (an item in more than 64 parts would take longer to join than to read)
    const I share = max((total + (I)gridDim.x - 1) / (I)gridDim.x, (I)((longest + kMostParts - 1) / kMostParts));
    // workgroups of one XCD take neighbouring ranges
    const int wg = (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3);
    const I begin = wg * share, end = min(begin + share, total);
    I at = begin;
    const uint32_t mv = magic64();

    while (at < end) {
        const int b = __builtin_amdgcn_readfirstlane(request_of(known, a.B, at));
        const Request q = known[b].uniform();
        const I before = known[b].before;
        const int steps = steps_of(q), tiles = tiles_of(q);
        const I item = (at - before) / steps, item0 = before + item * steps;
        const int head = (int)(item / tiles), tile = (int)(item % tiles);
        const int s0 = (int)(at - item0), s1 = (int)min((I)steps, end - item0);
        const int rows = min((int)min((long)q.n * a.G, (long)INT32_MAX) - tile * kRows, kRows);
        const int row = tile * kRows + col, tok = row / a.G;
        const int pos = col < rows ? q.len - q.n + tok : -1;
        const int low = first_seen(pos, a.window);
        // tokens that every row of the tile sees
        const int all_hi = q.len - q.n + tile * kRows / a.G;
        const int all_lo = first_seen(q.len - q.n + (tile * kRows + rows - 1) / a.G, a.window);

        // q as the second operand: lane's row, dims (D/4) h ..
        uint4 qv[D / 32];
        float qsum;
        {
            const uint16_t* src = a.q + (long)(q.row0 + tok) * a.ldq + ((long)head * a.G + row % a.G) * D + h * (D / 4);
#pragma unroll
            for (int i = 0; i < D / 32; ++i)
                qv[i] = col < rows ? reinterpret_cast<const uint4*>(src)[i] : make_uint4(0, 0, 0, 0);
        }
        f32x4_t o[NT], oz = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < NT; ++i)
            o[i] = f32x4_t{0, 0, 0, 0};
        float m = kNone, l = 0.0f;

        const int t0 = (first_step(q) + s0) * kStep + wave * 32;     // this wave's tokens: t0 + 128 i ..
        const int n = s1 - s0;
        // page numbers of 32 steps: lane 2 i + j has that of step i, tile j
        int pages = 0;
        auto load_pages = [&](int i) {
            const int t = t0 + (i + (lane >> 1)) * kStep + (lane & 1) * 16;     // (below 2^30 + 2^13)
            pages = a.table[(long)b * a.W + min(t >> lg, a.W - 1)];
        };
        Step<D> buf[3];                                   // two steps are under way while one is multiplied
        auto load = [&](Step<D>& d, int i) {
            if ((i & 31) == 0)
                load_pages(i);
            const int t = t0 + i * kStep;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int p = __builtin_amdgcn_readlane(pages, 2 * (i & 31) + j);
                d.hidden[j] = (uint32_t)p >= (uint32_t)a.cache.pages;
                load_tile<D>(d.tile[j], a, d.hidden[j] ? 0 : p, head, (t + 16 * j) & ((1 << lg) - 1));
            }
        };
        // (the first steps are under way before q is seen to)
        load(buf[0], 0);
        if (n > 1)
            load(buf[1], 1);
        auto quarters = [](float v) {
            v += __shfl_xor(v, 16, 64);
            return v + __shfl_xor(v, 32, 64);
        };
        float scale = a.scale * operand_rows(qv, a.bf, qsum, quarters, [](uint32_t v) {
            v |= __shfl_xor(v, 16, 64);
            return v | (uint32_t)__shfl_xor((int)v, 32, 64);
        }, [](uint32_t top) {                             // each row a power of its own
            top = max(top, (uint32_t)__shfl_xor((int)top, 16, 64));
            return max(top, (uint32_t)__shfl_xor((int)top, 32, 64));
        });

        // minus the row's sum, in the places of the first quarter
        uint32_t part3[3];
        three_bf16(-qsum, part3);
        const uint4 qz = h == 0 ? make_uint4(part3[0] | part3[1] << 16, part3[2], 0, 0) : make_uint4(0, 0, 0, 0);
        scale = scale == 0.0f ? 1.2e-38f : scale;         // (no score passes 2^-40 with it, and infinity times it is no NaN)
        const float away = scale < 0.0f ? INFINITY : -INFINITY;      // a score that weighs nothing

        auto multiply = [&](const Step<D>& s, int i) {
            const Tile<D>* cur = s.tile;
            const bool hid0 = s.hidden[0], hid1 = s.hidden[1];
            const int t = t0 + i * kStep;
            const bool full = t >= all_lo && t + 31 <= all_hi && !hid0 && !hid1;
            if (full || t < q.len) {
                // scores: tokens 16 j + 4 h + i of row `col`
                float x[8];
                uint32_t zz[4], sv[8];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    // the offset and the zero of a token, times the row's sum: one more step, in bfloat16 (64 + zero is exact there)
                    const uint32_t z = __float_as_uint(fma_hi(cur[j].kz, 1.0f, 64.0f)), zd = __builtin_amdgcn_perm(z, z, 0x03020302u);
                    f32x4_t acc = mfma16_bf(make_uint4(zd, zd, zd, zd), qz, f32x4_t{0, 0, 0, 0});
#pragma unroll
                    for (int w = 0; w < D / 32; ++w) {
                        uint32_t e[4];
                        pairs64(cur[j].k[w], mv, e);
                        acc = mfma16(make_uint4(e[0], e[1], e[2], e[3]), qv[w], acc);
                    }
#pragma unroll
                    for (int i4 = 0; i4 < 4; ++i4) {
                        x[4 * j + i4] = fma_lo(comp(cur[j].km, i4), acc[i4], 0.0f);
                        sv[4 * j + i4] = comp(cur[j].vm, i4);
                    }
                    zz[2 * j] = add2(highs(cur[j].vm.x, cur[j].vm.y), mv);
                    zz[2 * j + 1] = add2(highs(cur[j].vm.z, cur[j].vm.w), mv);
                }
                if (!full) {
                    // what a row does not see weighs nothing, whatever lies there
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const int j = t + (k >> 2) * 16 + 4 * h + (k & 3);
                        const bool there = j < q.len && !(k >> 2 ? hid1 : hid0);
                        if (!(there && j <= pos && j >= low)) {
                            x[k] = away;
                            sv[k] = 0x3C00u;
                        }
                        if (!there)
                            zz[k >> 1] &= k & 1 ? 0x0000FFFFu : 0xFFFF0000u;
                    }
                }
                float w[8], sum, top;
                auto weigh = [&](auto raw) {                  // x as it is, or already times the scale
                    sum = 0.0f;
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const float e = exp2_(decltype(raw)::value ? __builtin_fmaf(x[k], scale, -m) : x[k] - m);
                        w[k] = fma_lo(sv[k], e, 0.0f);
                        sum += e;
                    }
                    top = fmaxf(fmaxf(fmaxf(w[0], w[1]), fmaxf(w[2], w[3])), fmaxf(fmaxf(w[4], w[5]), fmaxf(w[6], w[7])));
                };
                weigh(std::true_type{});
                // (a scale of 0, as in an empty cache, hides a large weight from the first test)
                if (__ballot(top > kTop || sum > 8.0f * kTop * kLeast)) {
                    float best = kNone, most = kNone;
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        x[k] = rounded(x[k] * scale);
                        most = fmaxf(most, x[k]);
                        best = fmaxf(best, x[k] + log2_(fmaxf(h2f(sv[k] & 0xFFFFu), 1.0f / kLeast)));
                    }
                    most = fmaxf(most, __shfl_xor(most, 16, 64));
                    most = fmaxf(most, __shfl_xor(most, 32, 64));
                    best = fmaxf(best, __shfl_xor(best, 16, 64));
                    best = fmaxf(best, __shfl_xor(best, 32, 64));
                    const float mn = shifted(m, most, best), f = exp2_(m - mn);
                    m = mn;
                    l *= f;
                    oz *= f;
#pragma unroll
                    for (int d = 0; d < NT; ++d)
                        o[d] *= f;
                    weigh(std::false_type{});
                }
                l += sum;
                const uint4 p = make_uint4(pack2(w[0], w[1]), pack2(w[2], w[3]), pack2(w[4], w[5]), pack2(w[6], w[7]));
                oz = mfma16(make_uint4(zz[0], zz[1], zz[2], zz[3]), p, oz);
                if constexpr (D == 128) {
                    uint32_t lw[4], hw[4];
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        lw[2 * j] = lows(cur[j].v.x, cur[j].v.y);
                        lw[2 * j + 1] = lows(cur[j].v.z, cur[j].v.w);
                        hw[2 * j] = highs(cur[j].v.x, cur[j].v.y);
                        hw[2 * j + 1] = highs(cur[j].v.z, cur[j].v.w);
                    }
                    uint32_t ea[4][4];
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            pairs64(c ? hw[k] : lw[k], mv, ea[k]);
#pragma unroll
                        for (int f = 0; f < 4; ++f)
                            o[2 * f + c] = mfma16(make_uint4(ea[0][f], ea[1][f], ea[2][f], ea[3][f]), p, o[2 * f + c]);
                    }
                } else {
                    // lanes of the upper eight rows take the odd dims of the same words
                    const uint32_t sel = col & 8 ? 0x07060302u : 0x05040100u;
                    uint32_t ea[4][4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const uint4& v = cur[k >> 1].v;
                        pairs64(k & 1 ? __builtin_amdgcn_perm(v.w, v.z, sel) : __builtin_amdgcn_perm(v.y, v.x, sel), mv, ea[k]);
                    }
#pragma unroll
                    for (int f = 0; f < 4; ++f)
                        o[f] = mfma16(make_uint4(ea[0][f], ea[1][f], ea[2][f], ea[3][f]), p, o[f]);
                }
            }
        };
        for (int i = 0; i < n; i += 3) {
#pragma unroll
            for (int j = 0; j < 3; ++j)
                if (i + j < n) {
                    if (i + j + 2 < n)
                        load(buf[(j + 2) % 3], i + j + 2);
                    multiply(buf[j], i + j);
                }
        }

        // the four waves' parts, by row
        l = quarters(l);
        if (h == 0) {
            lm[wave][col] = m;
            ll[wave][col] = l;
        }
        float* my = lo + (wave * kRows + col) * LD;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = 4 * h + i;
            if constexpr (D == 128) {
                *reinterpret_cast<float4*>(my + 8 * r) = make_float4(o[0][i] - oz[i], o[1][i] - oz[i], o[2][i] - oz[i], o[3][i] - oz[i]);
                *reinterpret_cast<float4*>(my + 8 * r + 4) = make_float4(o[4][i] - oz[i], o[5][i] - oz[i], o[6][i] - oz[i], o[7][i] - oz[i]);
            } else {
#pragma unroll
                for (int f = 0; f < 4; ++f)
                    my[8 * (r & 7) + 2 * f + (r >> 3)] = o[f][i] - oz[i];
            }
        }
        __syncthreads();
        const bool whole = s0 == 0 && s1 == steps;
        const uint32_t place = kRows * (D + 2) * 4u;      // bytes of a part: [16][D], m [16], l [16]
        const uint32_t mine = (uint32_t)(2 * wg + (at == begin ? 0 : 1)) * place;
        const Rsrc rp = rsrc(a.part, 2 * gridDim.x * place);
        for (int c = tid; c < rows * (D / 4); c += 256) {
            const int r = c / (D / 4), d = 4 * (c % (D / 4));
            float mm = lm[0][r];
#pragma unroll
            for (int w = 1; w < 4; ++w)
                mm = fmaxf(mm, lm[w][r]);
            float ls = 0.0f, v[4] = {0, 0, 0, 0};
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float f = exp2_(lm[w][r] - mm);
                const float4 u = *reinterpret_cast<const float4*>(lo + (w * kRows + r) * LD + d);
                ls += f * ll[w][r];
                v[0] += f * u.x;
                v[1] += f * u.y;
                v[2] += f * u.z;
                v[3] += f * u.w;
            }
            if (whole) {
                const int rr = tile * kRows + r, g = head * a.G + rr % a.G;
                const float f = row_factor(a, g, mm, ls);
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    v[k] = ls == 0.0f ? 0.0f : v[k] * f;
                store4(a.y + (long)(q.row0 + rr / a.G) * a.ldy + (long)g * D + d, v, a.bf);
            } else {
                const w4 u = {__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
                __builtin_amdgcn_raw_buffer_store_b128(u, rp, mine + (uint32_t)(r * D + d) * 4u, 0, kDevice);
                if (d == 0) {
                    __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(mm), rp, mine + (uint32_t)(kRows * D + r) * 4u, 0, kDevice);
                    __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(ls), rp, mine + (uint32_t)(kRows * D + kRows + r) * 4u, 0, kDevice);
                }
            }
        }
        if (!whole) {
            // the part is out, then the item's counter: the last to come joins
            const int w0 = (int)(item0 / share), w1 = (int)((item0 + steps - 1) / share);
            __asm__ volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
            if (tid == 0)
                arrived = __hip_atomic_fetch_add(a.done + w0, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            __syncthreads();
            if (arrived == (uint32_t)(w1 - w0)) {
                if (tid == 0)
                    __hip_atomic_store(a.done + w0, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                // (an item begins at its first workgroup's range or inside it; later ones begin with it)
                auto part = [&](int w) { return (uint32_t)(2 * w + (w == w0 && item0 != w0 * share ? 1 : 0)) * place; };
                // each wave joins every fourth part, four numbers a lane, eight parts under way; then the waves meet in LDS
                for (int c0 = 0; c0 < rows * (D / 4); c0 += 64) {
                    const int c = min(c0 + lane, rows * (D / 4) - 1), r = c / (D / 4), d = 4 * (c % (D / 4));
                    float mm = kNone, ls = 0.0f, v[4] = {0, 0, 0, 0};
                    for (int w = w0 + wave; w <= w1; w += 4 * kAhead) {
                        w4 u[kAhead];
                        float pm[kAhead], pl[kAhead];
#pragma unroll
                        for (int k = 0; k < kAhead; ++k) {
                            const uint32_t at0 = part(min(w + 4 * k, w1));
                            u[k] = __builtin_amdgcn_raw_buffer_load_b128(rp, at0 + (uint32_t)(r * D + d) * 4u, 0, kDevice);
                            pm[k] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rp, at0 + (uint32_t)(kRows * D + r) * 4u, 0, kDevice));
                            pl[k] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rp, at0 + (uint32_t)(kRows * D + kRows + r) * 4u, 0, kDevice));
                        }
#pragma unroll
                        for (int k = 0; k < kAhead; ++k)
                            if (w + 4 * k <= w1) {
                                const float mn = fmaxf(mm, pm[k]), f0 = exp2_(mm - mn), f1 = exp2_(pm[k] - mn);
                                mm = mn;
                                ls = ls * f0 + pl[k] * f1;
#pragma unroll
                                for (int x = 0; x < 4; ++x)
                                    v[x] = v[x] * f0 + __uint_as_float(u[k][x]) * f1;
                            }
                    }
                    __syncthreads();                      // the last reads of LDS are over
                    float* my = lo + (wave * 64 + lane) * 8;
                    *reinterpret_cast<float4*>(my) = make_float4(v[0], v[1], v[2], v[3]);
                    *reinterpret_cast<float2*>(my + 4) = make_float2(mm, ls);
                    __syncthreads();
                    if (wave == 0 && c0 + lane < rows * (D / 4)) {
#pragma unroll
                        for (int w = 1; w < 4; ++w) {
                            const float* o = lo + (w * 64 + lane) * 8;
                            const float mn = fmaxf(mm, o[4]), f0 = exp2_(mm - mn), f1 = exp2_(o[4] - mn);
                            mm = mn;
                            ls = ls * f0 + o[5] * f1;
#pragma unroll
                            for (int x = 0; x < 4; ++x)
                                v[x] = v[x] * f0 + o[x] * f1;
                        }
                        const int rr = tile * kRows + r, g = head * a.G + rr % a.G;
                        const float f = row_factor(a, g, mm, ls);
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            v[k] = ls == 0.0f ? 0.0f : v[k] * f;
                        store4(a.y + (long)(q.row0 + rr / a.G) * a.ldy + (long)g * D + d, v, a.bf);
                    }
                }
            }
        }
        __syncthreads();                                  // LDS is the next item's
        at = item0 + s1;
    }
}

constexpr int kPerCu = 2;                                 // workgroups of a compute unit
int few_grid() { return (plan_cus() * kPerCu + 7) / 8 * 8; }

template <int D, typename I>
hipError_t launch_few(const AttnArgs& a, int limit, hipStream_t st) {
    const size_t lds = (size_t)4 * kRows * (D + 4) * 4 + (size_t)a.B * sizeof(Known<I>);
    const hipError_t e = set_lds(few_kernel<D, I>, lds + 1024);
    if (e != hipSuccess)
        return e;
    few_kernel<D, I><<<few_grid(), 256, lds, st>>>(a, limit);
    return hipGetLastError();
}

}  // namespace

// Requests of up to this many rows take the kernel above, those with more the one for many rows (kv_attention_rows.hip).
// 80 rows (5 tokens, 16 heads on one K/V head) of four requests of 30000 tokens: 38 us here, 98 us there, whose tile of 256 rows is
// then a third full and its items few; 20 tokens (80 rows a K/V head) after 15000: 37 and 68 us.  800 rows there: 120 us.
// (Every 16 rows read and unpack the cache again here: both are far from reading it once.)
constexpr int kFewRows = 128;

size_t kv_attention_bytes(int D, int G, int max_new) {
    const size_t few = (size_t)few_grid() * 2 * kRows * (D + 2) * 4, many = (long)max_new * G > kFewRows ? kv_rows_bytes(D) : 0;
    return (few > many ? few : many) + kCounters;
}

hipError_t launch_kv_attention(const AttnArgs& args, int max_new, hipStream_t st) {
    AttnArgs a = args;
    a.part = reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(a.done) + kCounters);
    const bool many = (long)max_new * a.G > kFewRows;
    if (many) {
        const hipError_t e = launch_kv_rows(a, kFewRows, st);
        if (e != hipSuccess)
            return e;
    }
    const int limit = many ? kFewRows : INT32_MAX;
    // the units of all requests at most: 32 bits hold them but for the longest tables with the most rows
    const double units = ((double)a.T * a.G / kRows + a.B) * a.cache.heads * (((double)((long)a.W << a.cache.page_log2)) / kStep + 2);
    const bool wide = units + few_grid() >= 2147483647.0;
    if (a.D == 128)
        return wide ? launch_few<128, int64_t>(a, limit, st) : launch_few<128, int32_t>(a, limit, st);
    return wide ? launch_few<64, int64_t>(a, limit, st) : launch_few<64, int32_t>(a, limit, st);
}

}  // namespace qmlp
