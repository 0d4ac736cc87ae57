// C ABI of the operators that choose weights per token: the linear with
// adapters of many requests, the router and the whole MoE layer.  As in
// api.hip every check runs before the first launch.
#include <stddef.h>
#include <stdint.h>

#include "lora_linear.h"
#include "moe_layer.h"
#include "qmlp.h"
#include "qmlp_internal.h"

namespace {

using namespace qmlp;

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }
inline bool aligned4(const void* p) { return ((uintptr_t)p & 3u) == 0; }
inline size_t round256(size_t v) { return (v + 255) & ~(size_t)255; }
qmlp_status from_hip(hipError_t e) { return e == hipSuccess ? QMLP_OK : QMLP_ERR_HIP; }
// An enumeration's number as a C caller passed it, any at all: to be refused it has to be looked at, and reading a
// number that the enumeration does not have is undefined in C++.
template <typename E>
inline int number(const E& e) {
    static_assert(sizeof(E) == sizeof(int), "an enumeration of the C interface");
    int v;
    __builtin_memcpy(&v, &e, sizeof v);
    return v;
}

// ---------------------------------------------------------------- linear with adapters

constexpr int kMaxRows = 1 << 20, kMaxStride = 1 << 21;    // 256 rows, or a column of 1024, within 32-bit offsets

qmlp_status check_lora(const qmlp_qweight* w, const qmlp_adapters* ad, int M, int dtype) {
    const qmlp_status s = weight_check(w, 0);
    if (s != QMLP_OK)
        return s;
    if (w->bits == 3 || (dtype != QMLP_F16 && dtype != QMLP_BF16))
        return QMLP_ERR_UNSUPPORTED;
    if (w->k_in % 64 != 0 || M < 0)
        return QMLP_ERR_SHAPE;
    if (M > kMaxRows || w->k_in > kMaxStride)
        return QMLP_ERR_UNSUPPORTED;
    if (!ad)
        return QMLP_OK;
    if (ad->count < 0)
        return QMLP_ERR_SHAPE;
    if (ad->count == 0)
        return QMLP_OK;
    if (ad->rank != 8 && ad->rank != 16 && ad->rank != 32 && ad->rank != 64)
        return QMLP_ERR_UNSUPPORTED;
    if (!ad->A || !ad->B)
        return QMLP_ERR_NULL;
    if (!aligned16(ad->A) || !aligned16(ad->B) || !aligned4(ad->scale))
        return QMLP_ERR_ALIGN;
    return QMLP_OK;
}

// Workspace: [t: M x R fp32, or as two bfloat16 terms][adapters of up to 16 rows,
// or sets of rows with several][2^-e: M fp32], then up to 16 rows [x in operand
// order][its group sums], past them [sums of shares of k, fp32] or [terms of
// the rows of those sets, fp32], and for bfloat16 [x 2^e: M x k binary16].
struct LoraSizes {
    size_t t, slots, xf, xo, xs, mixed, parts, x16;
    size_t all() const { return t + slots + xf + xo + xs + mixed + parts + x16; }
};
LoraSizes lora_sizes(const qmlp_qweight* w, const qmlp_adapters* ad, int M, int dtype) {
    const bool bf = dtype == QMLP_BF16, some = ad && ad->count > 0, few = lora_few_rows(M, w);
    LoraSizes z{};
    if (some) {
        z.t = round256((size_t)M * ad->rank * 4);
        z.slots = round256(((size_t)(M + 31) / 32 + kMixedSets) * 4);
    }
    if (bf)
        z.xf = round256((size_t)M * 4);
    if (few) {
        z.xo = round256((size_t)M * operand_row(w->k_in, w->bits) * 2);
        z.xs = round256((size_t)M * operand_sums(w->k_in, w->bits, w->group) * 4);
    } else {
        const int shares = lora_shares(M, w->n_out, w->k_in, plan_cus());
        if (lora_join(M, shares, some))
            z.parts = round256((size_t)shares * M * w->n_out * 4);
        else if (some)
            z.mixed = round256((size_t)lora_mixed_most(M) * 32 * w->n_out * 4);
        if (bf)
            z.x16 = round256((size_t)M * w->k_in * 2);
    }
    return z;
}

// A workspace for any number of rows up to M.  More rows can need less (fewer shares of k, none of them past 512 rows,
// terms of mixed sets instead), but between these numbers the need grows with M.
size_t lora_most_bytes(const qmlp_qweight* w, const qmlp_adapters* ad, int M, int dtype) {
    size_t most = lora_sizes(w, ad, M, dtype).all();
    for (const int m : {kLoraFewTokens, kLoraMidRows, 128, 256, 384, 512})
        if (m < M && lora_sizes(w, ad, m, dtype).all() > most)
            most = lora_sizes(w, ad, m, dtype).all();
    return most;
}

// ---------------------------------------------------------------- router

qmlp_status check_route(int M, int d, int E, int k, int score, int dtype) {
    if (M < 0 || d <= 0 || E < 1 || k < 1 || k > E || d % 8 != 0)
        return QMLP_ERR_SHAPE;
    if (M > kMaxRows || E > kMoeExperts || k > kMoeTopk || d > (1 << 20) || (dtype != QMLP_F16 && dtype != QMLP_BF16) ||
        score < QMLP_SCORE_TOPK_SOFTMAX || score > QMLP_SCORE_SIGMOID)
        return QMLP_ERR_UNSUPPORTED;
    return QMLP_OK;
}
// [logits fp64][norms of the rows of x][of the router's], the norms for many tokens
size_t route_bytes(int M, int E) { return round256((size_t)M * E * 8 + ((size_t)M + E) * 4); }

// ---------------------------------------------------------------- MoE layer

qmlp_status check_moe(const qmlp_moe* l, int M, int dtype) {
    if (!l)
        return QMLP_ERR_NULL;
    const qmlp_mlp& m = l->mlp;
    qmlp_status s;
    if ((s = weight_check(&m.gate, 0)) != QMLP_OK) return s;
    if ((s = weight_check(&m.up, m.gate.bits)) != QMLP_OK) return s;
    if ((s = weight_check(&m.down, 0)) != QMLP_OK) return s;
    const int E = l->experts, d = m.gate.k_in, f = m.down.k_in;
    if ((s = check_route(M, d, E, l->topk, l->score, dtype)) != QMLP_OK) return s;
    if (m.gate.bits == 3 || m.down.bits == 3 || dtype != QMLP_F16 || M > kMoeTokens)
        return QMLP_ERR_UNSUPPORTED;
    if ((long)E * f != m.gate.n_out || m.up.n_out != m.gate.n_out || m.up.k_in != d || (long)E * d != m.down.n_out ||
        m.up.group != m.gate.group || d % 64 != 0 || f % 64 != 0)
        return QMLP_ERR_SHAPE;
    if (m.rank != 0 && m.rank != 8 && m.rank != 16 && m.rank != 32)
        return QMLP_ERR_UNSUPPORTED;
    // one expert's arrays, and the instances' rows, take 32-bit offsets
    const long most = 1l << 31, w = (long)d * f;
    if (w * m.gate.bits / 8 >= most || w * m.down.bits / 8 >= most || w / m.gate.group * 4 >= most ||
        w / m.down.group * 4 >= most || (long)kMoeTokens * kMoeTopk * 2 * (d > f ? d : f) >= most)
        return QMLP_ERR_UNSUPPORTED;
    if (!l->router)
        return QMLP_ERR_NULL;
    if (!aligned16(l->router) || !aligned4(l->bias))
        return QMLP_ERR_ALIGN;
    if (m.rank > 0) {
        if (!m.A_gate || !m.B_gate || !m.A_up || !m.B_up)
            return QMLP_ERR_NULL;
        if (!aligned16(m.A_gate) || !aligned16(m.B_gate) || !aligned16(m.A_up) || !aligned16(m.B_up))
            return QMLP_ERR_ALIGN;
    }
    return QMLP_OK;
}

// Workspace: [logits fp64][expert of a slot][its weight][blocks][t][h][outputs of
// the instances, fp32][x in operand order][its group sums].
struct MoeSizes {
    size_t logits, idx, w, blocks, t, h, part, xo, xs;
    size_t all() const { return logits + idx + w + blocks + t + h + part + xo + xs; }
};
MoeSizes moe_sizes(const qmlp_moe* l, int M) {
    const size_t n = (size_t)M * l->topk;
    return {route_bytes(M, l->experts), round256(n * 4), round256(n * 4),
            round256((size_t)(1 + moe_blocks_most((int)n, l->experts)) * kBlkInts * 4),
            round256(n * 2 * l->mlp.rank * 4), round256(n * operand_row(l->mlp.down.k_in, l->mlp.down.bits) * 2), round256(n * l->mlp.gate.k_in * 4),
            round256((size_t)M * operand_row(l->mlp.gate.k_in, l->mlp.gate.bits) * 2),
            round256((size_t)M * operand_sums(l->mlp.gate.k_in, l->mlp.gate.bits, l->mlp.gate.group) * 4)};
}

}  // namespace

extern "C" {

size_t qmlp_linear_lora_workspace_bytes(const qmlp_qweight* w, const qmlp_adapters* ad, int M, qmlp_dtype dtype) {
    if (check_lora(w, ad, M, number(dtype)) != QMLP_OK)
        return 0;
    return lora_most_bytes(w, ad, M, number(dtype));
}

qmlp_status qmlp_linear_lora(const qmlp_qweight* w, const qmlp_adapters* ad, const int32_t* ids, const void* x,
                             int64_t ldx, int M, qmlp_dtype dtype, void* y, int64_t ldy, void* ws, size_t ws_bytes,
                             qmlp_stream stream) {
    const qmlp_status s = check_lora(w, ad, M, number(dtype));
    if (s != QMLP_OK)
        return s;
    if (M == 0)
        return QMLP_OK;
    const bool adapters = ad && ad->count > 0;
    if (!x || !y || (adapters && !ids))
        return QMLP_ERR_NULL;
    if (ldx < w->k_in || ldx % 8 != 0 || ldy < w->n_out)
        return QMLP_ERR_SHAPE;
    if (ldx > kMaxStride)
        return QMLP_ERR_UNSUPPORTED;
    if (!aligned16(x) || ((uintptr_t)y & 1u) != 0 || (adapters && !aligned4(ids)))
        return QMLP_ERR_ALIGN;
    const LoraSizes z = lora_sizes(w, ad, M, dtype);
    if (z.all() > 0 && (!ws || ws_bytes < z.all()))
        return QMLP_ERR_WORKSPACE;
    if (!aligned16(ws))
        return QMLP_ERR_ALIGN;
    char* base = static_cast<char*>(ws);
    LoraArgs a{};
    a.codes = static_cast<const uint32_t*>(w->codes);
    a.meta = static_cast<const uint32_t*>(w->meta);
    a.x = static_cast<const uint16_t*>(x);
    a.y = static_cast<uint16_t*>(y);
    if (adapters) {
        a.A = static_cast<const uint16_t*>(ad->A);
        a.B = static_cast<const uint16_t*>(ad->B);
        a.scale = ad->scale;
        a.ids = ids;
        a.T = ad->count;
        a.R = ad->rank;
    }
    a.ldx = ldx;
    a.ldy = ldy;
    a.M = M;
    a.n = w->n_out;
    a.k = w->k_in;
    a.bits = w->bits;
    a.g = w->group;
    a.bf = dtype == QMLP_BF16;
    a.cus = plan_cus();
    a.shares = lora_shares(M, a.n, a.k, a.cus);
    const bool few = lora_few_rows(M, w);
    const auto take = [&](size_t bytes) {
        char* at = base;
        base += bytes;
        return at;
    };
    char* t = take(z.t);
    a.t = few ? reinterpret_cast<float*>(t) : nullptr;
    a.tb = few ? nullptr : reinterpret_cast<uint16_t*>(t);
    a.slots = a.known = reinterpret_cast<int*>(take(z.slots));
    a.xf = reinterpret_cast<float*>(take(z.xf));
    a.xo = few ? reinterpret_cast<uint16_t*>(take(z.xo)) : nullptr;
    a.xs = reinterpret_cast<float*>(take(z.xs));
    a.mixed = reinterpret_cast<float*>(take(z.mixed));
    a.parts = z.parts ? reinterpret_cast<float*>(take(z.parts)) : nullptr;
    a.x16 = z.x16 ? reinterpret_cast<uint16_t*>(take(z.x16)) : nullptr;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    hipError_t e = launch_lora_prep(a, st);
    if (e == hipSuccess && !few && adapters && !a.parts)
        e = launch_lora_mixed(a, st);
    if (e != hipSuccess)
        return QMLP_ERR_HIP;
    e = few ? launch_lora_few(a, st) : launch_lora_gemm(a, st);
    return from_hip(e == hipSuccess && a.parts ? launch_lora_join(a, st) : e);
}

size_t qmlp_moe_route_workspace_bytes(int E, int M) {
    return M < 0 || M > kMaxRows || E < 1 || E > kMoeExperts ? 0 : route_bytes(M, E);
}

qmlp_status qmlp_moe_route(const void* router, const float* bias, const void* x, int M, int d, int E, int k,
                           qmlp_score score, qmlp_dtype dtype, int32_t* topk_idx, float* topk_w, void* ws,
                           size_t ws_bytes, qmlp_stream stream) {
    const qmlp_status s = check_route(M, d, E, k, number(score), number(dtype));
    if (s != QMLP_OK)
        return s;
    if (M == 0)
        return QMLP_OK;
    if (!router || !x || !topk_idx || !topk_w)
        return QMLP_ERR_NULL;
    if (!aligned16(router) || !aligned16(x) || !aligned4(bias) || !aligned4(topk_idx) || !aligned4(topk_w) || !aligned16(ws))
        return QMLP_ERR_ALIGN;
    if (!ws || ws_bytes < route_bytes(M, E))
        return QMLP_ERR_WORKSPACE;
    float* norms = reinterpret_cast<float*>(static_cast<double*>(ws) + (size_t)M * E);
    const RouteArgs a{static_cast<const uint16_t*>(x), static_cast<const uint16_t*>(router), bias, topk_idx, topk_w,
                      static_cast<double*>(ws), norms, norms + M, M, d, E, k, score, dtype == QMLP_BF16};
    return from_hip(launch_route(a, static_cast<hipStream_t>(stream)));
}

size_t qmlp_moe_layer_workspace_bytes(const qmlp_moe* layer, int M, qmlp_dtype dtype) {
    return check_moe(layer, M, number(dtype)) != QMLP_OK ? 0 : moe_sizes(layer, M).all();
}

qmlp_status qmlp_moe_layer(const qmlp_moe* layer, const void* x, int M, qmlp_dtype dtype, void* y, void* ws,
                           size_t ws_bytes, qmlp_stream stream) {
    const qmlp_status s = check_moe(layer, M, number(dtype));
    if (s != QMLP_OK)
        return s;
    if (M == 0)
        return QMLP_OK;
    if (!x || !y)
        return QMLP_ERR_NULL;
    if (!aligned16(x) || !aligned16(y) || !aligned16(ws))
        return QMLP_ERR_ALIGN;
    const MoeSizes z = moe_sizes(layer, M);
    if (!ws || ws_bytes < z.all())
        return QMLP_ERR_WORKSPACE;
    const qmlp_mlp& m = layer->mlp;
    char* p = static_cast<char*>(ws);
    const auto take = [&](size_t bytes) {
        char* at = p;
        p += bytes;
        return at;
    };
    RouteArgs r{};
    r.logits = reinterpret_cast<double*>(take(z.logits));
    r.idx = reinterpret_cast<int32_t*>(take(z.idx));
    r.w = reinterpret_cast<float*>(take(z.w));
    r.x = static_cast<const uint16_t*>(x);
    r.router = static_cast<const uint16_t*>(layer->router);
    r.bias = layer->bias;
    r.M = M;
    r.d = m.gate.k_in;
    r.E = layer->experts;
    r.k = layer->topk;
    r.score = layer->score;
    MoeArgs a{};
    a.cg = static_cast<const uint32_t*>(m.gate.codes);
    a.mg = static_cast<const uint32_t*>(m.gate.meta);
    a.cu = static_cast<const uint32_t*>(m.up.codes);
    a.mu = static_cast<const uint32_t*>(m.up.meta);
    a.cd = static_cast<const uint32_t*>(m.down.codes);
    a.md = static_cast<const uint32_t*>(m.down.meta);
    a.Ag = static_cast<const uint16_t*>(m.A_gate);
    a.Bg = static_cast<const uint16_t*>(m.B_gate);
    a.Au = static_cast<const uint16_t*>(m.A_up);
    a.Bu = static_cast<const uint16_t*>(m.B_up);
    a.x = r.x;
    a.y = static_cast<uint16_t*>(y);
    a.idx = r.idx;
    a.w = r.w;
    a.logits = r.logits;
    a.score = r.score;
    a.blocks = reinterpret_cast<int*>(take(z.blocks));
    a.t = reinterpret_cast<float*>(take(z.t));
    a.h = reinterpret_cast<uint16_t*>(take(z.h));
    a.part = reinterpret_cast<float*>(take(z.part));
    a.xo = reinterpret_cast<uint16_t*>(take(z.xo));
    a.xs = reinterpret_cast<float*>(take(z.xs));
    a.M = M;
    a.d = r.d;
    a.f = m.down.k_in;
    a.r = m.rank;
    a.E = r.E;
    a.k = r.k;
    a.gb = m.gate.bits;
    a.gg = m.gate.group;
    a.db = m.down.bits;
    a.dg = m.down.group;
    a.lora_scale = m.lora_scale;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const hipError_t e = launch_route_logits(r, st);
    return from_hip(e != hipSuccess ? e : launch_moe_experts(a, st));
}

}  // extern "C"
