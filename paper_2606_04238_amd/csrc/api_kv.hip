// C ABI of the operators over the 4-bit cache of keys and values.  As in
// api.hip every check runs before the first launch.
#include <math.h>
#include <stddef.h>
#include <stdint.h>

#include "kv_cache.h"
#include "qmlp.h"
#include "qmlp_internal.h"

namespace {

using namespace qmlp;

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }
inline bool aligned4(const void* p) { return ((uintptr_t)p & 3u) == 0; }
qmlp_status from_hip(hipError_t e) { return e == hipSuccess ? QMLP_OK : QMLP_ERR_HIP; }
// An enumeration's number as a C caller passed it (reading one that it does not have is undefined in C++).
template <typename E>
inline int number(const E& e) {
    static_assert(sizeof(E) == sizeof(int), "an enumeration of the C interface");
    int v;
    __builtin_memcpy(&v, &e, sizeof v);
    return v;
}

constexpr int kMaxRows = 1 << 20, kMaxHeads = 1 << 12;
constexpr int64_t kMaxStride = 1ll << 31;

bool page_ok(int page) { return page == 16 || page == 32 || page == 64 || page == 128 || page == 256; }
bool dim_ok(int d) { return d == 64 || d == 128; }
int log2_of(int page) { return __builtin_ctz((unsigned)page); }

qmlp_status check_cache_sizes(int pages, int heads, int dim, int page) {
    if (!dim_ok(dim) || !page_ok(page))
        return QMLP_ERR_UNSUPPORTED;
    if (pages < 1 || heads < 1)
        return QMLP_ERR_SHAPE;
    if (heads > kMaxHeads || (int64_t)pages * page >= (1ll << 31))
        return QMLP_ERR_UNSUPPORTED;
    return QMLP_OK;
}

qmlp_status check_cache(const qmlp_kv_cache* c) {
    if (!c)
        return QMLP_ERR_NULL;
    const qmlp_status s = check_cache_sizes(c->pages, c->kv_heads, c->head_dim, c->page);
    if (s != QMLP_OK)
        return s;
    if (!c->data)
        return QMLP_ERR_NULL;
    return aligned16(c->data) ? QMLP_OK : QMLP_ERR_ALIGN;
}

KvView view(const qmlp_kv_cache* c) {
    return KvView{static_cast<uint8_t*>(c->data), c->pages, c->kv_heads, log2_of(c->page)};
}

// Rows of `heads` heads, ld elements apart.
qmlp_status check_rows(const void* p, int64_t ld, int heads, int dim, int T) {
    if (!p)
        return QMLP_ERR_NULL;
    if ((T > 1 && ld < (int64_t)heads * dim) || ld < 0 || ld % 8 != 0)
        return QMLP_ERR_SHAPE;
    if (ld > kMaxStride)
        return QMLP_ERR_UNSUPPORTED;
    return aligned16(p) ? QMLP_OK : QMLP_ERR_ALIGN;
}

qmlp_status check_tokens(int T, int dtype) {
    if (T < 0)
        return QMLP_ERR_SHAPE;
    return T > kMaxRows || (dtype != QMLP_F16 && dtype != QMLP_BF16) ? QMLP_ERR_UNSUPPORTED : QMLP_OK;
}

}  // namespace

extern "C" {

size_t qmlp_kv_cache_bytes(int pages, int kv_heads, int head_dim, int page) {
    if (check_cache_sizes(pages, kv_heads, head_dim, page) != QMLP_OK)
        return 0;
    return (size_t)pages * kv_heads * 2 * page * (head_dim / 2 + 4);
}

qmlp_status qmlp_kv_plan(const qmlp_plan* p, qmlp_stream stream) {
    if (!p)
        return QMLP_ERR_NULL;
    if (!page_ok(p->page))
        return QMLP_ERR_UNSUPPORTED;
    if (p->B < 0 || p->W < 1 || p->N < 0 || p->tokens < 0)
        return QMLP_ERR_SHAPE;
    if (p->B > kKvRequests || p->W > (1 << 20) || (int64_t)p->W * p->page > (1ll << 30) || p->tokens > (1 << 24))
        return QMLP_ERR_UNSUPPORTED;
    if (p->B == 0)
        return QMLP_OK;
    if (!p->lens || !p->new_tokens || !p->table || !p->n_free || !p->starts || !p->lens_out || !p->n_free_out ||
        !p->short_out || (p->N > 0 && !p->free_pages) || (p->tokens > 0 && (!p->slots || !p->positions)))
        return QMLP_ERR_NULL;
    for (const int32_t* v : {p->lens, p->new_tokens, (const int32_t*)p->table, (const int32_t*)p->free_pages, p->n_free,
                             (const int32_t*)p->slots, (const int32_t*)p->positions, (const int32_t*)p->starts,
                             (const int32_t*)p->lens_out, (const int32_t*)p->n_free_out, (const int32_t*)p->short_out})
        if (!aligned4(v))
            return QMLP_ERR_ALIGN;
    const PlanArgs a{p->lens, p->new_tokens, p->n_free, p->table, p->free_pages, p->slots, p->positions, p->starts,
                     p->lens_out, p->n_free_out, p->short_out, p->B, log2_of(p->page), p->W, p->N, p->tokens};
    return from_hip(launch_kv_plan(a, static_cast<hipStream_t>(stream)));
}

qmlp_status qmlp_qk_norm_rope(const qmlp_heads* h, int T, qmlp_dtype dtype, const qmlp_kv_cache* cache,
                              qmlp_stream stream) {
    if (!h)
        return QMLP_ERR_NULL;
    const int dt = number(dtype);
    qmlp_status s = check_tokens(T, dt);
    if (s != QMLP_OK)
        return s;
    if (!dim_ok(h->head_dim) || h->heads > kMaxHeads || h->kv_heads > kMaxHeads ||
        (h->pairs != QMLP_PAIRS_HALF && h->pairs != QMLP_PAIRS_NEXT))
        return QMLP_ERR_UNSUPPORTED;
    if (h->heads < 0 || h->kv_heads < 0 || h->heads + h->kv_heads == 0)
        return QMLP_ERR_SHAPE;
    if (h->inv_freq && (h->rot < 16 || h->rot > h->head_dim || h->rot % 16 != 0))
        return QMLP_ERR_SHAPE;
    if (!(h->eps >= 0.0f) || !isfinite(h->eps) || !isfinite(h->mul))
        return QMLP_ERR_UNSUPPORTED;
    if (cache) {
        if ((s = check_cache(cache)) != QMLP_OK)
            return s;
        if (cache->kv_heads != h->kv_heads || cache->head_dim != h->head_dim)
            return QMLP_ERR_SHAPE;
    }
    if (T == 0)
        return QMLP_OK;
    if (h->heads) {
        if ((s = check_rows(h->q, h->ldq, h->heads, h->head_dim, T)) != QMLP_OK) return s;
        if ((s = check_rows(h->q_out, h->ldq_out, h->heads, h->head_dim, T)) != QMLP_OK) return s;
    }
    if (h->kv_heads) {
        if ((s = check_rows(h->k, h->ldk, h->kv_heads, h->head_dim, T)) != QMLP_OK) return s;
        if (h->k_out && (s = check_rows(h->k_out, h->ldk_out, h->kv_heads, h->head_dim, T)) != QMLP_OK) return s;
        if (!cache && !h->k_out)
            return QMLP_ERR_NULL;
    }
    if (cache) {
        if ((s = check_rows(h->v, h->ldv, h->kv_heads, h->head_dim, T)) != QMLP_OK) return s;
        if (!h->slots)
            return QMLP_ERR_NULL;
    }
    if (h->inv_freq && !h->positions)
        return QMLP_ERR_NULL;
    if (!aligned16(h->q_weight) || !aligned16(h->k_weight) || !aligned4(h->positions) || !aligned4(h->inv_freq) ||
        !aligned4(h->slots))
        return QMLP_ERR_ALIGN;
    HeadsArgs a{};
    a.q = static_cast<const uint16_t*>(h->q);
    a.k = h->kv_heads ? static_cast<const uint16_t*>(h->k) : nullptr;
    a.v = static_cast<const uint16_t*>(h->v);
    a.q_out = static_cast<uint16_t*>(h->q_out);
    a.k_out = static_cast<uint16_t*>(h->k_out);
    a.qw = static_cast<const uint16_t*>(h->q_weight);
    a.kw = static_cast<const uint16_t*>(h->k_weight);
    a.pos = h->positions;
    a.slots = h->slots;
    a.inv = h->inv_freq;
    a.ldq = h->ldq; a.ldk = h->ldk; a.ldv = h->ldv; a.ldqo = h->ldq_out; a.ldko = h->ldk_out;
    if (cache)
        a.cache = view(cache);
    a.T = T; a.Hq = h->heads; a.Hk = h->kv_heads; a.D = h->head_dim; a.rot = h->rot;
    a.next = h->pairs == QMLP_PAIRS_NEXT; a.bf = dt == QMLP_BF16; a.eps = h->eps; a.mul = h->mul;
    return from_hip(launch_qk_norm_rope(a, static_cast<hipStream_t>(stream)));
}

qmlp_status qmlp_kv_read(const qmlp_kv_cache* cache, const int32_t* slots, int T, qmlp_dtype dtype, void* k, void* v,
                         qmlp_stream stream) {
    const int dt = number(dtype);
    qmlp_status s = check_tokens(T, dt);
    if (s != QMLP_OK)
        return s;
    if ((s = check_cache(cache)) != QMLP_OK)
        return s;
    if ((int64_t)T * cache->kv_heads > (1ll << 27))        // threads of a launch stay within 32 bits
        return QMLP_ERR_UNSUPPORTED;
    if (T == 0)
        return QMLP_OK;
    if (!slots || (!k && !v))
        return QMLP_ERR_NULL;
    if (!aligned4(slots) || !aligned16(k) || !aligned16(v))
        return QMLP_ERR_ALIGN;
    return from_hip(launch_kv_read(view(cache), cache->head_dim, slots, T, dt == QMLP_BF16, static_cast<uint16_t*>(k),
                                   static_cast<uint16_t*>(v), static_cast<hipStream_t>(stream)));
}

static qmlp_status check_attention(const qmlp_kv_cache* c, int heads, int max_new) {
    const qmlp_status s = check_cache(c);
    if (s != QMLP_OK)
        return s;
    if (heads < 1 || heads % c->kv_heads != 0 || max_new < 0)
        return QMLP_ERR_SHAPE;
    return heads > kMaxHeads || max_new > kMaxRows ? QMLP_ERR_UNSUPPORTED : QMLP_OK;
}

size_t qmlp_kv_attention_workspace_bytes(const qmlp_kv_cache* cache, int heads, int max_new) {
    if (check_attention(cache, heads, max_new) != QMLP_OK)
        return 0;
    return kv_attention_bytes(cache->head_dim, heads / cache->kv_heads, max_new);
}

qmlp_status qmlp_kv_attention(const qmlp_kv_cache* cache, const qmlp_attention* p, qmlp_dtype dtype, qmlp_stream stream) {
    if (!p)
        return QMLP_ERR_NULL;
    const int dt = number(dtype);
    qmlp_status s = check_tokens(p->T, dt);
    if (s != QMLP_OK)
        return s;
    if ((s = check_attention(cache, p->heads, p->max_new)) != QMLP_OK)
        return s;
    if (p->B < 0 || p->W < 1 || p->window < 0 || (!p->starts && p->T != p->B))
        return QMLP_ERR_SHAPE;
    if (p->B > kKvRequests || (int64_t)p->W * cache->page > (1ll << 30) || !isfinite(p->scale))
        return QMLP_ERR_UNSUPPORTED;
    if (p->T == 0 || p->B == 0)
        return QMLP_OK;
    if (!p->table || !p->lens)
        return QMLP_ERR_NULL;
    if ((s = check_rows(p->q, p->ldq, p->heads, cache->head_dim, p->T)) != QMLP_OK)
        return s;
    if ((s = check_rows(p->y, p->ldy, p->heads, cache->head_dim, p->T)) != QMLP_OK)
        return s;
    if (!aligned4(p->table) || !aligned4(p->lens) || !aligned4(p->starts) || !aligned4(p->sinks))
        return QMLP_ERR_ALIGN;
    const int G = p->heads / cache->kv_heads;
    if (!p->ws || p->ws_bytes < kv_attention_bytes(cache->head_dim, G, p->max_new))
        return QMLP_ERR_WORKSPACE;
    if (!aligned16(p->ws))
        return QMLP_ERR_ALIGN;
    AttnArgs a{};
    a.cache = view(cache);
    a.q = static_cast<const uint16_t*>(p->q);
    a.y = static_cast<uint16_t*>(p->y);
    a.table = p->table; a.lens = p->lens; a.starts = p->starts; a.sinks = p->sinks;
    a.ldq = p->ldq; a.ldy = p->ldy;
    a.done = static_cast<uint32_t*>(p->ws);
    a.T = p->T; a.B = p->B; a.W = p->W; a.Hq = p->heads; a.G = G; a.D = cache->head_dim; a.bf = dt == QMLP_BF16;
    a.window = p->window;
    a.scale = (float)((double)p->scale * 1.4426950408889634);
    return from_hip(launch_kv_attention(a, p->max_new, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
