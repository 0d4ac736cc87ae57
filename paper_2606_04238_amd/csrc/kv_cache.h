// Argument blocks and launchers of the 4-bit cache of keys and values
// (kv_plan.hip, kv_write.hip, kv_attention.hip), and its addresses.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "qmlp.h"

namespace qmlp {

constexpr int kKvRequests = 2048;            // most requests of a call: their sums are kept in LDS

// A cache as the kernels see it.  `side` bytes hold one page of one head's K or V.
struct KvView {
    uint8_t* data;
    int pages, heads, page_log2;
    __host__ __device__ uint32_t side(int D) const { return (uint32_t)(D / 2 + 4) << page_log2; }
    // K of head h in page p; its V is side(D) further on
    __host__ __device__ uint8_t* at(int D, int p, int h) const {
        return data + ((size_t)p * heads + h) * (2 * (size_t)side(D));
    }
};

struct PlanArgs {
    const int32_t *lens, *add, *n_free;
    int32_t *table, *free_pages;
    int32_t *slots, *positions, *starts, *lens_out, *n_free_out, *short_out;
    int B, page_log2, W, N, T;
};
hipError_t launch_kv_plan(const PlanArgs& a, hipStream_t st);

struct HeadsArgs {
    const uint16_t *q, *k, *v;
    uint16_t *q_out, *k_out;                 // or null
    const uint16_t *qw, *kw;                 // or null
    const int32_t *pos, *slots;
    const float* inv;                        // or null
    long ldq, ldk, ldv, ldqo, ldko;
    KvView cache;                            // data null: none
    int T, Hq, Hk, D, rot, next, bf;
    float eps, mul;
};
hipError_t launch_qk_norm_rope(const HeadsArgs& a, hipStream_t st);
hipError_t launch_kv_read(const KvView& c, int D, const int32_t* slots, int T, int bf, uint16_t* k, uint16_t* v,
                          hipStream_t st);

struct AttnArgs {
    KvView cache;
    const uint16_t* q;
    uint16_t* y;
    const int32_t *table, *lens, *starts;    // starts null: one row a request
    const float* sinks;                      // or null
    long ldq, ldy;
    float* part;                             // workspace behind the counters
    uint32_t* done;                          // counters, zero between calls
    int T, B, W, Hq, G, D, bf, window;
    float scale;                             // times log2(e): scores are powers of two
};
constexpr size_t kCounters = 16384;           // bytes of counters at the workspace's start
size_t kv_attention_bytes(int D, int G, int max_new);
// The kernel for many rows: requests of more than `limit` rows; its part of the workspace.
hipError_t launch_kv_rows(const AttnArgs& a, int limit, hipStream_t st);
size_t kv_rows_bytes(int D);
hipError_t launch_kv_attention(const AttnArgs& a, int max_new, hipStream_t st);

}  // namespace qmlp
