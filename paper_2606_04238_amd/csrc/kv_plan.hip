// The pages of a step's tokens: what ended requests give back, what growing ones
// take, and the slot of every token (gfx950).
//
// A few thousand integers, so what it costs is the launch and the chain of
// dependent loads: one workgroup holds the requests' prefix sums in LDS (pages
// given back, new tokens, pages wanted) and then goes through pages and tokens,
// each finding its request by a binary search.  More workgroups would have to wait for
// one another, since lens and n_free may be overwritten in place.  8 requests with a token each take 3.7 us, 256 requests,
// 9 of them prompts, with 8192 slots 14 us: there a thread has eight tokens, and each waits for the one before it (a search in LDS,
// a load of the table, two stores, which the next load may not pass).
#include "kv_cache.h"
#include "qmlp_device.h"

namespace qmlp {
namespace {

constexpr int kPer = kKvRequests / 1024;                  // requests of a thread at most

// Exclusive sums over the workgroup's threads of v; the total goes to *all.
template <int NT>
__device__ __forceinline__ int64_t block_sum(int64_t v, int64_t* wsum, int64_t* all) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t inc = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int64_t o = __shfl_up(inc, d, 64);
        inc += lane >= d ? o : 0;
    }
    __syncthreads();                                      // wsum may still be read from the sum before
    if (lane == 63)
        wsum[wave] = inc;
    __syncthreads();
    int64_t before = 0, total = 0;
#pragma unroll
    for (int i = 0; i < NT / 64; ++i) {
        before += i < wave ? wsum[i] : 0;
        total += wsum[i];
    }
    *all = total;
    return before + inc - v;
}

// The last b in [0, B) with sums[b] <= i (sums rise from sums[0] = 0).
__device__ __forceinline__ int find(const int32_t* sums, int B, int i) {
    int lo = 0, hi = B;
    while (hi - lo > 1) {
        const int m = (lo + hi) >> 1;
        if (sums[m] <= i)
            lo = m;
        else
            hi = m;
    }
    return lo;
}

template <int NT>
__global__ void __launch_bounds__(NT) kv_plan_kernel(PlanArgs a) {
    __shared__ int32_t len[kKvRequests], begin[kKvRequests + 1], sums[kKvRequests + 1];
    __shared__ uint8_t served[kKvRequests];
    __shared__ int64_t wsum[NT / 64];
    __shared__ int refused, top;
    const int tid = threadIdx.x, lg = a.page_log2, page = 1 << lg;
    const int most = a.W << lg;
    const int per = (a.B + NT - 1) / NT, b0 = tid * per;
    if (tid == 0) {
        refused = 0;
        top = 0;
    }
    const int n_free = min(max(a.n_free[0], 0), a.N);
    int32_t l[kPer], add[kPer], used[kPer];
    int64_t back = 0, fresh = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        l[i] = add[i] = used[i] = 0;
        if (i < per && b0 + i < a.B) {
            l[i] = min(max(a.lens[b0 + i], 0), most);
            add[i] = a.add[b0 + i];
            used[i] = (l[i] + page - 1) >> lg;
            back += add[i] < 0 ? used[i] : 0;
            fresh += max(add[i], 0);
        }
    }
    int64_t backs, tokens;
    int64_t at = block_sum<NT>(back, wsum, &backs), first = block_sum<NT>(fresh, wsum, &tokens);
    backs = min(backs, (int64_t)(a.N - n_free));          // what would pass the stack's end is dropped
    const int have = n_free + (int)backs;
    int64_t want = 0, need[kPer];
    bool fits[kPer];
    int64_t f = first;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        need[i] = 0;
        fits[i] = false;
        if (i < per && b0 + i < a.B) {
            const int64_t n = max(add[i], 0);
            len[b0 + i] = l[i];
            begin[b0 + i] = (int)min(f, (int64_t)INT32_MAX);
            sums[b0 + i] = (int)min(at, (int64_t)INT32_MAX);
            at += add[i] < 0 ? used[i] : 0;
            f += n;
            fits[i] = add[i] >= 0 && l[i] + n <= most && f <= a.T;
            need[i] = fits[i] ? max((int64_t)0, ((l[i] + n + page - 1) >> lg) - used[i]) : 0;
            want += need[i];
        }
    }
    int64_t wants;
    int64_t p = block_sum<NT>(want, wsum, &wants);        // (its barriers also publish len, begin and sums)
    for (int j = tid; j < (int)backs; j += NT) {
        const int b = find(sums, a.B, j);
        a.free_pages[n_free + j] = a.table[(long)b * a.W + j - sums[b]];
    }
    __syncthreads();                                      // the stack is whole, and sums free for the next ones
#pragma unroll
    for (int i = 0; i < kPer; ++i)
        if (i < per && b0 + i < a.B) {
            const int b = b0 + i;
            sums[b] = (int)min(p, (int64_t)INT32_MAX);
            p += need[i];
            const bool ok = fits[i] && (need[i] == 0 || p <= have);
            served[b] = ok;
            if (ok && need[i])
                atomicMax(&top, (int)p);
            if (!ok && add[i] > 0)
                atomicAdd(&refused, 1);
            a.starts[b] = begin[b];
            a.lens_out[b] = add[i] < 0 ? 0 : ok ? l[i] + add[i] : l[i];
        }
    if (tid == 0) {
        begin[a.B] = (int)min(tokens, (int64_t)INT32_MAX);
        a.starts[a.B] = begin[a.B];
    }
    __syncthreads();
    const int taken = top;
    if (tid == 0) {
        a.n_free_out[0] = have - taken;
        a.short_out[0] = refused;
    }
    for (int j = tid; j < taken; j += NT) {
        const int b = find(sums, a.B, j);
        a.table[(long)b * a.W + ((len[b] + page - 1) >> lg) + j - sums[b]] = a.free_pages[have - 1 - j];
    }
    __syncthreads();
    const int all = min(begin[a.B], a.T);
    for (int i = tid; i < a.T; i += NT) {
        int pos = 0, slot = -1;
        if (i < all) {
            const int b = find(begin, a.B, i);
            const int64_t at64 = (int64_t)len[b] + i - begin[b];
            pos = (int)min(at64, (int64_t)INT32_MAX);
            if (served[b]) {
                const int p = a.table[(long)b * a.W + (pos >> lg)];
                if (p >= 0 && p <= INT32_MAX >> lg)       // (another one's slots are not numbers of 31 bits)
                    slot = (p << lg) | (pos & (page - 1));
            }
        }
        a.slots[i] = slot;
        a.positions[i] = pos;
    }
}

}  // namespace

hipError_t launch_kv_plan(const PlanArgs& a, hipStream_t st) {
    // small steps: four waves meet sooner than sixteen, long ones have turns to share (us in a row of replays, 256 and 1024 threads:
    // 8 requests, 8 tokens 3.4 and 5.6, 1024 tokens 5.4 and 6.1; 256 requests, 1024 tokens 7.5 and 7.1, 2048 11.2 and 8.5)
    if (a.B <= 256 && a.T <= 1024)
        kv_plan_kernel<256><<<1, 256, 0, st>>>(a);
    else
        kv_plan_kernel<1024><<<1, 1024, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace qmlp
