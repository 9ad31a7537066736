// slot_map.cu -- block tables, slot maps and positions of one serving step,
// built on the GPU from the requests' lengths (rfq_slot_map).
//
// Mathematics: three exclusive prefix sums over the requests (pages given
// back, pages wanted, tokens added).  A page given back goes on top of the
// stack of free pages at count + its prefix; the n-th wanted page is the n-th
// from the stack's top after that; a token finds its request by a binary
// search in the token prefix.  Every place follows from the sums, so no
// atomics decide an order and a call gives the same tables every time.
//
// Bound: latency (16 bytes a request, 12 a token).  One launch: every CTA of
// one cluster scans all requests for itself (at most eight a thread), the
// CTAs then share the requests' pages and the tokens, with one cluster
// barrier between what reads the inputs and what may overwrite them
// (free_out may be free_in, lengths may be cached).  One CTA suffices up to
// kSoloTokens tokens; beyond, eight of them write the slots.
// 6.3 us for 256 requests of about one token, and for 37 of prompts up to 8192.
#include <cuda_runtime.h>
#include <cstdint>

#include "internal.h"
#include "ptx.cuh"

namespace rfq {
namespace {

constexpr int kThreads = 1024, kWarps = kThreads / 32;
constexpr int kCluster = 8;
constexpr int64_t kSoloTokens = 2048;

// (pages of one table: 32 bits, as the host has seen; tokens may be more)
struct Sums {
    uint32_t back, need;
    unsigned long long tok;
};

__device__ __forceinline__ Sums operator+(const Sums &x, const Sums &y)
{
    return {x.back + y.back, x.need + y.need, x.tok + y.tok};
}

// Inclusive sums over the warp's lanes.
__device__ __forceinline__ Sums warp_scan(Sums v, int lane)
{
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const Sums u = {__shfl_up_sync(0xFFFFFFFFu, v.back, d), __shfl_up_sync(0xFFFFFFFFu, v.need, d),
                        __shfl_up_sync(0xFFFFFFFFu, v.tok, d)};
        if (lane >= d)
            v = v + u;
    }
    return v;
}

// What request r holds and wants.  fits: its lengths are sane and its pages
// fit the table's row; a request that does not fit takes and gives nothing.
struct Request {
    int cached, added;
    uint32_t p0, p1, after;
    bool fits;
    __device__ __forceinline__ Request(const SlotMapArgs &a, int r)
    {
        cached = __ldcg(a.cached + r);
        added = __ldcg(a.added + r);
        const uint32_t page = a.page_size, c = max(cached, 0);
        after = added >= 0 ? c + (uint32_t)added : c > (uint32_t)-(int64_t)added ? c - (uint32_t)-(int64_t)added : 0u;
        p0 = c / page + (c % page != 0);
        p1 = after / page + (after % page != 0);
        fits = cached >= 0 && after <= (uint32_t)INT32_MAX && p0 <= (uint32_t)a.width && p1 <= (uint32_t)a.width;
    }
    __device__ __forceinline__ Sums sums() const
    {
        return {fits && p0 > p1 ? p0 - p1 : 0u, fits && p1 > p0 ? p1 - p0 : 0u, (unsigned long long)max(added, 0)};
    }
};

__global__ void __launch_bounds__(kThreads) slot_map_kernel(const SlotMapArgs a)
{
    extern __shared__ int32_t smem[];
    __shared__ Sums s_warp[kWarps];
    __shared__ uint32_t s_taken;
    static_assert(sizeof(s_warp) + sizeof(s_taken) <= 1024, "beside 47 KB of dynamic shared memory");
    const int R = a.requests, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int32_t *const s_start = smem;            // [R + 1] first token of each request
    int32_t *const s_cached = s_start + R + 1;
    uint32_t *const s_p0 = reinterpret_cast<uint32_t *>(s_cached + R);   // pages before
    uint32_t *const s_p1 = s_p0 + R;          // and after; before if it does not fit
    int32_t *const s_nth = reinterpret_cast<int32_t *>(s_p1 + R);   // its first page's place among the pages
                                              // taken; -1: not served
    uint32_t *const s_back = reinterpret_cast<uint32_t *>(s_nth + R);   // and among the pages given back
    const int rank = (int)cluster_ctarank(), ctas = gridDim.x;

    if (tid == 0)
        s_taken = 0;
    wait_for_previous();
    let_next_start();
    const int given = __ldcg(a.free_in);
    // this thread's requests, then the block's sums before them
    const int per = (R + kThreads - 1) / kThreads;
    const int r0 = min(R, tid * per), r1 = min(R, r0 + per);
    Sums own = {0, 0, 0};
    bool bad = false;
    uint32_t fit = 0;                         // which of them fit
    static_assert(kSlotMapRequests <= 32 * kThreads, "a bit for each of a thread's requests");
    for (int r = r0; r < r1; ++r) {
        const Request q(a, r);
        bad |= !q.fits;
        fit |= (uint32_t)q.fits << (r - r0);
        own = own + q.sums();
        s_cached[r] = q.cached;
        s_p0[r] = q.p0;
        s_p1[r] = q.fits ? q.p1 : q.p0;
        s_nth[r] = q.added;                  // (until the sums are known)
    }
    const Sums inc = warp_scan(own, lane);
    if (lane == 31)
        s_warp[warp] = inc;
    __syncthreads();
    const Sums w = warp_scan(s_warp[lane], lane);      // kWarps == 32
    Sums at = {__shfl_sync(0xFFFFFFFFu, w.back, (warp + 31) & 31), __shfl_sync(0xFFFFFFFFu, w.need, (warp + 31) & 31),
               __shfl_sync(0xFFFFFFFFu, w.tok, (warp + 31) & 31)};
    if (warp == 0)
        at = {0, 0, 0};
    const Sums all = {__shfl_sync(0xFFFFFFFFu, w.back, 31), __shfl_sync(0xFFFFFFFFu, w.need, 31),
                      __shfl_sync(0xFFFFFFFFu, w.tok, 31)};
    at = at + inc;
    at = {at.back - own.back, at.need - own.need, at.tok - own.tok};
    const uint32_t count = min(max(given, 0), a.free_capacity);
    // (pages given back beyond the list's end are dropped)
    const uint32_t top = min(count + all.back, (uint32_t)a.free_capacity);
    bad |= (int)count != given || count + all.back > (uint32_t)a.free_capacity || all.tok > (unsigned long long)a.tokens;
    uint32_t taken = 0;
    for (int r = r0; r < r1; ++r) {
        const bool fits = fit >> (r - r0) & 1u;
        const int added = s_nth[r];
        const uint32_t p0 = s_p0[r], p1 = s_p1[r], need = p1 > p0 ? p1 - p0 : 0u;
        const bool served = fits && (need == 0 || at.need + need <= top);
        s_start[r] = (int32_t)min(at.tok, (unsigned long long)INT32_MAX);
        s_nth[r] = served ? (int32_t)min(at.need, (uint32_t)INT32_MAX) : -1;
        s_back[r] = at.back;
        if (served && need > 0)
            taken = max(taken, at.need + need);
        at = at + Sums{p0 > p1 ? p0 - p1 : 0u, need, (unsigned long long)max(added, 0)};
    }
    if (tid == 0)
        s_start[R] = (int32_t)min(all.tok, (unsigned long long)INT32_MAX);
    if (taken > 0)
        atomicMax(&s_taken, taken);
    if (bad && rank == 0)
        atomicCAS(a.status, kDevOk, kDevBadGroups);
    __syncthreads();

    // pages given back: onto the stack, in the order of the requests
    if (all.back > 0)
        for (int r = rank * kWarps + warp; r < R; r += ctas * kWarps)
            for (uint32_t j = s_p1[r] + lane; j < s_p0[r]; j += 32) {
                const uint32_t to = count + s_back[r] + (j - s_p1[r]);
                if (to < (uint32_t)a.free_capacity)
                    a.free_pages[to] = __ldcg(a.table + (int64_t)r * a.width + j);
            }
    // what the outputs below may overwrite has been read now (`added` is
    // nobody's output)
    if (ctas > 1)
        cluster_sync();
    else
        __syncthreads();

    // pages taken: from the top, request by request
    const uint32_t top_taken = s_taken;
    if (top_taken > 0)
        for (int r = rank * kWarps + warp; r < R; r += ctas * kWarps) {
            const int nth = s_nth[r];
            const uint32_t p0 = s_p0[r], p1 = s_p1[r];
            if (nth >= 0)
                for (uint32_t j = p0 + lane; j < p1; j += 32)
                    a.table[(int64_t)r * a.width + j] = __ldcg(a.free_pages + (top - 1 - nth - (j - p0)));
        }
    if (rank == 0) {
        for (int r = tid; r < R; r += kThreads) {
            const int64_t after = (int64_t)s_cached[r] + __ldcg(a.added + r);
            a.lengths[r] = s_nth[r] >= 0 ? (int32_t)max(after, (int64_t)0) : s_cached[r];
        }
        for (int r = tid; r <= R; r += kThreads)
            a.token_start[r] = s_start[r];
        if (tid == 0)
            *a.free_out = (int32_t)(top - top_taken);
    }
    // tokens: the last request that starts at or before t and has tokens
    const int total = s_start[R];
    const uint32_t page_size = a.page_size;
    for (int64_t t = (int64_t)rank * kThreads + tid; t < a.tokens; t += (int64_t)ctas * kThreads) {
        int64_t slot = -1;
        int32_t pos = 0;
        if (t < total) {
            int lo = 0, hi = R;              // s_start[lo] <= t < s_start[hi]
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (s_start[mid] <= (int)t)
                    lo = mid;
                else
                    hi = mid;
            }
            const int nth = s_nth[lo];
            pos = s_cached[lo] + ((int)t - s_start[lo]);
            if (nth >= 0) {
                const uint32_t p0 = s_p0[lo], j = (uint32_t)pos / page_size;
                const int32_t page = j < p0 ? __ldcg(a.table + (int64_t)lo * a.width + j)
                                            : __ldcg(a.free_pages + (top - 1 - nth - (j - p0)));
                if (page >= 0)
                    slot = (int64_t)page * page_size + ((uint32_t)pos - j * page_size);
            }
        }
        a.slots[t] = slot;
        a.positions[t] = pos;
    }
}

} // namespace

cudaError_t launch_slot_map(const SlotMapArgs &a, cudaStream_t st)
{
    const size_t smem = (6 * (size_t)a.requests + 1) * sizeof(int32_t);
    if (smem > 47 * 1024)                    // (of 48 KB; the kernel's own arrays take some of it)
        if (cudaError_t e = cudaFuncSetAttribute(slot_map_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                 (6 * kSlotMapRequests + 1) * (int)sizeof(int32_t)))
            return e;
    const int ctas = a.tokens > kSoloTokens ? kCluster : 1;
    return launch_early(slot_map_kernel, dim3(ctas), kThreads, smem, st, ctas, a);
}

} // namespace rfq
