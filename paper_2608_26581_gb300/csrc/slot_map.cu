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
#include <cuda_runtime.h>
#include <cstdint>

#include "internal.h"
#include "ptx.cuh"

namespace rfq {
namespace {

constexpr int kThreads = 1024, kWarps = kThreads / 32;
constexpr int kCluster = 8;
constexpr int64_t kSoloTokens = 2048;

struct Sums {
    long long back, need, tok;
};

__device__ __forceinline__ Sums operator+(const Sums &x, const Sums &y)
{
    return {x.back + y.back, x.need + y.need, x.tok + y.tok};
}

__device__ __forceinline__ Sums shfl_up(const Sums &x, int d)
{
    return {__shfl_up_sync(0xFFFFFFFFu, x.back, d), __shfl_up_sync(0xFFFFFFFFu, x.need, d),
            __shfl_up_sync(0xFFFFFFFFu, x.tok, d)};
}

// Inclusive sums over the warp's lanes.
__device__ __forceinline__ Sums warp_scan(Sums v, int lane)
{
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const Sums u = shfl_up(v, d);
        if (lane >= d)
            v = v + u;
    }
    return v;
}

// What request r holds and wants.  fits: its lengths are sane and its pages
// fit the table's row; a request that does not fit takes and gives nothing.
struct Request {
    long long cached, after, p0, p1;
    bool fits;
    __device__ Request(const SlotMapArgs &a, int r)
    {
        cached = a.cached[r];
        const long long n = cached + (long long)a.added[r];
        after = n > 0 ? n : 0;
        p0 = cached > 0 ? (cached + a.page_size - 1) / a.page_size : 0;
        p1 = (after + a.page_size - 1) / a.page_size;
        fits = cached >= 0 && p0 <= a.width && p1 <= a.width;
    }
    __device__ Sums sums(int added) const
    {
        return {fits && p0 > p1 ? p0 - p1 : 0, fits && p1 > p0 ? p1 - p0 : 0, added > 0 ? added : 0};
    }
};

__global__ void __launch_bounds__(kThreads) slot_map_kernel(const SlotMapArgs a)
{
    extern __shared__ int32_t smem[];
    __shared__ Sums s_warp[kWarps];
    __shared__ int s_taken;
    const int R = a.requests, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int32_t *const s_start = smem;            // [R + 1] first token of each request
    int32_t *const s_cached = s_start + R + 1;
    int32_t *const s_nth = s_cached + R;      // its first page's place among the pages taken; -1: not served
    int32_t *const s_back = s_nth + R;        // its first page's place among the pages given back
    const int rank = (int)cluster_ctarank(), ctas = gridDim.x;

    if (tid == 0)
        s_taken = 0;
    // this thread's requests, then the block's sums before them
    const int per = (R + kThreads - 1) / kThreads;
    const int r0 = min(R, tid * per), r1 = min(R, r0 + per);
    Sums own = {0, 0, 0};
    bool bad = false;
    for (int r = r0; r < r1; ++r) {
        const Request q(a, r);
        bad |= !q.fits;
        own = own + q.sums(a.added[r]);
    }
    const Sums inc = warp_scan(own, lane);
    if (lane == 31)
        s_warp[warp] = inc;
    __syncthreads();
    const Sums w = warp_scan(s_warp[lane], lane);      // kWarps == 32
    Sums before = {__shfl_sync(0xFFFFFFFFu, w.back, (warp + 31) & 31), __shfl_sync(0xFFFFFFFFu, w.need, (warp + 31) & 31),
                   __shfl_sync(0xFFFFFFFFu, w.tok, (warp + 31) & 31)};
    if (warp == 0)
        before = {0, 0, 0};
    const Sums all = {__shfl_sync(0xFFFFFFFFu, w.back, 31), __shfl_sync(0xFFFFFFFFu, w.need, 31),
                      __shfl_sync(0xFFFFFFFFu, w.tok, 31)};
    Sums at = before + inc;
    at = {at.back - own.back, at.need - own.need, at.tok - own.tok};
    const long long given = *a.free_in;
    const long long count = given < 0 ? 0 : given > a.free_capacity ? a.free_capacity : given;
    // (pages given back beyond the list's end are dropped)
    const long long top = min(count + all.back, (long long)a.free_capacity);
    bad |= count != given || count + all.back > a.free_capacity || all.tok > a.tokens;
    int taken = 0;
    for (int r = r0; r < r1; ++r) {
        const Request q(a, r);
        const Sums s = q.sums(a.added[r]);
        const bool served = q.fits && (s.need == 0 || at.need + s.need <= top);
        s_start[r] = (int32_t)min(at.tok, (long long)INT32_MAX);
        s_cached[r] = (int32_t)q.cached;
        s_nth[r] = served ? (int32_t)min(at.need, (long long)INT32_MAX) : -1;
        s_back[r] = (int32_t)min(at.back, (long long)INT32_MAX);
        if (served && s.need > 0)
            taken = max(taken, (int)(at.need + s.need));
        at = at + s;
    }
    if (tid == 0)
        s_start[R] = (int32_t)min(all.tok, (long long)INT32_MAX);
    if (taken > 0)
        atomicMax(&s_taken, taken);
    if (bad && rank == 0)
        atomicCAS(a.status, kDevOk, kDevBadGroups);
    __syncthreads();

    // pages given back: onto the stack, in the order of the requests
    if (all.back > 0)
        for (int r = rank * kWarps + warp; r < R; r += ctas * kWarps) {
            const Request q(a, r);
            if (!q.fits)
                continue;
            for (long long j = q.p1 + lane; j < q.p0; j += 32) {
                const long long to = count + s_back[r] + (j - q.p1);
                if (to < a.free_capacity)
                    a.free_pages[to] = a.table[(int64_t)r * a.width + j];
            }
        }
    // lengths that the outputs below may overwrite are in shared memory now;
    // `added` is read again, and is nobody's output
    cluster_sync();

    // pages taken: from the top, request by request
    if (s_taken > 0)
        for (int r = rank * kWarps + warp; r < R; r += ctas * kWarps) {
            if (s_nth[r] < 0)
                continue;
            const long long cached = s_cached[r], after = max(cached + (long long)a.added[r], 0ll);
            const long long p0 = (cached + a.page_size - 1) / a.page_size, p1 = (after + a.page_size - 1) / a.page_size;
            for (long long j = p0 + lane; j < p1; j += 32)
                a.table[(int64_t)r * a.width + j] = __ldcg(a.free_pages + (top - 1 - s_nth[r] - (j - p0)));
        }
    if (rank == 0) {
        for (int r = tid; r < R; r += kThreads) {
            const long long after = max((long long)s_cached[r] + a.added[r], 0ll);
            a.lengths[r] = s_nth[r] >= 0 ? (int32_t)after : s_cached[r];
        }
        for (int r = tid; r <= R; r += kThreads)
            a.token_start[r] = s_start[r];
        if (tid == 0)
            *a.free_out = (int32_t)(top - s_taken);
    }
    // tokens: the last request that starts at or before t and has tokens
    const long long total = min(all.tok, (long long)INT32_MAX);
    for (int64_t t = (int64_t)rank * kThreads + tid; t < a.tokens; t += (int64_t)ctas * kThreads) {
        int64_t slot = -1;
        int32_t pos = 0;
        if (t < total) {
            int lo = 0, hi = R;              // s_start[lo] <= t < s_start[hi]
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (s_start[mid] <= t)
                    lo = mid;
                else
                    hi = mid;
            }
            const long long cached = s_cached[lo], p = cached + (t - s_start[lo]);
            pos = (int32_t)p;
            if (s_nth[lo] >= 0) {
                const long long p0 = (cached + a.page_size - 1) / a.page_size, j = p / a.page_size;
                const int32_t page = j < p0 ? a.table[(int64_t)lo * a.width + j]
                                            : __ldcg(a.free_pages + (top - 1 - s_nth[lo] - (j - p0)));
                if (page >= 0)
                    slot = (int64_t)page * a.page_size + (p - j * a.page_size);
            }
        }
        a.slots[t] = slot;
        a.positions[t] = pos;
    }
}

} // namespace

cudaError_t launch_slot_map(const SlotMapArgs &a, cudaStream_t st)
{
    const size_t smem = (4 * (size_t)a.requests + 1) * sizeof(int32_t);
    if (smem > 48 * 1024)
        if (cudaError_t e = cudaFuncSetAttribute(slot_map_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                 (4 * kSlotMapRequests + 1) * (int)sizeof(int32_t)))
            return e;
    const int ctas = a.tokens > kSoloTokens ? kCluster : 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(ctas);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim = {(unsigned)ctas, 1, 1};
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, slot_map_kernel, a);
}

} // namespace rfq
