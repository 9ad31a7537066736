// moe_sort.cu -- pairs (token, choice) sorted by expert (rfq_moe_sort): the
// offsets of the experts' groups of rows, the row of each pair and the pair
// of each row.
//
// Mathematics: a stable counting sort.  Pair p of expert e goes to row
//     start[e] + (pairs of e before p),
// start being the exclusive sum of the groups' sizes, each rounded up to a
// multiple of `align`.  Every place follows from counts: no atomics decide an
// order, so the same ids give the same rows.
//
// Bound: latency (12 bytes a pair).  One launch of one cluster.  Each warp
// takes a run of the pairs and counts them by expert, 32 at a time: lanes of
// the same expert find each other with a match, the first one adds their
// number to the warp's own counters.  The counters are summed over the warps
// of a block and, through distributed shared memory, over the blocks; then
// the warps go through their pairs again and give out the rows.
#include <cuda_runtime.h>
#include <cstdint>

#include "internal.h"
#include "ptx.cuh"

namespace rfq {
namespace {

constexpr int kThreads = 1024, kWarps = kThreads / 32;
constexpr uint32_t kAll = 0xFFFFFFFFu;
constexpr int64_t kPairsPerCta = 4096;       // of a cluster that has room for more
constexpr int kMostCtas = 8;

__device__ __forceinline__ int ld_peer(uint32_t saddr, int rank)
{
    int v;
    asm volatile("ld.shared::cluster.b32 %0, [%1];" : "=r"(v) : "r"(mapa_shared(saddr, rank)) : "memory");
    return v;
}

__global__ void __launch_bounds__(kThreads) moe_sort_kernel(const MoeSortArgs a)
{
    __shared__ int s_count[kWarps][kMoeExperts];     // pairs of a warp; then those of the warps before it
    __shared__ int s_total[kMoeExperts];             // pairs of the block
    __shared__ int s_base[kMoeExperts];              // row of the block's first pair
    __shared__ int s_end[kMoeExperts], s_next[kMoeExperts];   // a group's end, and the next one's start
    __shared__ int s_scan[kMoeExperts / 32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = (int)cluster_ctarank(), ctas = gridDim.x;
    const int E = a.experts;
    for (int i = tid; i < kWarps * kMoeExperts; i += kThreads)
        (&s_count[0][0])[i] = 0;
    __syncthreads();
    wait_for_previous();
    let_next_start();

    // this warp's pairs, whole steps of 32
    const int64_t steps = (a.pairs + 31) / 32, per = (steps + ctas * kWarps - 1) / (ctas * kWarps);
    const int64_t p0 = min(a.pairs, (rank * kWarps + warp) * per * 32), p1 = min(a.pairs, p0 + per * 32);
    int *const mine = s_count[warp];
    auto expert = [&](int64_t p) {
        const int e = p < p1 ? a.ids[p] : -1;
        return e >= 0 && e < E ? e : -1;
    };
    for (int64_t p = p0; p < p1; p += 32) {
        const int e = expert(p + lane);
        const uint32_t same = __match_any_sync(kAll, e);
        if (e >= 0 && (same & ((1u << lane) - 1)) == 0)
            mine[e] += __popc(same);
        __syncwarp();
    }
    __syncthreads();
    int own = 0;                             // thread e: the block's pairs of expert e
    if (tid < kMoeExperts) {
        for (int w = 0; w < kWarps; ++w) {
            const int n = s_count[w][tid];
            s_count[w][tid] = own;
            own += n;
        }
        s_total[tid] = own;
    }
    if (ctas > 1)
        cluster_sync();
    int before = 0, all = own;
    if (tid < kMoeExperts && ctas > 1) {
        all = 0;
        for (int r = 0; r < ctas; ++r) {
            const int n = ld_peer(smem_u32(&s_total[tid]), r);
            before += r < rank ? n : 0;
            all += n;
        }
    }
    // exclusive sum over the experts of the groups' sizes
    const int size = (all + a.align - 1) / a.align * a.align;
    int inc = size;
    if (tid < kMoeExperts) {
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int u = __shfl_up_sync(kAll, inc, d);
            inc += lane >= d ? u : 0;
        }
        if (lane == 31)
            s_scan[warp] = inc;
    }
    __syncthreads();
    if (tid < kMoeExperts) {
        for (int w = 0; w < warp; ++w)
            inc += s_scan[w];
        const int start = inc - size;
        s_base[tid] = start + before;
        s_end[tid] = start + all;
        s_next[tid] = inc;
        if (rank == 0 && tid < E) {
            // (rows that are not there: the groups end where the whole ones do)
            const int most = (int)(a.rows / a.align * a.align);
            if (tid == 0)
                a.group_off[0] = 0;
            a.group_off[tid + 1] = min(inc, most);
            if (tid == E - 1 && inc > most)
                atomicCAS(a.status, kDevOk, kDevBadGroups);
        }
    }
    __syncthreads();
    for (int64_t p = p0; p < p1; p += 32) {
        const int e = expert(p + lane);
        const uint32_t same = __match_any_sync(kAll, e);
        const int nth = __popc(same & ((1u << lane) - 1));
        int row = -1;
        if (e >= 0) {
            row = s_base[e] + mine[e] + nth;
            row = row < a.rows / a.align * a.align ? row : -1;
        }
        __syncwarp();
        if (e >= 0 && nth == 0)
            mine[e] += __popc(same);
        __syncwarp();
        if (p + lane < p1) {
            a.row_of[p + lane] = row;
            if (row >= 0)
                a.pair_of[row] = (int)(p + lane);
        }
    }
    // rows of no pair: behind each group and behind the last
    for (int e = rank * kWarps + warp; e < E; e += ctas * kWarps)
        for (int64_t r = s_end[e] + lane; r < min((int64_t)s_next[e], a.rows); r += 32)
            a.pair_of[r] = -1;
    for (int64_t r = min((int64_t)s_next[E - 1], a.rows / a.align * a.align) + rank * kThreads + tid; r < a.rows; r += ctas * kThreads)
        a.pair_of[r] = -1;
    if (ctas > 1)
        cluster_sync();                      // (a block's shared memory is read by the others)
}

} // namespace

cudaError_t launch_moe_sort(const MoeSortArgs &a, cudaStream_t st)
{
    int ctas = 1;
    while (ctas < kMostCtas && ctas * kPairsPerCta < a.pairs)
        ctas *= 2;
    return launch_early(moe_sort_kernel, dim3(ctas), kThreads, 0, st, ctas, a);
}

} // namespace rfq
