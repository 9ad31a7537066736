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
// the same expert find each other by a ballot for each bit of its number (a
// match instruction took 62 clocks of the SM, 262144 pairs 67 us in all), the
// first one adds their number to the warp's own counters, and each pair's
// place among the warp's is kept.  The counters are summed over the warps of a
// block and, through distributed shared memory, over the blocks, which gives
// the rows.  Loads that do not depend on each other (pairs of eight steps, the
// warps' and the blocks' counters) are in flight together.
// 256 pairs of 128 experts: 2.5 us (4.1 with groups on 128 rows, 16512 in all);
// 32768: 8.5 us, of which 1.3 are the ballots, 1.3 the scattered stores of
// pair_of and 1 the rows of no pair; 262144: 42 us.
#include <cuda_runtime.h>
#include <cstdint>

#include "internal.h"
#include "ptx.cuh"

namespace rfq {
namespace {

constexpr uint32_t kAll = 0xFFFFFFFFu;
constexpr int kHeld = 8;                     // steps of 32 pairs in flight
constexpr int64_t kPairsPerCta = 512;        // of a cluster that has room for more; four rows count like a pair, most of a small call's hold
                                             // none (32 tokens of 8 pairs, 16512 rows: 4.1 us, with one block 6.4)
constexpr int kMostCtas = 8;

__device__ __forceinline__ int ld_peer(uint32_t saddr, int rank)
{
    int v;
    asm volatile("ld.shared::cluster.b32 %0, [%1];" : "=r"(v) : "r"(mapa_shared(saddr, rank)) : "memory");
    return v;
}

template <int THREADS>
__global__ void __launch_bounds__(THREADS) moe_sort_kernel(const MoeSortArgs a)
{
    static_assert(THREADS >= kMoeExperts, "a thread for each expert");
    constexpr int kWarps = THREADS / 32;
    __shared__ __align__(16) int s_count[kWarps][kMoeExperts];     // pairs of a warp; then those of the warps before it
    __shared__ int s_total[kMoeExperts];             // pairs of the block
    __shared__ int s_base[kMoeExperts];              // row of the block's first pair
    __shared__ int s_end[kMoeExperts], s_next[kMoeExperts];   // a group's end, and the next one's start
    __shared__ int s_scan[kMoeExperts / 32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = (int)cluster_ctarank(), ctas = gridDim.x;
    const int E = a.experts;
    // this warp's pairs, whole steps of 32
    const int64_t steps = (a.pairs + 31) / 32, per = (steps + ctas * kWarps - 1) / (ctas * kWarps);
    const int64_t p0 = min(a.pairs, (rank * kWarps + warp) * per * 32), p1 = min(a.pairs, p0 + per * 32);
    int *const mine = s_count[warp];
    int held[kHeld];                         // experts of the pairs of kHeld steps, -1 without one
    auto hold = [&](int64_t p) {
#pragma unroll
        for (int i = 0; i < kHeld; ++i)
            held[i] = p + 32 * i + lane < p1 ? a.ids[p + 32 * i + lane] : -1;
#pragma unroll
        for (int i = 0; i < kHeld; ++i)
            held[i] = held[i] >= 0 && held[i] < E ? held[i] : -1;
    };
    wait_for_previous();
    let_next_start();
    hold(p0);
    for (int i = tid; i < kWarps * kMoeExperts / 4; i += THREADS)
        reinterpret_cast<int4 *>(s_count)[i] = make_int4(0, 0, 0, 0);
    __syncthreads();
    // the place of each held pair among the warp's of its expert; of pairs that
    // are not held until the rows are given out, in the place of the row
    int place[kHeld];
    const bool kept = p1 - p0 <= 32 * kHeld;
    const int bits = 32 - __clz(E - 1);
#pragma unroll 1
    for (int64_t p = p0; p < p1; p += 32 * kHeld) {
        if (p > p0)
            hold(p);
#pragma unroll
        for (int i = 0; i < kHeld; ++i)
            if (p + 32 * i < p1) {
                const int e = held[i];
                uint32_t same = __ballot_sync(kAll, e >= 0);
                for (int b = 0; b < bits; ++b) {
                    const uint32_t set = __ballot_sync(kAll, e >> b & 1);
                    same &= e >> b & 1 ? set : ~set;
                }
                const int nth = __popc(same & ((1u << lane) - 1));
                place[i] = e >= 0 ? mine[e] + nth : 0;
                __syncwarp();
                if (e >= 0 && nth == 0)
                    mine[e] = place[i] + __popc(same);
                __syncwarp();
                if (!kept && p + 32 * i + lane < p1)
                    a.row_of[p + 32 * i + lane] = place[i];
            }
    }
    __syncthreads();
    int own = 0;                             // thread e: the block's pairs of expert e
    if (tid < kMoeExperts) {
        int n[kWarps];
#pragma unroll
        for (int w = 0; w < kWarps; ++w)
            n[w] = s_count[w][tid];
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            s_count[w][tid] = own;
            own += n[w];
        }
        s_total[tid] = own;
    }
    if (ctas > 1)
        cluster_sync();
    int before = 0, all = own;
    if (tid < kMoeExperts && ctas > 1) {
        int n[kMostCtas];
#pragma unroll
        for (int r = 0; r < kMostCtas; ++r)
            n[r] = r < ctas ? ld_peer(smem_u32(&s_total[tid]), r) : 0;
        all = 0;
#pragma unroll
        for (int r = 0; r < kMostCtas; ++r) {
            before += r < rank ? n[r] : 0;
            all += n[r];
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
    const int most = (int)(a.rows / a.align * a.align);
#pragma unroll 1
    for (int64_t p = p0; p < p1; p += 32 * kHeld) {
        if (!kept) {
            hold(p);
#pragma unroll
            for (int i = 0; i < kHeld; ++i)
                place[i] = p + 32 * i + lane < p1 ? a.row_of[p + 32 * i + lane] : 0;
        }
#pragma unroll
        for (int i = 0; i < kHeld; ++i) {
            const int64_t at = p + 32 * i + lane;
            if (at < p1) {
                const int e = held[i];
                int row = -1;
                if (e >= 0) {
                    row = s_base[e] + mine[e] + place[i];
                    row = row < most ? row : -1;
                }
                a.row_of[at] = row;
                if (row >= 0)
                    a.pair_of[row] = (int)at;
            }
        }
    }
    // rows of no pair: behind each group and behind the last
    const int w = rank * kWarps + warp, warps = ctas * kWarps;
    for (int e0 = w; e0 < E; e0 += 32 * warps) {
        const int e = e0 + lane * warps, end = e < E ? s_end[e] : 0, next = e < E ? s_next[e] : 0;
        for (uint32_t some = __ballot_sync(kAll, end < next); some; some &= some - 1) {
            const int64_t from = __shfl_sync(kAll, end, __ffs(some) - 1), to = __shfl_sync(kAll, next, __ffs(some) - 1);
            for (int64_t r = from + lane; r < min(to, a.rows); r += 32)
                a.pair_of[r] = -1;
        }
    }
    for (int64_t r = (int64_t)min(s_next[E - 1], most) + rank * THREADS + tid; r < a.rows; r += ctas * THREADS)
        a.pair_of[r] = -1;
    if (ctas > 1)
        cluster_sync();                      // (a block's shared memory is read by the others)
}

} // namespace

cudaError_t launch_moe_sort(const MoeSortArgs &a, cudaStream_t st)
{
    int ctas = 1;
    while (ctas < kMostCtas && ctas * kPairsPerCta < a.pairs + a.rows / 4)
        ctas *= 2;
    // (fewer threads pass barriers sooner, more have more pairs in flight: 256 pairs take 4.1 us with 256 threads, 5.7 with 1024;
    // 32768 pairs 8.5 with 512, 9.1 with 1024; 131072 pairs 24.7 and 23.1)
    return a.pairs <= 4096    ? launch_early(moe_sort_kernel<256>, dim3(ctas), 256, 0, st, ctas, a)
           : a.pairs <= 32768 ? launch_early(moe_sort_kernel<512>, dim3(ctas), 512, 0, st, ctas, a)
                              : launch_early(moe_sort_kernel<1024>, dim3(ctas), 1024, 0, st, ctas, a);
}

} // namespace rfq
