// kv_attention.cuh -- what the two attention kernels over the paged 4-bit
// cache share: how the work of ragged requests is laid end to end and split.
// A segment is one (request, key head, tile of rows); a row is one (token,
// query head) of the key head's group.  Its keys are cut into chunks of
// S::kChunk, each a unit of work, with S::kStart more units for the segment's
// start and end.
#pragma once

#include <cuda_bf16.h>
#include <cstdint>

#include "internal.h"
#include "ptx.cuh"

namespace rfq {

constexpr uint32_t kAll = 0xFFFFFFFFu;

// The reference m of a row's weights exp2(s - m), which are held in f16 (up to
// 2^16, all 11 bits down to 2^-14, multiples of 2^-24 below): kBelow octaves
// below the maximum when it is set, so that f16's range serves the small weights,
// and raised when a score passes it by more than kRoom.
constexpr float kBelow = 7.f, kRoom = 15.f;

__device__ __forceinline__ float ex2(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}

struct AttnParams {
    KvAttentionArgs a;
    int group;                 // query heads per key head
    int gran;                  // keys of one copy: they lie in one page
    int32_t *status;
    int32_t *counter;          // [CTAs] parts of a split segment that have arrived
    float *part;               // [2 CTAs] parts of split segments
    int least_rows, most_rows; // the requests taken: those with this many rows a key head
};

// The first key that a row sees of those before `end` (below zero: it sees none, and
// end - window may not fit 32 bits).
__device__ __forceinline__ int first_seen(int end, int window) { return max(0, max(0, end) - window); }

// One request: n new tokens (rows q0 .. of q) at the end of its L keys.
struct Request {
    int n, L, q0;
    // (true if q_start descends here)
    __device__ __forceinline__ bool load(const AttnParams &p, int r, int32_t *status)
    {
        const KvAttentionArgs &a = p.a;
        const int most = a.width * a.cache.page_size;      // (the host has seen that it fits an int)
        const int len = a.lengths[r];
        L = min(max(len, 0), most);
        q0 = r;
        n = 1;
        bool ok = len == L, descends = false;
        if (a.q_start) {
            q0 = a.q_start[r];
            const int q1 = a.q_start[r + 1];
            n = q1 - q0;
            descends = q0 > q1;
            if (q0 < 0 || q0 > q1 || q1 > a.tokens) {
                ok = false;
                n = 0;
            }
        }
        if (!ok && status)
            atomicCAS(status, kDevOk, kDevBadGroups);
        const int64_t rows = (int64_t)n * p.group;
        if (rows < p.least_rows || rows > p.most_rows)
            n = 0;
        return descends;
    }
    // Tiles of `rows` (token, head) rows
    __device__ __forceinline__ int tiles(int group, int rows) const { return (n * group + rows - 1) / rows; }
    // Keys [least, ke) that some row of the tile sees; kb is least rounded down to gran
    __device__ __forceinline__ void keys(int tile, const AttnParams &p, int rows, int &kb, int &ke, int &least) const
    {
        int first = 0, last = 0;
        if (n > 1) {
            first = tile * rows / p.group;
            last = min(n - 1, (tile * rows + rows - 1) / p.group);
        }
        ke = max(0, L - n + last + 1);
        least = first_seen(L - n + first + 1, p.a.window);
        kb = min(least & -p.gran, ke & -p.gran);
    }
    // Units of a tile: its chunks (one at least) and S::kStart more
    template <typename S>
    __device__ __forceinline__ uint32_t units(int tile, const AttnParams &p) const
    {
        int kb, ke, least;
        keys(tile, p, S::kRows, kb, ke, least);
        return max(1, (ke - kb + S::kChunk - 1) / S::kChunk) + S::kStart;
    }
};

__device__ __forceinline__ uint32_t warp_scan(uint32_t v, int lane)    // inclusive
{
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const uint32_t x = __shfl_up_sync(kAll, v, d);
        if (lane >= d)
            v += x;
    }
    return v;
}

// Units of one key head of a request (the whole warp together)
template <typename S>
__device__ __forceinline__ uint32_t head_units(const Request &q, const AttnParams &p, int lane)
{
    const int n = q.tiles(p.group, S::kRows);
    uint32_t s = 0;
#pragma unroll 1
    for (int t = lane; t < n; t += 32)
        s += q.template units<S>(t, p);
    return __reduce_add_sync(kAll, s);
}

// Walks requests [r, r1) with the whole warp until `rem` units lie behind:
// returns the units of all of them, or stops at the request in which rem
// runs out, with rem units of it.  Requests are taken 32 at a time, a lane
// each (of several tokens: those of many tiles are counted by the whole warp);
// one or two of several tokens one by one, which is less to do (256 requests
// of 512 keys, 32 heads on 8: with one token each 46 us, 11 more one by one, with
// 1 to 4 74 us, 17 more).
template <typename S>
__device__ __forceinline__ uint32_t seek(const AttnParams &p, int &r, int r1, uint32_t &rem, int lane, int32_t *status,
                                         bool &descends)
{
    constexpr int kFew = 4;
    uint32_t all = 0;
    const int H = p.a.cache.heads;
    // the 32 requests at r, `mine` units this lane's: are rem units in them?
    auto among = [&](uint32_t mine) {
        const uint32_t upto = warp_scan(mine, lane), sum = __shfl_sync(kAll, upto, 31);
        if (rem < sum) {
            const int at = __ffs(__ballot_sync(kAll, rem < upto)) - 1;
            rem -= __shfl_sync(kAll, upto - mine, at);
            r += at;
            return true;
        }
        rem -= sum;
        all += sum;
        return false;
    };
    if (!p.a.q_start) {
#pragma unroll 1
        for (; r < r1; r += 32) {
            uint32_t mine = 0;
            if (r + lane < r1) {
                Request q;
                q.load(p, r + lane, status);
                mine = H * (uint32_t)q.tiles(p.group, S::kRows) * q.template units<S>(0, p);
            }
            if (among(mine))
                return all;
        }
    } else if (r1 - r > 2) {
#pragma unroll 1
        for (; r < r1; r += 32) {
            uint32_t mine = 0;
            Request q = {0, 0, 0};
            if (r + lane < r1)
                descends |= q.load(p, r + lane, status);
            const int tiles = q.tiles(p.group, S::kRows);
            if (tiles <= kFew)
#pragma unroll 1
                for (int t = 0; t < tiles; ++t)
                    mine += q.template units<S>(t, p);
#pragma unroll 1
            for (uint32_t left = __ballot_sync(kAll, tiles > kFew); left; left &= left - 1) {
                const int src = __ffs(left) - 1;
                const Request one = {__shfl_sync(kAll, q.n, src), __shfl_sync(kAll, q.L, src), 0};
                const uint32_t sum = head_units<S>(one, p, lane);
                if (lane == src)
                    mine = sum;
            }
            if (among(H * mine))
                return all;
        }
    } else {
#pragma unroll 1
        for (; r < r1; ++r) {
            Request q;
            descends |= q.load(p, r, status);
            const uint32_t sum = H * head_units<S>(q, p, lane);
            if (rem < sum)
                return all;
            rem -= sum;
            all += sum;
        }
    }
    return all;
}

// The segments of a warp's run of units, one after the other.
template <typename S>
struct Walk {
    static constexpr int ROWS = S::kRows;
    int r, head, tile, ntiles;
    Request q;
    int kb, ke, chunks;        // of the segment
    int least;                 // no row of it sees a key below
    int i, i1;                 // the warp's chunks of it left
    uint32_t u, end;           // the segment's first unit; the end of the warp's units
    // from unit `first`, `rem` units into the segments of request r0
    __device__ __forceinline__ void start(const AttnParams &p, int r0, uint32_t rem, uint32_t first, uint32_t last, int lane)
    {
        r = r0;
        end = last;
        head = tile = i = i1 = 0;
        u = last;
        if (first >= last)
            return;
        q.load(p, r, nullptr);
        ntiles = q.tiles(p.group, ROWS);
        const uint32_t per = head_units<S>(q, p, lane);
        head = (int)(rem / per);
        rem -= head * per;
#pragma unroll 1
        for (;; tile += 32) {
            const uint32_t mine = tile + lane < ntiles ? q.template units<S>(tile + lane, p) : 0u;
            const uint32_t upto = warp_scan(mine, lane);
            const uint32_t hit = __ballot_sync(kAll, rem < upto);
            if (hit) {
                const int at = __ffs(hit) - 1;
                rem -= __shfl_sync(kAll, upto - mine, at);
                tile += at;
                break;
            }
            rem -= __shfl_sync(kAll, upto, 31);
        }
        u = first - rem;
        segment(p, first);
    }
    // the chunks of the segment at u that lie in [from, end): chunk k is unit u + kStart + k
    __device__ __forceinline__ void segment(const AttnParams &p, uint32_t from)
    {
        q.keys(tile, p, ROWS, kb, ke, least);
        chunks = max(1, (ke - kb + S::kChunk - 1) / S::kChunk);
        i = from > u + S::kStart ? (int)(from - u - S::kStart) : 0;
        i1 = end > u + S::kStart ? (int)min((uint32_t)chunks, end - u - S::kStart) : 0;
    }
    __device__ __forceinline__ bool more() const { return i < i1; }
    // on to the next segment that has a chunk here, if any, once more() is false
    __device__ __forceinline__ void next(const AttnParams &p)
    {
#pragma unroll 1
        while (i >= i1 && u < end) {
            u += chunks + S::kStart;
            if (u >= end)
                return;
            if (++tile == ntiles) {
                tile = 0;
                if (++head == p.a.cache.heads) {
                    head = 0;
#pragma unroll 1
                    do {               // (requests without new tokens have no segment)
                        ++r;
                        q.load(p, r, nullptr);
                        ntiles = q.tiles(p.group, ROWS);
                    } while (ntiles == 0);
                }
            }
            segment(p, u);
        }
    }
};

// A run of units, and where it starts: `rem` units into the segments of
// request r.
struct Share {
    uint32_t total, ctas, first, last, rem;
    int r;
};

// The share of this warp (ALL_WARPS) or of the CTA, found by the whole CTA of W
// warps; false if the CTA has none, and in every CTA if q_start descends
// somewhere (its requests' rows would overlap, and their units pass 32 bits:
// where it ascends the host has seen that they do not).  Each warp counts a run of requests, then
// finds its start in one of the runs.  (One loop for both: the second pass
// finds its code at hand.)  least: units of a CTA, at least: one with fewer
// would only add parts to join.
template <typename S, bool ALL_WARPS = true>
__device__ __forceinline__ bool find_share(const AttnParams &p, uint32_t *s_scan, int W, uint32_t least, Share &o)
{
    const KvAttentionArgs &a = p.a;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t cta = blockIdx.x;
    const int per = (a.requests + W - 1) / W;
    int run = warp;
    bool descends = false;
    o.rem = 0xFFFFFFFFu;
#pragma unroll 1
    for (int pass = 0;; ++pass) {
        o.r = min(a.requests, run * per);
        const uint32_t sum = seek<S>(p, o.r, min(a.requests, o.r + per), o.rem, lane,
                                     pass == 0 && cta == 0 ? p.status : nullptr, descends);
        if (pass == 1)
            return true;
        if (lane == 0)
            s_scan[warp] = sum;
        if (!a.q_start)
            __syncthreads();
        else if (__syncthreads_or(descends))
            return false;
        const uint32_t runs = warp_scan(lane < W ? s_scan[lane] : 0u, lane);
        o.total = __shfl_sync(kAll, runs, 31);
        o.ctas = min(gridDim.x, (o.total + least - 1) / least);
        if (cta >= o.ctas)
            return false;
        // total cta / ctas without a wide product
        const uint32_t each = o.total / o.ctas, more = o.total % o.ctas;
        const uint32_t u0 = each * cta + more * cta / o.ctas;
        const uint32_t un = each * (cta + 1) + more * (cta + 1) / o.ctas - u0;
        o.first = ALL_WARPS ? u0 + un / W * warp + un % W * warp / W : u0;
        o.last = ALL_WARPS ? u0 + un / W * (warp + 1) + un % W * (warp + 1) / W : u0 + un;
        run = min(W - 1, __popc(__ballot_sync(kAll, lane < W && runs <= o.first)));
        o.rem = o.first - (run ? __shfl_sync(kAll, runs, run - 1) : 0u);
        if (o.first >= o.last)
            o.rem = 0;
    }
}

// The CTA whose run holds unit u.
__device__ __forceinline__ int owner(const Share &s, uint32_t u)
{
    const uint32_t each = s.total / s.ctas, more = s.total % s.ctas;
    uint32_t k = min(s.ctas - 1, (uint32_t)((float)u * (float)s.ctas / (float)s.total));
    while (each * k + more * k / s.ctas > u)
        --k;
    while (each * (k + 1) + more * (k + 1) / s.ctas <= u)
        ++k;
    return (int)k;
}

// (m + log2 l) in nats: -inf for a row that saw no key, NaN for one whose wait ran out
__device__ __forceinline__ float log_sum(float m, float l)
{
    return l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
}
// Rows of no request, before q_start[0] and from q_start[requests] on (a step of
// fixed size has such): o = 0, lse = -inf, as for a row that sees no key.  A CTA's
// share, by `threads` of its threads.
__device__ __forceinline__ void clear_rest(const KvAttentionArgs &a, int thread, int threads)
{
    const int first = a.q_start[0], end = a.q_start[a.requests];
    if (first < 0 || end < first || end > a.tokens)
        return;                              // (the status says so)
    const int64_t rest = first + (a.tokens - end);
    const int row = a.heads * a.cache.head_dim / 8;
#pragma unroll 1
    for (int64_t i = blockIdx.x; i < rest; i += gridDim.x) {
        const int64_t t = i < first ? i : end + (i - first);
        uint4 *const out = static_cast<uint4 *>(a.out) + t * row;
#pragma unroll 1
        for (int j = thread; j < row; j += threads)
            out[j] = make_uint4(0, 0, 0, 0);
        if (a.lse)
#pragma unroll 1
            for (int j = thread; j < a.heads; j += threads)
                a.lse[t * a.heads + j] = -INFINITY;
    }
}

// 1 / l, 0 for a row that saw no key (and NaN for one whose wait ran out)
__device__ __forceinline__ float inverse(float l) { return l > 0.f ? 1.f / l : l; }

// kv_attention_tile.cu: the requests of p's row range, in tiles of 128 rows by
// 128 keys; a segment's start counts as 3 units
constexpr int kTileRowsEach = 128, kTileChunk = 128, kTileStart = 3;
size_t kv_attention_tile_part_bytes(int32_t head_dim);
cudaError_t launch_kv_attention_tile(const AttnParams &p, cudaStream_t st);

} // namespace rfq
