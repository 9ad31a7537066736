// kv_attention.cu -- attention over the paged 4-bit cache (rfq_kv_attention):
// o = softmax(scale q k^T) v for the last n tokens of every request over its
// cached keys, in one launch.
//
// Mathematics: one pass over the keys with a running maximum and sum
// (log2 domain).  Keys and values enter the tensor cores as their 4-bit codes
// in f16 (exact): S^T = K q^T and O^T = V^T P^T with K and V^T the A operand
// of mma.m16n8k16, 16 keys (or 16 dimensions) by 8 rows, a row being one
// (token, query head) of the key head's group.
//   K: a block's scale multiplies the fp32 sums over its 32 (MXFP4) or 64
//      (HiF4) dimensions: nothing is rounded.
//   q: made f16 by a power of two per row (maximum in [2^14, 2^15)): exact
//      down to 2^-28 of the maximum, off by less than 2^-39 of it below.
//   P: exp2(s - m) rounded to f16 (relative 2^-11; its sum l stays fp32); m
//      is raised only when a score passes it by 8, which f16 has room for.
//   V: codes times scale relative to a running power of two, exact in f16
//      while the scales of one 32-dimension block span less than 2^24 over
//      the keys seen so far; smaller ones fade out.
//
// Bound: HBM at long caches: 136 (MXFP4) or 144 (HiF4) bytes a key and head
// of 128.  An SM's share of the measured copy rate is one of these every 5.8
// clocks, so a key may cost at most 23 warp instructions.
//
// Work: the (request, key head, row tile) segments of all requests laid end
// to end, in units of 128 keys, are split evenly over the resident CTAs,
// however ragged the lengths.  A segment that one CTA holds whole is written
// by it; the parts of others go to the workspace, and the last CTA to finish
// adds them in the order of the keys (the split depends on the lengths
// alone: a call gives the same bits every time).  One producer warp copies the
// pages' contiguous bytes into a ring of stages; eight consumer warps take 16
// keys of a stage each and are joined once per segment.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <cstdint>

#include "internal.h"
#include "kv_layout.cuh"
#include "ptx.cuh"

namespace rfq {
namespace {

constexpr int kConsumers = 8, kThreads = 32 * (kConsumers + 1);
constexpr int kUnit = 16 * kConsumers;       // keys of a stage

__device__ __forceinline__ uint32_t movmatrix(uint32_t a)
{
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(a));
    return r;
}

__device__ __forceinline__ float ex2(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi)
{
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}

__device__ __forceinline__ void consumer_sync()
{
    asm volatile("bar.sync 1, %0;" ::"n"(32 * kConsumers) : "memory");
}

struct Params {
    KvAttentionArgs a;
    int group;                 // query heads per key head
    int gran;                  // keys of one copy: the largest power of two dividing a page, at most 128
    int32_t *status;
    int32_t *counter;          // [CTAs] parts of a split segment that have arrived
    float *part_ml;            // [2 CTAs][rows][2]
    float *part_o;             // [2 CTAs][rows][D]
};

template <int FMT, int D, int NT>
struct Shape {
    static constexpr int kRows = 8 * NT;
    static constexpr int kScale = FMT == RFQ_FMT_HIF4 ? D / 16 : D / 32;   // bytes a token
    static constexpr int kCode = D / 2;
    static constexpr int kVOff = kUnit * kCode, kKsOff = 2 * kVOff, kVsOff = kKsOff + kUnit * kScale;
    static constexpr int kStage = kVsOff + kUnit * kScale;
    static constexpr int kBlocksPerSm = NT == 1 ? 2 : 1;
    static constexpr int kMerge = kConsumers * 8 * D * 4;
    static constexpr int kQ = NT > 1 ? NT * D * 16 : 0;
    static constexpr int kStages = ((kBlocksPerSm == 2 ? 108 : 200) * 1024 - kMerge - kQ) / kStage;
    static constexpr int kSmem = kStages * kStage + kMerge + kQ;
};

// One request: n new tokens (rows q0 .. of q) at the end of its L keys.
struct Request {
    int n, L, q0;
    __device__ void load(const KvAttentionArgs &a, int r, int32_t *status)
    {
        const int64_t most = (int64_t)a.width * a.cache.page_size;
        const int len = __ldg(a.lengths + r);
        L = (int)min((int64_t)max(len, 0), most);
        int q1 = r + 1;
        q0 = r;
        if (a.q_start) {
            q0 = __ldg(a.q_start + r);
            q1 = __ldg(a.q_start + r + 1);
        }
        const bool rows_ok = q0 >= 0 && q0 <= q1 && q1 <= a.tokens;
        n = rows_ok ? q1 - q0 : 0;
        if ((len != L || !rows_ok) && status)
            atomicCAS(status, kDevOk, kDevBadGroups);
    }
    // Tiles of `rows` (token, head) rows
    __device__ int tiles(int group, int rows) const { return (int)(((int64_t)n * group + rows - 1) / rows); }
    // Keys [kb, ke) that some row of the tile sees, kb rounded down to gran
    __device__ void keys(int tile, int group, int rows, int window, int gran, int &kb, int &ke) const
    {
        const int first = (int)((int64_t)tile * rows / group);
        const int last = (int)min((int64_t)n - 1, ((int64_t)(tile + 1) * rows - 1) / group);
        ke = max(0, L - n + last + 1);
        kb = window > 0 ? max(0, L - n + first + 1 - window) / gran * gran : 0;
        kb = min(kb, ke / gran * gran);
    }
    __device__ int units(int tile, int group, int rows, int window, int gran) const
    {
        int kb, ke;
        keys(tile, group, rows, window, gran, kb, ke);
        return max(1, (ke - kb + kUnit - 1) / kUnit);
    }
    // Units of one key head
    __device__ long long all_units(int group, int rows, int window, int gran) const
    {
        long long s = 0;
        const int t = tiles(group, rows);
        for (int i = 0; i < t; ++i)
            s += units(i, group, rows, window, gran);
        return s;
    }
};

// The segments of a CTA's share of the units, one after the other.
template <int ROWS>
struct Walk {
    const Params &p;
    int r, head, tile, ntiles;
    Request q;
    int kb, ke, units;         // of the segment
    int i0, i1;                // this CTA's units of it
    long long u, u1;           // the CTA's units left
    __device__ Walk(const Params &pp, int r0, long long rem, long long first, long long last) : p(pp), r(r0), u(first), u1(last)
    {
        if (u >= u1)
            return;
        q.load(p.a, r, nullptr);
        ntiles = q.tiles(p.group, ROWS);
        const long long per = q.all_units(p.group, ROWS, p.a.window, p.gran);
        head = (int)(rem / per);
        rem -= head * per;
        for (tile = 0;; ++tile) {
            const int n = q.units(tile, p.group, ROWS, p.a.window, p.gran);
            if (rem < n)
                break;
            rem -= n;
        }
        segment((int)rem);
    }
    __device__ void segment(int from)
    {
        q.keys(tile, p.group, ROWS, p.a.window, p.gran, kb, ke);
        units = max(1, (ke - kb + kUnit - 1) / kUnit);
        i0 = from;
        i1 = (int)min((long long)units, from + (u1 - u));
    }
    __device__ bool more() const { return u < u1; }
    __device__ void next()
    {
        u += i1 - i0;
        if (u >= u1)
            return;
        if (++tile == ntiles) {
            tile = 0;
            if (++head == p.a.cache.heads) {
                head = 0;
                do {               // (requests without new tokens have no segment)
                    ++r;
                    q.load(p.a, r, nullptr);
                    ntiles = q.tiles(p.group, ROWS);
                } while (ntiles == 0);
            }
        }
        segment(0);
    }
};

template <int FMT, int D, int NT>
__global__ void __launch_bounds__(kThreads, Shape<FMT, D, NT>::kBlocksPerSm) kv_attention_kernel(const Params p)
{
    using S = Shape<FMT, D, NT>;
    constexpr bool HIF4 = FMT == RFQ_FMT_HIF4;
    constexpr int NB = D / 32, ROWS = S::kRows, MT = D / 16, STAGES = S::kStages;
    extern __shared__ __align__(128) uint8_t smem[];
    uint8_t *const s_ring = smem;
    float *const s_merge = reinterpret_cast<float *>(smem + STAGES * S::kStage);   // [warp][8][D]
    uint4 *const s_q = reinterpret_cast<uint4 *>(smem + STAGES * S::kStage + S::kMerge);
    __shared__ alignas(8) uint64_t s_full[STAGES], s_empty[STAGES];
    __shared__ float s_m[kConsumers][ROWS], s_l[kConsumers][ROWS], s_qs[ROWS];
    __shared__ long long s_scan[kConsumers + 1], s_rem;
    __shared__ int s_r0, s_flag;

    const KvAttentionArgs &a = p.a;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int H = a.cache.heads, G = p.group;

    if (tid == 0) {
        for (int i = 0; i < STAGES; ++i) {
            mbar_init(&s_full[i], 1);
            mbar_init(&s_empty[i], kConsumers);
        }
        fence_mbar_init();
    }
    // ---- this CTA's share: units of all requests, in order
    const int per = (a.requests + kThreads - 1) / kThreads;
    const int r0 = min(a.requests, tid * per), r1 = min(a.requests, r0 + per);
    long long mine = 0;
    for (int r = r0; r < r1; ++r) {
        Request q;
        q.load(a, r, blockIdx.x == 0 ? p.status : nullptr);
        mine += H * q.all_units(G, ROWS, a.window, p.gran);
    }
    long long inc = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const long long v = __shfl_up_sync(0xFFFFFFFFu, inc, d);
        if (lane >= d)
            inc += v;
    }
    if (lane == 31)
        s_scan[warp] = inc;
    __syncthreads();
    long long before = inc - mine, total = 0;
#pragma unroll
    for (int w = 0; w <= kConsumers; ++w) {
        if (w < warp)
            before += s_scan[w];
        total += s_scan[w];
    }
    const int ctas = (int)min((long long)gridDim.x, total), cta = blockIdx.x;
    if (cta >= ctas)
        return;
    const long long u0 = total * cta / ctas, u1 = total * (cta + 1) / ctas;
    if (before <= u0 && u0 < before + mine) {
        long long at = u0 - before;
        for (int r = r0;; ++r) {
            Request q;
            q.load(a, r, nullptr);
            const long long n = H * q.all_units(G, ROWS, a.window, p.gran);
            if (at < n) {
                s_r0 = r;
                s_rem = at;
                break;
            }
            at -= n;
        }
    }
    __syncthreads();
    Walk<ROWS> walk(p, s_r0, s_rem, u0, u1);
    const uint64_t limit = ws_wait_limit_ns(p.status);
    bool ok = true;
    uint32_t it = 0;                          // stages used so far

    if (warp == kConsumers) {
        // ---- producer: lane j copies granule j of a stage
        const int64_t token_row = (int64_t)a.cache.page_size;
        const uint32_t gbytes = p.gran * (2 * S::kCode + 2 * S::kScale);
        for (; walk.more(); walk.next()) {
            const int32_t *const row = a.table + (int64_t)walk.r * a.width;
            for (int i = walk.i0; i < walk.i1; ++i, ++it) {
                const int st = it % STAGES;
                const int key = walk.kb + i * kUnit + lane * p.gran;
                bool have = lane * p.gran < kUnit && key < walk.ke;
                int64_t at = 0;
                if (have) {
                    const int pg = key / a.cache.page_size, page = __ldg(row + pg);
                    if (page < 0 || page >= a.cache.pages) {
                        atomicCAS(p.status, kDevOk, kDevBadGroups);
                        have = false;
                    }
                    at = ((int64_t)page * H + walk.head) * token_row + (key - pg * a.cache.page_size);
                }
                const uint32_t granules = __popc(__ballot_sync(0xFFFFFFFFu, have));
                if (it >= STAGES)
                    ok = ok && mbar_wait(&s_empty[st], (it / STAGES - 1) & 1, limit);
                ok = __all_sync(0xFFFFFFFFu, ok);
                if (!ok)
                    have = false;
                if (lane == 0)
                    mbar_arrive_expect_tx(&s_full[st], ok ? granules * gbytes : 0);
                __syncwarp();
                if (have) {
                    uint8_t *const d = s_ring + st * S::kStage;
                    const int tok = lane * p.gran;
                    bulk_load(d + tok * S::kCode, static_cast<const uint8_t *>(a.cache.k_codes) + at * S::kCode,
                              p.gran * S::kCode, &s_full[st]);
                    bulk_load(d + S::kKsOff + tok * S::kScale,
                              static_cast<const uint8_t *>(a.cache.k_scales) + at * S::kScale, p.gran * S::kScale,
                              &s_full[st]);
                    bulk_load(d + S::kVOff + tok * S::kCode, static_cast<const uint8_t *>(a.cache.v_codes) + at * S::kCode,
                              p.gran * S::kCode, &s_full[st]);
                    bulk_load(d + S::kVsOff + tok * S::kScale,
                              static_cast<const uint8_t *>(a.cache.v_scales) + at * S::kScale, p.gran * S::kScale,
                              &s_full[st]);
                }
            }
        }
        // nothing leaves while a copy of its own is in flight
        for (uint32_t k = it > STAGES ? it - STAGES : 0; k < it; ++k)
            if (!mbar_wait(&s_full[k % STAGES], (k / STAGES) & 1, limit))
                ok = false;
        if (!ok && lane == 0)
            atomicExch(p.status, kDevTimeout);
        return;
    }

    // ---- consumers
    const int g = lane >> 2, c = lane & 3;
    for (; walk.more(); walk.next()) {
        const Request &q = walk.q;
        const int row0 = walk.tile * ROWS, rows = (int)min((int64_t)ROWS, (int64_t)q.n * G - row0);
        // q as f16, scaled by a power of two per row
        uint4 qf[NB];
        float qs[NT][2];
        int hi[NT][2];                        // keys that the thread's two rows see: [max(0, hi - window), hi)
        {
            const float base = a.scale * 1.4426950408889634f * (HIF4 ? 128.f : 1.f);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                if (NT == 1 || t == warp) {
                    const int rr = 8 * t + g, ri = row0 + rr;
                    uint4 raw[NB];
                    float mx = 0.f;
#pragma unroll
                    for (int b = 0; b < NB; ++b) {
                        raw[b] = make_uint4(0, 0, 0, 0);
                        if (rr < rows)
                            raw[b] = __ldg(reinterpret_cast<const uint4 *>(
                                static_cast<const __nv_bfloat16 *>(a.q) + (q.q0 + ri / G) * a.q_token +
                                (int64_t)(walk.head * G + ri % G) * a.q_head + 32 * b + 8 * c));
                        const uint32_t w[4] = {raw[b].x, raw[b].y, raw[b].z, raw[b].w};
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            mx = fmaxf(mx, fmaxf(fabsf(__uint_as_float(w[j] << 16)),
                                                 fabsf(__uint_as_float(w[j] & 0xFFFF0000u))));
                    }
                    mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, 1));
                    mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, 2));
                    const int e = max(min((int)(__float_as_uint(mx) >> 23) - 127 - 14, 126), -126);
                    const float mul = __uint_as_float((uint32_t)(127 - e) << 23);
                    const float undo = __uint_as_float((uint32_t)(127 + e) << 23) * base;
#pragma unroll
                    for (int b = 0; b < NB; ++b) {
                        const uint32_t w[4] = {raw[b].x, raw[b].y, raw[b].z, raw[b].w};
                        float f[8];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            f[2 * j] = __uint_as_float(w[j] << 16) * mul;
                            f[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u) * mul;
                        }
                        uint32_t h[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            // HiF4 codes decode in the order 0 2 | 1 3 | 4 6 | 5 7
                            const int lo = HIF4 ? (j >> 1) * 4 + (j & 1) : 2 * j, up = HIF4 ? lo + 2 : lo + 1;
                            h[j] = pack_f16(f[lo], f[up]);
                        }
                        qf[b] = make_uint4(h[0], h[1], h[2], h[3]);
                        if (NT > 1)
                            s_q[(t * NB + b) * 32 + lane] = qf[b];
                    }
                    if (NT == 1) {
                        qs[0][0] = __shfl_sync(0xFFFFFFFFu, undo, 8 * c);
                        qs[0][1] = __shfl_sync(0xFFFFFFFFu, undo, 8 * c + 4);
                    } else if (c == 0) {
                        s_qs[rr] = undo;
                    }
                }
            }
            if (NT > 1)
                consumer_sync();
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    if (NT > 1)
                        qs[t][j] = s_qs[8 * t + 2 * c + j];
                    const int ri = row0 + min(8 * t + 2 * c + j, rows - 1);
                    hi[t][j] = max(0, q.L - q.n + ri / G + 1);
                }
        }
        const int all_hi = max(0, q.L - q.n + row0 / G + 1);   // every row sees [all_lo, all_hi)
        const int all_lo = a.window > 0 ? max(0, q.L - q.n + (row0 + rows - 1) / G + 1 - a.window) : 0;

        float o[NT][MT][4], m[NT][2], l[NT][2];
        int vref = -1000;                     // V scale exponents are relative to it (the same in a row's quad)
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            m[t][0] = m[t][1] = -INFINITY;
            l[t][0] = l[t][1] = 0.f;
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    o[t][i][j] = 0.f;
        }

        for (int i = walk.i0; i < walk.i1; ++i, ++it) {
            const int st = it % STAGES;
            ok = ok && mbar_wait(&s_full[st], (it / STAGES) & 1, limit);
            const int key0 = walk.kb + i * kUnit + warp * 16;
            if (ok && key0 < walk.ke) {
                const uint8_t *const ring = s_ring + st * S::kStage;
                // ---- scores of 16 keys: rows g and g + 8 of the tile
                uint32_t k0[NB], k1[NB];
                {
                    const uint8_t *const kr = ring + (warp * 16 + g) * S::kCode + c * NB * 4;
                    if (D == 128) {
                        const uint4 x = *reinterpret_cast<const uint4 *>(kr);
                        const uint4 y = *reinterpret_cast<const uint4 *>(kr + 8 * S::kCode);
                        k0[0] = x.x, k0[1] = x.y, k0[NB - 2] = x.z, k0[NB - 1] = x.w;
                        k1[0] = y.x, k1[1] = y.y, k1[NB - 2] = y.z, k1[NB - 1] = y.w;
                    } else {
                        const uint2 x = *reinterpret_cast<const uint2 *>(kr);
                        const uint2 y = *reinterpret_cast<const uint2 *>(kr + 8 * S::kCode);
                        k0[0] = x.x, k0[1] = x.y;
                        k1[0] = y.x, k1[1] = y.y;
                    }
                }
                const uint8_t *const ks = ring + S::kKsOff + (warp * 16 + g) * S::kScale;
                float s[NT][4];
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        s[t][j] = 0.f;
                if (!HIF4) {
                    uint32_t sw0, sw1;
                    if (D == 128) {
                        sw0 = *reinterpret_cast<const uint32_t *>(ks);
                        sw1 = *reinterpret_cast<const uint32_t *>(ks + 8 * S::kScale);
                    } else {
                        sw0 = *reinterpret_cast<const uint16_t *>(ks);
                        sw1 = *reinterpret_cast<const uint16_t *>(ks + 8 * S::kScale);
                    }
#pragma unroll
                    for (int b = 0; b < NB; ++b) {
                        uint32_t h0[4], h1[4];
                        e2m1x8_f16(k0[b], h0);
                        e2m1x8_f16(k1[b], h1);
                        const float f0 = e8m0_f32((sw0 >> (8 * b)) & 0xFFu), f1 = e8m0_f32((sw1 >> (8 * b)) & 0xFFu);
#pragma unroll
                        for (int t = 0; t < NT; ++t) {
                            const uint4 qb = NT == 1 ? qf[b] : s_q[(t * NB + b) * 32 + lane];
                            float tmp[4] = {0.f, 0.f, 0.f, 0.f};
                            mma_f16(tmp, h0[0], h1[0], h0[1], h1[1], qb.x, qb.y);
                            mma_f16(tmp, h0[2], h1[2], h0[3], h1[3], qb.z, qb.w);
                            s[t][0] = fmaf(tmp[0], f0, s[t][0]);
                            s[t][1] = fmaf(tmp[1], f0, s[t][1]);
                            s[t][2] = fmaf(tmp[2], f1, s[t][2]);
                            s[t][3] = fmaf(tmp[3], f1, s[t][3]);
                        }
                    }
                } else {
#pragma unroll
                    for (int bb = 0; bb < NB / 2; ++bb) {   // HiF4 blocks of 64
                        const uint32_t w0 = *reinterpret_cast<const uint32_t *>(ks + 4 * bb);
                        const uint32_t w1 = *reinterpret_cast<const uint32_t *>(ks + 8 * S::kScale + 4 * bb);
                        float tmp[NT][4];
#pragma unroll
                        for (int t = 0; t < NT; ++t)
#pragma unroll
                            for (int j = 0; j < 4; ++j)
                                tmp[t][j] = 0.f;
#pragma unroll
                        for (int hb = 0; hb < 2; ++hb) {
                            const int b = 2 * bb + hb;
                            uint32_t h0[4], h1[4], t0, t1;
                            s1p2x8_f16(k0[b], h0);
                            s1p2x8_f16(k1[b], h1);
                            hif4_pow2_pair(w0, 4 * hb + c, t0, t1);
                            h0[0] = hmul2(h0[0], t0), h0[1] = hmul2(h0[1], t0);
                            h0[2] = hmul2(h0[2], t1), h0[3] = hmul2(h0[3], t1);
                            hif4_pow2_pair(w1, 4 * hb + c, t0, t1);
                            h1[0] = hmul2(h1[0], t0), h1[1] = hmul2(h1[1], t0);
                            h1[2] = hmul2(h1[2], t1), h1[3] = hmul2(h1[3], t1);
#pragma unroll
                            for (int t = 0; t < NT; ++t) {
                                const uint4 qb = NT == 1 ? qf[b] : s_q[(t * NB + b) * 32 + lane];
                                mma_f16(tmp[t], h0[0], h1[0], h0[1], h1[1], qb.x, qb.y);
                                mma_f16(tmp[t], h0[2], h1[2], h0[3], h1[3], qb.z, qb.w);
                            }
                        }
                        const float f0 = hif4_macro_f32(w0), f1 = hif4_macro_f32(w1);
#pragma unroll
                        for (int t = 0; t < NT; ++t) {
                            s[t][0] = fmaf(tmp[t][0], f0, s[t][0]);
                            s[t][1] = fmaf(tmp[t][1], f0, s[t][1]);
                            s[t][2] = fmaf(tmp[t][2], f1, s[t][2]);
                            s[t][3] = fmaf(tmp[t][3], f1, s[t][3]);
                        }
                    }
                }
                // ---- softmax: s[t][j] is key g + 8 (j / 2), row 2 c + j % 2
                const bool masked = key0 < all_lo || key0 + 16 > all_hi;
                bool raise = false;
#pragma unroll
                for (int t = 0; t < NT; ++t) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        s[t][j] *= qs[t][j & 1];
                        if (masked) {
                            const int key = key0 + g + 8 * (j >> 1), h = hi[t][j & 1];
                            if (key >= h || (a.window > 0 && key < h - a.window))
                                s[t][j] = -INFINITY;
                        }
                    }
                    raise |= fmaxf(s[t][0], s[t][2]) > m[t][0] + 8.f || fmaxf(s[t][1], s[t][3]) > m[t][1] + 8.f;
                }
                if (__any_sync(0xFFFFFFFFu, raise)) {
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            float mx = fmaxf(s[t][j], s[t][j + 2]);
                            mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, 4));
                            mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, 8));
                            mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, 16));
                            mx = fmaxf(mx, m[t][j]);
                            const float f = m[t][j] == -INFINITY ? 0.f : ex2(m[t][j] - mx);
                            m[t][j] = mx;
                            l[t][j] *= f;
#pragma unroll
                            for (int i2 = 0; i2 < MT; ++i2) {
                                o[t][i2][j] *= f;
                                o[t][i2][j + 2] *= f;
                            }
                        }
                }
                uint32_t pb[NT][2];
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    float e[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j)   // (a row that has seen no key yet: m is -inf and so is s)
                        e[j] = ex2(s[t][j] - (m[t][j & 1] == -INFINITY ? 0.f : m[t][j & 1]));
                    l[t][0] += e[0] + e[2];
                    l[t][1] += e[1] + e[3];
                    pb[t][0] = movmatrix(pack_f16(e[0], e[1]));
                    pb[t][1] = movmatrix(pack_f16(e[2], e[3]));
                }
                // ---- values: keys 2c, 2c + 1 (v0) and 2c + 8, 2c + 9 (v1), dimensions g D/8 ..
                constexpr int VW = D / 64;    // words a key
                uint32_t v0[2 * VW], v1[2 * VW];
                {
                    const uint8_t *const vr = ring + S::kVOff + warp * 8 * D + lane * (D / 8);
                    if (D == 128) {
                        const uint4 x = *reinterpret_cast<const uint4 *>(vr);
                        const uint4 y = *reinterpret_cast<const uint4 *>(vr + 4 * D);
                        v0[0] = x.x, v0[1] = x.y, v0[2 * VW - 2] = x.z, v0[2 * VW - 1] = x.w;
                        v1[0] = y.x, v1[1] = y.y, v1[2 * VW - 2] = y.z, v1[2 * VW - 1] = y.w;
                    } else {
                        const uint2 x = *reinterpret_cast<const uint2 *>(vr);
                        const uint2 y = *reinterpret_cast<const uint2 *>(vr + 4 * D);
                        v0[0] = x.x, v0[1] = x.y;
                        v1[0] = y.x, v1[1] = y.y;
                    }
                }
                const uint8_t *const vs = ring + S::kVsOff + (warp * 16 + 2 * c) * S::kScale;
                int ve[4];                    // exponents (MXFP4: byte; HiF4: E) of the four keys
                uint32_t vm[4];               // HiF4 metadata
                int top = -2000;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int tok = (j & 1) + 8 * (j >> 1), key = key0 + 2 * c + tok;
                    const bool seen = key < walk.ke && key >= walk.kb;
                    if (HIF4) {
                        vm[j] = *reinterpret_cast<const uint32_t *>(vs + tok * S::kScale + (g * (D / 8) / 64) * 4);
                        vm[j] = seen ? vm[j] : 0u;
                        ve[j] = seen ? (int)((vm[j] >> 2) & 63u) : -2000;
                    } else {
                        ve[j] = seen ? (int)vs[tok * S::kScale + g * (D / 8) / 32] : -2000;
                    }
                    top = max(top, ve[j]);
                }
                if (__any_sync(0xFFFFFFFFu, top > vref + 3)) {
                    top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
                    top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
                    top = max(top, vref);
                    const float f = ex2((float)(vref - top));
                    vref = top;
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int i2 = 0; i2 < MT; ++i2)
#pragma unroll
                            for (int j = 0; j < 4; ++j)
                                o[t][i2][j] *= f;
                }
                // f16 scale of each key: 2^(e - vref + 9)
                uint32_t sc[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    uint32_t x[2];
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const int f = ve[2 * j + k] - vref + 24;
                        x[k] = f > 0 ? ((uint32_t)f << 10) | (HIF4 ? (vm[2 * j + k] & 3u) << 8 : 0u) : 0u;
                    }
                    sc[j] = x[0] | (x[1] << 16);
                }
#pragma unroll
                for (int w = 0; w < VW; ++w) {
                    uint32_t a0[4], a1[4], a2[4], a3[4];   // even and odd dimensions of keys 2c ..; of keys 2c + 8 ..
                    if (!HIF4) {
                        const uint32_t x0 = v0[w], x1 = v0[VW + w], y0 = v1[w], y1 = v1[VW + w];
                        e2m1x8_f16((x0 & 0x0F0F0F0Fu) | ((x1 << 4) & 0xF0F0F0F0u), a0);
                        e2m1x8_f16(((x0 >> 4) & 0x0F0F0F0Fu) | (x1 & 0xF0F0F0F0u), a1);
                        e2m1x8_f16((y0 & 0x0F0F0F0Fu) | ((y1 << 4) & 0xF0F0F0F0u), a2);
                        e2m1x8_f16(((y0 >> 4) & 0x0F0F0F0Fu) | (y1 & 0xF0F0F0F0u), a3);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            a0[j] = hmul2(a0[j], sc[0]), a1[j] = hmul2(a1[j], sc[0]);
                            a2[j] = hmul2(a2[j], sc[1]), a3[j] = hmul2(a3[j], sc[1]);
                        }
                    } else {
#pragma unroll
                        for (int kk = 0; kk < 2; ++kk) {
                            const uint32_t x0 = kk ? v1[w] : v0[w], x1 = kk ? v1[VW + w] : v0[VW + w];
                            uint32_t(&ev)[4] = kk ? a2 : a0;
                            uint32_t(&od)[4] = kk ? a3 : a1;
                            const uint32_t e0 = s1p2_even_bytes(x0), e1 = s1p2_even_bytes(x1);
                            const uint32_t o0 = s1p2_odd_bytes(x0), o1 = s1p2_odd_bytes(x1);
                            const uint32_t ea = __byte_perm(e0, e1, 0x5140), eb = __byte_perm(e0, e1, 0x7362);
                            const uint32_t oa = __byte_perm(o0, o1, 0x5140), ob = __byte_perm(o0, o1, 0x7362);
                            ev[0] = e4m3x2_f16(ea), ev[1] = e4m3x2_f16(ea >> 16);
                            ev[2] = e4m3x2_f16(eb), ev[3] = e4m3x2_f16(eb >> 16);
                            od[0] = e4m3x2_f16(oa), od[1] = e4m3x2_f16(oa >> 16);
                            od[2] = e4m3x2_f16(ob), od[3] = e4m3x2_f16(ob >> 16);
                            // sub-group exponents of both keys, added to the scale's exponent field
                            const int gi = (g * (D / 8) / 8) % 8 + w;     // group of 8 in the 64-element block
                            const uint32_t m0 = vm[2 * kk], m1 = vm[2 * kk + 1];
                            const uint32_t e8 = ((m0 >> (8 + gi)) & 1u) | (((m1 >> (8 + gi)) & 1u) << 16);
                            const uint32_t q0 = m0 >> (16 + 2 * gi), q1 = m1 >> (16 + 2 * gi);
                            const uint32_t ta = e8 + ((q0 & 1u) | ((q1 & 1u) << 16));
                            const uint32_t tb = e8 + (((q0 >> 1) & 1u) | (((q1 >> 1) & 1u) << 16));
                            const uint32_t sa = sc[kk] + (ta << 10), sb = sc[kk] + (tb << 10);
                            ev[0] = hmul2(ev[0], sa), od[0] = hmul2(od[0], sa);
                            ev[1] = hmul2(ev[1], sa), od[1] = hmul2(od[1], sa);
                            ev[2] = hmul2(ev[2], sb), od[2] = hmul2(od[2], sb);
                            ev[3] = hmul2(ev[3], sb), od[3] = hmul2(od[3], sb);
                        }
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j)
#pragma unroll
                        for (int t = 0; t < NT; ++t)
                            mma_f16(o[t][4 * w + j], a0[j], a1[j], a2[j], a3[j], pb[t][0], pb[t][1]);
                }
            }
            __syncwarp();
            if (lane == 0)
                mbar_arrive(&s_empty[st]);
        }

        // ---- join the warps
        const float vunit = scalbnf(1.f, vref - (HIF4 ? 50 : 136));
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                float x = l[t][j];
                x += __shfl_xor_sync(0xFFFFFFFFu, x, 4);
                x += __shfl_xor_sync(0xFFFFFFFFu, x, 8);
                x += __shfl_xor_sync(0xFFFFFFFFu, x, 16);
                if (g == 0) {
                    s_m[warp][8 * t + 2 * c + j] = m[t][j];
                    s_l[warp][8 * t + 2 * c + j] = x;
                }
            }
        const bool whole = walk.i0 == 0 && walk.i1 == walk.units;
        const long long seg0 = walk.u - walk.i0;
        const int c0 = (int)(((seg0 + 1) * ctas - 1) / total), c1 = (int)(((seg0 + walk.units) * ctas - 1) / total);
        const int slot = 2 * cta + (walk.i0 == 0 ? 1 : 0);
        constexpr int VPR = D / 4;            // float4 a row
        const int mrow = tid / VPR, mcol = tid % VPR;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    *reinterpret_cast<float2 *>(s_merge + (warp * 8 + 2 * c + j) * D + g * (D / 8) + 2 * i) =
                        make_float2(o[t][i][j] * vunit, o[t][i][j + 2] * vunit);
            consumer_sync();
            if (mrow < 8) {
                const int row = 8 * t + mrow;
                float mx = -INFINITY;
#pragma unroll
                for (int w = 0; w < kConsumers; ++w)
                    mx = fmaxf(mx, s_m[w][row]);
                float sum = 0.f;
                float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int w = 0; w < kConsumers; ++w) {
                    const float f = s_m[w][row] == -INFINITY ? 0.f : ex2(s_m[w][row] - mx);
                    const float4 y = *reinterpret_cast<const float4 *>(s_merge + (w * 8 + mrow) * D + 4 * mcol);
                    sum = fmaf(f, s_l[w][row], sum);
                    x.x = fmaf(f, y.x, x.x), x.y = fmaf(f, y.y, x.y);
                    x.z = fmaf(f, y.z, x.z), x.w = fmaf(f, y.w, x.w);
                }
                if (!whole) {
                    const int64_t at = (int64_t)slot * ROWS + row;
                    __stcg(reinterpret_cast<float4 *>(p.part_o + at * D + 4 * mcol), x);
                    if (mcol == 0)
                        __stcg(reinterpret_cast<float2 *>(p.part_ml + at * 2), make_float2(mx, sum));
                } else if (row < rows) {
                    const int ri = row0 + row;
                    const int64_t at = (int64_t)(q.q0 + ri / G) * a.heads + walk.head * G + ri % G;
                    const float inv = sum > 0.f ? 1.f / sum : 0.f;
                    const __nv_bfloat162 lo = __floats2bfloat162_rn(x.x * inv, x.y * inv);
                    const __nv_bfloat162 up = __floats2bfloat162_rn(x.z * inv, x.w * inv);
                    *reinterpret_cast<uint2 *>(static_cast<__nv_bfloat16 *>(a.out) + at * D + 4 * mcol) = make_uint2(
                        *reinterpret_cast<const uint32_t *>(&lo), *reinterpret_cast<const uint32_t *>(&up));
                    if (a.lse && mcol == 0)
                        a.lse[at] = sum > 0.f ? (mx + log2f(sum)) * 0.69314718055994531f : -INFINITY;
                }
            }
            consumer_sync();
        }
        if (whole)
            continue;
        // ---- a split segment: the last of its CTAs adds the parts
        __threadfence();
        consumer_sync();
        if (tid == 0)
            s_flag = atomicAdd(p.counter + c0, 1) == c1 - c0;
        consumer_sync();
        if (s_flag) {
            __threadfence();
            for (int i = tid; i < rows * VPR; i += 32 * kConsumers) {
                const int row = i / VPR, col = i % VPR;
                float mx = -INFINITY;
                for (int k = c0; k <= c1; ++k)
                    mx = fmaxf(mx, __ldcg(p.part_ml + ((int64_t)(2 * k + (k == c0)) * ROWS + row) * 2));
                float sum = 0.f;
                float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
                for (int k = c0; k <= c1; ++k) {
                    const int64_t at = (int64_t)(2 * k + (k == c0)) * ROWS + row;
                    const float2 ml = __ldcg(reinterpret_cast<const float2 *>(p.part_ml + at * 2));
                    const float4 y = __ldcg(reinterpret_cast<const float4 *>(p.part_o + at * D + 4 * col));
                    const float f = ml.x == -INFINITY ? 0.f : ex2(ml.x - mx);
                    sum = fmaf(f, ml.y, sum);
                    x.x = fmaf(f, y.x, x.x), x.y = fmaf(f, y.y, x.y);
                    x.z = fmaf(f, y.z, x.z), x.w = fmaf(f, y.w, x.w);
                }
                const int ri = row0 + row;
                const int64_t at = (int64_t)(q.q0 + ri / G) * a.heads + walk.head * G + ri % G;
                const float inv = sum > 0.f ? 1.f / sum : 0.f;
                const __nv_bfloat162 lo = __floats2bfloat162_rn(x.x * inv, x.y * inv);
                const __nv_bfloat162 up = __floats2bfloat162_rn(x.z * inv, x.w * inv);
                *reinterpret_cast<uint2 *>(static_cast<__nv_bfloat16 *>(a.out) + at * D + 4 * col) = make_uint2(
                    *reinterpret_cast<const uint32_t *>(&lo), *reinterpret_cast<const uint32_t *>(&up));
                if (a.lse && col == 0)
                    a.lse[at] = sum > 0.f ? (mx + log2f(sum)) * 0.69314718055994531f : -INFINITY;
            }
            if (tid == 0)
                atomicExch(p.counter + c0, 0);
        }
        consumer_sync();
    }
}

constexpr int kMaxRows = 32, kMaxBlocksPerSm = 2;
constexpr size_t kWsCounters = 256;

size_t ws_parts_offset() { return kWsCounters + ((size_t)kMaxBlocksPerSm * num_sms() * 4 + 255) / 256 * 256; }

template <int FMT, int D, int NT>
cudaError_t launch(const KvAttentionArgs &a, cudaStream_t st)
{
    using S = Shape<FMT, D, NT>;
    static_assert(S::kStages >= 3, "the ring holds at least three stages");
    static bool ready = false;     // (per instantiation; setting it twice is harmless)
    if (!ready) {
        if (cudaError_t e = cudaFuncSetAttribute(kv_attention_kernel<FMT, D, NT>,
                                                 cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem))
            return e;
        ready = true;
    }
    const int ctas = S::kBlocksPerSm * num_sms();
    uint8_t *const ws = static_cast<uint8_t *>(a.workspace);
    Params p;
    p.a = a;
    p.group = a.heads / a.cache.heads;
    p.gran = a.cache.page_size & -a.cache.page_size;
    p.gran = p.gran < kUnit ? p.gran : kUnit;
    p.status = static_cast<int32_t *>(a.workspace);
    p.counter = reinterpret_cast<int32_t *>(ws + kWsCounters);
    p.part_o = reinterpret_cast<float *>(ws + ws_parts_offset());
    p.part_ml = p.part_o + (int64_t)2 * ctas * S::kRows * D;
    kv_attention_kernel<FMT, D, NT><<<ctas, kThreads, S::kSmem, st>>>(p);
    return cudaGetLastError();
}

template <int FMT, int D>
cudaError_t launch_rows(const KvAttentionArgs &a, cudaStream_t st)
{
    // rows of a request and key head: the group's heads times its new tokens
    const int64_t per = a.q_start ? (a.tokens + a.requests - 1) / a.requests : 1;
    const int64_t rows = per * (a.heads / a.cache.heads);
    return rows <= 8 ? launch<FMT, D, 1>(a, st) : rows <= 16 ? launch<FMT, D, 2>(a, st) : launch<FMT, D, 4>(a, st);
}

} // namespace

size_t kv_attention_workspace_bytes(int32_t heads, int32_t head_dim)
{
    (void)heads;
    return ws_parts_offset() + (size_t)2 * kMaxBlocksPerSm * num_sms() * kMaxRows * (head_dim + 2) * 4;
}

cudaError_t launch_kv_attention(const KvAttentionArgs &a, cudaStream_t st)
{
    const bool wide = a.cache.head_dim == 128;
    if (a.cache.fmt == RFQ_FMT_HIF4)
        return wide ? launch_rows<RFQ_FMT_HIF4, 128>(a, st) : launch_rows<RFQ_FMT_HIF4, 64>(a, st);
    return wide ? launch_rows<RFQ_FMT_MXFP4, 128>(a, st) : launch_rows<RFQ_FMT_MXFP4, 64>(a, st);
}

} // namespace rfq
