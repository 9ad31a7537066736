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
//   P: exp2(s - m) rounded to f16 (its sum l stays fp32), m 7 below the
//      maximum when it is set and raised only when a score passes it by 15:
//      weights down to 2^-21 of the largest are off by 2^-11 of themselves,
//      smaller ones by 2^-32 of the largest.
//   V: codes times scale relative to a running power of two, exact in f16
//      while the scales of one 32-dimension block span less than 2^24 over
//      the keys seen so far; smaller ones fade out (HiF4: but for their
//      sub-group exponents, which make 2^-21 of the largest scale at most;
//      taking those out as well costs 2% of a long request).
//
// Bound: HBM at long caches: 136 (MXFP4) or 144 (HiF4) bytes a key and head
// of 128.  An SM's share of the measured copy rate is one of these every 5.8
// clocks, so a key may cost at most 23 warp instructions, 11 of them on the
// pipe that converts codes.
//
// Work: the (request, key head, row tile) segments of all requests laid end
// to end, in chunks of 32 keys and one more unit a segment for its start, are
// split evenly over the CTAs (one a SM) and there over the warps, however
// ragged the lengths.  A warp copies the chunks of its run (contiguous pieces
// of pages) into its own small ring and waits for no other warp.  It writes
// the segments that it holds whole; the parts of others wait in shared memory
// for the CTA's end, when all warps join them, and the parts of segments that
// CTAs share go to the workspace, where the last CTA to finish joins them.
// The split and the order of every sum depend on the lengths alone: a call
// gives the same bits every time.
//
// Measured, 32 heads on 8, D = 128: 8 requests of 98304 to 131072 keys, MXFP4
// 218 us, 4.5 TB/s, 67% of the copy rate; HiF4, whose codes take more
// instructions to decode, 351 us at 44%.  One request of 777 keys: 10.4 us,
// the latency of its dependent steps.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <algorithm>
#include <cstdint>

#include "kv_attention.cuh"
#include "kv_layout.cuh"
#include "mxfp4_math.cuh"

namespace rfq {
namespace {

constexpr int kLeast = 8;                    // units of a CTA, at least
constexpr int kHalves = 2;                   // MMA tiles of 16 keys in a chunk

__device__ __forceinline__ uint32_t movmatrix(uint32_t a)
{
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(a));
    return r;
}

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi)
{
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}

template <int FMT, int D, int NT>
struct Shape {
    // 12 warps leave a thread 168 registers: with 16 the loop over the keys
    // spills at D = 128 (323 us against 230 at 8 x 131072 keys, MXFP4), and
    // eight hide less latency (275 us)
    static constexpr int kWarps = NT > 1 ? 8 : D == 64 ? 16 : 12, kThreads = 32 * kWarps;
    static constexpr int kRows = 8 * NT, kMt = D / 16, kChunk = 16 * kHalves, kStart = 1;
    static constexpr int kScale = FMT == RFQ_FMT_HIF4 ? D / 16 : D / 32;   // bytes a token
    static constexpr int kCode = D / 2;
    static constexpr int kVOff = kChunk * kCode, kKsOff = 2 * kVOff, kVsOff = kKsOff + kChunk * kScale;
    static constexpr int kBytes = kVsOff + kChunk * kScale;                // of a chunk
    static constexpr int kDepth = D == 64 ? 4 : 3;                              // chunks in a warp's ring
    // a part: NT D/16 float4 a lane, and a float4 (m, m, l, l) a lane and column tile
    static constexpr int kPart = NT * (kMt + 1) * 512;
    static constexpr int kQ = NT > 1 ? NT * D * 16 : 0;                    // of a warp
    static constexpr int kSmem = kWarps * (kDepth * kBytes + kPart + kQ);
    static_assert(kDepth * kBytes >= kPart, "a warp's last part lies over its ring");
};

// One warp's share of a row tile: O^T (dimensions g D/8 + 2i and + 1 by rows
// 2c, 2c + 1), the running maxima and the sums of weights.
template <int D, int NT>
struct Sums {
    static constexpr int MT = D / 16;
    float o[NT][MT][4], m[NT][2], l[NT][2];
    __device__ __forceinline__ void clear()
    {
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
    }
    // as a part, in shared memory
    __device__ __forceinline__ void store(uint8_t *dst, int lane) const
    {
        float4 *const d = reinterpret_cast<float4 *>(dst);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int i = 0; i < MT; ++i)
                d[(t * MT + i) * 32 + lane] = make_float4(o[t][i][0], o[t][i][1], o[t][i][2], o[t][i][3]);
            d[(NT * MT + t) * 32 + lane] = make_float4(m[t][0], m[t][1], l[t][0], l[t][1]);
        }
    }
    // adds a part
    __device__ __forceinline__ void join(const uint8_t *src, int lane)
    {
        const float4 *const d = reinterpret_cast<const float4 *>(src);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const float4 ml = d[(NT * MT + t) * 32 + lane];
            const float mm[2] = {ml.x, ml.y}, ll[2] = {ml.z, ml.w};
            float fa[2], fb[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float top = fmaxf(m[t][j], mm[j]);
                fa[j] = m[t][j] == -INFINITY ? 0.f : ex2(m[t][j] - top);
                fb[j] = mm[j] == -INFINITY ? 0.f : ex2(mm[j] - top);
                l[t][j] = l[t][j] * fa[j] + ll[j] * fb[j];
                m[t][j] = top;
            }
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                const float4 v = d[(t * MT + i) * 32 + lane];
                o[t][i][0] = o[t][i][0] * fa[0] + v.x * fb[0];
                o[t][i][1] = o[t][i][1] * fa[1] + v.y * fb[1];
                o[t][i][2] = o[t][i][2] * fa[0] + v.z * fb[0];
                o[t][i][3] = o[t][i][3] * fa[1] + v.w * fb[1];
            }
        }
    }
};

// What a warp left of a segment that it does not hold whole.
struct PartInfo {
    uint32_t seg;              // the segment's first unit
    int chunks, head, row0, rows, q0;
    int begins, ends;          // holds its first chunk, its last
};
constexpr uint32_t kNoPart = 0xFFFFFFFFu;

// One lane's share of the joined parts of column tile t: four sums, of
// dimensions g D/8 + 2i, + 1 and rows 2c, 2c + 1.
struct Joined {
    float o[4], m[2], l[2];
    __device__ __forceinline__ void clear()
    {
        o[0] = o[1] = o[2] = o[3] = l[0] = l[1] = 0.f;
        m[0] = m[1] = -INFINITY;
    }
    __device__ __forceinline__ void add(const float4 &v, const float4 &ml)
    {
        const float mm[2] = {ml.x, ml.y}, ll[2] = {ml.z, ml.w}, vv[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const float top = fmaxf(m[j], mm[j]);
            const float fa = m[j] == -INFINITY ? 0.f : ex2(m[j] - top), fb = mm[j] == -INFINITY ? 0.f : ex2(mm[j] - top);
            l[j] = l[j] * fa + ll[j] * fb;
            o[j] = o[j] * fa + vv[j] * fb;
            o[j + 2] = o[j + 2] * fa + vv[j + 2] * fb;
            m[j] = top;
        }
    }
};

template <int FMT, int D, int NT>
__global__ void __launch_bounds__(Shape<FMT, D, NT>::kThreads, 1)
    kv_attention_kernel(const __grid_constant__ AttnParams p)
{
    using S = Shape<FMT, D, NT>;
    constexpr bool HIF4 = FMT == RFQ_FMT_HIF4;
    constexpr int NB = D / 32, ROWS = S::kRows, MT = S::kMt, W = S::kWarps, DEPTH = S::kDepth, HV = kHalves, kChunk = S::kChunk;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ alignas(8) uint64_t s_full[W][DEPTH];
    __shared__ uint32_t s_scan[W];
    __shared__ int s_flag[2];
    __shared__ int2 s_c[2];
    __shared__ PartInfo s_info[W][2];        // of its first segment, of its last

    const KvAttentionArgs &a = p.a;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, c = lane & 3;
    const int H = a.cache.heads, G = p.group;
    uint8_t *const s_ring = smem + warp * DEPTH * S::kBytes;
    uint4 *const s_q = reinterpret_cast<uint4 *>(smem + W * DEPTH * S::kBytes + warp * S::kQ);
    // the parts of a warp's first segment (k = 0) and of its last (k = 1)
    auto part_of = [&](int w, int k) -> uint8_t * {
        return k ? smem + w * DEPTH * S::kBytes : smem + W * (DEPTH * S::kBytes + S::kQ) + w * S::kPart;
    };

    if (lane < 2)
        s_info[warp][lane].seg = kNoPart;
    if (lane == 0) {
#pragma unroll
        for (int i = 0; i < DEPTH; ++i)
            mbar_init(&s_full[warp][i], 1);
        fence_mbar_init();
    }
    wait_for_previous();
    let_next_start();
    // ---- this warp's share of the units of all requests, in order
    Share sh;
    if (!find_share<S>(p, s_scan, W, kLeast, sh))
        return;
    const uint32_t total = sh.total, ctas = sh.ctas, cta = blockIdx.x;
    Walk<S> walk, ahead;                  // what is computed, and what is copied
    walk.start(p, sh.r, sh.rem, sh.first, sh.last, lane);
    walk.next(p);
    ahead = walk;
    const uint64_t limit = ws_wait_limit_ns(p.status);
    bool ok = true;                          // no wait of this warp has run out

    // ---- copies: chunk ahead.i of segment `ahead` into slot fslot of this
    // warp's ring.  Lane (h, array), h < 32 / gran, copies keys 16 h .. of one
    // array; it keeps its place in the block table from chunk to chunk.
    const int arr = lane & 3, page_size = a.cache.page_size;
    const uint32_t unit = arr < 2 ? S::kCode : S::kScale;              // bytes a key
    const uint8_t *const src = static_cast<const uint8_t *>(arr == 0   ? a.cache.k_codes
                                                            : arr == 1 ? a.cache.v_codes
                                                            : arr == 2 ? a.cache.k_scales
                                                                       : a.cache.v_scales);
    const uint32_t dst = smem_u32(s_ring) + (arr == 0 ? 0 : arr == 1 ? S::kVOff : arr == 2 ? S::kKsOff : S::kVsOff) +
                         (lane >> 2) * 16 * unit;
    const uint32_t bytes = p.gran * unit;
    const uint64_t page_bytes = (uint64_t)H * page_size * unit;
    const bool copies = (lane >> 2) < kChunk / p.gran;
    const int32_t *entry = a.table;          // of the page of this lane's next key
    uint32_t off = 0;                        // that key in its page
    int key = 0;
    const uint8_t *from = src;               // the key head's bytes in page 0
    int page = -1;                           // *entry, read a chunk before it is used
    auto read_page = [&]() {
        if (copies && ahead.more() && key < ahead.ke)
            page = *entry;
    };
    auto place = [&]() {
        key = ahead.kb + ahead.i * kChunk + (lane >> 2) * 16;
        const uint32_t pg = (uint32_t)key / (uint32_t)page_size;
        off = key - pg * page_size;
        entry = a.table + (int64_t)ahead.r * a.width + pg;
        from = src + (uint64_t)ahead.head * page_size * unit;
        read_page();
    };
    int fslot = 0;
    if (walk.more())
        place();
    auto fetch = [&]() {
        if (!ahead.more())
            return;
        bool have = copies && key < ahead.ke;
        if (have && (page < 0 || page >= a.cache.pages)) {
            atomicCAS(p.status, kDevOk, kDevBadGroups);
            have = false;
        }
        const uint32_t granules = __popc(__ballot_sync(kAll, have)) >> 2;
        if (lane == 0)
            mbar_arrive_expect_tx(&s_full[warp][fslot], granules * p.gran * (2 * S::kCode + 2 * S::kScale));
        __syncwarp();
        if (have)
            bulk_load_at(dst + fslot * S::kBytes, from + page * page_bytes + off * unit, bytes, &s_full[warp][fslot]);
        if (++fslot == DEPTH)
            fslot = 0;
        if (++ahead.i == ahead.i1) {
            ahead.next(p);
            if (ahead.more())
                place();
            return;
        }
        key += kChunk;
        off += kChunk;
        if (off >= (uint32_t)page_size) {
            off -= page_size;
            ++entry;
            if (off >= (uint32_t)page_size) {    // (a page of 16 is shorter than a chunk)
                off -= page_size;
                ++entry;
            }
            read_page();
        }
    };
    // z, one lane's share of a segment's sums, to the output
    Sums<D, NT> z;
    auto write = [&](int row0, int rows, int q0, int head) {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int row = 8 * t + 2 * c + j, ri = row0 + row;
                if (row >= rows)
                    continue;
                const int64_t at = (int64_t)(q0 + ri / G) * a.heads + head * G + ri % G;
                const float inv = inverse(z.l[t][j]);
                uint32_t w[MT];
#pragma unroll
                for (int i = 0; i < MT; ++i)
                    w[i] = pack_bf16(z.o[t][i][j] * inv, z.o[t][i][j + 2] * inv);
                uint4 *const d = reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(a.out) + at * D + g * (D / 8));
#pragma unroll
                for (int i = 0; i < MT / 4; ++i)
                    d[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
                if (a.lse && g == 0)
                    a.lse[at] = log_sum(z.m[t][j], z.l[t][j]);
            }
    };
    int slot = 0, warm = DEPTH - 1;          // chunks to copy before the first is computed
    uint32_t parity = 0;
    bool fresh = true, loaded = false;       // a segment begins; its rows of q are on their way
    bool begins = walk.i == 0;
    Request q = {0, 0, 0};
    int row0 = 0, rows = 0;
    uint4 raw[NB];                           // eight of them, as they come and then as f16
    auto read_q = [&](int t) {
        const int rr = 8 * t + g, ri = row0 + rr, tok = ri / G;
        const __nv_bfloat16 *const at = static_cast<const __nv_bfloat16 *>(a.q) + (q.q0 + tok) * a.q_token +
                                        (int64_t)(walk.head * G + ri - tok * G) * a.q_head + 8 * c;
#pragma unroll
        for (int b = 0; b < NB; ++b)
            raw[b] = rr < rows ? *reinterpret_cast<const uint4 *>(at + 32 * b) : make_uint4(0, 0, 0, 0);
    };
    float qs[NT][2];
    int hi[NT][2];                           // keys that the thread's two rows see: [max(0, hi - window), hi)
    int all_hi = 0, all_lo = 0, least = 0;   // every row sees [all_lo, all_hi), none a key below least
    int vref = -1000;                        // V scale exponents are relative to it (the same in a row's quad)
#ifdef RFQ_DEBUG_BOUNDS
    // (the held start, by which a test makes a wait run out with nothing in flight,
    // costs 0.3 us of a short request: the debug build alone has it)
    ok = __all_sync(kAll, held_start_wait(p.status, limit));
#endif
#pragma unroll 1
    while (ok && walk.more()) {
        // the segment's rows of q, on their way while chunks are copied (of one
        // row tile: more would take the registers)
        if (fresh && !loaded) {
            loaded = true;
            begins = walk.i == 0;
            q = walk.q;
            row0 = walk.tile * ROWS;
            rows = min(ROWS, q.n * G - row0);
            if (NT == 1)
                read_q(0);
        }
        fetch();
        if (warm > 0) {
            --warm;
            continue;
        }
        if (fresh) {
            fresh = loaded = false;
            // ---- q as f16, scaled by a power of two per row
            const float base = a.scale * 1.4426950408889634f * (HIF4 ? 128.f : 1.f);
            __syncwarp();                     // (the rows of the segment before are done with)
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                if (NT > 1)
                    read_q(t);
                float mx = 0.f;
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    const uint32_t w[4] = {raw[b].x, raw[b].y, raw[b].z, raw[b].w};
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        mx = fmaxf(mx, fmaxf(fabsf(__uint_as_float(w[j] << 16)),
                                             fabsf(__uint_as_float(w[j] & 0xFFFF0000u))));
                }
                mx = fmaxf(mx, __shfl_xor_sync(kAll, mx, 1));
                mx = fmaxf(mx, __shfl_xor_sync(kAll, mx, 2));
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
                    raw[b] = make_uint4(h[0], h[1], h[2], h[3]);
                    if (NT > 1)
                        s_q[(t * NB + b) * 32 + lane] = raw[b];
                }
                qs[t][0] = __shfl_sync(kAll, undo, 8 * c);
                qs[t][1] = __shfl_sync(kAll, undo, 8 * c + 4);
            }
            __syncwarp();
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int ri = row0 + min(8 * t + 2 * c + j, rows - 1);
                    hi[t][j] = max(0, q.L - q.n + (q.n > 1 ? ri / G : 0) + 1);
                }
            all_hi = max(0, q.L - q.n + (q.n > 1 ? row0 / G : 0) + 1);
            least = first_seen(all_hi, a.window);
            all_lo = first_seen(q.L - q.n + (q.n > 1 ? (row0 + rows - 1) / G : 0) + 1, a.window);
            z.clear();
            vref = -1000;
        }

        // ---- one chunk
        {
            const int i = walk.i;
            const bool here = mbar_wait(&s_full[warp][slot], parity, limit);
            const int key0 = walk.kb + i * kChunk;
            const uint8_t *const ring = s_ring + slot * S::kBytes;
            // ---- scores: s[h][t][j] is key 16 h + g + 8 (j / 2), row 8 t + 2 c + j % 2
            float s[HV][NT][4];
            uint32_t kw[HV][2][NB];            // [h][row g, g + 8][sub-block]
#pragma unroll
            for (int h = 0; h < HV; ++h)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const uint8_t *const kr = ring + (16 * h + 8 * r + g) * S::kCode + c * NB * 4;
                    if (D == 128) {
                        const uint4 x = *reinterpret_cast<const uint4 *>(kr);
                        kw[h][r][0] = x.x, kw[h][r][1] = x.y, kw[h][r][NB - 2] = x.z, kw[h][r][NB - 1] = x.w;
                    } else {
                        const uint2 x = *reinterpret_cast<const uint2 *>(kr);
                        kw[h][r][0] = x.x, kw[h][r][1] = x.y;
                    }
                }
            const uint8_t *const ks = ring + S::kKsOff + g * S::kScale;
            if (!HIF4) {
                uint32_t sw[HV][2];
#pragma unroll
                for (int h = 0; h < HV; ++h)
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const uint8_t *const q8 = ks + (16 * h + 8 * r) * S::kScale;
                        sw[h][r] = D == 128 ? *reinterpret_cast<const uint32_t *>(q8)
                                            : *reinterpret_cast<const uint16_t *>(q8);
                    }
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    uint32_t k0[HV][4], k1[HV][4];
                    float f0[HV], f1[HV];
#pragma unroll
                    for (int h = 0; h < HV; ++h) {
                        e2m1x8_f16(kw[h][0][b], k0[h]);
                        e2m1x8_f16(kw[h][1][b], k1[h]);
                        f0[h] = e8m0_byte(sw[h][0], b);
                        f1[h] = e8m0_byte(sw[h][1], b);
                    }
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        const uint4 qb = NT == 1 ? raw[b] : s_q[(t * NB + b) * 32 + lane];
#pragma unroll
                        for (int h = 0; h < HV; ++h) {
                            float tmp[4];
                            mma_f16_first(tmp, k0[h][0], k1[h][0], k0[h][1], k1[h][1], qb.x, qb.y);
                            mma_f16(tmp, k0[h][2], k1[h][2], k0[h][3], k1[h][3], qb.z, qb.w);
                            if (b == 0) {
                                s[h][t][0] = tmp[0] * f0[h], s[h][t][1] = tmp[1] * f0[h];
                                s[h][t][2] = tmp[2] * f1[h], s[h][t][3] = tmp[3] * f1[h];
                            } else {
                                s[h][t][0] = fmaf(tmp[0], f0[h], s[h][t][0]);
                                s[h][t][1] = fmaf(tmp[1], f0[h], s[h][t][1]);
                                s[h][t][2] = fmaf(tmp[2], f1[h], s[h][t][2]);
                                s[h][t][3] = fmaf(tmp[3], f1[h], s[h][t][3]);
                            }
                        }
                    }
                }
            } else {
#pragma unroll
                for (int bb = 0; bb < NB / 2; ++bb) {   // HiF4 blocks of 64
                    float tmp[HV][NT][4];
                    uint32_t meta[HV][2];
#pragma unroll
                    for (int h = 0; h < HV; ++h)
#pragma unroll
                        for (int r = 0; r < 2; ++r)
                            meta[h][r] =
                                *reinterpret_cast<const uint32_t *>(ks + (16 * h + 8 * r) * S::kScale + 4 * bb);
#pragma unroll
                    for (int hb = 0; hb < 2; ++hb) {
                        const int b = 2 * bb + hb;
                        uint32_t k0[HV][4], k1[HV][4];
#pragma unroll
                        for (int h = 0; h < HV; ++h) {
                            uint32_t t0, t1;
                            s1p2x8_f16(kw[h][0][b], k0[h]);
                            hif4_pow2_pair(meta[h][0], 4 * hb + c, t0, t1);
                            k0[h][0] = hmul2(k0[h][0], t0), k0[h][1] = hmul2(k0[h][1], t0);
                            k0[h][2] = hmul2(k0[h][2], t1), k0[h][3] = hmul2(k0[h][3], t1);
                            s1p2x8_f16(kw[h][1][b], k1[h]);
                            hif4_pow2_pair(meta[h][1], 4 * hb + c, t0, t1);
                            k1[h][0] = hmul2(k1[h][0], t0), k1[h][1] = hmul2(k1[h][1], t0);
                            k1[h][2] = hmul2(k1[h][2], t1), k1[h][3] = hmul2(k1[h][3], t1);
                        }
#pragma unroll
                        for (int t = 0; t < NT; ++t) {
                            const uint4 qb = NT == 1 ? raw[b] : s_q[(t * NB + b) * 32 + lane];
#pragma unroll
                            for (int h = 0; h < HV; ++h) {
                                if (hb == 0)
                                    mma_f16_first(tmp[h][t], k0[h][0], k1[h][0], k0[h][1], k1[h][1], qb.x, qb.y);
                                else
                                    mma_f16(tmp[h][t], k0[h][0], k1[h][0], k0[h][1], k1[h][1], qb.x, qb.y);
                                mma_f16(tmp[h][t], k0[h][2], k1[h][2], k0[h][3], k1[h][3], qb.z, qb.w);
                            }
                        }
                    }
#pragma unroll
                    for (int h = 0; h < HV; ++h) {
                        const float f0 = hif4_macro_f32(meta[h][0]), f1 = hif4_macro_f32(meta[h][1]);
#pragma unroll
                        for (int t = 0; t < NT; ++t)
#pragma unroll
                            for (int j = 0; j < 4; ++j)
                                s[h][t][j] = bb == 0 ? tmp[h][t][j] * (j < 2 ? f0 : f1)
                                                     : fmaf(tmp[h][t][j], j < 2 ? f0 : f1, s[h][t][j]);
                    }
                }
            }
            // ---- softmax
            const bool whole = key0 >= all_lo && key0 + kChunk <= all_hi;   // every row sees every key
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int h = 0; h < HV; ++h)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        s[h][t][j] *= qs[t][j & 1];
            if (!whole) {
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int h = 0; h < HV; ++h)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const int key = key0 + 16 * h + g + 8 * (j >> 1), top = hi[t][j & 1];
                            if (key >= top || key < top - a.window)
                                s[h][t][j] = -INFINITY;
                        }
            }
            bool raise = !here;              // (one vote for both)
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    raise |= fmaxf(fmax3(s[0][t][j], s[0][t][j + 2], s[HV - 1][t][j]), s[HV - 1][t][j + 2]) > z.m[t][j] + kRoom;
            if (__any_sync(kAll, raise)) {
                if (!__all_sync(kAll, here)) {
                    ok = false;
                    break;
                }
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        float mx = fmaxf(fmax3(s[0][t][j], s[0][t][j + 2], s[HV - 1][t][j]), s[HV - 1][t][j + 2]);
                        mx = fmaxf(mx, __shfl_xor_sync(kAll, mx, 4));
                        mx = fmaxf(mx, __shfl_xor_sync(kAll, mx, 8));
                        mx = fmaxf(mx, __shfl_xor_sync(kAll, mx, 16));
                        mx = fmaxf(mx - kBelow, z.m[t][j]);
                        const float f = z.m[t][j] == -INFINITY ? 0.f : ex2(z.m[t][j] - mx);
                        z.m[t][j] = mx;
                        z.l[t][j] *= f;
#pragma unroll
                        for (int i2 = 0; i2 < MT; ++i2) {
                            z.o[t][i2][j] *= f;
                            z.o[t][i2][j + 2] *= f;
                        }
                    }
            }
            uint32_t pb[HV][NT][2];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                // (a row that has seen no key yet: m is -inf and so is s)
                const float m0 = z.m[t][0] == -INFINITY ? 0.f : z.m[t][0];
                const float m1 = z.m[t][1] == -INFINITY ? 0.f : z.m[t][1];
#pragma unroll
                for (int h = 0; h < HV; ++h) {
                    const float e0 = ex2(s[h][t][0] - m0), e1 = ex2(s[h][t][1] - m1);
                    const float e2 = ex2(s[h][t][2] - m0), e3 = ex2(s[h][t][3] - m1);
                    z.l[t][0] += e0 + e2;
                    z.l[t][1] += e1 + e3;
                    pb[h][t][0] = movmatrix(pack_f16(e0, e1));
                    pb[h][t][1] = movmatrix(pack_f16(e2, e3));
                }
            }
            // ---- values: this lane's keys are 16 h + 2 c, + 1 and + 8, + 9, its dimensions g D/8 ..
            const uint8_t *const vs = ring + S::kVsOff + 2 * c * S::kScale;
            int ve[HV][4];                    // exponents (MXFP4: byte; HiF4: E) of the keys
            uint32_t vm[HV][4];               // HiF4 metadata
            int top = -2000;
#pragma unroll
            for (int h = 0; h < HV; ++h)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int tok = 16 * h + (j & 1) + 8 * (j >> 1);
                    if (HIF4) {
                        vm[h][j] = *reinterpret_cast<const uint32_t *>(vs + tok * S::kScale + (g * (D / 8) / 64) * 4);
                        ve[h][j] = (int)((vm[h][j] >> 2) & 63u);
                    } else {
                        ve[h][j] = (int)vs[tok * S::kScale + g * (D / 8) / 32];
                    }
                }
            if (!whole) {                     // what no row sees is nothing, whatever its bytes
#pragma unroll
                for (int h = 0; h < HV; ++h)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int key = key0 + 16 * h + 2 * c + (j & 1) + 8 * (j >> 1);
                        if (key >= walk.ke || key < least) {
                            ve[h][j] = -2000;
                            if (HIF4)
                                vm[h][j] = 0;
                        }
                    }
            }
#pragma unroll
            for (int h = 0; h < HV; ++h)
                top = __vimax3_s32(__vimax3_s32(top, ve[h][0], ve[h][1]), ve[h][2], ve[h][3]);
            if (__any_sync(kAll, top > vref + 3)) {
                top = max(top, __shfl_xor_sync(kAll, top, 1));
                top = max(top, __shfl_xor_sync(kAll, top, 2));
                top = max(top, vref);
                const float f = ex2((float)(vref - top));
                vref = top;
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int i2 = 0; i2 < MT; ++i2)
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            z.o[t][i2][j] *= f;
            }
#pragma unroll
            for (int h = 0; h < HV; ++h) {
                constexpr int VW = D / 64;    // words a key
                uint32_t v0[2 * VW], v1[2 * VW];   // keys 2c, 2c + 1; 2c + 8, 2c + 9
                {
                    const uint8_t *const vr = ring + S::kVOff + h * 8 * D + lane * (D / 8);
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
                // f16 scales of the key pairs: 2^(e - vref + 9)
                uint32_t sc[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const uint32_t x = (uint32_t)__viaddmax_s32(ve[h][2 * j], 24 - vref, 0);
                    const uint32_t y = (uint32_t)__viaddmax_s32(ve[h][2 * j + 1], 24 - vref, 0);
                    sc[j] = x * 0x400u + y * 0x04000000u;
                    if (HIF4)                 // with the macro scale's two mantissa bits
                        sc[j] += (x ? (vm[h][2 * j] & 3u) << 8 : 0u) + (y ? (vm[h][2 * j + 1] & 3u) << 24 : 0u);
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
                            const uint32_t m0 = vm[h][2 * kk], m1 = vm[h][2 * kk + 1];
                            const uint32_t e8 = __byte_perm(m0, m1, 0x7531) >> gi;    // E1_8 bytes at 0 and 16
                            const uint32_t e16 = __byte_perm(m0, m1, 0x7632) >> (2 * gi);
                            const uint32_t t8 = e8 & 0x00010001u;
                            const uint32_t sa = sc[kk] + (t8 + (e16 & 0x00010001u)) * 0x400u;
                            const uint32_t sb = sc[kk] + (t8 + ((e16 >> 1) & 0x00010001u)) * 0x400u;
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
                            mma_f16(z.o[t][4 * w + j], a0[j], a1[j], a2[j], a3[j], pb[h][t][0], pb[h][t][1]);
                }
            }
            __syncwarp();                     // every lane has read the chunk
            if (++slot == DEPTH) {
                slot = 0;
                parity ^= 1;
            }
        }

        if (++walk.i < walk.i1)
            continue;
        // ---- the segment ends here: the warp's sums in plain units
        const float vunit = scalbnf(1.f, vref - (HIF4 ? 50 : 136));
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                float x = z.l[t][j];
                x += __shfl_xor_sync(kAll, x, 4);
                x += __shfl_xor_sync(kAll, x, 8);
                x += __shfl_xor_sync(kAll, x, 16);
                z.l[t][j] = x;
            }
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    z.o[t][i][j] *= vunit;
        }
        const bool ends = walk.i1 == walk.chunks;
        fresh = true;
        if (!begins || !ends) {
            // (over the ring only when nothing is left to copy: the run's last segment)
            const int k = begins ? 1 : 0;
            z.store(part_of(warp, k), lane);
            if (lane == 0)
                s_info[warp][k] = {walk.u, walk.chunks, walk.head, row0, rows, q.q0, begins, ends};
        } else {
            write(row0, rows, q.q0, walk.head);
        }
        walk.next(p);
    }

    // ---- a wait has run out: the warp copies nothing more and waits for nothing
    // more, and its segments from this one on are NaN
    if (!ok) {
        if (warm == 0) {                     // (its copies in flight, of slots slot .. fslot, land before a part lies over them)
            int i = slot;
            do {
                mbar_wait(&s_full[warp][i], parity, kWaitLimitNs);
                if (++i == DEPTH) {
                    i = 0;
                    parity ^= 1;
                }
            } while (i != fslot);
        }
        if (lane == 0)
            atomicExch(p.status, kDevTimeout);
#pragma unroll 1
        for (; walk.more(); walk.next(p), begins = true) {
            const bool ends = walk.i1 == walk.chunks;
            const float nan = __int_as_float(0x7FFFFFFF);
            row0 = walk.tile * ROWS;
            rows = min(ROWS, walk.q.n * G - row0);
            if (!begins || !ends) {
                const int k = begins ? 1 : 0;
                for (int i = lane; i < S::kPart / 16; i += 32)
                    reinterpret_cast<float4 *>(part_of(warp, k))[i] = make_float4(nan, nan, nan, nan);
                if (lane == 0)
                    s_info[warp][k] = {walk.u, walk.chunks, walk.head, row0, rows, walk.q.q0, begins, ends};
            } else {
                for (int i = lane; i < rows * D; i += 32) {
                    const int ri = row0 + i / D;
                    const int64_t at = (int64_t)(walk.q.q0 + ri / G) * a.heads + walk.head * G + ri % G;
                    static_cast<__nv_bfloat16 *>(a.out)[at * D + i % D] = __float2bfloat16_rn(nan);
                    if (a.lse && i % D == 0)
                        a.lse[at] = nan;
                }
            }
            walk.i = walk.i1;
        }
    }

    // ---- join the parts: of one segment they follow each other in the order of the warps
    __syncthreads();
    constexpr int64_t kFloats = S::kPart / 4;
    // lane e looks at entry e: entry 2w is warp w's first segment, 2w + 1 its last
    const uint32_t seg = lane < 2 * W ? s_info[lane >> 1][lane & 1].seg : kNoPart;
    const uint32_t have = __ballot_sync(kAll, seg != kNoPart);
    const uint32_t below = have & ((1u << lane) - 1);
    const uint32_t prev = __shfl_sync(kAll, seg, below ? 31 - __clz(below) : 0);
    const uint32_t starts = __ballot_sync(kAll, seg != kNoPart && (!below || prev != seg));   // of a segment's entries
    auto parts_of = [&](int e) {                                       // the entries of the segment that starts at e
        const uint32_t after = starts & ~((2u << e) - 1);
        return have & ~((1u << e) - 1) & (after ? (after & -after) - 1 : kAll);
    };
    auto part_at = [&](int k) -> const uint8_t * { return part_of(k >> 1, k & 1); };
    // At most two segments reach into other CTAs: the first entries' one, if
    // it began before this CTA, and the last entries' one.  All warps sum their
    // parts; the CTA's sums go to the workspace.
    int shared[2], nshared = 0;
    if (have) {
        const int e0 = __ffs(have) - 1, e1 = 31 - __clz(starts), le = 31 - __clz(have);
        if (!s_info[e0 >> 1][e0 & 1].begins)
            shared[nshared++] = e0;
        if (!s_info[le >> 1][le & 1].ends && (nshared == 0 || e1 != e0))
            shared[nshared++] = e1;
    }
#pragma unroll 1
    for (int n = 0; n < nshared; ++n) {
        const int e = n ? shared[1] : shared[0];
        const bool first_cta = s_info[e >> 1][e & 1].begins != 0;
        const uint32_t parts = parts_of(e);
        float4 *const mine = reinterpret_cast<float4 *>(p.part + (2 * cta + (first_cta ? 1 : 0)) * kFloats);
#pragma unroll 1
        for (int u = warp; u < NT * MT; u += W) {
            const int t = u / MT;
            Joined x;
            x.clear();
#pragma unroll 2
            for (uint32_t left = parts; left; left &= left - 1) {
                const float4 *const d = reinterpret_cast<const float4 *>(part_at(__ffs(left) - 1));
                x.add(d[u * 32 + lane], d[(NT * MT + t) * 32 + lane]);
            }
            __stcg(mine + u * 32 + lane, make_float4(x.o[0], x.o[1], x.o[2], x.o[3]));
            if (u % MT == 0)
                __stcg(mine + (NT * MT + t) * 32 + lane, make_float4(x.m[0], x.m[1], x.l[0], x.l[1]));
        }
    }
    if (nshared > 0) {
        __threadfence();
        __syncthreads();
        if (lane == 0 && warp < nshared) {
            const int e = warp ? shared[1] : shared[0];
            const PartInfo f = s_info[e >> 1][e & 1];
            const int c0 = owner(sh, f.seg + S::kStart), c1 = owner(sh, f.seg + S::kStart + f.chunks - 1);
            s_c[warp] = make_int2(c0, c1);
            s_flag[warp] = atomicAdd(p.counter + c0, 1) == c1 - c0;
        }
    }
    // A segment that warps of this CTA share among them starts in one warp's
    // last entry: that warp joins it.
    if (starts >> (2 * warp + 1) & 1) {
        const int e = 2 * warp + 1;
        const uint32_t parts = parts_of(e);
        const int le = 31 - __clz(parts);
        if (s_info[le >> 1][le & 1].ends) {
            z.clear();
#pragma unroll 1
            for (uint32_t left = parts; left; left &= left - 1)
                z.join(part_at(__ffs(left) - 1), lane);
            const PartInfo f = s_info[warp][1];
            write(f.row0, f.rows, f.q0, f.head);
        }
    }
    // The last CTA of a shared segment joins all its parts.
    if (nshared > 0) {
        __syncthreads();
#pragma unroll 1
        for (int n = 0; n < nshared; ++n) {
            if (!s_flag[n])
                continue;
            const int e = n ? shared[1] : shared[0];
            const PartInfo f = s_info[e >> 1][e & 1];
            const int c0 = s_c[n].x, c1 = s_c[n].y;
            __threadfence();
            if (tid == 0)
                atomicExch(p.counter + c0, 0);
#pragma unroll 1
            for (int u = warp; u < NT * MT; u += W) {
                const int t = u / MT, i = u % MT;
                Joined x;
                x.clear();
#pragma unroll 4
                for (int k = c0; k <= c1; ++k) {
                    const float4 *const d =
                        reinterpret_cast<const float4 *>(p.part + (2 * k + (k == c0 ? 1 : 0)) * kFloats);
                    x.add(__ldcg(d + u * 32 + lane), __ldcg(d + (NT * MT + t) * 32 + lane));
                }
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int row = 8 * t + 2 * c + j, ri = f.row0 + row;
                    if (row >= f.rows)
                        continue;
                    const int64_t at = (int64_t)(f.q0 + ri / G) * a.heads + f.head * G + ri % G;
                    const float inv = inverse(x.l[j]);
                    *reinterpret_cast<uint32_t *>(static_cast<__nv_bfloat16 *>(a.out) + at * D + g * (D / 8) + 2 * i) =
                        pack_bf16(x.o[j] * inv, x.o[j + 2] * inv);
                    if (a.lse && g == 0 && i == 0)
                        a.lse[at] = log_sum(x.m[j], x.l[j]);
                }
            }
        }
    }
}

// The rows of no request where no tile kernel runs to see to them: in the kernel
// above, whatever is added costs 2 to 3% of a long request.
constexpr int kRestThreads = 256;

__global__ void __launch_bounds__(kRestThreads) kv_attention_rest_kernel(const KvAttentionArgs a)
{
    wait_for_previous();
    let_next_start();
    clear_rest(a, threadIdx.x, kRestThreads);
}

constexpr size_t kWsCounters = 256;

size_t ws_parts_offset() { return kWsCounters + ((size_t)num_sms() * 4 + 255) / 256 * 256; }

template <int FMT, int D, int NT>
cudaError_t launch(AttnParams p, cudaStream_t st)
{
    using S = Shape<FMT, D, NT>;
    static_assert(S::kSmem <= 226 * 1024, "fits an SM");
    static PerDevice<bool> allowed;
    if (cudaError_t e = allow_smem(reinterpret_cast<const void *>(kv_attention_kernel<FMT, D, NT>), S::kSmem, allowed))
        return e;
    p.gran = p.a.cache.page_size % S::kChunk == 0 ? S::kChunk : 16;
    return launch_early(kv_attention_kernel<FMT, D, NT>, dim3(num_sms()), S::kThreads, S::kSmem, st, 1, p);
}

template <int FMT, int D>
cudaError_t launch_rows(const AttnParams &p, int64_t rows, cudaStream_t st)
{
    // (Four row tiles a warp and 16 keys a chunk: 283 us against 239 with two,
    // 256 new tokens over up to 8192, D = 128: the sums leave no registers.)
    return rows <= 8 ? launch<FMT, D, 1>(p, st) : launch<FMT, D, 2>(p, st);
}

// Rows of a request and key head (the group's heads times its new tokens) from
// which on kv_attention_tile.cu takes it: more than two of this kernel's tiles.
// 8 requests of 4096 keys, 32 heads on 8, D = 128, MXFP4, tiles against this
// kernel: 32 rows 38 against 33 us, 64 rows 39 against 40, 96 rows 40 against
// 73, 256 rows 50 against 96 (HiF4: 42 against 39, 43 against 49, 44 against
// 93, 54 against 125; D = 64, MXFP4: 33 against 25, 33 against 30, 34 against
// 55, 41 against 74).
constexpr int kTileRows = 33;

// The rows that a request of the call may have at most, as far as the host
// knows: each request has one token at least, or the tiles may be left out all the same.
int64_t most_rows(int64_t tokens, int32_t group, bool q_start, int32_t requests)
{
    return q_start ? (tokens - requests + 1) * group : group;
}

} // namespace

double kv_attention_most_units(int64_t tokens, int32_t group, bool q_start, int32_t requests, int32_t kv_heads, int64_t keys)
{
    // A request of r rows has ceil(r / 8) tiles here (of 16 rows, fewer), or
    // ceil(r / 128) there; a tile has a unit for each chunk of keys that is begun
    // (the first key may lie inside one) and those of its start.
    const double rows = (double)tokens * group, R = requests;
    const double here = kv_heads * (keys / 32.0 + 2), there = kv_heads * (keys / (double)kTileChunk + 1 + kTileStart);
    const bool tiles = most_rows(tokens, group, q_start, requests) >= kTileRows;
    if (!q_start)
        return tiles ? (R + rows / kTileRowsEach) * there : (R + rows / 8) * here;
    if (!tiles)
        return (R + rows / 8) * here;
    const double few = std::min(R + rows / 8, R * ((kTileRows - 1 + 7) / 8));   // of requests below kTileRows rows
    return std::max(few * here, (std::min(R, rows / kTileRows) + rows / kTileRowsEach) * there);
}

size_t kv_attention_workspace_bytes(int32_t heads, int32_t head_dim)
{
    (void)heads;
    const size_t part = (size_t)2 * (head_dim / 16 + 1) * 512, tile = kv_attention_tile_part_bytes(head_dim);
    return ws_parts_offset() + (size_t)2 * num_sms() * (part > tile ? part : tile);
}

cudaError_t launch_kv_attention(const KvAttentionArgs &a, cudaStream_t st)
{
    uint8_t *const ws = static_cast<uint8_t *>(a.workspace);
    AttnParams p = {a,
                    a.heads / a.cache.heads,
                    0,
                    static_cast<int32_t *>(a.workspace),
                    reinterpret_cast<int32_t *>(ws + kWsCounters),
                    reinterpret_cast<float *>(ws + ws_parts_offset()),
                    0,
                    INT32_MAX};
    if (a.window == 0)                       // (none: the kernels know windows alone)
        p.a.window = INT32_MAX;
    // Only the device knows who has how many new tokens.  Where each request
    // has one at least and none can have kTileRows rows, the tiles have nothing to do.
    if (a.requests > 0 && most_rows(a.tokens, p.group, a.q_start != nullptr, a.requests) >= kTileRows) {
        p.least_rows = kTileRows;
        if (cudaError_t e = launch_kv_attention_tile(p, st))
            return e;
        p.least_rows = 0;
        p.most_rows = kTileRows - 1;
        if (!a.q_start)
            return cudaSuccess;              // (every request has the same rows)
    } else if (a.q_start) {
        if (cudaError_t e = launch_early(kv_attention_rest_kernel, dim3(num_sms()), kRestThreads, 0, st, 1, a))
            return e;
        if (a.requests == 0)
            return cudaSuccess;
    }
    const int64_t rows = a.q_start ? (a.tokens + a.requests - 1) / a.requests * p.group : p.group;
    const bool wide = a.cache.head_dim == 128;
    if (a.cache.fmt == RFQ_FMT_HIF4)
        return wide ? launch_rows<RFQ_FMT_HIF4, 128>(p, rows, st) : launch_rows<RFQ_FMT_HIF4, 64>(p, rows, st);
    return wide ? launch_rows<RFQ_FMT_MXFP4, 128>(p, rows, st) : launch_rows<RFQ_FMT_MXFP4, 64>(p, rows, st);
}

} // namespace rfq
