// kv_attention_tile.cu -- rfq_kv_attention for requests with many rows (new
// tokens times the key head's query heads): tiles of 128 rows by 128 keys on
// the tensor cores.
//
// Mathematics: as in kv_attention.cu, one pass over the keys with a running
// maximum and sum in the log2 domain, with S = Q K^T and O += P V as
// tcgen05.mma of 128 x 128 x 16, f16 operands and fp32 sums.
//   Q: scaled by a power of two per row (maximum in [2^14, 2^15)): exact down
//      to 2^-28 of the maximum, off by less than 2^-39 of it below.
//   K: codes times scale relative to a running power of two, exact while the
//      scales span less than 2^24 over the keys seen so far; what lies below
//      counts as zero (a score is then off by what its fp32 sum is off by
//      beside a key of the largest scale).
//   P: exp2(s - m) rounded to f16 (its sum l stays fp32), m 7 below the maximum
//      when it is set and raised only when a score passes it by 15: weights down
//      to 2^-21 of the largest are off by 2^-11 of themselves, smaller ones by
//      2^-32 of the largest.
//   V: as K, the power of two per 32 dimensions.
//
// Work: the (request, key head, 128 rows) segments laid end to end in chunks
// of 128 keys, split evenly over the CTAs, one a SM.  In a CTA, warp by warp:
//   0-3    softmax: a thread has one row; S from TMEM twice (for its maximum,
//          then for its weights), P to TMEM
//   4-7    K codes to f16 (and Q, when a segment begins), dimensions contiguous
//   8-11   V codes to f16, dimensions contiguous
//   12     one thread issues the MMAs: S of the next chunk before P V of this
//   13     the running powers of two
//   14     copies the chunks' codes and scales, three ahead
// K, V, S and P have two buffers each.  A segment that CTAs share leaves its
// parts in the workspace, where the last CTA to finish joins them: the split
// and the order of every sum depend on the lengths alone.
//
// Bound: the instructions of 16384 scores and 32768 codes a chunk (3800 clocks
// in a long segment, of which the MMAs take 1000), and their fetch: the roles'
// loops have to fit the instruction caches together, so they stay rolled (all
// unrolled: 186 us before what else follows, against 135).
// 256 new tokens of 5 requests over 300 to 8192 keys, 32 heads on 8, D = 128,
// MXFP4, pages of 32: 78 us, 457 TFLOP/s; HiF4 87; one request of 4096 new
// tokens, MXFP4: 159 us, 658 TFLOP/s.  Tried there: eight warps for the
// softmax 83 us, for K and for V 95 against 92; one pass over the scores with
// the maximum so far, repeated where it was passed, 79; the units of a
// segment's start 1, 3, 5, 7: 107, 95, 96, 101.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <cstdint>

#include "kv_attention.cuh"
#include "kv_layout.cuh"
#include "mxfp4_math.cuh"

namespace rfq {
namespace {

constexpr int kLeast = 4;                    // units of a CTA, at least
constexpr int kKeys = 4, kValues = 8, kMma = 12, kUnits = 13, kWarps = 15;   // a role's first warp
constexpr uint32_t kTmemCols = 512;          // S: 0, 128; O: 256; P: 384, 448

template <int FMT, int D>
struct Tile {
    static constexpr int kRows = kTileRowsEach, kChunk = kTileChunk, kStart = kTileStart, kThreads = 32 * kWarps, kDepth = 3;
    static constexpr int kScale = FMT == RFQ_FMT_HIF4 ? D / 16 : D / 32;   // bytes a token
    static constexpr int kCode = D / 2;
    static constexpr int kVOff = kChunk * kCode, kKsOff = 2 * kVOff, kVsOff = kKsOff + kChunk * kScale;
    static constexpr int kBytes = kVsOff + kChunk * kScale;
    static constexpr int kOperand = 128 * D * 2;                           // bytes of Q, of a K and of a V
    static constexpr int kQ = 0, kK = kOperand, kV = 3 * kOperand, kRing = 5 * kOperand;
    static constexpr int kSmem = 1024 + kRing + kDepth * kBytes + 1024;    // (the operands lie on 1024 bytes)
    static constexpr int64_t kPart = 128 * (D + 2);                        // floats
};

struct Bars {
    uint64_t full[3], units[3], empty[3];    // the ring: copied, its powers of two found, read
    uint64_t k_full[2], k_empty[2], v_full[2], v_empty[2];
    uint64_t s_full[2], s_empty[2], p_full[2];
    uint64_t drain;
    uint64_t limit;                          // of a wait, in ns
    int32_t abort;                           // a wait has run out
};
extern __shared__ __align__(16) uint8_t smem_raw[];   // Bars, then the operands and the ring

// A segment that the CTA does not hold whole.
struct Shared {
    uint32_t seg;
    int chunks, head, row0, rows, q0, begins, c0, c1, last;
};

// The f16 scale 2^(e - ref + 9) of a scale byte or HiF4 metadata word, in both
// halves; HiF4 with its two mantissa bits.
template <bool HIF4>
__device__ __forceinline__ uint32_t f16_scale(uint32_t scale, int ref)
{
    const uint32_t x = (uint32_t)max((int)(HIF4 ? (scale >> 2) & 63u : scale) + 24 - ref, 0);
    return (HIF4 && x ? x << 10 | (scale & 3u) << 8 : x << 10) * 0x00010001u;
}

// Eight codes times f16_scale sc -> four f16 pairs: MXFP4 in order, HiF4
// elements (0, 2), (1, 3), (4, 6), (5, 7) of group gi of the block of meta.
template <bool HIF4>
__device__ __forceinline__ uint4 codes_f16(uint32_t w, uint32_t sc, uint32_t meta, int gi)
{
    uint32_t h[4];
    if (HIF4) {
        // (a scale that has faded out stays below 2^-12: its codes come as k 2^-9)
        const uint32_t e8 = (meta >> (8 + gi)) & 1u, e16 = meta >> (16 + 2 * gi);
        const uint32_t s0 = sc ? sc + (e8 + (e16 & 1u)) * 0x04000400u : 0u;
        const uint32_t s1 = sc ? sc + (e8 + ((e16 >> 1) & 1u)) * 0x04000400u : 0u;
        s1p2x8_f16(w, h);
        h[0] = hmul2(h[0], s0), h[1] = hmul2(h[1], s0);
        h[2] = hmul2(h[2], s1), h[3] = hmul2(h[3], s1);
    } else {
        e2m1x8_f16(w, h);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            h[e] = hmul2(h[e], sc);
    }
    return make_uint4(h[0], h[1], h[2], h[3]);
}

// Two fp32 operations in one instruction.
__device__ __forceinline__ void mul2(float &d0, float &d1, float a0, float a1, float b)
{
    asm("{\n\t.reg .b64 x, y;\n\t"
        "mov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %4};\n\t"
        "mul.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "=f"(d0), "=f"(d1)
        : "f"(a0), "f"(a1), "f"(b));
}
__device__ __forceinline__ void add2(float &d0, float &d1, float a0, float a1)
{
    asm("{\n\t.reg .b64 x, y;\n\t"
        "mov.b64 x, {%0, %1};\n\tmov.b64 y, {%2, %3};\n\t"
        "add.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "+f"(d0), "+f"(d1)
        : "f"(a0), "f"(a1));
}

// D[tmem] (+)= A[tmem] x B[smem], f16 operands, fp32 accumulator.
__device__ __forceinline__ void tc_mma_f16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc,
                                              uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\t"
                 "setp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
                 "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
                 : "memory");
}

// Instruction descriptor, kind::f16: f16 x f16 -> fp32, A K-major, B K-major
// or with N contiguous (bit 16).
__host__ __device__ constexpr uint32_t idesc_f16(int M, int N, bool n_major)
{
    return (1u << 4) | (n_major ? 1u << 16 : 0u) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

// Operand tile with N contiguous and the 128-byte swizzle: [N / 64][128 K rows
// of 128 bytes].  Leading offset: from 64 columns to the next; stride offset:
// from 8 K rows to the next.
__device__ __forceinline__ uint64_t sdesc_n_sw128(uint32_t saddr)
{
    return (uint64_t)((saddr & 0x3FFFFu) >> 4) | (uint64_t)(128 * 128 >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 |
           (uint64_t)1 << 46 | (uint64_t)2 << 61;
}

// Sixteen 32-bit columns of the thread's TMEM lane.
__device__ __forceinline__ void tmem_st_32x32b_x16(uint32_t taddr, const uint32_t (&r)[16])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
                 "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),
                 "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
                 "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
                 : "memory");
}
// x[b] without indexing registers
template <typename T, int N>
__device__ __forceinline__ T pick(const T (&x)[N], int b)
{
    T r = x[0];
#pragma unroll
    for (int i = 1; i < N; ++i)
        r = b == i ? x[i] : r;
    return r;
}

// Waits for the loads into r (tied to it: its uses stay behind the wait).
__device__ __forceinline__ void tmem_ld_ready(uint32_t (&r)[32])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                   "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14])
                 :
                 : "memory");
    asm volatile("" : "+r"(r[15]), "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]),
                      "+r"(r[22]), "+r"(r[23]), "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]),
                      "+r"(r[29]), "+r"(r[30]), "+r"(r[31]));
}

// Bits [lo, hi) of the word of columns at ..
__device__ __forceinline__ uint32_t visible(int at, int lo, int hi)
{
    lo = min(max(lo - at, 0), 32), hi = min(max(hi - at, 0), 32);
    return lo < hi ? (kAll >> (32 - hi)) & (kAll << lo) : 0u;
}

// The largest of the 128 scores at s_at: of ALL, or of those in columns [lo, hi).
template <bool ALL>
__device__ __forceinline__ float row_max(uint32_t s_at, int lo, int hi)
{
    float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll 1
    for (int q = 0; q < 128; q += 32) {
        uint32_t x[32];
        tmem_ld_32x32b_x32(s_at + q, x);
        tmem_ld_ready(x);
        const uint32_t seen = ALL ? kAll : visible(q, lo, hi);
#pragma unroll
        for (int i = 0; i < 32; i += 2) {
            const float x0 = ALL || (seen >> i & 1) ? __uint_as_float(x[i]) : -INFINITY;
            const float x1 = ALL || (seen >> i & 2) ? __uint_as_float(x[i + 1]) : -INFINITY;
            mx[i >> 1 & 1] = fmax3(mx[i >> 1 & 1], x0, x1);
        }
    }
    return fmaxf(mx[0], mx[1]);
}

// The weights exp2(c s - m) of the scores at s_at, to p_at as f16; their sum.
template <bool ALL>
__device__ __forceinline__ float row_weights(uint32_t s_at, uint32_t p_at, float c, float m, int lo, int hi)
{
    float l[2] = {0.f, 0.f};
#pragma unroll 1
    for (int q = 0; q < 128; q += 32) {
        uint32_t x[32], w[16];
        tmem_ld_32x32b_x32(s_at + q, x);
        tmem_ld_ready(x);
        const uint32_t seen = ALL ? kAll : visible(q, lo, hi);
#pragma unroll
        for (int i = 0; i < 32; i += 2) {
            float e0, e1;
            // (the product is rounded, as the maximum is)
            mul2(e0, e1, __uint_as_float(x[i]), __uint_as_float(x[i + 1]), c);
            add2(e0, e1, -m, -m);
            e0 = ex2(e0), e1 = ex2(e1);
            if (!ALL) {
                e0 = seen >> i & 1 ? e0 : 0.f;
                e1 = seen >> i & 2 ? e1 : 0.f;
            }
            add2(l[0], l[1], e0, e1);
            const __half2 h = __floats2half2_rn(e0, e1);
            w[i / 2] = *reinterpret_cast<const uint32_t *>(&h);
        }
        tmem_st_32x32b_x16(p_at + q / 2, w);
    }
    return l[0] + l[1];
}

// The rest of a wait that did not end at once: out of the way of the loops.
__device__ __noinline__ bool wait_on(uint32_t b, uint32_t parity)
{
    const Bars &bar = *reinterpret_cast<const Bars *>(smem_raw);
    const uint64_t t0 = globaltimer_ns();
    for (;;) {
        uint32_t done;
        asm volatile("{\n\t.reg .pred p;\n\t"
                     "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
                     "selp.u32 %0, 1, 0, p;\n\t}"
                     : "=r"(done)
                     : "r"(b), "r"(parity), "r"(1000u)             // (asleep for at most this many ns)
                     : "memory");
        if (done)
            return true;
        if (globaltimer_ns() - t0 > bar.limit || *reinterpret_cast<const volatile int32_t *>(&bar.abort))
            return false;
    }
}
// A warp waits as one, and every wait of the CTA gives up once one has run out.
__device__ __forceinline__ bool wait(uint64_t *b, uint32_t parity)
{
    const uint32_t at = smem_u32(b);
    if (__all_sync(kAll, mbar_try_wait(at, parity)))
        return true;
    if (__all_sync(kAll, wait_on(at, parity)))
        return true;
    *reinterpret_cast<volatile int32_t *>(&reinterpret_cast<Bars *>(smem_raw)->abort) = 1;
    return false;
}

template <int FMT, int D>
__global__ void __launch_bounds__(32 * kWarps, 1) kv_attention_tile_kernel(const __grid_constant__ AttnParams p)
{
    using S = Tile<FMT, D>;
    constexpr bool HIF4 = FMT == RFQ_FMT_HIF4;
    constexpr int NB = D / 32, DEPTH = S::kDepth;
    constexpr int kBias = HIF4 ? 50 : 136;   // operand = value 2^(kBias - exponent)
    Bars &bar = *reinterpret_cast<Bars *>(smem_raw);
    __shared__ uint32_t s_scan[kWarps], s_tmem;
    __shared__ int s_unit[DEPTH][NB + 1];    // the exponents that V (32 dimensions each) and K are relative to
    __shared__ int s_vref[2][NB], s_kref[4]; // the same by chunk, for the softmax
    __shared__ float s_qs[4][128];           // by segment: what a row of Q was divided by
    __shared__ Shared s_shared[2];
    __shared__ int s_nshared;
    static_assert(sizeof(Bars) <= 1024, "in front of the operands");
    uint8_t *const smem = smem_raw + 1024 + (-smem_u32(smem_raw) & 1023u);

    const KvAttentionArgs &a = p.a;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int H = a.cache.heads, G = p.group;

    if (tid == 0) {
        for (int i = 0; i < DEPTH; ++i) {
            mbar_init(&bar.full[i], 1);
            mbar_init(&bar.units[i], 1);
            mbar_init(&bar.empty[i], 8);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&bar.k_full[i], 4);
            mbar_init(&bar.k_empty[i], 1);
            mbar_init(&bar.v_full[i], 4);
            mbar_init(&bar.v_empty[i], 1);
            mbar_init(&bar.s_full[i], 1);
            mbar_init(&bar.s_empty[i], 4);
            mbar_init(&bar.p_full[i], 4);
        }
        mbar_init(&bar.drain, 1);
        fence_mbar_init();
        bar.abort = 0;
        s_nshared = 0;
    }
    wait_for_previous();
    let_next_start();
    Share sh;
    if (!find_share<S, false>(p, s_scan, kWarps, kLeast, sh)) {
        if (a.q_start)
            clear_rest(a, tid, S::kThreads);
        return;
    }
    if (tid == 0)
        bar.limit = ws_wait_limit_ns(p.status);
    // (TMEM only now: a kernel in front that is still to take its own has finished)
    if (warp == kMma) {
        tmem_alloc(&s_tmem, kTmemCols);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = s_tmem;
    Walk<S> walk;
    walk.start(p, sh.r, sh.rem, sh.first, sh.last, lane);
    walk.next(p);
    if (warp < kKeys) {
        // ------------------------------------------------ softmax and output
        const uint32_t lane_at = tmem + ((uint32_t)(warp * 32) << 16);
        const float base = fabsf(a.scale) * 1.4426950408889634f;
        bool ok = true;
        uint32_t j = 0, segs = 0;            // chunks and segments of the CTA so far
#pragma unroll 1
        for (; walk.more(); ++segs) {
            const bool begins = walk.i == 0, ends = walk.i1 == walk.chunks;
            const int row0 = walk.tile * 128, rows = min(128, walk.q.n * G - row0), n = walk.q.n, L = walk.q.L;
            const int ri = row0 + min(tid, rows - 1);
            const int hi = max(0, L - n + ri / G + 1), lo = first_seen(hi, a.window);
            const int all_hi = max(0, L - n + row0 / G + 1);
            const int all_lo = first_seen(L - n + (row0 + rows - 1) / G + 1, a.window);
            float m = -INFINITY, l = 0.f, qs = 0.f;
            int vref[NB];
#pragma unroll 1
            for (bool first = true; walk.i < walk.i1; ++walk.i, ++j, first = false) {
                const uint32_t buf = j & 1, ph = (j >> 1) & 1;
                const int key0 = walk.kb + walk.i * 128;
                const bool whole = key0 >= all_lo && key0 + 128 <= all_hi;
                const uint32_t s_at = lane_at + buf * 128, p_at = lane_at + 384 + buf * 64;
                ok = ok && wait(&bar.s_full[buf], ph);
                tc_fence_after();
                if (first)
                    qs = base * s_qs[segs & 3][tid];
                const float c = qs * ex2((float)(s_kref[j & 3] - kBias));
                // ---- the row's maximum
                const float mx = whole ? row_max<true>(s_at, 0, 0) : row_max<false>(s_at, lo - key0, hi - key0);
                const float top = mx == -INFINITY ? mx : mx * c;
                float f = 1.f;
                const bool raise = top > m + kRoom;
                if (raise) {
                    f = m == -INFINITY ? 0.f : ex2(m - (top - kBelow));
                    m = top - kBelow;
                    l *= f;
                }
                const float m0 = m == -INFINITY ? 0.f : m;
                // ---- its weights, over those of two chunks ago
                ok = ok && wait(&bar.v_empty[buf], ph ^ 1);
                tc_fence_after();
                l += whole ? row_weights<true>(s_at, p_at, c, m0, 0, 0)
                           : row_weights<false>(s_at, p_at, c, m0, lo - key0, hi - key0);
                tc_fence_before();
                __syncwarp();
                if (lane == 0)
                    mbar_arrive(&bar.s_empty[buf]);
                // ---- the sums so far, if the maximum or V's unit has changed
                ok = ok && wait(&bar.v_full[buf], ph);
                float unit[NB];
                bool change = raise && !first;
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    const int now = s_vref[buf][b];
                    unit[b] = f;
                    if (!first && now != vref[b]) {
                        unit[b] *= ex2((float)(vref[b] - now));
                        change = true;
                    }
                    vref[b] = now;
                }
                if (__any_sync(kAll, change)) {
                    ok = ok && wait(&bar.v_empty[buf ^ 1], ((j - 1) >> 1) & 1);
                    tc_fence_after();
#pragma unroll 1
                    for (int b = 0; b < NB; ++b) {
                        uint32_t x[32];
                        tmem_ld_32x32b_x32(lane_at + 256 + 32 * b, x);
                        tmem_ld_ready(x);
                        const float u = pick(unit, b);
#pragma unroll
                        for (int half = 0; half < 2; ++half) {
                            uint32_t y[16];
#pragma unroll
                            for (int i = 0; i < 16; ++i)
                                y[i] = __float_as_uint(__uint_as_float(x[16 * half + i]) * u);
                            tmem_st_32x32b_x16(lane_at + 256 + 32 * b + 16 * half, y);
                        }
                    }
                }
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0)
                    mbar_arrive(&bar.p_full[buf]);
            }
            // ---- the sums in plain units, to the output or as a part
            ok = ok && wait(&bar.v_empty[(j - 1) & 1], ((j - 1) >> 1) & 1);
            tc_fence_after();
            if (!ok)
                l = __int_as_float(0x7FFFFFFF);
            const bool part = !begins || !ends;
            float4 *const mine = reinterpret_cast<float4 *>(p.part + (2 * blockIdx.x + (begins ? 1 : 0)) * S::kPart);
            const int64_t at = (int64_t)(walk.q.q0 + ri / G) * a.heads + walk.head * G + ri % G;
            uint4 *const out = reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(a.out) + at * D);
            const float inv = part ? 1.f : inverse(l);
#pragma unroll 1
            for (int b = 0; b < NB; ++b) {
                uint32_t x[32];
                tmem_ld_32x32b_x32(lane_at + 256 + 32 * b, x);
                tmem_ld_ready(x);
                const float f = scalbnf(inv, pick(vref, b) - kBias);
#pragma unroll
                for (int k = 0; k < 4 && tid < rows; ++k) {
                    float y[8];              // (HiF4 columns stand in the order 0 2 | 1 3 | 4 6 | 5 7)
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        y[HIF4 ? (i & 4) + (i >> 1 & 1) + (i & 1) * 2 : i] = __uint_as_float(x[8 * k + i]) * f;
                    if (part) {
                        __stcg(mine + (8 * b + 2 * k) * 128 + tid, make_float4(y[0], y[1], y[2], y[3]));
                        __stcg(mine + (8 * b + 2 * k + 1) * 128 + tid, make_float4(y[4], y[5], y[6], y[7]));
                    } else {
                        out[4 * b + k] = make_uint4(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]),
                                                    pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7]));
                    }
                }
                __syncwarp();
            }
            if (part) {
                if (tid < rows)
                    __stcg(reinterpret_cast<float2 *>(mine + (D / 4) * 128) + tid, make_float2(m, l));
                if (tid == 0)
                    s_shared[s_nshared++] = {walk.u, walk.chunks, walk.head, row0, rows, walk.q.q0, begins, 0, 0, 0};
            } else if (a.lse && tid < rows) {
                a.lse[at] = log_sum(m, l);
            }
            tc_fence_before();               // (O is read before the next segment's P lets it be written)
            walk.next(p);
        }
        if (!ok && lane == 0)
            atomicExch(p.status, kDevTimeout);
    } else if (warp < kValues) {
        // ------------------------------------------------ K, and Q
        const int t = tid - 32 * kKeys, kc = lane & 3;
        // where a thread's pieces stand in a row of 128 bytes
        const uint32_t k_at0 = ((2 * kc) ^ (t >> 2 & 7)) << 4, k_at1 = k_at0 ^ 16u;
        const uint32_t sign = a.scale < 0.f ? 0x80008000u : 0u;
        uint32_t j = 0, segs = 0, slot = 0, ring = 0;
        bool ok = true;
#pragma unroll 1
        for (; walk.more(); ++segs) {
            // ---- the rows as f16, once all MMAs that read those before are done
            const int row0 = walk.tile * 128, rows = min(128, walk.q.n * G - row0);
            constexpr int C = D / 8, kStep = 128 / C;    // pieces of 8 dimensions, a lane each; rows at a time
            const int row = t / C, ch = t % C;
            uint4 x[C];
            {
                int tok = (row0 + row) / G, head = row0 + row - tok * G;
                const int more = kStep / G, rest = kStep - more * G;
                const __nv_bfloat16 *const q = static_cast<const __nv_bfloat16 *>(a.q) + walk.q.q0 * a.q_token +
                                               (int64_t)walk.head * G * a.q_head + 8 * ch;
#pragma unroll
                for (int u = 0; u < C; ++u) {
                    x[u] = make_uint4(0, 0, 0, 0);
                    if (kStep * u + row < rows)
                        x[u] = *reinterpret_cast<const uint4 *>(q + tok * a.q_token + head * a.q_head);
                    tok += more, head += rest;
                    if (head >= G)
                        head -= G, ++tok;
                }
            }
            if (j > 0 && !wait(&bar.k_empty[(j - 1) & 1], ((j - 1) >> 1) & 1))
                break;
            uint8_t *at = smem + S::kQ + (ch >> 3) * 16384 + row * 128;
            const int b = ch >> 2, even = (2 * (ch & 3) + (b & 1)) << 4;
#pragma unroll
            for (int u = 0; u < C; ++u)
                *reinterpret_cast<uint4 *>(at + u * (kStep * 128) + (even ^ ((kStep * u + row & 7) << 4))) = x[u];
#pragma unroll 1
            for (int u = row; u < 128; u += kStep, at += kStep * 128) {
                uint4 *const mine = reinterpret_cast<uint4 *>(at + (even ^ ((u & 7) << 4)));
                const uint4 y = *mine;
                const uint32_t w[4] = {y.x ^ sign, y.y ^ sign, y.z ^ sign, y.w ^ sign};
                float f[8], mx = 0.f;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    f[2 * i] = __uint_as_float(w[i] << 16);
                    f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
                    mx = fmax3(mx, fabsf(f[2 * i]), fabsf(f[2 * i + 1]));
                }
#pragma unroll
                for (int d = 1; d < C; d <<= 1)
                    mx = fmaxf(mx, __shfl_xor_sync(kAll, mx, d));
                const int e = max(min((int)(__float_as_uint(mx) >> 23) - 127 - 14, 126), -126);
                const float mul = __uint_as_float((uint32_t)(127 - e) << 23);
                uint32_t h[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    // HiF4 codes decode in the order 0 2 | 1 3 | 4 6 | 5 7
                    const int lo = HIF4 ? (i >> 1) * 4 + (i & 1) : 2 * i, up = HIF4 ? lo + 2 : lo + 1;
                    const __half2 z = __floats2half2_rn(f[lo] * mul, f[up] * mul);
                    h[i] = *reinterpret_cast<const uint32_t *>(&z);
                }
                *mine = make_uint4(h[0], h[1], h[2], h[3]);
                if (ch == 0)
                    s_qs[segs & 3][u] = __uint_as_float((uint32_t)(127 + e) << 23);
            }
            const int least = walk.least;
#pragma unroll 1
            for (; walk.i < walk.i1; ++walk.i, ++j) {
                const uint32_t buf = j & 1;
                ok = wait(&bar.full[slot], ring) && wait(&bar.units[slot], ring) &&
                     wait(&bar.k_empty[buf], ((j >> 1) & 1) ^ 1);
                if (!ok)
                    break;
                const uint8_t *src = smem + S::kRing + slot * S::kBytes + t * (4 * NB);
                const uint8_t *ks = smem + S::kRing + slot * S::kBytes + S::kKsOff + (t >> 2) * S::kScale;
                uint8_t *dst = smem + S::kK + buf * S::kOperand + (t >> 2) * 128;
                const int ref = s_unit[slot][NB], key0 = walk.kb + walk.i * 128;
                const int from = least - key0, to = walk.ke - key0;
                if (t == 0)
                    s_kref[j & 3] = ref;
#pragma unroll 1
                for (int key = t >> 2; key < 128; key += 32) {
                    uint32_t w[NB], sc[NB], meta[NB];
                    if (D == 128) {
                        const uint4 y = *reinterpret_cast<const uint4 *>(src);
                        w[0] = y.x, w[1] = y.y, w[NB - 2] = y.z, w[NB - 1] = y.w;
                    } else {
                        const uint2 y = *reinterpret_cast<const uint2 *>(src);
                        w[0] = y.x, w[1] = y.y;
                    }
                    const int far = key >= from && key < to ? ref : 1000;      // (what no row sees is nothing)
#pragma unroll
                    for (int b = 0; b < NB; ++b) {
                        meta[b] = HIF4 ? reinterpret_cast<const uint32_t *>(ks)[b >> 1] : ks[b];
                        sc[b] = f16_scale<HIF4>(meta[b], far);
                    }
#pragma unroll
                    for (int b = 0; b < NB; ++b)
                        *reinterpret_cast<uint4 *>(dst + (b >> 1) * 16384 + ((b & 1) ? k_at1 : k_at0)) =
                            codes_f16<HIF4>(w[b], sc[b], meta[b], 4 * (b & 1) + kc);
                    src += 32 * S::kCode, ks += 32 * S::kScale, dst += 32 * 128;
                }
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(&bar.k_full[buf]);
                    mbar_arrive(&bar.empty[slot]);
                }
                if (++slot == DEPTH) {
                    slot = 0;
                    ring ^= 1;
                }
            }
            if (!ok)
                break;
            walk.next(p);
        }
    } else if (warp < kMma) {
        // ------------------------------------------------ V
        // A thread has D / 8 dimensions of one key in 16: its place in the cache's tile of 16.
        const int t = tid - 32 * kValues, vg = (t >> 3) & 7, vb = vg * (D / 8) / 32;
        const int vkey = 8 * (t >> 6) + 2 * ((t >> 1) & 3) + (t & 1);
        const uint32_t v_at = ((vg * (D / 64) & 7) ^ (vkey & 7)) << 4;
        uint32_t j = 0, slot = 0, ring = 0;
        bool ok = true;
#pragma unroll 1
        while (walk.more()) {
            const int least = walk.least;
#pragma unroll 1
            for (; walk.i < walk.i1; ++walk.i, ++j) {
                const uint32_t buf = j & 1;
                ok = wait(&bar.full[slot], ring) && wait(&bar.units[slot], ring) &&
                     wait(&bar.v_empty[buf], ((j >> 1) & 1) ^ 1);
                if (!ok)
                    break;
                const int key0 = walk.kb + walk.i * 128, ref = s_unit[slot][vb];
                const int from = least - key0, to = walk.ke - key0;
                constexpr int VW = D / 64;   // words of a thread's piece of a key
                const uint8_t *src = smem + S::kRing + slot * S::kBytes + S::kVOff + t * (4 * VW);
                const uint8_t *vs = smem + S::kRing + slot * S::kBytes + S::kVsOff + vkey * S::kScale + (HIF4 ? (vb >> 1) * 4 : vb);
                uint8_t *dst = smem + S::kV + buf * S::kOperand + (vg * VW >> 3) * 16384 + vkey * 128;
                if (t < NB)
                    s_vref[buf][t] = s_unit[slot][t];
#pragma unroll 1
                for (int key = vkey; key < 128; key += 16) {
                    uint32_t w[VW];
                    if (D == 128) {
                        const uint2 y = *reinterpret_cast<const uint2 *>(src);
                        w[0] = y.x, w[VW - 1] = y.y;
                    } else {
                        w[0] = *reinterpret_cast<const uint32_t *>(src);
                    }
                    const uint32_t meta = HIF4 ? *reinterpret_cast<const uint32_t *>(vs) : *vs;
                    const uint32_t sc = f16_scale<HIF4>(meta, key >= from && key < to ? ref : 1000);
#pragma unroll
                    for (int k = 0; k < VW; ++k)
                        *reinterpret_cast<uint4 *>(dst + (v_at ^ (k << 4))) = codes_f16<HIF4>(w[k], sc, meta, (vg * VW & 7) + k);
                    src += 8 * D, vs += 16 * S::kScale, dst += 16 * 128;
                }
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(&bar.v_full[buf]);
                    mbar_arrive(&bar.empty[slot]);
                }
                if (++slot == DEPTH) {
                    slot = 0;
                    ring ^= 1;
                }
            }
            if (!ok)
                break;
            walk.next(p);
        }
    } else if (warp == kUnits) {
        // ------------------------------------------------ the powers of two
        uint32_t slot = 0, ring = 0;
        bool ok = true;
#pragma unroll 1
        while (walk.more()) {
            const int least = walk.least;
            int ref[NB + 1];
#pragma unroll
            for (int b = 0; b <= NB; ++b)
                ref[b] = -1000;
#pragma unroll 1
            for (; walk.i < walk.i1; ++walk.i) {
                ok = wait(&bar.full[slot], ring);
                if (!ok)
                    break;
                // the largest exponents of the keys that some row sees, with room to grow by 3
                const uint8_t *const src = smem + S::kRing + slot * S::kBytes;
                int top[NB + 1];
#pragma unroll
                for (int b = 0; b <= NB; ++b)
                    top[b] = -2000;
#pragma unroll 1
                for (int k = lane; k < 128; k += 32) {
                    const int key = walk.kb + walk.i * 128 + k;
                    if (key >= walk.ke || key < least)
                        continue;
                    const uint8_t *const ks = src + S::kKsOff + k * S::kScale, *const vs = src + S::kVsOff + k * S::kScale;
#pragma unroll
                    for (int b = 0; b < NB; ++b) {
                        const int at = HIF4 ? (b >> 1) * 4 : b;
                        top[b] = max(top[b], (int)(HIF4 ? (vs[at] >> 2) & 63 : vs[at]));
                        top[NB] = max(top[NB], (int)(HIF4 ? (ks[at] >> 2) & 63 : ks[at]));
                    }
                }
#pragma unroll
                for (int b = 0; b <= NB; ++b) {
                    const int e = __reduce_max_sync(kAll, top[b]);
                    if (e > ref[b] + 3)
                        ref[b] = e;
                    if (lane == 0)
                        s_unit[slot][b] = ref[b];
                }
                if (lane == 0)
                    mbar_arrive(&bar.units[slot]);
                if (++slot == DEPTH) {
                    slot = 0;
                    ring ^= 1;
                }
            }
            if (!ok)
                break;
            walk.next(p);
        }
    } else if (warp == kMma) {
        // ------------------------------------------------ MMAs
        constexpr uint32_t id_s = idesc_f16(128, 128, false), id_o = idesc_f16(128, D, true);
        const uint64_t q_desc = sdesc_k_sw128(smem_u32(smem + S::kQ));
        const uint32_t k_at = smem_u32(smem + S::kK), v_at = smem_u32(smem + S::kV);
        auto scores = [&](uint32_t j) {
            const uint32_t buf = j & 1, ph = (j >> 1) & 1;
            if (!wait(&bar.k_full[buf], ph) || !wait(&bar.s_empty[buf], ph ^ 1))
                return false;
            tc_fence_after();
            if (lane == 0) {
                const uint64_t k_desc = sdesc_k_sw128(k_at + buf * S::kOperand);
#pragma unroll
                for (int k = 0; k < D / 16; ++k) {           // (offsets in 16 bytes)
                    const int at = (k >> 2) * 1024 + (k & 3) * 2;
                    tc_mma_f16(tmem + buf * 128, q_desc + at, k_desc + at, id_s, k > 0);
                }
                tc_commit(&bar.k_empty[buf]);
                tc_commit(&bar.s_full[buf]);
            }
            __syncwarp();
            return true;
        };
        auto sums = [&](uint32_t j, bool first) {
            const uint32_t buf = j & 1, ph = (j >> 1) & 1;
            if (!wait(&bar.p_full[buf], ph) || !wait(&bar.v_full[buf], ph))
                return false;
            tc_fence_after();
            if (lane == 0) {
                const uint64_t v_desc = sdesc_n_sw128(v_at + buf * S::kOperand);
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    tc_mma_f16_ts(tmem + 256, tmem + 384 + buf * 64 + 8 * k, v_desc + 128 * k, id_o, !first || k > 0);
                tc_commit(&bar.v_empty[buf]);
            }
            __syncwarp();
            return true;
        };
        uint32_t j = 0;
        bool ok = true;
#pragma unroll 1
        while (ok && walk.more()) {
            const int n = walk.i1 - walk.i;
#pragma unroll 1
            for (int k = 0; ok && k <= n; ++k) {
                if (k < n)
                    ok = scores(j + k);
                if (ok && k > 0)
                    ok = sums(j + k - 1, k == 1);
            }
            j += n;
            walk.i = walk.i1;
            if (ok)
                walk.next(p);
        }
        if (lane == 0) {
            tc_commit(&bar.drain);           // (all of them, before TMEM goes back)
            mbar_wait(&bar.drain, 0, kWaitLimitNs);
        }
    } else {
        // ------------------------------------------------ copies
        // Lane (piece, array) copies gran keys of one array.
        const int arr = lane & 3, page_size = a.cache.page_size;
        const uint32_t unit = arr < 2 ? S::kCode : S::kScale;
        const uint8_t *const src = static_cast<const uint8_t *>(arr == 0   ? a.cache.k_codes
                                                                : arr == 1 ? a.cache.v_codes
                                                                : arr == 2 ? a.cache.k_scales
                                                                           : a.cache.v_scales);
        const uint32_t dst = smem_u32(smem + S::kRing) +
                             (arr == 0 ? 0 : arr == 1 ? S::kVOff : arr == 2 ? S::kKsOff : S::kVsOff) +
                             (lane >> 2) * p.gran * unit;
        const bool copies = (lane >> 2) < 128 / p.gran;
        const uint64_t head_bytes = (uint64_t)page_size * unit;
        uint32_t slot = 0, ring = 0, filled = 0;
        // a chunk's page, head and place in the page: read a chunk before they are used
        int page = -1, head = 0;
        uint32_t off = 0;
        bool in = false;
        auto next = [&]() {
            const int key = walk.kb + walk.i * 128 + (lane >> 2) * p.gran;
            in = copies && key < walk.ke;
            const uint32_t pg = (uint32_t)key / (uint32_t)page_size;
            head = walk.head;
            off = (key - pg * page_size) * unit;
            page = -1;
            if (in)
                page = a.table[(int64_t)walk.r * a.width + pg];
            if (++walk.i == walk.i1)
                walk.next(p);
        };
        bool left = walk.more();
        if (left && !__all_sync(kAll, held_start_wait(p.status, bar.limit))) {
            *reinterpret_cast<volatile int32_t *>(&bar.abort) = 1;
            left = false;
        }
        if (left)
            next();
#pragma unroll 1
        while (left) {
            const bool have = in && page >= 0 && page < a.cache.pages;
            if (in && !have)
                atomicCAS(p.status, kDevOk, kDevBadGroups);
            const uint8_t *const from = src + ((uint64_t)(have ? page : 0) * H + head) * head_bytes + off;
            left = walk.more();
            if (left)
                next();
            if (!wait(&bar.empty[slot], ring ^ 1))
                break;
            const uint32_t pieces = __popc(__ballot_sync(kAll, have)) >> 2;
            if (lane == 0)
                mbar_arrive_expect_tx(&bar.full[slot], pieces * p.gran * (2 * S::kCode + 2 * S::kScale));
            __syncwarp();
            if (have)
                bulk_load_at(dst + slot * S::kBytes, from, p.gran * unit, &bar.full[slot]);
            ++filled;
            if (++slot == DEPTH) {
                slot = 0;
                ring ^= 1;
            }
        }
        // (copies in flight land before the CTA's memory goes: fill f is phase f / DEPTH of its slot)
        for (uint32_t f = filled > DEPTH ? filled - DEPTH : 0; f < filled; ++f)
            mbar_wait(&bar.full[f % DEPTH], (f / DEPTH) & 1, kWaitLimitNs);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == kMma)
        tmem_dealloc(tmem, kTmemCols);

    // ---- the parts of segments that CTAs share (the first and the last of this one)
    if (a.q_start && warp == kUnits)
        clear_rest(a, lane, 32);
    const int nshared = s_nshared;
    if (nshared == 0)
        return;
    if (warp < kKeys)
        __threadfence();
    __syncthreads();
    if (tid < nshared) {
        Shared &f = s_shared[tid];
        f.c0 = owner(sh, f.seg + S::kStart);
        f.c1 = owner(sh, f.seg + S::kStart + f.chunks - 1);
        f.last = atomicAdd(p.counter + f.c0, 1) == f.c1 - f.c0;
    }
    __syncthreads();
#pragma unroll 1
    for (int s = 0; s < nshared; ++s) {
        const Shared f = s_shared[s];
        if (!f.last)
            continue;
        __threadfence();
        if (tid == 0)
            atomicExch(p.counter + f.c0, 0);
        // a thread takes every third 8 dimensions of a row
        constexpr int kThird = 3, kPieces = (D / 8 + kThird - 1) / kThird;
        const int row = tid & 127, ch0 = tid >> 7, ri = f.row0 + row;
        if (ch0 >= kThird || row >= f.rows)
            continue;
        float y[kPieces][8], m = -INFINITY, l = 0.f;
#pragma unroll
        for (int i = 0; i < 8 * kPieces; ++i)
            y[i / 8][i % 8] = 0.f;
#pragma unroll 1
        for (int k = f.c0; k <= f.c1; ++k) {
            const float4 *const d = reinterpret_cast<const float4 *>(p.part + (2 * k + (k == f.c0 ? 1 : 0)) * S::kPart);
            const float2 ml = __ldcg(reinterpret_cast<const float2 *>(d + (D / 4) * 128) + row);
            float4 x[kPieces][2];
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                const int ch = min(ch0 + kThird * i, D / 8 - 1);
                x[i][0] = __ldcg(d + 2 * ch * 128 + row), x[i][1] = __ldcg(d + (2 * ch + 1) * 128 + row);
            }
            const float top = fmaxf(m, ml.x);
            const float fa = m == -INFINITY ? 0.f : ex2(m - top), fb = ml.x == -INFINITY ? 0.f : ex2(ml.x - top);
            l = l * fa + ml.y * fb;
            m = top;
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                const float z[8] = {x[i][0].x, x[i][0].y, x[i][0].z, x[i][0].w, x[i][1].x, x[i][1].y, x[i][1].z, x[i][1].w};
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    y[i][e] = y[i][e] * fa + z[e] * fb;
            }
        }
        const int64_t at = (int64_t)(f.q0 + ri / G) * a.heads + f.head * G + ri % G;
        const float inv = inverse(l);
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int ch = ch0 + kThird * i;
            if (ch < D / 8)
                reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(a.out) + at * D)[ch] =
                    make_uint4(pack_bf16(y[i][0] * inv, y[i][1] * inv), pack_bf16(y[i][2] * inv, y[i][3] * inv),
                               pack_bf16(y[i][4] * inv, y[i][5] * inv), pack_bf16(y[i][6] * inv, y[i][7] * inv));
        }
        if (a.lse && ch0 == 0)
            a.lse[at] = log_sum(m, l);
    }
}

template <int FMT, int D>
cudaError_t launch(const AttnParams &p, cudaStream_t st)
{
    using S = Tile<FMT, D>;
    static_assert(S::kSmem <= 226 * 1024, "fits an SM");
    static PerDevice<bool> allowed;
    if (cudaError_t e = allow_smem(reinterpret_cast<const void *>(kv_attention_tile_kernel<FMT, D>), S::kSmem, allowed))
        return e;
    return launch_early(kv_attention_tile_kernel<FMT, D>, dim3(num_sms()), S::kThreads, S::kSmem, st, 1, p);
}

} // namespace

size_t kv_attention_tile_part_bytes(int32_t head_dim) { return (size_t)128 * (head_dim + 2) * 4; }

cudaError_t launch_kv_attention_tile(const AttnParams &p, cudaStream_t st)
{
    AttnParams t = p;
    // the longest piece that never crosses a page: a power of two that divides it
    // (a copy costs its thread some 100 clocks, whatever its size)
    const int page = p.a.cache.page_size, pow2 = page & -page;
    t.gran = pow2 < 128 ? pow2 : 128;
    const bool wide = p.a.cache.head_dim == 128;
    if (p.a.cache.fmt == RFQ_FMT_HIF4)
        return wide ? launch<RFQ_FMT_HIF4, 128>(t, st) : launch<RFQ_FMT_HIF4, 64>(t, st);
    return wide ? launch<RFQ_FMT_MXFP4, 128>(t, st) : launch<RFQ_FMT_MXFP4, 64>(t, st);
}

} // namespace rfq
