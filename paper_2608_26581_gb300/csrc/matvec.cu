// matvec.cu -- y = x W~^T for a few rows of x (rfq_matvec): the linear layer
// of a decoding step, x kept in bf16 and W~ in 4 bits with its group scales.
//
// Bound: HBM, the N K (1/2 + 1/32 or 1/16) bytes of W~.  At the measured copy
// rate an SM has 44 codes to decode per clock with 128 lanes, so the ALUs may
// spend 2.9 operations on a code: W~ is the A operand of mma.m16n8k16 (16
// rows of W~, 8 rows of x in B), its codes converted to f16 two at a time by
// one instruction and multiplied unscaled.  A block's scale multiplies the
// fp32 sums of its 32 (MXFP4) or 64 (HiF4) products, so neither the scale nor
// the codes are rounded.  x is made f16 by a power of two per row of x and
// step of K, 512 codes up to 8 rows and 256 beyond (its maximum lands in
// [2^14, 2^15)): bf16 values down to 2^-28 of the maximum are exact, the rest
// are off by less than 2^-39 of it.
//
// Each of a CTA's 16 warps streams its own boxes, 16 rows of W~ x 256 codes,
// through a ring that it alone fills (TMA, 128-byte swizzle) and empties
// (ldmatrix hands every lane its 8 codes of a 32-code block without a bank
// conflict), so nothing in the main loop waits for another warp.  A CTA has a
// run of 16-row tiles and one share of K; its boxes, tile by tile, are dealt
// to the warps in equal contiguous runs, and the parts of a tile that two
// warps share are added in the order of the warps.  x lies in shared memory
// in the order of the B operand.  K is split over a cluster only where that
// pays (split_of): the CTAs' parts are then added over distributed shared
// memory, in the order of the ranks.  All sums have a fixed order: a call
// gives the same bits every time.
//
// Measured, MXFP4: 1 x 4096 x 24576 12.8 us, 4.2 TB/s, 62% of the copy rate;
// 8 x 5120 x 13824 13.0 us; 32 rows 30.7 us; 13 x 12288 x 4096 in HiF4 18.6 us.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <cstdint>
#include <cstdlib>

#include "internal.h"
#include "kv_layout.cuh"
#include "mxfp4_math.cuh"
#include "ptx.cuh"

namespace rfq {
namespace {

constexpr int kWarps = 16, kThreads = 32 * kWarps;
constexpr int kTile = 16;                    // rows of W~ per tile
constexpr int kBoxK = 256;                   // codes per row of a box (128 bytes)
constexpr int kBoxBytes = kTile * kBoxK / 2;
constexpr int kMaxDepth = 6;                 // steps in a warp's ring
constexpr int kSmemBytes = 225 * 1024;
// MP: rows of x rounded up to a power of two.  The eight columns of an MMA
// hold min(MP, 8) rows of x times kCb blocks of 32 codes: column n is row
// n / kCb and block n % kCb of a group of kCb, and a block's MMAs see x in
// its own columns and zeros in the others.  With one row the sums of all
// eight blocks of a box thus stay apart in one accumulator, and the scales
// multiply four numbers a lane and box instead of 32.
template <int MP>
struct Shape {
    static constexpr int kNt = MP > 8 ? MP / 8 : 1;                // column tiles
    static constexpr int kCb = MP < 8 ? 8 / MP : 1;
    static constexpr int kPart = kNt * 512;  // bytes of one tile's sums: [tile][lane][4] fp32
    static constexpr int kTiles = 48 / kNt;  // most tiles of a CTA
    // a step of the loop is two boxes along K, or one where x takes the room
    static constexpr int kBx = kNt == 1 ? 2 : 1;
    static constexpr int kStepK = kBx * kBoxK, kStepBytes = kBx * kBoxBytes;
    static constexpr int kBlockX = MP * 64;  // bytes of a block of 32 codes' x: [row][4][16 bytes]
    static constexpr int kStepX = kStepK / 32 * kBlockX;
    static constexpr int kZero = MP < 8 ? kStepX : 0;              // zeros that the other blocks' columns read
    // bytes of x in shared memory: with several column tiles all that leaves
    // rings of two steps (a second phase costs more than the deeper rings give:
    // 13 x 12288 x 4096, HiF4, 18.9 us with 12 steps of x, 22.7 with 9)
    static constexpr int kMaxX = kNt > 1 ? kSmemBytes - 1024 - (kWarps + kTiles) * kPart - 2 * kWarps * kStepBytes
                                         : 80 * 1024;
};

__device__ __forceinline__ void ldmatrix_x4(uint32_t addr, uint32_t (&r)[4])
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr));
}

struct Params {
    const __nv_bfloat16 *x;
    int64_t x_row;
    int M;
    int N, K;
    const uint8_t *scales;
    int mma_layout;
    int words;             // four blocks' E8M0 bytes are an aligned word
    void *y;
    int bf16;
    int tiles;             // of W~
    int steps;             // along K
    int phase;             // steps of K at a time (what of x fits)
    int depth;             // of the rings
#ifdef RFQ_DEBUG_BOUNDS
    int hold_us;           // not 0: no box is copied, and a wait lasts this long
#endif
};

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi)
{
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}

// A box's scale words that a lane needs, and where the next box's lie.
//   MXFP4  the words (four blocks) of rows g and g + 8 that hold the blocks of
//          its columns: one half of the box with kCb = 8, else both
//   HiF4   block c of the box, rows g and g + 8 (the others by shuffles)
template <int FMT, int CB, int BX>
struct Scales {
    static constexpr bool kHif4 = FMT == RFQ_FMT_HIF4;
    static constexpr int kHalves = kHif4 || CB == 8 ? 1 : 2;
    static constexpr int kN = 2 * kHalves;       // words a box
    const uint8_t *at[2];      // rows g and g + 8
    int64_t step, half;        // bytes to the next box, to the other half
    int k;                     // code of at[]'s first word
    bool in[2];                // rows of W~
    __device__ __forceinline__ void tile(const Params &p, int n, int step0, int c)   // n: row g of the tile
    {
        k = step0 * BX * kBoxK + (kHif4 ? 64 * c : CB == 8 ? 128 * (c >> 1) : 0);
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int m = n + 8 * r;
            in[r] = m < p.N;
            if (kHif4) {
                const int64_t pad = (p.N + 127) / 128 * 128;
                at[r] = p.scales + 4 * (p.mma_layout ? (int64_t)(k / 64) * pad + m : (int64_t)m * (p.K / 64) + k / 64);
                step = p.mma_layout ? 16 * pad : 16;
                half = 0;
            } else {
                at[r] = p.scales + (p.mma_layout ? sf_mma_offset(m, k / 32, p.K / 128) : (int64_t)m * (p.K / 32) + k / 32);
                step = p.mma_layout ? 1024 : 8;
                half = p.mma_layout ? 512 : 4;
            }
        }
    }
    // the words of a step: [box][half][row]
    __device__ __forceinline__ void load(const Params &p, uint32_t (&w)[BX * kN])
    {
#pragma unroll
        for (int b = 0; b < BX; ++b)
#pragma unroll
            for (int h = 0; h < kHalves; ++h)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const uint8_t *const s = at[r] + b * step + h * half;
                    const int kk = k + b * kBoxK + 128 * h;
                    uint32_t v = 0;
                    if (kHif4 || p.words) {
                        if (in[r] && kk < p.K)
                            v = *reinterpret_cast<const uint32_t *>(s);
                    } else if (in[r]) {    // row-major E8M0 rows that are not whole words
                        for (int j = 0; j < 4; ++j)
                            if (kk + 32 * j < p.K)
                                v |= (uint32_t)s[j] << (8 * j);
                    }
                    w[b * kN + 2 * h + r] = v;
                }
        at[0] += BX * step;
        at[1] += BX * step;
        k += BX * kBoxK;
    }
};

// Waits for a ring's boxes in flight, of slots `slot` to `end`: they land before
// sums are laid over them and before the CTA's memory goes.
__device__ __forceinline__ void let_land(uint64_t *full, int depth, int slot, uint32_t parity, int end, uint64_t limit)
{
    do {
        mbar_wait(full + slot, parity, limit);
        if (++slot == depth) {
            slot = 0;
            parity ^= 1;
        }
    } while (slot != end);
}

template <int FMT, int MP>
__global__ void __launch_bounds__(kThreads, 1) matvec_kernel(const __grid_constant__ CUtensorMap wmap, const Params p)
{
    using S = Shape<MP>;
    constexpr bool HIF4 = FMT == RFQ_FMT_HIF4;
    constexpr int NT = S::kNt, CB = S::kCb, BX = S::kBx, kStepK = S::kStepK, kStepBytes = S::kStepBytes;
    constexpr uint32_t kAll = 0xFFFFFFFFu;
    extern __shared__ uint8_t smem_raw[];
    __shared__ alignas(8) uint64_t s_full[kWarps][kMaxDepth];
    __shared__ int4 s_run[kWarps];           // [first box, end) of each warp, its first and last tile
    uint8_t *const smem = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, c = lane & 3;
    const int M = MP == 1 ? 1 : p.M;
    uint8_t *const s_ring = smem + warp * p.depth * kStepBytes;
    // a warp's part of its first tile, in s_head; of its last, over its ring (all read by then)
    uint8_t *const s_head = smem + kWarps * p.depth * kStepBytes;
    uint8_t *const s_tot = s_head + kWarps * S::kPart;             // [tile] sums
    uint8_t *const s_zero = s_tot + S::kTiles * S::kPart;
    uint8_t *const s_x = s_zero + S::kZero;                        // [block][row][4][16 bytes]
    float *const s_xs = reinterpret_cast<float *>(s_x + p.phase * S::kStepX);   // [step][row] undoes x's power of two

    const int split = (int)gridDim.x, rank = blockIdx.x;           // a cluster spans x
    const int t0 = (int)((uint32_t)p.tiles * blockIdx.y / gridDim.y);
    const int nt = (int)((uint32_t)p.tiles * (blockIdx.y + 1) / gridDim.y) - t0;
    const int b0 = (uint32_t)p.steps * rank / split, b1 = (uint32_t)p.steps * (rank + 1) / split;

    if (lane == 0) {
        for (int i = 0; i < p.depth; ++i)
            mbar_init(&s_full[warp][i], 1);
        fence_mbar_init();
    }
    for (int i = tid; i < S::kZero / 16; i += kThreads)
        reinterpret_cast<uint4 *>(s_zero)[i] = make_uint4(0, 0, 0, 0);
    __syncwarp();
    if (tid == 0)
        prefetch_tmap(&wmap);
    wait_for_previous();
    let_next_start();
#ifdef RFQ_DEBUG_BOUNDS
    const bool held = p.hold_us > 0;
    const uint64_t limit = held ? p.hold_us * 1000ull : kWaitLimitNs;
#else
    constexpr bool held = false;
    constexpr uint64_t limit = kWaitLimitNs;
#endif
    // No wait of this lane has run out.  One that has waits for nothing more, its
    // sums are NaN from then on, and if it is lane 0 the warp copies nothing more.
    bool ok = true;
    int slot = 0;                                                  // of the ring, and its phase
    uint32_t parity = 0;

    for (int pb = b0; pb < b1; pb += p.phase) {
        const int nb = min(p.phase, b1 - pb);                      // steps of a tile in this phase
        const uint32_t all = nt * nb;
        const int f0 = (int)(all * warp / kWarps), f1 = (int)(all * (warp + 1) / kWarps);
        const int first = f0 / nb, last = f1 > f0 ? (f1 - 1) / nb : first;   // this warp's tiles
        // what comes next into the ring: step fstep of tile ftile, at slot fslot
        int fstep = f0 - first * nb, ftile = first, fslot = slot, left = f1 - f0;
        auto fetch = [&]() {
            if (left <= 0)
                return;
            if (lane == 0 && ok && !held) {
                mbar_arrive_expect_tx(&s_full[warp][fslot], kStepBytes);
#pragma unroll
                for (int i = 0; i < BX; ++i)
                    tma_load_2d(s_ring + fslot * kStepBytes + i * kBoxBytes, &wmap, &s_full[warp][fslot],
                                (pb + fstep) * (kStepK / 2) + i * (kBoxK / 2), (t0 + ftile) * kTile);
            }
            --left;
            if (++fstep == nb) {
                fstep = 0;
                ++ftile;
            }
            if (++fslot == p.depth)
                fslot = 0;
        };
        // x of the phase as f16, each (row, step) scaled by a power of two
        auto load_x = [&](int i, uint4 (&u)[BX]) {
            const int st = i / M, m = i - st * M, k = (pb + st) * kStepK + lane * 8;
#pragma unroll
            for (int j = 0; j < BX; ++j)
                u[j] = make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int j = 0; j < BX; ++j)
                if (k + j * kBoxK < p.K)       // (volatile: where it stands)
                    asm volatile("ld.global.v4.b32 {%0, %1, %2, %3}, [%4];"
                                 : "=r"(u[j].x), "=r"(u[j].y), "=r"(u[j].z), "=r"(u[j].w)
                                 : "l"(p.x + m * p.x_row + k + j * kBoxK));
        };
        auto store_x = [&](int i, const uint4 (&u)[BX]) {
            const int st = i / M, m = i - st * M;
            float f[BX][8], mx = 0.f;
#pragma unroll
            for (int j = 0; j < BX; ++j) {
                bf16x8_to_f32(u[j], f[j]);
                mx = fmaxf(mx, absmax8(f[j]));
            }
            // (non-negative floats compare as integers)
            mx = __uint_as_float(__reduce_max_sync(kAll, __float_as_uint(mx)));
            const int e = (int)(__float_as_uint(mx) >> 23) - 127 - 14;   // x 2^-e: the maximum in [2^14, 2^15)
            const int ec = max(min(e, 119), -126);
            const float mul = __uint_as_float((uint32_t)(127 - ec) << 23);
            if (lane == 0)                                         // (HiF4: a code's 2^-9 and the 1/4 of its step)
                s_xs[st * MP + m] = __uint_as_float((uint32_t)(127 + ec + (HIF4 ? 7 : 0)) << 23);
#pragma unroll
            for (int j = 0; j < BX; ++j) {
                uint32_t h[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    // HiF4 codes decode in the order 0 2 | 1 3 | 4 6 | 5 7
                    const int lo = HIF4 ? (q >> 1) * 4 + (q & 1) : 2 * q, hi = HIF4 ? lo + 2 : lo + 1;
                    h[q] = pack_f16(f[j][lo] * mul, f[j][hi] * mul);
                }
                *reinterpret_cast<uint4 *>(s_x + st * S::kStepX + (8 * j + g) * S::kBlockX + ((m * 4 + c) << 4)) =
                    make_uint4(h[0], h[1], h[2], h[3]);
            }
        };
        // (loops, not unrolled: a short kernel pays for every line of code it
        // fetches; four rows in flight where there are many, 32 x 5120 x 13824
        // 30.3 us against 31.9 with two)
        constexpr int kAhead = MP < 4 ? 1 : MP < 16 ? 2 : 4;
        const int tasks = nb * M;
#pragma unroll 1
        for (int i = warp; i < tasks; i += kAhead * kWarps) {
            uint4 u[kAhead][BX];
#pragma unroll
            for (int j = 0; j < kAhead; ++j)
                load_x(min(i + j * kWarps, tasks - 1), u[j]);
#pragma unroll
            for (int j = 0; j < kAhead; ++j)
                store_x(min(i + j * kWarps, tasks - 1), u[j]);
        }
        // W~ only now: its boxes in front of x in the memory's queues would
        // hold up every warp (15.0 us against 13.5 at 1 x 4096 x 24576)
        if (pb > b0)                                               // (the rings held parts of tiles)
            fence_proxy_async_smem();
#pragma unroll 1
        for (int i = 0; i < p.depth; ++i)
            fetch();
        Scales<FMT, CB, BX> sc;
        uint32_t next[BX * sc.kN];
        if (f0 < f1) {
            sc.tile(p, (t0 + first) * kTile + g, pb + f0 - first * nb, c);
            sc.load(p, next);
        }
        if (lane == 0)
            s_run[warp] = make_int4(f0, f1, first, last);
        __syncthreads();

        float acc[NT][4];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                acc[t][i] = 0.f;
        // this lane's column of B: row of x (past the last one: the last, a
        // column that nobody reads) and block of a group; for the other blocks
        // it reads zeros
        uint32_t xbase[NT][CB], xstep[CB];
        int xcol[NT][2];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int j = 0; j < CB; ++j)
                xbase[t][j] = (CB == 1 || g % CB == j) ? smem_u32(s_x) + ((min(8 * t + g / CB, M - 1) * 4 + c) << 4)
                                                       : smem_u32(s_zero);
            xcol[t][0] = min(8 * t + 2 * c / CB, M - 1);
            xcol[t][1] = min(8 * t + (2 * c + 1) / CB, M - 1);
        }
#pragma unroll
        for (int j = 0; j < CB; ++j)
            xstep[j] = CB == 1 || g % CB == j ? S::kStepX : 0;
        auto flush = [&](int t) {
            float4 *const d = reinterpret_cast<float4 *>(t == first  ? s_head + warp * S::kPart
                                                         : t == last ? s_ring
                                                                     : s_tot + t * S::kPart);
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                float4 v = make_float4(acc[j][0], acc[j][1], acc[j][2], acc[j][3]);
                if (!ok)
                    v.x = v.y = v.z = v.w = __int_as_float(0x7FFFFFFF);
                if (t != first && t != last && pb > b0) {
                    const float4 u = d[j * 32 + lane];
                    v.x += u.x, v.y += u.y, v.z += u.z, v.w += u.w;
                }
                d[j * 32 + lane] = v;
                acc[j][0] = acc[j][1] = acc[j][2] = acc[j][3] = 0.f;
            }
        };
        // ldmatrix: matrix lane / 8 = (8 rows (lane / 8) % 2, block parity lane / 16)
        const int row = ((lane >> 3) & 1) * 8 + (lane & 7);
        uint32_t aoff[4];
#pragma unroll
        for (int q = 0; q < 4; ++q)
            aoff[q] = smem_u32(s_ring) + row * 128 + (((q * 2 + (lane >> 4)) ^ (row & 7)) << 4);

        int tile = first, step = f0 - first * nb;
#pragma unroll 1
        for (int f = f0; f < f1; ++f) {
            uint32_t cur[BX * sc.kN];
#pragma unroll
            for (int i = 0; i < BX * sc.kN; ++i)
                cur[i] = next[i];
            if (f + 1 < f1) {
                if (step + 1 == nb)
                    sc.tile(p, (t0 + tile + 1) * kTile + g, pb, c);
                sc.load(p, next);
            }
            uint32_t xat[NT][CB];
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int j = 0; j < CB; ++j)
                    xat[t][j] = xbase[t][j] + step * xstep[j];
            if (ok && !mbar_wait(&s_full[warp][slot], parity, limit)) {
                ok = false;
                let_land(s_full[warp], p.depth, slot, parity, fslot, limit);
            }
            float win[NT][4];
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    win[t][i] = 0.f;
#pragma unroll
            for (int b = 0; b < BX; ++b) {
                float tmp[NT][4];
                const uint32_t *const w = cur + b * sc.kN;         // [half][row]
#pragma unroll
                for (int pair = 0; pair < 4; ++pair) {             // two 32-code blocks
                    uint32_t a[4];
                    ldmatrix_x4(aoff[pair] + slot * kStepBytes + b * kBoxBytes, a);
                    uint32_t m0 = 0, m1 = 0;                       // HiF4 metadata of rows g and g + 8
                    if (HIF4) {
                        m0 = __shfl_sync(kAll, w[0], 4 * g + pair);
                        m1 = __shfl_sync(kAll, w[1], 4 * g + pair);
                    }
#pragma unroll
                    for (int s = 0; s < 2; ++s) {
                        const int blk = pair * 2 + s;
                        uint32_t h0[4], h1[4];                     // rows g and g + 8
                        if (HIF4) {
                            s1p2x8_f16(a[2 * s], h0);
                            s1p2x8_f16(a[2 * s + 1], h1);
                            uint32_t e0, e1;
                            hif4_pow2_pair(m0, 4 * s + c, e0, e1);
                            h0[0] = hmul2(h0[0], e0), h0[1] = hmul2(h0[1], e0);
                            h0[2] = hmul2(h0[2], e1), h0[3] = hmul2(h0[3], e1);
                            hif4_pow2_pair(m1, 4 * s + c, e0, e1);
                            h1[0] = hmul2(h1[0], e0), h1[1] = hmul2(h1[1], e0);
                            h1[2] = hmul2(h1[2], e1), h1[3] = hmul2(h1[3], e1);
                        } else {
                            e2m1x8_f16(a[2 * s], h0);
                            e2m1x8_f16(a[2 * s + 1], h1);
                        }
                        // (a HiF4 block of 64 is two of these: with one block a
                        // column its sums stay in tmp until the second)
                        constexpr int GROUP = CB > 1 ? CB : HIF4 ? 2 : 1;
#pragma unroll
                        for (int t = 0; t < NT; ++t) {
                            uint4 x;
                            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                                         : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w)
                                         : "r"(xat[t][blk % CB] + (8 * b + blk) * S::kBlockX));
                            if (blk % GROUP == 0)
                                mma_f16_first(tmp[t], h0[0], h1[0], h0[1], h1[1], x.x, x.y);
                            else
                                mma_f16(tmp[t], h0[0], h1[0], h0[1], h1[1], x.x, x.y);
                            mma_f16(tmp[t], h0[2], h1[2], h0[3], h1[3], x.z, x.w);
                        }
                        if (blk % GROUP == GROUP - 1) {
                            // scales of this lane's four sums: rows g, g + 8, columns 2c, 2c + 1
                            float u[2][2];
#pragma unroll
                            for (int r = 0; r < 2; ++r) {
                                if (HIF4) {             // CB 8: 64-code block c; 4: block c % 2 of the half box;
                                                        // 2 and 1: the one at hand
                                    u[r][0] = u[r][1] = hif4_macro_f32(
                                        CB == 8   ? w[r]
                                        : CB == 4 ? __shfl_sync(kAll, w[r], 4 * g + (blk >> 2) * 2 + (c & 1))
                                        : r       ? m1
                                                  : m0);
                                } else if (CB >= 4) {   // 8: blocks 2c, 2c + 1; 4: (blk / 4) 4 + 2c % 4, + 1
                                    const uint32_t v = w[(CB == 8 ? 0 : (blk >> 2) * 2) + r] >> (16 * (c & 1));
                                    u[r][0] = e8m0_byte(v, 0), u[r][1] = e8m0_byte(v, 1);
                                } else {
                                    const uint32_t v = w[(blk >> 2) * 2 + r];
                                    u[r][0] = e8m0_byte(v, CB == 2 ? (blk & 2) : blk & 3);
                                    u[r][1] = CB == 2 ? e8m0_byte(v, (blk & 2) + 1) : u[r][0];
                                }
                            }
#pragma unroll
                            for (int t = 0; t < NT; ++t)
#pragma unroll
                                for (int i = 0; i < 4; ++i)
                                    win[t][i] = fmaf(tmp[t][i], u[i >> 1][i & 1], win[t][i]);
                        }
                    }
                }
            }
            __syncwarp();                                          // every lane has read the step
            fetch();
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const float x0 = s_xs[step * MP + xcol[t][0]], x1 = CB > 1 ? x0 : s_xs[step * MP + xcol[t][1]];
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    acc[t][i] = fmaf(win[t][i], i & 1 ? x1 : x0, acc[t][i]);
            }
            if (++slot == p.depth) {
                slot = 0;
                parity ^= 1;
            }
            if (++step == nb || f + 1 == f1) {
                flush(tile);
                if (step == nb) {
                    step = 0;
                    ++tile;
                }
            }
        }
        __syncthreads();
        // tiles that a warp began or ended with: the warps' parts in order
        for (int t = warp; t < nt; t += kWarps) {
            float4 *const d = reinterpret_cast<float4 *>(s_tot + t * S::kPart);
            float4 v[NT];
#pragma unroll
            for (int j = 0; j < NT; ++j)
                v[j] = pb > b0 ? d[j * 32 + lane] : make_float4(0.f, 0.f, 0.f, 0.f);
            bool inner = false;
            for (int w = 0; w < kWarps; ++w) {
                const int4 run = s_run[w];
                if (run.x == run.y || t < run.z || t > run.w)
                    continue;
                if (t != run.z && t != run.w) {
                    inner = true;
                    break;
                }
                const float4 *const q =
                    reinterpret_cast<const float4 *>(t == run.z ? s_head + w * S::kPart : smem + w * p.depth * kStepBytes);
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    const float4 u = q[j * 32 + lane];
                    v[j].x += u.x, v[j].y += u.y, v[j].z += u.z, v[j].w += u.w;
                }
            }
            if (!inner)
#pragma unroll
                for (int j = 0; j < NT; ++j)
                    d[j * 32 + lane] = v[j];
        }
        // a tile's y is written by the warp that summed it, unless other CTAs
        // or another phase add to it
        if (split > 1 || pb + p.phase < b1)
            __syncthreads();
    }

    // ---- y: with a cluster, the ranks' sums in order, each rank a share of the tiles
    if (split > 1)
        cluster_sync();
    for (int t = rank * kWarps + warp; t < nt; t += split * kWarps) {
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            float v[4] = {0.f, 0.f, 0.f, 0.f};
            const uint32_t at = smem_u32(s_tot) + t * S::kPart + (j * 32 + lane) * 16;
            // (all ranks' loads in flight before the first sum)
            float u[8][4];
#pragma unroll
            for (int q = 0; q < 8; ++q)
                if (q < split)
                    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                                 : "=f"(u[q][0]), "=f"(u[q][1]), "=f"(u[q][2]), "=f"(u[q][3])
                                 : "r"(split > 1 ? mapa_shared(at, q) : at));
#pragma unroll
            for (int q = 0; q < 8; ++q)
                if (q < split)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        v[i] += u[q][i];
            // the columns of a row of x
            if (CB >= 2) {
                v[0] += v[1];
                v[2] += v[3];
            }
            if (CB >= 4) {
                v[0] += __shfl_xor_sync(kAll, v[0], 1);
                v[2] += __shfl_xor_sync(kAll, v[2], 1);
            }
            if (CB >= 8) {
                v[0] += __shfl_xor_sync(kAll, v[0], 2);
                v[2] += __shfl_xor_sync(kAll, v[2], 2);
            }
            const bool owner = CB < 4 || 2 * c % CB == 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (CB >= 2 && (i & 1))
                    continue;
                const int m = 8 * j + (2 * c + (i & 1)) / CB, n = (t0 + t) * kTile + g + (i >> 1) * 8;
                if (owner && m < M && n < p.N) {
                    if (p.bf16)
                        static_cast<__nv_bfloat16 *>(p.y)[(int64_t)m * p.N + n] = __float2bfloat16_rn(v[i]);
                    else
                        static_cast<float *>(p.y)[(int64_t)m * p.N + n] = v[i];
                }
            }
        }
    }
    if (split > 1)
        cluster_sync();
}

// CTAs along K (a cluster): the choice with the least time by a count of
// clocks of one SM: a box costs the decoding of its codes, and more with
// HiF4's sub-group scales or several column tiles; a row of x and step costs
// its conversion; a cluster its barriers and the sums over distributed shared
// memory, more the wider it is; a phase after the first (x does not fit at
// once) a pause.  Measured in us with 1, 2, 4 and 8 CTAs along K, MXFP4:
// 4 x 12288 x 4096 15.8, 11.8, 11.3, 13.5; 16 x 4096 x 4096 14.1, 9.9, 9.0,
// 12.3; 8 x 4096 x 4096 7.3, 7.4, 7.5, 9.8; 1 x 4096 x 24576 13.5, 17.0.
constexpr int kRowClocks = 25, kClusterClocks = 1000, kPhaseClocks = 3000;

// Clusters of `split` CTAs that the GPU holds at once (a GPC holds whole
// clusters only: 152 SMs are not 19 clusters of eight).
template <int FMT, int MP>
int clusters_at_once(int split)
{
    struct Counts {
        int n[4];                  // by log2(split), 0: not asked yet
    };
    static PerDevice<Counts> known;
    int &n = known.here().n[split == 1 ? 0 : split == 2 ? 1 : split == 4 ? 2 : 3];
    if (n == 0) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(split, num_sms());
        cfg.blockDim = dim3(kThreads);
        cfg.dynamicSmemBytes = kSmemBytes;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim = {(unsigned)split, 1, 1};
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        int got = 0;
        if (split == 1 || cudaOccupancyMaxActiveClusters(&got, matvec_kernel<FMT, MP>, &cfg) != cudaSuccess || got < 1)
            got = num_sms() / split;
        n = got;
    }
    return n;
}

template <int FMT, int MP>
int split_of(int64_t tiles, int steps, int phase, int M)
{
    using S = Shape<MP>;
    int best = 1;
    int64_t least = INT64_MAX;
    for (int s = 1; s <= 8 && s <= steps; s *= 2) {
        const int64_t groups = clusters_at_once<FMT, MP>(s);
        const int64_t waves = (tiles + groups * S::kTiles - 1) / (groups * S::kTiles);
        const int64_t rounds = (tiles + groups - 1) / groups, nb = (steps + s - 1) / s;
        const int64_t box = (FMT == RFQ_FMT_HIF4 ? 140 : 85) + 35 * (S::kNt - 1);
        const int64_t t = rounds * nb * S::kBx * box + waves * (M * nb * kRowClocks + (s > 1 ? s * kClusterClocks : 0) +
                                                                ((nb + phase - 1) / phase - 1) * kPhaseClocks);
        if (t < least) {
            least = t;
            best = s;
        }
    }
    return best;
}

template <int FMT, int MP>
cudaError_t launch(const MatvecArgs &a, cudaStream_t st)
{
    using S = Shape<MP>;
    const int64_t N = a.w.rows, K = a.w.k;
    const int64_t tiles = (N + kTile - 1) / kTile;
    const int steps = (int)((K + S::kStepK - 1) / S::kStepK);
    const int step_x = S::kStepX + MP * 4;                         // shared bytes of x a step
    const int most = S::kMaxX / step_x;
    static PerDevice<bool> allowed;
    if (cudaError_t e = allow_smem(reinterpret_cast<const void *>(matvec_kernel<FMT, MP>), kSmemBytes, allowed))
        return e;
    const int split = split_of<FMT, MP>(tiles, steps, most, a.M);
    const int nb = (steps + split - 1) / split, phase = nb < most ? nb : most;
    int64_t groups = clusters_at_once<FMT, MP>(split);
    if (groups > tiles)
        groups = tiles;
    if ((tiles + groups - 1) / groups > S::kTiles)
        groups = (tiles + S::kTiles - 1) / S::kTiles;
    const int fixed = 1024 + (kWarps + S::kTiles) * S::kPart + S::kZero + phase * step_x;
    int depth = (kSmemBytes - fixed) / (kWarps * S::kStepBytes);
    depth = depth < kMaxDepth ? depth : kMaxDepth;
    const bool mma = a.w.scale_layout == RFQ_SCALE_MMA;
    const Params p = {static_cast<const __nv_bfloat16 *>(a.x), a.x_row, a.M, (int)N, (int)K,
                      static_cast<const uint8_t *>(a.w.scales), mma, mma || K % 128 == 0, a.y, a.bf16,
                      (int)tiles, steps, phase, depth,
#ifdef RFQ_DEBUG_BOUNDS
                      getenv("RFQ_DEBUG_HOLD_US") ? atoi(getenv("RFQ_DEBUG_HOLD_US")) : 0
#endif
    };
    CUtensorMap map;
    if (!encode_tmap_2d_u8(&map, a.w.codes, (uint64_t)K / 2, (uint64_t)N, (uint64_t)K / 2, kBoxK / 2, kTile, 128))
        return cudaErrorInvalidValue;
    return launch_early(matvec_kernel<FMT, MP>, dim3(split, (unsigned)groups), kThreads,
                        (size_t)fixed + depth * kWarps * S::kStepBytes, st, split, map, p);
}

template <int FMT>
cudaError_t launch_rows(const MatvecArgs &a, cudaStream_t st)
{
    return a.M == 1   ? launch<FMT, 1>(a, st)
           : a.M == 2 ? launch<FMT, 2>(a, st)
           : a.M <= 4 ? launch<FMT, 4>(a, st)
           : a.M <= 8 ? launch<FMT, 8>(a, st)
           : a.M <= 16 ? launch<FMT, 16>(a, st)
                       : launch<FMT, 32>(a, st);
}

} // namespace

cudaError_t launch_matvec(const MatvecArgs &a, cudaStream_t st)
{
    return a.w.fmt == RFQ_FMT_HIF4 ? launch_rows<RFQ_FMT_HIF4>(a, st) : launch_rows<RFQ_FMT_MXFP4>(a, st);
}

} // namespace rfq
