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
// window of K (its maximum lands in [2^14, 2^15)): bf16 values down to 2^-28
// of the maximum are exact, the rest are off by less than 2^-39 of it.
//
// A CTA takes 64 rows of W~ and one share of K (a cluster of up to eight CTAs
// splits K and adds its parts in shared memory, in the order of the ranks, so
// a call gives the same bits every time).  W~ arrives in boxes of 64 rows x
// 256 codes by TMA with the 128-byte swizzle; ldmatrix then hands every lane
// its 8 codes of a 32-code block without a bank conflict.  Eight warps: four
// row tiles of 16, two halves of the window's boxes.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <cstdint>

#include "internal.h"
#include "kv_layout.cuh"
#include "ptx.cuh"

namespace rfq {
namespace {

constexpr int kWarps = 8, kThreads = 32 * kWarps;
constexpr int kRows = 64;                    // rows of W~ per CTA
constexpr int kBoxK = 256;                   // codes per row of a box (128 bytes)
constexpr int kBoxBytes = kRows * kBoxK / 2;

// NT: tiles of 8 rows of x.  Boxes per window: the x of a window is
// 8 NT boxes 512 bytes.
template <int NT>
struct Shape {
    static constexpr int kBoxes = NT >= 4 ? 2 : 4;
    static constexpr int kWinK = kBoxes * kBoxK;
    static constexpr int kXBytes = 8 * NT * kWinK * 2;
    static constexpr int kScaleWords = kRows * kWinK / 64;   // HiF4 (MXFP4: half)
    static constexpr int kStage = kBoxes * kBoxBytes;
    // two windows of W~, one of x and of scales
    static constexpr int kSmem = 1024 + 2 * kStage + kXBytes + kScaleWords * 4;
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
    int64_t N, K;
    const uint8_t *scales;
    int mma_layout;
    void *y;
    int bf16;
    int win_per_cta;       // windows of K per cluster rank
};

// Scale word of row n and the 128 (MXFP4) or 64 (HiF4) codes at k.
template <int FMT>
__device__ __forceinline__ uint32_t scale_word(const Params &p, int64_t n, int64_t k)
{
    if (n >= p.N || k >= p.K)
        return 0;
    if (FMT == RFQ_FMT_HIF4) {
        const int64_t at = p.mma_layout ? (k / 64) * ((p.N + 127) / 128 * 128) + n : n * (p.K / 64) + k / 64;
        return __ldg(reinterpret_cast<const uint32_t *>(p.scales) + at);
    }
    if (p.mma_layout)
        return __ldg(reinterpret_cast<const uint32_t *>(p.scales + sf_mma_offset(n, k / 32, p.K / 128)));
    uint32_t w = 0;
    const uint8_t *const s = p.scales + n * (p.K / 32) + k / 32;
    if (p.K % 128 == 0)
        return __ldg(reinterpret_cast<const uint32_t *>(s));
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (k + 32 * j < p.K)
            w |= (uint32_t)__ldg(s + j) << (8 * j);
    return w;
}

// Eight elements of an x row at k as fp32 (zero past its end).
__device__ __forceinline__ void load_x8(const Params &p, int m, int64_t k, float (&f)[8])
{
    uint32_t w[4] = {0, 0, 0, 0};
    if (m < p.M && k < p.K) {
        const __nv_bfloat16 *const s = p.x + m * p.x_row + k;
        const uint4 u = __ldg(reinterpret_cast<const uint4 *>(s));
        w[0] = u.x, w[1] = u.y, w[2] = u.z, w[3] = u.w;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi)
{
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}

template <int FMT, int NT>
__global__ void __launch_bounds__(kThreads) matvec_kernel(const __grid_constant__ CUtensorMap wmap, const Params p)
{
    using S = Shape<NT>;
    constexpr bool HIF4 = FMT == RFQ_FMT_HIF4;
    constexpr int WINK = S::kWinK;
    extern __shared__ uint8_t smem_raw[];
    __shared__ alignas(8) uint64_t s_full[2];
    __shared__ float s_xscale[8 * NT];
    uint8_t *const smem = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
    uint8_t *const s_w = smem;                                 // [2][boxes][64 rows][128 bytes]
    uint8_t *const s_x = s_w + 2 * S::kStage;                  // [block][tile][lane][16 bytes]
    uint32_t *const s_sc = reinterpret_cast<uint32_t *>(s_x + S::kXBytes);

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, c = lane & 3;
    const int split = (int)gridDim.x, rank = blockIdx.x;       // the cluster spans x
    const int64_t n0 = (int64_t)blockIdx.y * kRows;
    const int windows = (int)((p.K + WINK - 1) / WINK);
    const int w0 = min(windows, rank * p.win_per_cta), w1 = min(windows, w0 + p.win_per_cta);

    if (tid == 0) {
        mbar_init(&s_full[0], 1);
        mbar_init(&s_full[1], 1);
        fence_mbar_init();
    }
    __syncthreads();
    auto fetch = [&](int w) {                                  // one thread
        const int b = (w - w0) & 1;
        mbar_arrive_expect_tx(&s_full[b], S::kStage);
#pragma unroll
        for (int i = 0; i < S::kBoxes; ++i)
            tma_load_2d(s_w + b * S::kStage + i * kBoxBytes, &wmap, &s_full[b], (w * WINK + i * kBoxK) / 2, (int)n0);
    };
    if (tid == 0) {
        if (w0 < w1)
            fetch(w0);
        if (w0 + 1 < w1)
            fetch(w0 + 1);
    }

    const int rt = warp & 3, half = warp >> 2;                 // rows 16 rt .., every second box
    float acc[NT][4];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            acc[t][i] = 0.f;
    bool ok = true;                                            // no wait has run out

    for (int w = w0; w < w1; ++w) {
        const int64_t k0 = (int64_t)w * WINK;
        const int b = (w - w0) & 1;
        // scales of the window: [k word][row]
        constexpr int KW = WINK / (HIF4 ? 64 : 128);
        for (int i = tid; i < KW * kRows; i += kThreads)
            s_sc[i] = scale_word<FMT>(p, n0 + i % kRows, k0 + (int64_t)(i / kRows) * (HIF4 ? 64 : 128));
        // x of the window as f16, each row scaled by a power of two: one warp a row
        for (int m = warp; m < 8 * NT; m += kWarps) {
            float f[WINK / 256][8];
            float mx = 0.f;
#pragma unroll
            for (int i = 0; i < WINK / 256; ++i) {
                load_x8(p, m, k0 + i * 256 + lane * 8, f[i]);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    mx = fmaxf(mx, fabsf(f[i][j]));
            }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1)
                mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, o));
            const int e = (int)(__float_as_uint(mx) >> 23) - 127 - 14;   // x 2^-e: the maximum in [2^14, 2^15)
            const int ec = max(min(e, 126), -126);
            const float mul = __uint_as_float((uint32_t)(127 - ec) << 23);
            if (lane == 0)
                s_xscale[m] = __uint_as_float((uint32_t)(127 + ec) << 23);
#pragma unroll
            for (int i = 0; i < WINK / 256; ++i) {
                uint32_t h[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    // HiF4 codes decode in the order 0 2 | 1 3 | 4 6 | 5 7
                    const int lo = HIF4 ? (j >> 1) * 4 + (j & 1) : 2 * j, hi = HIF4 ? lo + 2 : lo + 1;
                    h[j] = pack_f16(f[i][lo] * mul, f[i][hi] * mul);
                }
                const int blk = i * 8 + (lane >> 2), cc = lane & 3;
                *reinterpret_cast<uint4 *>(s_x + (((blk * NT + (m >> 3)) * 32 + (m & 7) * 4 + cc) << 4)) =
                    make_uint4(h[0], h[1], h[2], h[3]);
            }
        }
        __syncthreads();
        ok = ok && mbar_wait(&s_full[b], ((w - w0) >> 1) & 1, kWaitLimitNs);
        if (!ok)                                               // (once more before its copies' memory may go)
            mbar_wait(&s_full[b], ((w - w0) >> 1) & 1, kWaitLimitNs);
        if (ok) {
            float win[NT][4];
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    win[t][i] = 0.f;
#pragma unroll 1
            for (int box = half; box < S::kBoxes; box += 2) {
                const uint32_t base = smem_u32(s_w) + b * S::kStage + box * kBoxBytes;
                // ldmatrix: matrix lane / 8 = (8 rows (lane / 8) % 2, block parity lane / 16)
                const int row = rt * 16 + ((lane >> 3) & 1) * 8 + (lane & 7);
#pragma unroll
                for (int pair = 0; pair < 4; ++pair) {         // two 32-code blocks
                    const int chunk = pair * 2 + (lane >> 4);  // 16 bytes
                    uint32_t a[4];
                    ldmatrix_x4(base + row * 128 + ((chunk ^ (row & 7)) << 4), a);
                    float tmp[NT][4];
                    if (HIF4) {
#pragma unroll
                        for (int t = 0; t < NT; ++t)
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                tmp[t][i] = 0.f;
                    }
                    const int kw = HIF4 ? box * 4 + pair : box * 2 + (pair >> 1);
                    const uint32_t sw0 = s_sc[kw * kRows + rt * 16 + g], sw1 = s_sc[kw * kRows + rt * 16 + g + 8];
#pragma unroll
                    for (int s = 0; s < 2; ++s) {
                        uint32_t h0[4], h1[4];                 // rows g and g + 8
                        if (HIF4) {
                            s1p2x8_f16(a[2 * s], h0);
                            s1p2x8_f16(a[2 * s + 1], h1);
                            uint32_t t0, t1;
                            hif4_pow2_pair(sw0, 4 * s + c, t0, t1);
                            h0[0] = hmul2(h0[0], t0), h0[1] = hmul2(h0[1], t0);
                            h0[2] = hmul2(h0[2], t1), h0[3] = hmul2(h0[3], t1);
                            hif4_pow2_pair(sw1, 4 * s + c, t0, t1);
                            h1[0] = hmul2(h1[0], t0), h1[1] = hmul2(h1[1], t0);
                            h1[2] = hmul2(h1[2], t1), h1[3] = hmul2(h1[3], t1);
                        } else {
                            e2m1x8_f16(a[2 * s], h0);
                            e2m1x8_f16(a[2 * s + 1], h1);
#pragma unroll
                            for (int t = 0; t < NT; ++t)
#pragma unroll
                                for (int i = 0; i < 4; ++i)
                                    tmp[t][i] = 0.f;
                        }
                        const int blk = box * 8 + pair * 2 + s;
#pragma unroll
                        for (int t = 0; t < NT; ++t) {
                            const uint4 xb =
                                *reinterpret_cast<const uint4 *>(s_x + (((blk * NT + t) * 32 + lane) << 4));
                            mma_f16(tmp[t], h0[0], h1[0], h0[1], h1[1], xb.x, xb.y);
                            mma_f16(tmp[t], h0[2], h1[2], h0[3], h1[3], xb.z, xb.w);
                        }
                        if (!HIF4) {
                            const int sh = ((pair & 1) * 2 + s) * 8;
                            const float f0 = e8m0_f32((sw0 >> sh) & 0xFFu), f1 = e8m0_f32((sw1 >> sh) & 0xFFu);
#pragma unroll
                            for (int t = 0; t < NT; ++t) {
                                win[t][0] = fmaf(tmp[t][0], f0, win[t][0]);
                                win[t][1] = fmaf(tmp[t][1], f0, win[t][1]);
                                win[t][2] = fmaf(tmp[t][2], f1, win[t][2]);
                                win[t][3] = fmaf(tmp[t][3], f1, win[t][3]);
                            }
                        }
                    }
                    if (HIF4) {
                        const float f0 = hif4_macro_f32(sw0), f1 = hif4_macro_f32(sw1);
#pragma unroll
                        for (int t = 0; t < NT; ++t) {
                            win[t][0] = fmaf(tmp[t][0], f0, win[t][0]);
                            win[t][1] = fmaf(tmp[t][1], f0, win[t][1]);
                            win[t][2] = fmaf(tmp[t][2], f1, win[t][2]);
                            win[t][3] = fmaf(tmp[t][3], f1, win[t][3]);
                        }
                    }
                }
            }
            // HiF4: a code's 2^-9 and the 1/4 of its step
            constexpr float kUnit = HIF4 ? 128.f : 1.f;
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const float u0 = s_xscale[8 * t + 2 * c] * kUnit, u1 = s_xscale[8 * t + 2 * c + 1] * kUnit;
                acc[t][0] = fmaf(win[t][0], u0, acc[t][0]);
                acc[t][1] = fmaf(win[t][1], u1, acc[t][1]);
                acc[t][2] = fmaf(win[t][2], u0, acc[t][2]);
                acc[t][3] = fmaf(win[t][3], u1, acc[t][3]);
            }
        }
        __syncthreads();
        if (tid == 0 && w + 2 < w1)
            fetch(w + 2);
    }

    if (!ok)
#pragma unroll
        for (int t = 0; t < NT; ++t)
            acc[t][0] = acc[t][1] = acc[t][2] = acc[t][3] = __int_as_float(0x7FFFFFFF);
    // the CTA's part: [half][x row][row of W~], over the codes' shared memory
    float *const s_part = reinterpret_cast<float *>(smem);
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            s_part[(half * 8 * NT + 8 * t + 2 * c + (i & 1)) * kRows + rt * 16 + g + (i >> 1) * 8] = acc[t][i];
    cluster_sync();
    // each rank finishes its share of the elements, all ranks' parts added in order
    const int elems = p.M * kRows;
    const uint32_t part = smem_u32(s_part);
    for (int i = rank * kThreads + tid; i < elems; i += split * kThreads) {
        const int m = i / kRows, r = i % kRows;
        float sum = 0.f;
        for (int q = 0; q < split; ++q)
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
                float v;
                asm volatile("ld.shared::cluster.f32 %0, [%1];"
                             : "=f"(v)
                             : "r"(mapa_shared(part + ((hf * 8 * NT + m) * kRows + r) * 4, q)));
                sum += v;
            }
        if (n0 + r < p.N) {
            const int64_t o = (int64_t)m * p.N + n0 + r;
            if (p.bf16)
                static_cast<__nv_bfloat16 *>(p.y)[o] = __float2bfloat16_rn(sum);
            else
                static_cast<float *>(p.y)[o] = sum;
        }
    }
    cluster_sync();
}

template <int FMT, int NT>
cudaError_t launch(const MatvecArgs &a, cudaStream_t st)
{
    using S = Shape<NT>;
    const int64_t N = a.w.rows, K = a.w.k;
    const int windows = (int)((K + S::kWinK - 1) / S::kWinK);
    const int64_t tiles = (N + kRows - 1) / kRows;
    // split K until every SM has a few CTAs
    int split = 1;
    while (split < 8 && split * 2 <= windows && tiles * split < 4 * (int64_t)num_sms())
        split *= 2;
    Params p = {static_cast<const __nv_bfloat16 *>(a.x), a.x_row, a.M, N, K, static_cast<const uint8_t *>(a.w.scales),
                a.w.scale_layout == RFQ_SCALE_MMA, a.y, a.bf16, (windows + split - 1) / split};
    CUtensorMap map;
    if (!encode_tmap_2d_u8(&map, a.w.codes, (uint64_t)K / 2, (uint64_t)N, (uint64_t)K / 2, kBoxK / 2, kRows, 128))
        return cudaErrorInvalidValue;
    static bool ready = false;     // (per instantiation; setting it twice is harmless)
    if (!ready) {
        if (cudaError_t e = cudaFuncSetAttribute(matvec_kernel<FMT, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                 S::kSmem))
            return e;
        ready = true;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(split, (unsigned)tiles);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = S::kSmem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim = {(unsigned)split, 1, 1};
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, matvec_kernel<FMT, NT>, map, p);
}

template <int FMT>
cudaError_t launch_rows(const MatvecArgs &a, cudaStream_t st)
{
    return a.M <= 8 ? launch<FMT, 1>(a, st) : a.M <= 16 ? launch<FMT, 2>(a, st) : launch<FMT, 4>(a, st);
}

} // namespace

cudaError_t launch_matvec(const MatvecArgs &a, cudaStream_t st)
{
    return a.w.fmt == RFQ_FMT_HIF4 ? launch_rows<RFQ_FMT_HIF4>(a, st) : launch_rows<RFQ_FMT_MXFP4>(a, st);
}

} // namespace rfq
