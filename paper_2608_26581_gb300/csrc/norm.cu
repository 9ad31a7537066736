// norm.cu -- layer norm and RMS norm of rows (rfq_norm) and their gradients
// (rfq_norm_grad).
//
// Forward:   m = mean x (RMS: 0),  r = 1 / sqrt(mean (x - m)^2 + eps),
//            y = (x - m) r w + b.
// Backward:  g = dy w,  h = (x - m) r,
//            dx = r (g - mean g - h mean(g h))   (RMS: without mean g),
//            dw = sum over rows of dy h,  db = sum over rows of dy.
//
// Bound: HBM (x read and y written once; dy and x read and dx written once).
// Persistent blocks take rows in turn.  The threads that share a row hold it
// in registers, so the mean and the squared distances from it are two passes
// over registers.  Rows that come next are on their way to shared memory: a
// thread copies (cp.async) and reads its own 16-byte chunks alone, so the ring
// needs no barrier.  Where strides and sizes allow no more, chunks are words, and
// the next row's are loaded into registers (a row of bf16 that starts in the
// middle of a word takes two words for each chunk, and joins them).  A thread's
// chunks lie a fixed distance apart, which leaves one address a row; arithmetic
// is on pairs of fp32 values.  The weight's gradient is summed in fp32 in
// registers by threads that keep their columns over all their rows; the blocks'
// sums go through the workspace and a second kernel adds them, both in a fixed
// order.
//
// 32760 rows of 5120 bf16: forward 112 us, 6.0 TB/s, 89% of the copy rate;
// backward 166 us with both sums, 89% (148 us without weights and sums: the
// partial sums of 304 blocks, 12 MB there and back, and their kernel take 8 of
// the 18, the weights' loads the rest).  Issue slots are 65% busy at that.
// At 16384 rows: 32 heads of 128 bf16 forward 83%, backward 92% (fp32 89 and
// 98%); 4096 elements bf16 80 and 81% (fp32 83 and 89%).
// Slower are, at floors of 59.5 us (2^26 elements of bf16, 2^25 of fp32), rows
// beyond 5120 elements backwards: bf16 8192 77%, 9216 70%, 13824 61%, fp32 8192
// 92%, 9216 88%, 13824 69%: one block on an SM, beyond 8192 the row is read from
// shared memory twice.  And backwards, calls as large as a prompt: the partial
// sums are 7 to 12 MB whatever the rows, their kernel has a block for 64 columns,
// and both sums are kept where one is asked for.  RMS with a weight, bf16: 4096
// rows of 2048 17.3 us of 7.4, 8192 of 1024 18.7 of 7.5, 1531 of 4096 15.5 of 5.6,
// 2000 of 5120 20.0 of 9.1; 700 of 5120 fp32 17.5 of 6.4; 4096 of 32 heads of 128
// 22.0 of 15.0.  (Forward, 4096 of 2048: 5.7 of 5.0; one to 32 rows: 2.3, latency.)
// Rows of words are bound by instructions: 65536 rows of 1023 fp32 78% forward
// and 89% backward, bf16 38 and 41%, 54123 of 620 bf16 37 and 33%; 16384 rows of
// 1023 fp32 72 and 73%, bf16 35 and 36% (words by cp.async took longer, 45 us
// instead of 29 for the first of these).
// The narrow backward kernels of blocks of 1024 threads (64 registers) spill 56 to
// 192 bytes, and the forward one of 16-byte bf16 rows that take a block 8.
// (Measured and not kept: tiles of several rows gone through twice, first by
// rows, then by columns, 188 us backwards; weights in shared memory, 197; the
// next row asked for after this one's sums, 184 to 220; weights loaded ahead of
// the row or held, 183; for fewer partial sums, one block of 640 threads on an SM
// that several rows share, 258, and clusters that add theirs first, 184.)
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <cstdint>

#include "internal.h"
#include "ptx.cuh"
#include "rows.cuh"

namespace rfq {
namespace {

constexpr int kThreads = 256;                // of a block whose rows take a warp or less
constexpr size_t kMostSmem = 200 * 1024;     // of an SM's blocks together
constexpr size_t kPlainSmem = 47 * 1024;     // dynamic, beside the kernels' own (512 bytes at most), without asking

struct Pair {
    float x, y;
};
__device__ __forceinline__ Pair operator+(const Pair &a, const Pair &b) { return {a.x + b.x, a.y + b.y}; }
__device__ __forceinline__ float shfl_xor(float v, int d) { return __shfl_xor_sync(0xFFFFFFFFu, v, d); }
__device__ __forceinline__ Pair shfl_xor(const Pair &v, int d) { return {shfl_xor(v.x, d), shfl_xor(v.y, d)}; }

// How a row lies over threads: TPR of them share it, NV chunks of VEC elements
// each, TPR chunks apart; with TPR = 64 it takes all warps of the block, each
// of them 32 NV chunks that lie together.
template <typename T_, int VEC_, int NV_, int TPR_>
struct Split {
    using T = T_;
    static constexpr int VEC = VEC_, NV = NV_, TPR = TPR_;
    static constexpr int kChunk = VEC * (int)sizeof(T);               // bytes: 16, or 4
    static constexpr bool kNarrow = kChunk == 4, kHalves = kNarrow && VEC == 2;
    static constexpr bool kBlock = TPR > 32;
    static constexpr int kStep = kBlock ? 32 : TPR;                   // chunks between a thread's
    static constexpr int kLanesOf = kLanes<VEC>;
    using F = Lane<VEC>;
    int group, first;                                                 // row of the block's; this thread's first chunk
    __device__ __forceinline__ Split()
        : group(kBlock ? 0 : threadIdx.x / TPR),
          first(kBlock ? (threadIdx.x >> 5) * 32 * NV + (threadIdx.x & 31) : threadIdx.x % TPR)
    {
    }
    static __device__ __forceinline__ int groups() { return kBlock ? 1 : blockDim.x / TPR; }
    __device__ __forceinline__ bool leads() const { return first == 0; }
    // chunk i of this thread is one of the row's
    __device__ __forceinline__ bool has(int i, int chunks) const { return first + i * kStep < chunks; }

    // Sum over the row's threads.  A block's go through `part` (32 values, zero
    // where it has no warp); two sums in a row take different ones, which makes
    // one barrier a sum enough: who writes has passed the barrier behind the
    // last use.
    template <typename V>
    __device__ __forceinline__ V sum(V v, V *part) const
    {
#pragma unroll
        for (int d = kStep / 2; d > 0; d >>= 1)
            v = v + shfl_xor(v, d);
        if constexpr (kBlock) {
            if ((threadIdx.x & 31) == 0)
                part[threadIdx.x >> 5] = v;
            __syncthreads();
            v = part[0];
            const int n = blockDim.x >> 5;
#pragma unroll
            for (int i = 1; i < 4; ++i)
                v = v + part[i];
#pragma unroll 1
            for (int i = 4; i < n; i += 4)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    v = v + part[i + j];
        }
        return v;
    }
};

// Rows in steps, as (token, head): rows lie [tokens][heads] with two strides in
// elements.  (A division for each row costs as much as its 8 elements.)
struct Walk {
    uint32_t token, head, tokens_on, heads_on, heads;
    __device__ __forceinline__ Walk(uint32_t row, uint32_t step, uint32_t h)
        : token(row / h), head(row - token * h), tokens_on(step / h), heads_on(step - tokens_on * h), heads(h)
    {
    }
    __device__ __forceinline__ void next()
    {
        token += tokens_on;
        head += heads_on;
        if (head >= heads) {
            head -= heads;
            ++token;
        }
    }
    template <typename T>
    __device__ __forceinline__ T *at(T *p, int64_t token_stride, int64_t head_stride) const
    {
        return p + token * token_stride + head * head_stride;
    }
};

// The same without a state, for rows of a whole block.
struct Place {
    uint32_t row, step, heads;
    __device__ __forceinline__ Place(uint32_t r, uint32_t s, uint32_t h) : row(r), step(s), heads(h) {}
    __device__ __forceinline__ void next() { row += step; }
    template <typename T>
    __device__ __forceinline__ T *at(T *p, int64_t token_stride, int64_t head_stride) const
    {
        if (heads == 1)
            return p + row * token_stride;
        const uint32_t t = row / heads;
        return p + t * token_stride + (row - t * heads) * head_stride;
    }
};

// The end of an array of rows (for chunks that are words of two elements).
template <typename P, typename T>
__device__ __forceinline__ const T *array_end(const T *p, int64_t token_stride, int64_t head_stride, uint32_t rows, uint32_t heads, int dim)
{
    return P::kHalves ? p + (int64_t)(rows / heads - 1) * token_stride + (int64_t)(heads - 1) * head_stride + dim : nullptr;
}

__device__ __forceinline__ F2 first_only(F2 v)
{
    float a, b;
    f2unpack(v.v, a, b);
    return {f2pack(a, 0.f)};
}

template <typename P>
using Rows = std::conditional_t<P::kBlock, Place, Walk>;

// VEC parameters from column c on (of dim), in fp32.
template <int VEC>
__device__ __forceinline__ void load_params(const void *p, bool bf16, int c, int dim, Lane<VEC> *v)
{
    if (VEC == 2 && c + 1 == dim) {          // (the last of an odd number)
        const float one = bf16 ? to_f32(static_cast<const __nv_bfloat16 *>(p)[c]) : static_cast<const float *>(p)[c];
        if constexpr (VEC == 2)
            v[0] = {f2pack(one, 0.f)};
    } else if (bf16)
        unpack<__nv_bfloat16, VEC>(load_vec<__nv_bfloat16, VEC>(static_cast<const __nv_bfloat16 *>(p) + c), v);
    else {
        constexpr int F = VEC < 4 ? VEC : 4;
#pragma unroll
        for (int g = 0; g < VEC / F; ++g)
            unpack<float, F>(load_vec<float, F>(static_cast<const float *>(p) + c + g * F), v + g * kLanes<F>);
    }
}

__device__ __forceinline__ uint4 lds128(uint32_t at)
{
    uint4 u;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w) : "r"(at) : "memory");
    return u;
}

// Rows on their way, S deep, N arrays: 16-byte chunks copied ahead into shared memory.
template <typename P, int N, int S>
struct Ring {
    using T = typename P::T;
    uint32_t base, row;                      // shared address of this thread's chunks; bytes of a row of all threads
    __device__ __forceinline__ Ring(const void *smem)
        : base(smem_u32(smem) + ((threadIdx.x >> 5) * 32 * P::NV + (threadIdx.x & 31)) * 16), row(blockDim.x * P::NV * 16)
    {
    }
    static constexpr size_t bytes(int threads) { return (size_t)S * N * P::NV * 16 * threads; }
    __device__ __forceinline__ void copy(const P &p, int slot, int n, const T *x, bool there, int chunks) const
    {
        const uint32_t to = base + (slot * N + n) * row;
#pragma unroll
        for (int i = 0; i < P::NV; ++i)
            if (there && p.has(i, chunks))
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + i * 512), "l"(x + (p.first + i * P::kStep) * P::VEC) : "memory");
    }
    __device__ __forceinline__ void read(int slot, int n, int i, bool there, typename P::F *x) const
    {
        uint4 u = make_uint4(0, 0, 0, 0);
        if (there)
            u = lds128(base + (slot * N + n) * row + i * 512);
        unpack<T, P::VEC>(*reinterpret_cast<Vec<T, P::VEC> *>(&u), x);
    }
};

// A row that starts in the middle of a word (of bf16 elements).
__device__ __forceinline__ uint32_t half_off(const void *row) { return (uint32_t)reinterpret_cast<uintptr_t>(row) & 2u; }

// A thread's words of a row.
template <typename P>
struct Words {
    using T = typename P::T;
    uint32_t low[P::NV], high[P::kHalves ? P::NV : 1], off;
    // The word of bf16 elements at `from`, or its first half alone.
    static __device__ __forceinline__ uint32_t halves(const char *from, bool both)
    {
        return both ? *reinterpret_cast<const uint32_t *>(from) : (uint32_t)*reinterpret_cast<const uint16_t *>(from);
    }
    // x: the row; end: of its array (which a word that holds the last element may pass)
    __device__ __forceinline__ void load(const P &p, const T *x, const T *end, bool there, int chunks, int dim)
    {
        off = P::kHalves ? half_off(x) : 0;
        const int most = P::kHalves && x + dim == end ? dim : INT32_MAX;      // elements that may be read, from x on
        const char *const word = reinterpret_cast<const char *>(x + p.first * P::VEC) - off;
        const int e = p.first * 2 - (off ? 1 : 0);                             // the first word's first element
#pragma unroll
        for (int i = 0; i < P::NV; ++i) {
            low[i] = 0;
            if constexpr (P::kHalves)
                high[i] = 0;
            if (there && p.has(i, chunks)) {
                if constexpr (P::kHalves) {
                    low[i] = halves(word + i * P::kStep * 4, e + i * P::kStep * 2 + 1 < most);
                    if (off && 2 * (p.first + i * P::kStep) + 1 < dim)
                        high[i] = halves(word + i * P::kStep * 4 + 4, e + i * P::kStep * 2 + 3 < most);
                } else
                    low[i] = *reinterpret_cast<const uint32_t *>(word + i * P::kStep * 4);
            }
        }
    }
    __device__ __forceinline__ void get(const P &p, int i, int dim, typename P::F *v) const
    {
        uint32_t u = low[i];
        if constexpr (P::kHalves) {
            if (off)
                u = __funnelshift_r(u, high[i], 16);
            if (2 * (p.first + i * P::kStep) + 1 == dim)
                u &= 0xFFFFu;                // (zero behind the last of an odd number)
        }
        unpack<T, P::VEC>(*reinterpret_cast<Vec<T, P::VEC> *>(&u), v);
    }
};

__device__ __forceinline__ void ring_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void ring_wait() // until no more than N rows are on their way
{
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// Chunk i of a result's row.
template <typename P>
__device__ __forceinline__ void store_chunk(const P &p, typename P::T *row, int i, int dim, const typename P::F *v)
{
    const int c = (p.first + i * P::kStep) * P::VEC;
    const auto u = pack<typename P::T, P::VEC>(v);
    if constexpr (P::kHalves) {
        if (half_off(row) || c + 1 == dim) {
            row[c] = u.v[0];
            if (c + 1 < dim)
                row[c + 1] = u.v[1];
            return;
        }
    }
    store_once<typename P::T, P::VEC>(row + c, u);
}

// Narrow rows of up to so many elements go with 8 elements a thread, longer ones with 16.
constexpr int kFewForward = 4096, kFewBackward = 8192;

// The most threads of a forward block.
template <typename P>
constexpr int kMostThreads = P::kBlock ? (P::NV * P::VEC == 8 ? kFewForward : kNormDim) / (P::NV * P::VEC) : kThreads;

// Rows of the forward ring.  (Deeper ones take L1 from the weights: with three
// rows of 5120 elements a layer norm of 32760 takes 116 us, with two 112.)
template <typename P>
constexpr int kForwardRows = P::kNarrow ? 0 : P::NV == 2 ? 4 : 2;

template <typename P>
__global__ void __launch_bounds__(kMostThreads<P>, P::kBlock ? (kMostThreads<P> <= 512 ? 2 : 1) : 4) norm_kernel(const NormArgs a)
{
    using T = typename P::T;
    using F = typename P::F;
    constexpr int S = kForwardRows<P>, NV = P::NV, L = P::kLanesOf;
    extern __shared__ __align__(16) uint8_t s_ring[];
    __shared__ float s_part[2][32];
    const P p;
    const Ring<P, 1, S> ring(s_ring);
    const int chunks = (a.dim + P::VEC - 1) / P::VEC;
    const uint32_t rows = (uint32_t)a.rows, step = gridDim.x * p.groups();
    const float inv = 1.f / (float)a.dim;
    uint32_t first = blockIdx.x * p.groups();
    Rows<P> here(first + p.group, step, a.heads), next = here;        // this turn's row; the one that is copied next
    const T *const x = static_cast<const T *>(a.x), *const x_end = array_end<P>(x, a.x_token, a.x_head, rows, a.heads, a.dim);
    Words<P> words;                          // of the next row
    auto ahead = [&](int slot, uint32_t r) {
        if constexpr (P::kNarrow)
            words.load(p, next.at(x, a.x_token, a.x_head), x_end, r < rows, chunks, a.dim);
        else {
            ring.copy(p, slot, 0, next.at(x, a.x_token, a.x_head), r < rows, chunks);
            ring_commit();
        }
        next.next();
    };
    if (P::kBlock && threadIdx.x < 32)
        s_part[0][threadIdx.x] = s_part[1][threadIdx.x] = 0.f;
    wait_for_previous();
    let_next_start();
#pragma unroll 1
    for (int s = 0; s < (P::kNarrow ? 1 : S - 1); ++s)
        ahead(s, first + p.group + s * step);
    if (P::kBlock)
        __syncthreads();
    // (few lanes a row: many rows for the same few weights)
    constexpr bool HELD = P::kNarrow ? NV * P::VEC <= 8 : !P::kBlock && NV == 2;
    F held[HELD ? NV : 1][L];
    if (HELD && a.weight)
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (p.has(i, chunks))
                load_params<P::VEC>(a.weight, a.w_bf16, (p.first + i * P::kStep) * P::VEC, a.dim, held[HELD ? i : 0]);
    int slot = 0, turn = 0;
    // (every thread of the block takes part in the sums of every turn)
#pragma unroll 1
    for (; first < rows; first += step, turn ^= 1, here.next()) {
        const uint32_t row = first + p.group;
        const bool there = P::kBlock || row < rows;
        F d[NV][L];
        if constexpr (P::kNarrow) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
                words.get(p, i, a.dim, d[i]);
            ahead(0, row + step);
        } else {
            ring_wait<S - 2>();
#pragma unroll
            for (int i = 0; i < NV; ++i)
                ring.read(slot, 0, i, there && p.has(i, chunks), d[i]);
            ahead(slot == 0 ? S - 1 : slot - 1, row + (S - 1) * step);
            slot = slot == S - 1 ? 0 : slot + 1;
        }
        float mean = 0.f;
        if (!a.rms) {
            F s = all_of<P::VEC>(0.f);
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int e = 0; e < L; ++e)
                    s = s + d[i][e];
            mean = p.sum(both(s), s_part[0]) * inv;
        }
        const F less = all_of<P::VEC>(-mean);
        F q = all_of<P::VEC>(0.f);
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (p.has(i, chunks))
#pragma unroll
                for (int e = 0; e < L; ++e) {
                    d[i][e] = d[i][e] + less;
                    if constexpr (P::kHalves)
                        if (2 * (p.first + i * P::kStep) + 1 == a.dim)
                            d[i][e] = first_only(d[i][e]);
                    q = fused(d[i][e], d[i][e], q);
                }
        // (two sums a turn, or with RMS one; rsqrtf is off by two steps of fp32 at most)
        const float rstd = rsqrtf(p.sum(both(q), s_part[a.rms ? turn : 1]) * inv + a.eps);
        if (!there)
            continue;
        if (p.leads()) {
            if (a.mean)
                a.mean[row] = mean;
            if (a.rstd)
                a.rstd[row] = rstd;
        }
        const F scale = all_of<P::VEC>(rstd);
        T *const y = here.at(static_cast<T *>(a.y), a.y_token, a.y_head);
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (p.has(i, chunks)) {
                const int c = (p.first + i * P::kStep) * P::VEC;
                F f[L];
#pragma unroll
                for (int e = 0; e < L; ++e)
                    d[i][e] = d[i][e] * scale;
                if (a.weight) {
                    if (!HELD)
                        load_params<P::VEC>(a.weight, a.w_bf16, c, a.dim, f);
#pragma unroll
                    for (int e = 0; e < L; ++e)
                        d[i][e] = d[i][e] * (HELD ? held[HELD ? i : 0][e] : f[e]);
                }
                if (a.bias) {
                    load_params<P::VEC>(a.bias, a.w_bf16, c, a.dim, f);
#pragma unroll
                    for (int e = 0; e < L; ++e)
                        d[i][e] = d[i][e] + f[e];
                }
                store_chunk(p, y, i, a.dim, d[i]);
            }
    }
}

// Whether a row is read from the ring a second time for dx instead of staying
// in registers (24 elements a thread or more; 9216 bf16 in registers: 96 us
// instead of 85, 8192 bf16, which stays there, from the ring: 90 instead of 77).
template <typename P>
constexpr bool kTwice = P::NV * P::VEC > 16;

// The backward kernel for blocks of up to THREADS threads: blocks on an SM and
// rows of its ring (of two arrays).
template <typename P, int THREADS>
struct Backward {
    static constexpr int kBlocks = THREADS <= 320 ? 2 : 1;
    static constexpr bool kAhead = P::kNarrow && P::NV * P::VEC <= 8;    // the next row's words in registers
    static constexpr size_t kRow = (size_t)P::NV * 2 * 16;    // bytes of a thread
    // (three rows of a block's: 189 us instead of 166)
    static constexpr int rows()
    {
        const size_t n = kMostSmem / kBlocks / THREADS / kRow, most = P::kBlock ? 2 : 3;
        return P::kNarrow ? 0 : (int)(n < most ? n : most);
    }
    static constexpr int kRows = rows();
    static_assert(P::kNarrow || kRows >= (kTwice<P> ? 1 : 2), "a row on its way beside one that has been read");
    static constexpr size_t bytes(int threads) { return kRows * kRow * threads; }
};

template <int VEC>
__device__ __forceinline__ void store_sums(float *to, const Lane<VEC> *v)
{
    if constexpr (VEC <= 2)
        *reinterpret_cast<Lane<VEC> *>(to) = v[0];
    else
#pragma unroll
        for (int e = 0; e < kLanes<VEC>; e += 2)
            *reinterpret_cast<ulonglong2 *>(to + 2 * e) = {v[e].v, v[e + 1].v};
}

// Columns of a part in the workspace: whole 16-byte words.
__host__ __device__ __forceinline__ int padded_dim(int dim) { return (dim + 3) / 4 * 4; }

// Blocks take rows in turn; a thread keeps its columns.  Partial sums of the
// weight's gradient: a.partial [blocks][2][padded dim].
template <typename P, int THREADS>
__global__ void __launch_bounds__(THREADS, Backward<P, THREADS>::kBlocks) norm_grad_kernel(const NormGradArgs a)
{
    using T = typename P::T;
    using F = typename P::F;
    using B = Backward<P, THREADS>;
    constexpr int S = B::kRows, NV = P::NV, L = P::kLanesOf, VEC = P::VEC;
    constexpr bool TWICE = kTwice<P>;
    extern __shared__ __align__(16) uint8_t smem[];      // ring; after the last row: [groups][2][padded dim] sums where a block has several groups
    __shared__ Pair s_part[2][32];
    const P p;
    const Ring<P, 2, S> ring(smem);
    const int chunks = (a.dim + VEC - 1) / VEC, groups = p.groups();
    const uint32_t rows = (uint32_t)a.rows, step = gridDim.x * groups;
    const float inv = 1.f / (float)a.dim;
    uint32_t first = blockIdx.x * groups;
    Rows<P> here(first + p.group, step, a.heads), next = here;        // this turn's row; the one that is copied next
    const T *const x = static_cast<const T *>(a.x), *const x_end = array_end<P>(x, a.x_token, a.x_head, rows, a.heads, a.dim);
    const T *const dy = static_cast<const T *>(a.dy), *const dy_end = array_end<P>(dy, a.dy_token, a.dy_head, rows, a.heads, a.dim);
    Words<P> words_x, words_dy;              // of the next row
    auto ahead = [&](int slot, uint32_t r) {
        if constexpr (P::kNarrow) {
            words_x.load(p, next.at(x, a.x_token, a.x_head), x_end, r < rows, chunks, a.dim);
            words_dy.load(p, next.at(dy, a.dy_token, a.dy_head), dy_end, r < rows, chunks, a.dim);
        } else {
            ring.copy(p, slot, 0, next.at(x, a.x_token, a.x_head), r < rows, chunks);
            ring.copy(p, slot, 1, next.at(dy, a.dy_token, a.dy_head), r < rows, chunks);
            ring_commit();
        }
        next.next();
    };
    if (P::kBlock && threadIdx.x < 32)
        s_part[0][threadIdx.x] = s_part[1][threadIdx.x] = {0.f, 0.f};
    wait_for_previous();
    let_next_start();
#pragma unroll 1
    for (int s = 0; s < (P::kNarrow ? B::kAhead : TWICE ? S : S - 1); ++s)
        ahead(s, first + p.group + s * step);
    F dw[NV][L], db[NV][L];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
#pragma unroll
        for (int e = 0; e < L; ++e)
            dw[i][e] = db[i][e] = all_of<VEC>(0.f);
    }
    F held[B::kAhead ? NV : 1][L];           // weights, where there is room for them
    if (B::kAhead && a.weight)
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (p.has(i, chunks))
                load_params<VEC>(a.weight, a.w_bf16, (p.first + i * P::kStep) * VEC, a.dim, held[B::kAhead ? i : 0]);
    // (a row's statistics are loaded one row ahead)
    float next_rstd = 0.f, next_mean = 0.f;
    auto stats = [&](uint32_t r) {
        if (r < rows) {
            next_rstd = a.rstd[r];
            next_mean = a.rms ? 0.f : a.mean[r];
        }
    };
    stats(first + p.group);
    if (P::kBlock)
        __syncthreads();
    int slot = 0, turn = 0;
    // (every thread of the block takes part in the sums of every turn)
#pragma unroll 1
    for (; first < rows; first += step, turn ^= 1, here.next()) {
        const uint32_t row = first + p.group;
        const bool there = P::kBlock || row < rows;
        const F less = all_of<VEC>(-next_mean);
        const float rstd = next_rstd;
        const F scale = all_of<VEC>(rstd);
        stats(row + step);
        constexpr int KEPT = TWICE ? 1 : NV;
        F h[KEPT][L], g[KEPT][L];
        auto fetch = [&](int i) {
            const int k = TWICE ? 0 : i;
            const bool in = there && p.has(i, chunks);
            if constexpr (P::kNarrow) {
                words_x.get(p, i, a.dim, h[k]);
                words_dy.get(p, i, a.dim, g[k]);
            } else {
                ring.read(slot, 0, i, in, h[k]);
                ring.read(slot, 1, i, in, g[k]);
            }
        };
        auto weighted = [&](int i) {
            if (a.weight) {
                F w[L];
                if (B::kAhead) {
#pragma unroll
                    for (int e = 0; e < L; ++e)
                        w[e] = held[B::kAhead ? i : 0][e];
                } else
                    load_params<VEC>(a.weight, a.w_bf16, (p.first + i * P::kStep) * VEC, a.dim, w);
#pragma unroll
                for (int e = 0; e < L; ++e)
                    g[TWICE ? 0 : i][e] = g[TWICE ? 0 : i][e] * w[e];
            }
        };
        if constexpr (P::kNarrow) {
            if constexpr (!B::kAhead)
                ahead(0, row);
        } else {
            if constexpr (!TWICE)
                ahead(slot == 0 ? S - 1 : slot - 1, row + (S - 1) * step);
            ring_wait<S - 1>();
        }
        if constexpr (!TWICE) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
                fetch(i);
            slot = slot == S - 1 ? 0 : slot + 1;
            if constexpr (B::kAhead)
                ahead(0, row + step);
        }
        F sg = all_of<VEC>(0.f), sh = sg;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int k = TWICE ? 0 : i;
            if constexpr (TWICE)
                fetch(i);
            if (there && p.has(i, chunks)) {
#pragma unroll
                for (int e = 0; e < L; ++e) {
                    h[k][e] = (h[k][e] + less) * scale;
                    dw[i][e] = fused(g[k][e], h[k][e], dw[i][e]);
                    db[i][e] = db[i][e] + g[k][e];
                }
                weighted(i);
#pragma unroll
                for (int e = 0; e < L; ++e) {
                    sg = sg + g[k][e];
                    sh = fused(g[k][e], h[k][e], sh);
                }
            }
        }
        const Pair s = p.sum(Pair{both(sg), both(sh)}, s_part[turn]);
        if (there) {
            // (g - mean g - h mean(g h)) rstd
            const F to_g = all_of<VEC>(a.rms ? 0.f : -(s.x * inv) * rstd), to_h = all_of<VEC>(-(s.y * inv) * rstd);
            T *const dx = here.at(static_cast<T *>(a.dx), a.dx_token, a.dx_head);
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (p.has(i, chunks)) {
                    const int k = TWICE ? 0 : i;
                    if constexpr (TWICE) {
                        fetch(i);
                        weighted(i);
#pragma unroll
                        for (int e = 0; e < L; ++e)
                            h[k][e] = (h[k][e] + less) * scale;
                    }
#pragma unroll
                    for (int e = 0; e < L; ++e)
                        g[k][e] = fused(h[k][e], to_h, fused(g[k][e], scale, to_g));
                    store_chunk(p, dx, i, a.dim, g[k]);
                }
        }
        if constexpr (TWICE) {
            ahead(slot, row + S * step);
            slot = slot == S - 1 ? 0 : slot + 1;
        }
    }
    if (!a.partial)
        return;
    const int padded = padded_dim(a.dim);
    float *const out = a.partial + (int64_t)blockIdx.x * 2 * padded;
    float *const s_sums = reinterpret_cast<float *>(smem);
    if (groups > 1) {
        if constexpr (!P::kNarrow)
            asm volatile("cp.async.wait_all;" ::: "memory");   // (the sums take the ring's place)
        __syncthreads();
    }
    float *const to = groups > 1 ? s_sums + p.group * 2 * padded : out;
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (p.has(i, chunks)) {
            const int c = (p.first + i * P::kStep) * VEC;
            store_sums<VEC>(to + c, dw[i]);
            store_sums<VEC>(to + padded + c, db[i]);
        }
    if (groups > 1) {
        __syncthreads();
        for (int i = threadIdx.x; i < 2 * padded; i += blockDim.x) {
            float s = 0.f;
            for (int g = 0; g < groups; ++g)
                s += s_sums[g * 2 * padded + i];
            out[i] = s;
        }
    }
}

// dw, db: sums of the blocks' parts.  A block takes 64 of the columns, its
// warps shares of the parts, a lane two columns.
constexpr int kSumWarps = 32;
__global__ void __launch_bounds__(kSumWarps * 32) norm_sum_kernel(const float *partial, int parts, int dim, float *dweight, float *dbias)
{
    __shared__ float2 s[kSumWarps][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, padded = padded_dim(dim);
    const int i = (blockIdx.x * 32 + lane) * 2;
    wait_for_previous();
    let_next_start();
    float2 v = {0.f, 0.f};
    if (i < 2 * padded)
#pragma unroll 10
        for (int p = warp; p < parts; p += kSumWarps) {
            const float2 u = *reinterpret_cast<const float2 *>(partial + (int64_t)p * 2 * padded + i);
            v = {v.x + u.x, v.y + u.y};
        }
    s[warp][lane] = v;
    __syncthreads();
    if (threadIdx.x < 64) {
        const int at = blockIdx.x * 64 + threadIdx.x;
        const float *const column = reinterpret_cast<const float *>(s) + threadIdx.x;
        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < kSumWarps; ++k)
            sum += column[k * 64];
        if (dweight && at < dim)
            dweight[at] = sum;
        if (dbias && at >= padded && at < padded + dim)
            dbias[at - padded] = sum;
    }
}

// Blocks of the backward kernel on an SM: 640 threads, or one block that is
// larger than half of them.
int backward_blocks(int threads) { return threads > 320 ? 1 : 640 / threads; }

// Calls go(split) with the way a row of `chunks` lies over threads: a few
// lanes with two chunks each, a warp, or a block whose warps take 32 NV
// chunks each.  LONG: rows that always take a block.
template <typename T, int VEC, int NV, bool LONG, typename G>
cudaError_t with_split(int chunks, G &&go)
{
    if constexpr (!LONG) {
        static_assert(NV == 2 || NV == 4 || NV == 8, "a warp's splits below");
        if (chunks <= 2)
            return go((Split<T, VEC, 2, 1> *)nullptr);
        if (chunks <= 8)
            return go((Split<T, VEC, 2, 4> *)nullptr);
        if (chunks <= 16)
            return go((Split<T, VEC, 2, 8> *)nullptr);
        if (chunks <= 32)
            return go((Split<T, VEC, 2, 16> *)nullptr);
        if (chunks <= 64)
            return go((Split<T, VEC, 2, 32> *)nullptr);
        if constexpr (NV >= 4)
            if (chunks <= 128)
                return go((Split<T, VEC, 4, 32> *)nullptr);
        if constexpr (NV >= 8)
            if (chunks <= 256)
                return go((Split<T, VEC, 8, 32> *)nullptr);
    }
    return go((Split<T, VEC, NV, 64> *)nullptr);
}

template <typename P>
int threads_of(int chunks)
{
    return P::kBlock ? (chunks + 32 * P::NV - 1) / (32 * P::NV) * 32 : kThreads;
}

template <typename T, int VEC, int MOST, bool LONG = false>
cudaError_t launch_forward(const NormArgs &a, cudaStream_t st)
{
    const int chunks = (a.dim + VEC - 1) / VEC;
    return with_split<T, VEC, MOST, LONG>(chunks, [&](auto split) -> cudaError_t {
        using P = std::remove_pointer_t<decltype(split)>;
        const int threads = threads_of<P>(chunks), groups = P::kBlock ? 1 : threads / P::TPR;
        const int64_t turns = (a.rows + groups - 1) / groups;
        const size_t smem = Ring<P, 1, kForwardRows<P>>::bytes(threads);
        static PerDevice<bool> allowed;
        if (smem > kPlainSmem)
            if (cudaError_t e = allow_smem((const void *)norm_kernel<P>, (int)kMostSmem, allowed))
                return e;
        const int64_t most = (int64_t)num_sms() * max(1, min(1024 / threads, (int)(kMostSmem / max(smem, (size_t)1))));
        const int64_t blocks = turns < most ? turns : most;
        return launch_early(norm_kernel<P>, dim3((unsigned)blocks), threads, smem, st, 1, a);
    });
}

template <typename P, int THREADS>
cudaError_t launch_backward_of(const NormGradArgs &a, int threads, int blocks, cudaStream_t st)
{
    const int groups = P::kBlock ? 1 : threads / P::TPR;
    const size_t parts = a.partial && groups > 1 ? (size_t)groups * 2 * padded_dim(a.dim) * sizeof(float) : 0;
    const size_t rows = Backward<P, THREADS>::bytes(threads), smem = rows > parts ? rows : parts;
    static PerDevice<bool> allowed;
    if (smem > kPlainSmem)
        if (cudaError_t e = allow_smem((const void *)norm_grad_kernel<P, THREADS>, (int)kMostSmem, allowed))
            return e;
    return launch_early(norm_grad_kernel<P, THREADS>, dim3((unsigned)blocks), threads, smem, st, 1, a);
}

template <typename T, int VEC, int MOST, bool LONG = false>
cudaError_t launch_backward(const NormGradArgs &given, cudaStream_t st)
{
    NormGradArgs a = given;
    const bool sums = a.dweight || a.dbias;
    a.partial = sums ? static_cast<float *>(a.workspace) : nullptr;
    int blocks = 0;
    if (a.rows > 0) {
        const cudaError_t e = with_split<T, VEC, MOST, LONG>((a.dim + VEC - 1) / VEC, [&](auto split) -> cudaError_t {
            using P = std::remove_pointer_t<decltype(split)>;
            const int threads = threads_of<P>((a.dim + VEC - 1) / VEC), groups = P::kBlock ? 1 : threads / P::TPR;
            const int64_t turns = (a.rows + groups - 1) / groups, most = (int64_t)num_sms() * (kTwice<P> ? 1 : backward_blocks(threads));
            // (all blocks take as many turns; four of them, if each SM has that many, halve the partial sums and more: 1531 rows of
            // 1024 bf16 take 7.8 us instead of 11.9)
            const int64_t few = turns / num_sms() < 4 ? turns / num_sms() : 4, least = sums && few > 1 ? few : 1;
            const int64_t each = (turns + most - 1) / most > least ? (turns + most - 1) / most : least;
            blocks = (int)((turns + each - 1) / each);
            if constexpr (LONG)
                return launch_backward_of<P, P::kNarrow ? 1024 : 512>(a, threads, blocks, st);
            else if constexpr (P::kBlock) {
                if constexpr (P::kNarrow)
                    if (threads > 512)
                        return launch_backward_of<P, 1024>(a, threads, blocks, st);
                if (threads > 320)
                    return launch_backward_of<P, 512>(a, threads, blocks, st);
                return launch_backward_of<P, 320>(a, threads, blocks, st);
            } else
                return launch_backward_of<P, 256>(a, threads, blocks, st);
        });
        if (e != cudaSuccess)
            return e;
    }
    if (!sums)
        return cudaSuccess;
    return launch_early(norm_sum_kernel, dim3((unsigned)((2 * padded_dim(a.dim) + 63) / 64)), kSumWarps * 32, 0, st, 1, static_cast<const float *>(a.workspace), blocks, a.dim, a.dweight, a.dbias);
}

bool wide(int64_t bits, bool bf16) { return bits % (bf16 ? 8 : 4) == 0; }

} // namespace

size_t norm_grad_workspace_bytes(int32_t dim)
{
    // (whatever the type and strides: a row of a block has a warp for at most 512 elements, and two of them at least; rows beyond
    // 8192, which can have fewer warps, take one block an SM)
    const int threads = dim > 1024 ? (dim + 511) / 512 * 32 : dim > 256 ? 64 : kThreads;
    return (size_t)num_sms() * backward_blocks(threads) * 2 * (size_t)padded_dim(dim) * sizeof(float);
}

cudaError_t launch_norm(const NormArgs &a, cudaStream_t st)
{
    const bool w = wide(a.x_token | a.x_head | a.y_token | a.y_head | a.dim, a.bf16), few = a.dim <= kFewForward;
    if (a.bf16)
        return w ? launch_forward<__nv_bfloat16, 8, 4>(a, st) : few ? launch_forward<__nv_bfloat16, 2, 4>(a, st) : launch_forward<__nv_bfloat16, 2, 8, true>(a, st);
    return w ? launch_forward<float, 4, 4>(a, st) : few ? launch_forward<float, 1, 8>(a, st) : launch_forward<float, 1, 16, true>(a, st);
}

cudaError_t launch_norm_grad(const NormGradArgs &a, cudaStream_t st)
{
    const bool w = wide(a.dy_token | a.dy_head | a.x_token | a.x_head | a.dx_token | a.dx_head | a.dim, a.bf16), few = a.dim <= kFewBackward;
    // (Elements of a thread: the fewest that need no more than 512 threads.  At 2^26 elements, of which copies take 59.5 us: rows of
    // 9216 bf16 with 16 take 133 us, with 24 85, with 32 130; 13824 with 16 119, with 24 119, with 32 98.)
    const int of_thread = a.dim <= 512 * 16 ? 16 : a.dim <= 512 * 24 ? 24 : 32;
    if (a.bf16)
        return !w                ? (few ? launch_backward<__nv_bfloat16, 2, 4>(a, st) : launch_backward<__nv_bfloat16, 2, 8, true>(a, st))
               : of_thread == 16 ? launch_backward<__nv_bfloat16, 8, 2>(a, st)
               : of_thread == 24 ? launch_backward<__nv_bfloat16, 8, 3, true>(a, st)
                                 : launch_backward<__nv_bfloat16, 8, 4, true>(a, st);
    return !w                ? (few ? launch_backward<float, 1, 8>(a, st) : launch_backward<float, 1, 16, true>(a, st))
           : of_thread == 16 ? launch_backward<float, 4, 4>(a, st)
           : of_thread == 24 ? launch_backward<float, 4, 6, true>(a, st)
                             : launch_backward<float, 4, 8, true>(a, st);
}

} // namespace rfq
