// Product of 8-bit matrices with a scale for every token and channel: sums of 8-bit products in 32-bit integers, exact in
// any order, so that tiles, splits and schedules are free; then three roundings in binary32 and one to the type.
//
// Three kernels.  One and two tokens are bound by reading the weights once and need nothing but loads and integer dot products
// (k_matmul8_few).  Up to a few hundred tokens, the weights still are most of what is read: blocks of 128 channels
// and up to 128 tokens (k_matmul8).  Beyond, the tensor cores are the bound: pairs of SMs on tiles of 256 x 256 (k_matmul8_pair).
#include <cuda.h>

#include <atomic>
#include <type_traits>

#include "cluster.cuh"
#include "elements.cuh"

namespace cdadam {

constexpr int kRowsP = 128, kBytesK = 128, kMaxRing = 8;

__device__ __forceinline__ void tma_2d(void *dst, const CUtensorMap *map, int x, int y, uint64_t *bar)
{
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(smem_addr(dst)), "l"(map), "r"(x), "r"(y), "r"(smem_addr(bar)) : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void commit(uint64_t *bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_addr(bar)) : "memory");
}
// Operand in shared memory: rows of 128 bytes, 16-byte vectors swizzled within groups of eight rows (1024 bytes apart).
__device__ __forceinline__ uint64_t operand(const void *p)
{
    return (uint64_t)((smem_addr(p) >> 4) & 0x3fff) | (uint64_t)1 << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
// Signed 8-bit operands, both with the summed index along rows, 32-bit integer sums.
__host__ __device__ constexpr uint32_t shape8(int m, int n)
{
    return 2u << 4 | 1u << 7 | 1u << 10 | (uint32_t)(n >> 3) << 17 | (uint32_t)(m >> 4) << 24;
}
__device__ __forceinline__ void mma8(uint32_t d, uint64_t a, uint64_t b, uint32_t shape, bool add)
{
    asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\n"
                 "tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n}"
                 ::"r"(d), "l"(a), "l"(b), "r"(shape), "r"((uint32_t)add) : "memory");
}
__device__ __forceinline__ void read_sums(uint32_t addr, int (&v)[16])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n"
                 "tcgen05.wait::ld.sync.aligned;"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
                   "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
                 : "r"(addr) : "memory");
}
__device__ __forceinline__ void read_sums32(uint32_t addr, int (&v)[32])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,"
                 "%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];\n"
                 "tcgen05.wait::ld.sync.aligned;"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
                   "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]),
                   "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]),
                   "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
                 : "r"(addr) : "memory");
}
// What has become of a thread's waits: 0: all in time; 1: one ran out and the thread waited a second time, with the
// default limit: the block's results are NaN; 2: that was in vain too: nothing more is waited for or started.
__device__ __noinline__ int wait_again(uint64_t *bar, uint32_t parity, int limit, int late)
{
    if (late == 2 || (limit > 0 && mbar_wait_bounded(bar, parity, limit))) return late;
    return mbar_wait_bounded(bar, parity) ? 1 : 2;
}
// After a wait in vain, whichever thread's it was: the copies that may still be under way (of the last stages of a ring, of
// `started` in all) land before the block leaves its shared memory.
__device__ __noinline__ void land(uint64_t *full, int started, int ring)
{
    for (int k = max(0, started - ring); k < started; ++k) mbar_wait_bounded(&full[k % ring], k / ring & 1);
}
__device__ __forceinline__ int wait_for(uint64_t *bar, uint32_t parity, int limit, int late)
{
    if (limit != 0 && mbar_try_wait(bar, parity)) return late;
    return wait_again(bar, parity, limit < 0 ? kWaitLimit : limit, late);
}

// An output, in the documented steps (packed products and sums would be contracted by the assembler).  Without a bias, -0: that
// sum is the other term, whichever zero it may be.
constexpr float kNoBias = -0.0f;
__device__ __forceinline__ float output(int sum, float x_scale, float w_scale, float bias)
{
    return __fadd_rn(__fmul_rn(__fmul_rn((float)sum, x_scale), w_scale), bias);
}
// Four channels' outputs of a token; `vec`: every four of them start on a multiple of their size, n of them are there.
template <typename T>
__device__ __forceinline__ void store4(T *to, const float (&f)[4], bool vec, int n)
{
    if (vec && n >= 4) {
        if constexpr (sizeof(T) == 4) *reinterpret_cast<float4 *>(to) = make_float4(f[0], f[1], f[2], f[3]);
        else *reinterpret_cast<uint2 *>(to) = make_uint2(Vec<T>::down(make_float2(f[0], f[1])), Vec<T>::down(make_float2(f[2], f[3])));
        return;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e < n) to[e] = narrow<T>(f[e]);
}

// ---------------------------------------------------------------------------------------------
// A block takes 128 channels and BN tokens: the weights are the first operand of the tensor core's product (its 128
// rows), the tokens the second, so that few tokens cost a narrow product and every weight is read once per BN
// tokens.  One thread fills a ring of stages (128 bytes of every row) by tiled bulk copies, one issues the products,
// the sums stay in tensor memory.  Where there are few tiles, a cluster of blocks shares the rows' length; its blocks fetch
// each other's sums from shared memory, 16 bytes at a time.
// Measured: 64 tokens x 131072 channels x 4096 97 us (5.7 TB/s), 64 x 30522 x 4096 26 to 28 us (4.8 TB/s; what is beside
// the weights' 19 us is the launch, the first copy's way and the last tile's outputs), 64 x 4096 x 4096 10 us,
// 509 x 2003 x 1021 8.4 us.
// ---------------------------------------------------------------------------------------------
template <typename T, int BN>
__global__ void __launch_bounds__(128) k_matmul8(const __grid_constant__ CUtensorMap wmap, const __grid_constant__ CUtensorMap xmap, Matmul8 a,
                                                 int ring, int splits, int token_tiles)
{
    constexpr int STAGE = (kRowsP + BN) * kBytesK, COLUMNS = BN < 32 ? 32 : BN;
    extern __shared__ char raw[];
    char *const stages = raw + (-smem_addr(raw) & 1023);
    __shared__ uint64_t full[kMaxRing], empty[kMaxRing], done;
    __shared__ uint32_t tmem;
    __shared__ int lates[2], any_late;
    __shared__ float x_scale[BN];
    __shared__ __align__(16) float w_scale[kRowsP], bias[kRowsP];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, rank = blockIdx.x % splits;
    const int64_t tile = blockIdx.x / splits, channel0 = tile / token_tiles * kRowsP, token0 = tile % token_tiles * BN;
    const int blocks = (int)((a.inner + kBytesK - 1) / kBytesK);
    const int first = (int)((int64_t)blocks * rank / splits), n = (int)((int64_t)blocks * (rank + 1) / splits) - first;
    auto fill = [&](int i, int s) {
        mbar_arrive_expect_tx(&full[s], STAGE);
        char *to = stages + s * STAGE;
        tma_2d(to, &wmap, (first + i) * kBytesK, (int)channel0, &full[s]);
        tma_2d(to + kRowsP * kBytesK, &xmap, (first + i) * kBytesK, (int)token0, &full[s]);
    };
    if (threadIdx.x == 0) {
        for (int i = 0; i < ring; ++i) {
            mbar_init(&full[i], 1);
            mbar_init(&empty[i], 1);
        }
        mbar_init(&done, 1);
        mbar_fence_init();
        for (int i = 0; i < min(n, ring); ++i) fill(i, i);
        any_late = 0;
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&tmem)), "r"(COLUMNS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    for (int i = threadIdx.x; i < BN; i += 128) x_scale[i] = token0 + i < a.tokens ? a.x.scale[token0 + i] : 0.0f;
    {
        const int64_t c = channel0 + threadIdx.x;
        w_scale[threadIdx.x] = c < a.channels ? a.w.scale[c] : 0.0f;
        bias[threadIdx.x] = c < a.channels && a.bias.p ? any_at(a.bias, c) : kNoBias;
    }
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t sums = tmem;
    int late = 0, started = 0;
    if (threadIdx.x == 0) {
        int s = 0, phase = 0;
        for (started = min(n, ring); started < n; ++started) {
            late = wait_for(&empty[s], phase, a.wait_limit, late);
            if (late == 2) break;
            fill(started, s);
            if (++s == ring) { s = 0; phase ^= 1; }
        }
        lates[0] = late;
    } else if (threadIdx.x == 32) {
        int s = 0, phase = 0;
        for (int i = 0; i < n; ++i) {
            late = wait_for(&full[s], phase, a.wait_limit, late);
            if (late == 2) break;
            fence_after();
            const uint64_t w = operand(stages + s * STAGE), x = operand(stages + s * STAGE + kRowsP * kBytesK);
#pragma unroll
            for (int k = 0; k < kBytesK / 32; ++k) mma8(sums, w + 2 * k, x + 2 * k, shape8(kRowsP, BN), i > 0 || k > 0);
            commit(&empty[s]);
            if (++s == ring) { s = 0; phase ^= 1; }
        }
        commit(&done);
        lates[1] = late;
    }
    __syncwarp();
    late = wait_for(&done, 0, a.wait_limit, 0);
    if (late) any_late = 1;
    __syncthreads();
    fence_after();
    // The sums take the stages' place, a row of 128 channels for every token.  Every block of a cluster adds up a share of
    // the tokens from all of them; a warp takes a token at a time, a lane four channels.
    if (threadIdx.x == 0 && (lates[0] | lates[1])) {
        any_late = 1;
        if (max(lates[0], lates[1]) == 2) land(full, started, ring);
    }
    __syncwarp();
    int *const left = reinterpret_cast<int *>(stages);
    const int n_tokens = (int)min((int64_t)BN, a.tokens - token0);
#pragma unroll 1
    for (int c = 0; c < BN; c += 16) {
        int v[16];
        if (c >= n_tokens) break;
        read_sums(sums + ((uint32_t)warp << 21) + c, v);
#pragma unroll
        for (int e = 0; e < 16; ++e) left[(c + e) * kRowsP + threadIdx.x] = v[e];
    }
    __syncwarp();
    if (splits > 1) cluster_barrier();
    else __syncthreads();
    const float4 ws = *reinterpret_cast<const float4 *>(&w_scale[4 * lane]), bs = *reinterpret_cast<const float4 *>(&bias[4 * lane]);
    bool none = any_late != 0;
    if (splits > 1)
        for (int r = 0; r < splits; ++r) none |= load_at(at_rank(&any_late, r)) != 0;
    const int share = BN / splits, channels = (int)min((int64_t)4, max((int64_t)0, a.channels - channel0 - 4 * lane));
    const bool vec = (((uintptr_t)a.y | (uintptr_t)(a.y_stride * sizeof(T))) & (4 * sizeof(T) - 1)) == 0;
    T *const to = static_cast<T *>(a.y) + token0 * a.y_stride + channel0 + 4 * lane;
    const int last = min(n_tokens, (rank + 1) * share);
#pragma unroll 2
    for (int c = rank * share + warp; c < last; c += 4) {
        int4 v;
        if (splits == 1) {
            v = *reinterpret_cast<const int4 *>(&left[c * kRowsP + 4 * lane]);
        } else {
            int4 u[8];
#pragma unroll
            for (int r = 0; r < 8; ++r) u[r] = r < splits ? load4_at(at_rank(&left[c * kRowsP + 4 * lane], r)) : make_int4(0, 0, 0, 0);
            v = u[0];
#pragma unroll
            for (int r = 1; r < 8; ++r) v = make_int4(v.x + u[r].x, v.y + u[r].y, v.z + u[r].z, v.w + u[r].w);
        }
        const float x = none ? __uint_as_float(0x7fc00000u) : x_scale[c];
        const float f[4] = {output(v.x, x, ws.x, bs.x), output(v.y, x, ws.y, bs.y), output(v.z, x, ws.z, bs.z), output(v.w, x, ws.w, bs.w)};
        store4<T>(to + c * a.y_stride, f, vec, channels);
    }
    __syncwarp();
    if (splits > 1) cluster_barrier();                  // no block leaves while others read from it
    fence_before();
    __syncthreads();
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(sums), "r"(COLUMNS));
}

// ---------------------------------------------------------------------------------------------
// Many tokens: pairs of blocks, one on each SM, that stay and take one tile of 256 tokens and 256 channels after
// the other.  Here the tokens are the first operand: a thread then has a token's channels side by side, and they
// are packed without passing through others.  Each block holds half of the tokens' rows and half of the channels', the
// tensor cores of the two read both halves, and each ends up with the sums of its 128 tokens and all 256 channels.  Two
// sets of sums in tensor memory: eight warps turn one into outputs while the other is being added up, each 32 tokens and
// 128 channels, 128 bytes of a row at a time through shared memory.  The first block of a pair issues the products
// for both; its `full` barriers count the copies of both, `empty` and `ready` are told to both, `drained` counts the
// warps of both.
// Measured: 4096 tokens x 131072 channels x 4096 bf16 1.42 to 1.49 ms (2.96 POP/s; back to back under the power limit 1.6 to 1.7),
// 4096 x 30528 x 768 90 to 104 us, 4096 x 30522 x 768 (rows that are no whole vectors) 115 to 145 (from GPU to
// GPU); a library's 8-bit product with 32-bit integer output and no scales 1.38 ms for the first.
// ---------------------------------------------------------------------------------------------
constexpr int kPairTile = 256, kPairRing = 5, kPairStage = 2 * kRowsP * kBytesK, kPairThreads = 320, kLeaveBytes = 4096;

__device__ __forceinline__ void tma_2d_pair(void *dst, const CUtensorMap *map, int x, int y, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(smem_addr(dst)), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
__device__ __forceinline__ void commit_pair(uint64_t *bar)
{
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(smem_addr(bar)), "h"((uint16_t)3) : "memory");
}
__device__ __forceinline__ void mma8_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t shape, bool add)
{
    asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\n"
                 "tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n}"
                 ::"r"(d), "l"(a), "l"(b), "r"(shape), "r"((uint32_t)add) : "memory");
}

__device__ __forceinline__ void half_barrier(int half) { asm volatile("bar.sync %0, 128;" ::"r"(half + 1) : "memory"); }

// 32 channels' outputs of the thread's token to its warp's staging place: row `lane` of 128 bytes, its 16-byte vectors
// swizzled as the copy engine wants them; the first goes to vector `at`.
template <typename T>
__device__ __forceinline__ void leave_channels(char *place, int lane, int at, const int (&v)[32], float x_scale, const float *w_scale, const float *bias)
{
    constexpr int N = 16 / sizeof(T);
#pragma unroll
    for (int i = 0; i < 32 / N; ++i) {
        float2 f[N / 2];
#pragma unroll
        for (int e = 0; e < N; e += 4) {
            const int c = i * N + e;
            const float4 w = *reinterpret_cast<const float4 *>(w_scale + c);
            if (bias) {
                const float4 b = *reinterpret_cast<const float4 *>(bias + c);
                f[e / 2] = make_float2(output(v[c], x_scale, w.x, b.x), output(v[c + 1], x_scale, w.y, b.y));
                f[e / 2 + 1] = make_float2(output(v[c + 2], x_scale, w.z, b.z), output(v[c + 3], x_scale, w.w, b.w));
            } else {
                f[e / 2] = mul2(mul2(make_float2((float)v[c], (float)v[c + 1]), both(x_scale)), make_float2(w.x, w.y));
                f[e / 2 + 1] = mul2(mul2(make_float2((float)v[c + 2], (float)v[c + 3]), both(x_scale)), make_float2(w.z, w.w));
            }
        }
        *reinterpret_cast<uint4 *>(place + lane * 128 + (((at + i) ^ (lane & 7)) << 4)) = Vec<T>::pack(f);
    }
}

// Staged rows of 128 bytes from shared memory to rows that are no whole vectors: rows `first`, first + step, ..,
// by words; ODD: they begin between two words, and so each word is put together from two.  No branch in between: rows
// overlap.
__device__ __forceinline__ uint32_t staged_word(const char *place, int row, int lane)
{
    return *reinterpret_cast<const uint32_t *>(place + row * 128 + ((((lane >> 2) ^ row) & 7) << 4) + (lane & 3) * 4);
}
template <bool ODD>
__device__ __forceinline__ void leave_words(const char *place, unsigned short *p, int64_t stride, int first, int step, int tokens, int lane)
{
    constexpr int ROWS = 8;
    p += first * stride;
#pragma unroll 1
    for (int i = first; i < tokens; i += ROWS * step) {
        uint32_t w[ROWS], before[ROWS];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) w[r] = staged_word(place, (i + r * step) & 31, lane);
        if (ODD)
#pragma unroll
            for (int r = 0; r < ROWS; ++r) before[r] = __shfl_up_sync(0xffffffffu, w[r], 1);
#pragma unroll
        for (int r = 0; r < ROWS; ++r, p += step * stride) {
            if (i + r * step >= tokens) break;
            if (!ODD) {
                reinterpret_cast<uint32_t *>(p)[lane] = w[r];
            } else {
                if (lane > 0) reinterpret_cast<uint32_t *>(p - 1)[lane] = __funnelshift_l(before[r], w[r], 16);
                if ((lane + 1 & 31) < 2) p[lane ? 63 : 0] = (unsigned short)(lane ? w[r] >> 16 : w[r]);
            }
        }
    }
}
// `tokens` staged rows of `channels` outputs to anywhere.
template <typename T>
__device__ __forceinline__ void leave_rows(const char *place, T *p, int64_t stride, int tokens, int channels, int lane)
{
    if (sizeof(T) == 2 && channels == 64) {
        unsigned short *u = reinterpret_cast<unsigned short *>(p);
        const int odd = (int)((uintptr_t)p >> 1 & 1);
        if (stride & 1) {
            leave_words<false>(place, u, stride, odd, 2, tokens, lane);
            leave_words<true>(place, u, stride, 1 - odd, 2, tokens, lane);
        } else if (odd) {
            leave_words<true>(place, u, stride, 0, 1, tokens, lane);
        } else {
            leave_words<false>(place, u, stride, 0, 1, tokens, lane);
        }
        return;
    }
    if (sizeof(T) == 4 && channels == 32) {
        leave_words<false>(place, reinterpret_cast<unsigned short *>(p), 2 * stride, 0, 1, tokens, lane);
        return;
    }
#pragma unroll 1
    for (int i = 0; i < tokens; ++i, p += stride) {
        const uint32_t w = staged_word(place, i, lane);
        if constexpr (sizeof(T) == 4) {
            if (lane < channels) p[lane] = __uint_as_float(w);
        } else {
            unsigned short *u = reinterpret_cast<unsigned short *>(p) + 2 * lane;
            if (2 * lane < channels) u[0] = (unsigned short)w;
            if (2 * lane + 1 < channels) u[1] = (unsigned short)(w >> 16);
        }
    }
}

// TILED: the outputs' rows are whole 16-byte vectors and leave by tiled bulk copies.
template <typename T, bool TILED>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kPairThreads, 1)
k_matmul8_pair(const __grid_constant__ CUtensorMap wmap, const __grid_constant__ CUtensorMap xmap, const __grid_constant__ CUtensorMap ymap, Matmul8 a,
               int tiles, int token_tiles)
{
    extern __shared__ char raw[];
    char *const stages = raw + (-smem_addr(raw) & 1023);
    __shared__ uint64_t full[kPairRing], empty[kPairRing], ready[2], drained[2];
    __shared__ uint32_t tmem;
    __shared__ int lates[2];
    __shared__ __align__(16) float w_scale[2][kPairTile], bias[2][kPairTile];
    const int warp = threadIdx.x >> 5, rank = blockIdx.x & 1, pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    const int blocks = (int)((a.inner + kBytesK - 1) / kBytesK);
    if (threadIdx.x == 0) {
        for (int i = 0; i < kPairRing; ++i) {
            mbar_init(&full[i], 1);
            mbar_init(&empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&ready[i], 1);
            mbar_init(&drained[i], 16);
            lates[i] = 0;
        }
        mbar_fence_init();
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&tmem)), "r"(2 * kPairTile) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    }
    fence_before();
    __syncthreads();
    cluster_barrier();
    fence_after();
    const uint32_t sums = tmem;
    int late = 0, started = 0;
    if (threadIdx.x == 0) {
        int s = 0, phase = 1;
        for (int tile = pair; tile < tiles && late < 2; tile += pairs) {
            const int channel = tile / token_tiles * kPairTile + rank * kRowsP, token = tile % token_tiles * kPairTile + rank * kRowsP;
            for (int b = 0; b < blocks; ++b, ++started) {
                if (started >= kPairRing) late = wait_for(&empty[s], phase, a.wait_limit, late);
                if (late == 2) break;
                if (rank == 0) mbar_arrive_expect_tx(&full[s], 2 * kPairStage);
                char *to = stages + s * kPairStage;
                const uint32_t bar = at_rank(&full[s], 0);
                tma_2d_pair(to, &xmap, b * kBytesK, token, bar);
                tma_2d_pair(to + kRowsP * kBytesK, &wmap, b * kBytesK, channel, bar);
                if (++s == kPairRing) { s = 0; phase ^= 1; }
            }
        }
        lates[0] = late;
    } else if (threadIdx.x == 32 && rank == 0) {
        int set = 0, s = 0, phase = 0;
        for (int tile = pair; tile < tiles && late < 2; tile += pairs, ++set) {
            const int buffer = set & 1;
            if (set >= 2) late = wait_for(&drained[buffer], (set >> 1 & 1) ^ 1, a.wait_limit, late);
            fence_after();
            for (int b = 0; b < blocks; ++b) {
                late = wait_for(&full[s], phase, a.wait_limit, late);
                if (late == 2) break;
                fence_after();
                const uint64_t x = operand(stages + s * kPairStage), w = operand(stages + s * kPairStage + kRowsP * kBytesK);
#pragma unroll
                for (int k = 0; k < kBytesK / 32; ++k)
                    mma8_pair(sums + buffer * kPairTile, x + 2 * k, w + 2 * k, shape8(2 * kRowsP, kPairTile), b > 0 || k > 0);
                commit_pair(&empty[s]);
                if (++s == kPairRing) { s = 0; phase ^= 1; }
            }
            if (late < 2) commit_pair(&ready[buffer]);
        }
        lates[1] = late;
    } else if (warp >= 2) {
        constexpr int CHUNK = 128 / (int)sizeof(T), HALF = kPairTile / 2;     // channels that leave together: 32 or 64
        const int lane = threadIdx.x & 31, quarter = warp & 3, half = (warp - 2) >> 2, thread = quarter * 32 + lane;
        char *const place = stages + kPairRing * kPairStage + (warp - 2) * kLeaveBytes;
        int set = 0;
        for (int tile = pair; tile < tiles; tile += pairs, ++set) {
            const int buffer = set & 1;
            const int64_t token0 = (int64_t)(tile % token_tiles) * kPairTile + rank * kRowsP + quarter * 32;
            const int64_t channel0 = (int64_t)(tile / token_tiles) * kPairTile + half * HALF;
            float x_scale = token0 + lane < a.tokens ? a.x.scale[token0 + lane] : 0.0f;
            const bool real = channel0 + thread < a.channels;
            w_scale[buffer][half * HALF + thread] = real ? a.w.scale[channel0 + thread] : 0.0f;
            if (a.bias.p) bias[buffer][half * HALF + thread] = real ? any_at(a.bias, channel0 + thread) : 0.0f;
            half_barrier(half);
            late = wait_for(&ready[buffer], set >> 1 & 1, a.wait_limit, late);
            if (late) x_scale = __uint_as_float(0x7fc00000u);
            __syncwarp();
            fence_after();
            const uint32_t at = sums + buffer * kPairTile + half * HALF + ((uint32_t)quarter << 21);
            const int tokens = (int)min((int64_t)32, a.tokens - token0);
#pragma unroll 1
            for (int c = 0; c < HALF; c += CHUNK) {
                if (tokens <= 0 || channel0 + c >= a.channels) break;
#pragma unroll
                for (int d = 0; d < CHUNK; d += 32) {
                    int v[32];
                    read_sums32(at + c + d, v);
                    if (d == 0) {                       // what was here before has left
                        if (TILED && lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
                        __syncwarp();
                    }
                    const int first = half * HALF + c + d;
                    leave_channels<T>(place, lane, d * (int)sizeof(T) / 16, v, x_scale, &w_scale[buffer][first],
                                      a.bias.p ? &bias[buffer][first] : nullptr);
                }
                if (TILED) {
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) {
                        asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];"
                                     ::"l"(&ymap), "r"((int)channel0 + c), "r"((int)token0), "r"(smem_addr(place)) : "memory");
                        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                    }
                } else {
                    __syncwarp();
                    leave_rows<T>(place, static_cast<T *>(a.y) + token0 * a.y_stride + channel0 + c, a.y_stride, tokens,
                                  (int)min((int64_t)CHUNK, a.channels - channel0 - c), lane);
                    __syncwarp();
                }
            }
            // The products may overwrite the set: all of it is in registers.  Nothing but those reads is handed over, and their
            // order is that of tensor memory: the reads' wait, the fence, an arrival; on the other side a wait, the fence, the
            // product.  So the arrival is relaxed.  A release, even right behind the last read, also waits for the outputs
            // stored so far (on one GPU: 4096 x 30528 x 768 133 us instead of 102, 4096 x 30522 x 768 174 instead of 145); a
            // relaxed one there gains nothing (104 and 144).
            fence_before();
            __syncwarp();
            if (lane == 0)
                asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(at_rank(&drained[buffer], 0)) : "memory");
        }
        if (TILED && lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    }
    __syncwarp();
    fence_before();
    __syncthreads();
    // (the barriers of the first block count the copies of both; of a stage that it gave up, the second may have started its
    // half all the same: that barrier stays open, but the limit lasts longer than any copy)
    if (threadIdx.x == 0 && rank == 0 && max(lates[0], lates[1]) == 2) {
        land(full, started, kPairRing);
        if (lates[0] == 2) mbar_wait_bounded(&full[started % kPairRing], started / kPairRing & 1);
    }
    __syncwarp();
    cluster_barrier();
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(sums), "r"(2 * kPairTile));
}

// ---------------------------------------------------------------------------------------------
// One and two tokens: the weights are streamed once, 16 bytes a lane, and multiplied four at a time; what the kernels above
// need before their first byte arrives and after their last (tensor memory, barriers) costs more than their products are worth
// here.  From three tokens on the dot products would be the bound (16 a clock and SM: 4 x 30522 x 4096 31 us, by k_matmul8 24).
// A warp takes kFewChannels channels and every `slices`-th stretch of 512 bytes of them; the slices' sums meet in shared memory.
// Measured, one token: 131072 x 4096 82 us (6.5 TB/s), 30522 x 768 8 us, 4096 x 4096 4.7 us, 1000 x 768 2.5 us.
// ---------------------------------------------------------------------------------------------
constexpr int kFewWarps = 8, kFewChannels = 4;

// 16 bytes of a row, 0 beyond its end.
template <bool KEEP>
__device__ __forceinline__ int4 load16(const int8_t *row, int k, int inner)
{
    if (k + 16 <= inner) {
        const int4 *p = reinterpret_cast<const int4 *>(row + k);
        return KEEP ? __ldg(p) : __ldcs(p);
    }
    int w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (k + i < inner) w[i / 4] |= (int)(uint8_t)row[k + i] << (i % 4 * 8);
    return make_int4(w[0], w[1], w[2], w[3]);
}

template <typename T, int TOKENS>
__global__ void __launch_bounds__(kFewWarps * 32, 4) k_matmul8_few(Matmul8 a, int slices)
{
    constexpr int C = kFewChannels;
    __shared__ int parts[kFewWarps][C * TOKENS];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, slice = warp % slices, inner = (int)a.inner;
    const int64_t channel0 = ((int64_t)blockIdx.x * (kFewWarps / slices) + warp / slices) * C;
    const int8_t *w[C], *x[TOKENS];
#pragma unroll
    for (int c = 0; c < C; ++c) w[c] = a.w.p + min(channel0 + c, a.channels - 1) * a.w.stride;
#pragma unroll
    for (int t = 0; t < TOKENS; ++t) x[t] = a.x.p + min((int64_t)t, a.tokens - 1) * a.x.stride;
    int sums[C][TOKENS] = {};
    if (channel0 < a.channels)
#pragma unroll 2
        for (int k = (slice * 32 + lane) * 16; k < inner; k += slices * 512) {
            int4 v[C];
#pragma unroll
            for (int c = 0; c < C; ++c) v[c] = load16<false>(w[c], k, inner);
#pragma unroll
            for (int t = 0; t < TOKENS; ++t) {
                const int4 u = load16<true>(x[t], k, inner);
#pragma unroll
                for (int c = 0; c < C; ++c)
                    sums[c][t] = __dp4a(v[c].w, u.w, __dp4a(v[c].z, u.z, __dp4a(v[c].y, u.y, __dp4a(v[c].x, u.x, sums[c][t]))));
            }
        }
    int mine = 0;                                       // lane c TOKENS + t has channel c, token t
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int t = 0; t < TOKENS; ++t) {
            const int v = __reduce_add_sync(0xffffffffu, sums[c][t]);
            if (lane == c * TOKENS + t) mine = v;
        }
    if (slices > 1) {
        if (lane < C * TOKENS) parts[warp][lane] = mine;
        __syncthreads();
        if (slice != 0) return;
        mine = 0;
        if (lane < C * TOKENS)
            for (int i = 0; i < slices; ++i) mine += parts[warp + i][lane];
    }
    const int token = lane % TOKENS;
    const int64_t channel = channel0 + lane / TOKENS;
    if (lane < C * TOKENS && channel < a.channels && token < a.tokens) {
        const float bias = a.bias.p ? any_at(a.bias, channel) : kNoBias;
        static_cast<T *>(a.y)[token * a.y_stride + channel] =
            narrow<T>(output(mine, a.x.scale[token], a.w.scale[channel], bias));
    }
}

// ---------------------------------------------------------------------------------------------
// Launches
// ---------------------------------------------------------------------------------------------
typedef CUresult (*EncodeTiled)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// Kept for the process once it is found; NULL: not this time (where the look-up failed, the reason stays for the caller's
// cudaGetLastError()), and the next call looks again.
static EncodeTiled encode_tiled()
{
    static std::atomic<EncodeTiled> kept{nullptr};
    EncodeTiled fn = kept.load(std::memory_order_acquire);
    if (fn) return fn;
    void *p = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess)
        return nullptr;
    fn = reinterpret_cast<EncodeTiled>(p);
    kept.store(fn, std::memory_order_release);
    return fn;
}
// Boxes of 128 bytes of `rows` rows; what lies beyond a row's end or the last row reads as 0.
static bool describe(CUtensorMap *map, const Rows8 &m, int64_t rows, int64_t inner, int box_rows)
{
    const EncodeTiled fn = encode_tiled();
    if (!fn) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)inner, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)(rows > 1 ? m.stride : (inner + 15) / 16 * 16)};
    const cuuint32_t box[2] = {kBytesK, (cuuint32_t)box_rows}, ones[2] = {1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, m.p, dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T> static CUtensorMapDataType type_of()
{
    return std::is_same<T, float>::value ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
           : std::is_same<T, bf16>::value ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
}
// Boxes of 128 bytes of 32 tokens.
static bool describe_outputs(CUtensorMap *map, const Matmul8 &a, CUtensorMapDataType type, int size)
{
    const EncodeTiled fn = encode_tiled();
    if (!fn) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)a.channels, (cuuint64_t)a.tokens};
    const cuuint64_t strides[1] = {(cuuint64_t)(a.tokens > 1 ? a.y_stride * size : (a.channels * size + 15) / 16 * 16)};
    const cuuint32_t box[2] = {(cuuint32_t)(128 / size), 32}, ones[2] = {1, 1};
    return fn(map, type, 2, a.y, dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
              CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Blocks of 128 x BN tiles that fill the GPU's 148 SMs, one or two to each.
constexpr int64_t kEnoughTiles = 128, kMostBlocks = 296;

static int64_t tiles_of(const Matmul8 &a, int tokens, int channels)
{
    return (a.tokens + tokens - 1) / tokens * ((a.channels + channels - 1) / channels);
}
static int blocks_of(const Matmul8 &a) { return (int)((a.inner + kBytesK - 1) / kBytesK); }

template <typename T, int BN>
static bool product_as(const Matmul8 &a, cudaStream_t st)
{
    CUtensorMap wmap, xmap;
    if (!describe(&wmap, a.w, a.channels, a.inner, kRowsP) || !describe(&xmap, a.x, a.tokens, a.inner, BN)) return false;
    const int64_t token_tiles = (a.tokens + BN - 1) / BN, tiles = tiles_of(a, BN, kRowsP);
    // long rows are shared by up to four blocks (eight where even those are few): 64 x 4096 x 4096 by one 15.1 us, two 12.7,
    // four 9.8, eight 10.5; rows of up to 1024 bytes are not (256 x 2003 x 1021 7.7 by one, 8.7 by two)
    int splits = 1;
    if (blocks_of(a) > 8)
        while (splits < 8 && tiles * splits * 2 <= (splits < 4 ? kMostBlocks : kEnoughTiles)) splits *= 2;
    constexpr int STAGE = (kRowsP + BN) * kBytesK;
    int ring = 104 * 1024 / STAGE;
    ring = ring < kMaxRing ? ring : kMaxRing;
    const size_t smem = (size_t)ring * STAGE + 1024;
    auto kernel = k_matmul8<T, BN>;
    allow_shared(kernel, smem);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(tiles * splits));
    cfg.blockDim = dim3(128);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)splits;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cudaLaunchKernelEx(&cfg, kernel, wmap, xmap, a, ring, splits, (int)token_tiles);
    return true;
}
template <typename T>
static bool product_by_pairs(const Matmul8 &a, cudaStream_t st)
{
    CUtensorMap wmap, xmap;
    if (!describe(&wmap, a.w, a.channels, a.inner, kRowsP) || !describe(&xmap, a.x, a.tokens, a.inner, kRowsP)) return false;
    const int64_t token_tiles = (a.tokens + kPairTile - 1) / kPairTile, tiles = tiles_of(a, kPairTile, kPairTile);
    CUtensorMap ymap = {};
    // (a tiled copy writes whole 16-byte vectors: of a row that ends inside one it would overwrite what lies behind)
    const bool tiled = ((uintptr_t)a.y & 15) == 0 && a.channels * (int64_t)sizeof(T) % 16 == 0 &&
                       (a.tokens == 1 || a.y_stride * (int64_t)sizeof(T) % 16 == 0);
    if (tiled && !describe_outputs(&ymap, a, type_of<T>(), sizeof(T))) return false;
    const size_t smem = kPairRing * kPairStage + 8 * kLeaveBytes + 1024;
    auto kernel = tiled ? k_matmul8_pair<T, true> : k_matmul8_pair<T, false>;
    allow_shared(kernel, smem);
    queue(kernel, dim3((unsigned)(2 * (tiles < 74 ? tiles : 74))), kPairThreads, smem, st, wmap, xmap, ymap, a, (int)tiles, (int)token_tiles);
    return true;
}
template <typename T, int TOKENS>
static bool product_of_few(const Matmul8 &a, cudaStream_t st)
{
    // warps for about 24 to an SM, as far as the rows' length allows
    const int64_t channels = (a.channels + kFewChannels - 1) / kFewChannels;
    int slices = 1;
    while (slices < kFewWarps && channels * slices < 148 * 24 && a.inner > slices * 512) slices *= 2;
    const int64_t blocks = (channels * slices + kFewWarps - 1) / kFewWarps;
    queue(k_matmul8_few<T, TOKENS>, dim3((unsigned)blocks), kFewWarps * 32, 0, st, a, slices);
    return true;
}
template <typename T>
static bool product(const Matmul8 &a, cudaStream_t st)
{
    // 30522 x 768: one token 8.0 us this way and 8.9 by tiles of 16 tokens, two 9.6 and 9.1; 1000 x 768 2.5 and 8.5; 131072 x 4096 82 and 89
    if (a.tokens == 1) return product_of_few<T, 1>(a, st);
    if (a.tokens == 2) return product_of_few<T, 2>(a, st);
    // pairs, as soon as there are tiles for 32 of the 74 (512 x 4096 x 1024 9.4 us, by smaller tiles 9.5; 1024 x 4096 x 4096
    // 19.1 and 22.2; with 16 tiles, 256 x 4096 x 4096, 17.4 and 13.7)
    if (a.tokens > 128 && tiles_of(a, kPairTile, kPairTile) >= 32) return product_by_pairs<T>(a, st);
    // else the widest tiles of which there are enough: fewer blocks read the same weights (128 x 30522 x 768 12.5 us by 128
    // tokens, 16.3 by 64; 256 x 2003 x 1021 9.9 by 128, 8.4 by 64, 7.7 by 32)
    if (a.tokens > 64 && tiles_of(a, 128, kRowsP) >= kEnoughTiles) return product_as<T, 128>(a, st);
    if (a.tokens > 32 && (tiles_of(a, 64, kRowsP) >= kEnoughTiles || blocks_of(a) > 8)) return product_as<T, 64>(a, st);
    if (a.tokens > 16 && (tiles_of(a, 32, kRowsP) >= kEnoughTiles || blocks_of(a) > 8)) return product_as<T, 32>(a, st);
    return product_as<T, 16>(a, st);
}
bool launch_matmul8(const Matmul8 &a, int type, cudaStream_t st)
{
    return type == 0 ? product<float>(a, st) : type == 1 ? product<bf16>(a, st) : product<f16>(a, st);
}

}  // namespace cdadam
