// Product of 8-bit matrices with a scale for every token and channel.
//
// A block takes 128 channels and BN tokens: the weights are the first operand of the tensor core's product (its 128
// rows), the tokens the second, so that few tokens cost a narrow product and every weight is read once per BN
// tokens.  One thread fills a ring of stages (128 bytes of every row) by tiled bulk copies, one issues the products,
// the sums stay in tensor memory as 32-bit integers, exact in any order.  Where there are few tiles, a
// cluster of blocks shares the row's length and adds its sums up through shared memory.
#include <cuda.h>

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
__device__ __forceinline__ void cluster_barrier()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ int load_peer(const void *p, int rank)
{
    uint32_t at;
    int v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_addr(p)), "r"(rank));
    asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
    return v;
}

// What has become of a thread's waits: 0: all in time; 1: one ran out and the thread waited a second time, with the
// default limit: the block's results are NaN; 2: that was in vain too: nothing more is waited for or started.
__device__ __noinline__ int wait_again(uint64_t *bar, uint32_t parity, int limit, int late)
{
    if (late == 2 || (limit > 0 && mbar_wait_bounded(bar, parity, limit))) return late;
    return mbar_wait_bounded(bar, parity) ? 1 : 2;
}
__device__ __forceinline__ int wait_for(uint64_t *bar, uint32_t parity, int limit, int late)
{
    if (limit != 0 && mbar_try_wait(bar, parity)) return late;
    return wait_again(bar, parity, limit < 0 ? kWaitLimit : limit, late);
}

template <typename T>
__device__ __forceinline__ void store_product(const Matmul8 &a, int64_t token, int64_t channel, int sum, float x_scale, float w_scale, float bias,
                                              bool late)
{
    const float v = __fadd_rn(__fmul_rn(__fmul_rn((float)sum, x_scale), w_scale), bias);
    static_cast<T *>(a.y)[token * a.y_stride + channel] = narrow<T>(late ? __uint_as_float(0x7fc00000u) : v);
}

template <typename T, int BN>
__global__ void __launch_bounds__(128) k_matmul8(const __grid_constant__ CUtensorMap wmap, const __grid_constant__ CUtensorMap xmap, Matmul8 a,
                                                 int ring, int splits, int token_tiles)
{
    constexpr int STAGE = (kRowsP + BN) * kBytesK, COLUMNS = BN < 32 ? 32 : BN;
    extern __shared__ char raw[];
    char *const stages = raw + (-smem_addr(raw) & 1023);
    __shared__ uint64_t full[kMaxRing], empty[kMaxRing], done;
    __shared__ uint32_t tmem;
    __shared__ int lates[2];
    __shared__ float x_scale[BN];
    const int warp = threadIdx.x >> 5, rank = blockIdx.x % splits;
    const int64_t tile = blockIdx.x / splits, channel0 = tile / token_tiles * kRowsP, token0 = tile % token_tiles * BN;
    const int blocks = (int)((a.inner + kBytesK - 1) / kBytesK);
    const int first = (int)((int64_t)blocks * rank / splits), n = (int)((int64_t)blocks * (rank + 1) / splits) - first;
    if (threadIdx.x == 0) {
        for (int i = 0; i < ring; ++i) {
            mbar_init(&full[i], 1);
            mbar_init(&empty[i], 1);
        }
        mbar_init(&done, 1);
        mbar_fence_init();
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&tmem)), "r"(COLUMNS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    for (int i = threadIdx.x; i < BN; i += 128) x_scale[i] = token0 + i < a.tokens ? a.x.scale[token0 + i] : 0.0f;
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t sums = tmem;
    int late = 0;
    if (threadIdx.x == 0) {
        for (int i = 0; i < n; ++i) {
            const int s = i % ring, phase = i / ring & 1;
            if (i >= ring) late = wait_for(&empty[s], phase ^ 1, a.wait_limit, late);
            if (late == 2) {                            // what is under way lands before the block leaves
                for (int k = max(0, i - ring); k < i; ++k) mbar_wait_bounded(&full[k % ring], k / ring & 1);
                break;
            }
            mbar_arrive_expect_tx(&full[s], STAGE);
            char *to = stages + s * STAGE;
            tma_2d(to, &wmap, (first + i) * kBytesK, (int)channel0, &full[s]);
            tma_2d(to + kRowsP * kBytesK, &xmap, (first + i) * kBytesK, (int)token0, &full[s]);
        }
        lates[0] = late;
    } else if (threadIdx.x == 32) {
        for (int i = 0; i < n; ++i) {
            const int s = i % ring, phase = i / ring & 1;
            late = wait_for(&full[s], phase, a.wait_limit, late);
            if (late == 2) break;
            fence_after();
            const uint64_t w = operand(stages + s * STAGE), x = operand(stages + s * STAGE + kRowsP * kBytesK);
#pragma unroll
            for (int k = 0; k < kBytesK / 32; ++k) mma8(sums, w + 2 * k, x + 2 * k, shape8(kRowsP, BN), i > 0 || k > 0);
            commit(&empty[s]);
        }
        commit(&done);
        lates[1] = late;
    }
    __syncwarp();
    late = wait_for(&done, 0, a.wait_limit, 0);
    __syncthreads();
    fence_after();
    const int64_t channel = channel0 + threadIdx.x;
    const bool mine = channel < a.channels;
    const float w_scale = mine ? a.w.scale[channel] : 0.0f, bias = mine && a.bias.p ? any_at(a.bias, channel) : 0.0f;
    const uint32_t lane_at = sums + ((uint32_t)warp << 21);
    bool none = (late | lates[0] | lates[1]) != 0;
    if (splits == 1) {
#pragma unroll 1
        for (int c = 0; c < BN; c += 16) {
            if (token0 + c >= a.tokens) break;
            int v[16];
            __syncwarp();
            read_sums(lane_at + c, v);
#pragma unroll
            for (int e = 0; e < 16; ++e)
                if (mine && token0 + c + e < a.tokens)
                    store_product<T>(a, token0 + c + e, channel, v[e], x_scale[c + e], w_scale, bias, none);
        }
    } else {
        // every block leaves its sums in the stages' place and adds up a share of the tokens
        int *const left = reinterpret_cast<int *>(stages);
        __shared__ int any_late;
        if (threadIdx.x == 0) any_late = 0;
        __syncthreads();
        if (none) any_late = 1;
#pragma unroll 1
        for (int c = 0; c < BN; c += 16) {
            int v[16];
            read_sums(lane_at + c, v);
#pragma unroll
            for (int e = 0; e < 16; ++e) left[(c + e) * kRowsP + threadIdx.x] = v[e];
        }
        cluster_barrier();
        for (int r = 0; r < splits; ++r) none |= load_peer(&any_late, r) != 0;
        for (int c = BN * rank / splits; c < BN * (rank + 1) / splits; ++c) {
            if (token0 + c >= a.tokens) break;
            int v = 0;
            for (int r = 0; r < splits; ++r) v += load_peer(&left[c * kRowsP + threadIdx.x], r);
            if (mine) store_product<T>(a, token0 + c, channel, v, x_scale[c], w_scale, bias, none);
        }
        __syncwarp();
        cluster_barrier();                              // no block leaves while others read from it
    }
    fence_before();
    __syncthreads();
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(sums), "r"(COLUMNS));
}

// ---------------------------------------------------------------------------------------------
// Launches
// ---------------------------------------------------------------------------------------------
typedef CUresult (*EncodeTiled)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

static EncodeTiled encode_tiled()
{
    static EncodeTiled fn = [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess)
            p = nullptr;
        return reinterpret_cast<EncodeTiled>(p);
    }();
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

template <typename T, int BN>
static bool product_as(const Matmul8 &a, cudaStream_t st)
{
    CUtensorMap wmap, xmap;
    if (!describe(&wmap, a.w, a.channels, a.inner, kRowsP) || !describe(&xmap, a.x, a.tokens, a.inner, BN)) return false;
    const int64_t token_tiles = (a.tokens + BN - 1) / BN, tiles = (a.channels + kRowsP - 1) / kRowsP * token_tiles;
    const int blocks = (int)((a.inner + kBytesK - 1) / kBytesK);
    int splits = 1;
    while (splits < 8 && tiles * splits * 2 <= 296 && blocks >= splits * 4) splits *= 2;
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
static bool product(const Matmul8 &a, cudaStream_t st)
{
    if (a.tokens <= 16) return product_as<T, 16>(a, st);
    if (a.tokens <= 32) return product_as<T, 32>(a, st);
    if (a.tokens <= 64) return product_as<T, 64>(a, st);
    return product_as<T, 128>(a, st);
}
bool launch_matmul8(const Matmul8 &a, int type, cudaStream_t st)
{
    return type == 0 ? product<float>(a, st) : type == 1 ? product<bf16>(a, st) : product<f16>(a, st);
}

}  // namespace cdadam
