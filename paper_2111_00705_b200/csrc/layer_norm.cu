// Layer norm, forward and backward.
//
// A row is held in registers: a group of THREADS threads (a warp, or a whole block) has N elements
// of it each, loaded once, so mean, squared deviations and output come from one read.  Elements
// are loaded in units of W consecutive ones: W elements of 16 bytes where every row starts on a
// multiple of 16 bytes (and the row is a whole number of units), else single elements.
#include "elements.cuh"

namespace cdadam {

// ---------------------------------------------------------------------------------------------
// W consecutive elements, as they are in memory.
// ---------------------------------------------------------------------------------------------
template <typename T, int W> struct Unit;

template <typename T>
struct Unit<T, 1> {
    T v;
    __device__ __forceinline__ void load(const T *p) { v = *p; }
    __device__ __forceinline__ void zero() { v = narrow<T>(0.0f); }
    __device__ __forceinline__ void wide(float (&f)[1]) const { f[0] = widen(v); }
    static __device__ __forceinline__ void store(T *p, const float (&f)[1]) { *p = narrow<T>(f[0]); }
};

template <typename T, int W>
struct Unit {
    static_assert(W == Vec<T>::n, "16 bytes");
    uint4 u;
    __device__ __forceinline__ void load(const T *p)
    {
        asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                     : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w) : "l"(p) : "memory");
    }
    __device__ __forceinline__ void zero() { u = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ void wide(float (&f)[W]) const
    {
        float2 g[W / 2];
        Vec<T>::wide(u, g);
#pragma unroll
        for (int i = 0; i < W / 2; ++i) { f[2 * i] = g[i].x; f[2 * i + 1] = g[i].y; }
    }
    static __device__ __forceinline__ void store(T *p, const float (&f)[W])
    {
        float2 g[W / 2];
#pragma unroll
        for (int i = 0; i < W / 2; ++i) g[i] = make_float2(f[2 * i], f[2 * i + 1]);
        const uint4 u = Vec<T>::pack(g);
        asm volatile("st.global.cs.v4.u32 [%0], {%1,%2,%3,%4};" ::"l"(p), "r"(u.x), "r"(u.y), "r"(u.z), "r"(u.w) : "memory");
    }
};

// W consecutive parameters as binary32; `wide4`: binary32 parameters that start on 16 bytes.
template <int W>
__device__ __forceinline__ void parameters(const AnyVec &v, bool wide4, int64_t j, float absent, float (&f)[W])
{
    if (!v.p) {
#pragma unroll
        for (int i = 0; i < W; ++i) f[i] = absent;
    } else if (W >= 4 && wide4) {
#pragma unroll
        for (int i = 0; i < W / 4; ++i) {
            const float4 q = __ldg(reinterpret_cast<const float4 *>(static_cast<const float *>(v.p) + j) + i);
            f[4 * i] = q.x; f[(4 * i + 1) % W] = q.y; f[(4 * i + 2) % W] = q.z; f[(4 * i + 3) % W] = q.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < W; ++i) f[i] = any_at(v, j + i);
    }
}
__device__ __forceinline__ bool is_wide4(const AnyVec &v) { return v.type == 0 && ((uintptr_t)v.p & 15) == 0; }

// Sum over a row's threads, the same in each: a warp's lanes, or the block (`sh`: 32 floats that
// nothing else uses before the next barrier).
template <int THREADS>
__device__ __forceinline__ float row_sum(float v, float *sh)
{
    return THREADS == 32 ? warp_sum(v) : block_sum_all<THREADS < 32 ? 32 : THREADS>(v, sh);
}
template <int THREADS>
__device__ __forceinline__ float2 row_sum2(float a, float b, float2 *sh)
{
    a = warp_sum(a);
    b = warp_sum(b);
    if (THREADS == 32) return make_float2(a, b);
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = make_float2(a, b);
    __syncthreads();
    const int lane = threadIdx.x & 31;
    const float2 v = lane < THREADS / 32 ? sh[lane] : make_float2(0.0f, 0.0f);
    return make_float2(warp_sum(v.x), warp_sum(v.y));
}

// ---------------------------------------------------------------------------------------------
// Forward.  THREADS = 32: a block of 256 threads has eight rows; else a block has one.  U units of W
// elements a thread.
// ---------------------------------------------------------------------------------------------
template <int THREADS> constexpr int kBlockOf = THREADS == 32 ? 256 : THREADS;

template <typename T, int W, int U, int THREADS>
__global__ void __launch_bounds__(kBlockOf<THREADS>) k_norm(NormForward a)
{
    __shared__ float sh[2][32];
    const int t = threadIdx.x % THREADS;
    const int64_t row = (int64_t)blockIdx.x * (kBlockOf<THREADS> / THREADS) + threadIdx.x / THREADS;
    if (THREADS == 32 && row >= a.rows) return;
    const T *x = static_cast<const T *>(a.x) + row * a.x_stride;
    const int cols = (int)a.cols;
    Unit<T, W> u[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const int j = (t + i * THREADS) * W;
        if (j < cols) u[i].load(x + j);
        else u[i].zero();
    }
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < U; ++i) {
        float f[W];
        u[i].wide(f);
#pragma unroll
        for (int e = 0; e < W; ++e) s += f[e];
    }
    const float mean = row_sum<THREADS>(s, sh[0]) / (float)cols;
    s = 0.0f;
#pragma unroll
    for (int i = 0; i < U; ++i) {
        float f[W];
        u[i].wide(f);
        const bool in = (t + i * THREADS) * W < cols;
#pragma unroll
        for (int e = 0; e < W; ++e) {
            const float c = in ? f[e] - mean : 0.0f;
            s = fmaf(c, c, s);
        }
    }
    const float rstd = 1.0f / sqrtf(row_sum<THREADS>(s, sh[1]) / (float)cols + a.eps);
    T *y = static_cast<T *>(a.y) + row * a.y_stride;
    const bool w4 = is_wide4(a.weight), b4 = is_wide4(a.bias);
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const int j = (t + i * THREADS) * W;
        if (j < cols) {
            float f[W], w[W], b[W];
            u[i].wide(f);
            parameters<W>(a.weight, w4, j, 1.0f, w);
            parameters<W>(a.bias, b4, j, 0.0f, b);
#pragma unroll
            for (int e = 0; e < W; ++e) f[e] = fmaf((f[e] - mean) * rstd, w[e], b[e]);
            Unit<T, W>::store(y + j, f);
        }
    }
    if (t == 0) {
        if (a.mean) a.mean[row] = mean;
        if (a.rstd) a.rstd[row] = rstd;
    }
}

// Rows too long for the registers of a block: three passes, the later two from L2.
constexpr int kLongBlock = 1024;

template <typename T>
__global__ void __launch_bounds__(kLongBlock) k_norm_long(NormForward a)
{
    __shared__ float sh[2][32];
    const int64_t row = blockIdx.x;
    const T *x = static_cast<const T *>(a.x) + row * a.x_stride;
    T *y = static_cast<T *>(a.y) + row * a.y_stride;
    float s = 0.0f;
    for (int64_t j = threadIdx.x; j < a.cols; j += kLongBlock) s += widen(x[j]);
    const float mean = block_sum_all<kLongBlock>(s, sh[0]) / (float)a.cols;
    s = 0.0f;
    for (int64_t j = threadIdx.x; j < a.cols; j += kLongBlock) {
        const float c = widen(x[j]) - mean;
        s = fmaf(c, c, s);
    }
    const float rstd = 1.0f / sqrtf(block_sum_all<kLongBlock>(s, sh[1]) / (float)a.cols + a.eps);
    for (int64_t j = threadIdx.x; j < a.cols; j += kLongBlock) {
        const float w = a.weight.p ? any_at(a.weight, j) : 1.0f, b = a.bias.p ? any_at(a.bias, j) : 0.0f;
        y[j] = narrow<T>(fmaf((widen(x[j]) - mean) * rstd, w, b));
    }
    if (threadIdx.x == 0) {
        if (a.mean) a.mean[row] = mean;
        if (a.rstd) a.rstd[row] = rstd;
    }
}

// ---------------------------------------------------------------------------------------------
// Backward.  A block works on rows of one group, one after the other, and every thread keeps the
// sums over rows of its own columns in registers, so x and dy are read once for dx, dweight and
// dbias together.  THREADS = 32: the block's warps have a row each and add their sums up at the
// end, in order.  `blocks` blocks share a group; with more than one each leaves its sums in the
// workspace and k_norm_sums adds them, in order: no atomics, the same bits every time.
// ---------------------------------------------------------------------------------------------
__device__ __forceinline__ void store_grad(void *p, int64_t i, int type, int accumulate, float v)
{
    if (type == 0) {
        float *q = static_cast<float *>(p) + i;
        *q = accumulate ? *q + v : v;
    } else if (type == 1) {
        bf16 *q = static_cast<bf16 *>(p) + i;
        *q = narrow<bf16>(accumulate ? widen(*q) + v : v);
    } else {
        f16 *q = static_cast<f16 *>(p) + i;
        *q = narrow<f16>(accumulate ? widen(*q) + v : v);
    }
}

// The sums w, b of column j of group g from this block.
__device__ __forceinline__ void leave_sums(const NormBackward &a, int64_t g, int blocks, int64_t j, float w, float b)
{
    if (blocks > 1) {
        float *p = a.parts + ((g * blocks + blockIdx.x) * 2) * a.cols;
        p[j] = w;
        p[a.cols + j] = b;
    } else {
        if (a.dweight) store_grad(a.dweight, g * a.dweight_stride + j, a.grad_type, a.accumulate, w);
        if (a.dbias) store_grad(a.dbias, g * a.dbias_stride + j, a.grad_type, a.accumulate, b);
    }
}

template <typename T, int W, int U, int THREADS>
__global__ void __launch_bounds__(kBlockOf<THREADS>) k_norm_backward(NormBackward a, int blocks)
{
    constexpr int BT = kBlockOf<THREADS>, ROWS = BT / THREADS;
    constexpr bool AHEAD = W > 1 ? U <= 2 : U <= 8;     // registers for the next row
    extern __shared__ __align__(16) float wide_w[];     // the weight, binary32; at the end the block's sums
    __shared__ float2 sh[2][32];
    const int t = threadIdx.x % THREADS, sub = threadIdx.x / THREADS, cols = (int)a.cols;
    const int64_t per = a.rows / a.groups, first = blockIdx.y * per, end = first + per;
    for (int j = threadIdx.x; j < (cols + 3) / 4 * 4; j += BT) wide_w[j] = a.weight.p && j < cols ? any_at(a.weight, j) : 1.0f;
    __syncthreads();
    const T *x = static_cast<const T *>(a.x), *dy = static_cast<const T *>(a.dy);
    float aw[U][W], ab[U][W];
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
        for (int e = 0; e < W; ++e) aw[i][e] = ab[i][e] = 0.0f;

    Unit<T, W> ux[U], ud[U], nx[AHEAD ? U : 1], nd[AHEAD ? U : 1];
    auto fetch = [&](int64_t row, Unit<T, W> *px, Unit<T, W> *pd) {
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int j = (t + i * THREADS) * W;
            if (j < cols) {
                px[i].load(x + row * a.x_stride + j);
                pd[i].load(dy + row * a.dy_stride + j);
            } else {
                px[i].zero();
                pd[i].zero();
            }
        }
    };
    const int64_t step = (int64_t)blocks * ROWS;
    int64_t row = first + (int64_t)blockIdx.x * ROWS + sub;
    float mean = 0.0f, rstd = 0.0f;
    if (row < end) {
        fetch(row, ux, ud);
        mean = a.mean[row];
        rstd = a.rstd[row];
    }
    for (int flip = 0; row < end; row += step, flip ^= 1) {
        float nmean = 0.0f, nrstd = 0.0f;
        if (AHEAD && row + step < end) {
            fetch(row + step, nx, nd);
            nmean = a.mean[row + step];
            nrstd = a.rstd[row + step];
        }
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int j = (t + i * THREADS) * W;
            float fx[W], fd[W];
            ux[i].wide(fx);
            ud[i].wide(fd);
#pragma unroll
            for (int e = 0; e < W; ++e) {
                const float xh = (fx[e] - mean) * rstd, h = fd[e] * (j < cols ? wide_w[j + e] : 0.0f);
                s1 += h;
                s2 = fmaf(h, xh, s2);
                aw[i][e] = fmaf(fd[e], xh, aw[i][e]);
                ab[i][e] += fd[e];
            }
        }
        if (a.dx) {
            const float2 s = row_sum2<THREADS>(s1, s2, sh[flip]);
            const float c1 = s.x / (float)cols, c2 = s.y / (float)cols;
            T *dx = static_cast<T *>(a.dx) + row * a.dx_stride;
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const int j = (t + i * THREADS) * W;
                if (j < cols) {
                    float fx[W], fd[W];
                    ux[i].wide(fx);
                    ud[i].wide(fd);
#pragma unroll
                    for (int e = 0; e < W; ++e) {
                        const float xh = (fx[e] - mean) * rstd, h = fd[e] * wide_w[j + e];
                        fx[e] = rstd * (h - c1 - xh * c2);
                    }
                    Unit<T, W>::store(dx + j, fx);
                }
            }
        }
        if (AHEAD) {
#pragma unroll
            for (int i = 0; i < U; ++i) { ux[i] = nx[i]; ud[i] = nd[i]; }
            mean = nmean;
            rstd = nrstd;
        } else if (row + step < end) {
            fetch(row + step, ux, ud);
            mean = a.mean[row + step];
            rstd = a.rstd[row + step];
        }
    }
    grid_dep_launch();
    if (!a.dweight && !a.dbias) return;
    if (ROWS > 1) {
        float *sw = wide_w, *sb = wide_w + cols;
        for (int r = 0; r < ROWS; ++r) {
            __syncthreads();
            if (sub == r) {
#pragma unroll
                for (int i = 0; i < U; ++i)
#pragma unroll
                    for (int e = 0; e < W; ++e) {
                        const int j = (t + i * THREADS) * W + e;
                        if (j < cols) {
                            sw[j] = r == 0 ? aw[i][e] : sw[j] + aw[i][e];
                            sb[j] = r == 0 ? ab[i][e] : sb[j] + ab[i][e];
                        }
                    }
            }
        }
        __syncthreads();
        for (int j = threadIdx.x; j < cols; j += BT) leave_sums(a, blockIdx.y, blocks, j, sw[j], sb[j]);
    } else {
#pragma unroll
        for (int i = 0; i < U; ++i)
#pragma unroll
            for (int e = 0; e < W; ++e) {
                const int j = (t + i * THREADS) * W + e;
                if (j < cols) leave_sums(a, blockIdx.y, blocks, j, aw[i][e], ab[i][e]);
            }
    }
}

// The blocks' sums of a group, added in the order of the blocks: 32 columns a block, the 32 warps
// a share of the blocks each.
__global__ void __launch_bounds__(1024) k_norm_sums(NormBackward a, int blocks)
{
    __shared__ float sh[32][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t j = (int64_t)blockIdx.x * 32 + lane, n = 2 * a.cols;      // columns of dweight, then of dbias
    const float *p = a.parts + blockIdx.y * (int64_t)blocks * n + j;
    const int share = (blocks + 31) / 32, lo = warp * share, hi = min(blocks, lo + share);
    grid_dep_wait();
    float s = 0.0f;
    if (j < n)
#pragma unroll 8
        for (int b = lo; b < hi; ++b) s += __ldcg(p + b * n);
    sh[warp][lane] = s;
    __syncthreads();
    s = warp_sum(sh[lane][warp]);                       // column `warp` of the block's 32
    const int64_t c = (int64_t)blockIdx.x * 32 + warp;
    if (lane == 0 && c < n) {
        if (c < a.cols) {
            if (a.dweight) store_grad(a.dweight, blockIdx.y * a.dweight_stride + c, a.grad_type, a.accumulate, s);
        } else if (a.dbias) {
            store_grad(a.dbias, blockIdx.y * a.dbias_stride + c - a.cols, a.grad_type, a.accumulate, s);
        }
    }
}

// Rows too long for that: the sums over rows first (dx may overwrite what they read), then dx.
constexpr int kNormBlock = 256;

template <typename T>
__global__ void __launch_bounds__(kNormBlock) k_norm_dw(NormBackward a)
{
    __shared__ float sw[kNormBlock / 32][33], sb[kNormBlock / 32][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t j = (int64_t)blockIdx.x * 32 + lane, per = a.rows / a.groups, first = blockIdx.y * per;
    float w = 0.0f, b = 0.0f;
    if (j < a.cols)
        for (int64_t r = first + warp; r < first + per; r += kNormBlock / 32) {
            const float dy = widen(static_cast<const T *>(a.dy)[r * a.dy_stride + j]);
            const float x = widen(static_cast<const T *>(a.x)[r * a.x_stride + j]);
            w = fmaf(dy, (x - a.mean[r]) * a.rstd[r], w);
            b += dy;
        }
    sw[warp][lane] = w;
    sb[warp][lane] = b;
    __syncthreads();
    if (warp == 0 && j < a.cols) {
        w = b = 0.0f;
        for (int i = 0; i < kNormBlock / 32; ++i) { w += sw[i][lane]; b += sb[i][lane]; }
        leave_sums(a, blockIdx.y, 1, j, w, b);
    }
}

template <typename T>
__global__ void __launch_bounds__(kLongBlock) k_norm_dx(NormBackward a)
{
    __shared__ float2 sh[32];
    const int64_t row = blockIdx.x;
    const T *x = static_cast<const T *>(a.x) + row * a.x_stride;
    const T *dy = static_cast<const T *>(a.dy) + row * a.dy_stride;
    T *dx = static_cast<T *>(a.dx) + row * a.dx_stride;
    const float mean = a.mean[row], rstd = a.rstd[row];
    float s1 = 0.0f, s2 = 0.0f;
    for (int64_t j = threadIdx.x; j < a.cols; j += kLongBlock) {
        const float h = widen(dy[j]) * (a.weight.p ? any_at(a.weight, j) : 1.0f);
        s1 += h;
        s2 = fmaf(h, (widen(x[j]) - mean) * rstd, s2);
    }
    const float2 s = row_sum2<kLongBlock>(s1, s2, sh);
    const float c1 = s.x / (float)a.cols, c2 = s.y / (float)a.cols;
    for (int64_t j = threadIdx.x; j < a.cols; j += kLongBlock) {
        const float h = widen(dy[j]) * (a.weight.p ? any_at(a.weight, j) : 1.0f);
        const float xh = (widen(x[j]) - mean) * rstd;
        dx[j] = narrow<T>(rstd * (h - c1 - xh * c2));
    }
}

// ---------------------------------------------------------------------------------------------
// Launches
// ---------------------------------------------------------------------------------------------
constexpr int kSums = 2 * 148;          // blocks that leave sums, at most (two for each SM)

// Blocks that share a group's rows: as many as the GPU holds, no more than there are rows.
static int blocks_per_group(int64_t rows, int64_t groups)
{
    int64_t n = kSums / groups;
    if (n > rows / groups) n = rows / groups;
    return n < 1 ? 1 : (int)n;
}

int64_t layer_norm_workspace(int64_t rows, int64_t cols, int64_t groups)
{
    const int n = blocks_per_group(rows, groups);
    return n > 1 ? groups * n * cols * 8 : 0;
}

// Whether every row of a matrix starts on 16 bytes.
static bool aligned(const void *p, int64_t stride, int64_t rows, int size)
{
    return ((uintptr_t)p & 15) == 0 && (rows <= 1 || stride * size % 16 == 0);
}

template <typename T, int W, int U, int THREADS>
static bool try_forward(const NormForward &a, cudaStream_t st)
{
    if (a.cols > (int64_t)W * U * THREADS) return false;
    constexpr int block = kBlockOf<THREADS>, rows = block / THREADS;
    k_norm<T, W, U, THREADS><<<(unsigned)((a.rows + rows - 1) / rows), block, 0, st>>>(a);
    return true;
}

template <typename T>
static void forward(const NormForward &a, cudaStream_t st)
{
    constexpr int W = Vec<T>::n, F = 8 / W;             // binary32 needs twice the units
    if (a.cols % W == 0 && aligned(a.x, a.x_stride, a.rows, sizeof(T)) && aligned(a.y, a.y_stride, a.rows, sizeof(T))) {
        if (try_forward<T, W, 1 * F, 32>(a, st) || try_forward<T, W, 2 * F, 32>(a, st) || try_forward<T, W, 4 * F, 32>(a, st) ||
            try_forward<T, W, 2 * F, 128>(a, st) || try_forward<T, W, 4 * F, 128>(a, st) || try_forward<T, W, 4 * F, 256>(a, st) ||
            try_forward<T, W, 4 * F, 512>(a, st) || try_forward<T, W, 4 * F, 1024>(a, st))
            return;
    } else if (try_forward<T, 1, 8, 32>(a, st) || try_forward<T, 1, 32, 32>(a, st) || try_forward<T, 1, 16, 256>(a, st) ||
               try_forward<T, 1, 32, 256>(a, st) || try_forward<T, 1, 32, 1024>(a, st)) {
        return;
    }
    k_norm_long<T><<<(unsigned)a.rows, kLongBlock, 0, st>>>(a);
}

template <typename T, int W, int U, int THREADS>
static bool try_backward(const NormBackward &a, int blocks, cudaStream_t st)
{
    if (a.cols > (int64_t)W * U * THREADS) return false;
    constexpr int BT = kBlockOf<THREADS>;
    const int64_t per = a.rows / a.groups;
    if (blocks > (per + BT / THREADS - 1) / (BT / THREADS)) blocks = (int)((per + BT / THREADS - 1) / (BT / THREADS));
    if (blocks < 1) blocks = 1;
    const size_t smem = ((size_t)a.cols + 3) / 4 * 4 * 4 * (BT > THREADS ? 2 : 1);
    cudaFuncSetAttribute(k_norm_backward<T, W, U, THREADS>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    k_norm_backward<T, W, U, THREADS><<<dim3((unsigned)blocks, (unsigned)a.groups), BT, smem, st>>>(a, blocks);
    if (blocks > 1 && (a.dweight || a.dbias))
        launch_after(k_norm_sums, dim3((unsigned)((2 * a.cols + 31) / 32), (unsigned)a.groups), dim3(1024), 0, st, a, blocks);
    return true;
}

template <typename T>
static void backward(const NormBackward &a, cudaStream_t st)
{
    constexpr int W = Vec<T>::n, F = 8 / W;
    const int n = blocks_per_group(a.rows, a.groups);
    if (a.cols % W == 0 && aligned(a.x, a.x_stride, a.rows, sizeof(T)) && aligned(a.dy, a.dy_stride, a.rows, sizeof(T)) &&
        (!a.dx || aligned(a.dx, a.dx_stride, a.rows, sizeof(T)))) {
        if (try_backward<T, W, 1 * F, 32>(a, n, st) || try_backward<T, W, 3 * F, 32>(a, n, st) ||
            try_backward<T, W, 1 * F, 256>(a, n, st) || try_backward<T, W, 1 * F, 512>(a, n, st) ||
            try_backward<T, W, 2 * F, 512>(a, n, st) || try_backward<T, W, 4 * F, 512>(a, n, st))
            return;
    } else if (try_backward<T, 1, 8, 32>(a, n, st) || try_backward<T, 1, 4, 256>(a, n, st) || try_backward<T, 1, 8, 256>(a, n, st) ||
               try_backward<T, 1, 8, 512>(a, n, st) || try_backward<T, 1, 16, 512>(a, n, st)) {
        return;
    }
    if (a.dweight || a.dbias)
        k_norm_dw<T><<<dim3((unsigned)((a.cols + 31) / 32), (unsigned)a.groups), kNormBlock, 0, st>>>(a);
    if (a.dx && a.rows) k_norm_dx<T><<<(unsigned)a.rows, kLongBlock, 0, st>>>(a);
}

void launch_layer_norm(const NormForward &a, int type, cudaStream_t st)
{
    if (type == 0) forward<float>(a, st);
    else if (type == 1) forward<bf16>(a, st);
    else forward<f16>(a, st);
}

void launch_layer_norm_backward(const NormBackward &a, int type, cudaStream_t st)
{
    if (type == 0) backward<float>(a, st);
    else if (type == 1) backward<bf16>(a, st);
    else backward<f16>(a, st);
}

}  // namespace cdadam
