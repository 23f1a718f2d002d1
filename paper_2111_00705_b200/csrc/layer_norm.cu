// Layer norm, forward and backward.
//
// A row is held in registers: a group of threads has 8 or 16 elements of it each, loaded once,
// so mean, squared deviations and output come from one read.  Elements are loaded in units of W
// consecutive ones: 16 bytes where every row starts on a multiple of 16 bytes and is a whole
// number of units, else single elements.
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

// ---------------------------------------------------------------------------------------------
// THREADS threads of a block (whole warps) work on a row; a block of BT threads has BT / THREADS
// such groups.  Sums over a group: within warps by shuffles, then through shared memory behind a
// barrier of the group's own.  `slot` has to alternate from one sum of a group to the next.
// ---------------------------------------------------------------------------------------------
template <int THREADS>
__device__ __forceinline__ void group_barrier(int group)
{
    asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "n"(THREADS) : "memory");
}

template <int THREADS>
__device__ __forceinline__ float group_sum(float v, float *slot, int group)
{
    constexpr int N = THREADS / 32;
    v = warp_sum(v);
    if (N == 1) return v;
    const int lane = threadIdx.x & 31, warp = threadIdx.x / 32 % N;
    if (lane == 0) slot[warp] = v;
    group_barrier<THREADS>(group);
    if (N <= 4) {
        v = slot[0];
#pragma unroll
        for (int i = 1; i < N; ++i) v += slot[i];
        return v;
    }
    v = slot[lane % N];
#pragma unroll
    for (int d = N / 2; d >= 1; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}

// Two sums at once: after the first exchange the lower half of a warp carries one, the upper half
// the other.
template <int THREADS>
__device__ __forceinline__ float2 group_sum2(float a, float b, float2 *slot, int group)
{
    constexpr int N = THREADS / 32;
    const int lane = threadIdx.x & 31, warp = threadIdx.x / 32 % N;
    const bool upper = lane & 16;
    float v = (upper ? b : a) + __shfl_xor_sync(0xffffffffu, upper ? a : b, 16);
#pragma unroll
    for (int d = 8; d >= 1; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    if (N == 1) return make_float2(__shfl_sync(0xffffffffu, v, 0), __shfl_sync(0xffffffffu, v, 16));
    float *at = reinterpret_cast<float *>(slot);
    if ((lane & 15) == 0) at[2 * warp + (upper ? 1 : 0)] = v;
    group_barrier<THREADS>(group);
    if (N <= 4) {
        float2 s = slot[0];
#pragma unroll
        for (int i = 1; i < N; ++i) s = add2(s, slot[i]);
        return s;
    }
    v = at[2 * (lane % N) + (upper ? 1 : 0)];       // N is 8 or 16: both halves of the warp cover all warps
#pragma unroll
    for (int d = (N > 16 ? 16 : N) / 2; d >= 1; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return make_float2(__shfl_sync(0xffffffffu, v, 0), __shfl_sync(0xffffffffu, v, 16));
}

// What a thread holds of a row: U units of W elements, N = U W, as N / 2 pairs when widened.
template <typename T, int W, int U, int THREADS>
struct Held {
    static constexpr int N = U * W;
    Unit<T, W> u[U];
    __device__ __forceinline__ void load(const T *row, int t, int cols)
    {
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int j = (t + i * THREADS) * W;
            if (j < cols) u[i].load(row + j);
            else u[i].zero();
        }
    }
    __device__ __forceinline__ void wide(float2 (&f)[N / 2]) const
    {
#pragma unroll
        for (int i = 0; i < U; ++i) {
            float g[W];
            u[i].wide(g);
#pragma unroll
            for (int e = 0; e < W; ++e) (((i * W + e) & 1) ? f[(i * W + e) / 2].y : f[(i * W + e) / 2].x) = g[e];
        }
    }
    static __device__ __forceinline__ void store(T *row, int t, int cols, const float2 (&f)[N / 2])
    {
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int j = (t + i * THREADS) * W;
            if (j < cols) {
                float g[W];
#pragma unroll
                for (int e = 0; e < W; ++e) g[e] = ((i * W + e) & 1) ? f[(i * W + e) / 2].y : f[(i * W + e) / 2].x;
                Unit<T, W>::store(row + j, g);
            }
        }
    }
    static __device__ __forceinline__ void params(const AnyVec &v, int t, int cols, float absent, float2 (&f)[N / 2])
    {
        const bool wide4 = is_wide4(v);
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int j = (t + i * THREADS) * W;
            float g[W];
#pragma unroll
            for (int e = 0; e < W; ++e) g[e] = 0.0f;
            if (j < cols) parameters<W>(v, wide4, j, absent, g);
#pragma unroll
            for (int e = 0; e < W; ++e) (((i * W + e) & 1) ? f[(i * W + e) / 2].y : f[(i * W + e) / 2].x) = g[e];
        }
    }
    // whether pair p's elements are columns of the row (N / 2 pairs; both of a pair when W > 1)
    static __device__ __forceinline__ bool in(int i, int t, int cols) { return (t + i / W * THREADS) * W + i % W < cols; }
};

// ---------------------------------------------------------------------------------------------
// Forward.  Every group takes rows at a distance of all groups, the next row on its way while one
// is normalised.  KEEP: the parameters stay in registers (read for every row, 8 bytes of them
// beside 4 of data, they took most of the time: 20000 x 4096 bf16 82 us); rows of more than 8192
// columns leave no registers for them and for the next row.
// ---------------------------------------------------------------------------------------------
template <typename T, int W, int U, int THREADS, int BT, int PER_SM, bool KEEP>
__global__ void __launch_bounds__(BT, PER_SM) k_norm(NormForward a)
{
    typedef Held<T, W, U, THREADS> H;
    constexpr int N = H::N, GROUPS = BT / THREADS;
    constexpr bool AHEAD = KEEP;
    __shared__ float sh[GROUPS][2][THREADS / 32];
    const int t = threadIdx.x % THREADS, group = threadIdx.x / THREADS, cols = (int)a.cols;
    const int64_t step = (int64_t)gridDim.x * GROUPS;
    int64_t row = (int64_t)blockIdx.x * GROUPS + group;
    const T *x = static_cast<const T *>(a.x);
    H h, ahead;
    float2 w[KEEP ? N / 2 : 1], b[KEEP ? N / 2 : 1];
    if (row < a.rows) h.load(x + row * a.x_stride, t, cols);
    if constexpr (KEEP) {
        H::params(a.weight, t, cols, 1.0f, w);
        H::params(a.bias, t, cols, 0.0f, b);
    }
    const float over = 1.0f / (float)cols;
    for (; row < a.rows; row += step) {
        if (AHEAD && row + step < a.rows) ahead.load(x + (row + step) * a.x_stride, t, cols);
        float2 f[N / 2], s = both(0.0f);
        h.wide(f);
#pragma unroll
        for (int i = 0; i < N / 2; ++i) s = add2(s, f[i]);
        const float mean = group_sum<THREADS>(s.x + s.y, sh[group][0], group) * over;
        s = both(0.0f);
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            f[i] = add2(f[i], both(-mean));
            if (!H::in(2 * i, t, cols)) f[i].x = 0.0f;
            if (!H::in(2 * i + 1, t, cols)) f[i].y = 0.0f;
            s = fma2(f[i], f[i], s);
        }
        const float rstd = 1.0f / sqrtf(fmaf(group_sum<THREADS>(s.x + s.y, sh[group][1], group), over, a.eps));
        if constexpr (KEEP) {
#pragma unroll
            for (int i = 0; i < N / 2; ++i) f[i] = fma2(mul2(f[i], both(rstd)), w[i], b[i]);
        } else {
            float2 p[N / 2];
            H::params(a.weight, t, cols, 1.0f, p);
#pragma unroll
            for (int i = 0; i < N / 2; ++i) f[i] = mul2(mul2(f[i], both(rstd)), p[i]);
            H::params(a.bias, t, cols, 0.0f, p);
#pragma unroll
            for (int i = 0; i < N / 2; ++i) f[i] = add2(f[i], p[i]);
        }
        H::store(static_cast<T *>(a.y) + row * a.y_stride, t, cols, f);
        if (t == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
        if (AHEAD) h = ahead;
        else if (row + step < a.rows) h.load(x + (row + step) * a.x_stride, t, cols);
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

template <typename T, int W, int U, int THREADS, int BT, int PER_SM>
__global__ void __launch_bounds__(BT, PER_SM) k_norm_backward(NormBackward a, int blocks)
{
    typedef Held<T, W, U, THREADS> H;
    constexpr int N = H::N, GROUPS = BT / THREADS;
    extern __shared__ __align__(16) float sums[];       // GROUPS > 1: the block's sums, 2 x cols
    __shared__ float2 sh[GROUPS][2][THREADS / 32];
    const int t = threadIdx.x % THREADS, group = threadIdx.x / THREADS, cols = (int)a.cols;
    const int64_t per = a.rows / a.groups, first = blockIdx.y * per, end = first + per;
    const T *x = static_cast<const T *>(a.x), *dy = static_cast<const T *>(a.dy);
    float2 aw[N / 2], ab[N / 2], w[N / 2];
#pragma unroll
    for (int i = 0; i < N / 2; ++i) aw[i] = ab[i] = both(0.0f);

    H hx, hd, nx, nd;
    const int64_t step = (int64_t)blocks * GROUPS;
    int64_t row = first + (int64_t)blockIdx.x * GROUPS + group;
    float mean = 0.0f, rstd = 0.0f;
    auto fetch = [&](int64_t r, H &px, H &pd, float &m, float &s) {
        px.load(x + r * a.x_stride, t, cols);
        pd.load(dy + r * a.dy_stride, t, cols);
        m = a.mean[r];
        s = a.rstd[r];
    };
    if (row < end) fetch(row, hx, hd, mean, rstd);
    H::params(a.weight, t, cols, 1.0f, w);
    const float over = 1.0f / (float)cols;
    for (int flip = 0; row < end; row += step, flip ^= 1) {
        float nmean = 0.0f, nrstd = 0.0f;
        if (row + step < end) fetch(row + step, nx, nd, nmean, nrstd);
        float2 s1 = both(0.0f), s2 = both(0.0f), fx[N / 2], fd[N / 2];
        hx.wide(fx);
        hd.wide(fd);
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            const float2 xh = mul2(add2(fx[i], both(-mean)), both(rstd)), h = mul2(fd[i], w[i]);
            s1 = add2(s1, h);
            s2 = fma2(h, xh, s2);
            aw[i] = fma2(fd[i], xh, aw[i]);
            ab[i] = add2(ab[i], fd[i]);
        }
        if (a.dx) {
            const float2 s = group_sum2<THREADS>(s1.x + s1.y, s2.x + s2.y, sh[group][flip], group);
            const float2 c1 = both(-s.x * over), c2 = both(-s.y * over);
            hx.wide(fx);                                // widened again rather than kept: registers
            hd.wide(fd);
#pragma unroll
            for (int i = 0; i < N / 2; ++i) {
                const float2 xh = mul2(add2(fx[i], both(-mean)), both(rstd));
                const float2 h = fma2(fd[i], w[i], c1);
                fx[i] = mul2(fma2(xh, c2, h), both(rstd));
            }
            H::store(static_cast<T *>(a.dx) + row * a.dx_stride, t, cols, fx);
        }
        hx = nx;
        hd = nd;
        mean = nmean;
        rstd = nrstd;
    }
    grid_dep_launch();
    if (!a.dweight && !a.dbias) return;
    if (GROUPS > 1) {
        for (int r = 0; r < GROUPS; ++r) {
            __syncthreads();
            if (group == r) {
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const int j = (t + i / W * THREADS) * W + i % W;
                    if (j < cols) {
                        const float vw = i & 1 ? aw[i / 2].y : aw[i / 2].x, vb = i & 1 ? ab[i / 2].y : ab[i / 2].x;
                        sums[j] = r == 0 ? vw : sums[j] + vw;
                        sums[cols + j] = r == 0 ? vb : sums[cols + j] + vb;
                    }
                }
            }
        }
        __syncthreads();
        for (int j = threadIdx.x; j < cols; j += BT) leave_sums(a, blockIdx.y, blocks, j, sums[j], sums[cols + j]);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int j = (t + i / W * THREADS) * W + i % W;
            if (j < cols)
                leave_sums(a, blockIdx.y, blocks, j, i & 1 ? aw[i / 2].y : aw[i / 2].x, i & 1 ? ab[i / 2].y : ab[i / 2].x);
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
    __shared__ float sh[2][32];
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
    const float c1 = block_sum_all<kLongBlock>(s1, sh[0]) / (float)a.cols, c2 = block_sum_all<kLongBlock>(s2, sh[1]) / (float)a.cols;
    for (int64_t j = threadIdx.x; j < a.cols; j += kLongBlock) {
        const float h = widen(dy[j]) * (a.weight.p ? any_at(a.weight, j) : 1.0f);
        const float xh = (widen(x[j]) - mean) * rstd;
        dx[j] = narrow<T>(rstd * (h - c1 - xh * c2));
    }
}

// ---------------------------------------------------------------------------------------------
// Launches
// ---------------------------------------------------------------------------------------------
constexpr int kSMs = 148;
constexpr int kSums = 2 * kSMs;         // blocks that leave sums, at most (two for each SM)

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

template <typename T, int W, int U, int THREADS, int BT, int PER_SM, bool KEEP = true>
static bool try_forward(const NormForward &a, cudaStream_t st)
{
    if (a.cols > (int64_t)W * U * THREADS) return false;
    constexpr int groups = BT / THREADS;
    int64_t blocks = (a.rows + groups - 1) / groups;
    if (blocks > kSMs * PER_SM) blocks = kSMs * PER_SM;
    k_norm<T, W, U, THREADS, BT, PER_SM, KEEP><<<(unsigned)blocks, BT, 0, st>>>(a);
    return true;
}

template <typename T>
static void forward(const NormForward &a, cudaStream_t st)
{
    constexpr int W = Vec<T>::n, F = 8 / W;             // binary32 needs twice the units
    if (a.cols % W == 0 && aligned(a.x, a.x_stride, a.rows, sizeof(T)) && aligned(a.y, a.y_stride, a.rows, sizeof(T))) {
        if (try_forward<T, W, 1 * F, 32, 512, 2>(a, st) || try_forward<T, W, 1 * F, 64, 512, 2>(a, st) ||
            try_forward<T, W, 1 * F, 96, 480, 2>(a, st) || try_forward<T, W, 1 * F, 128, 512, 2>(a, st) ||
            try_forward<T, W, 1 * F, 256, 512, 2>(a, st) || try_forward<T, W, 1 * F, 512, 512, 2>(a, st) ||
            try_forward<T, W, 2 * F, 512, 512, 1>(a, st) || try_forward<T, W, 2 * F, 1024, 1024, 1, false>(a, st))
            return;
    } else if (try_forward<T, 1, 8, 32, 512, 2>(a, st) || try_forward<T, 1, 16, 32, 256, 2>(a, st) ||
               try_forward<T, 1, 16, 64, 256, 2>(a, st) || try_forward<T, 1, 16, 128, 256, 2>(a, st) ||
               try_forward<T, 1, 16, 256, 256, 2>(a, st) || try_forward<T, 1, 16, 512, 512, 1>(a, st) ||
               try_forward<T, 1, 16, 1024, 1024, 1, false>(a, st)) {
        return;
    }
    k_norm_long<T><<<(unsigned)a.rows, kLongBlock, 0, st>>>(a);
}

template <typename T, int W, int U, int THREADS, int BT, int PER_SM>
static bool try_backward(const NormBackward &a, int blocks, cudaStream_t st)
{
    if (a.cols > (int64_t)W * U * THREADS) return false;
    constexpr int groups = BT / THREADS;
    const int64_t per = a.rows / a.groups, most = (per + groups - 1) / groups;
    if (PER_SM == 1 && blocks > 1) blocks = (blocks + 1) / 2;
    if (blocks > most) blocks = (int)most;
    if (blocks < 1) blocks = 1;
    const size_t smem = groups > 1 ? (size_t)a.cols * 8 : 0;
    auto *kernel = k_norm_backward<T, W, U, THREADS, BT, PER_SM>;
    kernel<<<dim3((unsigned)blocks, (unsigned)a.groups), BT, smem, st>>>(a, blocks);
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
        if (try_backward<T, W, 1 * F, 32, 512, 2>(a, n, st) || try_backward<T, W, 1 * F, 64, 512, 2>(a, n, st) ||
            try_backward<T, W, 1 * F, 96, 480, 2>(a, n, st) || try_backward<T, W, 1 * F, 128, 512, 2>(a, n, st) ||
            try_backward<T, W, 1 * F, 256, 512, 2>(a, n, st) || try_backward<T, W, 1 * F, 512, 512, 2>(a, n, st) ||
            try_backward<T, W, 2 * F, 512, 512, 1>(a, n, st))
            return;
    } else if (try_backward<T, 1, 8, 32, 256, 2>(a, n, st) || try_backward<T, 1, 16, 32, 256, 2>(a, n, st) ||
               try_backward<T, 1, 16, 64, 256, 2>(a, n, st) || try_backward<T, 1, 16, 128, 256, 2>(a, n, st) ||
               try_backward<T, 1, 16, 256, 256, 2>(a, n, st) || try_backward<T, 1, 16, 512, 512, 1>(a, n, st)) {
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
