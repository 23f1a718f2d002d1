// Root-mean-square norm with the residual's addition, its gradient, and the 8-bit formats of rows.
//
// All are bound by memory: every matrix is read once and written once.  A group of 32 to 512 threads
// takes a row at a time, every thread up to four units of eight columns, and asks for its next row's units
// before it works on the present ones.
#include "eight_bits.cuh"

namespace cdadam {

constexpr int kSms = 148;

// Sum and maximum over a group's threads; `slot` alternates from one row to the next.
template <int THREADS>
__device__ __forceinline__ void group_wait(int group)
{
    if (THREADS > 32) asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "n"(THREADS) : "memory");
}
template <int THREADS>
__device__ __forceinline__ void group_sum_max(float &sum, uint32_t &top, float2 *slot, int group)
{
    constexpr int N = THREADS / 32;
    sum = warp_sum(sum);
    top = __reduce_max_sync(0xffffffffu, top);
    if (N == 1) return;
    if ((threadIdx.x & 31) == 0) slot[threadIdx.x / 32 % N] = make_float2(sum, __uint_as_float(top));
    group_wait<THREADS>(group);
    float2 v = slot[0];
    sum = v.x;
    top = __float_as_uint(v.y);
#pragma unroll
    for (int i = 1; i < N; ++i) {
        v = slot[i];
        sum += v.x;
        top = max(top, __float_as_uint(v.y));
    }
}
template <int THREADS>
__device__ __forceinline__ float group_sum(float sum, float *slot, int group)
{
    constexpr int N = THREADS / 32;
    sum = warp_sum(sum);
    if (N == 1) return sum;
    if ((threadIdx.x & 31) == 0) slot[threadIdx.x / 32 % N] = sum;
    group_wait<THREADS>(group);
    sum = slot[0];
#pragma unroll
    for (int i = 1; i < N; ++i) sum += slot[i];
    return sum;
}

// 1 / sqrt(v): the approximation and one Newton step, within 1 ulp or so; 0 gives infinity, infinity 0.
__device__ __forceinline__ float inverse_root(float v)
{
    const float r = rsqrtf(v);
    return r > 0.0f && r < 3e38f ? __fmul_rn(r, fmaf(__fmul_rn(__fmul_rn(-0.5f, r), v), r, 1.5f)) : r;
}

// The weight, widened, in shared memory, 0 beyond the row: columns 0 .. 3 of the units in one plane, 4 .. 7
// in another, so that a warp's 16-byte reads are adjacent.
__device__ __forceinline__ void fill_weight(float *w, const AnyVec &v, int cols, int units)
{
    for (int j = threadIdx.x; j < 8 * units; j += blockDim.x)
        w[(j & 4 ? 4 * units : 0) + (j >> 3) * 4 + (j & 3)] = j >= cols ? 0.0f : v.p ? any_at(v, j) : 1.0f;
}
__device__ __forceinline__ void weight8(const float *w, int u, int units, float (&f)[8])
{
    const float4 a = *reinterpret_cast<const float4 *>(w + 4 * u), b = *reinterpret_cast<const float4 *>(w + 4 * (units + u));
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
    f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
}

template <typename T>
__device__ __forceinline__ T *row_of(const Matrix &m, int64_t r) { return static_cast<T *>(m.p) + r * m.stride; }

// h of a unit: x, or the sum with the residual as the activations' type holds it.
template <typename T>
__device__ __forceinline__ void add_residual(float (&f)[8], const Raw8<T> &r)
{
    float g[8];
    widen8<T>(r, g);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = widen(narrow<T>(__fadd_rn(f[e], g[e])));
}

// A block of 32 columns of a checkpoint: four neighbouring threads' units.
template <typename T>
__device__ __forceinline__ void keep8(const Kept8 &k, int64_t row, int64_t j, int64_t cols, const float (&f)[8], bool vec)
{
    uint32_t m = magnitude8(f);
    m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
    m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
    const uint32_t e = kept_exponent(m);
    store_bytes(k.p + row * k.stride, j, cols, vec, to_kept8(f, e));
    if ((threadIdx.x & 3) == 0 && j < cols) k.exponents[row * k.exponents_stride + (j >> 5)] = (uint8_t)e;
}

// What follows from a row's statistics.
struct RowStats {
    float s;
    Step step;
    bool finite;
    __device__ __forceinline__ float scale() const
    {
        return finite ? __fmul_rn(__fdiv_rn(step.m, 127.0f), s) : __uint_as_float(0x7fc00000u);
    }
};
__device__ __forceinline__ RowStats stats_of(const RmsNorm &a, float squares, uint32_t top)
{
    RowStats r;
    r.s = a.normalise ? inverse_root(__fadd_rn(__fmul_rn(squares, __frcp_rn((float)a.cols)), a.eps)) : 1.0f;
    r.step = step_of(top);
    r.finite = top < kInfBits;
    return r;
}
template <typename T, bool VEC>
__device__ __forceinline__ void finish8(const RmsNorm &a, const RowStats &st, int64_t row, int64_t j, const float (&p)[8], bool q_vec)
{
    if (a.y.p) {
        float f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = __fmul_rn(p[e], st.s);
        store8<T, VEC>(row_of<T>(a.y, row), j, a.cols, narrow8<T>(f));
    }
    if (a.q.p) store_bytes(a.q.p + row * a.q.stride, j, a.cols, q_vec, st.finite ? to_rows8(p, st.step) : make_uint2(0, 0));
}

// ---------------------------------------------------------------------------------------------
// Forward.
// ---------------------------------------------------------------------------------------------
template <typename T, int THREADS, int STEPS, int BT, bool VEC>
__global__ void __launch_bounds__(BT, BT == 256 ? 2 : 1) k_rms_norm(RmsNorm a)
{
    constexpr int GROUPS = BT / THREADS, UNITS = THREADS * STEPS;
    constexpr bool AHEAD = STEPS * sizeof(T) < 16;       // the next row's units fit into the registers
    extern __shared__ __align__(16) float w[];
    __shared__ float2 slots[GROUPS][2][THREADS / 32];
    const int t = threadIdx.x % THREADS, group = threadIdx.x / THREADS, cols = (int)a.cols;
    const int64_t step = (int64_t)gridDim.x * GROUPS;
    const bool q_vec = on(a.q.p, a.q.stride, 8), kept_vec = on(a.kept.p, a.kept.stride, 8);
    int64_t row = (int64_t)blockIdx.x * GROUPS + group;
    Raw8<T> x[STEPS], r[STEPS];
    auto fetch = [&](int64_t n) {
#pragma unroll
        for (int k = 0; k < STEPS; ++k) x[k] = load8<T, VEC>(row_of<T>(a.x, n), 8 * (t + k * THREADS), cols);
        if (a.residual.p)
#pragma unroll
            for (int k = 0; k < STEPS; ++k) r[k] = load8<T, VEC>(row_of<T>(a.residual, n), 8 * (t + k * THREADS), cols);
    };
    if (AHEAD && row < a.rows) fetch(row);
    fill_weight(w, a.weight, cols, UNITS);
    __syncthreads();
    for (int slot = 0; row < a.rows; row += step, slot ^= 1) {
        float p[STEPS][8], squares = 0.0f;
        uint32_t top = 0;
        if (!AHEAD) fetch(row);
#pragma unroll
        for (int k = 0; k < STEPS; ++k) {
            widen8<T>(x[k], p[k]);
            if (a.residual.p) add_residual<T>(p[k], r[k]);
        }
        if (AHEAD && row + step < a.rows) fetch(row + step);
#pragma unroll
        for (int k = 0; k < STEPS; ++k) {
            const int u = t + k * THREADS;
            if (a.total.p) store8<T, VEC>(row_of<T>(a.total, row), 8 * u, cols, narrow8<T>(p[k]));
            if (a.kept.p) keep8<T>(a.kept, row, 8 * u, cols, p[k], kept_vec);
            float f[8];
            weight8(w, u, UNITS, f);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                squares = fmaf(p[k][e], p[k][e], squares);
                p[k][e] = __fmul_rn(p[k][e], f[e]);
            }
            if (a.q.p) top = max(top, magnitude8(p[k]));
        }
        group_sum_max<THREADS>(squares, top, slots[group][slot], group);
        const RowStats st = stats_of(a, squares, top);
#pragma unroll
        for (int k = 0; k < STEPS; ++k) finish8<T, VEC>(a, st, row, 8 * (t + k * THREADS), p[k], q_vec);
        if (t == 0) {
            if (a.rstd) a.rstd[row] = st.s;
            if (a.q.scale) a.q.scale[row] = st.scale();
        }
    }
}

// Rows too long for the registers of a block: read twice, the second time from the caches.
constexpr int kLongThreads = 1024;

__device__ __forceinline__ void weight8_long(const AnyVec &v, int64_t j, int64_t cols, float (&f)[8])
{
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = j + e >= cols ? 0.0f : v.p ? any_at(v, j + e) : 1.0f;
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(kLongThreads, 1) k_rms_norm_long(RmsNorm a)
{
    __shared__ float2 slots[kLongThreads / 32];
    const int64_t row = blockIdx.x, cols = a.cols;
    const bool q_vec = on(a.q.p, a.q.stride, 8), kept_vec = on(a.kept.p, a.kept.stride, 8);
    float f[8], w[8], squares = 0.0f;
    uint32_t top = 0;
    for (int64_t base = 0; base < cols; base += 8 * kLongThreads) {
        const int64_t j = base + 8 * threadIdx.x;
        widen8<T>(load8<T, VEC>(row_of<T>(a.x, row), j, cols), f);
        if (a.residual.p) add_residual<T>(f, load8<T, VEC>(row_of<T>(a.residual, row), j, cols));
        if (a.total.p) store8<T, VEC>(row_of<T>(a.total, row), j, cols, narrow8<T>(f));
        if (a.kept.p) keep8<T>(a.kept, row, j, cols, f, kept_vec);
        weight8_long(a.weight, j, cols, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            squares = fmaf(f[e], f[e], squares);
            w[e] = __fmul_rn(f[e], w[e]);
        }
        top = max(top, magnitude8(w));
    }
    group_sum_max<kLongThreads>(squares, top, slots, 0);
    const RowStats st = stats_of(a, squares, top);
    if (threadIdx.x == 0) {
        if (a.rstd) a.rstd[row] = st.s;
        if (a.q.scale) a.q.scale[row] = st.scale();
    }
    if (!a.y.p && !a.q.p) return;
    for (int64_t j = 8 * threadIdx.x; j < cols; j += 8 * kLongThreads) {
        if (a.total.p) {                                // may have been written over x
            widen8<T>(load8<T, VEC>(row_of<T>(a.total, row), j, cols), f);
        } else {
            widen8<T>(load8<T, VEC>(row_of<T>(a.x, row), j, cols), f);
            if (a.residual.p) add_residual<T>(f, load8<T, VEC>(row_of<T>(a.residual, row), j, cols));
        }
        weight8_long(a.weight, j, cols, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = __fmul_rn(f[e], w[e]);
        finish8<T, VEC>(a, st, row, j, w, q_vec);
    }
}

// ---------------------------------------------------------------------------------------------
// Backward.  A block works on rows of one group of rows, and every thread keeps the sums over rows of
// its own columns in registers, so everything is read once.  `parts` blocks share a group; with more than one each
// leaves its sums in the workspace and k_rms_sums adds them in order: the same bits every time.
// ---------------------------------------------------------------------------------------------
__device__ __forceinline__ void store_gradient(void *p, int64_t i, int type, int accumulate, float v)
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

// A unit of the activations, as they were or as a checkpoint.
template <typename T, bool KEPT> struct Source {
    Raw8<T> u;
    __device__ __forceinline__ void load(const RmsNormBackward &a, int64_t row, int64_t j, int64_t cols, bool)
    {
        u = load8<T, false>(row_of<T>(a.x, row), j, cols);
    }
    __device__ __forceinline__ void load_vec(const RmsNormBackward &a, int64_t row, int64_t j, int64_t cols, bool)
    {
        u = load8<T, true>(row_of<T>(a.x, row), j, cols);
    }
    __device__ __forceinline__ void values(float s, float (&f)[8]) const
    {
        widen8<T>(u, f);
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = __fmul_rn(f[e], s);
    }
};
template <typename T> struct Source<T, true> {
    uint2 u;
    uint32_t exponent;
    __device__ __forceinline__ void load(const RmsNormBackward &a, int64_t row, int64_t j, int64_t cols, bool vec)
    {
        u = load_bytes(a.kept.p + row * a.kept.stride, j, cols, vec);
        exponent = j < cols ? __ldg(a.kept.exponents + row * a.kept.exponents_stride + (j >> 5)) : 1;
    }
    __device__ __forceinline__ void load_vec(const RmsNormBackward &a, int64_t row, int64_t j, int64_t cols, bool vec)
    {
        load(a, row, j, cols, vec);
    }
    __device__ __forceinline__ void values(float s, float (&f)[8]) const
    {
        const float step = kept_step(exponent);
        unpack_bytes(u, f);
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = __fmul_rn(__fmul_rn(f[e], step), s);
    }
};

template <typename T, int THREADS, int STEPS, int BT, bool VEC, bool KEPT>
__global__ void __launch_bounds__(BT, BT == 256 ? 2 : 1) k_rms_norm_backward(RmsNormBackward a)
{
    constexpr int GROUPS = BT / THREADS, UNITS = THREADS * STEPS;
    extern __shared__ __align__(16) float w[];          // the weight; at the end the groups' sums
    __shared__ float slots[GROUPS][2][THREADS / 32];
    const int t = threadIdx.x % THREADS, group = threadIdx.x / THREADS, cols = (int)a.cols;
    const int64_t per = a.rows / a.groups, end = (blockIdx.y + 1) * per, step = (int64_t)gridDim.x * GROUPS;
    const bool vec = KEPT && on(a.kept.p, a.kept.stride, 8);
    const float over = __frcp_rn((float)cols);
    int64_t row = blockIdx.y * per + (int64_t)blockIdx.x * GROUPS + group;
    Raw8<T> dy[STEPS];
    Source<T, KEPT> x[STEPS];
    float rstd = 0.0f;
    auto fetch = [&](int64_t n) {
        rstd = __ldg(a.rstd + n);
#pragma unroll
        for (int k = 0; k < STEPS; ++k) {
            const int j = 8 * (t + k * THREADS);
            dy[k] = load8<T, VEC>(row_of<T>(a.dy, n), j, cols);
            if (VEC) x[k].load_vec(a, n, j, cols, vec); else x[k].load(a, n, j, cols, vec);
        }
    };
    if (row < end) fetch(row);
    fill_weight(w, a.weight, cols, UNITS);
    __syncthreads();
    float sums[STEPS][8];
#pragma unroll
    for (int k = 0; k < STEPS; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) sums[k][e] = 0.0f;
    for (int slot = 0; row < end; row += step, slot ^= 1) {
        float dot = 0.0f;
        const float s = rstd;
        Raw8<T> dy_now[STEPS], more[STEPS];
        Source<T, KEPT> x_now[STEPS];
#pragma unroll
        for (int k = 0; k < STEPS; ++k) {
            dy_now[k] = dy[k];
            x_now[k] = x[k];
        }
        if (a.dtotal.p)
#pragma unroll
            for (int k = 0; k < STEPS; ++k) more[k] = load8<T, VEC>(row_of<T>(a.dtotal, row), 8 * (t + k * THREADS), cols);
        if (row + step < end) fetch(row + step);
#pragma unroll
        for (int k = 0; k < STEPS; ++k) {
            float g[8], xh[8], f[8];
            x_now[k].values(s, xh);
            widen8<T>(dy_now[k], g);
            weight8(w, t + k * THREADS, UNITS, f);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                sums[k][e] = fmaf(g[e], xh[e], sums[k][e]);
                dot = fmaf(__fmul_rn(g[e], f[e]), xh[e], dot);
            }
        }
        if (!a.dx.p) continue;
        const float mean = __fmul_rn(group_sum<THREADS>(dot, slots[group][slot], group), over);
#pragma unroll
        for (int k = 0; k < STEPS; ++k) {
            float g[8], xh[8], f[8];
            x_now[k].values(s, xh);
            widen8<T>(dy_now[k], g);
            weight8(w, t + k * THREADS, UNITS, f);
#pragma unroll
            for (int e = 0; e < 8; ++e) g[e] = fmaf(-xh[e], mean, __fmul_rn(g[e], f[e]));
            if (a.dtotal.p) widen8<T>(more[k], f);
#pragma unroll
            for (int e = 0; e < 8; ++e) g[e] = a.dtotal.p ? fmaf(g[e], s, f[e]) : __fmul_rn(g[e], s);
            store8<T, VEC>(row_of<T>(a.dx, row), 8 * (t + k * THREADS), cols, narrow8<T>(g));
        }
    }
    if (!a.dweight) return;
    // the groups' sums one after the other, as planes
    for (int i = 0; i < GROUPS; ++i) {
        __syncthreads();
        if (i == group)
#pragma unroll
            for (int k = 0; k < STEPS; ++k)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float4 *p = reinterpret_cast<float4 *>(w + 4 * (h * UNITS + t + k * THREADS));
                    float4 v = i ? *p : make_float4(0, 0, 0, 0);
                    v.x += sums[k][4 * h]; v.y += sums[k][4 * h + 1]; v.z += sums[k][4 * h + 2]; v.w += sums[k][4 * h + 3];
                    *p = v;
                }
    }
    __syncthreads();
    for (int j = threadIdx.x; j < cols; j += BT) {
        const float v = w[(j & 4 ? 4 * UNITS : 0) + (j >> 3) * 4 + (j & 3)];
        if (gridDim.x > 1) a.parts[((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * cols + j] = v;
        else store_gradient(a.dweight, blockIdx.y * a.dweight_stride + j, a.grad_type, a.accumulate, v);
    }
}

// Rows too long for a block's registers: dx a row at a time, read twice; the weight's gradient column by column.
template <typename T, bool VEC, bool KEPT>
__global__ void __launch_bounds__(kLongThreads, 1) k_rms_dx_long(RmsNormBackward a)
{
    __shared__ float slots[kLongThreads / 32];
    const int64_t row = blockIdx.x, cols = a.cols;
    const bool vec = KEPT && on(a.kept.p, a.kept.stride, 8);
    const float s = a.rstd[row];
    Source<T, KEPT> x;
    float g[8], xh[8], w[8], dot = 0.0f;
    auto take = [&](int64_t j) {
        if (VEC) x.load_vec(a, row, j, cols, vec); else x.load(a, row, j, cols, vec);
        x.values(s, xh);
        widen8<T>(load8<T, VEC>(row_of<T>(a.dy, row), j, cols), g);
        weight8_long(a.weight, j, cols, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) g[e] = __fmul_rn(g[e], w[e]);
    };
    for (int64_t j = 8 * threadIdx.x; j < cols; j += 8 * kLongThreads) {
        take(j);
#pragma unroll
        for (int e = 0; e < 8; ++e) dot = fmaf(g[e], xh[e], dot);
    }
    const float mean = __fmul_rn(group_sum<kLongThreads>(dot, slots, 0), __frcp_rn((float)cols));
    for (int64_t j = 8 * threadIdx.x; j < cols; j += 8 * kLongThreads) {
        take(j);
        if (a.dtotal.p) widen8<T>(load8<T, VEC>(row_of<T>(a.dtotal, row), j, cols), w);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float d = fmaf(-xh[e], mean, g[e]);
            g[e] = a.dtotal.p ? fmaf(d, s, w[e]) : __fmul_rn(d, s);
        }
        store8<T, VEC>(row_of<T>(a.dx, row), j, cols, narrow8<T>(g));
    }
}
constexpr int kLongRows = 128;         // rows of a block of the next kernel, at least
template <typename T, bool VEC, bool KEPT>
__global__ void __launch_bounds__(128) k_rms_dw_long(RmsNormBackward a)
{
    const int64_t per = a.rows / a.groups, cols = a.cols, j = 8 * ((int64_t)blockIdx.x * 128 + threadIdx.x);
    const int parts = gridDim.y, part = blockIdx.y;
    const int64_t first = blockIdx.z * per + per * part / parts, end = blockIdx.z * per + per * (part + 1) / parts;
    const bool vec = KEPT && on(a.kept.p, a.kept.stride, 8);
    float sums[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (j >= cols) return;
#pragma unroll 4
    for (int64_t row = first; row < end; ++row) {
        Source<T, KEPT> x;
        float g[8], xh[8];
        if (VEC) x.load_vec(a, row, j, cols, vec); else x.load(a, row, j, cols, vec);
        widen8<T>(load8<T, VEC>(row_of<T>(a.dy, row), j, cols), g);
        x.values(__ldg(a.rstd + row), xh);
#pragma unroll
        for (int e = 0; e < 8; ++e) sums[e] = fmaf(g[e], xh[e], sums[e]);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if (j + e >= cols) break;
        if (parts > 1) a.parts[((int64_t)blockIdx.z * parts + part) * cols + j + e] = sums[e];
        else store_gradient(a.dweight, blockIdx.z * a.dweight_stride + j + e, a.grad_type, a.accumulate, sums[e]);
    }
}

// Sums of a group's parts, in a fixed order: 32 columns a block, a warp every 32nd part, then the warps in turn.
__global__ void __launch_bounds__(1024) k_rms_sums(RmsNormBackward a, int parts)
{
    __shared__ float sh[32][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t j = (int64_t)blockIdx.x * 32 + lane;
    float v = 0.0f;
    grid_dep_wait();
    if (j < a.cols)
#pragma unroll 4
        for (int i = warp; i < parts; i += 32) v += __ldcg(a.parts + ((int64_t)blockIdx.y * parts + i) * a.cols + j);
    sh[warp][lane] = v;
    __syncthreads();
    v = warp_sum(sh[lane][warp]);                       // column `warp` of the block
    if (lane == 0 && (int64_t)blockIdx.x * 32 + warp < a.cols)
        store_gradient(a.dweight, blockIdx.y * a.dweight_stride + (int64_t)blockIdx.x * 32 + warp, a.grad_type, a.accumulate, v);
}

// ---------------------------------------------------------------------------------------------
// The formats by themselves, unit by unit.  Rows are padded to whole blocks of four units, so that a
// checkpoint's block is four neighbouring threads.
// ---------------------------------------------------------------------------------------------
constexpr int kFlat = 256;

template <typename T, bool VEC>
__global__ void __launch_bounds__(kFlat) k_checkpoint8(Matrix x, Kept8 kept, int64_t rows, int64_t cols)
{
    const unsigned units = (unsigned)((cols + 31) / 32 * 4);
    const bool vec = on(kept.p, kept.stride, 8);
    const int64_t all = rows * units;
    for (int64_t base = (int64_t)blockIdx.x * kFlat; base < all; base += (int64_t)gridDim.x * kFlat) {
        const int64_t i = base + threadIdx.x;
        const int64_t row = i < all ? (all >> 32 ? i / units : (unsigned)i / units) : rows - 1, j = i < all ? 8 * (i - row * units) : cols;
        float f[8];
        widen8<T>(load8<T, VEC>(row_of<T>(x, row), j, cols), f);
        keep8<T>(kept, row, j, cols, f, vec);
    }
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(kFlat) k_restore8(Rows8 q, Kept8 kept, Matrix to, int64_t rows, int64_t cols)
{
    const unsigned units = (unsigned)((cols + 7) / 8);
    const int8_t *p = kept.p ? kept.p : q.p;
    const int64_t stride = kept.p ? kept.stride : q.stride, all = rows * units;
    const bool vec = on(p, stride, 8);
    for (int64_t i = (int64_t)blockIdx.x * kFlat + threadIdx.x; i < all; i += (int64_t)gridDim.x * kFlat) {
        const int64_t row = all >> 32 ? i / units : (unsigned)i / units, j = 8 * (i - row * units);
        float f[8];
        const uint2 b = load_bytes(p + row * stride, j, cols, vec);
        const float s = kept.p ? kept_step(__ldg(kept.exponents + row * kept.exponents_stride + (j >> 5))) : __ldg(q.scale + row);
        unpack_bytes(b, f);
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = __fmul_rn(f[e], s);
        store8<T, VEC>(row_of<T>(to, row), j, cols, narrow8<T>(f));
    }
}

// ---------------------------------------------------------------------------------------------
// Launches
// ---------------------------------------------------------------------------------------------
static bool starts_on_16(const Matrix &m, int64_t rows, int size)
{
    return !m.p || (((uintptr_t)m.p & 15) == 0 && (rows <= 1 || (m.stride * size & 15) == 0));
}

template <typename T, int THREADS, int STEPS, int BT>
static void forward_as(const RmsNorm &a, bool vec, cudaStream_t st)
{
    auto kernel = vec ? k_rms_norm<T, THREADS, STEPS, BT, true> : k_rms_norm<T, THREADS, STEPS, BT, false>;
    const int64_t groups = BT / THREADS, need = (a.rows + groups - 1) / groups, most = kSms * (BT == 256 ? 4 : BT == 512 ? 2 : 1);
    const size_t smem = (size_t)THREADS * STEPS * 32;
    allow_shared(kernel, smem);
    queue(kernel, dim3((unsigned)(need < most ? need : most)), BT, smem, st, a);
}
template <typename T>
static void forward(const RmsNorm &a, cudaStream_t st)
{
    const int size = sizeof(T);
    const bool vec = starts_on_16(a.x, a.rows, size) && starts_on_16(a.residual, a.rows, size) && starts_on_16(a.total, a.rows, size) &&
                     starts_on_16(a.y, a.rows, size);
    const int64_t units = (a.cols + 7) / 8;
    if (units <= 32) forward_as<T, 32, 1, 256>(a, vec, st);
    else if (units <= 64) forward_as<T, 32, 2, 256>(a, vec, st);
    else if (units <= 96) forward_as<T, 32, 3, 256>(a, vec, st);
    else if (units <= 128) forward_as<T, 32, 4, 256>(a, vec, st);
    else if (units <= 192) forward_as<T, 64, 3, 256>(a, vec, st);
    else if (units <= 256) forward_as<T, 64, 4, 256>(a, vec, st);
    else if (units <= 384) forward_as<T, 128, 3, 256>(a, vec, st);
    else if (units <= 512) forward_as<T, 128, 4, 256>(a, vec, st);
    else if (units <= 768) forward_as<T, 256, 3, 256>(a, vec, st);
    else if (units <= 1024) forward_as<T, 256, 4, 256>(a, vec, st);
    else if (units <= 1536) forward_as<T, 512, 3, 512>(a, vec, st);
    else if (units <= 2048) forward_as<T, 512, 4, 512>(a, vec, st);
    else queue(vec ? k_rms_norm_long<T, true> : k_rms_norm_long<T, false>, dim3((unsigned)a.rows), kLongThreads, 0, st, a);
}
void launch_rms_norm(const RmsNorm &a, int type, cudaStream_t st)
{
    if (type == 0) forward<float>(a, st);
    else if (type == 1) forward<bf16>(a, st);
    else forward<f16>(a, st);
}

// Threads that take a row together (0: too long for them), and blocks that share a group of rows.
static int backward_threads(int64_t cols)
{
    const int64_t units = (cols + 7) / 8;
    return units <= 64 ? 32 : units <= 128 ? 64 : units <= 256 ? 128 : units <= 512 ? 256 : units <= 1024 ? 512 : 0;
}
static int backward_block(int threads) { return threads > 256 ? threads : 256; }
static int64_t backward_parts(int64_t rows, int64_t cols, int64_t groups)
{
    const int64_t per = rows / groups;
    const int threads = backward_threads(cols);
    int64_t most, parts;
    if (threads == 0) {
        most = (kSms * 16 * 1024 + cols * groups - 1) / (cols * groups);
        parts = per / kLongRows;
    } else {
        const int block = backward_block(threads), at_once = block == 256 ? 2 : 1;
        most = kSms * at_once / groups;
        parts = (per + block / threads - 1) / (block / threads);
    }
    parts = parts < most ? parts : most;
    return parts < 1 ? 1 : parts > 65535 ? 65535 : parts;
}
int64_t rms_norm_workspace(int64_t rows, int64_t cols, int64_t groups)
{
    const int64_t parts = backward_parts(rows, cols, groups);
    return parts > 1 ? parts * groups * cols * 4 : 0;
}

template <typename T, int THREADS, int STEPS, int BT>
static bool backward_as(const RmsNormBackward &a, int parts, bool vec, cudaStream_t st)
{
    auto kernel = a.kept.p ? (vec ? k_rms_norm_backward<T, THREADS, STEPS, BT, true, true> : k_rms_norm_backward<T, THREADS, STEPS, BT, false, true>)
                           : (vec ? k_rms_norm_backward<T, THREADS, STEPS, BT, true, false> : k_rms_norm_backward<T, THREADS, STEPS, BT, false, false>);
    const size_t smem = (size_t)THREADS * STEPS * 32;
    allow_shared(kernel, smem);
    return queue(kernel, dim3((unsigned)parts, (unsigned)a.groups), BT, smem, st, a);
}
template <typename T, bool VEC, bool KEPT>
static bool backward_long(const RmsNormBackward &a, int parts, cudaStream_t st)
{
    // the weight's gradient first: dx may overwrite what it reads
    if (a.dweight && !queue(k_rms_dw_long<T, VEC, KEPT>, dim3((unsigned)((a.cols + 1023) / 1024), (unsigned)parts, (unsigned)a.groups), 128, 0, st, a))
        return false;
    return !a.dx.p || a.rows == 0 || queue(k_rms_dx_long<T, VEC, KEPT>, dim3((unsigned)a.rows), kLongThreads, 0, st, a);
}
template <typename T>
static void backward(const RmsNormBackward &a, cudaStream_t st)
{
    const int size = sizeof(T);
    const bool vec = starts_on_16(a.dy, a.rows, size) && starts_on_16(a.x, a.rows, size) && starts_on_16(a.dtotal, a.rows, size) &&
                     starts_on_16(a.dx, a.rows, size);
    const int64_t units = (a.cols + 7) / 8;
    const int parts = (int)backward_parts(a.rows, a.cols, a.groups);
    bool queued;
    if (units <= 32) queued = backward_as<T, 32, 1, 256>(a, parts, vec, st);
    else if (units <= 64) queued = backward_as<T, 32, 2, 256>(a, parts, vec, st);
    else if (units <= 128) queued = backward_as<T, 64, 2, 256>(a, parts, vec, st);
    else if (units <= 256) queued = backward_as<T, 128, 2, 256>(a, parts, vec, st);
    else if (units <= 512) queued = backward_as<T, 256, 2, 256>(a, parts, vec, st);
    else if (units <= 1024) queued = backward_as<T, 512, 2, 512>(a, parts, vec, st);
    else if (a.kept.p) queued = vec ? backward_long<T, true, true>(a, parts, st) : backward_long<T, false, true>(a, parts, st);
    else queued = vec ? backward_long<T, true, false>(a, parts, st) : backward_long<T, false, false>(a, parts, st);
    if (queued && a.dweight && parts > 1)
        launch_after(k_rms_sums, dim3((unsigned)((a.cols + 31) / 32), (unsigned)a.groups), dim3(1024), 0, st, a, parts);
}
void launch_rms_norm_backward(const RmsNormBackward &a, int type, cudaStream_t st)
{
    if (type == 0) backward<float>(a, st);
    else if (type == 1) backward<bf16>(a, st);
    else backward<f16>(a, st);
}

static dim3 flat_grid(int64_t rows, int64_t units)
{
    const int64_t need = (rows * units + kFlat - 1) / kFlat, most = kSms * 64;
    return dim3((unsigned)(need < most ? need : most));
}
template <typename T>
static void checkpoint(const Matrix &x, const Kept8 &kept, int64_t rows, int64_t cols, cudaStream_t st)
{
    auto kernel = starts_on_16(x, rows, sizeof(T)) ? k_checkpoint8<T, true> : k_checkpoint8<T, false>;
    queue(kernel, flat_grid(rows, (cols + 31) / 32 * 4), kFlat, 0, st, x, kept, rows, cols);
}
void launch_checkpoint8(const Matrix &x, const Kept8 &kept, int64_t rows, int64_t cols, int type, cudaStream_t st)
{
    if (type == 0) checkpoint<float>(x, kept, rows, cols, st);
    else if (type == 1) checkpoint<bf16>(x, kept, rows, cols, st);
    else checkpoint<f16>(x, kept, rows, cols, st);
}
template <typename T>
static void restore(const Rows8 &q, const Kept8 &kept, const Matrix &to, int64_t rows, int64_t cols, cudaStream_t st)
{
    auto kernel = starts_on_16(to, rows, sizeof(T)) ? k_restore8<T, true> : k_restore8<T, false>;
    queue(kernel, flat_grid(rows, (cols + 7) / 8), kFlat, 0, st, q, kept, to, rows, cols);
}
void launch_restore8(const Rows8 &q, const Kept8 &kept, const Matrix &to, int64_t rows, int64_t cols, int type, cudaStream_t st)
{
    if (type == 0) restore<float>(q, kept, to, rows, cols, st);
    else if (type == 1) restore<bf16>(q, kept, to, rows, cols, st);
    else restore<f16>(q, kept, to, rows, cols, st);
}

}  // namespace cdadam
