// Root-mean-square norm with the residual's addition, its gradient, and the 8-bit formats of rows.
//
// All are bound by memory: every matrix is read once and written once.  A group of 32 to 1024 threads
// takes a row at a time, every thread up to four units of eight columns, and asks for its next row's units
// before it works on the present ones (where the registers hold both).
#include "cluster.cuh"
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
__device__ __forceinline__ float2 group_sum_max(float sum, uint32_t top, float2 *slot, int group)
{
    constexpr int N = THREADS / 32;
    sum = warp_sum(sum);
    top = __reduce_max_sync(0xffffffffu, top);
    if (N == 1) return make_float2(sum, __uint_as_float(top));
    if ((threadIdx.x & 31) == 0) slot[threadIdx.x / 32 % N] = make_float2(sum, __uint_as_float(top));
    group_wait<THREADS>(group);
    if (N > 8) {
        const float2 v = (threadIdx.x & 31) < N ? slot[threadIdx.x & 31] : both(0.0f);
        return make_float2(warp_sum(v.x), __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(v.y))));
    }
    float2 v = slot[0];
#pragma unroll
    for (int i = 1; i < N; ++i) {
        const float2 f = slot[i];
        v.x += f.x;
        v.y = __uint_as_float(max(__float_as_uint(v.y), __float_as_uint(f.y)));
    }
    return v;
}
template <int THREADS>
__device__ __forceinline__ float group_sum(float sum, float *slot, int group)
{
    constexpr int N = THREADS / 32;
    sum = warp_sum(sum);
    if (N == 1) return sum;
    if ((threadIdx.x & 31) == 0) slot[threadIdx.x / 32 % N] = sum;
    group_wait<THREADS>(group);
    if (N > 8) return warp_sum((threadIdx.x & 31) < N ? slot[threadIdx.x & 31] : 0.0f);
    sum = slot[0];
#pragma unroll
    for (int i = 1; i < N; ++i) sum += slot[i];
    return sum;
}

// The weight, widened, in shared memory, 0 beyond the row: columns 0 .. 3 of the units in one plane, 4 .. 7
// in another, so that a warp's 16-byte reads are adjacent.
__device__ __forceinline__ void fill_weight(float *w, const AnyVec &v, int cols, int units)
{
    for (int j = threadIdx.x; j < 8 * units; j += blockDim.x)
        w[(j & 4 ? 4 * units : 0) + (j >> 3) * 4 + (j & 3)] = j >= cols ? 0.0f : v.p ? any_at(v, j) : 1.0f;
}
__device__ __forceinline__ void weight8(const float *w, int u, int units, float2 (&f)[4])
{
    const float4 a = *reinterpret_cast<const float4 *>(w + 4 * u), b = *reinterpret_cast<const float4 *>(w + 4 * (units + u));
    f[0] = make_float2(a.x, a.y);
    f[1] = make_float2(a.z, a.w);
    f[2] = make_float2(b.x, b.y);
    f[3] = make_float2(b.z, b.w);
}

// The sum with the residual, as the activations' type holds it.
template <typename T>
__device__ __forceinline__ Raw8<T> sum8(const Raw8<T> &x, const Raw8<T> &residual)
{
    float2 f[4], g[4];
    widen8<T>(x, f);
    widen8<T>(residual, g);
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = add2(f[e], g[e]);
    return narrow8<T>(f);
}

// A block of 32 columns of a checkpoint: four neighbouring threads' units.
template <bool VEC>
__device__ __forceinline__ void keep8(const Kept8 &k, int64_t row, int j, int cols, const float2 (&f)[4], bool vec)
{
    uint32_t m = __float_as_uint(largest8(0.0f, f));
    m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
    m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
    const uint32_t e = kept_exponent(m);
    store_bytes<VEC>(k.p + row * k.stride, j, cols, vec, to_kept8(f, m, e));
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
__device__ __forceinline__ void finish8(const RmsNorm &a, const Place<T> &y, const RowStats &st, int64_t row, int j, const float2 (&p)[4], bool q_vec)
{
    if (a.y.p) {
        float2 f[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = mul2(p[e], both(st.s));
        store8<T, VEC, true>(y, row, j, (int)a.cols, narrow8<T>(f));
    }
    if (a.q.p) store_bytes<VEC>(a.q.p + row * a.q.stride, j, (int)a.cols, q_vec, st.finite ? to_rows8(p, st.step) : make_uint2(0, 0));
}

// ---------------------------------------------------------------------------------------------
// Forward: one read of x and residual, one write of each output.  What is quantised is p = h w and not p s, so that
// it does not wait for the sum: the sum of squares and the largest |p| go through the same exchange, and the rounding of s
// cannot move a value across a half.
// Measured: 16384 x 4096 bf16 with residual and sum in 8 bits 90 us (5.2 TB/s; 113 with reading back, which alone takes 32);
// 30000 x 768 bf16 32 us (5.7 TB/s), 8000 x 4096 f32 105 (5.0); 3001 x 1021 f32 15 us, 20000 x 1022 bf16 54 (3.0 TB/s; rows that start
// anywhere cost 460 instructions a unit and warp instead of 190).
// ---------------------------------------------------------------------------------------------
// Blocks an SM holds.  A thread's units of 16 bits fit into 80 registers, 768 threads (16384 x 4096 bf16 in 8 bits 112 us; with
// 64 registers and 1024 threads, some of them in memory, 120).
constexpr int forward_blocks(int size, int steps, int threads)
{
    return threads > 512 ? 1 : (size * steps <= 4 ? 768 : 512) / threads;
}

template <typename T, int THREADS, int STEPS, int BT, bool VEC>
__global__ void __launch_bounds__(BT, forward_blocks(sizeof(T), STEPS, BT)) k_rms_norm(RmsNorm a)
{
    constexpr int GROUPS = BT / THREADS, UNITS = THREADS * STEPS;
    constexpr bool AHEAD = BT < 1024 || sizeof(T) == 2;       // the next row's units fit into the registers
    extern __shared__ __align__(16) float w[];
    __shared__ float2 slots[GROUPS][2][THREADS / 32];
    const int t = threadIdx.x % THREADS, group = threadIdx.x / THREADS, cols = (int)a.cols;
    const int64_t step = (int64_t)gridDim.x * GROUPS;
    const bool q_vec = on(a.q.p, a.q.stride, 8), kept_vec = on(a.kept.p, a.kept.stride, 8);
    const Place<T> x_ = place<T>(a.x, a.rows), residual_ = place<T>(a.residual, a.rows), total_ = place<T>(a.total, a.rows), y_ = place<T>(a.y, a.rows);
    int64_t row = (int64_t)blockIdx.x * GROUPS + group;
    Unit<T, VEC> x[STEPS], r[STEPS];
    auto fetch = [&](int64_t n) {
        const bool edge = !VEC && x_.edge(n), r_edge = !VEC && residual_.edge(n);
#pragma unroll
        for (int k = 0; k < STEPS; ++k) x[k].ask(x_, n, 8 * (t + k * THREADS), cols, edge);
        if (a.residual.p)
#pragma unroll
            for (int k = 0; k < STEPS; ++k) r[k].ask(residual_, n, 8 * (t + k * THREADS), cols, r_edge);
    };
    if (AHEAD && row < a.rows) fetch(row);
    fill_weight(w, a.weight, cols, UNITS);
    __syncthreads();
    for (int slot = 0; row < a.rows; row += step, slot ^= 1) {
        float2 p[STEPS][4], squares = both(0.0f);
        float top = 0.0f;
        if (!AHEAD) fetch(row);
        const bool edge = !VEC && x_.edge(row), r_edge = !VEC && residual_.edge(row);
#pragma unroll
        for (int k = 0; k < STEPS; ++k) {
            const int j = 8 * (t + k * THREADS);
            Raw8<T> h = x[k].take(x_, row, j, cols, edge);
            if (a.residual.p) h = sum8<T>(h, r[k].take(residual_, row, j, cols, r_edge));
            if (a.total.p) store8<T, VEC, true>(total_, row, j, cols, h);
            widen8<T>(h, p[k]);
        }
        if (AHEAD && row + step < a.rows) fetch(row + step);
#pragma unroll
        for (int k = 0; k < STEPS; ++k) {
            const int u = t + k * THREADS;
            if (a.kept.p) keep8<VEC>(a.kept, row, 8 * u, cols, p[k], kept_vec);
            float2 f[4];
            weight8(w, u, UNITS, f);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                squares = fma2(p[k][e], p[k][e], squares);
                p[k][e] = mul2(p[k][e], f[e]);
            }
            if (a.q.p) top = largest8(top, p[k]);
        }
        const float2 sums = group_sum_max<THREADS>(squares.x + squares.y, __float_as_uint(top), slots[group][slot], group);
        const RowStats st = stats_of(a, sums.x, __float_as_uint(sums.y));
#pragma unroll
        for (int k = 0; k < STEPS; ++k) finish8<T, VEC>(a, y_, st, row, 8 * (t + k * THREADS), p[k], q_vec);
        if (t == 0) {
            if (a.rstd) a.rstd[row] = st.s;
            if (a.q.scale) a.q.scale[row] = st.scale();
        }
    }
}

// Rows too long for the registers of a block: read twice, the second time from the caches.  4000 x 20000 bf16 with residual and
// sum 272 us (2.4 TB/s), 4000 x 20001 405; 64 x 200000 f32 104.
constexpr int kLongThreads = 1024;

__device__ __forceinline__ void weight8_long(const AnyVec &v, int j, int cols, float2 (&f)[4])
{
#pragma unroll
    for (int e = 0; e < 8; ++e) (e & 1 ? f[e / 2].y : f[e / 2].x) = j + e >= cols ? 0.0f : v.p ? any_at(v, j + e) : 1.0f;
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(kLongThreads, 1) k_rms_norm_long(RmsNorm a)
{
    __shared__ float2 slots[kLongThreads / 32];
    const int64_t row = blockIdx.x;
    const int cols = (int)a.cols;
    const bool q_vec = on(a.q.p, a.q.stride, 8), kept_vec = on(a.kept.p, a.kept.stride, 8);
    const Place<T> x_ = place<T>(a.x, a.rows), residual_ = place<T>(a.residual, a.rows), total_ = place<T>(a.total, a.rows), y_ = place<T>(a.y, a.rows);
    float2 f[4], w[4], squares = both(0.0f);
    float top = 0.0f;
    for (int base = 0; base < cols; base += 8 * kLongThreads) {
        const int j = base + 8 * (int)threadIdx.x;
        Raw8<T> h = load8<T, VEC>(x_, row, j, cols);
        if (a.residual.p) h = sum8<T>(h, load8<T, VEC>(residual_, row, j, cols));
        if (a.total.p) store8<T, VEC, true>(total_, row, j, cols, h);
        widen8<T>(h, f);
        if (a.kept.p) keep8<VEC>(a.kept, row, j, cols, f, kept_vec);
        weight8_long(a.weight, j, cols, w);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            squares = fma2(f[e], f[e], squares);
            w[e] = mul2(f[e], w[e]);
        }
        top = largest8(top, w);
    }
    const float2 sums = group_sum_max<kLongThreads>(squares.x + squares.y, __float_as_uint(top), slots, 0);
    const RowStats st = stats_of(a, sums.x, __float_as_uint(sums.y));
    if (threadIdx.x == 0) {
        if (a.rstd) a.rstd[row] = st.s;
        if (a.q.scale) a.q.scale[row] = st.scale();
    }
    if (!a.y.p && !a.q.p) return;
    if (!VEC && a.total.p) __syncthreads();             // units are put together with their neighbours' threads
    for (int base = 0; base < cols; base += 8 * kLongThreads) {
        const int j = base + 8 * (int)threadIdx.x;
        Raw8<T> h;
        if (a.total.p) {                                // may have been written over x
            h = load8<T, VEC>(total_, row, j, cols);
        } else {
            h = load8<T, VEC>(x_, row, j, cols);
            if (a.residual.p) h = sum8<T>(h, load8<T, VEC>(residual_, row, j, cols));
        }
        widen8<T>(h, f);
        weight8_long(a.weight, j, cols, w);
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = mul2(f[e], w[e]);
        finish8<T, VEC>(a, y_, st, row, j, w, q_vec);
    }
}

// ---------------------------------------------------------------------------------------------
// Backward.  A block works on rows of one group of rows, and every thread keeps the sums over rows of
// its own columns, so everything is read once.  (In registers up to 8192 columns, but for up to 132 bytes, most in binary32; beyond, up to
// 144 bytes of a thread's 16-bit whole vectors are in memory, 828 of rows that start anywhere, 240 to 740 in binary32.)  `parts`
// blocks share a group.  Up to eight are a cluster and add their sums up through shared memory; of more (eight_of), each leaves its
// sums in the workspace and k_rms_sums adds them.  All in order: the same bits every time.
// Measured: 32768 x 4096 bf16 from a checkpoint, with dtotal, 161 us (5.9 TB/s); 16384 x 768 bf16 for 8 workers 25 us, of which
// k_rms_sums 4; 16384 x 1536 bf16 43 us (4.6 TB/s), 8000 x 4096 f32 96 (5.5); 20000 x 1022 bf16 57, 3001 x 1021 f16 from a checkpoint
// 16.6 us (two launches, three rows a group).
// ---------------------------------------------------------------------------------------------
// A unit of the activations times s, as they were or as a checkpoint.
template <typename T, bool VEC, bool KEPT> struct Source {
    Unit<T, VEC> u;
    __device__ __forceinline__ void ask(const RmsNormBackward &, const Place<T> &x, int64_t row, int j, int cols, bool)
    {
        u.ask(x, row, j, cols, !VEC && x.edge(row));
    }
    __device__ __forceinline__ void take(const RmsNormBackward &, const Place<T> &x, int64_t row, int j, int cols, Raw8<T> &now) const
    {
        now = u.take(x, row, j, cols, !VEC && x.edge(row));
    }
    typedef Raw8<T> Now;
    static __device__ __forceinline__ void values(const Now &now, float s, float2 (&f)[4])
    {
        widen8<T>(now, f);
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = mul2(f[e], both(s));
    }
};
struct Kept {
    uint2 u;
    uint32_t exponent;
};
__device__ __forceinline__ void anew(Kept &k)
{
    anew(k.u.x);
    anew(k.u.y);
}
template <typename T, bool VEC> struct Source<T, VEC, true> {
    Kept u;
    __device__ __forceinline__ void ask(const RmsNormBackward &a, const Place<T> &, int64_t row, int j, int cols, bool vec)
    {
        u.u = load_bytes<VEC>(a.kept.p + row * a.kept.stride, j, cols, vec);
        u.exponent = j < cols ? __ldg(a.kept.exponents + row * a.kept.exponents_stride + (j >> 5)) : 1;
    }
    typedef Kept Now;
    __device__ __forceinline__ void take(const RmsNormBackward &, const Place<T> &, int64_t, int, int, Kept &now) const { now = u; }
    static __device__ __forceinline__ void values(const Kept &now, float s, float2 (&f)[4])
    {
        const float step = kept_step(now.exponent);
        unpack_bytes(now.u, f);
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = mul2(mul2(f[e], both(step)), both(s));
    }
};

constexpr int kClusterParts = 8;

template <typename T, int THREADS, int STEPS, int BT, bool VEC, bool KEPT>
__global__ void __launch_bounds__(BT, BT > 512 ? 1 : 512 / BT) k_rms_norm_backward(RmsNormBackward a)
{
    constexpr int GROUPS = BT / THREADS, UNITS = THREADS * STEPS;
    constexpr bool AHEAD = STEPS * BT <= 1024 && (VEC || sizeof(T) == 2);    // the next row's units fit into the registers
    extern __shared__ __align__(16) float w[];          // the weight; at the end the groups' sums
    __shared__ float slots[GROUPS][2][THREADS / 32];
    const int t = threadIdx.x % THREADS, group = threadIdx.x / THREADS, cols = (int)a.cols;
    const int64_t per = a.rows / a.groups, end = (blockIdx.y + 1) * per, step = (int64_t)gridDim.x * GROUPS;
    const bool vec = KEPT && on(a.kept.p, a.kept.stride, 8);
    const float over = __frcp_rn((float)cols);
    const Place<T> dy_ = place<T>(a.dy, a.rows), x_ = place<T>(a.x, a.rows), dtotal_ = place<T>(a.dtotal, a.rows), dx_ = place<T>(a.dx, a.rows);
    int64_t row = blockIdx.y * per + (int64_t)blockIdx.x * GROUPS + group;
    Unit<T, VEC> dy[STEPS], more[STEPS];
    Source<T, VEC, KEPT> x[STEPS];
    float rstd = 0.0f;
    auto fetch = [&](int64_t n) {
        rstd = __ldg(a.rstd + n);
        const bool edge = !VEC && dy_.edge(n), more_edge = !VEC && dtotal_.edge(n);
#pragma unroll
        for (int k = 0; k < STEPS; ++k) {
            const int j = 8 * (t + k * THREADS);
            dy[k].ask(dy_, n, j, cols, edge);
            x[k].ask(a, x_, n, j, cols, vec);
            if (AHEAD && a.dtotal.p) more[k].ask(dtotal_, n, j, cols, more_edge);
        }
    };
    if (a.dweight && gridDim.x > kClusterParts) grid_dep_launch();  // of k_rms_sums, which waits for all of this
    if (AHEAD && row < end) fetch(row);
    fill_weight(w, a.weight, cols, UNITS);
    __syncthreads();
    float2 sums[STEPS][4];
#pragma unroll
    for (int k = 0; k < STEPS; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) sums[k][e] = both(0.0f);
    for (int slot = 0; row < end; row += step, slot ^= 1) {
        if (!AHEAD) fetch(row);
        float2 dot = both(0.0f);
        const float s = rstd;
        Raw8<T> dy_now[STEPS], more_now[STEPS];
        typename Source<T, VEC, KEPT>::Now x_now[STEPS];
        const bool edge = !VEC && dy_.edge(row), more_edge = !VEC && dtotal_.edge(row);
#pragma unroll
        for (int k = 0; k < STEPS; ++k) {
            const int j = 8 * (t + k * THREADS);
            dy_now[k] = dy[k].take(dy_, row, j, cols, edge);
            x[k].take(a, x_, row, j, cols, x_now[k]);
            if (AHEAD && a.dtotal.p) more_now[k] = more[k].take(dtotal_, row, j, cols, more_edge);
        }
        if (AHEAD && row + step < end) fetch(row + step);
#pragma unroll
        for (int k = 0; k < STEPS; ++k) {
            float2 g[4], xh[4], f[4];
            Source<T, VEC, KEPT>::values(x_now[k], s, xh);
            widen8<T>(dy_now[k], g);
            weight8(w, t + k * THREADS, UNITS, f);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                sums[k][e] = fma2(g[e], xh[e], sums[k][e]);
                dot = fma2(mul2(g[e], f[e]), xh[e], dot);
            }
        }
        if (!a.dx.p) continue;
        if (!AHEAD && a.dtotal.p)
#pragma unroll
            for (int k = 0; k < STEPS; ++k) more[k].ask(dtotal_, row, 8 * (t + k * THREADS), cols, more_edge);
        const float mean = __fmul_rn(group_sum<THREADS>(dot.x + dot.y, slots[group][slot], group), over);
#pragma unroll
        for (int k = 0; k < STEPS; ++k) {
            float2 g[4], xh[4], f[4];
            anew(x_now[k]);
            anew(dy_now[k]);
            Source<T, VEC, KEPT>::values(x_now[k], s, xh);
            widen8<T>(dy_now[k], g);
            weight8(w, t + k * THREADS, UNITS, f);
#pragma unroll
            for (int e = 0; e < 4; ++e) g[e] = fma2(xh[e], both(-mean), mul2(g[e], f[e]));
            if (!AHEAD && a.dtotal.p) more_now[k] = more[k].take(dtotal_, row, 8 * (t + k * THREADS), cols, more_edge);
            if (a.dtotal.p) widen8<T>(more_now[k], f);
#pragma unroll
            for (int e = 0; e < 4; ++e) g[e] = a.dtotal.p ? fma2(g[e], both(s), f[e]) : mul2(g[e], both(s));
            store8<T, VEC, true>(dx_, row, 8 * (t + k * THREADS), cols, narrow8<T>(g));
        }
    }
    if (!a.dweight) return;
    // the groups' sums one after the other, as planes
#pragma unroll 1
    for (int i = 0; i < GROUPS; ++i) {
        __syncthreads();
        if (i == group)
#pragma unroll
            for (int k = 0; k < STEPS; ++k)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float4 *p = reinterpret_cast<float4 *>(w + 4 * (h * UNITS + t + k * THREADS));
                    float4 v = i ? *p : make_float4(0, 0, 0, 0);
                    v.x += sums[k][2 * h].x; v.y += sums[k][2 * h].y; v.z += sums[k][2 * h + 1].x; v.w += sums[k][2 * h + 1].y;
                    *p = v;
                }
    }
    __syncthreads();
    const int parts = (int)gridDim.x;
    if (parts > 1 && parts <= kClusterParts) {
        cluster_barrier();
        for (int j = (int)blockIdx.x * BT + threadIdx.x; j < cols; j += parts * BT) {
            const float *const at = &w[(j & 4 ? 4 * UNITS : 0) + (j >> 3) * 4 + (j & 3)];
            float f[kClusterParts], v = 0.0f;
#pragma unroll
            for (int r = 0; r < kClusterParts; ++r) f[r] = r < parts ? __int_as_float(load_at(at_rank(at, r))) : 0.0f;
#pragma unroll
            for (int r = 0; r < kClusterParts; ++r) v += f[r];
            store_grad(a.dweight, blockIdx.y * a.dweight_stride + j, a.grad_type, a.accumulate, v);
        }
        __syncwarp();
        cluster_barrier();                              // no block leaves while others read from it
        return;
    }
    for (int j = threadIdx.x; j < cols; j += BT) {
        const float v = w[(j & 4 ? 4 * UNITS : 0) + (j >> 3) * 4 + (j & 3)];
        if (parts > 1) a.parts[((int64_t)blockIdx.y * parts + blockIdx.x) * cols + j] = v;
        else store_grad(a.dweight, blockIdx.y * a.dweight_stride + j, a.grad_type, a.accumulate, v);
    }
}

// Rows too long for a block's registers: dx a row at a time, read twice; the weight's gradient column by column.  4000 x 20000 bf16
// with dtotal 376 us (of which k_rms_dx_long 200, k_rms_dw_long 85 by themselves), from a checkpoint 377; 4000 x 20001 530 and 510.
template <typename T, bool VEC, bool KEPT>
__global__ void __launch_bounds__(kLongThreads, 1) k_rms_dx_long(RmsNormBackward a)
{
    __shared__ float slots[kLongThreads / 32];
    const int64_t row = blockIdx.x;
    const int cols = (int)a.cols;
    const bool vec = KEPT && on(a.kept.p, a.kept.stride, 8);
    const Place<T> dy_ = place<T>(a.dy, a.rows), x_ = place<T>(a.x, a.rows), dtotal_ = place<T>(a.dtotal, a.rows), dx_ = place<T>(a.dx, a.rows);
    const float s = a.rstd[row];
    float2 g[4], xh[4], w[4], dot = both(0.0f);
    auto take = [&](int j) {
        Source<T, VEC, KEPT> x;
        typename Source<T, VEC, KEPT>::Now now;
        x.ask(a, x_, row, j, cols, vec);
        x.take(a, x_, row, j, cols, now);
        x.values(now, s, xh);
        widen8<T>(load8<T, VEC>(dy_, row, j, cols), g);
        weight8_long(a.weight, j, cols, w);
#pragma unroll
        for (int e = 0; e < 4; ++e) g[e] = mul2(g[e], w[e]);
    };
    for (int j = 8 * (int)threadIdx.x; j < cols; j += 8 * kLongThreads) {
        take(j);
#pragma unroll
        for (int e = 0; e < 4; ++e) dot = fma2(g[e], xh[e], dot);
    }
    const float mean = __fmul_rn(group_sum<kLongThreads>(dot.x + dot.y, slots, 0), __frcp_rn((float)cols));
    for (int base = 0; base < cols; base += 8 * kLongThreads) {
        const int j = base + 8 * (int)threadIdx.x;
        take(j);
        if (a.dtotal.p) widen8<T>(load8<T, VEC>(dtotal_, row, j, cols), w);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 d = fma2(xh[e], both(-mean), g[e]);
            g[e] = a.dtotal.p ? fma2(d, both(s), w[e]) : mul2(d, both(s));
        }
        store8<T, VEC, true>(dx_, row, j, cols, narrow8<T>(g));
    }
}
constexpr int kLongRows = 128;         // rows of a block of the next kernel, at least
template <typename T, bool VEC, bool KEPT>
__global__ void __launch_bounds__(128) k_rms_dw_long(RmsNormBackward a)
{
    const int64_t per = a.rows / a.groups;
    const int cols = (int)a.cols, j = 8 * (int)(blockIdx.x * 128 + threadIdx.x);
    const int parts = gridDim.y, part = blockIdx.y;
    const int64_t first = blockIdx.z * per + per * part / parts, end = blockIdx.z * per + per * (part + 1) / parts;
    const bool vec = KEPT && on(a.kept.p, a.kept.stride, 8);
    const Place<T> dy_ = place<T>(a.dy, a.rows), x_ = place<T>(a.x, a.rows);
    float2 sums[4] = {both(0.0f), both(0.0f), both(0.0f), both(0.0f)};
    if (j >= cols) return;
#pragma unroll 4
    for (int64_t row = first; row < end; ++row) {
        Source<T, VEC, KEPT> x;
        typename Source<T, VEC, KEPT>::Now now;
        float2 g[4], xh[4];
        x.ask(a, x_, row, j, cols, vec);
        widen8<T>(load8<T, VEC>(dy_, row, j, cols), g);
        x.take(a, x_, row, j, cols, now);
        x.values(now, __ldg(a.rstd + row), xh);
#pragma unroll
        for (int e = 0; e < 4; ++e) sums[e] = fma2(g[e], xh[e], sums[e]);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if (j + e >= cols) break;
        const float v = e & 1 ? sums[e / 2].y : sums[e / 2].x;
        if (parts > 1) a.parts[((int64_t)blockIdx.z * parts + part) * cols + j + e] = v;
        else store_grad(a.dweight, blockIdx.z * a.dweight_stride + j + e, a.grad_type, a.accumulate, v);
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
        for (int i = warp; i < parts; i += 32 * 10) {   // 296 parts at once
            float f[10];
#pragma unroll
            for (int k = 0; k < 10; ++k)
                f[k] = i + 32 * k < parts ? __ldcg(a.parts + ((int64_t)blockIdx.y * parts + i + 32 * k) * a.cols + j) : 0.0f;
#pragma unroll
            for (int k = 0; k < 10; ++k) v += f[k];
        }
    sh[warp][lane] = v;
    __syncthreads();
    v = warp_sum(sh[lane][warp]);                       // column `warp` of the block
    if (lane == 0 && (int64_t)blockIdx.x * 32 + warp < a.cols)
        store_grad(a.dweight, blockIdx.y * a.dweight_stride + (int64_t)blockIdx.x * 32 + warp, a.grad_type, a.accumulate, v);
}

// ---------------------------------------------------------------------------------------------
// The formats by themselves, unit by unit.  Rows are padded to whole blocks of four units, so that a
// checkpoint's block is four neighbouring threads.  Measured: 32768 x 4096 bf16 into a checkpoint and back 128 to 130 us (6.3 TB/s, the
// copy rate less 4 %), 1023 x 5001 f32 20 us (two launches, rows that start anywhere).
// ---------------------------------------------------------------------------------------------
constexpr int kFlat = 256;
// Units that a thread asks for before it works on the first: what fits into 64 registers (8000 x 5001 f32 109 us by four, 98 by
// two; 100000 x 100 bf16 41 and 36).
template <typename T, bool VEC> constexpr int kAhead = VEC ? 4 : 2;
constexpr int kWideUnits = 64;             // of a row: from there on a warp's 128 units in one row are half used at least

// Where a thread's A units are.  WIDE: a warp takes 32 A units of one row, lane l the units l, l + 32, .. of them; rows of fewer units, one behind the other, 32 units a warp at a time.  Number i of a sequence of n to a row
// is in row i / n, for i < 2^31 by a product (`magic` = ceil(2^(31 + s) / n), 2^s >= n: the excess adds less than 1 / n).
struct Units {
    unsigned n, magic, shift;
    int64_t all;
};
static Units units_of(int64_t rows, int64_t units, int each)
{
    const int64_t n = units >= kWideUnits ? (units + 32 * each - 1) / (32 * each) : units;
    unsigned s = 0;
    while (((int64_t)1 << s) < n) ++s;
    return {(unsigned)n, (unsigned)((((uint64_t)1 << (31 + s)) + n - 1) / n), s, rows * n};
}
struct UnitAt {
    int64_t row;
    int j;          // cols: none
};
__device__ __forceinline__ int64_t row_of(int64_t i, const Units &u)
{
    return u.all >> 31 ? i / u.n : u.shift ? __umulhi((unsigned)i, u.magic) >> (u.shift - 1) : i;
}
template <bool WIDE, int A>
__device__ __forceinline__ void units_at(int64_t warp, const Units &u, int cols, UnitAt (&at)[A])
{
    const int lane = threadIdx.x & 31;
    if (WIDE) {
        const int64_t row = row_of(warp, u);
        const int j = ((int)(warp - row * u.n) * 32 * A + lane) * 8;
#pragma unroll
        for (int k = 0; k < A; ++k) at[k] = {row, min(j + k * 256, cols)};
    } else {
#pragma unroll
        for (int k = 0; k < A; ++k) {
            const int64_t i = (warp * A + k) * 32 + lane, row = row_of(i, u);
            at[k] = {row, (int)(i - row * u.n) * 8};
            if (i >= u.all) at[k] = {0, cols};
        }
    }
}
// What the warps of a launch take in turn.
template <bool WIDE, int A>
__device__ __forceinline__ int64_t items(const Units &u) { return WIDE ? u.all : (u.all + 32 * A - 1) / (32 * A); }

template <typename T, bool VEC, bool WIDE>
__global__ void __launch_bounds__(kFlat) k_checkpoint8(Matrix x, Kept8 kept, int64_t rows, int cols, Units n)
{
    constexpr int A = kAhead<T, VEC>;
    const bool vec = on(kept.p, kept.stride, 8);
    const Place<T> x_ = place<T>(x, rows);
    const int64_t all = items<WIDE, A>(n), step = (int64_t)gridDim.x * (kFlat / 32);
    for (int64_t i = (int64_t)blockIdx.x * (kFlat / 32) + threadIdx.x / 32; i < all; i += step) {
        UnitAt at[A];
        Unit<T, VEC> u[A];
        units_at<WIDE, A>(i, n, cols, at);
#pragma unroll
        for (int k = 0; k < A; ++k) u[k].ask(x_, at[k].row, at[k].j, cols, !VEC && x_.edge(at[k].row));
#pragma unroll
        for (int k = 0; k < A; ++k) {
            float2 f[4];
            widen8<T>(u[k].take(x_, at[k].row, at[k].j, cols, !VEC && x_.edge(at[k].row)), f);
            keep8<VEC>(kept, at[k].row, at[k].j, cols, f, vec);
        }
    }
}

template <typename T, bool VEC, bool WIDE>
__global__ void __launch_bounds__(kFlat) k_restore8(Rows8 q, Kept8 kept, Matrix to, int64_t rows, int cols, Units n)
{
    constexpr int A = kAhead<T, VEC>;
    const int8_t *p = kept.p ? kept.p : q.p;
    const int64_t stride = kept.p ? kept.stride : q.stride;
    const bool vec = on(p, stride, 8);
    const Place<T> to_ = place<T>(to, rows);
    const int64_t all = items<WIDE, A>(n), step = (int64_t)gridDim.x * (kFlat / 32);
    for (int64_t i = (int64_t)blockIdx.x * (kFlat / 32) + threadIdx.x / 32; i < all; i += step) {
        UnitAt at[A];
        uint2 b[A];
        float s[A];
        units_at<WIDE, A>(i, n, cols, at);
#pragma unroll
        for (int k = 0; k < A; ++k) {
            b[k] = load_bytes<VEC>(p + at[k].row * stride, at[k].j, cols, vec);
            s[k] = 0.0f;
            if (at[k].j < cols)
                s[k] = kept.p ? kept_step(__ldg(kept.exponents + at[k].row * kept.exponents_stride + (at[k].j >> 5))) : __ldg(q.scale + at[k].row);
        }
#pragma unroll
        for (int k = 0; k < A; ++k) {
            float2 f[4];
            unpack_bytes(b[k], f);
#pragma unroll
            for (int e = 0; e < 4; ++e) f[e] = mul2(f[e], both(s[k]));
            store8<T, VEC, WIDE>(to_, at[k].row, at[k].j, cols, narrow8<T>(f));
        }
    }
}

// ---------------------------------------------------------------------------------------------
// Launches
// ---------------------------------------------------------------------------------------------
static bool starts_on(int bytes, const void *p, int64_t rows, int64_t row_bytes)
{
    return !p || (((uintptr_t)p & (uintptr_t)(bytes - 1)) == 0 && (rows <= 1 || (row_bytes & (bytes - 1)) == 0));
}
static bool starts_on_16(const Matrix &m, int64_t rows, int size) { return starts_on(16, m.p, rows, m.stride * size); }

template <typename T, int THREADS, int STEPS, int BT>
static void forward_as(const RmsNorm &a, bool vec, cudaStream_t st)
{
    auto kernel = vec ? k_rms_norm<T, THREADS, STEPS, BT, true> : k_rms_norm<T, THREADS, STEPS, BT, false>;
    const int64_t groups = BT / THREADS, need = (a.rows + groups - 1) / groups, most = kSms * forward_blocks(sizeof(T), STEPS, BT);
    const size_t smem = (size_t)THREADS * STEPS * 32;
    allow_shared(kernel, smem);
    queue(kernel, dim3((unsigned)(need < most ? need : most)), BT, smem, st, a);
}
// Rows of more than 384 units.
template <typename T>
static void forward_wide(const RmsNorm &a, bool vec, cudaStream_t st)
{
    const int64_t units = (a.cols + 7) / 8;
    if (units <= 512) forward_as<T, 256, 2, 256>(a, vec, st);
    else if (units <= 768) forward_as<T, 256, 3, 256>(a, vec, st);
    else if (units <= 1024) forward_as<T, 512, 2, 512>(a, vec, st);
    else if (units <= 1536) forward_as<T, 512, 3, 512>(a, vec, st);
    else if (units <= 2048) forward_as<T, 1024, 2, 1024>(a, vec, st);
    else queue(vec ? k_rms_norm_long<T, true> : k_rms_norm_long<T, false>, dim3((unsigned)a.rows), kLongThreads, 0, st, a);
}
template <typename T>
static void forward(const RmsNorm &a, cudaStream_t st)
{
    const int size = sizeof(T);
    const bool vec = starts_on_16(a.x, a.rows, size) && starts_on_16(a.residual, a.rows, size) && starts_on_16(a.total, a.rows, size) &&
                     starts_on_16(a.y, a.rows, size) && starts_on(8, a.q.p, a.rows, a.q.stride) &&
                     starts_on(8, a.kept.p, a.rows, a.kept.stride) && a.cols % 8 == 0;
    const int64_t units = (a.cols + 7) / 8;
    // Binary32: one unit a thread up to 384 units (20000 x 1021 61 us, two units 72; 8000 x 3000 66 and 80; 30000 x 500 45 and 49; of
    // more two, 8000 x 4096 in 8 bits 115 us, by one 126).  16 bits: two or three (16384 x 4096 in 8 bits 113 us, by one 162;
    // 16000 x 2048 45 and 50; 30000 x 768 32 and 36).  By the width alone: the order of the sums, so their bits, go by the sizes.
    if (units <= 32) forward_as<T, 32, 1, 256>(a, vec, st);
    else if constexpr (sizeof(T) == 4) {
        if (units <= 64) forward_as<T, 64, 1, 256>(a, vec, st);
        else if (units <= 96) forward_as<T, 96, 1, 192>(a, vec, st);
        else if (units <= 128) forward_as<T, 128, 1, 256>(a, vec, st);
        else if (units <= 192) forward_as<T, 192, 1, 192>(a, vec, st);
        else if (units <= 256) forward_as<T, 256, 1, 256>(a, vec, st);
        else if (units <= 384) forward_as<T, 384, 1, 384>(a, vec, st);
        else forward_wide<T>(a, vec, st);
    } else {
        if (units <= 64) forward_as<T, 32, 2, 256>(a, vec, st);
        else if (units <= 96) forward_as<T, 32, 3, 256>(a, vec, st);
        else if (units <= 128) forward_as<T, 64, 2, 256>(a, vec, st);
        else if (units <= 192) forward_as<T, 64, 3, 256>(a, vec, st);
        else if (units <= 256) forward_as<T, 128, 2, 256>(a, vec, st);
        else if (units <= 384) forward_as<T, 128, 3, 256>(a, vec, st);
        else forward_wide<T>(a, vec, st);
    }
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
    return units <= 64 ? 32 : units <= 128 ? 64 : units <= 256 ? 128 : units <= 512 ? 256 : units <= 2048 ? 512 : 0;
}
static int backward_block(int threads) { return threads > 256 ? threads : 256; }
static int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
// Whether nine to 24 blocks a group are a cluster of eight instead.  Each then has more rows, but nothing goes through the
// workspace and k_rms_sums, whose time grows with the columns and the groups (device time by eight and by all, bf16; n: groups).
// Few rows: the second launch is 2 us of the host's (64 x 4096 of one 10.5 and 9.0 us, with the host 10.5 and 11.6).
// More: by what the others would save (n = 16: 2048 x 4096 21 and 28 us, 4096 x 4096 35 and 34, 16384 x 4096 122 and 90, 8192 x 768
// 16.6 and 13.5; n = 24: 6144 x 4096 36 and 45, 12288 x 4096 71 and 76, 24000 x 768 29 and 24).
// Blocks that have an SM to themselves: the GPU holds 15 clusters of them (8192 columns, 1024 rows a group: n = 15 152 and 163 us,
// n = 16 286 and 170).
static bool eight_of(int64_t per, int64_t cols, int64_t groups, int64_t parts, int together, int at_once)
{
    if (parts > 3 * kClusterParts) return false;
    const int64_t rows = ceil_div(per, kClusterParts * together), saved = rows - ceil_div(per, parts * together);
    if (rows <= 9) return true;
    if (at_once == 1 && groups > 15) return false;
    const int64_t worth = cols * (groups > 16 ? groups : 16) / 3200;
    return saved <= (worth > 4 ? worth : 4);
}
static int64_t backward_parts(int64_t rows, int64_t cols, int64_t groups)
{
    const int64_t per = rows / groups;
    const int threads = backward_threads(cols);
    const int together = threads ? backward_block(threads) / threads : 0, at_once = backward_block(threads) == 256 ? 2 : 1;
    // three rows a group of threads, or more
    const int64_t most = threads ? kSms * at_once / groups : ceil_div(kSms * 16 * 1024, cols * groups);
    int64_t parts = threads ? ceil_div(per, 3 * together) : per / kLongRows;
    parts = parts < most ? parts : most;
    parts = parts < 1 ? 1 : parts > 65535 ? 65535 : parts;
    if (threads && (parts <= kClusterParts || eight_of(per, cols, groups, parts, together, at_once)))
        parts = parts > 4 ? 8 : parts > 2 ? 4 : parts;
    return parts;
}
static bool in_a_cluster(int64_t cols, int64_t parts) { return backward_threads(cols) && parts <= kClusterParts; }
int64_t rms_norm_workspace(int64_t rows, int64_t cols, int64_t groups)
{
    const int64_t parts = backward_parts(rows, cols, groups);
    return parts > 1 && !in_a_cluster(cols, parts) ? parts * groups * cols * 4 : 0;
}

template <typename T, int THREADS, int STEPS, int BT>
static bool backward_as(const RmsNormBackward &a, int parts, bool vec, cudaStream_t st)
{
    auto kernel = a.kept.p ? (vec ? k_rms_norm_backward<T, THREADS, STEPS, BT, true, true> : k_rms_norm_backward<T, THREADS, STEPS, BT, false, true>)
                           : (vec ? k_rms_norm_backward<T, THREADS, STEPS, BT, true, false> : k_rms_norm_backward<T, THREADS, STEPS, BT, false, false>);
    const size_t smem = (size_t)THREADS * STEPS * 32;
    allow_shared(kernel, smem);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)parts, (unsigned)a.groups);
    cfg.blockDim = dim3(BT);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)parts;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = parts > 1 && parts <= kClusterParts;
    return cudaLaunchKernelEx(&cfg, kernel, a) == cudaSuccess;
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
                     starts_on_16(a.dx, a.rows, size) && starts_on(8, a.kept.p, a.rows, a.kept.stride) && a.cols % 8 == 0;
    const int64_t units = (a.cols + 7) / 8;
    const int parts = (int)backward_parts(a.rows, a.cols, a.groups);
    bool queued;
    // two units a thread (32768 x 4096 bf16 161 us, by one and 512 threads 208; 20000 x 2048 from a checkpoint 56 and 61; 16384 x 1536
    // 43 and 44; 16384 x 768 for 8 workers 24.7 and, with 96 threads, 23.9, not enough for variants of its own)
    if (units <= 32) queued = backward_as<T, 32, 1, 256>(a, parts, vec, st);
    else if (units <= 64) queued = backward_as<T, 32, 2, 256>(a, parts, vec, st);
    else if (units <= 128) queued = backward_as<T, 64, 2, 256>(a, parts, vec, st);
    else if (units <= 256) queued = backward_as<T, 128, 2, 256>(a, parts, vec, st);
    else if (units <= 512) queued = backward_as<T, 256, 2, 256>(a, parts, vec, st);
    else if (units <= 1024) queued = backward_as<T, 512, 2, 512>(a, parts, vec, st);
    else if (units <= 2048) {
        if constexpr (sizeof(T) == 2) queued = backward_as<T, 512, 4, 512>(a, parts, vec, st);
        else queued = backward_as<T, 1024, 2, 1024>(a, parts, vec, st);
    }
    else if (a.kept.p) queued = vec ? backward_long<T, true, true>(a, parts, st) : backward_long<T, false, true>(a, parts, st);
    else queued = vec ? backward_long<T, true, false>(a, parts, st) : backward_long<T, false, false>(a, parts, st);
    if (queued && a.dweight && parts > 1 && !in_a_cluster(a.cols, parts))
        launch_after(k_rms_sums, dim3((unsigned)((a.cols + 31) / 32), (unsigned)a.groups), dim3(1024), 0, st, a, parts);
}
void launch_rms_norm_backward(const RmsNormBackward &a, int type, cudaStream_t st)
{
    if (type == 0) backward<float>(a, st);
    else if (type == 1) backward<bf16>(a, st);
    else backward<f16>(a, st);
}

static dim3 flat_grid(const Units &n, bool wide, int ahead)
{
    const int64_t each = kFlat / 32 * (wide ? 1 : 32 * ahead), need = (n.all + each - 1) / each, most = kSms * 32;
    return dim3((unsigned)(need < most ? need : most));
}
template <typename T>
static void checkpoint(const Matrix &x, const Kept8 &kept, int64_t rows, int64_t cols, cudaStream_t st)
{
    const int64_t units = (cols + 31) / 32 * 4;
    const bool vec = starts_on_16(x, rows, sizeof(T)) && starts_on(8, kept.p, rows, kept.stride) && cols % 8 == 0, wide = units >= kWideUnits;
    auto kernel = wide ? (vec ? k_checkpoint8<T, true, true> : k_checkpoint8<T, false, true>)
                       : (vec ? k_checkpoint8<T, true, false> : k_checkpoint8<T, false, false>);
    const int each = vec ? kAhead<T, true> : kAhead<T, false>;
    const Units n = units_of(rows, units, each);
    queue(kernel, flat_grid(n, wide, each), kFlat, 0, st, x, kept, rows, (int)cols, n);
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
    const int64_t units = (cols + 7) / 8;
    const bool vec = starts_on_16(to, rows, sizeof(T)) && starts_on(8, q.p, rows, q.stride) && starts_on(8, kept.p, rows, kept.stride) && cols % 8 == 0;
    const bool wide = units >= kWideUnits;
    auto kernel = wide ? (vec ? k_restore8<T, true, true> : k_restore8<T, false, true>)
                       : (vec ? k_restore8<T, true, false> : k_restore8<T, false, false>);
    const int each = vec ? kAhead<T, true> : kAhead<T, false>;
    const Units n = units_of(rows, units, each);
    queue(kernel, flat_grid(n, wide, each), kFlat, 0, st, q, kept, to, rows, (int)cols, n);
}
void launch_restore8(const Rows8 &q, const Kept8 &kept, const Matrix &to, int64_t rows, int64_t cols, int type, cudaStream_t st)
{
    if (type == 0) restore<float>(q, kept, to, rows, cols, st);
    else if (type == 1) restore<bf16>(q, kept, to, rows, cols, st);
    else restore<f16>(q, kept, to, rows, cols, st);
}

}  // namespace cdadam
