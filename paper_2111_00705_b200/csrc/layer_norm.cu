// Layer norm, forward and backward.
//
// Both are bound by memory: a row is read once and its output written once.  An SM runs one block
// of 512 to 768 threads in groups; a group works on a row or two at a time, every thread on 8, 16 or
// 24 elements of a row.  Rows reach a group through a ring of stages in shared memory, filled by bulk copies
// that its first thread issues several rows ahead, so that what is on its way from memory does not
// depend on registers or on where the warps are.  A bulk copy moves whole 16-byte vectors: of a row
// that starts or ends between two it takes the neighbours' bytes along, and only at the very ends
// of the matrix, where there are none, the row's last elements are read from memory directly.
//
// Elements are taken from the stage in units of W consecutive ones: 16 bytes where every row
// starts on a multiple of 16 bytes and is a whole number of units, else two where rows allow that,
// else one by one.
#include <type_traits>

#include "elements.cuh"

namespace cdadam {

// ---------------------------------------------------------------------------------------------
// Rows of a matrix on their way through a group's stages.  A stage holds a chunk of up to 32 rows,
// `pitch` bytes apart, each at its address modulo 16; lane i of the group's first warp issues the
// copy of row i.
// ---------------------------------------------------------------------------------------------
template <typename T>
struct Rows {
    const T *base;
    int64_t stride;
    unsigned rows, near;        // within `near` rows of an end a copy's vectors may reach beyond the matrix
    int cols;

    __device__ __forceinline__ Rows(const void *p, int64_t row_stride, unsigned n, int c)
        : base(static_cast<const T *>(p)), stride(row_stride), rows(n), cols(c)
    {
        near = stride * (int64_t)sizeof(T) >= 16 ? 1 : stride == 0 ? n : 16;
    }
    __device__ __forceinline__ const T *row(unsigned r) const { return base + r * stride; }
    __device__ __forceinline__ bool edge(unsigned r) const { return r < near || rows - 1 - r < near; }
    // The whole vectors around row r that lie within the matrix: [lo, hi).
    __device__ __forceinline__ void window(unsigned r, uintptr_t &lo, uintptr_t &hi) const
    {
        lo = (uintptr_t)row(r) & ~(uintptr_t)15;
        hi = ((uintptr_t)(row(r) + cols) + 15) & ~(uintptr_t)15;
        if (edge(r)) {
            if (lo < (uintptr_t)base) lo += 16;
            if (hi > (uintptr_t)(row(rows - 1) + cols)) hi -= 16;
            if (hi < lo) hi = lo;
        }
    }
    __device__ __forceinline__ uint32_t bytes(unsigned r) const
    {
        uintptr_t lo, hi;
        window(r, lo, hi);
        return (uint32_t)(hi - lo);
    }
    __device__ __forceinline__ void start(unsigned r, char *to, uint64_t *bar) const
    {
        uintptr_t lo, hi;
        window(r, lo, hi);
        if (hi > lo)
            bulk_copy_g2s(to + (lo - ((uintptr_t)row(r) & ~(uintptr_t)15)), reinterpret_cast<const void *>(lo), (uint32_t)(hi - lo), bar);
    }
    // Where row r's first element is in the stage.
    __device__ __forceinline__ const T *find(unsigned r, const char *at) const
    {
        return reinterpret_cast<const T *>(at + ((uintptr_t)row(r) & 15));
    }
    // Puts into the stage what the copy of row r could not bring; thread t of n.
    __device__ __forceinline__ void complete(unsigned r, const char *at, int t, int n) const
    {
        uintptr_t lo, hi;
        window(r, lo, hi);
        T *to = const_cast<T *>(find(r, at));
        for (int j = t; j < cols; j += n)
            if ((uintptr_t)(row(r) + j) < lo || (uintptr_t)(row(r) + j) >= hi) to[j] = row(r)[j];
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");    // a later copy writes there
    }
};

// Bytes from row to row of a stage.
__host__ __device__ __forceinline__ int row_pitch(int cols, int size) { return (cols * size + 30) & ~15; }

// ---------------------------------------------------------------------------------------------
// A group: THREADS threads of a block (whole warps).  Sums over it: within warps by shuffles, then
// through shared memory behind a barrier of the group's own.  `slot` has to alternate from one sum
// of a group to the next.
// ---------------------------------------------------------------------------------------------
template <int THREADS>
__device__ __forceinline__ void group_barrier(int group)
{
    if (THREADS == 32) __syncwarp();
    else asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "n"(THREADS) : "memory");
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
    // each half of the warp adds up one of the sums: lane l of it has warp l's
    v = (lane & 15) < N ? at[2 * (lane & 15) + (upper ? 1 : 0)] : 0.0f;
#pragma unroll
    for (int d = 8; d >= 1; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return make_float2(__shfl_sync(0xffffffffu, v, 0), __shfl_sync(0xffffffffu, v, 16));
}


// Two adjacent elements (their address a multiple of their size together).
template <typename T> struct Two {
    static __device__ __forceinline__ float2 wide(const T *p) { return Vec<T>::up(*reinterpret_cast<const uint32_t *>(p)); }
    static __device__ __forceinline__ void store(T *p, float2 f) { *reinterpret_cast<uint32_t *>(p) = Vec<T>::down(f); }
};
template <> struct Two<float> {
    static __device__ __forceinline__ float2 wide(const float *p) { return *reinterpret_cast<const float2 *>(p); }
    static __device__ __forceinline__ void store(float *p, float2 f) { *reinterpret_cast<float2 *>(p) = f; }
};

// ---------------------------------------------------------------------------------------------
// A thread's N elements of a row, in STEPS steps of E (E / 2 pairs).  BIG (W elements are 16 bytes):
// a step is a unit, unit k of thread t starts at column (t + k THREADS) W.  W = 1 and 2: a step is
// 8 / W units, unit i of step k starts at column (t + (8 k / W + i) THREADS) W.  A launch with N =
// 16 (24) has at least 8 (16) THREADS columns, `fits` sees to that, so that all but a thread's last 8
// elements need no check.
// ---------------------------------------------------------------------------------------------
template <typename T, int W, int N_, int THREADS>
struct Mine {
    static constexpr bool BIG = W * sizeof(T) == 16;
    static constexpr int N = N_, E = BIG ? W : 8, STEPS = N / E, P = E / 2, SURE = N > 8 ? N - 8 : 0;
    static bool fits(int64_t cols) { return cols >= (int64_t)SURE * THREADS && cols <= (int64_t)N * THREADS; }
    static __device__ __forceinline__ int column(int k, int e, int t)
    {
        return BIG ? (t + k * THREADS) * W + e : (t + (k * (E / W) + e / W) * THREADS) * W + e % W;
    }
    static __device__ __forceinline__ bool in(int k, int e, int t, int cols)    // rows are whole units
    {
        return k * E + e / W * W < SURE || column(k, e / W * W, t) < cols;
    }
    // From the stage; 0 beyond the row.
    static __device__ __forceinline__ void load(const T *staged, int k, int t, int cols, float2 (&f)[P])
    {
        if constexpr (BIG) {
            uint4 u = make_uint4(0, 0, 0, 0);
            if (in(k, 0, t, cols)) u = *reinterpret_cast<const uint4 *>(staged + column(k, 0, t));
            Vec<T>::wide(u, f);
        } else if constexpr (W == 2) {
#pragma unroll
            for (int e = 0; e < E; e += 2) {
                f[e / 2] = both(0.0f);
                if (in(k, e, t, cols)) f[e / 2] = Two<T>::wide(staged + column(k, e, t));
            }
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float v = in(k, e, t, cols) ? widen(staged[column(k, e, t)]) : 0.0f;
                if (e & 1) f[e / 2].y = v; else f[e / 2].x = v;
            }
        }
    }
    static __device__ __forceinline__ void store(T *row, int k, int t, int cols, const float2 (&f)[P])
    {
        if constexpr (BIG) {
            if (in(k, 0, t, cols)) __stcs(reinterpret_cast<uint4 *>(row + column(k, 0, t)), Vec<T>::pack(f));
        } else if constexpr (W == 2) {
#pragma unroll
            for (int e = 0; e < E; e += 2)
                if (in(k, e, t, cols)) Two<T>::store(row + column(k, e, t), f[e / 2]);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (in(k, e, t, cols)) row[column(k, e, t)] = narrow<T>(e & 1 ? f[e / 2].y : f[e / 2].x);
        }
    }
};

// Parameters, widened, in shared memory, 0 beyond the row: of units of 8 the first four floats in one
// plane, the last four in another, so that a warp's 16-byte reads are adjacent.
template <typename M, int W, int THREADS>
struct Planes {
    static constexpr int floats = M::N * THREADS, plane = floats / 2;
    template <int BT>
    static __device__ __forceinline__ void fill(float *p, const AnyVec &v, int cols, float absent)
    {
        constexpr int each = (floats + BT - 1) / BT;    // all loads of a thread on their way at once
        float f[each];
#pragma unroll
        for (int i = 0; i < each; ++i) {
            const int j = threadIdx.x + i * BT;
            f[i] = j >= cols ? 0.0f : absent;
            if (v.p && v.type == 0 && j < cols) f[i] = __ldg(static_cast<const float *>(v.p) + j);
        }
        if (v.p && v.type != 0)
#pragma unroll
            for (int i = 0; i < each; ++i)
                if (threadIdx.x + i * BT < cols) f[i] = any_at(v, threadIdx.x + i * BT);
#pragma unroll
        for (int i = 0; i < each; ++i) {
            const int j = threadIdx.x + i * BT;
            if (j >= floats) break;
            if (W == 8) p[(j & 4 ? plane : 0) + (j >> 3) * 4 + (j & 3)] = f[i];
            else p[j] = f[i];
        }
    }
    static __device__ __forceinline__ void load(const float *p, int k, int t, float2 (&f)[M::P])
    {
        if constexpr (M::BIG) {
#pragma unroll
            for (int h = 0; h < W / 4; ++h) {
                const float4 q = *reinterpret_cast<const float4 *>(p + h * plane + (t + k * THREADS) * 4);
                f[2 * h] = make_float2(q.x, q.y);
                f[2 * h + 1] = make_float2(q.z, q.w);
            }
        } else if constexpr (W == 2) {
#pragma unroll
            for (int e = 0; e < M::E; e += 2) f[e / 2] = *reinterpret_cast<const float2 *>(p + M::column(k, e, t));
        } else {
#pragma unroll
            for (int e = 0; e < M::E; ++e) {
                const float v = p[M::column(k, e, t)];
                if (e & 1) f[e / 2].y = v; else f[e / 2].x = v;
            }
        }
    }
};

// Rows of a chunk, stages of a ring, bytes from row to row: the shape of a launch's rings; polls of a
// wait for a chunk.
struct Ring {
    int rows, stages, pitch, wait_limit;
};
constexpr int kMaxStages = 6;

// What has become of a thread's waits for its group's chunks (`late`): 0: all came; 1: from one on
// a wait ran out, the thread then waited a second time, with the default limit: its rows are NaN;
// 2: that was in vain too: the thread waits for nothing any more, after the other stages' copies
// (rows up to `end`), so that no block leaves with copies in flight, and its group's first warp
// starts nothing.  All of a wait behind the first poll is in a function, for the loop's registers'
// sake (inline: 32768 x 4096 bf16 backward 151 us instead of 145).
__device__ __noinline__ int wait_slowly(uint64_t *bars, int stages, int limit, int late, int s, int phase, unsigned row0,
                                        unsigned step, unsigned end)
{
    if (late == 2 || mbar_wait_bounded(&bars[s], phase, limit)) return late;
    if (mbar_wait_bounded(&bars[s], phase)) return 1;
    for (int i = 1; i < stages && row0 + (uint64_t)i * step < end; ++i)
        mbar_wait_bounded(&bars[(s + i) % stages], s + i < stages ? phase : phase ^ 1);
    return 2;
}
__device__ __forceinline__ int wait_chunk(uint64_t *bars, const Ring &ring, int late, int s, int phase, unsigned row0, unsigned step,
                                          unsigned end)
{
    if (ring.wait_limit != 0 && mbar_try_wait(&bars[s], phase)) return late;
    return wait_slowly(bars, ring.stages, ring.wait_limit, late, s, phase, row0, step, end);
}

// 1 / sqrt(v): the approximation and one Newton step, within 1 ulp or so and a third of the
// instructions of the correctly rounded quotient and root.  0 and infinity have no step to take (0
// times infinity): v = 0 gives infinity, a sum of squares that overflowed gives 0.
__device__ __forceinline__ float inverse_root(float v)
{
    const float r = rsqrtf(v);
    return r > 0.0f && r < 3e38f ? r * fmaf(-0.5f * r * v, r, 1.5f) : r;
}

// ---------------------------------------------------------------------------------------------
// Forward.  A group works on two rows at a time: their sums go through the same shuffles and
// barriers, and parameters are taken from shared memory once for both (20000 x 4096 bf16: 71 us a
// row at a time, 61 us so, 5.3 TB/s or 82 % of the copy rate; 16384 x 768 f32 20 us, bf16 14.5, of
// which 9 are the rows at 5.7 TB/s and the rest is the start of the rings and the end of the
// launch).  Rows that do not start on 16 bytes cost about twice the instructions: 20000 x 1021 bf16
// 29 us, 43 %.
// ---------------------------------------------------------------------------------------------
template <typename T, int W, int N, int THREADS, int BT>
__global__ void __launch_bounds__(BT, 1) k_norm(NormForward a, Ring ring)
{
    typedef Mine<T, W, N, THREADS> M;
    typedef Planes<M, W, THREADS> PL;
    constexpr int GROUPS = BT / THREADS;
    extern __shared__ __align__(16) char smem[];        // weight, bias; the rings
    __shared__ float2 sh[GROUPS][2][THREADS / 32];
    __shared__ uint64_t bars[GROUPS][kMaxStages];
    const int t = threadIdx.x % THREADS, group = threadIdx.x / THREADS, cols = (int)a.cols;
    const unsigned rows = (unsigned)a.rows, step = gridDim.x * GROUPS * ring.rows;
    const Rows<T> x(a.x, a.x_stride, rows, cols);
    float *const w = reinterpret_cast<float *>(smem), *const b = w + PL::floats;
    const int stage_bytes = ring.rows * ring.pitch;
    char *stages = smem + 2 * PL::floats * 4 + group * ring.stages * stage_bytes;
    const uint32_t row_bytes = cols * (uint32_t)sizeof(T);
    // the group's first warp: chunk at row r into stage s
    auto start = [&](unsigned r, int s) {
        const int n = min((unsigned)ring.rows, rows - r);
        char *to = stages + s * stage_bytes + t * ring.pitch;
        if (M::BIG) {                                   // rows of whole vectors
            if (t == 0) mbar_arrive_expect_tx(&bars[group][s], n * row_bytes);
            __syncwarp();
            if (t < n) bulk_copy_g2s(to, x.row(r + t), row_bytes, &bars[group][s]);
            return;
        }
        uint32_t sum = t < n ? x.bytes(r + t) : 0;
        sum = __reduce_add_sync(0xffffffffu, sum);
        if (t == 0) mbar_arrive_expect_tx(&bars[group][s], sum);
        __syncwarp();
        if (t < n) x.start(r + t, to, &bars[group][s]);
    };
    unsigned row0 = (blockIdx.x * GROUPS + group) * ring.rows;
    if (t < 32) {
        if (t == 0) {
            for (int i = 0; i < ring.stages; ++i) mbar_init(&bars[group][i], 1);
            mbar_fence_init();
        }
        __syncwarp();
        for (int i = 0; i < ring.stages; ++i)
            if (row0 + (uint64_t)i * step < rows) start(row0 + i * step, i);
    }
    PL::template fill<BT>(w, a.weight, cols, 1.0f);
    PL::template fill<BT>(b, a.bias, cols, 0.0f);
    __syncthreads();
    const float over = 1.0f / (float)cols;
    int s = 0, phase = 0, late = 0;
    for (; row0 < rows; row0 = row0 + (uint64_t)step < rows ? row0 + step : rows) {
        late = wait_chunk(bars[group], ring, late, s, phase, row0, step, rows);
        const float none = late ? NAN : 0.0f;           // one thread that was late is enough for the row
        const int n = min((unsigned)ring.rows, rows - row0);
        for (int i = 0; i < n; i += 2) {
            const bool two = i + 1 < n;
            float2 f[2][M::STEPS][M::P], v[2] = {both(none), both(none)};
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                if (r == 1 && !two) break;
                const unsigned row = row0 + i + r;
                const char *at = stages + s * stage_bytes + (i + r) * ring.pitch;
                const T *staged = M::BIG ? reinterpret_cast<const T *>(at) : x.find(row, at);
                if (!M::BIG && x.edge(row)) {
                    x.complete(row, at, t, THREADS);
                    group_barrier<THREADS>(group);
                }
#pragma unroll
                for (int k = 0; k < M::STEPS; ++k) M::load(staged, k, t, cols, f[r][k]);
#pragma unroll
                for (int k = 0; k < M::STEPS; ++k)
#pragma unroll
                    for (int e = 0; e < M::P; ++e) v[r] = add2(v[r], f[r][k][e]);
            }
            const float2 mean = mul2(group_sum2<THREADS>(v[0].x + v[0].y, v[1].x + v[1].y, sh[group][0], group), both(over));
            if (i + 2 >= n && t < 32 && row0 + (uint64_t)ring.stages * step < rows && __all_sync(0xffffffffu, late < 2))
                start(row0 + ring.stages * step, s);    // all have read
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const float m = r ? mean.y : mean.x;
                v[r] = both(0.0f);
                if (r == 1 && !two) break;
#pragma unroll
                for (int k = 0; k < M::STEPS; ++k)
#pragma unroll
                    for (int e = 0; e < M::P; ++e) {
                        const float2 d = add2(f[r][k][e], both(-m));
                        if (M::in(k, 2 * e + 1, t, cols)) v[r] = fma2(d, d, v[r]);
                        else if (W == 1 && M::in(k, 2 * e, t, cols)) v[r].x = fmaf(d.x, d.x, v[r].x);
                        f[r][k][e] = d;
                    }
            }
            const float2 squares = group_sum2<THREADS>(v[0].x + v[0].y, v[1].x + v[1].y, sh[group][1], group);
            const float2 rstd = make_float2(inverse_root(fmaf(squares.x, over, a.eps)), inverse_root(fmaf(squares.y, over, a.eps)));
            T *y = static_cast<T *>(a.y) + (int64_t)(row0 + i) * a.y_stride;
#pragma unroll
            for (int k = 0; k < M::STEPS; ++k) {
                float2 pw[M::P], pb[M::P];
                PL::load(w, k, t, pw);
                PL::load(b, k, t, pb);
#pragma unroll
                for (int e = 0; e < M::P; ++e) f[0][k][e] = fma2(mul2(f[0][k][e], both(rstd.x)), pw[e], pb[e]);
                M::store(y, k, t, cols, f[0][k]);
                if (two) {
#pragma unroll
                    for (int e = 0; e < M::P; ++e) f[1][k][e] = fma2(mul2(f[1][k][e], both(rstd.y)), pw[e], pb[e]);
                    M::store(y + a.y_stride, k, t, cols, f[1][k]);
                }
            }
            if (t < (two ? 2 : 1)) {
                if (a.mean) a.mean[row0 + i + t] = t ? mean.y : mean.x;
                if (a.rstd) a.rstd[row0 + i + t] = t ? rstd.y : rstd.x;
            }
        }
        if (++s == ring.stages) { s = 0; phase ^= 1; }
    }
}

// Rows too long for the registers of a block: three passes, the later two from the caches, by
// vectors of 16 bytes where rows are whole ones (4000 x 16384 bf16 69 us, 58 % of the copy rate;
// 16383 columns, one by one, 147, 27 %).
constexpr int kLongBlock = 512;

// V elements: 16 bytes or one.
template <typename T, int V> struct RawOf { typedef uint4 type; };
template <typename T> struct RawOf<T, 1> { typedef T type; };
template <typename T, int V> using Raw = typename RawOf<T, V>::type;

template <typename T>
__device__ __forceinline__ void widen_all(const uint4 &u, float (&f)[Vec<T>::n])
{
    float2 g[Vec<T>::n / 2];
    Vec<T>::wide(u, g);
#pragma unroll
    for (int e = 0; e < Vec<T>::n; ++e) f[e] = e & 1 ? g[e / 2].y : g[e / 2].x;
}
template <typename T>
__device__ __forceinline__ void widen_all(const T &u, float (&f)[1]) { f[0] = widen(u); }
template <typename T, int V>
__device__ __forceinline__ void take(const T *p, float (&f)[V]) { widen_all<T>(*reinterpret_cast<const Raw<T, V> *>(p), f); }
template <typename T, int V>
__device__ __forceinline__ void put(T *p, const float (&f)[V])
{
    if constexpr (V > 1) {
        float2 g[V / 2];
#pragma unroll
        for (int e = 0; e < V; e += 2) g[e / 2] = make_float2(f[e], f[e + 1]);
        __stcs(reinterpret_cast<uint4 *>(p), Vec<T>::pack(g));
    } else {
        *p = narrow<T>(f[0]);
    }
}
template <int V>
__device__ __forceinline__ void take(const AnyVec &v, int64_t j, float absent, float (&f)[V])
{
    if (V > 1 && v.p && v.type == 0 && ((uintptr_t)v.p & 15) == 0) {
#pragma unroll
        for (int e = 0; e + 3 < V; e += 4) {
            const float4 q = __ldg(reinterpret_cast<const float4 *>(static_cast<const float *>(v.p) + j + e));
            f[e] = q.x; f[e + 1] = q.y; f[e + 2] = q.z; f[e + 3] = q.w;
        }
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e) f[e] = v.p ? any_at(v, j + e) : absent;
    }
}

template <typename T, int V>
__global__ void __launch_bounds__(kLongBlock) k_norm_long(NormForward a)
{
    __shared__ float sh[2][32];
    const int64_t row = blockIdx.x;
    const T *x = static_cast<const T *>(a.x) + row * a.x_stride;
    T *y = static_cast<T *>(a.y) + row * a.y_stride;
    float s = 0.0f, f[V], w[V], b[V];
#pragma unroll 4
    for (int64_t j = threadIdx.x * V; j < a.cols; j += kLongBlock * V) {
        take(x + j, f);
#pragma unroll
        for (int e = 0; e < V; ++e) s += f[e];
    }
    const float mean = block_sum_all<kLongBlock>(s, sh[0]) / (float)a.cols;
    s = 0.0f;
#pragma unroll 4
    for (int64_t j = threadIdx.x * V; j < a.cols; j += kLongBlock * V) {
        take(x + j, f);
#pragma unroll
        for (int e = 0; e < V; ++e) s = fmaf(f[e] - mean, f[e] - mean, s);
    }
    const float rstd = 1.0f / sqrtf(block_sum_all<kLongBlock>(s, sh[1]) / (float)a.cols + a.eps);
    for (int64_t j = threadIdx.x * V; j < a.cols; j += kLongBlock * V) {
        take(x + j, f);
        take(a.weight, j, 1.0f, w);
        take(a.bias, j, 0.0f, b);
#pragma unroll
        for (int e = 0; e < V; ++e) f[e] = fmaf((f[e] - mean) * rstd, w[e], b[e]);
        put(y + j, f);
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
// Measured: 32768 x 4096 bf16 145 to 156 us (5.2 to 5.5 TB/s, 79 to 85 % of the copy rate); 16384 x 768
// bf16 for 8 workers 25 us, of which the rows take 12, the second kernel 5 and the start of the
// rings 3; 30000 x 1021 f16 60 us (47 %: single elements).  Narrow rows, from two numbers of rows each:
// 1024 columns 6.3 TB/s and 16 us beside that, 500 columns 6.0 TB/s and 15 us, 128 columns 3.4 TB/s (the
// sums over a row) and 12 us: 32768 rows take 48, 31 and 19.5 us.
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

template <typename T, int W, int N, int THREADS, int BT>
__global__ void __launch_bounds__(BT, 1) k_norm_backward(NormBackward a, int blocks, Ring ring)
{
    typedef Mine<T, W, N, THREADS> M;
    typedef Planes<M, W, THREADS> PL;
    constexpr int GROUPS = BT / THREADS, STEPS = M::STEPS, P = M::P;
    extern __shared__ __align__(16) char smem[];        // weight; the rings; at the end the groups' sums
    __shared__ float2 sh[GROUPS][2][THREADS / 32];
    __shared__ uint64_t bars[GROUPS][kMaxStages];
    const int t = threadIdx.x % THREADS, group = threadIdx.x / THREADS, lane = threadIdx.x & 31, cols = (int)a.cols;
    const unsigned rows = (unsigned)a.rows, per = rows / (unsigned)a.groups, end = (blockIdx.y + 1) * per;
    const unsigned step = (unsigned)blocks * GROUPS * ring.rows;
    const Rows<T> x(a.x, a.x_stride, rows, cols), dy(a.dy, a.dy_stride, rows, cols);
    float *const w = reinterpret_cast<float *>(smem);
    const int half = ring.rows * ring.pitch, stage_bytes = 2 * half;
    const uint32_t row_bytes = cols * (uint32_t)sizeof(T);
    char *stages = smem + PL::floats * 4 + group * ring.stages * stage_bytes;
    auto start = [&](unsigned r, int s) {
        const int n = min((unsigned)ring.rows, end - r);
        char *to = stages + s * stage_bytes + t * ring.pitch;
        if (M::BIG) {                                   // rows of whole vectors
            if (t == 0) mbar_arrive_expect_tx(&bars[group][s], 2 * n * row_bytes);
            __syncwarp();
            if (t < n) {
                bulk_copy_g2s(to, x.row(r + t), row_bytes, &bars[group][s]);
                bulk_copy_g2s(to + half, dy.row(r + t), row_bytes, &bars[group][s]);
            }
            return;
        }
        uint32_t sum = t < n ? x.bytes(r + t) + dy.bytes(r + t) : 0;
        sum = __reduce_add_sync(0xffffffffu, sum);
        if (t == 0) mbar_arrive_expect_tx(&bars[group][s], sum);
        __syncwarp();
        if (t < n) {
            x.start(r + t, to, &bars[group][s]);
            dy.start(r + t, to + half, &bars[group][s]);
        }
    };
    unsigned row0 = blockIdx.y * per + (blockIdx.x * GROUPS + group) * ring.rows;
    if (t < 32) {
        if (t == 0) {
            for (int i = 0; i < ring.stages; ++i) mbar_init(&bars[group][i], 1);
            mbar_fence_init();
        }
        __syncwarp();
        for (int i = 0; i < ring.stages; ++i)
            if (row0 + (uint64_t)i * step < end) start(row0 + i * step, i);
    }
    PL::template fill<BT>(w, a.weight, cols, 1.0f);
    // lane l of every warp has the statistics of the chunk's row l, a chunk ahead
    float mean_next = 0.0f, rstd_next = 0.0f;
    if (row0 < end && lane < ring.rows && row0 + lane < end) { mean_next = a.mean[row0 + lane]; rstd_next = a.rstd[row0 + lane]; }
    float2 aw[STEPS][P], ab[STEPS][P];
#pragma unroll
    for (int k = 0; k < STEPS; ++k)
#pragma unroll
        for (int e = 0; e < P; ++e) aw[k][e] = ab[k][e] = both(0.0f);
    __syncthreads();
    const float over = 1.0f / (float)cols;
    int s = 0, phase = 0, flip = 0, late = 0;
    while (row0 < end) {
        const float means = mean_next, rstds = rstd_next;
        const unsigned next = row0 + (uint64_t)step < end ? row0 + step : end;
        if (lane < ring.rows && next + lane < end) { mean_next = a.mean[next + lane]; rstd_next = a.rstd[next + lane]; }
        late = wait_chunk(bars[group], ring, late, s, phase, row0, step, end);
        const int n = min((unsigned)ring.rows, end - row0);
        for (int i = 0; i < n; ++i, flip ^= 1) {
            const unsigned row = row0 + i;
            const float mean = __shfl_sync(0xffffffffu, means, i);
            float rstd = __shfl_sync(0xffffffffu, rstds, i);
            if (late) rstd = NAN;                       // and with it the group's sums over the row
            const char *at = stages + s * stage_bytes + i * ring.pitch;
            const T *sx = M::BIG ? reinterpret_cast<const T *>(at) : x.find(row, at);
            const T *sd = M::BIG ? reinterpret_cast<const T *>(at + half) : dy.find(row, at + half);
            if (!M::BIG && (x.edge(row) || dy.edge(row))) {
                x.complete(row, at, t, THREADS);
                dy.complete(row, at + half, t, THREADS);
                group_barrier<THREADS>(group);
            }
            float2 s1 = both(0.0f), s2 = both(0.0f), fx[STEPS][P], fd[STEPS][P];
#pragma unroll
            for (int k = 0; k < STEPS; ++k) {
                float2 pw[P];
                M::load(sx, k, t, cols, fx[k]);
                M::load(sd, k, t, cols, fd[k]);
                PL::load(w, k, t, pw);
#pragma unroll
                for (int e = 0; e < P; ++e) {
                    const float2 xh = mul2(add2(fx[k][e], both(-mean)), both(rstd)), h = mul2(fd[k][e], pw[e]);
                    s1 = add2(s1, h);
                    s2 = fma2(h, xh, s2);
                    aw[k][e] = fma2(fd[k][e], xh, aw[k][e]);
                    ab[k][e] = add2(ab[k][e], fd[k][e]);
                    fx[k][e] = xh;
                    fd[k][e] = h;
                }
            }
            float2 v = both(0.0f);
            if (a.dx) v = group_sum2<THREADS>(s1.x + s1.y, s2.x + s2.y, sh[group][flip], group);
            else group_barrier<THREADS>(group);
            if (i == n - 1 && t < 32 && row0 + (uint64_t)ring.stages * step < end && __all_sync(0xffffffffu, late < 2))
                start(row0 + ring.stages * step, s);    // all have read
            if (a.dx) {
                const float2 c1 = both(-v.x * over), c2 = both(-v.y * over);
                T *dx = static_cast<T *>(a.dx) + row * a.dx_stride;
#pragma unroll
                for (int k = 0; k < STEPS; ++k) {
#pragma unroll
                    for (int e = 0; e < P; ++e) fx[k][e] = mul2(fma2(fx[k][e], c2, add2(fd[k][e], c1)), both(rstd));
                    M::store(dx, k, t, cols, fx[k]);
                }
            }
        }
        row0 = next;
        if (++s == ring.stages) { s = 0; phase ^= 1; }
    }
    if (late) {
#pragma unroll
        for (int k = 0; k < STEPS; ++k)
#pragma unroll
            for (int e = 0; e < P; ++e) aw[k][e] = ab[k][e] = both(NAN);
    }
    grid_dep_launch();
    if (!a.dweight && !a.dbias) return;
    float *sums = reinterpret_cast<float *>(smem);              // GROUPS x 2 x cols
    if (GROUPS > 1) __syncthreads();                            // the rings are empty
#pragma unroll
    for (int k = 0; k < STEPS; ++k) {
        float *gw = sums + (group * 2) * cols, *gb = gw + cols;
        if (GROUPS > 1 && M::BIG) {                             // 16 bytes at a time
            const int j = M::column(k, 0, t);
            if (j < cols)
#pragma unroll
                for (int e = 0; e < P; e += 2) {
                    *reinterpret_cast<float4 *>(gw + j + 2 * e) = make_float4(aw[k][e].x, aw[k][e].y, aw[k][e + 1].x, aw[k][e + 1].y);
                    *reinterpret_cast<float4 *>(gb + j + 2 * e) = make_float4(ab[k][e].x, ab[k][e].y, ab[k][e + 1].x, ab[k][e + 1].y);
                }
        } else {
#pragma unroll
            for (int e = 0; e < M::E; ++e) {
                const int j = M::column(k, e, t);
                const float vw = e & 1 ? aw[k][e / 2].y : aw[k][e / 2].x, vb = e & 1 ? ab[k][e / 2].y : ab[k][e / 2].x;
                if (j < cols) {
                    if (GROUPS > 1) {
                        gw[j] = vw;
                        gb[j] = vb;
                    } else {
                        leave_sums(a, blockIdx.y, blocks, j, vw, vb);
                    }
                }
            }
        }
    }
    if (GROUPS > 1) {
        __syncthreads();
        for (int j = threadIdx.x; j < cols; j += BT) {
            float vw = 0.0f, vb = 0.0f;
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) {
                vw += sums[(g * 2) * cols + j];
                vb += sums[(g * 2 + 1) * cols + j];
            }
            leave_sums(a, blockIdx.y, blocks, j, vw, vb);
        }
    }
}

// The blocks' sums of a group, added in the order of the blocks: 32 columns a block, its 8 warps a
// share of the blocks each.
constexpr int kSumWarps = 8;

__global__ void __launch_bounds__(32 * kSumWarps) k_norm_sums(NormBackward a, int blocks)
{
    __shared__ float sh[kSumWarps][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t j = (int64_t)blockIdx.x * 32 + lane, n = 2 * a.cols;      // columns of dweight, then of dbias
    const float *p = a.parts + blockIdx.y * (int64_t)blocks * n + j;
    const int share = (blocks + kSumWarps - 1) / kSumWarps, lo = warp * share, hi = min(blocks, lo + share);
    grid_dep_wait();
    float s = 0.0f;
    if (j < n)
#pragma unroll 10
        for (int b = lo; b < hi; ++b) s += __ldcg(p + b * n);
    sh[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && j < n) {
        s = 0.0f;
#pragma unroll
        for (int w = 0; w < kSumWarps; ++w) s += sh[w][lane];
        if (j < a.cols) {
            if (a.dweight) store_grad(a.dweight, blockIdx.y * a.dweight_stride + j, a.grad_type, a.accumulate, s);
        } else if (a.dbias) {
            store_grad(a.dbias, blockIdx.y * a.dbias_stride + j - a.cols, a.grad_type, a.accumulate, s);
        }
    }
}

// Rows too long for that: the sums over rows first (dx may overwrite what they read), then dx; V as
// in k_norm_long.  8192 x 16384 bf16 256 us, where reading x and dy twice takes 205 at the copy
// rate; 16383 columns, one by one, 696.
//
// The sums: a block has 32 V columns and a share of a group's rows, its warps every eighth row of
// that, AHEAD on their way at a time; the warps' sums are added in order.
constexpr int kNormBlock = 256;

template <typename T, int V>
__global__ void __launch_bounds__(kNormBlock, 3) k_norm_dw(NormBackward a, int blocks)
{
    constexpr int WARPS = kNormBlock / 32, AHEAD = V > 1 ? 4 : 8;
    __shared__ float sw[WARPS][32 * V], sb[WARPS][32 * V];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t j0 = (int64_t)blockIdx.z * 32 * V, j = j0 + lane * V, per = a.rows / a.groups;
    const int64_t share = (per + blocks - 1) / blocks, end = (blockIdx.y + 1) * per;
    const int64_t first = blockIdx.y * per + blockIdx.x * share, last = first + share < end ? first + share : end;
    float w[V], b[V];
#pragma unroll
    for (int e = 0; e < V; ++e) w[e] = b[e] = 0.0f;
    if (j < a.cols) {
        const T *x = static_cast<const T *>(a.x) + j, *dy = static_cast<const T *>(a.dy) + j;
        auto rows = [&](int64_t r, auto count) {
            constexpr int n = decltype(count)::value;
            Raw<T, V> ux[n], ud[n];
            float mean[n], rstd[n], fx[V], fd[V];
#pragma unroll
            for (int i = 0; i < n; ++i) {
                const int64_t q = r + i * WARPS;
                ux[i] = *reinterpret_cast<const Raw<T, V> *>(x + q * a.x_stride);
                ud[i] = *reinterpret_cast<const Raw<T, V> *>(dy + q * a.dy_stride);
                mean[i] = a.mean[q];
                rstd[i] = a.rstd[q];
            }
#pragma unroll
            for (int i = 0; i < n; ++i) {
                widen_all<T>(ux[i], fx);
                widen_all<T>(ud[i], fd);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    w[e] = fmaf(fd[e], (fx[e] - mean[i]) * rstd[i], w[e]);
                    b[e] += fd[e];
                }
            }
        };
        int64_t r = first + warp;
        for (; r + (AHEAD - 1) * WARPS < last; r += AHEAD * WARPS) rows(r, std::integral_constant<int, AHEAD>());
        for (; r < last; r += WARPS) rows(r, std::integral_constant<int, 1>());
    }
#pragma unroll
    for (int e = 0; e < V; ++e) {
        sw[warp][lane * V + e] = w[e];
        sb[warp][lane * V + e] = b[e];
    }
    __syncthreads();
    for (int c = threadIdx.x; c < 32 * V; c += kNormBlock) {
        float tw = 0.0f, tb = 0.0f;
        for (int i = 0; i < WARPS; ++i) { tw += sw[i][c]; tb += sb[i][c]; }
        if (j0 + c < a.cols) leave_sums(a, blockIdx.y, blocks, j0 + c, tw, tb);
    }
}

template <typename T, int V>
__global__ void __launch_bounds__(kLongBlock) k_norm_dx(NormBackward a)
{
    __shared__ float sh[2][32];
    const int64_t row = blockIdx.x;
    const T *x = static_cast<const T *>(a.x) + row * a.x_stride;
    const T *dy = static_cast<const T *>(a.dy) + row * a.dy_stride;
    T *dx = static_cast<T *>(a.dx) + row * a.dx_stride;
    const float mean = a.mean[row], rstd = a.rstd[row];
    float s1 = 0.0f, s2 = 0.0f, fx[V], fd[V], w[V];
#pragma unroll 2
    for (int64_t j = threadIdx.x * V; j < a.cols; j += kLongBlock * V) {
        take(x + j, fx);
        take(dy + j, fd);
        take(a.weight, j, 1.0f, w);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const float h = fd[e] * w[e];
            s1 += h;
            s2 = fmaf(h, (fx[e] - mean) * rstd, s2);
        }
    }
    const float c1 = block_sum_all<kLongBlock>(s1, sh[0]) / (float)a.cols, c2 = block_sum_all<kLongBlock>(s2, sh[1]) / (float)a.cols;
    for (int64_t j = threadIdx.x * V; j < a.cols; j += kLongBlock * V) {
        take(x + j, fx);
        take(dy + j, fd);
        take(a.weight, j, 1.0f, w);
#pragma unroll
        for (int e = 0; e < V; ++e) fx[e] = rstd * (fd[e] * w[e] - c1 - (fx[e] - mean) * rstd * c2);
        put(dx + j, fx);
    }
}

// ---------------------------------------------------------------------------------------------
// Launches
// ---------------------------------------------------------------------------------------------
constexpr int kSMs = 148;
constexpr int kSums = kSMs;             // blocks that leave sums, at most

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

// Whether every row of a matrix starts on a multiple of `to` bytes.
static bool aligned(const void *p, int64_t stride, int64_t rows, int size, int to)
{
    return (uintptr_t)p % to == 0 && (rows <= 1 || stride * size % to == 0);
}

// Rows in chunks of about 4 KB (`least` rows where they are longer), fewer where that would leave groups
// without a chunk; two stages to six, until the rings take 160 KB or the shared memory is full.
static Ring ring_of(int64_t rows, int64_t groups, int pitch, int all_groups_and_matrices, int parameter_bytes, int least, int wait_limit)
{
    Ring r;
    r.wait_limit = wait_limit < 0 ? kWaitLimit : wait_limit;
    r.pitch = pitch;
    r.rows = pitch * least >= 4096 ? least : 4096 / pitch;
    if (r.rows > 32) r.rows = 32;
    if (r.rows > rows / groups) r.rows = rows / groups < 1 ? 1 : (int)(rows / groups);
    while (r.rows > 1 && r.rows * pitch * all_groups_and_matrices > 80 * 1024) --r.rows;
    const int bytes = r.rows * pitch * all_groups_and_matrices, room = kSharedLimit - parameter_bytes,
              n = (room < 160 * 1024 ? room : 160 * 1024) / bytes;
    r.stages = n < 2 ? 2 : n > kMaxStages ? kMaxStages : n;
    return r;
}

template <typename T, int W, int N, int THREADS, int BT>
static bool try_forward(const NormForward &a, cudaStream_t st)
{
    if (!Mine<T, W, N, THREADS>::fits(a.cols)) return false;
    constexpr int groups = BT / THREADS;
    const int cols = (int)a.cols;
    const Ring r = ring_of(a.rows, (int64_t)kSMs * groups, row_pitch(cols, sizeof(T)), groups, 2 * N * THREADS * 4, 2, a.wait_limit);
    const int64_t need = ((a.rows + r.rows - 1) / r.rows + groups - 1) / groups;
    const int smem = 2 * N * THREADS * 4 + r.stages * r.rows * r.pitch * groups;
    auto *kernel = k_norm<T, W, N, THREADS, BT>;
    allow_shared(kernel, smem);
    kernel<<<(unsigned)(need < kSMs ? need : kSMs), BT, smem, st>>>(a, r);
    return true;
}

// Rows that start on 16 bytes and are whole units of that go by those, others of an even number of
// elements that start on two by two (20000 x 1022 bf16 25 us, one by one 29; 20000 x 4098 112 and
// 141 us; backward of 32768 x 4090 199 and 233 us), the rest one by one.
//
// A row has the smallest group of 32, 64, 128, 256 or 512 threads whose 16 elements a thread hold
// it (8 up to 256 columns), with two exceptions where more of a group's elements would be empty than
// in use: 24 elements a thread of one warp for 513 to 768 columns, 384 threads for 4097 to 6144.  bf16, 82 M elements,
// us with and without them:
//     columns        520       640       768       518       766       519       767
//     24 elements    67/100    62/84     63/69     77/134    61/95     100/162   70/114
//     columns        4104      5120      6144      4098      6142      4099      6143
//     384 threads    79/108    67/90     61/79     110/132   81/98     141/170   102/122
template <typename T, int W>
static bool forward_by(const NormForward &a, cudaStream_t st)
{
    const int to = W * (int)sizeof(T);
    if (a.cols % W || !aligned(a.x, a.x_stride, a.rows, sizeof(T), to) || !aligned(a.y, a.y_stride, a.rows, sizeof(T), to)) return false;
    return try_forward<T, W, 8, 32, 768>(a, st) || try_forward<T, W, 16, 32, 768>(a, st) || try_forward<T, W, 24, 32, 512>(a, st) ||
           try_forward<T, W, 16, 64, 768>(a, st) || try_forward<T, W, 16, 128, 768>(a, st) || try_forward<T, W, 16, 256, 768>(a, st) ||
           try_forward<T, W, 16, 384, 768>(a, st) || try_forward<T, W, 16, 512, 512>(a, st);
}

template <typename T>
static void forward(const NormForward &a, cudaStream_t st)
{
    if (forward_by<T, Vec<T>::n>(a, st) || forward_by<T, 2>(a, st) || forward_by<T, 1>(a, st)) return;
    constexpr int V = Vec<T>::n;
    if (a.cols % V == 0 && aligned(a.x, a.x_stride, a.rows, sizeof(T), 16) && aligned(a.y, a.y_stride, a.rows, sizeof(T), 16))
        k_norm_long<T, V><<<(unsigned)a.rows, kLongBlock, 0, st>>>(a);
    else
        k_norm_long<T, 1><<<(unsigned)a.rows, kLongBlock, 0, st>>>(a);
}

template <typename T, int W, int N, int THREADS, int BT>
static bool try_backward(const NormBackward &a, int blocks, cudaStream_t st)
{
    if (!Mine<T, W, N, THREADS>::fits(a.cols)) return false;
    constexpr int groups = BT / THREADS;
    const int64_t per = a.rows / a.groups;
    const int cols = (int)a.cols;
    const Ring r = ring_of(per, (int64_t)blocks * groups, row_pitch(cols, sizeof(T)), 2 * groups, N * THREADS * 4, 1, a.wait_limit);
    const int64_t most = ((per + r.rows - 1) / r.rows + groups - 1) / groups;
    if (blocks > most) blocks = (int)most;
    if (blocks < 1) blocks = 1;
    const int rings = N * THREADS * 4 + 2 * r.stages * r.rows * r.pitch * groups, sums = groups > 1 ? groups * 2 * cols * 4 : 0;
    const int smem = rings > sums ? rings : sums;
    auto *kernel = k_norm_backward<T, W, N, THREADS, BT>;
    allow_shared(kernel, smem);
    const bool queued = queue(kernel, dim3((unsigned)blocks, (unsigned)a.groups), BT, smem, st, a, blocks, r);
    if (queued && blocks > 1 && (a.dweight || a.dbias))
        launch_after(k_norm_sums, dim3((unsigned)((2 * a.cols + 31) / 32), (unsigned)a.groups), dim3(32 * kSumWarps), 0, st, a, blocks);
    return true;
}

// Three blocks of k_norm_dw fit on an SM.  A share has 32 rows or more, one batch of a block's warps.
template <typename T, int V>
static void backward_long(const NormBackward &a, int most, cudaStream_t st)
{
    if (a.dweight || a.dbias) {
        const int64_t per = a.rows / a.groups, columns = (a.cols + 32 * V - 1) / (32 * V);
        int64_t blocks = 3 * kSMs / (a.groups * columns);
        if (blocks > per / 32) blocks = per / 32;
        if (blocks > most) blocks = most;
        if (blocks < 1) blocks = 1;
        if (!queue(k_norm_dw<T, V>, dim3((unsigned)blocks, (unsigned)a.groups, (unsigned)columns), kNormBlock, 0, st, a, (int)blocks))
            return;                 // dx may overwrite what the sums were to be taken from
        if (blocks > 1)
            k_norm_sums<<<dim3((unsigned)((2 * a.cols + 31) / 32), (unsigned)a.groups), 32 * kSumWarps, 0, st>>>(a, (int)blocks);
    }
    if (a.dx && a.rows) k_norm_dx<T, V><<<(unsigned)a.rows, kLongBlock, 0, st>>>(a);
}

// As forward, but the sums over rows beside the row leave no room for 24 elements a thread, and the
// exceptions are others.  96 threads of 8 elements for 513 to 768 columns of whole vectors; two by
// two or one by one is slower so.  320 threads for 4097 to 5120 columns that go two by two or one
// by one, although up to 90 bytes of every thread's registers go to memory; whole vectors of 16-bit
// elements would gain less, those of binary32 lose.  bf16 of 100 M elements (f32: 67 M), us with and
// without them (*: not taken):
//     columns        520       640       768       518       766       519       767
//     96 threads     151/160   126/134   116/121   285*/200  242*/153  256*/227  210*/172
//     columns        4104      5120      4104 f32  4098      5118      4099      5119
//     320 threads    184*/211  163*/173  160*/155  230/274   200/223   257/316   224/266
template <typename T, int W>
static bool backward_by(const NormBackward &a, int n, cudaStream_t st)
{
    const int to = W * (int)sizeof(T);
    if (a.cols % W || !aligned(a.x, a.x_stride, a.rows, sizeof(T), to) || !aligned(a.dy, a.dy_stride, a.rows, sizeof(T), to) ||
        (a.dx && !aligned(a.dx, a.dx_stride, a.rows, sizeof(T), to)))
        return false;
    if (try_backward<T, W, 8, 32, 768>(a, n, st) || try_backward<T, W, 16, 32, 512>(a, n, st)) return true;
    if constexpr (W * sizeof(T) == 16)
        if (try_backward<T, W, 8, 96, 768>(a, n, st)) return true;
    if (try_backward<T, W, 16, 64, 512>(a, n, st) || try_backward<T, W, 16, 128, 512>(a, n, st) ||
        try_backward<T, W, 16, 256, 512>(a, n, st))
        return true;
    if constexpr (W * sizeof(T) != 16)
        if (try_backward<T, W, 16, 320, 640>(a, n, st)) return true;
    return try_backward<T, W, 16, 512, 512>(a, n, st);
}

template <typename T>
static void backward(const NormBackward &a, cudaStream_t st)
{
    const int n = blocks_per_group(a.rows, a.groups);
    if (backward_by<T, Vec<T>::n>(a, n, st) || backward_by<T, 2>(a, n, st) || backward_by<T, 1>(a, n, st)) return;
    constexpr int V = Vec<T>::n;
    if (a.cols % V == 0 && aligned(a.x, a.x_stride, a.rows, sizeof(T), 16) && aligned(a.dy, a.dy_stride, a.rows, sizeof(T), 16) &&
        (!a.dx || aligned(a.dx, a.dx_stride, a.rows, sizeof(T), 16)))
        backward_long<T, V>(a, n, st);
    else
        backward_long<T, 1>(a, n, st);
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
