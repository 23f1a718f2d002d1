// Operators on rows of logits: log probabilities of given tokens with entropy and the most
// probable alternatives, its gradient, and distillation from a teacher's listed tokens.
//
// A row of logits is what bounds all three: each has to be read once, and its gradient written
// once.  The log probabilities read it in one streaming pass with a running maximum and sums, and
// their gradient needs no more than the saved normaliser.  The distillation's gradient needs the
// sums of the whole row, so there the row is held on the chip: a thread-block cluster of 1, 2, 4
// or 8 blocks takes it, every block a slice in its shared memory, and the blocks exchange a few
// sums through distributed shared memory.
#include <cooperative_groups.h>

#include "elements.cuh"

namespace cdadam {

constexpr int kMaxList = 128;
constexpr double kLn2 = 0.693147180559945309417;

__device__ __forceinline__ int64_t index_at(const void *p, int64_t i, int index64)
{
    return index64 ? static_cast<const int64_t *>(p)[i] : (int64_t)static_cast<const int32_t *>(p)[i];
}
__device__ __forceinline__ void store_index(void *p, int64_t i, int index64, int32_t v)
{
    if (index64) static_cast<int64_t *>(p)[i] = v;
    else static_cast<int32_t *>(p)[i] = v;
}

// Order of the alternatives: larger value first, then lower index; -0 counts as +0.  Larger
// keys come first.
__device__ __forceinline__ uint64_t order_key(float z, int32_t i)
{
    const uint32_t b = __float_as_uint(z + 0.0f);
    const uint32_t o = (b & 0x80000000u) ? ~b : (b | 0x80000000u);
    return ((uint64_t)o << 32) | (uint32_t)~i;
}
__device__ __forceinline__ float key_value(uint64_t key)
{
    const uint32_t o = (uint32_t)(key >> 32);
    return __uint_as_float((o & 0x80000000u) ? (o & 0x7fffffffu) : ~o);
}
__device__ __forceinline__ int32_t key_index(uint64_t key) { return (int32_t)~(uint32_t)key; }


namespace cg = cooperative_groups;

// Cluster barrier in two halves, for threads that need not be converged: writes before an
// arrival, also to other blocks' shared memory, are visible after the wait.
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_arrive_relaxed() { asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory"); }
// Stores into block `rank`'s shared memory (at the place of `here` in this block's) that are
// counted on its barrier `bar`: no fence, the receiver waits for the bytes.
__device__ __forceinline__ uint32_t cluster_addr(const void *here, int rank)
{
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_addr(here)), "r"(rank));
    return a;
}
__device__ __forceinline__ void send32(const void *here, int rank, uint64_t *bar, float v)
{
    asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.b32 [%0], %1, [%2];" ::"r"(cluster_addr(here, rank)),
                 "r"(__float_as_uint(v)), "r"(cluster_addr(bar, rank)) : "memory");
}
__device__ __forceinline__ void send64(const void *here, int rank, uint64_t *bar, float x, float y)
{
    asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.b64 [%0], %1, [%2];" ::"r"(cluster_addr(here, rank)),
                 "l"(bits64(make_float2(x, y))), "r"(cluster_addr(bar, rank)) : "memory");
}
// As mbar_wait_bounded, for what other blocks of the cluster have sent.
__device__ __forceinline__ bool wait_told(uint64_t *bar, int limit)
{
    for (int spin = 0; spin < limit; ++spin) {
        uint32_t done;
        asm volatile("{\n.reg .pred p;\n"
                     "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n"
                     "selp.u32 %0, 1, 0, p;\n}"
                     : "=r"(done) : "r"(smem_addr(bar)), "r"(0) : "memory");
        if (done) return true;
    }
    return false;
}
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }

// ---------------------------------------------------------------------------------------------
// A row in slices.  The row is cut into 16-byte vectors at multiples of 16 bytes of its address
// (`off` elements of the first vector lie before the row), and the vectors into `parts` equal
// slices, one for each block of the cluster.  Elements of a vector outside the row are -inf: they
// add nothing to a sum and are never an alternative.  A vector belongs to one thread (number
// v mod NT) from the load to the last pass over it.
// ---------------------------------------------------------------------------------------------
constexpr int kMaxParts = 8;

template <typename T>
struct Slice {
    static constexpr int V = Vec<T>::n;
    const T *row;
    int off, vocab, nv;
    int start;              // column of the slice's first element (negative where off > 0)

    // parts = 2^log_parts
    __device__ __forceinline__ Slice(const void *z, int64_t stride, int64_t r, int64_t n, int part, int log_parts)
    {
        row = static_cast<const T *>(z) + r * stride;
        vocab = (int)n;
        off = (int)(((uintptr_t)row & 15) / sizeof(T));
        const int nvec = (off + vocab + V - 1) / V, per = (nvec + (1 << log_parts) - 1) >> log_parts, first = part * per;
        nv = max(0, min(per, nvec - first));
        start = first * V - off;
    }
    __device__ __forceinline__ bool whole(int v) const
    {
        const int c = start + v * V;
        return c >= 0 && c + V <= vocab;
    }
};

// Thread 0 starts the copies of the whole vectors, in order; the (at most two) vectors that reach
// beyond the row are filled by threads.  The copies of a block are bulk copies because these are
// served one after the other: of several blocks on an SM one has its slice early and computes
// while the next one's is on its way.  (Copies issued by all threads share the bandwidth evenly,
// all blocks then wait together and compute together.)
// A copy that does not arrive within the limit of a wait (seconds) makes the row one without a
// distribution: its maximum counts as +inf, its outputs are NaN.  A second wait, with the default limit,
// follows at once, so that nothing is still in flight when the slice is written or the block leaves.
constexpr float kLate = __builtin_huge_valf();
constexpr uint32_t kCopyBytes = 16 * 1024;

template <typename T, int NT>
__device__ __forceinline__ void start_slice(const Slice<T> &s, uint4 *buf, uint64_t *bar)
{
    constexpr int V = Vec<T>::n;
    const int v0 = s.nv > 0 && !s.whole(0) ? 1 : 0, v1 = s.nv > v0 && !s.whole(s.nv - 1) ? s.nv - 1 : max(s.nv, v0);
    if (threadIdx.x == 0) {
        mbar_init(bar, 1);
        mbar_fence_init();
        const uint32_t bytes = (uint32_t)(v1 - v0) * 16;
        mbar_arrive_expect_tx(bar, bytes);
        const char *from = reinterpret_cast<const char *>(s.row + s.start + v0 * V);
        char *to = reinterpret_cast<char *>(buf + v0);
        for (uint32_t at = 0; at < bytes; at += kCopyBytes)
            bulk_copy_g2s(to + at, from + at, min(kCopyBytes, bytes - at), bar);
    }
    if (threadIdx.x >= NT - 2 * V) {
        const int i = threadIdx.x - (NT - 2 * V), v = i < V ? 0 : s.nv - 1, c = s.start + v * V + i % V;
        if (i < V ? v0 == 1 : v1 < s.nv && v >= v0)
            reinterpret_cast<T *>(buf)[v * V + i % V] = c >= 0 && c < s.vocab ? s.row[c] : minus_inf<T>();
    }
}

// Bytes of shared memory of a slice of a row of `vocab` elements, whatever the row's address.
template <typename T>
static size_t slice_bytes(int64_t vocab, int parts)
{
    const int64_t nvec = (vocab + Vec<T>::n - 1 + Vec<T>::n - 1) / Vec<T>::n;
    return (size_t)((nvec + parts - 1) / parts) * 16;
}

template <typename T, int NT>
__device__ __forceinline__ float slice_max(const uint4 *buf, int nv)
{
    typename Vec<T>::running m = Vec<T>::lowest();
#pragma unroll 4
    for (int v = threadIdx.x; v < nv; v += NT) m = Vec<T>::max(m, Vec<T>::top(buf[v]));
    return Vec<T>::value(m);
}

// Exponentials are taken relative to a slice's maximum m: t = z s - c with c = m s rounded to
// binary32, one fused operation; the same c is used wherever sums of slices are joined, so its
// rounding cancels.  The rounding is also what t is at the maximum itself: at most 64 while |c| is
// below 2^31, which leaves binary32's sums of 2^t room on both sides, but hundreds, and 2^t infinite
// or 0, from 2^32 or so on (a mask of -1e10).  Where |m s| is not below that bound, or there is
// nothing but masked logits (m is -inf), the origin is far: t = (z - m) s.  (What lies between kNear
// and kFar keeps a near maximum and a bound of -kFar on c further apart than 2^t reaches.)
constexpr float kFar = 2147483648.0f, kNear = kFar - 4096.0f;       // 2^31

struct Origin {
    float m, c;
    bool far;               // m itself is the origin, not c
    __device__ __forceinline__ Origin(float top, float s)
    {
        far = !(fabsf(top) * s < kNear);
        m = top == kNegInf ? 0.0f : top;
        c = m * s;
    }
    // What t is relative to (products of two binary32 values are exact in 64 bits).
    __device__ __forceinline__ double at(float s) const { return far ? (double)m * (double)s : (double)c; }
};
template <bool FAR>
__device__ __forceinline__ float2 exponents(float2 z, const Origin &o, float s)
{
    return FAR ? mul2(add2(z, both(-o.m)), both(s)) : fma2(z, both(s), both(-o.c));
}
// Exponent of slice p's origin relative to the row's, at least -1e4.
__device__ __forceinline__ float shift(const Origin &p, const Origin &row, float s)
{
    const float d = row.far ? (p.far ? (p.m - row.m) * s : -fmaf(row.m, s, -p.c)) : p.far ? fmaf(p.m, s, -row.c) : p.c - row.c;
    return fmaxf(d, -1e4f);
}
// z relative to the row's origin, in 64 bits.
__device__ __forceinline__ double exponent64(float z, const Origin &row, float s)
{
    return (double)z * (double)s - row.at(s);
}

// ---------------------------------------------------------------------------------------------
// Alternatives.  Every slice gives its k first tokens in descending order to all blocks of the
// cluster, and each places its own among them.  Within a slice each of the NT threads meets a largest value; the k-th largest
// of these is one that at least k elements reach, and in a row without structure hardly more (NT ln(
// NT / (NT - k)) are expected: 74 for NT = 256, k = 64).  It is found in the upper 16 bits of the
// values' order (a bound a little too low only lets a few more in).  A thread keeps a copy of the
// best batch of its even and of its odd rounds; almost all elements that reach the bound are in
// these, and the few other batches that do are read again.  Counting for each collected element how
// many are greater sorts them.  Only where more than kCap are collected (thousands of equal values,
// or the largest all in a few threads' vectors) the slice is walked again in order, the best k so
// far always kept.
// ---------------------------------------------------------------------------------------------
constexpr int kCap = 512;

// The upper 16 bits of the order of the k-th largest of the 32 N values of a warp's lanes (1 <= k <=
// 32 N), by bisection between the smallest and the largest.
template <int N>
__device__ __forceinline__ int kth_of_groups(const float (&g)[N], int k)
{
    int o[N], lo = 0xFFFF, hi = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        o[i] = (int)(order_key(g[i], 0) >> 48);
        lo = min(lo, o[i]);
        hi = max(hi, o[i]);
    }
    lo = __reduce_min_sync(0xffffffffu, lo);
    hi = __reduce_max_sync(0xffffffffu, hi);
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        int n = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) n += o[i] >= mid;
        if (__reduce_add_sync(0xffffffffu, n) >= k) lo = mid; else hi = mid - 1;
    }
    return lo;
}

__device__ __forceinline__ int rank_of(uint64_t key, const uint64_t *keys, int n)
{
    int r = 0;
#pragma unroll 8
    for (int i = 0; i < n; ++i) r += keys[i] > key;
    return r;
}

template <typename T, int NT>
__device__ __noinline__ int collect_in_order(const Slice<T> &sl, float reach, int k, uint64_t *cand, int *count)
{
    constexpr int step = kCap - kMaxList, per = (kCap + NT - 1) / NT;
    const int lo = max(0, sl.start), hi = min(sl.vocab, sl.start + sl.nv * Vec<T>::n);
    int kept = 0;
    uint64_t above = 0;
    for (int base = lo; base < hi; base += step) {
        __syncthreads();
        if (threadIdx.x == 0) *count = kept;
        __syncthreads();
        for (int c = base + threadIdx.x; c < min(base + step, hi); c += NT) {
            const float z = widen(sl.row[c]);
            const uint64_t key = order_key(z, c);
            if (z >= reach && z > kNegInf && key > above) cand[atomicAdd(count, 1)] = key;
        }
        __syncthreads();
        kept = *count;
        if (kept > kMaxList) {
            uint64_t key[per];
            int rank[per];
#pragma unroll
            for (int i = 0; i < per; ++i) {
                const int at = threadIdx.x + i * NT;
                key[i] = at < kept ? cand[at] : 0;
                rank[i] = at < kept ? rank_of(key[i], cand, kept) : kMaxList;
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < per; ++i)
                if (rank[i] < k) cand[rank[i]] = key[i];
            __syncthreads();
            kept = k;
            above = cand[k - 1];
        }
    }
    return kept;
}

// ---------------------------------------------------------------------------------------------
// The forward pass reads every logit once, in batches of kBatch vectors a thread, the next batch
// on its way while one is worked on.  A thread's sums are relative to the largest value it has
// met, c = max(m s, -kFar), and are rescaled when a batch raises it (about ten operations for 32
// logits): no barrier and no second look at a logit, so memory is never waited for together.
// (A thread that meets nothing above the bound, in the masked part of a row, adds up 0 or, near it, finite
// values that the row's maximum makes 0.)
//   e = sum 2^t, h = sum 2^t t, t = z s - c (one fused operation for two logits).
// Masked logits must not make 0 times -inf in h.  LOW raises them (four packed operations for
// eight) to a value whose t is finite and far below -150; binary16 has no such value next to its
// lowest and bounds t itself.  Rows whose maximum is a far origin (where all is masked by -1e10, for
// instance) are added up again relative to it.
// For the alternatives each batch leaves the upper 16 bits of its maximum's order in shared
// memory, and the batch itself where it is the best so far of its thread's even or odd rounds: with
// 4 blocks on every SM, each at its own row of 256 KB, a row's beginning has left L2 when its end
// arrives.
// Measured: 4096 x 131072 bf16 without alternatives 0.166 ms (6.5 TB/s, 98 % of the copy rate: bound
// by memory); with 64 of them 0.240 to 0.255 ms: what follows the pass, some 12,000 warp instructions in
// short dependent pieces, does not all hide behind the other blocks' loads.  One row of 30522 with
// 20 alternatives 10 us.
// ---------------------------------------------------------------------------------------------
constexpr int kBatch = 4;

template <typename T>
__device__ __noinline__ uint4 edge_vector(const Slice<T> sl, int v)
{
    constexpr int V = Vec<T>::n;
    const int c = sl.start + v * V;
    __align__(16) T e[V];
#pragma unroll
    for (int i = 0; i < V; ++i) e[i] = v < sl.nv && c + i >= 0 && c + i < sl.vocab ? sl.row[c + i] : minus_inf<T>();
    return *reinterpret_cast<uint4 *>(e);
}

// A log probability, an entropy: rounding takes neither beyond 0.  NaN stays.
__device__ __forceinline__ float at_most_0(double v) { return v > 0.0 ? 0.0f : (float)v; }
__device__ __forceinline__ float at_least_0(double v) { return v < 0.0 ? 0.0f : (float)v; }

__device__ __forceinline__ uint4 ld_stream(const void *p)
{
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

template <typename T, int NT>
__device__ __forceinline__ void load_batch(const Slice<T> &sl, int v, uint4 (&u)[kBatch])
{
    constexpr int V = Vec<T>::n;
    const int first = v - (int)threadIdx.x;             // of the block's batch
    const T *p = sl.row + (sl.start + v * V);
    if (sl.start + first * V >= 0 && sl.start + (first + kBatch * NT) * V <= sl.vocab && first + kBatch * NT <= sl.nv) {
#pragma unroll
        for (int i = 0; i < kBatch; ++i) u[i] = ld_stream(p + i * NT * V);
    } else {
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const int w = v + i * NT;
            if (w < sl.nv && sl.whole(w)) u[i] = ld_stream(p + i * NT * V);
            else u[i] = edge_vector(sl, w);
        }
    }
}

struct Running {
    float m, c;
    float2 e, h;
};

// Sums of a slice: m its maximum, c the origin of t, e = sum 2^t, h = sum 2^t t.
struct Sums {
    float m, c, e, h;
    int n;                  // entries of the slice's list of alternatives
};

// The sums of a warp's lanes, each relative to its own c, relative to the largest c.  (An origin
// infinitely far below belongs to sums of 0.)
__device__ __forceinline__ void join_warp(float &c, float &e, float &h)
{
    const float n = warp_max(c), d = c - n, f = exp2_fast(d);
    h = warp_sum(f == 0.0f && e == e ? 0.0f : f * fmaf(d, e, h));
    e = warp_sum(f * e);
    c = n;
}

template <typename T, int NT, bool TOP>
__global__ void __launch_bounds__(NT, 1024 / NT) k_logprobs(Logprobs a, int log_parts, int rounds)
{
    const int parts = 1 << log_parts;
    constexpr int V = Vec<T>::n;
    constexpr bool LOW = Vec<T>::wide_range;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ float sh[4][NT / 32];
    __shared__ Sums sums[kMaxParts];
    __shared__ int count[2], reach_sh;
    uint4 *kept = reinterpret_cast<uint4 *>(smem);                  // every group's best batch
    uint64_t *cand = reinterpret_cast<uint64_t *>(kept + 2 * kBatch * NT);  // kCap keys; before that the groups' maxima
    int2 *hits = reinterpret_cast<int2 *>(cand + kCap);             // kCap batches
    uint16_t *kept_at = reinterpret_cast<uint16_t *>(hits + kCap);  // the round of every group's best batch
    uint16_t *keys = kept_at + 2 * NT;                              // one of every batch
    uint64_t *lists = reinterpret_cast<uint64_t *>(keys + rounds * NT);     // of all slices: parts x k keys
    const int part = (int)(blockIdx.x & (unsigned)(parts - 1));
    const int64_t row = blockIdx.x >> log_parts;
    cg::cluster_group cluster = cg::this_cluster();
    if (parts > 1) cluster_arrive();                // a block runs before anything is written to it

    const Slice<T> sl(a.z, a.stride, row, a.vocab, part, log_parts);
    const float s = (float)a.scale2, inv_s = 1.0f / s;
    Running r = {kNegInf, -kFar, {0.0f, 0.0f}, {0.0f, 0.0f}};
    float best[2] = {kNegInf, kNegInf}, second[2] = {kNegInf, kNegInf};     // of the even and the odd rounds
    uint4 u[kBatch], next[kBatch];
    if (sl.nv > 0) load_batch<T, NT>(sl, threadIdx.x, u);
#pragma unroll 2
    for (int i = 0, v = threadIdx.x; i < rounds && i * (kBatch * NT) < sl.nv; ++i, v += kBatch * NT) {
        if ((i + 1) * (kBatch * NT) < sl.nv) load_batch<T, NT>(sl, v + kBatch * NT, next);
        typename Vec<T>::running mx = Vec<T>::top(u[0]);
#pragma unroll
        for (int b = 1; b < kBatch; ++b) mx = Vec<T>::max(mx, Vec<T>::top(u[b]));
        const float top = Vec<T>::value(mx);
        if (TOP) {
            keys[i * NT + threadIdx.x] = (uint16_t)(order_key(top, 0) >> 48);
            const float was = i & 1 ? best[1] : best[0], next2 = fmaxf(i & 1 ? second[1] : second[0], fminf(was, top));
            if (i & 1) second[1] = next2; else second[0] = next2;
            if (top > was) {
                if (i & 1) best[1] = top; else best[0] = top;
                kept_at[(i & 1) * NT + threadIdx.x] = (uint16_t)i;
#pragma unroll
                for (int b = 0; b < kBatch; ++b) kept[((i & 1) * kBatch + b) * NT + threadIdx.x] = u[b];
            }
        }
        r.m = fmaxf(r.m, top);
        const float c = fmaxf(r.m * s, -kFar), d = r.c - c, f = exp2_fast(d);
        r.c = c;
        r.h = mul2(fma2(both(d), r.e, r.h), both(f));
        r.e = mul2(r.e, both(f));
        const typename Vec<T>::running low = Vec<T>::below((c - fmaxf(200.0f, 0.015625f * fabsf(c))) * inv_s);
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            float2 z[V / 2];
            Vec<T>::wide(LOW ? Vec<T>::at_least(u[b], low) : u[b], z);
#pragma unroll
            for (int j = 0; j < V / 2; ++j) {
                float2 t = fma2(z[j], both(s), both(-c));
                const float2 p = make_float2(exp2_fast(t.x), exp2_fast(t.y));
                r.e = add2(r.e, p);
                if (!LOW) t = make_float2(fmaxf(t.x, -1e4f), fmaxf(t.y, -1e4f));
                r.h = fma2(p, t, r.h);
            }
        }
#pragma unroll
        for (int b = 0; b < kBatch; ++b) u[b] = next[b];
    }

    const int lane = threadIdx.x & 31;
    // the block's sums, and the threshold of its alternatives
    float c = r.c, e = r.e.x + r.e.y, h = r.h.x + r.h.y;
    float m = warp_max(r.m);
    join_warp(c, e, h);
    if ((threadIdx.x & 31) == 0) {
        const int w = threadIdx.x >> 5;
        sh[0][w] = m; sh[1][w] = c; sh[2][w] = e; sh[3][w] = h;
    }
    int n = 0;
    if (TOP) {
        reinterpret_cast<float *>(cand)[threadIdx.x] = r.m;
        __syncthreads();
        if (threadIdx.x < 32) {
            float g[NT / 32];
#pragma unroll
            for (int i = 0; i < NT / 32; ++i) g[i] = reinterpret_cast<const float *>(cand)[threadIdx.x + 32 * i];
            const int t = kth_of_groups<NT / 32>(g, a.k);
            if (threadIdx.x == 0) { reach_sh = t; count[0] = count[1] = 0; }
        }
        __syncthreads();
        const int reach16 = max(reach_sh, 0x80);                    // 0x7F: the order of -inf
        const float reach = key_value((uint64_t)reach16 << 48);
        // list the batches that reach it: where the first vector of a kept one is (the others of the
        // batch are NT V elements apart there as in the row) and its column; -1 where it is not kept
        const int place = (int)threadIdx.x * V, column = sl.start + place;
#pragma unroll
        for (int o = 0; o < 2; ++o) {
            const bool in = best[o] >= reach;
            const unsigned all = __ballot_sync(0xffffffffu, in);
            if (all == 0) continue;
            int at = 0;
            if (lane == 0) at = atomicAdd(&count[0], __popc(all));
            at = __shfl_sync(0xffffffffu, at, 0) + __popc(all & ((1u << lane) - 1));
            if (in) {
                const int own = kept_at[o * NT + threadIdx.x];
                if (at < kCap) hits[at] = make_int2(o * (kBatch * NT * V) + place, own * (kBatch * NT * V) + column);
                if (second[o] >= reach)
                    for (int i = o; i < rounds && i * (kBatch * NT) < sl.nv; i += 2)
                        if (keys[i * NT + threadIdx.x] >= reach16 && i != own) {
                            const int to = atomicAdd(&count[0], 1);
                            if (to < kCap) hits[to] = make_int2(-1, i * (kBatch * NT * V) + column);
                        }
            }
        }
        __syncthreads();
        const int noted = count[0];
        if (noted <= kCap) {
            // a warp looks at kAhead batches at a time, a lane at one element of each
            constexpr int kAhead = 8, W = NT / 32;
            const T *elem = reinterpret_cast<const T *>(kept);
            const int mine = lane / V * (NT * V) + lane % V, lo = max(sl.start, 0), hi = min(sl.vocab, sl.start + sl.nv * V);
            for (int i = threadIdx.x >> 5; i < noted; i += kAhead * W) {
                T raw[kAhead];                      // all on their way before the first is looked at
                int at[kAhead];
#pragma unroll
                for (int o = 0; o < kAhead; ++o) {
                    const bool there = i + o * W < noted && lane < kBatch * V;
                    const int2 h = hits[there ? i + o * W : 0];
                    at[o] = h.y + mine;
                    const bool in = there && at[o] >= lo && at[o] < hi;
                    const T *p = h.x >= 0 ? elem + (h.x + mine) : sl.row + at[o];
                    raw[o] = minus_inf<T>();
                    if (in) raw[o] = *p;
                }
                float z[kAhead];
#pragma unroll
                for (int o = 0; o < kAhead; ++o) z[o] = widen(raw[o]);
                // one reservation for all of them
                int total = 0, to = 0;
                unsigned all[kAhead];
#pragma unroll
                for (int o = 0; o < kAhead; ++o) {
                    all[o] = __ballot_sync(0xffffffffu, z[o] >= reach);
                    total += __popc(all[o]);
                }
                if (lane == 0 && total) to = atomicAdd(&count[1], total);
                to = __shfl_sync(0xffffffffu, to, 0);
#pragma unroll
                for (int o = 0; o < kAhead; ++o) {
                    if (z[o] >= reach) {
                        const int here = to + __popc(all[o] & ((1u << lane) - 1));
                        if (here < kCap) cand[here] = order_key(z[o], at[o]);
                    }
                    to += __popc(all[o]);
                }
            }
            __syncthreads();
            n = count[1];
        }
        if (noted > kCap || n > kCap) n = collect_in_order<T, NT>(sl, reach, a.k, cand, &count[1]);
    }
    __syncthreads();
    if (parts > 1) cluster_wait();
    // every block gets all slices' lists and sums, and places its own alternatives among them
    if (TOP)
        for (int i = threadIdx.x; i < n; i += NT) {
            const uint64_t key = cand[i];
            const int at = rank_of(key, cand, n);
            if (at >= a.k) continue;
            if (parts == 1) lists[at] = key;
            else
                for (int o = 0; o < parts; ++o) cluster.map_shared_rank(lists, o)[part * a.k + at] = key;
        }
    if (threadIdx.x < 32) {
        const bool is = threadIdx.x < NT / 32;
        m = warp_max(is ? sh[0][threadIdx.x] : kNegInf);
        c = is ? sh[1][threadIdx.x] : -kFar;
        e = is ? sh[2][threadIdx.x] : 0.0f;
        h = is ? sh[3][threadIdx.x] : 0.0f;
        join_warp(c, e, h);
        // (without alternatives to the first block alone: the others do not wait for anything)
        if (lane < (TOP ? parts : 1)) (parts > 1 ? cluster.map_shared_rank(sums, lane) : sums)[part] = Sums{m, c, e, h, min(n, a.k)};
    }
    if (parts > 1) {
        cluster_arrive();
        if (!TOP && part != 0) return;               // nothing is sent to this block
        cluster_wait();
    } else {
        __syncthreads();
    }

    // the row
    const bool is = lane < parts;
    const Sums p = sums[is ? lane : 0];
    float M = warp_max(p.m), C = p.c, E = is ? p.e : 0.0f, H = is ? p.h : 0.0f;
    join_warp(C, E, H);
    const int total = TOP ? (int)__reduce_add_sync(0xffffffffu, is ? p.n : 0) : 0;
    Origin all(M, s);
    all.c = C;
    all.far &= M > kNegInf && M <= 3.402823466e38f;
    if (all.far) {                                   // relative to the maximum, by this block alone
        e = h = 0.0f;
        for (int64_t i = threadIdx.x; i < a.vocab; i += NT) {
            const float t = (widen(static_cast<const T *>(sl.row)[i]) - M) * s, p = exp2_fast(t);
            e += p;
            h = fmaf(p, fmaxf(t, -1e4f), h);
        }
        __syncthreads();
        E = block_sum_all<NT>(e, sh[0]);
        H = block_sum_all<NT>(h, sh[1]);
    }
    if ((int)(threadIdx.x & ~31u) >= (TOP ? a.k : 1)) return;
    const bool none = E != E || M > 3.402823466e38f, empty = !none && E == 0.0f;
    const double l2 = none ? (double)NAN : empty ? (double)kNegInf : log2((double)E);
    if (threadIdx.x == 0 && part == 0) {
        if (a.logprob) {
            const int64_t t = index_at(a.tokens, row, a.index64);
            a.logprob[row] = t < 0 ? 0.0f : t >= a.vocab || none ? NAN : empty ? kNegInf
                : at_most_0((exponent64(widen(sl.row[t]), all, s) - l2) * kLn2);
        }
        if (a.entropy) a.entropy[row] = empty ? 0.0f : at_least_0((l2 - (double)H / (double)E) * kLn2);
        // z s - c - l2 is the log of p_i for s as rounded; the exact scale for the origin itself
        if (a.lse) a.lse[row] = (float)(((all.far ? (double)all.m * a.scale2 : (double)all.c * (a.scale2 / (double)s)) + l2) * kLn2);
    }
    if (!TOP) return;
    for (int j = threadIdx.x; j < (none ? 0 : sums[part].n); j += NT) {
        const uint64_t key = lists[part * a.k + j];
        int at = j;
        for (int o = 0; o < parts; ++o) {
            if (o == part) continue;
            int lo = 0, hi = sums[o].n;              // first entry of list o that is not greater
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                if (lists[o * a.k + mid] > key) lo = mid + 1; else hi = mid;
            }
            at += lo;
        }
        if (at < a.k) {
            store_index(a.top_ids, row * a.k + at, a.index64, key_index(key));
            a.top_logprobs[row * a.k + at] = at_most_0((exponent64(key_value(key), all, s) - l2) * kLn2);
        }
    }
    for (int t = threadIdx.x; t < a.k && part == 0; t += NT)
        if (none || t >= total) {
            store_index(a.top_ids, row * a.k + t, a.index64, -1);
            a.top_logprobs[row * a.k + t] = none ? NAN : kNegInf;
        }
}

// ---------------------------------------------------------------------------------------------
// Gradient of log probability and entropy.  With t = (z - lse T) s, p = 2^t,
//   dz_i = p (a t + b) (+ g at the token),   a = -u ln2 / T,  b = -(g + u H) / T,
// one pass over the logits: a block has kGradVecs vectors for each of its threads.  lse T s is taken
// off in two parts, and with s as rounded for the logits, so that t has a relative error of 2^-23
// however large z and lse are (beside what lse's own rounding means).  Bound by memory: 4096 x
// 30522 bf16 with both gradients 86 to 91 us (5.5 to 5.8 TB/s, 84 to 89 % of the copy rate).
// ---------------------------------------------------------------------------------------------
constexpr int kGradVecs = 4;
constexpr float kLost = 16777216.0f;        // |lse| from which binary32 says nothing about p

template <typename T, int NT>
__global__ void __launch_bounds__(NT) k_logprobs_backward(LogprobsBackward a, int chunks)
{
    constexpr int V = Vec<T>::n;
    const int64_t row = chunks == 1 ? blockIdx.x : blockIdx.x / (unsigned)chunks;
    const int chunk = chunks == 1 ? 0 : (int)(blockIdx.x - (unsigned)row * (unsigned)chunks);
    const Slice<T> sl(a.z, a.stride, row, a.vocab, 0, 0);
    T *out = static_cast<T *>(a.dz) + row * a.dz_stride;
    const bool same = (((uintptr_t)out - (uintptr_t)sl.row) & 15) == 0;

    const int64_t at = a.dlogprob ? index_at(a.tokens, row, a.index64) : -1;
    const int token = at >= 0 && at < a.vocab ? (int)at : -0x40000000;
    const float lse = a.lse[row], g = token >= 0 ? a.dlogprob[row] : 0.0f;
    const float u = a.dentropy ? a.dentropy[row] : 0.0f, H = a.dentropy ? a.entropy[row] : 0.0f;
    const bool zero = (g == 0.0f && u == 0.0f) || fabsf(lse) >= kLost;
    const float s = (float)a.scale2;
    const double l2 = (double)lse * a.lse_scale;
    const float hi = (float)l2, lo = (float)(l2 - (double)hi);
    const float ca = -u * ((float)kLn2 * a.inv_temperature), cb = -(fmaf(u, H, g)) * a.inv_temperature, cg = g * a.inv_temperature;
    // a row without a distribution, or a gradient that is not finite: 0 times that is NaN, and masked logits have 0
    const bool careful = lse != lse || !(fabsf(ca) + fabsf(cb) < __builtin_huge_valf());

    const int v0 = chunk * (NT * kGradVecs) + threadIdx.x;
    uint4 q[kGradVecs];
    if (!zero) {
#pragma unroll
        for (int i = 0; i < kGradVecs; ++i) {
            const int v = v0 + i * NT, c = sl.start + v * V;
            if (v < sl.nv) {
                if (sl.whole(v)) {
                    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                                 : "=r"(q[i].x), "=r"(q[i].y), "=r"(q[i].z), "=r"(q[i].w) : "l"(sl.row + c) : "memory");
                } else {
                    __align__(16) T e[V];
#pragma unroll
                    for (int j = 0; j < V; ++j) e[j] = c + j >= 0 && c + j < sl.vocab ? sl.row[c + j] : minus_inf<T>();
                    q[i] = *reinterpret_cast<uint4 *>(e);
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < kGradVecs; ++i) {
        const int v = v0 + i * NT, c = sl.start + v * V;
        if (v >= sl.nv) break;
        float2 f[V / 2];
        if (zero) {
#pragma unroll
            for (int j = 0; j < V / 2; ++j) f[j] = both(0.0f);
        } else {
            Vec<T>::wide(q[i], f);
            const int k = token - c;                // which of the vector's elements is the token, if one is
            float at_token = kNegInf;
            if (k >= 0 && k < V) at_token = widen(sl.row[token]);
            if (careful) {
#pragma unroll
                for (int j = 0; j < V / 2; ++j) {
                    const float2 t = add2(fma2(f[j], both(s), both(-hi)), both(-lo));
                    const float x = exp2_fast(t.x) * fmaf(fmaxf(t.x, -1e4f), ca, cb), y = exp2_fast(t.y) * fmaf(fmaxf(t.y, -1e4f), ca, cb);
                    f[j] = make_float2(f[j].x == kNegInf ? 0.0f : x, f[j].y == kNegInf ? 0.0f : y);
                }
            } else if (ca == 0.0f) {
#pragma unroll
                for (int j = 0; j < V / 2; ++j) {
                    const float2 t = add2(fma2(f[j], both(s), both(-hi)), both(-lo));
                    f[j] = mul2(make_float2(exp2_fast(t.x), exp2_fast(t.y)), both(cb));
                }
            } else {
#pragma unroll
                for (int j = 0; j < V / 2; ++j) {
                    const float2 t = add2(fma2(f[j], both(s), both(-hi)), both(-lo));
                    f[j] = mul2(make_float2(exp2_fast(t.x), exp2_fast(t.y)),
                                fma2(make_float2(fmaxf(t.x, -1e4f), fmaxf(t.y, -1e4f)), both(ca), both(cb)));
                }
            }
            if (at_token != kNegInf) {              // (a masked token has no gradient)
#pragma unroll
                for (int j = 0; j < V / 2; ++j) {
                    if (2 * j == k) f[j].x += cg;
                    if (2 * j + 1 == k) f[j].y += cg;
                }
            }
        }
        const uint4 r = Vec<T>::pack(f);
        if (same && sl.whole(v)) {
            __stcs(reinterpret_cast<uint4 *>(out + c), r);
        } else {
            __align__(16) T e[V];
            *reinterpret_cast<uint4 *>(e) = r;
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (c + j >= 0 && c + j < sl.vocab) out[c + j] = e[j];
        }
    }
}

// ---------------------------------------------------------------------------------------------
// Distillation.  The listed tokens are taken out of the slice (set to -inf) before its maximum
// and sum are formed, so that the rest of the vocabulary has its own maximum and sum: R comes
// from a sum of positive terms instead of from 1 - sum p_j, and neither part underflows however
// far the other is above it.  The gradient replaces the slice in shared memory, the listed
// tokens' entries are put in afterwards, and the slice leaves as one bulk copy.
// Measured: 4096 x 131072 bf16, 64 listed, loss and gradient 0.405 to 0.440 ms (4.9 to 5.3 TB/s, 75 to
// 81 % of the copy rate), the loss alone 0.274 (60 %); 1023 x 50021 f16 48 us, the loss alone 33.  A
// block's own chain (list, slice, maximum, sum, the cluster's sums, gradient) is about four times
// as long as its slice takes in memory, and six blocks on an SM do not quite cover that.  Half of what an exchange through cluster barriers cost was their fences:
// the sums go out as stores that the receiver's mbarrier counts (0.538 -> 0.439 ms).  Exponentials
// by arithmetic for a quarter of the logits, to spare the special function unit: 0.457 instead of
// 0.439 ms, the passes are bound by issue, not by that unit.
// ---------------------------------------------------------------------------------------------
struct Rest {
    float m, e;
};

__device__ __forceinline__ double warp_sum64(double v)
{
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}

template <typename T, int NT, bool FAR>
__device__ __forceinline__ float slice_sum(const uint4 *buf, int nv, const Origin &o, float s)
{
    constexpr int V = Vec<T>::n;
    float2 e2[V / 2];           // a sum for each pair: short chains of dependent additions
#pragma unroll
    for (int i = 0; i < V / 2; ++i) e2[i] = both(0.0f);
#pragma unroll 4
    for (int v = threadIdx.x; v < nv; v += NT) {
        float2 f[V / 2];
        Vec<T>::wide(buf[v], f);
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
            const float2 t = exponents<FAR>(f[i], o, s);
            e2[i] = add2(e2[i], make_float2(exp2_fast(t.x), exp2_fast(t.y)));
        }
    }
#pragma unroll
    for (int i = 1; i < V / 2; ++i) e2[0] = add2(e2[0], e2[i]);
    return e2[0].x + e2[0].y;
}

// The slice becomes scale 2^t.
template <typename T, int NT, bool FAR>
__device__ __forceinline__ void slice_gradient(uint4 *buf, int nv, const Origin &o, float s, float scale)
{
    constexpr int V = Vec<T>::n;
#pragma unroll 4
    for (int v = threadIdx.x; v < nv; v += NT) {
        float2 f[V / 2];
        Vec<T>::wide(buf[v], f);
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
            const float2 t = exponents<FAR>(f[i], o, s);
            f[i] = mul2(make_float2(exp2_fast(t.x), exp2_fast(t.y)), both(scale));
        }
        buf[v] = Vec<T>::pack(f);
    }
}

template <typename T, int NT>
__global__ void __launch_bounds__(NT) k_distill(Distill a, int log_parts)
{
    constexpr int V = Vec<T>::n, kWarps = kMaxList / 32;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ float sh[2][NT / 32], top32[kWarps], zl[kMaxList];
    __shared__ __align__(16) int32_t id[kMaxList];
    __shared__ double w[kMaxList], sum64[2][kWarps];
    __shared__ __align__(8) Rest rest_sh[kMaxParts];
    __shared__ uint64_t bar, told;              // the slice has arrived; the cluster's sums have
    __shared__ bool listed[kMaxList];
    __shared__ int repeated;
    uint4 *buf = reinterpret_cast<uint4 *>(smem);
    T *elem = reinterpret_cast<T *>(smem);
    const int parts = 1 << log_parts, part = (int)(blockIdx.x & (unsigned)(parts - 1)), j = threadIdx.x, k = a.k, lane = j & 31;
    const int64_t row = blockIdx.x >> log_parts;
    cg::cluster_group cluster = cg::this_cluster();
    const Slice<T> sl(a.z, a.stride, row, a.vocab, part, log_parts);

    // The list is asked for ahead of the slice, and worked on while that is on its way: the teacher's
    // distribution.  Thread j < k has entry j; an index listed again is left to its first entry.
    // Unused: id -1, weight 0.
    int mine = -1;
    float lq = kNegInf;
    double q = 0.0;
    int64_t listed_id = -1;
    if (j < k) {
        listed_id = index_at(a.ids, row * k + j, a.index64);
        lq = a.teacher[row * k + j];
    }
    if (j == 0) {
        repeated = 0;
        mbar_init(&told, 1);
    }
    start_slice<T, NT>(sl, buf, &bar);
    if (parts > 1) cluster_arrive_relaxed();            // this block runs, its barriers exist
    if (j < kMaxList) {
        mine = listed_id >= 0 && listed_id < a.vocab && (a.rest || lq != kNegInf) ? (int)listed_id : -1;
        if (mine < 0) lq = kNegInf;
        id[j] = mine;
        if (!a.rest) {
            const float m = warp_max(lq);
            if (lane == 0) top32[j >> 5] = m;
        }
    }
    const float g = a.dz ? a.dloss[row] * a.inv_temperature : 0.0f;
    __syncthreads();
    bool again = false;
    if (j < kMaxList) {
        float top = 0.0f;
        if (!a.rest) {
            top = fmaxf(fmaxf(top32[0], top32[1]), fmaxf(top32[2], top32[3]));
            if (top == kNegInf) top = 0.0f;
        }
        if (mine >= 0) {
            q = exp((double)lq - (double)top);
#pragma unroll 4
            for (int i = 0; i < j; i += 4) {
                const int4 d = *reinterpret_cast<const int4 *>(id + i);
                again |= (d.x == mine) | (d.y == mine && i + 1 < j) | (d.z == mine && i + 2 < j) | (d.w == mine && i + 3 < j);
            }
            if (again) repeated = 1;
        }
        w[j] = q;
        listed[j] = mine >= 0 && !again;
        const double sum = warp_sum64(q);
        if (lane == 0) sum64[0][j >> 5] = sum;
    }
    const bool first = mine >= 0 && !again, here = first && mine >= sl.start && mine < sl.start + sl.nv * V;
    bool late = !mbar_wait_bounded(&bar, 0, a.wait_limit);
    if (late) mbar_wait_bounded(&bar, 0);
    const int used = __syncthreads_count(first);
    float zj = kNegInf;
    if (here) {
        zj = widen(elem[mine - sl.start]);
        elem[mine - sl.start] = minus_inf<T>();
    }
    __syncthreads();
    const float s = (float)a.scale2;
    const float m = block_max_all<NT>(late ? kLate : slice_max<T, NT>(buf, sl.nv), sh[0]);
    const Origin own(m, s);
    float e = own.far ? slice_sum<T, NT, true>(buf, sl.nv, own, s) : slice_sum<T, NT, false>(buf, sl.nv, own, s);
    e = block_sum_all<NT>(e, sh[1]);

    // every block learns the others' sums and the listed tokens' logits
    if (parts > 1) {
        cluster_wait();
        if (j == 0) mbar_arrive_expect_tx(&told, (uint32_t)(parts * sizeof(Rest) + used * sizeof(float)));
        for (int i = 0; i < parts; ++i) {
            if (here) send32(&zl[j], i, &told, zj);
            if (j == i) send64(&rest_sh[part], i, &told, m, e);
        }
    } else {
        if (here) zl[j] = zj;
        if (j == 0) rest_sh[0] = Rest{m, e};
    }
    // meanwhile the teacher's weights of this thread's entry
    if (repeated && mine >= 0) {
        if (again) q = 0.0;
        else
            for (int i = j + 1; i < k; ++i)
                if (id[i] == mine) q += w[i];
    }
    const double mass = (sum64[0][0] + sum64[0][1]) + (sum64[0][2] + sum64[0][3]);
    if (!a.rest && mass != 0.0) q /= mass;
    const double r = !a.rest || used >= a.vocab ? 0.0 : mass != mass ? mass : fmax(0.0, 1.0 - mass);
    if (parts > 1) {
        if (!wait_told(&told, a.wait_limit)) {
            late = true;
            wait_told(&told, kWaitLimit);
        }
    } else {
        __syncthreads();
    }

    // Rest and list, each relative to its own origin; then both relative to the larger.  Every warp
    // does this for itself.
    const Rest mine_rest = rest_sh[lane < parts ? lane : 0];
    const float mr = warp_max(mine_rest.m);
    float zk[kWarps], ml = kNegInf;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) {
        zk[i] = listed[lane + 32 * i] ? zl[lane + 32 * i] : kNegInf;
        ml = fmaxf(ml, zk[i]);
    }
    ml = warp_max(ml);
    const Origin rest(mr, s), top(fmaxf(mr, ml), s);
    const float mlu = ml == kNegInf ? 0.0f : ml;
    float er = mine_rest.e != mine_rest.e ? mine_rest.e : mine_rest.e == 0.0f || lane >= parts ? 0.0f
        : exp2_fast(shift(Origin(mine_rest.m, s), rest, s)) * mine_rest.e;
    float el = 0.0f;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) el += zk[i] == kNegInf ? 0.0f : exp2_fast((zk[i] - mlu) * s);
    er = warp_sum(er);
    el = warp_sum(el);
    const bool bad = late || er != er || el != el || fmaxf(mr, ml) > 3.402823466e38f, empty = !bad && fmaxf(mr, ml) == kNegInf;
    // the list's sum is relative to ml s, the origin's c is rounded: exponents of the difference
    const float fr = er == 0.0f ? 0.0f : exp2_fast(shift(rest, top, s)), fl = el == 0.0f ? 0.0f
        : exp2_fast(top.far ? (mlu - top.m) * s : fmaf(mlu, s, -top.c));
    const float E = fmaf(fr, er, fl * el);

    if (a.dz) {
        const bool zero = g == 0.0f || empty || (used == 0 && !bad);
        const float others = er == 0.0f ? 0.0f : g * (fr / E - (float)r / er);
        if (zero || bad || !(fabsf(others) < __builtin_huge_valf())) {      // (0 times infinity is no masked logit's gradient)
            const float all = zero ? 0.0f : bad ? NAN : others;
            for (int v = threadIdx.x; v < sl.nv; v += NT) {
                float2 f[V / 2];
                Vec<T>::wide(buf[v], f);
#pragma unroll
                for (int i = 0; i < V / 2; ++i) f[i] = make_float2(f[i].x == kNegInf ? 0.0f : all, f[i].y == kNegInf ? 0.0f : all);
                buf[v] = Vec<T>::pack(f);
            }
        } else if (rest.far) {
            slice_gradient<T, NT, true>(buf, sl.nv, rest, s, others);
        } else {
            slice_gradient<T, NT, false>(buf, sl.nv, rest, s, others);
        }
        __syncthreads();
        if (here) {
            const float t = top.far ? (zj - top.m) * s : fmaf(zj, s, -top.c);
            const float d = zero || zj == kNegInf ? 0.0f : bad ? NAN : g * (exp2_fast(t) / E - (float)q);
            elem[mine - sl.start] = narrow<T>(d);
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");    // the bulk copy reads what the threads wrote
        __syncthreads();
        T *out = static_cast<T *>(a.dz) + row * a.dz_stride;
        const int lo = max(0, sl.start), hi = min(sl.vocab, sl.start + sl.nv * V);     // columns of the slice
        if ((((uintptr_t)out - (uintptr_t)sl.row) & 15) == 0) {
            const int v0 = sl.nv > 0 && !sl.whole(0) ? 1 : 0, v1 = sl.nv > v0 && !sl.whole(sl.nv - 1) ? sl.nv - 1 : sl.nv;
            if (threadIdx.x == 0 && v1 > v0) {
                asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;\n"
                             "cp.async.bulk.commit_group;" ::"l"(out + sl.start + v0 * V), "r"(smem_addr(buf + v0)),
                             "r"((v1 - v0) * 16) : "memory");
            }
            if (threadIdx.x < 2 * V) {                                  // a first and a last vector that are not whole
                const int v = threadIdx.x < V ? 0 : sl.nv - 1, c = sl.start + v * V + (int)threadIdx.x % V;
                if ((threadIdx.x < V ? v0 == 1 : v1 < sl.nv) && c >= lo && c < hi) out[c] = elem[c - sl.start];
            }
        } else {
            for (int c = lo + threadIdx.x; c < hi; c += NT) out[c] = elem[c - sl.start];
        }
    }
    if (part == 0 && a.loss) {
        if (j < kMaxList) {
            // relative to `top` and in 64 bits: the only roundings are those of the sums
            const double l2 = log2((double)E);
            double t = 0.0;
            if (first && !(q == 0.0)) t = q * (log(q) - (exponent64(zl[j], top, s) - l2) * kLn2);
            if (j == 0 && r > 0.0) {
                t += r * (log(r) - (rest.at(s) - top.at(s) + log2((double)er) - l2) * kLn2);
            }
            if (j == 0 && r != r) t = r;
            t = warp_sum64(t);
            if (lane == 0) sum64[1][j >> 5] = t;
        }
        __syncthreads();
        if (j == 0)
            a.loss[row] = bad ? NAN : used == 0 ? 0.0f : empty ? INFINITY
                : (float)((sum64[1][0] + sum64[1][1]) + (sum64[1][2] + sum64[1][3]));
    }
    if (a.dz && threadIdx.x == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
}

// ---------------------------------------------------------------------------------------------
// Launches
// ---------------------------------------------------------------------------------------------
constexpr int kSliceBytes = 32 * 1024;           // six blocks share an SM
// Slices of the forward pass up to this: blocks of 128 threads instead of 256.  bf16, us with 128 / 256
// threads, without alternatives and with 64: 40000 x 1000 134/275, 428/686; 8192 x 4001 31/62, 88/139;
// 4096 x 30522 54/61, 104/112; 2000 x 131072 95/92, 145/129; 1000 x 250000 88/92, 169/134.
constexpr int64_t kShortSlice = 64 * 1024;

// Blocks per row of the forward pass, as a power of two: one where the rows alone fill the GPU
// (two for each SM); fewer rows are shared by up to 8 blocks of at least 8 KB.  bf16, us with / without
// sharing, 0 and 20 alternatives: 1 x 30522 9.7/10.2, 10.3/12.3; 8 x 131072 8.9/12.0, 12.3/17.0; 64 x 131072
// 11.2/15.1, 16.5/21.4; 200 x 30522 9.3/10.8, 14.1/15.8; 250 x 131072 18.7/18.1, 26.3/26.6.
static int log_parts_for_rows(int64_t rows, int64_t bytes)
{
    int n = 0;
    while (n < 3 && rows << n < 2 * 148 && bytes >> (n + 1) >= 8 * 1024) ++n;
    return n;
}

// Blocks per row where the row is held in shared memory: as few as hold it in slices of 32 KB, up
// to 8.  (Slices of 64 KB and 256 threads, three to an SM: 0.442 instead of 0.412 ms for 4096 x
// 131072 bf16, each block waits for its cluster and its barriers as long as a smaller one.)
static int log_parts_for_slices(int64_t bytes)
{
    int n = 0;
    while (n < 3 && ((bytes - 1) >> n) + 1 > kSliceBytes) ++n;
    return n;
}

template <typename F>
static void launch_rows(F kernel, int64_t rows, int parts, int threads, size_t smem, cudaStream_t st, const void *args[])
{
    allow_shared(kernel, smem);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(rows * parts));
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = (unsigned)parts;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = parts > 1 ? 1 : 0;
    cudaLaunchKernelExC(&cfg, reinterpret_cast<const void *>(kernel), const_cast<void **>(args));
}

// The grid holds at most 2^31 - 1 blocks: more rows go in several launches.
template <typename F>
static void for_row_blocks(int64_t rows, int parts, F f)
{
    const int64_t most = 0x7fffffff / parts;
    for (int64_t at = 0; at < rows; at += most) f(at, rows - at < most ? rows - at : most);
}

template <typename T, int NT>
static void logprobs(const Logprobs &a, int log_parts, cudaStream_t st)
{
    const int parts = 1 << log_parts;
    int rounds = (int)((slice_bytes<T>(a.vocab, parts) / 16 + kBatch * NT - 1) / (kBatch * NT));
    const size_t smem = a.k ? 2 * kBatch * NT * 16 + kCap * 16 + (size_t)(rounds + 2) * NT * 2 + (size_t)parts * a.k * 8 : 0;
    for_row_blocks(a.rows, parts, [&](int64_t at, int64_t n) {
        Logprobs b = a;
        b.z = static_cast<const T *>(a.z) + at * a.stride;
        b.tokens = a.tokens ? static_cast<const char *>(a.tokens) + at * (a.index64 ? 8 : 4) : nullptr;
        if (a.logprob) b.logprob += at;
        if (a.entropy) b.entropy += at;
        if (a.lse) b.lse += at;
        if (a.k) {
            b.top_ids = static_cast<char *>(a.top_ids) + at * a.k * (a.index64 ? 8 : 4);
            b.top_logprobs += at * a.k;
        }
        const void *args[] = {&b, &log_parts, &rounds};
        if (a.k) launch_rows(k_logprobs<T, NT, true>, n, parts, NT, smem, st, args);
        else launch_rows(k_logprobs<T, NT, false>, n, parts, NT, smem, st, args);
    });
}

template <typename T>
static void logprobs(const Logprobs &a, cudaStream_t st)
{
    const int64_t bytes = a.vocab * (int64_t)sizeof(T);
    const int log_parts = log_parts_for_rows(a.rows, bytes);
    if (bytes >> log_parts <= kShortSlice) logprobs<T, 128>(a, log_parts, st);
    else logprobs<T, 256>(a, log_parts, st);
}

template <typename T>
static void distill(const Distill &a, cudaStream_t st)
{
    int log_parts = log_parts_for_slices(a.vocab * (int64_t)sizeof(T)), parts = 1 << log_parts;
    const size_t smem = slice_bytes<T>(a.vocab, parts);
    for_row_blocks(a.rows, parts, [&](int64_t at, int64_t n) {
        Distill b = a;
        if (a.wait_limit < 0) b.wait_limit = kWaitLimit;
        b.z = static_cast<const T *>(a.z) + at * a.stride;
        b.ids = static_cast<const char *>(a.ids) + at * a.k * (a.index64 ? 8 : 4);
        b.teacher += at * a.k;
        if (a.dloss) b.dloss += at;
        if (a.loss) b.loss += at;
        if (a.dz) b.dz = static_cast<T *>(a.dz) + at * a.dz_stride;
        const void *args[] = {&b, &log_parts};
        // longer slices than 48 KB (8 blocks do not hold the row in less): 256 threads; us with them / with 128:
        // 2000 x 131072 f32 402/424, 1000 x 393216 bf16 385/430, 700 x 393216 f32 653/749
        if (smem > 48 * 1024) launch_rows(k_distill<T, 256>, n, parts, 256, smem, st, args);
        else launch_rows(k_distill<T, 128>, n, parts, 128, smem, st, args);
    });
}

void launch_token_logprobs(const Logprobs &a, int type, cudaStream_t st)
{
    if (type == 0) logprobs<float>(a, st);
    else if (type == 1) logprobs<bf16>(a, st);
    else logprobs<f16>(a, st);
}

void launch_distill(const Distill &a, int type, cudaStream_t st)
{
    if (type == 0) distill<float>(a, st);
    else if (type == 1) distill<bf16>(a, st);
    else distill<f16>(a, st);
}

template <typename T>
static void logprobs_backward(const LogprobsBackward &a, cudaStream_t st)
{
    constexpr int V = Vec<T>::n;
    constexpr int NT = 128;
    const int64_t vecs = (a.vocab + 2 * V - 2) / V;
    const int chunks = (int)((vecs + NT * kGradVecs - 1) / (NT * kGradVecs));
    for_row_blocks(a.rows, chunks, [&](int64_t at, int64_t n) {
        LogprobsBackward b = a;
        b.z = static_cast<const T *>(a.z) + at * a.stride;
        b.dz = static_cast<T *>(a.dz) + at * a.dz_stride;
        b.tokens = a.tokens ? static_cast<const char *>(a.tokens) + at * (a.index64 ? 8 : 4) : nullptr;
        b.lse += at;
        if (a.entropy) b.entropy += at;
        if (a.dlogprob) b.dlogprob += at;
        if (a.dentropy) b.dentropy += at;
        k_logprobs_backward<T, NT><<<(unsigned)(n * chunks), NT, 0, st>>>(b, chunks);
    });
}

void launch_token_logprobs_backward(const LogprobsBackward &a, int type, cudaStream_t st)
{
    if (type == 0) logprobs_backward<float>(a, st);
    else if (type == 1) logprobs_backward<bf16>(a, st);
    else logprobs_backward<f16>(a, st);
}

}  // namespace cdadam
