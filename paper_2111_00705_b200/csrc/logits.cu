// Operators on rows of logits: log probabilities of given tokens with entropy and the most
// probable alternatives, its gradient, and distillation from a teacher's listed tokens.
//
// A row of logits is what bounds all three: each has to be read once, and its gradient written
// once.  The sums need the row's maximum first, the gradient needs the sums, so a row is
// worked on two or three times.  To read it from memory once it is held on the chip: a
// thread-block cluster of 1, 2, 4 or 8 blocks takes a row, every block a slice of it in its
// shared memory, and the blocks exchange a few sums through distributed shared memory.
#include <cooperative_groups.h>

#include "elements.cuh"

namespace cdadam {

constexpr int kRowBlock = 256;
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

    __device__ __forceinline__ Slice(const void *z, int64_t stride, int64_t r, int64_t n, int part, int parts)
    {
        row = static_cast<const T *>(z) + r * stride;
        vocab = (int)n;
        off = (int)(((uintptr_t)row & 15) / sizeof(T));
        const int nvec = (off + vocab + V - 1) / V, per = (nvec + parts - 1) / parts, first = part * per;
        nv = max(0, min(per, nvec - first));
        start = first * V - off;
    }
    __device__ __forceinline__ bool whole(int v) const
    {
        const int c = start + v * V;
        return c >= 0 && c + V <= vocab;
    }
};

template <typename T, int NT>
__device__ __forceinline__ void load_slice(const Slice<T> &s, uint4 *buf)
{
    constexpr int V = Vec<T>::n;
    for (int v = threadIdx.x; v < s.nv; v += NT) {
        const int c = s.start + v * V;
        if (s.whole(v)) {
            copy16(buf + v, s.row + c);
        } else {
            T *e = reinterpret_cast<T *>(buf + v);
#pragma unroll
            for (int i = 0; i < V; ++i) e[i] = c + i >= 0 && c + i < s.vocab ? s.row[c + i] : minus_inf<T>();
        }
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

// Sums of a slice: e = sum 2^t, h = sum 2^t t with t = (z - mu) s.
struct Sums {
    float m, e, h;
    int n;                  // entries of the slice's list of alternatives
};

// ---------------------------------------------------------------------------------------------
// Alternatives.  Every slice gives its k first tokens in descending order, the cluster's first
// block merges them.  Within a slice: 128 groups of threads have each met a largest value; the
// k-th largest of these 128 is a value that at least k elements reach, and in a row without
// structure hardly more (128 ln(128 / (128 - k)) are expected: 89 for k = 64).  The pass that
// adds up the exponentials collects the elements that reach it, and counting for each how many
// are greater sorts them.  Only where more than kCap are collected (thousands of equal values, or
// the largest all in a few threads' vectors) the slice is walked again in order, the best k so
// far always kept.
// ---------------------------------------------------------------------------------------------
constexpr int kCap = 512;
constexpr int kGroups = 128;

template <typename T>
__device__ __forceinline__ void collect(const uint4 &u, int c, float reach, uint64_t *cand, int *count, uint64_t above)
{
    float2 f[Vec<T>::n / 2];
    Vec<T>::wide(u, f);
#pragma unroll
    for (int i = 0; i < Vec<T>::n; ++i) {
        const float v = i & 1 ? f[i / 2].y : f[i / 2].x;
        if (v >= reach && v > kNegInf) {
            const uint64_t key = order_key(v, c + i);
            if (key > above) {
                const int at = atomicAdd(count, 1);
                if (at < kCap) cand[at] = key;
            }
        }
    }
}

__device__ __forceinline__ int rank_of(uint64_t key, const uint64_t *keys, int n)
{
    int r = 0;
#pragma unroll 8
    for (int i = 0; i < n; ++i) r += keys[i] > key;
    return r;
}

template <typename T, int NT>
__device__ __noinline__ int collect_in_order(const uint4 *buf, int nv, int start, int k, uint64_t *cand, int *count)
{
    constexpr int V = Vec<T>::n, step = (kCap - kMaxList) / V, per = (kCap + NT - 1) / NT;
    static_assert(step <= NT, "one vector per thread and step");
    int kept = 0;
    uint64_t above = 0;
    for (int base = 0; base < nv; base += step) {
        __syncthreads();
        if (threadIdx.x == 0) *count = kept;
        __syncthreads();
        const int v = base + (int)threadIdx.x;
        if (threadIdx.x < step && v < nv) collect<T>(buf[v], start + v * V, kNegInf, cand, count, above);
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

template <typename T, int NT, bool TOP>
__global__ void __launch_bounds__(NT) k_logprobs(Logprobs a, int parts, int slice)
{
    constexpr int V = Vec<T>::n;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ float sh[3][NT / 32], reach_sh;
    __shared__ __align__(16) float group[kGroups];
    __shared__ Sums sums[kMaxParts];
    __shared__ int count;
    uint4 *buf = reinterpret_cast<uint4 *>(smem);
    uint64_t *cand = reinterpret_cast<uint64_t *>(smem + slice);    // kCap keys; before that every thread's maximum
    uint64_t *lists = cand + kCap;                                  // first block: parts x k keys
    const int part = (int)(blockIdx.x % (unsigned)parts);
    const int64_t row = blockIdx.x / (unsigned)parts;
    cg::cluster_group cluster = cg::this_cluster();
    if (parts > 1) cluster_arrive();        // the first block runs before anything is written to it

    const Slice<T> sl(a.z, a.stride, row, a.vocab, part, parts);
    load_slice<T, NT>(sl, buf);
    copies_done();
    float m = slice_max<T, NT>(buf, sl.nv);
    if (TOP) reinterpret_cast<float *>(cand)[threadIdx.x] = m;
    m = block_max_all<NT>(m, sh[0]);
    float reach = 0.0f;
    if (TOP) {
        if (threadIdx.x < kGroups) {
            const float *all = reinterpret_cast<const float *>(cand);
            float g = all[threadIdx.x];
#pragma unroll
            for (int i = kGroups; i < NT; i += kGroups) g = fmaxf(g, all[threadIdx.x + i]);
            group[threadIdx.x] = g;
            asm volatile("bar.sync 1, %0;" ::"n"(kGroups) : "memory");
            int gt = 0, ge = 0;
#pragma unroll 8
            for (int i = 0; i < kGroups; i += 4) {
                const float4 q = *reinterpret_cast<const float4 *>(group + i);
                gt += (q.x > g) + (q.y > g) + (q.z > g) + (q.w > g);
                ge += (q.x >= g) + (q.y >= g) + (q.z >= g) + (q.w >= g);
            }
            if (gt < a.k && a.k <= ge) reach_sh = g;
            if (threadIdx.x == 0) count = 0;
        }
        __syncthreads();
        reach = reach_sh;
    }

    const float s = (float)a.scale2, mu = m == kNegInf ? 0.0f : m;
    const typename Vec<T>::running reach2 = Vec<T>::all(reach);
    float2 e2 = both(0.0f), h2 = both(0.0f);
#pragma unroll 2
    for (int v = threadIdx.x; v < sl.nv; v += NT) {
        const uint4 u = buf[v];
        float2 f[V / 2];
        Vec<T>::wide(u, f);
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
            const float2 t = mul2(add2(f[i], both(-mu)), both(s));
            const float2 p = make_float2(exp2_fast(t.x), exp2_fast(t.y));
            e2 = add2(e2, p);
            h2 = fma2(p, make_float2(fmaxf(t.x, -1e4f), fmaxf(t.y, -1e4f)), h2);   // 0 times -inf is 0 here
        }
        if (TOP && Vec<T>::reaches(Vec<T>::top(u), reach2)) collect<T>(u, sl.start + v * V, reach, cand, &count, 0);
    }
    float e = warp_sum(e2.x + e2.y), h = warp_sum(h2.x + h2.y);
    if ((threadIdx.x & 31) == 0) { sh[1][threadIdx.x >> 5] = e; sh[2][threadIdx.x >> 5] = h; }
    __syncthreads();
    int n = 0;
    if (TOP) {
        n = count;
        if (n > kCap) n = collect_in_order<T, NT>(buf, sl.nv, sl.start, a.k, cand, &count);
        __syncthreads();
    }
    if (parts > 1) cluster_wait();
    uint64_t *list = parts > 1 ? cluster.map_shared_rank(lists, 0) : lists;
    if (TOP)
        for (int i = threadIdx.x; i < n; i += NT) {
            const uint64_t key = cand[i];
            const int r = rank_of(key, cand, n);
            if (r < a.k) list[part * a.k + r] = key;
        }
    if (threadIdx.x < 32) {
        e = warp_sum(threadIdx.x < NT / 32 ? sh[1][threadIdx.x] : 0.0f);
        h = warp_sum(threadIdx.x < NT / 32 ? sh[2][threadIdx.x] : 0.0f);
        if (threadIdx.x == 0) {
            Sums *to = parts > 1 ? cluster.map_shared_rank(sums, 0) : sums;
            to[part] = Sums{m, e, h, min(n, a.k)};
        }
    }
    if (parts > 1) {
        cluster_arrive();
        if (part != 0) return;                       // nothing reads this block's shared memory
        cluster_wait();
    } else {
        __syncthreads();
    }

    // the row: slices relative to the row's maximum
    const int todo = TOP ? max(1, parts * a.k) : 1;
    if ((int)(threadIdx.x & ~31u) >= max(todo, a.k)) return;
    float M = kNegInf, E = 0.0f, H = 0.0f;
    int total = 0;
    for (int i = 0; i < parts; ++i) { M = fmaxf(M, sums[i].m); total += sums[i].n; }
    const float Mu = M == kNegInf ? 0.0f : M;
    for (int i = 0; i < parts; ++i) {
        const Sums p = sums[i];
        if (p.e == 0.0f) continue;                   // all masked
        const float d = fmaxf((p.m - Mu) * s, -1e4f), f = p.m == kNegInf ? 1.0f : exp2_fast(d);
        E = fmaf(f, p.e, E);
        H += f * fmaf(d, p.e, p.h);
    }
    const bool none = E != E || M > 3.402823466e38f, empty = !none && E == 0.0f;
    const double l2 = none ? (double)NAN : empty ? (double)kNegInf : log2((double)E);
    if (threadIdx.x == 0) {
        if (a.logprob) {
            const int64_t t = index_at(a.tokens, row, a.index64);
            a.logprob[row] = t < 0 ? 0.0f : t >= a.vocab || none ? NAN : empty ? kNegInf
                : (float)((((double)widen(sl.row[t]) - (double)Mu) * (double)s - l2) * kLn2);
        }
        if (a.entropy) a.entropy[row] = empty ? 0.0f : (float)((l2 - (double)H / (double)E) * kLn2);
        if (a.lse) a.lse[row] = (float)((double)Mu * (a.scale2 * kLn2) + l2 * kLn2);
    }
    if (!TOP) return;
    for (int t = threadIdx.x; t < parts * a.k; t += NT) {
        const int r = t / a.k, j = t - r * a.k;
        if (none || j >= sums[r].n) continue;
        const uint64_t key = lists[t];
        int at = j;
        for (int o = 0; o < parts; ++o) {
            if (o == r) continue;
            int lo = 0, hi = sums[o].n;              // first entry of list o that is not greater
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                if (lists[o * a.k + mid] > key) lo = mid + 1; else hi = mid;
            }
            at += lo;
        }
        if (at < a.k) {
            store_index(a.top_ids, row * a.k + at, a.index64, key_index(key));
            a.top_logprobs[row * a.k + at] = (float)((((double)key_value(key) - (double)Mu) * (double)s - l2) * kLn2);
        }
    }
    for (int t = threadIdx.x; t < a.k; t += NT)
        if (none || t >= total) {
            store_index(a.top_ids, row * a.k + t, a.index64, -1);
            a.top_logprobs[row * a.k + t] = none ? NAN : kNegInf;
        }
}

// One block per row.  dz_i = (g ([i = token] - p_i) - u p_i (log p_i + H)) / T.
template <typename T>
__global__ void __launch_bounds__(kRowBlock) k_logprobs_backward(LogprobsBackward a)
{
    const int64_t row = blockIdx.x;
    const T *z = static_cast<const T *>(a.z) + row * a.stride;
    T *dz = static_cast<T *>(a.dz) + row * a.dz_stride;
    int64_t token = a.dlogprob ? index_at(a.tokens, row, a.index64) : -1;
    if (token >= a.vocab) token = -1;
    const float lse = a.lse[row], g = token >= 0 ? a.dlogprob[row] : 0.0f;
    const float u = a.dentropy ? a.dentropy[row] : 0.0f, H = a.dentropy ? a.entropy[row] : 0.0f;
    const float s = (float)a.scale2;
    const bool still = (g == 0.0f && u == 0.0f) || fabsf(lse) >= 16777216.0f;    // no gradient, or none that lse could give
    const double l2 = (double)lse / kLn2;
    const float hi = (float)l2, lo = lse == kNegInf ? 0.0f : (float)(l2 - (double)hi);
    for (int64_t i = threadIdx.x; i < a.vocab; i += kRowBlock) {
        const float v = widen(z[i]);
        const float t = fmaf(v, s, -hi) - lo, p = exp2f(t);
        const float lp = fmaxf(t, -1e4f) * (float)kLn2;
        float d = -p * fmaf(u, lp + H, g);
        if (i == token) d += g;
        dz[i] = narrow<T>(v == kNegInf || still ? 0.0f : d * a.inv_temperature);
    }
}

// ---------------------------------------------------------------------------------------------
// Distillation.  The listed tokens are taken out of the slice (set to -inf) before its maximum
// and sum are formed, so that the rest of the vocabulary has its own maximum and sum: R comes
// from a sum of positive terms instead of from 1 - sum p_j, and neither part underflows however
// far the other is above it.  The gradient replaces the slice in shared memory, the listed
// tokens' entries are put in afterwards, and the slice leaves as one bulk copy.
// ---------------------------------------------------------------------------------------------
struct Rest {
    float m, e;
};

template <typename T, int NT>
__global__ void __launch_bounds__(NT) k_distill(Distill a, int parts)
{
    constexpr int V = Vec<T>::n, kWarps = kMaxList / 32;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ float sh[2][NT / 32], shm[kWarps], she[kWarps];
    __shared__ int32_t id[kMaxList];
    __shared__ double lq[kMaxList], w[kMaxList], terms[kWarps], mass_sh;
    __shared__ Rest rest_sh[kMaxParts];
    uint4 *buf = reinterpret_cast<uint4 *>(smem);
    T *elem = reinterpret_cast<T *>(smem);
    const int part = (int)(blockIdx.x % (unsigned)parts), j = threadIdx.x, k = a.k;
    const int64_t row = blockIdx.x / (unsigned)parts;
    cg::cluster_group cluster = cg::this_cluster();
    if (parts > 1) cluster_arrive();

    const Slice<T> sl(a.z, a.stride, row, a.vocab, part, parts);
    load_slice<T, NT>(sl, buf);

    // while the slice is on its way, the teacher's distribution over the list: thread j < k has
    // entry j, an index listed twice is taken together by its first entry
    int mine = -1;
    double q = 0.0;
    float zj = kNegInf;
    if (j < k) {
        const int64_t i = index_at(a.ids, row * k + j, a.index64);
        const float t = a.teacher[row * k + j];
        mine = i >= 0 && i < a.vocab && (a.rest || t != kNegInf) ? (int)i : -1;
        if (mine >= 0) zj = widen(sl.row[mine]);
        id[j] = mine;
        lq[j] = mine >= 0 ? (double)t : (double)kNegInf;
    }
    __syncthreads();
    if (j < k) {
        double top = 0.0;
        if (!a.rest) {
            top = (double)kNegInf;
            for (int i = 0; i < k; ++i) top = fmax(top, lq[i]);
            if (top == (double)kNegInf) top = 0.0;
        }
        w[j] = exp(lq[j] - top);
    }
    __syncthreads();
    bool first = mine >= 0;
    if (j < k) {
        double sum = 0.0;
        for (int i = 0; i < k; ++i) {
            sum += w[i];
            if (id[i] == mine) {
                q += w[i];
                if (i < j) first = false;
            }
        }
        if (!a.rest && sum != 0.0) q /= sum;
        if (j == 0) mass_sh = sum;
        if (!first) { q = 0.0; zj = kNegInf; }
    }
    copies_done();
    const int used = __syncthreads_count(first);
    const double mass = mass_sh, r = !a.rest || used >= a.vocab ? 0.0 : mass != mass ? mass : fmax(0.0, 1.0 - mass);
    const float s = (float)a.scale2;
    if (first && mine >= sl.start && mine < sl.start + sl.nv * V) elem[mine - sl.start] = minus_inf<T>();
    if (j < kMaxList) {
        const float m = warp_max(zj), p = zj == kNegInf ? 0.0f : exp2_fast((zj - m) * s);
        const float e = warp_sum(zj != zj ? zj : p);
        if ((j & 31) == 0) { shm[j >> 5] = m; she[j >> 5] = e; }
    }
    __syncthreads();

    float m = block_max_all<NT>(slice_max<T, NT>(buf, sl.nv), sh[0]);
    const float mu = m == kNegInf ? 0.0f : m;
    float2 e2 = both(0.0f);
#pragma unroll 4
    for (int v = threadIdx.x; v < sl.nv; v += NT) {
        float2 f[V / 2];
        Vec<T>::wide(buf[v], f);
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
            const float2 t = mul2(add2(f[i], both(-mu)), both(s));
            e2 = add2(e2, make_float2(exp2_fast(t.x), exp2_fast(t.y)));
        }
    }
    float e = block_sum_all<NT>(e2.x + e2.y, sh[1]);
    if (parts > 1) {
        cluster_wait();
        if (j < parts) cluster.map_shared_rank(rest_sh, j)[part] = Rest{m, e};
        cluster_arrive();
        cluster_wait();
    } else {
        if (j == 0) rest_sh[0] = Rest{m, e};
        __syncthreads();
    }

    // rest and list, each relative to its own maximum; both relative to the larger of these
    float mr = kNegInf, er = 0.0f, ml = kNegInf, el = 0.0f;
    for (int i = 0; i < parts; ++i) mr = fmaxf(mr, rest_sh[i].m);
    for (int i = 0; i < kWarps; ++i) ml = fmaxf(ml, shm[i]);
    const float mru = mr == kNegInf ? 0.0f : mr, mlu = ml == kNegInf ? 0.0f : ml;
    for (int i = 0; i < parts; ++i) {
        const Rest p = rest_sh[i];
        if (p.e != 0.0f) er = fmaf(p.m == kNegInf ? 1.0f : exp2_fast((p.m - mru) * s), p.e, er);
    }
    for (int i = 0; i < kWarps; ++i)
        if (she[i] != 0.0f) el = fmaf(shm[i] == kNegInf ? 1.0f : exp2_fast((shm[i] - mlu) * s), she[i], el);
    const float top = fmaxf(mr, ml);
    const bool bad = er != er || el != el || top > 3.402823466e38f, empty = !bad && top == kNegInf;
    const float fr = er == 0.0f ? 0.0f : exp2_fast((mru - top) * s), fl = el == 0.0f ? 0.0f : exp2_fast((mlu - top) * s);
    const float E = fmaf(fr, er, fl * el);

    const bool loss = part == 0 && a.loss;
    if (loss && j < kMaxList) {
        // relative to `top` and in 64 bits: the only rounding is that of the sums
        const double l2 = log2((double)E);
        double t = 0.0;
        if (first && !(q == 0.0)) t = q * (log(q) - (((double)zj - (double)top) * (double)s - l2) * kLn2);
        if (j == 0 && r > 0.0)
            t += r * (log(r) - (((double)mru - (double)top) * (double)s + log2((double)er) - l2) * kLn2);
        if (j == 0 && r != r) t = r;
#pragma unroll
        for (int d = 16; d >= 1; d >>= 1) t += __shfl_xor_sync(0xffffffffu, t, d);
        if ((j & 31) == 0) terms[j >> 5] = t;
    }

    if (a.dz) {
        const float g = a.dloss[row] * a.inv_temperature;
        const bool zero = g == 0.0f || empty || (used == 0 && !bad);
        const float others = er == 0.0f ? 0.0f : g * (fr / E - (float)r / er);
#pragma unroll 2
        for (int v = threadIdx.x; v < sl.nv; v += NT) {
            float2 f[V / 2];
            Vec<T>::wide(buf[v], f);
#pragma unroll
            for (int i = 0; i < V / 2; ++i) {
                if (zero) f[i] = both(0.0f);
                else if (bad) f[i] = make_float2(f[i].x == kNegInf ? 0.0f : NAN, f[i].y == kNegInf ? 0.0f : NAN);
                else {
                    const float2 t = mul2(add2(f[i], both(-mru)), both(s));
                    f[i] = mul2(make_float2(exp2_fast(t.x), exp2_fast(t.y)), both(others));
                }
            }
            buf[v] = Vec<T>::pack(f);
        }
        __syncthreads();
        if (first && mine >= sl.start && mine < sl.start + sl.nv * V) {
            const float d = zero || zj == kNegInf ? 0.0f : bad ? NAN : g * (exp2_fast((zj - top) * s) / E - (float)q);
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
    } else {
        __syncthreads();
    }
    if (loss && j == 0) {
        double t = 0.0;
        for (int i = 0; i < kWarps; ++i) t += terms[i];
        a.loss[row] = bad ? NAN : used == 0 ? 0.0f : empty ? INFINITY : (float)t;
    }
    if (a.dz && threadIdx.x == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
}

// ---------------------------------------------------------------------------------------------
// Launches
// ---------------------------------------------------------------------------------------------
constexpr int kSliceBytes = 64 * 1024 + 64;      // three blocks share an SM
constexpr int kRowThreads = 256;

// Blocks per row: as few as hold the row in slices of 64 KB.
static int parts_for(int64_t bytes)
{
    int parts = 1;
    while (parts < kMaxParts && (bytes + parts - 1) / parts > kSliceBytes - 64) parts *= 2;
    return parts;
}

template <typename F>
static void launch_rows(F kernel, int64_t rows, int parts, int threads, size_t smem, cudaStream_t st, const void *args[])
{
    cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
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

template <typename T>
static void logprobs(const Logprobs &a, cudaStream_t st)
{
    int parts = parts_for(a.vocab * (int64_t)sizeof(T)), slice = (int)slice_bytes<T>(a.vocab, parts);
    const size_t smem = slice + (a.k ? kCap * 8 + (size_t)parts * a.k * 8 : 0);
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
        const void *args[] = {&b, &parts, &slice};
        if (a.k) launch_rows(k_logprobs<T, kRowThreads, true>, n, parts, kRowThreads, smem, st, args);
        else launch_rows(k_logprobs<T, kRowThreads, false>, n, parts, kRowThreads, smem, st, args);
    });
}

template <typename T>
static void distill(const Distill &a, cudaStream_t st)
{
    int parts = parts_for(a.vocab * (int64_t)sizeof(T));
    const size_t smem = slice_bytes<T>(a.vocab, parts);
    for_row_blocks(a.rows, parts, [&](int64_t at, int64_t n) {
        Distill b = a;
        b.z = static_cast<const T *>(a.z) + at * a.stride;
        b.ids = static_cast<const char *>(a.ids) + at * a.k * (a.index64 ? 8 : 4);
        b.teacher += at * a.k;
        if (a.dloss) b.dloss += at;
        if (a.loss) b.loss += at;
        if (a.dz) b.dz = static_cast<T *>(a.dz) + at * a.dz_stride;
        const void *args[] = {&b, &parts};
        launch_rows(k_distill<T, kRowThreads>, n, parts, kRowThreads, smem, st, args);
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

void launch_token_logprobs_backward(const LogprobsBackward &a, int type, cudaStream_t st)
{
    const unsigned g = (unsigned)a.rows;
    if (g == 0) return;
    if (type == 0) k_logprobs_backward<float><<<g, kRowBlock, 0, st>>>(a);
    else if (type == 1) k_logprobs_backward<bf16><<<g, kRowBlock, 0, st>>>(a);
    else k_logprobs_backward<f16><<<g, kRowBlock, 0, st>>>(a);
}

}  // namespace cdadam
