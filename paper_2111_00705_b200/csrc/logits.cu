// Operators on rows of logits: log probabilities of given tokens with entropy and the most
// probable alternatives, its gradient, and distillation from a teacher's listed tokens.
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

// One block per row.
template <typename T>
__global__ void __launch_bounds__(kRowBlock) k_logprobs(Logprobs a)
{
    __shared__ float sh[3][kRowBlock / 32];
    __shared__ unsigned long long best;
    const int64_t row = blockIdx.x;
    const T *z = static_cast<const T *>(a.z) + row * a.stride;
    const float s = (float)a.scale2;
    float m = kNegInf;
    for (int64_t i = threadIdx.x; i < a.vocab; i += kRowBlock) m = fmaxf(m, widen(z[i]));
    m = block_max_all<kRowBlock>(m, sh[0]);
    const float mu = m == kNegInf ? 0.0f : m;
    float e = 0.0f, h = 0.0f;
    for (int64_t i = threadIdx.x; i < a.vocab; i += kRowBlock) {
        const float t = fmaxf((widen(z[i]) - mu) * s, -1e4f), p = widen(z[i]) == widen(z[i]) ? exp2f(t) : NAN;
        e += p;
        h = fmaf(p, t, h);
    }
    e = block_sum_all<kRowBlock>(e, sh[1]);
    h = block_sum_all<kRowBlock>(h, sh[2]);
    const bool none = e != e || m > 3.402823466e38f, empty = !none && e == 0.0f;
    const double l2 = empty ? (double)kNegInf : none ? (double)NAN : log2((double)e);
    if (threadIdx.x == 0) {
        if (a.logprob) {
            const int64_t t = index_at(a.tokens, row, a.index64);
            a.logprob[row] = t < 0 ? 0.0f : t >= a.vocab || none ? NAN : empty ? kNegInf
                : (float)((((double)widen(z[t]) - mu) * (double)s - l2) * kLn2);
        }
        if (a.entropy) a.entropy[row] = empty ? 0.0f : (float)((l2 - (double)h / (double)e) * kLn2);
        if (a.lse) a.lse[row] = (float)((double)mu * (a.scale2 * kLn2) + l2 * kLn2);
    }
    if (!a.top_ids) return;
    uint64_t last = ~0ull;
    for (int j = 0; j < a.k; ++j) {
        __syncthreads();
        if (threadIdx.x == 0) best = 0;
        __syncthreads();
        unsigned long long mine = 0;
        if (!none)
            for (int64_t i = threadIdx.x; i < a.vocab; i += kRowBlock) {
                const float v = widen(z[i]);
                const uint64_t key = order_key(v, (int32_t)i);
                if (v > kNegInf && key < last && key > mine) mine = key;
            }
        atomicMax(&best, mine);
        __syncthreads();
        last = best;
        if (threadIdx.x == 0) {
            const bool got = last != 0;
            store_index(a.top_ids, row * a.k + j, a.index64, got ? key_index(last) : -1);
            a.top_logprobs[row * a.k + j] = none ? NAN : !got ? kNegInf
                : (float)((((double)key_value(last) - mu) * (double)s - l2) * kLn2);
        }
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

// One block per row.
template <typename T>
__global__ void __launch_bounds__(kRowBlock) k_distill(Distill a)
{
    __shared__ float sh[4][kRowBlock / 32];
    __shared__ int32_t id[kMaxList];
    __shared__ double lq[kMaxList], q[kMaxList], list[3];
    __shared__ float zl[kMaxList];
    const int64_t row = blockIdx.x;
    const T *z = static_cast<const T *>(a.z) + row * a.stride;
    const float s = (float)a.scale2;
    const int k = a.k;
    for (int j = threadIdx.x; j < k; j += kRowBlock) {
        const int64_t i = index_at(a.ids, row * k + j, a.index64);
        id[j] = i >= 0 && i < a.vocab ? (int32_t)i : -1;
        lq[j] = (double)a.teacher[row * k + j];
        if (!a.rest && lq[j] == (double)kNegInf) id[j] = -1;
        zl[j] = id[j] >= 0 ? widen(z[id[j]]) : 0.0f;
    }
    __syncthreads();
    // the teacher's distribution over the list, an index listed twice taken together
    if (threadIdx.x == 0) {
        double top = -INFINITY, sum = 0.0, mass = 0.0;
        for (int j = 0; j < k; ++j) if (id[j] >= 0) top = fmax(top, lq[j]);
        if (a.rest || top == -INFINITY) top = 0.0;
        for (int j = 0; j < k; ++j) if (id[j] >= 0) sum += exp(lq[j] - top);
        const double norm = a.rest || sum == 0.0 ? 0.0 : top + log(sum);
        int used = 0;
        for (int j = 0; j < k; ++j) {
            if (id[j] < 0) continue;
            double v = exp(lq[j] - norm);
            lq[j] -= norm;
            for (int i = j + 1; i < k; ++i)
                if (id[i] == id[j]) { v += exp(lq[i] - norm); id[i] = -1; lq[j] = log(v); }
            q[j] = v;
            mass += v;
            ++used;
        }
        list[0] = a.rest && used < a.vocab ? fmax(0.0, 1.0 - mass) : 0.0;
        if (mass != mass) list[0] = mass;
        list[1] = mass;
        list[2] = used;
    }
    __syncthreads();
    const double r = list[0];
    // the student: listed tokens and all others apart, each relative to its own maximum
    float mr = kNegInf, ml = kNegInf;
    for (int64_t i = threadIdx.x; i < a.vocab; i += kRowBlock) {
        bool in = false;
        for (int j = 0; j < k; ++j) in |= id[j] == i;
        const float v = widen(z[i]);
        if (in) ml = fmaxf(ml, v); else mr = fmaxf(mr, v);
    }
    mr = block_max_all<kRowBlock>(mr, sh[0]);
    ml = block_max_all<kRowBlock>(ml, sh[1]);
    const float mru = mr == kNegInf ? 0.0f : mr, mlu = ml == kNegInf ? 0.0f : ml;
    float er = 0.0f, el = 0.0f;
    for (int64_t i = threadIdx.x; i < a.vocab; i += kRowBlock) {
        bool in = false;
        for (int j = 0; j < k; ++j) in |= id[j] == i;
        const float v = widen(z[i]);
        if (in) el += exp2f((v - mlu) * s); else er += exp2f((v - mru) * s);
    }
    er = block_sum_all<kRowBlock>(er, sh[2]);
    el = block_sum_all<kRowBlock>(el, sh[3]);
    const double rest2 = er == 0.0f ? (double)kNegInf : (double)mru * (double)s + log2((double)er);
    const double list2 = el == 0.0f ? (double)kNegInf : (double)mlu * (double)s + log2((double)el);
    const double top2 = fmax(rest2, list2);
    double lse2 = top2 == (double)kNegInf ? top2 : top2 + log2(exp2(rest2 - top2) + exp2(list2 - top2));
    if (er != er || el != el || fmaxf(mr, ml) > 3.402823466e38f) lse2 = NAN;
    if (threadIdx.x == 0 && a.loss) {
        double loss = 0.0;
        for (int j = 0; j < k; ++j)
            if (id[j] >= 0 && !(q[j] == 0.0)) loss += q[j] * (lq[j] - ((double)zl[j] * (double)s - lse2) * kLn2);
        if (r > 0.0) loss += r * (log(r) - (rest2 - lse2) * kLn2);
        if (lse2 != lse2) loss = NAN;
        else if (list[2] == 0.0) loss = 0.0;
        else if (top2 == (double)kNegInf) loss = INFINITY;
        a.loss[row] = (float)loss;
    }
    if (!a.dz) return;
    T *dz = static_cast<T *>(a.dz) + row * a.dz_stride;
    const double g = (double)a.dloss[row] * (double)a.inv_temperature;
    // p_i (1 - r / R) = 2^(z_i s - rest2) (2^(rest2 - lse2) - r), from the maximum of the others
    const double share = rest2 == (double)kNegInf ? 0.0 : (exp2(rest2 - lse2) - r) / (double)er;
    const float others = list[2] == 0.0 && lse2 == lse2 ? 0.0f : (float)(g * share);
    for (int64_t i = threadIdx.x; i < a.vocab; i += kRowBlock) {
        int at = -1;
        for (int j = 0; j < k; ++j) if (id[j] == i) at = j;
        const float v = widen(z[i]);
        float d;
        if (at < 0) d = others * exp2f((v - mru) * s);
        else d = (float)(g * (exp2((double)v * (double)s - lse2) - q[at]));
        dz[i] = narrow<T>(v == kNegInf || g == 0.0 ? 0.0f : d);
    }
}

void launch_token_logprobs(const Logprobs &a, int type, cudaStream_t st)
{
    const unsigned g = (unsigned)a.rows;
    if (g == 0) return;
    if (type == 0) k_logprobs<float><<<g, kRowBlock, 0, st>>>(a);
    else if (type == 1) k_logprobs<bf16><<<g, kRowBlock, 0, st>>>(a);
    else k_logprobs<f16><<<g, kRowBlock, 0, st>>>(a);
}

void launch_token_logprobs_backward(const LogprobsBackward &a, int type, cudaStream_t st)
{
    const unsigned g = (unsigned)a.rows;
    if (g == 0) return;
    if (type == 0) k_logprobs_backward<float><<<g, kRowBlock, 0, st>>>(a);
    else if (type == 1) k_logprobs_backward<bf16><<<g, kRowBlock, 0, st>>>(a);
    else k_logprobs_backward<f16><<<g, kRowBlock, 0, st>>>(a);
}

void launch_distill(const Distill &a, int type, cudaStream_t st)
{
    const unsigned g = (unsigned)a.rows;
    if (g == 0 || (!a.loss && !a.dz)) return;
    if (type == 0) k_distill<float><<<g, kRowBlock, 0, st>>>(a);
    else if (type == 1) k_distill<bf16><<<g, kRowBlock, 0, st>>>(a);
    else k_distill<f16><<<g, kRowBlock, 0, st>>>(a);
}

}  // namespace cdadam
