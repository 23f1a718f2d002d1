// Eight consecutive columns of a row, the unit in which the root-mean-square norm and the 8-bit formats
// take rows: how they are read, written, and turned into the two formats of 8 bits.
#pragma once
#include "elements.cuh"

namespace cdadam {

// A unit as it stands in memory.
template <typename T> struct Raw8 { uint32_t w[2 * sizeof(T)]; };

// Makes the compiler take the unit apart anew, instead of keeping what it is made of.
__device__ __forceinline__ void anew(uint32_t &w) { asm volatile("" : "+r"(w)); }
template <typename T>
__device__ __forceinline__ void anew(Raw8<T> &u)
{
#pragma unroll
    for (int i = 0; i < 2 * (int)sizeof(T); ++i) anew(u.w[i]);
}

template <typename T>
__device__ __forceinline__ void widen8(const Raw8<T> &u, float2 (&f)[4])
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if constexpr (sizeof(T) == 4) f[e] = make_float2(__uint_as_float(u.w[2 * e]), __uint_as_float(u.w[2 * e + 1]));
        else f[e] = Vec<T>::up(u.w[e]);
    }
}
template <typename T>
__device__ __forceinline__ Raw8<T> narrow8(const float2 (&f)[4])
{
    Raw8<T> u;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if constexpr (sizeof(T) == 4) {
            u.w[2 * e] = __float_as_uint(f[e].x);
            u.w[2 * e + 1] = __float_as_uint(f[e].y);
        } else {
            u.w[e] = Vec<T>::down(f[e]);
        }
    }
    return u;
}

__device__ __forceinline__ uint32_t element_bits(const float *p) { return __float_as_uint(__ldcs(p)); }
__device__ __forceinline__ uint32_t element_bits(const bf16 *p) { return __ldcs(reinterpret_cast<const unsigned short *>(p)); }
__device__ __forceinline__ uint32_t element_bits(const f16 *p) { return __ldcs(reinterpret_cast<const unsigned short *>(p)); }

// A matrix as units are taken from it.  VEC: every row starts on 16 bytes and is whole units (8-bit rows start on 8
// bytes), a unit is one or two vectors.  Otherwise a
// unit is cut out of the aligned vectors around it (and put into those that it shares with its
// neighbours, which are the neighbouring threads' units): a third of the time of eight elements one by one.  A
// vector may hold bytes of the rows before and after; of the first and last rows, where those would lie
// outside the matrix, what is not inside the row is taken element by element.
template <typename T> struct Place {
    T *p;
    int64_t stride, rows, near;     // rows this near to an end of the matrix have no neighbours on both sides
    __device__ __forceinline__ T *row(int64_t r) const { return p + r * stride; }
    __device__ __forceinline__ bool edge(int64_t r) const { return r < near || rows - 1 - r < near; }
};
template <typename T>
__device__ __forceinline__ Place<T> place(const Matrix &m, int64_t rows)
{
    // the vectors around a unit reach less than 48 bytes beyond it
    return {static_cast<T *>(m.p), m.stride, rows, m.stride > 0 ? 47 / (m.stride * (int64_t)sizeof(T)) + 1 : rows};
}

// f with the constant k in the place of the number, 0 <= k < 4 (mostly the same for a whole warp): cheaper than
// selecting among registers.
template <int K> struct Words { static constexpr int n = K; };
template <typename F>
__device__ __forceinline__ void by_words(unsigned k, F f)
{
    if (k == 0) f(Words<0>());
    else if (k == 1) f(Words<1>());
    else if (k == 2) f(Words<2>());
    else f(Words<3>());
}

template <typename T>
__device__ __forceinline__ Raw8<T> load_elements(const T *row, int j, int cols)
{
    Raw8<T> u;
#pragma unroll
    for (int i = 0; i < 2 * (int)sizeof(T); ++i) u.w[i] = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (j + e < cols) u.w[e * sizeof(T) / 4] |= element_bits(row + j + e) << (e * sizeof(T) % 4 * 8);
    return u;
}

// Columns j .. j + 7 of row r on their way: the aligned vectors around them, or the elements where a vector would reach
// beyond the matrix.  Asking for them and taking them are two steps with branches in the second alone, so that a thread
// can have several on their way at once.
template <typename T, bool VEC> struct Unit {
    static constexpr int W = 2 * (int)sizeof(T);
    uint32_t w[VEC ? W : W + 4];

    // not `edge`: row r is none of those at the matrix's ends
    __device__ __forceinline__ void ask(const Place<T> &m, int64_t r, int j, int cols, bool edge)
    {
        const T *const row = m.row(r);
        const uint4 *p = reinterpret_cast<const uint4 *>((uintptr_t)(row + j) & ~(uintptr_t)15);
        const bool some = j < cols;
        if (VEC || !edge) {
#pragma unroll
            for (int i = 0; i < (VEC ? W / 4 : W / 4 + 1); ++i) {
                uint4 v = make_uint4(0, 0, 0, 0);
                if (some) v = VEC ? __ldcs(p + i) : p[i];   // else also the neighbour's next one: in the first-level cache
                w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
            }
        } else {
            const Raw8<T> u = load_elements(row, j, cols);
#pragma unroll
            for (int i = 0; i < W; ++i) w[i] = u.w[i];
        }
    }
    // 0 beyond the row's end
    __device__ __forceinline__ Raw8<T> take(const Place<T> &m, int64_t r, int j, int cols, bool edge) const
    {
        Raw8<T> u;
        if constexpr (VEC) {
#pragma unroll
            for (int i = 0; i < W; ++i) u.w[i] = w[i];
        } else {
            const unsigned at = edge ? 0 : (unsigned)(uintptr_t)m.row(r), bits = sizeof(T) == 4 ? 0 : (at & 3) * 8;
            by_words(at >> 2 & 3, [&](auto words) {
                constexpr int k = decltype(words)::n;
#pragma unroll
                for (int i = 0; i < W; ++i) u.w[i] = sizeof(T) == 4 ? w[i + k] : __funnelshift_r(w[i + k], w[(i + k + 1) % (W + 4)], bits);
            });
            if (j + 8 > cols)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (j + e >= cols) u.w[e * sizeof(T) / 4] &= sizeof(T) == 4 ? 0u : e & 1 ? 0x0000ffffu : 0xffff0000u;
        }
        return u;
    }
};
template <typename T, bool VEC>
__device__ __forceinline__ Raw8<T> load8(const Place<T> &m, int64_t r, int j, int cols)
{
    const bool edge = !VEC && m.edge(r);
    Unit<T, VEC> u;
    u.ask(m, r, j, cols, edge);
    return u.take(m, r, j, cols, edge);
}

template <typename T>
__device__ __forceinline__ void store_element(T *row, int j, const Raw8<T> &u, int e)
{
    if constexpr (sizeof(T) == 4) reinterpret_cast<uint32_t *>(row)[j + e] = u.w[e];
    else reinterpret_cast<unsigned short *>(row)[j + e] = (unsigned short)(u.w[e / 2] >> (e % 2 * 16));
}
// All lanes of the warp call it (with j >= cols: nothing is stored).  SEQ: they have one row's units one behind the other;
// else lane l + 1 has the unit behind lane l's or one of another row.
template <typename T, bool VEC, bool SEQ>
__device__ __forceinline__ void store8(const Place<T> &m, int64_t r, int j, int cols, const Raw8<T> &u)
{
    constexpr int W = 2 * sizeof(T), EACH = 16 / sizeof(T);     // elements of a vector
    T *const row = m.row(r);
    if (VEC) {
        if (j < cols) {
            uint4 *p = reinterpret_cast<uint4 *>(row + j);
#pragma unroll
            for (int i = 0; i < W / 4; ++i) __stcs(p + i, make_uint4(u.w[4 * i], u.w[4 * i + 1], u.w[4 * i + 2], u.w[4 * i + 3]));
        }
        return;
    }
    // the aligned vectors that end in the unit: the first begins with the last `over` elements of the unit before, whose
    // lane leaves them to this one
    const uintptr_t at = (uintptr_t)(row + j);
    const int over = (int)((unsigned)(at & 15) / (unsigned)sizeof(T)), lane = threadIdx.x & 31;
    uint32_t w[W + 4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __shfl_up_sync(0xffffffffu, u.w[W - 4 + i], 1);
#pragma unroll
    for (int i = 0; i < W; ++i) w[4 + i] = u.w[i];
    bool before = lane > 0 && j > 0;
    if (!SEQ) before &= __shfl_up_sync(0xffffffffu, j, 1) == j - 8;
    const bool v0 = (before || over == 0) && j + EACH - over <= cols, v1 = j + 8 - over <= cols;  // vectors that it can store
    uint4 *const p = reinterpret_cast<uint4 *>(at & ~(uintptr_t)15);
    const unsigned from = 16 - (unsigned)(at & 15), bits = (from & 3) * 8;      // byte of w where the vectors begin
    auto put = [&](const uint32_t (&v)[W]) {
        if (v0) __stcs(p, make_uint4(v[0], v[1], v[2], v[3]));
        if constexpr (W == 8)
            if (v1) __stcs(p + 1, make_uint4(v[4], v[5], v[6], v[7]));
    };
    if (over == 0) {
        put(u.w);
    } else {
        by_words(from >> 2, [&](auto words) {
            constexpr int k = decltype(words)::n;
            uint32_t v[W];
#pragma unroll
            for (int i = 0; i < W; ++i) v[i] = sizeof(T) == 4 ? w[i + k] : __funnelshift_r(w[i + k], w[(i + k + 1) % (W + 4)], bits);
            put(v);
        });
    }
    // elements in no vector: lane 0's first ones and lane 31's last ones, and what is around the ends of a row
    const unsigned stored = __ballot_sync(0xffffffffu, v0);
    bool next = lane < 31 && (stored >> (lane + 1 & 31) & 1);
    if (!SEQ) next &= __shfl_down_sync(0xffffffffu, j, 1) == j + 8;
    const unsigned open = __ballot_sync(0xffffffffu, j < cols && (!v0 || (W == 8 && !v1) || (over > 0 && !next)));
    if (open == 0) return;
    const int j31 = j + 8 * (31 - lane);
    if (SEQ && open == 0x80000001u && j31 + 8 <= cols) {
        // as many as a vector has: a lane for each
        const bool head = lane < EACH - over;
        uint32_t v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __shfl_sync(0xffffffffu, W == 8 && lane == 31 ? u.w[W - 4 + i] : u.w[i], head ? 0 : 31);
        const int i = sizeof(T) == 4 ? lane : lane >> 1;
        const uint32_t one = i & 2 ? (i & 1 ? v[3] : v[2]) : (i & 1 ? v[1] : v[0]);
        if (lane < EACH) {
            T *const to = row + (head ? j31 - 248 : j31 + 8 - EACH) + lane;
            if constexpr (sizeof(T) == 4) *reinterpret_cast<uint32_t *>(to) = one;
            else *reinterpret_cast<unsigned short *>(to) = (unsigned short)(lane & 1 ? one >> 16 : one);
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const bool done = e < EACH - over ? v0 : e < 8 - over ? v1 : next;
        if (!done && j + e < cols) store_element(row, j, u, e);
    }
}

// Eight bytes; `vec`: rows start on 8 bytes (known with VEC).
template <bool VEC>
__device__ __forceinline__ uint2 load_bytes(const int8_t *row, int j, int cols, bool vec)
{
    if (VEC) return j < cols ? __ldcs(reinterpret_cast<const uint2 *>(row + j)) : make_uint2(0, 0);
    if (vec && j + 8 <= cols) return __ldcs(reinterpret_cast<const uint2 *>(row + j));
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (j + e < cols) w[e / 4] |= (uint32_t)(uint8_t)row[j + e] << (e % 4 * 8);
    return make_uint2(w[0], w[1]);
}
template <bool VEC>
__device__ __forceinline__ void store_bytes(int8_t *row, int j, int cols, bool vec, uint2 v)
{
    if (VEC) {
        if (j < cols) *reinterpret_cast<uint2 *>(row + j) = v;
        return;
    }
    if (vec && j + 8 <= cols) {
        *reinterpret_cast<uint2 *>(row + j) = v;
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (j + e < cols) row[j + e] = (int8_t)((e < 4 ? v.x : v.y) >> (e % 4 * 8));
}
// The low bytes of eight words.
__device__ __forceinline__ uint2 low_bytes(const uint32_t (&q)[8])
{
    uint2 v;
    v.x = __byte_perm(__byte_perm(q[0], q[1], 0x0040), __byte_perm(q[2], q[3], 0x0040), 0x5410);
    v.y = __byte_perm(__byte_perm(q[4], q[5], 0x0040), __byte_perm(q[6], q[7], 0x0040), 0x5410);
    return v;
}
// A byte b of v ^ 0x80 in the last place of 2^23 is 2^23 + 128 + (signed) b.
__device__ __forceinline__ void unpack_bytes(uint2 v, float2 (&f)[4])
{
    v.x ^= 0x80808080u;
    v.y ^= 0x80808080u;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t w = e < 2 ? v.x : v.y;
        f[e] = add2(make_float2(__uint_as_float(__byte_perm(w, 0x4B000000u, 0x7440 | e % 2 * 2)),
                                __uint_as_float(__byte_perm(w, 0x4B000000u, 0x7441 | e % 2 * 2))), both(-8388736.0f));
    }
}
// t + kWhole, |t| < 2^22, is t rounded to the nearest integer (to even at a half) and has that integer's lowest byte as its own.
constexpr float kWhole = 12582912.0f;       // 3 * 2^22
__device__ __forceinline__ bool on(const void *p, int64_t stride_bytes, int bytes)
{
    return (((uintptr_t)p | (uintptr_t)stride_bytes) & (uintptr_t)(bytes - 1)) == 0;
}

// The largest of m and |f|; NaN if any is NaN.  As bits, NaN is above infinity and that above all others.
__device__ __forceinline__ float largest(float m, float2 f)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(m), "f"(fabsf(f.x)), "f"(fabsf(f.y)));
    return r;
}
__device__ __forceinline__ float largest8(float m, const float2 (&f)[4])
{
    return largest(largest(largest(largest(m, f[0]), f[1]), f[2]), f[3]);
}
constexpr uint32_t kInfBits = 0x7f800000u;

// Rows format.  127 p / m in binary32 is off by less than 127 (2^-23 + 2^-47) < 2^-15.9 (a quotient and a product, each
// rounded once): only where it is that near to a half can its nearest integer be another than the exact quotient's.
// There 254 |p| against (2 k + 1) m decides, both exact in binary64 (9 and 24 bits); so it does for all of a row
// whose m is so small that 127 / m is beyond binary32.  Products h w are that near to a half once in 25000, but 16-bit p by
// themselves (rows of activations, a weight of ones) often lie on one: 16384 x 4096 bf16 155 us, f16 93, f32 80.
struct Step {
    float m, inverse;
    bool tiny;
};
__device__ __forceinline__ Step step_of(uint32_t bits)
{
    Step s;
    s.m = __uint_as_float(bits);
    s.inverse = __fdiv_rn(127.0f, s.m);
    s.tiny = s.m < 1e-36f;
    return s;
}
__device__ __noinline__ inline int nearest_exactly(float p, float m)
{
    const double a = 254.0 * fabs((double)p), b = (double)m;
    int k = b > 0.0 ? (int)(a / (2.0 * b)) : 0;                 // floor, or one more where the quotient is next to an integer
    if (2.0 * k * b > a) --k;
    const double half = (2.0 * k + 1.0) * b;
    if (b > 0.0 && (a > half || (a == half && (k & 1)))) ++k;
    return p < 0.0f ? -k : k;
}
__device__ __noinline__ inline uint2 to_rows8_exactly(float2 a, float2 b, float2 c, float2 d, float m)
{
    const float p[8] = {a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
    uint32_t q[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) q[e] = (uint32_t)nearest_exactly(p[e], m);
    return low_bytes(q);
}
__device__ __forceinline__ uint2 to_rows8(const float2 (&p)[4], const Step &s)
{
    float off = 0.0f;                       // furthest from an integer; NaN where 127 / m is beyond binary32
    uint32_t q[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float2 t = mul2(p[e], both(s.inverse)), n = add2(t, both(kWhole));
        q[2 * e] = __float_as_uint(n.x);
        q[2 * e + 1] = __float_as_uint(n.y);
        const float2 whole = add2(n, both(-kWhole));
        off = largest(off, add2(t, make_float2(-whole.x, -whole.y)));
    }
    if (off <= 0.49998f && !s.tiny) return low_bytes(q);
    return to_rows8_exactly(p[0], p[1], p[2], p[3], s.m);
}

// Checkpoint.  All steps are exact but the rounding itself: a power of two scales.
__device__ __forceinline__ uint32_t kept_exponent(uint32_t bits) { return bits >= kInfBits ? 255u : max((int)(bits >> 23) - 6, 1); }
// m: the bits of the block's largest magnitude.  Only where that is above 127 steps can a value round to 128.
__device__ __forceinline__ uint2 to_kept8(const float2 (&x)[4], uint32_t m, uint32_t exponent)
{
    if (exponent == 255) return make_uint2(0, 0);
    const float up = __uint_as_float((254u - exponent) << 23);
    const bool clamp = (m & 0x7fffffu) >= 0x7e0000u;
    uint32_t q[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        float2 t = mul2(x[e], both(up));
        if (clamp) t = make_float2(fminf(fmaxf(t.x, -127.0f), 127.0f), fminf(fmaxf(t.y, -127.0f), 127.0f));
        const float2 n = add2(t, both(kWhole));
        q[2 * e] = __float_as_uint(n.x);
        q[2 * e + 1] = __float_as_uint(n.y);
    }
    return low_bytes(q);
}
__device__ __forceinline__ float kept_step(uint32_t exponent)
{
    return exponent == 255 ? __uint_as_float(0x7fc00000u) : __uint_as_float(exponent << 23);
}

}  // namespace cdadam
