// Eight consecutive columns of a row, the unit in which the root-mean-square norm and the 8-bit formats
// take rows: how they are read, written, and turned into the two formats of 8 bits.
#pragma once
#include "elements.cuh"

namespace cdadam {

// A unit as it stands in memory.
template <typename T> struct Raw8 { uint32_t w[2 * sizeof(T)]; };

template <typename T>
__device__ __forceinline__ void widen8(const Raw8<T> &u, float (&f)[8])
{
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = __uint_as_float(u.w[e]);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 v = Vec<T>::up(u.w[e]);
            f[2 * e] = v.x;
            f[2 * e + 1] = v.y;
        }
    }
}
template <typename T>
__device__ __forceinline__ Raw8<T> narrow8(const float (&f)[8])
{
    Raw8<T> u;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < 8; ++e) u.w[e] = __float_as_uint(f[e]);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) u.w[e] = Vec<T>::down(make_float2(f[2 * e], f[2 * e + 1]));
    }
    return u;
}

__device__ __forceinline__ uint32_t element_bits(const float *p) { return __float_as_uint(__ldcs(p)); }
__device__ __forceinline__ uint32_t element_bits(const bf16 *p) { return __ldcs(reinterpret_cast<const unsigned short *>(p)); }
__device__ __forceinline__ uint32_t element_bits(const f16 *p) { return __ldcs(reinterpret_cast<const unsigned short *>(p)); }

// Columns j .. j + 7 of a row, 0 beyond its end.  VEC: every row starts on 16 bytes.
template <typename T, bool VEC>
__device__ __forceinline__ Raw8<T> load8(const T *row, int64_t j, int64_t cols)
{
    Raw8<T> u;
    if (VEC && j + 8 <= cols) {
        const uint4 *p = reinterpret_cast<const uint4 *>(row + j);
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
            const uint4 v = __ldcs(p + i);
            u.w[4 * i] = v.x; u.w[4 * i + 1] = v.y; u.w[4 * i + 2] = v.z; u.w[4 * i + 3] = v.w;
        }
        return u;
    }
#pragma unroll
    for (int i = 0; i < 2 * (int)sizeof(T); ++i) u.w[i] = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (j + e < cols) u.w[e * sizeof(T) / 4] |= element_bits(row + j + e) << (e * sizeof(T) % 4 * 8);
    return u;
}
template <typename T, bool VEC>
__device__ __forceinline__ void store8(T *row, int64_t j, int64_t cols, const Raw8<T> &u)
{
    if (VEC && j + 8 <= cols) {
        uint4 *p = reinterpret_cast<uint4 *>(row + j);
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) __stcs(p + i, make_uint4(u.w[4 * i], u.w[4 * i + 1], u.w[4 * i + 2], u.w[4 * i + 3]));
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (j + e < cols) {
            if constexpr (sizeof(T) == 4) reinterpret_cast<uint32_t *>(row)[j + e] = u.w[e];
            else reinterpret_cast<unsigned short *>(row)[j + e] = (unsigned short)(u.w[e / 2] >> (e % 2 * 16));
        }
}

// Eight bytes; `vec`: rows start on 8 bytes.
__device__ __forceinline__ uint2 load_bytes(const int8_t *row, int64_t j, int64_t cols, bool vec)
{
    if (vec && j + 8 <= cols) return __ldcs(reinterpret_cast<const uint2 *>(row + j));
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (j + e < cols) w[e / 4] |= (uint32_t)(uint8_t)row[j + e] << (e % 4 * 8);
    return make_uint2(w[0], w[1]);
}
__device__ __forceinline__ void store_bytes(int8_t *row, int64_t j, int64_t cols, bool vec, uint2 v)
{
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
__device__ __forceinline__ void unpack_bytes(uint2 v, float (&f)[8])
{
    v.x ^= 0x80808080u;
    v.y ^= 0x80808080u;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        f[e] = __fadd_rn(__uint_as_float(__byte_perm(e < 4 ? v.x : v.y, 0x4B000000u, 0x7440 | e % 4)), -8388736.0f);
}
// t + kWhole, |t| < 2^22, is t rounded to the nearest integer (to even at a half) and has that integer's lowest byte as its own.
constexpr float kWhole = 12582912.0f;       // 3 * 2^22
__device__ __forceinline__ bool on(const void *p, int64_t stride_bytes, int bytes)
{
    return (((uintptr_t)p | (uintptr_t)stride_bytes) & (uintptr_t)(bytes - 1)) == 0;
}

__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }   // ordered as |v|, NaN largest
__device__ __forceinline__ uint32_t magnitude8(const float (&f)[8])
{
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) m = max(m, magnitude(f[e]));
    return m;
}
constexpr uint32_t kInfBits = 0x7f800000u;

// Rows format.  127 p / m in binary32 is off by less than 127 (2^-23 + 2^-47) < 2^-15.9 (a quotient and a product, each
// rounded once): only where it is that near to a half can its nearest integer be another than the exact quotient's.
// There 254 |p| against (2 k + 1) m decides, both exact in binary64 (9 and 24 bits); so it does for all of a row
// whose m is so small that 127 / m is beyond binary32.
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
__device__ __forceinline__ uint2 to_rows8(const float (&p)[8], const Step &s)
{
    bool near = s.tiny;
    uint32_t q[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float t = __fmul_rn(p[e], s.inverse), n = __fadd_rn(t, kWhole);
        q[e] = __float_as_uint(n);
        near |= fabsf(__fsub_rn(t, __fsub_rn(n, kWhole))) > 0.49998f;
    }
    if (near)
#pragma unroll
        for (int e = 0; e < 8; ++e) q[e] = (uint32_t)nearest_exactly(p[e], s.m);
    return low_bytes(q);
}

// Checkpoint.  All steps are exact but the rounding itself: a power of two scales.
__device__ __forceinline__ uint32_t kept_exponent(uint32_t bits) { return bits >= kInfBits ? 255u : max((int)(bits >> 23) - 6, 1); }
__device__ __forceinline__ uint2 to_kept8(const float (&x)[8], uint32_t exponent)
{
    if (exponent == 255) return make_uint2(0, 0);
    const float up = __uint_as_float((254u - exponent) << 23);
    uint32_t q[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)
        q[e] = __float_as_uint(__fadd_rn(fminf(fmaxf(__fmul_rn(x[e], up), -127.0f), 127.0f), kWhole));
    return low_bytes(q);
}
__device__ __forceinline__ float kept_step(uint32_t exponent)
{
    return exponent == 255 ? __uint_as_float(0x7fc00000u) : __uint_as_float(exponent << 23);
}

}  // namespace cdadam
