// Device helpers of the layer operators: rows of fp32 / bf16 / f16 as fp32 vectors of 8 or 16, the
// activations and their derivatives from the pre-activation, and the 8-bit form (e4m3 numbers, one
// power-of-two scale for 32 columns).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "leapfrog.h"

namespace lfrow {

// ---- eight consecutive elements <-> fp32 ----------------------------------------------------------
__device__ __forceinline__ float2 unpack2(unsigned v, __nv_bfloat16)
{
    return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xFFFF0000u));
}
__device__ __forceinline__ float2 unpack2(unsigned v, __half)
{
    return __half22float2(*reinterpret_cast<const __half2*>(&v));
}
__device__ __forceinline__ unsigned pack2(float lo, float hi, __nv_bfloat16)
{
    unsigned r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ unsigned pack2(float lo, float hi, __half)
{
    unsigned r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
template <typename T>
struct vec8 {      // 16-bit types: one 128-bit access
    uint4 u;
    __device__ __forceinline__ void load(const T* p) { u = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ void zero() { u = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ void get(float (&v)[8]) const
    {
        const unsigned w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = unpack2(w[i], T());
            v[2 * i] = f.x; v[2 * i + 1] = f.y;
        }
    }
    __device__ __forceinline__ void set(const float (&v)[8])
    {
        u = make_uint4(pack2(v[0], v[1], T()), pack2(v[2], v[3], T()), pack2(v[4], v[5], T()), pack2(v[6], v[7], T()));
    }
    __device__ __forceinline__ void store(T* p) const { *reinterpret_cast<uint4*>(p) = u; }
};
template <>
struct vec8<float> {
    float4 a, b;
    __device__ __forceinline__ void load(const float* p)
    {
        a = reinterpret_cast<const float4*>(p)[0];
        b = reinterpret_cast<const float4*>(p)[1];
    }
    __device__ __forceinline__ void zero() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
    __device__ __forceinline__ void get(float (&v)[8]) const
    {
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    }
    __device__ __forceinline__ void set(const float (&v)[8])
    {
        a = make_float4(v[0], v[1], v[2], v[3]);
        b = make_float4(v[4], v[5], v[6], v[7]);
    }
    __device__ __forceinline__ void store(float* p) const
    {
        reinterpret_cast<float4*>(p)[0] = a;
        reinterpret_cast<float4*>(p)[1] = b;
    }
};
// ---- sixteen consecutive elements in 256-bit accesses (32-byte aligned) -----------------------------
__device__ __forceinline__ void ld256(const void* p, unsigned (&r)[8])
{
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "l"(p));
}
__device__ __forceinline__ void st256(void* p, const unsigned (&r)[8])
{
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"l"(p), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}
template <typename T>
struct vec16 {
    unsigned u[8];
    __device__ __forceinline__ void load(const T* p) { ld256(p, u); }
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] = 0;
    }
    __device__ __forceinline__ void get(float (&v)[16]) const
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float2 f = unpack2(u[i], T());
            v[2 * i] = f.x; v[2 * i + 1] = f.y;
        }
    }
    __device__ __forceinline__ void set(const float (&v)[16])
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] = pack2(v[2 * i], v[2 * i + 1], T());
    }
    __device__ __forceinline__ void store(T* p) const { st256(p, u); }
};
template <>
struct vec16<float> {
    unsigned a[8], b[8];
    __device__ __forceinline__ void load(const float* p) { ld256(p, a); ld256(p + 8, b); }
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) a[i] = b[i] = 0;
    }
    __device__ __forceinline__ void get(float (&v)[16]) const
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) { v[i] = __uint_as_float(a[i]); v[8 + i] = __uint_as_float(b[i]); }
    }
    __device__ __forceinline__ void set(const float (&v)[16])
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) { a[i] = __float_as_uint(v[i]); b[i] = __float_as_uint(v[8 + i]); }
    }
    __device__ __forceinline__ void store(float* p) const { st256(p, a); st256(p + 8, b); }
};
// a lane's piece of a row: W = 16 or 8 columns
template <typename T, int W> struct piece_of { typedef vec16<T> type; };
template <typename T> struct piece_of<T, 8> { typedef vec8<T> type; };

// the largest finite number of a type (what lf_unpack8 saturates to)
__device__ __forceinline__ float max_finite(float) { return 3.402823466e38f; }
__device__ __forceinline__ float max_finite(__nv_bfloat16) { return 3.389531389e38f; }
__device__ __forceinline__ float max_finite(__half) { return 65504.f; }
// the smallest scale byte of a group whose values may lie beyond the type: 448 * 2^e > max_finite
__device__ __forceinline__ unsigned overflow_byte(float) { return 127u + 120u; }
__device__ __forceinline__ unsigned overflow_byte(__nv_bfloat16) { return 127u + 120u; }
__device__ __forceinline__ unsigned overflow_byte(__half) { return 127u + 8u; }
__device__ __forceinline__ float clamp_keep_nan(float v, float m)
{
    return v > m ? m : (v < -m ? -m : v);
}

// ---- activations from the pre-activation ----------------------------------------------------------
// Two elements at a time: multiplies and additions as packed fp32 (fma.rn.f32x2), which halves their issue slots.
// FAST: e^t and the reciprocal from the special-function unit (about 1e-6 relative, far below the
// rounding of a 16-bit result); otherwise the library functions, for fp32 results.
__device__ __forceinline__ float2 f2(float v) { return make_float2(v, v); }
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) { return __ffma2_rn(a, b, c); }
__device__ __forceinline__ float2 mul2(float2 a, float2 b) { return __fmul2_rn(a, b); }
__device__ __forceinline__ float2 add2(float2 a, float2 b) { return __fadd2_rn(a, b); }
__device__ __forceinline__ float ex2(float t)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(t));
    return r;
}
__device__ __forceinline__ float rcp(float t)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(t));
    return r;
}
constexpr float LOG2E = 1.4426950408889634f;
// 1 / (1 + 2^t): the logistic function of -t ln 2
__device__ __forceinline__ float2 logistic2(float2 t)
{
    const float2 d = add2(f2(1.f), make_float2(ex2(t.x), ex2(t.y)));
    return make_float2(rcp(d.x), rcp(d.y));
}
constexpr float GELU_C = 1.5957691216057308f;            // 2 sqrt(2 / pi)
constexpr float GELU_D = GELU_C * 0.044715f;
// a = sigmoid(g(z)) of the three activations built on it: g(z) = z, or GELU's cubic, as (1 + tanh u) / 2 = sigmoid(2 u)
template <bool FAST>
__device__ __forceinline__ float2 sigmoid_of(float2 z, float2 zz, bool cubic)
{
    if (FAST) {
        const float2 p = cubic ? fma2(zz, f2(-LOG2E * GELU_D), f2(-LOG2E * GELU_C)) : f2(-LOG2E);
        return logistic2(mul2(z, p));
    }
    const float2 t = cubic ? mul2(z, fma2(zz, f2(GELU_D), f2(GELU_C))) : z;
    return make_float2(1.0f / (1.0f + expf(-t.x)), 1.0f / (1.0f + expf(-t.y)));
}
// tanh z = 1 - 2 / (1 + e^{2 z}); below 1/16, where that cancels, the Taylor polynomial (next term 17/315 z^7: 3e-9 relative)
__device__ __forceinline__ float2 tanh_fast(float2 z)
{
    const float2 zz = mul2(z, z), r = logistic2(mul2(z, f2(2.f * LOG2E)));
    const float2 t = fma2(r, f2(-2.f), f2(1.f));
    const float2 p = fma2(mul2(z, zz), fma2(zz, f2(2.f / 15.f), f2(-1.f / 3.f)), z);
    return make_float2(fabsf(z.x) < 0.0625f ? p.x : t.x, fabsf(z.y) < 0.0625f ? p.y : t.y);
}
template <bool FAST, int KIND>
__device__ __forceinline__ float2 act2(float2 z)
{
    if (KIND == LF_ACT_SIGMOID) return sigmoid_of<FAST>(z, z, false);
    if (KIND == LF_ACT_TANH) return FAST ? tanh_fast(z) : make_float2(tanhf(z.x), tanhf(z.y));
    if (KIND == LF_ACT_RELU) return make_float2(z.x < 0.f ? 0.f : z.x, z.y < 0.f ? 0.f : z.y);     // NaN stays
    if (KIND == LF_ACT_SILU) return mul2(z, sigmoid_of<FAST>(z, z, false));
    if (KIND == LF_ACT_GELU) return mul2(z, sigmoid_of<FAST>(z, mul2(z, z), true));
    return z;
}
// |z| <= 448 * 2^28 (prime_byte) or NaN; `nan`: 0, or NaN where z is not a number
template <bool FAST, int KIND>
__device__ __forceinline__ float2 act_prime2(float2 z, float nan)
{
    if (KIND == LF_ACT_TANH || KIND == LF_ACT_SIGMOID) {
        // even functions of z: a (1 - a) with a = sigmoid(-|z|) <= 1/2, where 1 - a does not cancel; tanh' = 4 a (1 - a) at 2 z
        const float k = KIND == LF_ACT_TANH ? 2.f : 1.f;
        const float2 a = sigmoid_of<FAST>(make_float2(-k * fabsf(z.x), -k * fabsf(z.y)), z, false);
        return mul2(mul2(a, f2(k * k)), fma2(a, f2(-1.f), f2(1.f)));
    }
    if (KIND == LF_ACT_RELU) return make_float2(z.x > 0.f ? 1.f : nan, z.y > 0.f ? 1.f : nan);
    if (KIND == LF_ACT_NONE) return f2(1.f);
    // a + z a (1 - a) g'(z)
    const float2 zz = mul2(z, z);
    const float2 a = sigmoid_of<FAST>(z, zz, KIND == LF_ACT_GELU);
    const float2 na = fma2(a, f2(-1.f), f2(1.f));
    const float2 zn = KIND == LF_ACT_GELU ? mul2(mul2(z, na), fma2(zz, f2(3.f * GELU_D), f2(GELU_C))) : mul2(z, na);
    return fma2(a, zn, a);
}
// Over NE elements.  (Half of the exponentials as a polynomial on the multiply-add units, to relieve the
// special-function unit, was 5 % slower, one reciprocal for two elements, 1 / (p q), 4 %: the issue slots are as scarce.)
template <bool FAST, int NE, int KIND>
__device__ __forceinline__ void act_all(float* v)
{
#pragma unroll
    for (int i = 0; i < NE; i += 2) {
        const float2 z = make_float2(v[i], v[i + 1]);
        const float2 r = act2<FAST, KIND>(z);
        v[i] = r.x; v[i + 1] = r.y;
    }
}
// ... with the choice of the activation at run time, outside of the loop
template <bool FAST, int NE>
__device__ __forceinline__ void act_n(float* v, int kind)
{
    switch (kind) {
        case LF_ACT_SIGMOID: act_all<FAST, NE, LF_ACT_SIGMOID>(v); break;
        case LF_ACT_TANH: act_all<FAST, NE, LF_ACT_TANH>(v); break;
        case LF_ACT_RELU: act_all<FAST, NE, LF_ACT_RELU>(v); break;
        case LF_ACT_SILU: act_all<FAST, NE, LF_ACT_SILU>(v); break;
        case LF_ACT_GELU: act_all<FAST, NE, LF_ACT_GELU>(v); break;
        default: break;
    }
}
// d *= sigma'(z)
template <bool FAST, int NE, int KIND>
__device__ __forceinline__ void prime_all(float* d, const float* z, float nan)
{
#pragma unroll
    for (int i = 0; i < NE; i += 2) {
        const float2 zi = make_float2(z[i], z[i + 1]);
        const float2 r = mul2(make_float2(d[i], d[i + 1]), act_prime2<FAST, KIND>(zi, nan));
        d[i] = r.x; d[i + 1] = r.y;
    }
}
// ---- 8 bits -------------------------------------------------------------------------------------
__device__ __forceinline__ unsigned abs_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }
// the scale byte of a group from the bits of its largest magnitude (NaN > infinity > finite as integers):
// amax = m 2^E, e = E - 8 for m <= 1.75 (448 = 1.75 * 2^8), else E - 7, at least -127
__device__ __forceinline__ unsigned scale_byte(unsigned amax_bits)
{
    if (amax_bits >= 0x7F800000u) return 255u;
    const int b = (int)(amax_bits >> 23) - 8 + ((amax_bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return b > 0 ? (unsigned)b : 0u;
}
__device__ __forceinline__ float inv_scale(unsigned byte)     // 2^-e; NaN for a group that is not finite
{
    return byte == 255u ? __uint_as_float(0x7FC00000u) : __uint_as_float((254u - byte) << 23);
}
__device__ __forceinline__ float scale(unsigned byte)         // 2^e
{
    return __uint_as_float(byte == 255u ? 0x7FC00000u : (byte == 0u ? 0x00400000u : byte << 23));
}
// The byte whose scale sigma' is taken with: at most 2^28, so that GELU's cubic stays finite (z a (1 - a) g'(z) needs |z| < 1e13).
// From e = 28 on every value but zero is beyond 2^19, where sigma' is 0 or 1 to the last bit for all activations.
__device__ __forceinline__ unsigned prime_byte(unsigned byte) { return byte < 127u + 28u || byte == 255u ? byte : 127u + 28u; }
// what is added to the rectifier's sigma', a comparison, which does not see NaN
__device__ __forceinline__ float prime_nan(unsigned byte) { return byte == 255u ? __uint_as_float(0x7FC00000u) : 0.f; }
__device__ __forceinline__ unsigned to_e4m3x4(float a, float b, float c, float d)
{
    unsigned short lo, hi;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
    return (unsigned)lo | ((unsigned)hi << 16);
}
__device__ __forceinline__ void from_e4m3x4(unsigned q, float s, float& a, float& b, float& c, float& d)
{
    unsigned h0, h1;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h0) : "h"((unsigned short)(q & 0xFFFFu)));
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h1) : "h"((unsigned short)(q >> 16)));
    const float2 f0 = __half22float2(*reinterpret_cast<const __half2*>(&h0));
    const float2 f1 = __half22float2(*reinterpret_cast<const __half2*>(&h1));
    const float2 g0 = __fmul2_rn(f0, make_float2(s, s)), g1 = __fmul2_rn(f1, make_float2(s, s));
    a = g0.x; b = g0.y; c = g1.x; d = g1.y;
}
// W columns held by one lane; the 32 / W lanes of a group are neighbours
template <int W>
__device__ __forceinline__ unsigned group_byte(const float (&v)[W])
{
    unsigned m = 0;
#pragma unroll
    for (int i = 0; i < W; ++i) m = max(m, abs_bits(v[i]));
#pragma unroll
    for (int o = 1; o < 32 / W; o <<= 1) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
    return scale_byte(m);
}
__device__ __forceinline__ uint2 quantize8(const float (&v)[8], unsigned byte)
{
    const float r = inv_scale(byte);
    return make_uint2(to_e4m3x4(v[0] * r, v[1] * r, v[2] * r, v[3] * r), to_e4m3x4(v[4] * r, v[5] * r, v[6] * r, v[7] * r));
}
__device__ __forceinline__ void dequantize8(uint2 q, unsigned byte, float (&v)[8])
{
    const float s = scale(byte);
    from_e4m3x4(q.x, s, v[0], v[1], v[2], v[3]);
    from_e4m3x4(q.y, s, v[4], v[5], v[6], v[7]);
}
}  // namespace lfrow
