// 16-byte groups of a matrix row in fp16, bf16 or fp32, and the 8-bit codes of a row.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cstdint>

#include "fq_internal.cuh"

namespace fq {

// Two at a time.
__device__ __forceinline__ unsigned long long two(float2 v)
{
    unsigned long long r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(v.x), "f"(v.y));
    return r;
}
__device__ __forceinline__ float2 apart(unsigned long long v)
{
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
    return r;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b)
{
    unsigned long long r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(two(a)), "l"(two(b)));
    return apart(r);
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b)
{
    unsigned long long r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(two(a)), "l"(two(b)));
    return apart(r);
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    unsigned long long r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(two(a)), "l"(two(b)), "l"(two(c)));
    return apart(r);
}

// ------------------------------------------------------------------------------- 16 bytes of a row
template <class T> struct Group;
template <> struct Group<float> {
    static constexpr int N = 4;
    static constexpr int kKeyBits = 32;          // upper bits of a value, as a float, that tell it from others of its sign
    static __device__ __forceinline__ void unpack(const uint4& v, float2 (&f)[2])
    {
        f[0] = make_float2(__uint_as_float(v.x), __uint_as_float(v.y));
        f[1] = make_float2(__uint_as_float(v.z), __uint_as_float(v.w));
    }
    static __device__ __forceinline__ uint4 pack(const float2 (&f)[2])
    {
        return make_uint4(__float_as_uint(f[0].x), __float_as_uint(f[0].y), __float_as_uint(f[1].x), __float_as_uint(f[1].y));
    }
    // running maximum (NaN is not seen)
    using Max = float;
    static __device__ __forceinline__ Max lowest() { return -INFINITY; }
    static __device__ __forceinline__ void take_max(Max& m, const uint4& v)
    {
        m = fmaxf(fmaxf(m, fmaxf(__uint_as_float(v.x), __uint_as_float(v.y))), fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
    }
    static __device__ __forceinline__ float of_max(Max m) { return m; }
    // running largest absolute value (NaN stays), from 0
    static __device__ __forceinline__ Max nothing() { return 0.0f; }
    static __device__ __forceinline__ void take_abs(Max& m, const uint4& v);
    static __device__ __forceinline__ float of_abs(Max m) { return m; }
    static __device__ __forceinline__ uint4 fill() { return make_uint4(0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u); }      // -inf
    static __device__ __forceinline__ float to_f(float v) { return v; }
    static __device__ __forceinline__ float from_f(float v) { return v; }
};
template <> struct Group<__nv_bfloat16> {
    static constexpr int N = 8;
    static constexpr int kKeyBits = 16;
    static __device__ __forceinline__ void unpack(const uint4& v, float2 (&f)[4])
    {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; i++) f[i] = make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
    }
    static __device__ __forceinline__ uint4 pack(const float2 (&f)[4])
    {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(f[i].x, f[i].y);
            w[i] = *reinterpret_cast<const uint32_t*>(&h);
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    using Max = __nv_bfloat162;
    static __device__ __forceinline__ Max lowest() { return __float2bfloat162_rn(-INFINITY); }
    static __device__ __forceinline__ void take_max(Max& m, const uint4& v)
    {
        const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&v);
        m = __hmax2(m, __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3])));
    }
    static __device__ __forceinline__ float of_max(Max m) { return fmaxf(__low2float(m), __high2float(m)); }
    static __device__ __forceinline__ Max nothing() { return __float2bfloat162_rn(0.0f); }
    static __device__ __forceinline__ void take_abs(Max& m, const uint4& v)
    {
        const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&v);
#pragma unroll
        for (int i = 0; i < 4; i++) m = __hmax2_nan(m, __habs2(h[i]));
    }
    static __device__ __forceinline__ float of_abs(Max m);
    static __device__ __forceinline__ uint4 fill() { return make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u); }      // -inf
    // a value whose exponential is 0 wherever that of -inf is, as long as the largest is far enough above it
    static constexpr float kFloor = -1e30f;
    static __device__ __forceinline__ uint4 above_floor(uint4 v)                                                  // (NaN stays)
    {
        __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&v);
        const __nv_bfloat162 low = __float2bfloat162_rn(kFloor);
#pragma unroll
        for (int i = 0; i < 4; i++) h[i] = __hmax2_nan(h[i], low);
        return v;
    }
    static __device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
    static __device__ __forceinline__ __nv_bfloat16 from_f(float v) { return __float2bfloat16_rn(v); }
};
template <> struct Group<__half> {
    static constexpr int N = 8;
    static constexpr int kKeyBits = 19;
    static __device__ __forceinline__ void unpack(const uint4& v, float2 (&f)[4])
    {
        const __half2* h = reinterpret_cast<const __half2*>(&v);
#pragma unroll
        for (int i = 0; i < 4; i++) f[i] = __half22float2(h[i]);
    }
    static __device__ __forceinline__ uint4 pack(const float2 (&f)[4])
    {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const __half2 h = __floats2half2_rn(f[i].x, f[i].y);
            w[i] = *reinterpret_cast<const uint32_t*>(&h);
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    using Max = __half2;
    static __device__ __forceinline__ Max lowest() { return __float2half2_rn(-INFINITY); }
    static __device__ __forceinline__ void take_max(Max& m, const uint4& v)
    {
        const __half2* h = reinterpret_cast<const __half2*>(&v);
        m = __hmax2(m, __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3])));
    }
    static __device__ __forceinline__ float of_max(Max m) { return fmaxf(__low2float(m), __high2float(m)); }
    static __device__ __forceinline__ Max nothing() { return __float2half2_rn(0.0f); }
    static __device__ __forceinline__ void take_abs(Max& m, const uint4& v)
    {
        const __half2* h = reinterpret_cast<const __half2*>(&v);
#pragma unroll
        for (int i = 0; i < 4; i++) m = __hmax2_nan(m, __habs2(h[i]));
    }
    static __device__ __forceinline__ float of_abs(Max m);
    static __device__ __forceinline__ uint4 fill() { return make_uint4(0xfc00fc00u, 0xfc00fc00u, 0xfc00fc00u, 0xfc00fc00u); }      // -inf
    // a value whose exponential is 0 wherever that of -inf is, as long as the largest is far enough above it
    static constexpr float kFloor = -65504.0f;
    static __device__ __forceinline__ uint4 above_floor(uint4 v)                                                  // (NaN stays)
    {
        __half2* h = reinterpret_cast<__half2*>(&v);
        const __half2 low = __float2half2_rn(kFloor);
#pragma unroll
        for (int i = 0; i < 4; i++) h[i] = __hmax2_nan(h[i], low);
        return v;
    }
    static __device__ __forceinline__ float to_f(__half v) { return __half2float(v); }
    static __device__ __forceinline__ __half from_f(float v) { return __float2half_rn(v); }
};

// The larger one, NaN if either is one.
__device__ __forceinline__ float max_nan(float a, float b)
{
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}
__device__ __forceinline__ void Group<float>::take_abs(float& m, const uint4& v)
{
    m = max_nan(max_nan(m, max_nan(fabsf(__uint_as_float(v.x)), fabsf(__uint_as_float(v.y)))), max_nan(fabsf(__uint_as_float(v.z)), fabsf(__uint_as_float(v.w))));
}
__device__ __forceinline__ float Group<__nv_bfloat16>::of_abs(__nv_bfloat162 m) { return max_nan(__low2float(m), __high2float(m)); }
__device__ __forceinline__ float Group<__half>::of_abs(__half2 m) { return max_nan(__low2float(m), __high2float(m)); }
__device__ __forceinline__ float warp_max_nan(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = max_nan(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}

// Codes of a row whose largest absolute value is `a` (fq_quant_rows.cu says how).
struct RowScale {
    float a, r;                  // r: 127 / a, a little off, or 0 where fp32 does not serve (0, an infinity or a NaN, or products out of range)
    __device__ __forceinline__ explicit RowScale(float largest)
    {
        a = largest < INFINITY ? largest : 0.0f;                 // (rows with an infinity or a NaN get codes 0, as those of zeros do)
        float inverse;
        asm("rcp.approx.f32 %0, %1;" : "=f"(inverse) : "f"(a));
        r = a >= 1e-30f && a <= 1e30f ? 127.0f * inverse : 0.0f;
    }
    static __device__ __forceinline__ float scale(float largest) { return largest < INFINITY ? largest / 127.0f : NAN; }
    // x * r rounded to the nearest integer: with 1.5 * 2^23 added a product keeps its integer part in its low bits.
    static constexpr float kMagic = 12582912.0f;
    // x * r is off by at most 127 * 2^-22 = 3.1e-5: further than that from a border the integer is the quotient's.
    static constexpr float kClear = 0.49995f;
    __device__ __forceinline__ float near(float x) const { return fmaf(x, r, kMagic); }
    __device__ __forceinline__ float off(float x, float u) const { return fmaf(x, r, kMagic - u); }
    // Four codes, one to a byte.
    __device__ __forceinline__ uint32_t four(float2 x, float2 y) const
    {
        const float2 rr = make_float2(r, r), magic = make_float2(kMagic, kMagic), minus = make_float2(-1.0f, -1.0f);
        float2 u = fma2(x, rr, magic), v = fma2(y, rr, magic);
        const float2 d = fma2(x, rr, fma2(u, minus, magic)), e = fma2(y, rr, fma2(v, minus, magic));
        if (r == 0.0f) return beyond(x.x) | beyond(x.y) << 8 | beyond(y.x) << 16 | beyond(y.y) << 24;
        if (fmaxf(fmaxf(fabsf(d.x), fabsf(d.y)), fmaxf(fabsf(e.x), fabsf(e.y))) > kClear) {
            u = make_float2(settled(x.x, u.x, d.x), settled(x.y, u.y, d.y));
            v = make_float2(settled(y.x, v.x, e.x), settled(y.y, v.y, e.y));
        }
        return __byte_perm(__byte_perm(__float_as_uint(u.x), __float_as_uint(u.y), 0x0040), __byte_perm(__float_as_uint(v.x), __float_as_uint(v.y), 0x0040), 0x5410);
    }
    __device__ __forceinline__ int8_t one(float x) const
    {
        const float u = near(x);
        return (int8_t)(r == 0.0f ? beyond(x) : __float_as_uint(settled(x, u, off(x, u))) & 255u);
    }
    // The quotient 127 x / a is close to q = u - 1.5 * 2^23, on the side of it that d says.  Whether it passes the border b half a step
    // on is the sign of 127 x - b a, which two products and what each lost in rounding (so little that their difference is exact)
    // give exactly.
    __device__ __forceinline__ float settled(float x, float u, float d) const
    {
        const float q = u - kMagic, step = copysignf(1.0f, d), b = q + copysignf(0.5f, d);
        const float w = 127.0f * x, wl = fmaf(127.0f, x, -w), p = b * a, pl = fmaf(b, a, -p);
        const float past = ((w - p) + (wl - pl)) * step;
        return past > 0.0f || (past == 0.0f && ((int)q & 1)) ? u + step : u;
    }
    // From the quotient in 64 bits.
    __device__ __noinline__ uint32_t beyond(float x) const { return a > 0.0f ? (uint32_t)__double2int_rn(127.0 * (double)x / (double)a) & 255u : 0u; }
};

inline int type_size(int dtype) { return dtype == FQ_DT_F32 ? 4 : dtype == FQ_DT_F16 || dtype == FQ_DT_BF16 ? 2 : 0; }

}  // namespace fq
