// 16-byte groups of a matrix row in fp16, bf16 or fp32, and the 8-bit codes of a row.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cstdint>

#include "fq_internal.cuh"

namespace fq {

// ------------------------------------------------------------------------------- 16 bytes of a row
template <class T> struct Group;
template <> struct Group<float> {
    static constexpr int N = 4;
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
    static __device__ __forceinline__ uint4 fill() { return make_uint4(0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u); }      // -inf
    static constexpr float kFloor = -1e30f;
    static __device__ __forceinline__ uint4 above_floor(const uint4& v) { return v; }                                             // (not used)
    static __device__ __forceinline__ float to_f(float v) { return v; }
    static __device__ __forceinline__ float from_f(float v) { return v; }
};
template <> struct Group<__nv_bfloat16> {
    static constexpr int N = 8;
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
__device__ __forceinline__ float warp_max_nan(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = max_nan(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}

// The code of x in a row whose largest absolute value is a, from the quotient in 64 bits.
static __device__ __noinline__ int exact_code(float x, float a) { return __double2int_rn(127.0 * (double)x / (double)a); }

// Codes of a row whose largest absolute value is `a` (fq_quant_rows.cu says how).
struct RowScale {
    float a, r, scale;
    bool fine;                   // fp32 serves: 127 / a is a normal number
    __device__ __forceinline__ explicit RowScale(float largest) : a(largest)
    {
        const bool finite = largest < INFINITY;                  // (false for NaN)
        scale = finite ? largest / 127.0f : NAN;
        fine = largest >= 1e-30f;
        r = finite && fine ? 127.0f / largest : 0.0f;            // rows of zeros, and those with an infinity or a NaN, get codes 0
        if (!finite) { a = 0.0f; fine = true; }
    }
    __device__ __forceinline__ int code(float x) const
    {
        if (!fine) return a > 0.0f ? exact_code(x, a) : 0;
        if (r == 0.0f) return 0;                                 // (0 * inf is NaN)
        const float t = x * r, q = rintf(t);
        if (fabsf(fabsf(t - q) - 0.5f) < 3.2e-5f) return exact_code(x, a);
        return (int)q;
    }
};

inline int type_size(int dtype) { return dtype == FQ_DT_F32 ? 4 : dtype == FQ_DT_F16 || dtype == FQ_DT_BF16 ? 2 : 0; }

}  // namespace fq
