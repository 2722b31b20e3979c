// Symmetric 8-bit quantiser of matrix rows:  a = max |x|,  scale = a / 127,  code = rint(127 x / a), ties to even.
//
// A code is that of the exact quotient: in fp32 alone a value next to the border between two codes could fall on either side, and
// 127 x / a does meet borders (x = a / 2 is 63.5).  t = x * fp32(127 / a) is off by at most 127 * 2^-23; only where t is
// closer than that to a border, one value in some ten thousand, the quotient is taken in 64 bits, where operands of 24 bits keep
// every quotient that is not on the border off it.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "fq_internal.cuh"
#include "fq_rowtypes.cuh"

namespace fq {
namespace {

constexpr int kQuantThreads = 256;

struct QuantArgs {
    const void* x;
    long long ldx;
    int rows, cols;
    int8_t* codes;
    long long ldc;
    float* scales;
};

__device__ __forceinline__ float block_max(float m, float* red)
{
    m = warp_max_nan(m);
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = m;
    __syncthreads();
    m = red[0];
#pragma unroll
    for (int w = 1; w < kQuantThreads / 32; w++) m = max_nan(m, red[w]);
    return m;
}

// Rows of any length and alignment: read twice, the second time from the caches.
template <class T>
__global__ void __launch_bounds__(kQuantThreads) quantize_rows_kernel(const QuantArgs a)
{
    __shared__ float red[kQuantThreads / 32];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");    // (whoever reads the codes waits for the end of this kernel)
    const long long r = blockIdx.x;
    const T* x = static_cast<const T*>(a.x) + r * a.ldx;
    float m = 0.0f;
    for (int c = threadIdx.x; c < a.cols; c += kQuantThreads) m = max_nan(m, fabsf(Group<T>::to_f(x[c])));
    const RowScale s(block_max(m, red));
    int8_t* q = a.codes + r * a.ldc;
    for (int c = threadIdx.x; c < a.cols; c += kQuantThreads) q[c] = (int8_t)s.code(Group<T>::to_f(x[c]));
    if (threadIdx.x == 0) a.scales[r] = s.scale;
}

// Rows that stay in registers, U pieces of 8 values to a thread: pieces are 16-byte aligned on both sides, and there is a whole number of them.
template <class T, int U>
__global__ void __launch_bounds__(kQuantThreads) quantize_rows_kept_kernel(const QuantArgs a)
{
    __shared__ float red[kQuantThreads / 32];
    constexpr int G = 8 / Group<T>::N;                   // 16-byte groups of a piece
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const long long r = blockIdx.x;
    const T* x = static_cast<const T*>(a.x) + r * a.ldx;
    const int pieces = a.cols / 8;
    uint4 v[U][G];
#pragma unroll
    for (int u = 0; u < U; u++)
#pragma unroll
        for (int g = 0; g < G; g++) {
            v[u][g] = make_uint4(0u, 0u, 0u, 0u);
            const int p = u * kQuantThreads + threadIdx.x;
            if (p < pieces) v[u][g] = *reinterpret_cast<const uint4*>(x + p * 8 + g * Group<T>::N);
        }
    float m = 0.0f;
#pragma unroll
    for (int u = 0; u < U; u++)
#pragma unroll
        for (int g = 0; g < G; g++) {
            float2 f[Group<T>::N / 2];
            Group<T>::unpack(v[u][g], f);
#pragma unroll
            for (int i = 0; i < Group<T>::N / 2; i++) m = max_nan(m, max_nan(fabsf(f[i].x), fabsf(f[i].y)));
        }
    const RowScale s(block_max(m, red));
    int8_t* q = a.codes + r * a.ldc;
#pragma unroll
    for (int u = 0; u < U; u++) {
        const int p = u * kQuantThreads + threadIdx.x;
        if (p >= pieces) break;
        uint32_t w[2];
#pragma unroll
        for (int g = 0; g < G; g++) {
            float2 f[Group<T>::N / 2];
            Group<T>::unpack(v[u][g], f);
#pragma unroll
            for (int i = 0; i < Group<T>::N / 4; i++) {
                const uint32_t c0 = (uint32_t)s.code(f[2 * i].x) & 255u, c1 = (uint32_t)s.code(f[2 * i].y) & 255u;
                const uint32_t c2 = (uint32_t)s.code(f[2 * i + 1].x) & 255u, c3 = (uint32_t)s.code(f[2 * i + 1].y) & 255u;
                w[g * (Group<T>::N / 4) + i] = c0 | c1 << 8 | c2 << 16 | c3 << 24;
            }
        }
        *reinterpret_cast<uint2*>(q + p * 8) = make_uint2(w[0], w[1]);
    }
    if (threadIdx.x == 0) a.scales[r] = s.scale;
}

template <class T>
void launch_typed(const QuantArgs& a, cudaStream_t st)
{
    const int per_thread = (a.cols / 8 + kQuantThreads - 1) / kQuantThreads;
    const bool pieces = a.cols % 8 == 0 && aligned(a.x, 16) && a.ldx * sizeof(T) % 16 == 0 && aligned(a.codes, 8) && a.ldc % 8 == 0;
    if (pieces && per_thread <= 1) quantize_rows_kept_kernel<T, 1><<<(unsigned)a.rows, kQuantThreads, 0, st>>>(a);
    else if (pieces && per_thread <= 2) quantize_rows_kept_kernel<T, 2><<<(unsigned)a.rows, kQuantThreads, 0, st>>>(a);
    else if (pieces && per_thread <= 4) quantize_rows_kept_kernel<T, 4><<<(unsigned)a.rows, kQuantThreads, 0, st>>>(a);
    else if (pieces && per_thread <= 8) quantize_rows_kept_kernel<T, 8><<<(unsigned)a.rows, kQuantThreads, 0, st>>>(a);
    else quantize_rows_kernel<T><<<(unsigned)a.rows, kQuantThreads, 0, st>>>(a);
}

}  // namespace

int launch_quantize_rows(const void* x, int dtype, int rows, int cols, long long ldx, int8_t* codes, long long ldc, float* scales,
                         cudaStream_t st)
{
    const QuantArgs a{x, ldx, rows, cols, codes, ldc, scales};
    if (dtype == FQ_DT_F32) launch_typed<float>(a, st);
    else if (dtype == FQ_DT_F16) launch_typed<__half>(a, st);
    else launch_typed<__nv_bfloat16>(a, st);
    return cudaGetLastError() == cudaSuccess ? FQ_OK : FQ_ERR_CUDA;
}

}  // namespace fq

using namespace fq;

extern "C" int fq_quantize_rows(fq_ctx* ctx, const void* x_dev, int dtype, int rows, int cols, long long ldx, int8_t* codes_dev,
                                long long ldc, float* scales_dev, void* stream)
{
    const int size = type_size(dtype);
    if (!ctx || !x_dev || !codes_dev || !scales_dev || !size) return FQ_ERR_ARG;
    if (rows < 1 || rows > FQ_MAX_ROWS || cols < 1 || cols > (1 << 20) || ldx < cols || ldc < cols) return FQ_ERR_SHAPE;
    if (!aligned(x_dev, (size_t)size) || !aligned(scales_dev, 4)) return FQ_ERR_ALIGN;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return FQ_ERR_CUDA;
    return launch_quantize_rows(x_dev, dtype, rows, cols, ldx, codes_dev, ldc, scales_dev, (cudaStream_t)stream);
}
