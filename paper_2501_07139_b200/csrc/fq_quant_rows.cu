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

template <class T>
__global__ void __launch_bounds__(kQuantThreads) quantize_rows_kernel(const QuantArgs a)
{
    __shared__ float red[kQuantThreads / 32];
    const long long r = blockIdx.x;
    const T* x = static_cast<const T*>(a.x) + r * a.ldx;
    float m = 0.0f;
    for (int c = threadIdx.x; c < a.cols; c += kQuantThreads) m = max_nan(m, fabsf(Group<T>::to_f(x[c])));
    m = warp_max_nan(m);
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = m;
    __syncthreads();
    m = red[0];
    for (int w = 1; w < kQuantThreads / 32; w++) m = max_nan(m, red[w]);
    const RowScale s(m);
    int8_t* q = a.codes + r * a.ldc;
    for (int c = threadIdx.x; c < a.cols; c += kQuantThreads) q[c] = (int8_t)s.code(Group<T>::to_f(x[c]));
    if (threadIdx.x == 0) a.scales[r] = s.scale;
}

}  // namespace

int launch_quantize_rows(const void* x, int dtype, int rows, int cols, long long ldx, int8_t* codes, long long ldc, float* scales,
                         cudaStream_t st)
{
    const QuantArgs a{x, ldx, rows, cols, codes, ldc, scales};
    if (dtype == FQ_DT_F32) quantize_rows_kernel<float><<<(unsigned)rows, kQuantThreads, 0, st>>>(a);
    else if (dtype == FQ_DT_F16) quantize_rows_kernel<__half><<<(unsigned)rows, kQuantThreads, 0, st>>>(a);
    else quantize_rows_kernel<__nv_bfloat16><<<(unsigned)rows, kQuantThreads, 0, st>>>(a);
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
