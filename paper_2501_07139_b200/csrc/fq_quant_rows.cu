// Symmetric 8-bit quantiser of matrix rows:  a = max |x|,  scale = a / 127,  code = rint(127 x / a), ties to even.
//
// A code is that of the exact quotient: in fp32 alone a value next to the border between two codes could fall on either side, and
// 127 x / a does meet borders (x = a / 2 is 63.5; among 4096 bf16 values some seven are).  x times a little inexact 127 / a is off by at most
// 3.1e-5; where it is closer than 5e-5 to a border, the side is settled by the exact sign of 127 x - border a.
#include <algorithm>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "fq_internal.cuh"
#include "fq_rowtypes.cuh"

namespace fq {
namespace {


struct QuantArgs {
    const void* x;
    long long ldx;
    int rows, cols;
    int8_t* codes;
    long long ldc;
    float* scales;
};

// (`red` is free again after the CTA's next barrier.)
template <int THREADS>
__device__ __forceinline__ float block_max(float m, float* red)
{
    constexpr int W = THREADS / 32;
    m = warp_max_nan(m);
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = m;
    __syncthreads();
    m = red[threadIdx.x & (W - 1)];
#pragma unroll
    for (int o = 1; o < W; o <<= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
    return m;
}

// Rows of any length and alignment: read twice, the second time from the caches.
template <class T, int THREADS>
__global__ void __launch_bounds__(THREADS) quantize_rows_kernel(const QuantArgs a)
{
    __shared__ float red[THREADS / 32];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");    // (whoever reads the codes waits for the end of this kernel)
    const long long r = blockIdx.x;
    const T* x = static_cast<const T*>(a.x) + r * a.ldx;
    float m = 0.0f;
    for (int c = threadIdx.x; c < a.cols; c += THREADS) m = max_nan(m, fabsf(Group<T>::to_f(x[c])));
    m = block_max<THREADS>(m, red);
    const RowScale s(m);
    int8_t* q = a.codes + r * a.ldc;
    for (int c = threadIdx.x; c < a.cols; c += THREADS) q[c] = s.one(Group<T>::to_f(x[c]));
    if (threadIdx.x == 0) a.scales[r] = RowScale::scale(m);
}

// Rows that stay in registers, U pieces of 8 values to a thread: pieces are 16-byte aligned on both sides, and there is a whole number of them.
// Many rows: four pieces, so that a row's maximum, two reductions and a reciprocal, is shared by 32 values of a thread (8192 x 4096 bf16 27 us,
// of which HBM needs 16, with one piece a thread 45 us; the next row on its way while one is worked on gains nothing).  What is left are phases: a
// row's loads, its maximum behind a barrier, its codes (issue slots 63 %, HBM 36 %; most stalls are waits for loads).  Few rows: one or two, for the latency.
template <class T, int U>
__global__ void __launch_bounds__(1024, 1) quantize_rows_kept_kernel(const QuantArgs a)
{
    __shared__ float red[2][32];
    constexpr int G = 8 / Group<T>::N;                   // 16-byte groups of a piece
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int pieces = a.cols / 8, threads = blockDim.x, lane = threadIdx.x & 31, warps = threads >> 5;
    const auto load = [&](uint4 (&v)[U][G], int r) {
        const T* x = static_cast<const T*>(a.x) + (long long)r * a.ldx;
#pragma unroll
        for (int u = 0; u < U; u++)
#pragma unroll
            for (int g = 0; g < G; g++) {
                v[u][g] = make_uint4(0u, 0u, 0u, 0u);
                const int p = u * threads + threadIdx.x;
                if (p < pieces && r < a.rows) v[u][g] = *reinterpret_cast<const uint4*>(x + p * 8 + g * Group<T>::N);
            }
    };
    uint4 v[U][G];
    load(v, (int)blockIdx.x);
    int turn = 0;
    for (int r = blockIdx.x; r < a.rows; r += gridDim.x, turn ^= 1) {
        typename Group<T>::Max most = Group<T>::nothing();
#pragma unroll
        for (int u = 0; u < U; u++)
#pragma unroll
            for (int g = 0; g < G; g++) Group<T>::take_abs(most, v[u][g]);
        float m = warp_max_nan(Group<T>::of_abs(most));
        if (lane == 0) red[turn][threadIdx.x >> 5] = m;
        __syncthreads();                                 // (a warp writes to the other half next, which all have left by then)
        m = warp_max_nan(lane < warps ? red[turn][lane] : 0.0f);
        const RowScale s(m);
        int8_t* q = a.codes + (long long)r * a.ldc;
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int p = u * threads + threadIdx.x;
            uint32_t w[2];
#pragma unroll
            for (int g = 0; g < G; g++) {
                float2 f[Group<T>::N / 2];
                Group<T>::unpack(v[u][g], f);
#pragma unroll
                for (int i = 0; i < Group<T>::N / 4; i++)
                    w[g * (Group<T>::N / 4) + i] = s.four(f[2 * i], f[2 * i + 1]);
            }
            if (p < pieces) *reinterpret_cast<uint2*>(q + p * 8) = make_uint2(w[0], w[1]);
        }
        if (threadIdx.x == 0) a.scales[r] = RowScale::scale(m);
        if (r + (int)gridDim.x < a.rows) load(v, r + (int)gridDim.x);
    }
}

template <class T, int U>
int launch_kept(const QuantArgs& a, int sm_count, cudaStream_t st)
{
    const int pieces = a.cols / 8, threads = std::max(32, ((pieces + U - 1) / U + 31) / 32 * 32);
    const int most = sm_count * (1024 / threads);
    quantize_rows_kept_kernel<T, U><<<(unsigned)std::min(a.rows, most), threads, 0, st>>>(a);
    return cudaGetLastError() == cudaSuccess ? FQ_OK : FQ_ERR_CUDA;
}

template <class T>
int launch_typed(const QuantArgs& a, int sm_count, cudaStream_t st)
{
    const int pieces = a.cols / 8;
    const bool kept = a.cols % 8 == 0 && aligned(a.x, 16) && a.ldx * sizeof(T) % 16 == 0 && aligned(a.codes, 8) && a.ldc % 8 == 0;
    if (kept && a.rows <= sm_count && pieces <= 1024) return launch_kept<T, 1>(a, sm_count, st);
    if (kept && a.rows <= sm_count && pieces <= 2048) return launch_kept<T, 2>(a, sm_count, st);
    if (kept && pieces <= 4096) return launch_kept<T, 4>(a, sm_count, st);
    quantize_rows_kernel<T, 256><<<(unsigned)a.rows, 256, 0, st>>>(a);
    return cudaGetLastError() == cudaSuccess ? FQ_OK : FQ_ERR_CUDA;
}

}  // namespace

int launch_quantize_rows(const void* x, int dtype, int rows, int cols, long long ldx, int8_t* codes, long long ldc, float* scales,
                         int sm_count, cudaStream_t st)
{
    const QuantArgs a{x, ldx, rows, cols, codes, ldc, scales};
    if (dtype == FQ_DT_F32) return launch_typed<float>(a, sm_count, st);
    if (dtype == FQ_DT_F16) return launch_typed<__half>(a, sm_count, st);
    return launch_typed<__nv_bfloat16>(a, sm_count, st);
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
    return launch_quantize_rows(x_dev, dtype, rows, cols, ldx, codes_dev, ldc, scales_dev, ctx->sm_count, (cudaStream_t)stream);
}
