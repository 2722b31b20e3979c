// 8-bit layers, a few tokens:  Y[m][n] = (sum_k xc[m][k] wc[n][k]) * sx[m] * sw[n]  for M <= 4.
//
// Bound by reading the weights once.  A CTA takes a run of output rows, and each of its warps the same columns of all of them: 512 columns, 16 to a
// lane, some slices of that kind where K is wide.  A lane's codes of the tokens then stay in registers for the whole kernel, a row costs a
// warp one 512-byte load per slice and four 4-way products per token, and rows depend on nothing, so that sixteen loads are on their
// way per lane.  The warps' sums meet in shared memory.  Sums are integers: their order does not matter.
//
// Activations that are not codes yet are quantised by every CTA for itself, while its first weights are on their way: that is a few
// thousand values from the L2, and saves a launch.
#include <algorithm>
#include <atomic>

#include "fq_internal.cuh"
#include "fq_rowtypes.cuh"

namespace fq {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kSliceCols = 512;                          // columns of a warp's load
constexpr int kRowsAtATime = 8;
constexpr int kMaxRows = 512;                            // output rows of a CTA
constexpr int kMaxSlices = 4;                            // slices of a warp

struct GemvArgs {
    const void* x;               // codes (int8) or activations
    long long ldx;
    const float* sx;             // scales of the codes
    const int8_t* w;
    long long ldw;
    const float* sw;
    void* y;
    long long ldy;
    int y_dtype;
    int N, K, rows;              // rows: output rows of a CTA
};

// Largest absolute values of the tokens, then their codes, zero behind the last column.
template <class T, int M>
__device__ __forceinline__ void quantise_here(const GemvArgs& a, int cols, int8_t* codes, float (&red)[M][kWarps], float (&scale)[M])
{
    const T* x = static_cast<const T*>(a.x);
    float m[M];
#pragma unroll
    for (int t = 0; t < M; t++) {
        m[t] = 0.0f;
        for (int c = threadIdx.x; c < a.K; c += kThreads) m[t] = max_nan(m[t], fabsf(Group<T>::to_f(x[t * a.ldx + c])));
        m[t] = warp_max_nan(m[t]);
        if ((threadIdx.x & 31) == 0) red[t][threadIdx.x >> 5] = m[t];
    }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < M; t++) {
        float largest = red[t][0];
#pragma unroll
        for (int w = 1; w < kWarps; w++) largest = max_nan(largest, red[t][w]);
        const RowScale s(largest);
        scale[t] = s.scale;
        for (int c = threadIdx.x; c < cols; c += kThreads)
            codes[t * cols + c] = c < a.K ? (int8_t)s.code(Group<T>::to_f(x[t * a.ldx + c])) : (int8_t)0;
    }
    __syncthreads();
}

template <class T, int M, int S>
__global__ void __launch_bounds__(kThreads, 2) gemv_i8_kernel(const GemvArgs a)
{
    extern __shared__ __align__(16) int8_t smem[];       // [M][columns] codes, then int [warps][rows][M]
    __shared__ float red[M][kWarps];
    constexpr int R = M * S <= 4 ? kRowsAtATime : kRowsAtATime / 2;
    constexpr bool kCodes = sizeof(T) == 1;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int r0 = (int)blockIdx.x * a.rows, r1 = min(a.N, r0 + a.rows);
    const int n_slices = (a.K + kSliceCols - 1) / kSliceCols, cols = n_slices * kSliceCols;
    int* part = reinterpret_cast<int*>(smem + (kCodes ? 0 : M * cols));
    const int col0 = warp * kSliceCols + lane * 16;      // of slice s: + s * kWarps * kSliceCols

    const auto load = [&](uint4 (&w)[R], int r, int s) {
        const int c = col0 + s * kWarps * kSliceCols;
#pragma unroll
        for (int i = 0; i < R; i++) {
            w[i] = make_uint4(0u, 0u, 0u, 0u);
            if (r + i < r1 && c < a.K)
                asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w[i].x), "=r"(w[i].y), "=r"(w[i].z), "=r"(w[i].w)
                             : "l"(a.w + (long long)(r + i) * a.ldw + c) : "memory");
        }
    };
    uint4 w[R];
    load(w, r0, 0);
    uint4 xq[S][M];
    float scale[M];
    if constexpr (kCodes) {
#pragma unroll
        for (int t = 0; t < M; t++) scale[t] = a.sx[t];
#pragma unroll
        for (int s = 0; s < S; s++)
#pragma unroll
            for (int t = 0; t < M; t++) {
                const int c = col0 + s * kWarps * kSliceCols, left = a.K - c;
                xq[s][t] = make_uint4(0u, 0u, 0u, 0u);
                if (left > 0) xq[s][t] = *reinterpret_cast<const uint4*>(static_cast<const int8_t*>(a.x) + t * a.ldx + c);
                if (left < 16) {                         // what lies behind the last column does not count
                    uint32_t* q = &xq[s][t].x;
#pragma unroll
                    for (int i = 0; i < 4; i++) q[i] = left >= 4 * i + 4 ? q[i] : left <= 4 * i ? 0u : q[i] & ((1u << 8 * (left - 4 * i)) - 1u);
                }
            }
    } else {
        quantise_here<T, M>(a, cols, smem, red, scale);
#pragma unroll
        for (int s = 0; s < S; s++)
#pragma unroll
            for (int t = 0; t < M; t++) {
                const int c = col0 + s * kWarps * kSliceCols;
                xq[s][t] = c < cols ? *reinterpret_cast<const uint4*>(smem + t * cols + c) : make_uint4(0u, 0u, 0u, 0u);
            }
    }
    for (int r = r0; r < r1; r += R) {
        int acc[R][M] = {};
#pragma unroll
        for (int s = 0; s < S; s++) {
            uint4 next[R];
            if (s + 1 < S) load(next, r, s + 1); else load(next, r + R, 0);
#pragma unroll
            for (int i = 0; i < R; i++)
#pragma unroll
                for (int t = 0; t < M; t++) {
                    acc[i][t] = __dp4a((int)w[i].x, (int)xq[s][t].x, acc[i][t]);
                    acc[i][t] = __dp4a((int)w[i].y, (int)xq[s][t].y, acc[i][t]);
                    acc[i][t] = __dp4a((int)w[i].z, (int)xq[s][t].z, acc[i][t]);
                    acc[i][t] = __dp4a((int)w[i].w, (int)xq[s][t].w, acc[i][t]);
                }
#pragma unroll
            for (int i = 0; i < R; i++) w[i] = next[i];
        }
#pragma unroll
        for (int i = 0; i < R; i++)
#pragma unroll
            for (int t = 0; t < M; t++) {
                const int sum = __reduce_add_sync(0xffffffffu, acc[i][t]);
                if (lane == 0 && r + i < r1) part[(warp * a.rows + r - r0 + i) * M + t] = sum;
            }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < (r1 - r0) * M; i += kThreads) {
        const int t = i / (r1 - r0), n = i % (r1 - r0);
        int sum = 0;
#pragma unroll
        for (int k = 0; k < kWarps; k++) sum += part[(k * a.rows + n) * M + t];
        float sx = scale[0];
#pragma unroll
        for (int j = 1; j < M; j++) sx = t == j ? scale[j] : sx;
        const float v = (float)sum * sx * a.sw[r0 + n];
        const long long at = t * a.ldy + r0 + n;
        if (a.y_dtype == FQ_DT_F32) static_cast<float*>(a.y)[at] = v;
        else if (a.y_dtype == FQ_DT_F16) static_cast<__half*>(a.y)[at] = __float2half_rn(v);
        else static_cast<__nv_bfloat16*>(a.y)[at] = __float2bfloat16_rn(v);
    }
}

template <class T, int M, int S>
int launch(const Ctx* ctx, GemvArgs a, cudaStream_t st)
{
    const int cols = (a.K + kSliceCols - 1) / kSliceCols * kSliceCols, ctas = 2 * ctx->sm_count;
    // the rows in even shares for two CTAs on every SM; a share is a whole number of loads at a time where that leaves no SM idle
    a.rows = std::min(kMaxRows, std::max(1, (a.N + ctas - 1) / ctas));
    const size_t smem = (sizeof(T) == 1 ? 0 : (size_t)M * cols) + sizeof(int) * kWarps * (size_t)a.rows * M;
    static std::atomic<bool> ready[64];
    if (!ready[ctx->device].load(std::memory_order_acquire)) {
        if (cudaFuncSetAttribute(gemv_i8_kernel<T, M, S>, cudaFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024) != cudaSuccess) return FQ_ERR_CUDA;
        ready[ctx->device].store(true, std::memory_order_release);
    }
    gemv_i8_kernel<T, M, S><<<(unsigned)((a.N + a.rows - 1) / a.rows), kThreads, smem, st>>>(a);
    return cudaGetLastError() == cudaSuccess ? FQ_OK : FQ_ERR_CUDA;
}

template <class T, int M>
int launch_slices(const Ctx* ctx, const GemvArgs& a, cudaStream_t st)
{
    const int per_warp = ((a.K + kSliceCols - 1) / kSliceCols + kWarps - 1) / kWarps;
    return per_warp == 1 ? launch<T, M, 1>(ctx, a, st) : per_warp == 2 ? launch<T, M, 2>(ctx, a, st) : launch<T, M, kMaxSlices>(ctx, a, st);
}

// (M is the number of tokens, exactly: a kernel for four would read a fourth one)
template <class T>
int launch_tokens(const Ctx* ctx, int M, const GemvArgs& a, cudaStream_t st)
{
    return M == 1 ? launch_slices<T, 1>(ctx, a, st) : M == 2 ? launch_slices<T, 2>(ctx, a, st) : M == 3 ? launch_slices<T, 3>(ctx, a, st)
                  : launch_slices<T, 4>(ctx, a, st);
}

}  // namespace

bool gemv_i8_takes(int M, int k_in) { return M <= 4 && k_in <= kMaxSlices * kWarps * kSliceCols; }

// x_dtype: FQ_DT_*, or -1 for codes with their scales
int launch_gemv_i8(const Ctx* ctx, const void* x, int x_dtype, long long ldx, const float* sx, int M, const int8_t* w, const float* sw, int n_out,
                   int k_in, long long ldw, void* y, int y_dtype, long long ldy, cudaStream_t st)
{
    if (ctx->device >= 64) return FQ_ERR_ARG;
    const GemvArgs a{x, ldx, sx, w, ldw, sw, y, ldy, y_dtype, n_out, k_in, 0};
    if (x_dtype == FQ_DT_F32) return launch_tokens<float>(ctx, M, a, st);
    if (x_dtype == FQ_DT_F16) return launch_tokens<__half>(ctx, M, a, st);
    if (x_dtype == FQ_DT_BF16) return launch_tokens<__nv_bfloat16>(ctx, M, a, st);
    return launch_tokens<int8_t>(ctx, M, a, st);
}

}  // namespace fq
