// 8-bit layers, a few tokens:  Y[m][n] = (sum_k xc[m][k] wc[n][k]) * sx[m] * sw[n]  for M <= 4.
//
// Bound by reading the weights once.  A CTA takes a run of output rows, and each of its warps the same columns of all of them: 512 columns, 16 to a
// lane, some slices of that kind where K is wide.  A lane's codes of the tokens then stay in registers for the whole kernel, a row costs a
// warp one 512-byte load per slice and four 4-way products per token, and rows depend on nothing, so that sixteen loads are on their
// way per lane.  The warps' sums meet in shared memory.  Sums are integers: their order does not matter.  1 x 4096 x 4096 4.7 us from codes and
// 5.5 us from fp16 (16.8 MB: 2.6 us at the rate of a copy), 1 x 13824 x 5120 12.4 us (11.0 us).
//
// One token that is not codes yet is quantised by every CTA for itself, while its first weights are on their way: that is a few
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
    int x_groups;                // the activations of a token come in 16-byte groups
};

// The largest absolute value of one token of up to kWarps * kSliceCols columns, then its codes, zero behind the last column.  Values stay in registers in
// between where they come in 16-byte groups of 16-bit ones, two for every thread.
template <class T>
__device__ __forceinline__ void quantise_here(const GemvArgs& a, int8_t* codes, float (&red)[kWarps], float& scale)
{
    constexpr int cols = kWarps * kSliceCols, U = 2;
    const T* x = static_cast<const T*>(a.x);
    const bool groups = sizeof(T) == 2 && a.x_groups;
    uint4 v[U];
#pragma unroll
    for (int u = 0; u < U; u++) {
        const int c = (u * kThreads + (int)threadIdx.x) * 8;
        v[u] = make_uint4(0u, 0u, 0u, 0u);
        if (groups && c < a.K) v[u] = *reinterpret_cast<const uint4*>(x + c);
    }
    float m = 0.0f;
    if (groups) {
        typename Group<T>::Max most = Group<T>::nothing();
#pragma unroll
        for (int u = 0; u < U; u++) Group<T>::take_abs(most, v[u]);
        m = Group<T>::of_abs(most);
    } else {
        for (int c = threadIdx.x; c < a.K; c += kThreads) m = max_nan(m, fabsf(Group<T>::to_f(x[c])));
    }
    m = warp_max_nan(m);
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = m;
    __syncthreads();
    m = red[0];
#pragma unroll
    for (int w = 1; w < kWarps; w++) m = max_nan(m, red[w]);
    const RowScale s(m);
    scale = RowScale::scale(m);
    if (groups) {
#pragma unroll
        for (int u = 0; u < U; u++) {
            float2 f[Group<T>::N / 2];
            Group<T>::unpack(v[u], f);
            const uint32_t lo = s.four(f[0], f[1]);
            const uint32_t hi = Group<T>::N == 8 ? s.four(f[Group<T>::N / 2 - 2], f[Group<T>::N / 2 - 1]) : 0u;
            *reinterpret_cast<uint2*>(codes + (u * kThreads + (int)threadIdx.x) * 8) = make_uint2(lo, hi);
        }
    } else {
        for (int c = threadIdx.x; c < cols; c += kThreads) codes[c] = c < a.K ? s.one(Group<T>::to_f(x[c])) : (int8_t)0;
    }
    __syncthreads();
}

template <class T, int M, int S>
__global__ void __launch_bounds__(kThreads, 2) gemv_i8_kernel(const GemvArgs a)
{
    extern __shared__ __align__(16) int8_t smem[];       // the codes of a token that is quantised here, then int [warps][rows][M]
    __shared__ float red[kWarps];
    constexpr int R = S <= 2 && M * S <= 4 ? kRowsAtATime : kRowsAtATime / 2;
    constexpr bool kCodes = sizeof(T) == 1;
    static_assert(kCodes || (M == 1 && S == 1), "one token of one slice a warp is quantised here");
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int r0 = (int)blockIdx.x * a.rows, r1 = min(a.N, r0 + a.rows);
    int* part = reinterpret_cast<int*>(smem + (kCodes ? 0 : kWarps * kSliceCols));
    const int col0 = warp * kSliceCols + lane * 16;      // of slice s: + s * kWarps * kSliceCols

    const auto load = [&](uint4 (&w)[R], int r, int s) {
        const int c = col0 + s * kWarps * kSliceCols;
        const int8_t* at = a.w + (long long)r * a.ldw + c;
#pragma unroll
        for (int i = 0; i < R; i++, at += a.ldw) {
            w[i] = make_uint4(0u, 0u, 0u, 0u);
            if (r + i < r1 && c < a.K)
                asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w[i].x), "=r"(w[i].y), "=r"(w[i].z), "=r"(w[i].w)
                             : "l"(at) : "memory");
        }
    };
    // two loads of R rows are always on their way: step i is slice i % S of rows r0 + (i / S) R, ...
    uint4 w[2][R];
    load(w[0], r0, 0);
    load(w[1], S == 1 ? r0 + R : r0, S == 1 ? 0 : 1);
    asm volatile("griddepcontrol.wait;" ::: "memory");   // (behind the quantiser: only its codes have to be waited for)
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
        quantise_here<T>(a, smem, red, scale[0]);
        xq[0][0] = *reinterpret_cast<const uint4*>(smem + col0);
    }
    const auto multiply = [&](const uint4 (&v)[R], int s, int (&acc)[R][M]) {
#pragma unroll
        for (int i = 0; i < R; i++)
#pragma unroll
            for (int t = 0; t < M; t++) {
                acc[i][t] = __dp4a((int)v[i].x, (int)xq[s][t].x, acc[i][t]);
                acc[i][t] = __dp4a((int)v[i].y, (int)xq[s][t].y, acc[i][t]);
                acc[i][t] = __dp4a((int)v[i].z, (int)xq[s][t].z, acc[i][t]);
                acc[i][t] = __dp4a((int)v[i].w, (int)xq[s][t].w, acc[i][t]);
            }
    };
    const auto finish = [&](int r, int (&acc)[R][M]) {
#pragma unroll
        for (int i = 0; i < R; i++)
#pragma unroll
            for (int t = 0; t < M; t++) {
                const int sum = __reduce_add_sync(0xffffffffu, acc[i][t]);
                if (lane == 0 && r + i < r1) part[(warp * a.rows + r - r0 + i) * M + t] = sum;
            }
    };
    if constexpr (S == 1) {
        for (int r = r0; r < r1; r += 2 * R)
#pragma unroll
            for (int h = 0; h < 2; h++) {
                int acc[R][M] = {};
                multiply(w[h], 0, acc);
                load(w[h], r + (2 + h) * R, 0);
                finish(r + h * R, acc);
            }
    } else {
        for (int r = r0; r < r1; r += R) {
            int acc[R][M] = {};
#pragma unroll
            for (int s = 0; s < S; s++) {
                multiply(w[s & 1], s, acc);
                load(w[s & 1], s + 2 < S ? r : r + R, s + 2 < S ? s + 2 : s + 2 - S);
            }
            finish(r, acc);
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
int launch(const Ctx* ctx, GemvArgs a, bool early, cudaStream_t st)
{
    const int ctas = 2 * ctx->sm_count;
    // the rows in even shares for two CTAs on every SM
    a.rows = std::min(kMaxRows, std::max(1, (a.N + ctas - 1) / ctas));
    const size_t smem = (sizeof(T) == 1 ? 0 : (size_t)kWarps * kSliceCols) + sizeof(int) * kWarps * (size_t)a.rows * M;
    static std::atomic<bool> ready[64];
    if (!ready[ctx->device].load(std::memory_order_acquire)) {
        if (cudaFuncSetAttribute(gemv_i8_kernel<T, M, S>, cudaFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024) != cudaSuccess) return FQ_ERR_CUDA;
        ready[ctx->device].store(true, std::memory_order_release);
    }
    cudaLaunchAttribute overlap{};
    overlap.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    overlap.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)((a.N + a.rows - 1) / a.rows)); cfg.blockDim = dim3(kThreads); cfg.dynamicSmemBytes = smem;
    cfg.stream = st; cfg.attrs = &overlap; cfg.numAttrs = early ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, gemv_i8_kernel<T, M, S>, a) == cudaSuccess ? FQ_OK : FQ_ERR_CUDA;
}

template <int M>
int launch_slices(const Ctx* ctx, const GemvArgs& a, bool early, cudaStream_t st)
{
    const int per_warp = ((a.K + kSliceCols - 1) / kSliceCols + kWarps - 1) / kWarps;
    if constexpr (M <= 2) {
        if (per_warp > 2) return launch<int8_t, M, kMaxSlices>(ctx, a, early, st);
    }
    return per_warp == 1 ? launch<int8_t, M, 1>(ctx, a, early, st) : launch<int8_t, M, 2>(ctx, a, early, st);
}

}  // namespace

// (Codes of four tokens and four slices do not fit beside the loads: 4 x 4096 x 11008 takes 17 us here and 12 us in strips.)
bool gemv_i8_takes(int M, int k_in) { return M <= 4 && k_in <= (M <= 2 ? kMaxSlices : 2) * kWarps * kSliceCols; }
// One token of up to 4096 columns.  More of them take every CTA longer than a launch of the quantiser does, behind which this kernel starts early (4
// tokens x 4096 columns, 4096 outputs: 11.8 us against 8.1 us).
bool gemv_i8_quantises(int M, int k_in) { return M == 1 && k_in <= kWarps * kSliceCols; }

// x_dtype: FQ_DT_*, or -1 for codes with their scales
int launch_gemv_i8(const Ctx* ctx, const void* x, int x_dtype, long long ldx, const float* sx, int M, const int8_t* w, const float* sw, int n_out,
                   int k_in, long long ldw, void* y, int y_dtype, long long ldy, bool early, cudaStream_t st)
{
    if (ctx->device >= 64) return FQ_ERR_ARG;
    const GemvArgs a{x, ldx, sx, w, ldw, sw, y, ldy, y_dtype, n_out, k_in, 0, k_in % 8 == 0 && aligned(x, 16)};
    if (x_dtype == FQ_DT_F32) return launch<float, 1, 1>(ctx, a, early, st);
    if (x_dtype == FQ_DT_F16) return launch<__half, 1, 1>(ctx, a, early, st);
    if (x_dtype == FQ_DT_BF16) return launch<__nv_bfloat16, 1, 1>(ctx, a, early, st);
    return M == 1 ? launch_slices<1>(ctx, a, early, st) : M == 2 ? launch_slices<2>(ctx, a, early, st) : M == 3 ? launch_slices<3>(ctx, a, early, st)
                  : launch_slices<4>(ctx, a, early, st);
}

}  // namespace fq
