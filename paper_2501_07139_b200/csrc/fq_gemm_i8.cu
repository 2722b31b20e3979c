// 8-bit layers:  Y[m][n] = (sum_k xc[m][k] wc[n][k]) * sx[m] * sw[n],  int8 codes, exact int32 sums in TMEM.
//
// gemm_i8_pair_kernel is the persistent, warp-specialised tcgen05 GEMM over pairs of SMs of fq_gemm.cu with 8-bit operands: a stage of
// 128 bytes of K holds 128 columns instead of 64, so the same copies feed twice the products.  The scales are applied where an
// accumulator leaves TMEM, an epilogue of 1400 instructions a warp beside 16000 cycles of MMAs (K = 4096).  8192 x 11008 x 4096: 230 us
// (3.2 PTOP/s) from a cool start, 250 us back to back, where the clock is what the power limit leaves; tensor pipe 90 %.
// Prompts of 129 .. 2047 tokens are two to five times their floor (512 x 4096 x 4096 15 us for the product, 18 us with the quantiser in front of it;
// floor 5.2 us): where a pair has one tile, nothing covers its epilogue, 1 us for 32 outputs, and the weights wait for the quantiser too.
// Every mbarrier wait is bounded by a timer; when one runs out the kernel records FQ_ERR_TIMEOUT, all roles
// leave their loops, and the TMEM allocation is released before the CTA exits.
#include <cuda.h>
#include <cudaTypedefs.h>

#include <algorithm>
#include <atomic>

#include "fq_cluster.cuh"
#include "fq_internal.cuh"
#include "fq_ptx.cuh"
#include "fq_rowtypes.cuh"
#include "fq_umma.cuh"

namespace fq {
namespace {

#define FQ_CUDA_OK(expr) do { if ((expr) != cudaSuccess) return FQ_ERR_CUDA; } while (0)

constexpr int kBM = 128;                 // tokens per CTA (UMMA M = 256 over the pair)
constexpr int kBN = 256;                 // outputs per tile, at most (UMMA N)
constexpr int kBK = 128;                 // K per stage: one 128-byte swizzle span
constexpr int kMaxStages = 8;
constexpr int kThreads = 192;            // warp 0: TMA, warp 1: TMEM owner, of the leading CTA also MMA; warps 2..5: epilogue
constexpr int kTmemCols = 512;           // two accumulators of up to kBN columns

// A stage holds 128 tokens and half of the tile's outputs: six stages of 256 outputs, seven or eight of fewer, where a tile's time is that of
// its loads more than that of its products (512 x 4096 x 4096, 128 outputs: 15.7 us with six stages, 15.0 us with eight).
struct PairSmem {
    static constexpr int kABytes = kBM * kBK;                      // 16 KB
    static constexpr int kTiles = 6 * (kABytes + kBN / 2 * kBK);   // 192 KB
    static constexpr int oBars = kTiles;                           // full[S], empty[S], tmem_full[2], tmem_empty[2]
    static constexpr int oTmemPtr = oBars + (2 * kMaxStages + 4) * 8;
    static constexpr int oFlag = oTmemPtr + 8;
    static constexpr int kTotal = oFlag + 8 + 1024;                // + slack for the 1024-byte alignment of the tiles
};
static_assert(PairSmem::kTotal <= 232448, "int8 GEMM: shared memory over the per-CTA limit");

struct I8Args {
    const float* sx;
    const float* sw;
    void* y;
    int M, N, K;
    long long ldy;
    int tile_n;
    int* status;
};

__device__ __forceinline__ void tmem_ld32(uint32_t (&v)[32], uint32_t addr)
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
          "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]),
          "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]),
          "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
        : "r"(addr) : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

__device__ __forceinline__ void tmem_ld16(uint32_t (&v)[16], uint32_t addr)
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
          "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
        : "r"(addr) : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar)
{
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
        ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}

// 32 neighbouring outputs of a row: `n` of them exist, dst is 16-byte aligned.
template <class T>
__device__ __forceinline__ void store_outputs(T* dst, const float (&f)[32], int n)
{
    constexpr int G = Group<T>::N;
    if (n >= 32) {
#pragma unroll
        for (int g = 0; g < 32 / G; g++) {
            float2 p[G / 2];
#pragma unroll
            for (int e = 0; e < G / 2; e++) p[e] = make_float2(f[g * G + 2 * e], f[g * G + 2 * e + 1]);
            reinterpret_cast<uint4*>(dst)[g] = Group<T>::pack(p);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 32; e++)
            if (e < n) dst[e] = Group<T>::from_f(f[e]);
    }
}

// Four neighbouring outputs, dst aligned to four of them.
template <class T>
__device__ __forceinline__ void store_four(T* dst, const float (&f)[4], int n)
{
    if (n >= 4) {
        if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<float4*>(dst) = make_float4(f[0], f[1], f[2], f[3]);
        } else {
            T h[4] = {Group<T>::from_f(f[0]), Group<T>::from_f(f[1]), Group<T>::from_f(f[2]), Group<T>::from_f(f[3])};
            *reinterpret_cast<uint2*>(dst) = *reinterpret_cast<const uint2*>(h);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; i++)
            if (i < n) dst[i] = Group<T>::from_f(f[i]);
    }
}

template <class T>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
gemm_i8_pair_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w, const I8Args a)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = (int)cluster_rank(), pair = (int)(blockIdx.x >> 1), n_pairs = (int)(gridDim.x >> 1);
    const uint32_t bars = g_smem_u32(smem + PairSmem::oBars);
    // a stage's "full" and an accumulator's "empty" barriers are those of the leading CTA, the others exist in both
    const uint32_t full0 = bars, empty0 = bars + 8 * kMaxStages;
    const uint32_t tfull0 = bars + 16 * kMaxStages, tempty0 = tfull0 + 16;
    const int tile_n = a.tile_n, stage_bytes = PairSmem::kABytes + tile_n / 2 * kBK;
    const int stages = min(kMaxStages, PairSmem::kTiles / stage_bytes);
    volatile uint32_t* tmem_ptr = reinterpret_cast<volatile uint32_t*>(smem + PairSmem::oTmemPtr);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + PairSmem::oFlag);

    if (threadIdx.x == 0) {
        for (int s = 0; s < stages; s++) {
            mbar_init(full0 + 8 * s, 1);
            mbar_init(empty0 + 8 * s, 1);
        }
        for (int b = 0; b < 2; b++) {
            mbar_init(tfull0 + 8 * b, 1);
            mbar_init(tempty0 + 8 * b, 8);                              // one arrival per epilogue warp of both CTAs
        }
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) {                     // this warp owns the TMEM allocation
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;"
                     ::"r"(g_smem_u32(const_cast<uint32_t*>(tmem_ptr))), "n"(kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    cluster_sync();                      // the peer's barriers exist, its TMEM is allocated
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem_base = *tmem_ptr;
    asm volatile("griddepcontrol.wait;" ::: "memory");                  // the codes are the previous kernel's output

    const int m_blocks = (a.M + 2 * kBM - 1) / (2 * kBM), n_blocks = (a.N + tile_n - 1) / tile_n;
    const int n_tiles = m_blocks * n_blocks;
    const int k_steps = (a.K + kBK - 1) / kBK;

    if (warp == 0) {
        // ================================================================== TMA producer
        if (lane == 0) {
            const uint32_t bytes = 2u * (uint32_t)stage_bytes;        // of both CTAs
            int stage = 0;
            uint32_t wraps = 0;
            bool ok = true;
            for (int t = pair; t < n_tiles && ok; t += n_pairs) {
                const int mb = t % m_blocks, nb = t / m_blocks;        // m fastest: the weight tile stays in L2
                for (int ks = 0; ks < k_steps; ks++) {
                    if (wraps > 0 && !g_wait(empty0 + 8 * stage, (wraps - 1u) & 1u, abort_flag)) { ok = false; break; }
                    const uint32_t full = in_leader(full0 + 8 * stage);
                    const uint32_t a_dst = g_smem_u32(smem + stage * stage_bytes);
                    if (rank == 0) mbar_expect_tx(full0 + 8 * stage, bytes);
                    tma_load_pair(a_dst, &map_x, ks * kBK, mb * (2 * kBM) + rank * kBM, full);
                    tma_load_pair(a_dst + PairSmem::kABytes, &map_w, ks * kBK, nb * tile_n + rank * (tile_n / 2), full);
                    if (++stage == stages) { stage = 0; wraps++; }
                }
            }
            if (!ok) { atomicCAS(a.status, 0, FQ_ERR_TIMEOUT); *abort_flag = 1; }
        }
    } else if (warp == 1) {
        if (rank == 0) {
            // ============================================================== MMA issuer (for both CTAs)
            const uint32_t idesc = umma_idesc_i8(2 * kBM, tile_n);
            const uint64_t adesc0 = umma_desc_sw128(g_smem_u32(smem)), bdesc0 = umma_desc_sw128(g_smem_u32(smem) + PairSmem::kABytes);
            int stage = 0;
            uint32_t wraps = 0;
            int local = 0;
            bool ok = true;
            for (int t = pair; t < n_tiles && ok; t += n_pairs, local++) {
                const int buf = local & 1;
                const uint32_t use = (uint32_t)(local >> 1);           // how often this accumulator was used before
                if (use > 0) ok = __all_sync(0xffffffffu, g_wait(tempty0 + 8 * buf, (use - 1u) & 1u, abort_flag));
                if (!ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t d_tmem = tmem_base + (uint32_t)(buf * kBN);
                for (int ks = 0; ks < k_steps; ks++) {
                    ok = __all_sync(0xffffffffu, g_wait(full0 + 8 * stage, wraps & 1u, abort_flag));
                    if (!ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint64_t step = (uint64_t)(uint32_t)(stage * (stage_bytes >> 4));
                    const uint32_t more = ks > 0 ? 1u : 0u;
                    if (elect_one()) {
#pragma unroll
                        for (int kk = 0; kk < kBK / 32; kk++)
                            asm volatile(
                                "{\n\t.reg .pred p;\n\t"
                                "setp.ne.b32 p, %4, 0;\n\t"
                                "tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}"
                                ::"r"(d_tmem), "l"(adesc0 + step + (uint64_t)(kk * 2)), "l"(bdesc0 + step + (uint64_t)(kk * 2)), "r"(idesc),
                                  "r"(kk > 0 ? 1u : more) : "memory");
                        commit_pair(empty0 + 8 * stage);               // the stage may be refilled once these MMAs have read it
                    }
                    __syncwarp();
                    if (++stage == stages) { stage = 0; wraps++; }
                }
                if (!ok) break;
                if (elect_one()) commit_pair(tfull0 + 8 * buf);
                __syncwarp();
            }
            if (!ok && lane == 0) { atomicCAS(a.status, 0, FQ_ERR_TIMEOUT); *abort_flag = 1; }
        }
    } else {
        // ================================================================== epilogue (warps 2..5)
        const int quarter = warp & 3;                                   // TMEM lanes 32*quarter .. +31 belong to this warp
        int local = 0;
        bool ok = true;
        for (int t = pair; t < n_tiles && ok; t += n_pairs, local++) {
            const int mb = t % m_blocks, nb = t / m_blocks;
            const int buf = local & 1;
            const uint32_t use = (uint32_t)(local >> 1);
            ok = __all_sync(0xffffffffu, g_wait<64>(tfull0 + 8 * buf, use & 1u, abort_flag));
            if (!ok) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const int row = mb * (2 * kBM) + rank * kBM + quarter * 32 + lane;      // token
            const float sx = row < a.M ? a.sx[row] : 0.0f;
            const uint32_t taddr0 = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(buf * kBN);
#pragma unroll 1
            for (int cb = 0; cb < tile_n / 32; cb++) {
                const int col0 = nb * tile_n + cb * 32;
                const float sw = col0 + lane < a.N ? a.sw[col0 + lane] : 0.0f;
                uint32_t v[32];
                tmem_ld32(v, taddr0 + (uint32_t)(cb * 32));
                float f[32];
#pragma unroll
                for (int e = 0; e < 32; e++) f[e] = (float)(int)v[e] * sx * __shfl_sync(0xffffffffu, sw, e);
                if (row < a.M && col0 < a.N) store_outputs(static_cast<T*>(a.y) + (long long)row * a.ldy + col0, f, a.N - col0);
            }
            // the accumulator may be overwritten
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0)
                asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(in_leader(tempty0 + 8 * buf)) : "memory");
        }
        if (!ok && lane == 0) { atomicCAS(a.status, 0, FQ_ERR_TIMEOUT); *abort_flag = 1; }
    }

    // every path ends here.  After a wait that ran out, copies may still be on their way into shared memory: they land within
    // microseconds, the CTAs leave much later.
    __syncthreads();
    if (*abort_flag) let_copies_land();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    cluster_sync();                      // nobody reads this CTA's shared memory or arrives at its barriers any more
    if (warp == 1) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "n"(kTmemCols) : "memory");
    }
}

// ------------------------------------------------------------------------------- some tokens: weights in strips
// Up to kStripTokens tokens: the weights are the larger operand by far, and the time is that of reading them.  Roles change places: a tile is 128
// outputs (UMMA M) x all the tokens (UMMA N, a multiple of 16), and K is split over the CTAs of a cluster so that all SMs read at once.
// The CTAs' sums, 32-bit integers whose order does not matter, meet in distributed shared memory: CTA r of the cluster adds up
// and writes the tokens r, r + S, ...
//
// 8 x 11008 x 4096 12.4 us, 77 x 4096 x 11008 15.8 us, of which 8 us are HBM's; the rest is launch, first bytes and the exchange.  (The kernel for pairs of
// SMs takes 24 us and 34 us: its tiles leave most SMs idle.)
//
// Behind the quantiser the kernel starts early and fetches weights while the tokens are still being quantised: the quantiser has waited for everything
// before it, so that the weights are there; only the codes have to be waited for.
constexpr int kStripTokens = 128;
constexpr int kStripTmemCols = 128;
constexpr int kStripStageW = 128 * kBK;                  // 16 KB
constexpr int kStripMaxStages = 12, kMaxSplits = 8;

struct StripArgs {
    I8Args a;
    int nt;                      // tokens of a tile
    int stages;
    int splits;                  // CTAs of a cluster
    int early;                   // the previous kernel writes the codes, and nothing else that is read here
};

constexpr int strip_bars_bytes() { return (2 * kStripMaxStages + 1) * 8 + 16; }

template <class T>
__global__ void __launch_bounds__(kThreads) gemm_i8_strip_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w,
                                                                 const StripArgs q)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = q.splits > 1 ? (int)cluster_rank() : 0, tile = (int)blockIdx.x / q.splits, m0 = (int)blockIdx.y * q.nt;
    const int stage_bytes = kStripStageW + q.nt * kBK;
    uint8_t* tail = smem + q.stages * stage_bytes;
    const uint32_t bars = g_smem_u32(tail), full0 = bars, empty0 = bars + 8 * kStripMaxStages, done = bars + 16 * kStripMaxStages;
    volatile uint32_t* tmem_ptr = reinterpret_cast<volatile uint32_t*>(tail + (2 * kStripMaxStages + 1) * 8);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_ptr + 1);
    const I8Args& a = q.a;

    if (threadIdx.x == 0) {
        for (int s = 0; s < q.stages; s++) {
            mbar_init(full0 + 8 * s, 1);
            mbar_init(empty0 + 8 * s, 1);
        }
        mbar_init(done, 1);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) {                     // this warp owns the TMEM allocation
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                     ::"r"(g_smem_u32(const_cast<uint32_t*>(tmem_ptr))), "n"(kStripTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem_base = *tmem_ptr;

    const int k_steps = (a.K + kBK - 1) / kBK;
    const int k0 = (int)((long long)k_steps * rank / q.splits), k1 = (int)((long long)k_steps * (rank + 1) / q.splits);
    if (!q.early) asm volatile("griddepcontrol.wait;" ::: "memory");

    if (warp == 0) {
        // ================================================================== TMA producer
        if (lane == 0) {
            const auto stage_at = [&](int s) { return g_smem_u32(smem + s * stage_bytes); };
            const int ahead = k1 - k0 < q.stages ? k1 - k0 : q.stages;
            for (int s = 0; s < ahead; s++) {
                mbar_expect_tx(full0 + 8 * s, (uint32_t)stage_bytes);
                tma_load_2d(stage_at(s), &map_w, (k0 + s) * kBK, tile * 128, full0 + 8 * s);
            }
            if (q.early) asm volatile("griddepcontrol.wait;" ::: "memory");
            for (int s = 0; s < ahead; s++) tma_load_2d(stage_at(s) + kStripStageW, &map_x, (k0 + s) * kBK, m0, full0 + 8 * s);
            int stage = 0;
            uint32_t wraps = 0;
            bool ok = true;
            for (int ks = k0 + ahead; ks < k1 && ok; ks++) {
                ok = g_wait(empty0 + 8 * stage, wraps & 1u, abort_flag);
                if (!ok) break;
                mbar_expect_tx(full0 + 8 * stage, (uint32_t)stage_bytes);
                tma_load_2d(stage_at(stage), &map_w, ks * kBK, tile * 128, full0 + 8 * stage);
                tma_load_2d(stage_at(stage) + kStripStageW, &map_x, ks * kBK, m0, full0 + 8 * stage);
                if (++stage == q.stages) { stage = 0; wraps++; }
            }
            if (!ok) { atomicCAS(a.status, 0, FQ_ERR_TIMEOUT); *abort_flag = 1; }
        }
    } else if (warp == 1) {
        // ================================================================== MMA issuer
        const uint32_t idesc = umma_idesc_i8(128, q.nt);
        const uint64_t adesc0 = umma_desc_sw128(g_smem_u32(smem)), bdesc0 = umma_desc_sw128(g_smem_u32(smem) + kStripStageW);
        int stage = 0;
        uint32_t wraps = 0;
        bool ok = true;
        for (int ks = k0; ks < k1; ks++) {
            ok = __all_sync(0xffffffffu, g_wait(full0 + 8 * stage, wraps & 1u, abort_flag));
            if (!ok) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint64_t step = (uint64_t)((uint32_t)(stage * stage_bytes) >> 4);
            const uint32_t more = ks > k0 ? 1u : 0u;
            if (elect_one()) {
#pragma unroll
                for (int kk = 0; kk < kBK / 32; kk++)
                    asm volatile(
                        "{\n\t.reg .pred p;\n\t"
                        "setp.ne.b32 p, %4, 0;\n\t"
                        "tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}"
                        ::"r"(tmem_base), "l"(adesc0 + step + (uint64_t)(kk * 2)), "l"(bdesc0 + step + (uint64_t)(kk * 2)), "r"(idesc),
                          "r"(kk > 0 ? 1u : more) : "memory");
                umma_commit(empty0 + 8 * stage);
            }
            __syncwarp();
            if (++stage == q.stages) { stage = 0; wraps++; }
        }
        if (ok && elect_one()) umma_commit(done);
        __syncwarp();
        if (!ok && lane == 0) { atomicCAS(a.status, 0, FQ_ERR_TIMEOUT); *abort_flag = 1; }
    } else {
        // ================================================================== epilogue (warps 2..5)
        const int quarter = warp & 3, row = quarter * 32 + lane, n = tile * 128 + row;      // output
        const bool ok = __all_sync(0xffffffffu, g_wait<64>(done, 0, abort_flag));
        if (ok) {
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const float sw = n < a.N ? a.sw[n] : 0.0f;
            if (q.early) asm volatile("griddepcontrol.wait;" ::: "memory");                 // the tokens' scales
            int* part = reinterpret_cast<int*>(smem);                                        // [token][128]; every copy and every MMA is done
#pragma unroll 1
            for (int t0 = 0; t0 < q.nt; t0 += 16) {
                uint32_t v[16];
                tmem_ld16(v, tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)t0);
#pragma unroll
                for (int t = 0; t < 16; t++) {
                    if (q.splits > 1) {
                        part[(t0 + t) * 128 + row] = (int)v[t];
                    } else if (n < a.N && m0 + t0 + t < a.M) {
                        static_cast<T*>(a.y)[(long long)(m0 + t0 + t) * a.ldy + n] = Group<T>::from_f((float)(int)v[t] * a.sx[m0 + t0 + t] * sw);
                    }
                }
            }
        } else if (lane == 0) {
            atomicCAS(a.status, 0, FQ_ERR_TIMEOUT);
            *abort_flag = 1;
        }
    }
    if (q.splits > 1) {
        cluster_arrive();
        cluster_wait();                  // all CTAs' sums are in their shared memory
        if (warp >= 2) {
            // a warp takes a token, a lane four of its outputs
            const int n = tile * 128 + 4 * lane, end = a.M - m0 < q.nt ? a.M - m0 : q.nt;
            float sw[4];
#pragma unroll
            for (int i = 0; i < 4; i++) sw[i] = n + i < a.N ? a.sw[n + i] : 0.0f;
            const uint32_t at = g_smem_u32(smem) + (uint32_t)lane * 16;
            for (int t = rank + q.splits * (warp - 2); t < end; t += q.splits * 4) {
                int4 v[kMaxSplits];
#pragma unroll
                for (int c = 0; c < kMaxSplits; c++) {
                    v[c] = make_int4(0, 0, 0, 0);
                    if (c < q.splits) v[c] = cluster_ld_s32x4(cluster_map(at, (uint32_t)c) + (uint32_t)t * 512);
                }
#pragma unroll
                for (int c = 1; c < kMaxSplits; c++) {
                    v[0].x += v[c].x; v[0].y += v[c].y; v[0].z += v[c].z; v[0].w += v[c].w;
                }
                const float sx = a.sx[m0 + t];
                const float f[4] = {(float)v[0].x * sx * sw[0], (float)v[0].y * sx * sw[1], (float)v[0].z * sx * sw[2], (float)v[0].w * sx * sw[3]};
                store_four(static_cast<T*>(a.y) + (long long)(m0 + t) * a.ldy + n, f, a.N - n);
            }
        }
        cluster_arrive();
        cluster_wait();                  // nobody's shared memory is read any more
    }
    // every path ends here.  After a wait that ran out, copies may still be on their way into shared memory.
    __syncthreads();
    if (*abort_flag) let_copies_land();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (warp == 1) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "n"(kStripTmemCols) : "memory");
    }
}

// ------------------------------------------------------------------------------- host side
// K is split until there are two to three CTAs for every SM, which then share its memory: one waits, adds up or writes while others read.
struct StripPlan { int nt, blocks, splits, stages; size_t smem; };
StripPlan strip_plan(const Ctx* ctx, int M, int N, int K)
{
    StripPlan p{};
    p.blocks = (M + kStripTokens - 1) / kStripTokens;
    p.nt = ((M + p.blocks - 1) / p.blocks + 15) / 16 * 16;
    const int tiles = (N + 127) / 128 * p.blocks, k_steps = (K + kBK - 1) / kBK, stage = kStripStageW + p.nt * kBK;
    p.splits = 1;
    while (p.splits < kMaxSplits && tiles * p.splits * 2 <= 3 * ctx->sm_count && k_steps >= 4 * p.splits) p.splits *= 2;
    const int per = std::min(3, (tiles * p.splits + ctx->sm_count - 1) / ctx->sm_count);
    const int room = (per == 1 ? 220 : per == 2 ? 110 : 72) * 1024 - 1024 - strip_bars_bytes();
    p.stages = room / stage;
    if (p.stages > kStripMaxStages) p.stages = kStripMaxStages;
    p.smem = (size_t)p.stages * stage + strip_bars_bytes() + 1024;
    return p;
}

// Strips up to 128 tokens, and up to 256 where the pairs' tiles, one row of them, would leave many SMs idle (256 tokens, 4096 x 11008: 21 us
// against 27 us; 11008 x 4096: 26 us against 19 us).
bool takes_strips(const Ctx* ctx, int M, int N)
{
    return M <= kStripTokens || (M <= 2 * kStripTokens && (N + 127) / 128 * 10 <= ctx->sm_count / 2 * 6);
}

template <class T>
int launch_strip(const Ctx* ctx, const int8_t* xc, long long ldx, const int8_t* wc, long long ldw, const I8Args& a, bool early, cudaStream_t st)
{
    static std::atomic<bool> ready[64];
    if (ctx->device >= 64) return FQ_ERR_ARG;
    if (!ready[ctx->device].load(std::memory_order_acquire)) {
        FQ_CUDA_OK(cudaFuncSetAttribute(gemm_i8_strip_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, 220 * 1024));
        ready[ctx->device].store(true, std::memory_order_release);
    }
    const StripPlan p = strip_plan(ctx, a.M, a.N, a.K);
    CUtensorMap map_x, map_w;
    int rc = make_map_i8(&map_x, xc, a.M, a.K, ldx, p.nt);
    if (rc != FQ_OK) return rc;
    rc = make_map_i8(&map_w, wc, a.N, a.K, ldw, 128);
    if (rc != FQ_OK) return rc;
    const StripArgs q{a, p.nt, p.stages, p.splits, early};
    cudaLaunchAttribute attr[2]{};
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)p.splits; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)((a.N + 127) / 128 * p.splits), (unsigned)p.blocks); cfg.blockDim = dim3(kThreads); cfg.dynamicSmemBytes = p.smem;
    cfg.stream = st; cfg.attrs = attr; cfg.numAttrs = early ? 2 : 1;
    FQ_CUDA_OK(cudaLaunchKernelEx(&cfg, gemm_i8_strip_kernel<T>, map_x, map_w, q));
    return FQ_OK;
}

// Outputs per tile: the width for which the last wave leaves the least idle (the time of a wave goes with the width, plus
// something for a tile's ends).
int pair_tile_n(int M, int n_out, int pairs)
{
    const long long m_blocks = (M + 2 * kBM - 1) / (2 * kBM);
    int best = 256;
    long long least = -1;
    for (int w = 256; w >= 128; w -= 32) {
        const long long waves = (m_blocks * ((n_out + w - 1) / w) + pairs - 1) / pairs, cost = waves * (w + 16);
        if (least < 0 || cost < least) { best = w; least = cost; }
    }
    return best;
}

template <class T>
int launch_pair(const Ctx* ctx, const int8_t* xc, long long ldx, const int8_t* wc, long long ldw, I8Args a, cudaStream_t st)
{
    static std::atomic<int> pairs_on[64];                // pairs of SMs that can be resident together
    if (ctx->device >= 64) return FQ_ERR_ARG;
    int pairs = pairs_on[ctx->device].load(std::memory_order_acquire);
    if (!pairs) {
        FQ_CUDA_OK(cudaFuncSetAttribute(gemm_i8_pair_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, PairSmem::kTotal));
        cudaLaunchConfig_t probe{};
        probe.gridDim = dim3((unsigned)(ctx->sm_count / 2 * 2)); probe.blockDim = dim3(kThreads);
        probe.dynamicSmemBytes = PairSmem::kTotal;
        int n = 0;
        FQ_CUDA_OK(cudaOccupancyMaxActiveClusters(&n, gemm_i8_pair_kernel<T>, &probe));
        if (n < 1) return FQ_ERR_CUDA;
        pairs = n < ctx->sm_count / 2 ? n : ctx->sm_count / 2;
        pairs_on[ctx->device].store(pairs, std::memory_order_release);
    }
    a.tile_n = pair_tile_n(a.M, a.N, pairs);
    CUtensorMap map_x, map_w;
    int rc = make_map_i8(&map_x, xc, a.M, a.K, ldx, kBM);
    if (rc != FQ_OK) return rc;
    rc = make_map_i8(&map_w, wc, a.N, a.K, ldw, a.tile_n / 2);
    if (rc != FQ_OK) return rc;
    const long long tiles = (long long)((a.M + 2 * kBM - 1) / (2 * kBM)) * ((a.N + a.tile_n - 1) / a.tile_n);
    const int grid = 2 * (int)(tiles < pairs ? tiles : pairs);
    cudaLaunchAttribute overlap{};                       // set up while the kernel before it drains
    overlap.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    overlap.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)grid); cfg.blockDim = dim3(kThreads); cfg.dynamicSmemBytes = PairSmem::kTotal;
    cfg.stream = st; cfg.attrs = &overlap; cfg.numAttrs = 1;
    FQ_CUDA_OK(cudaLaunchKernelEx(&cfg, gemm_i8_pair_kernel<T>, map_x, map_w, a));
    return FQ_OK;
}

int check_weights(const fq_ctx* ctx, const int8_t* wc, const float* sw, int M, int n_out, int k_in, long long ldw, const void* y, int y_dtype,
                  long long ldy)
{
    const int size = type_size(y_dtype);
    if (!ctx || !wc || !sw || !y || !size) return FQ_ERR_ARG;
    if (M < 1 || M > (1 << 20) || n_out < 1 || n_out > (1 << 20) || k_in < 1 || k_in > 131071) return FQ_ERR_SHAPE;
    if (ldw < k_in || ldw % 16 || ldy < n_out || ldy * size % 16) return FQ_ERR_SHAPE;
    if (!aligned(wc, 16) || !aligned(sw, 4) || !aligned(y, 16)) return FQ_ERR_ALIGN;
    return FQ_OK;
}

int check_codes(const int8_t* xc, const float* sx, int k_in, long long ldx)
{
    if (!xc || !sx) return FQ_ERR_ARG;
    if (ldx < k_in || ldx % 16) return FQ_ERR_SHAPE;
    if (!aligned(xc, 16) || !aligned(sx, 4)) return FQ_ERR_ALIGN;
    return FQ_OK;
}

int launch_any(const Ctx* ctx, const int8_t* xc, long long ldx, const int8_t* wc, long long ldw, int y_dtype, const I8Args& a, bool early,
               cudaStream_t st)
{
    if (takes_strips(ctx, a.M, a.N)) {
        if (y_dtype == FQ_DT_F32) return launch_strip<float>(ctx, xc, ldx, wc, ldw, a, early, st);
        if (y_dtype == FQ_DT_F16) return launch_strip<__half>(ctx, xc, ldx, wc, ldw, a, early, st);
        return launch_strip<__nv_bfloat16>(ctx, xc, ldx, wc, ldw, a, early, st);
    }
    if (y_dtype == FQ_DT_F32) return launch_pair<float>(ctx, xc, ldx, wc, ldw, a, st);
    if (y_dtype == FQ_DT_F16) return launch_pair<__half>(ctx, xc, ldx, wc, ldw, a, st);
    return launch_pair<__nv_bfloat16>(ctx, xc, ldx, wc, ldw, a, st);
}

}  // namespace
}  // namespace fq

using namespace fq;

extern "C" {

int fq_gemm_i8(fq_ctx* ctx, const int8_t* x_codes_dev, const float* x_scales_dev, int M, long long ldx, const int8_t* w_codes_dev,
               const float* w_scales_dev, int n_out, int k_in, long long ldw, void* Y_dev, int y_dtype, long long ldy, void* stream)
{
    int rc = check_weights(ctx, w_codes_dev, w_scales_dev, M, n_out, k_in, ldw, Y_dev, y_dtype, ldy);
    if (rc == FQ_OK) rc = check_codes(x_codes_dev, x_scales_dev, k_in, ldx);
    if (rc != FQ_OK) return rc;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return FQ_ERR_CUDA;
    if (gemv_i8_takes(M, k_in))
        return launch_gemv_i8(ctx, x_codes_dev, -1, ldx, x_scales_dev, M, w_codes_dev, w_scales_dev, n_out, k_in, ldw, Y_dev, y_dtype, ldy, false,
                              (cudaStream_t)stream);
    const I8Args a{x_scales_dev, w_scales_dev, Y_dev, M, n_out, k_in, ldy, 0, ctx->status_dev};
    return launch_any(ctx, x_codes_dev, ldx, w_codes_dev, ldw, y_dtype, a, false, (cudaStream_t)stream);
}

int fq_linear_i8(fq_ctx* ctx, const void* X_dev, int x_dtype, int M, long long ldx, const int8_t* w_codes_dev, const float* w_scales_dev,
                 int n_out, int k_in, long long ldw, int8_t* codes_dev, long long ldc, float* scales_dev, void* Y_dev, int y_dtype,
                 long long ldy, void* stream)
{
    const int size = type_size(x_dtype);
    int rc = check_weights(ctx, w_codes_dev, w_scales_dev, M, n_out, k_in, ldw, Y_dev, y_dtype, ldy);
    if (rc == FQ_OK) rc = check_codes(codes_dev, scales_dev, k_in, ldc);
    if (rc != FQ_OK) return rc;
    if (!X_dev || !size) return FQ_ERR_ARG;
    if (ldx < k_in) return FQ_ERR_SHAPE;
    if (!aligned(X_dev, (size_t)size)) return FQ_ERR_ALIGN;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return FQ_ERR_CUDA;
    const cudaStream_t st = (cudaStream_t)stream;
    if (gemv_i8_takes(M, k_in) && gemv_i8_quantises(M, k_in))
        return launch_gemv_i8(ctx, X_dev, x_dtype, ldx, nullptr, M, w_codes_dev, w_scales_dev, n_out, k_in, ldw, Y_dev, y_dtype, ldy, false, st);
    rc = launch_quantize_rows(X_dev, x_dtype, M, k_in, ldx, codes_dev, ldc, scales_dev, ctx->sm_count, st);
    if (rc != FQ_OK) return rc;
    if (gemv_i8_takes(M, k_in))
        return launch_gemv_i8(ctx, codes_dev, -1, ldc, scales_dev, M, w_codes_dev, w_scales_dev, n_out, k_in, ldw, Y_dev, y_dtype, ldy, true, st);
    const I8Args a{scales_dev, w_scales_dev, Y_dev, M, n_out, k_in, ldy, 0, ctx->status_dev};
    return launch_any(ctx, codes_dev, ldc, w_codes_dev, ldw, y_dtype, a, true, st);
}

}  // extern "C"
