// Attention of a sequence's last tokens over its paged cache, many query rows to a key head (large trees, shared key heads, prompts): tensor cores.
//
// A CTA an SM.  A unit is NQ tiles of 128 query rows (TMEM lanes) against one key head's cells, KEYS at a time:
//   warps 0 .. 4 NQ - 1   softmax, a thread a row: scores from TMEM, weights back into the same columns, running maximum and sum in registers; values
//                         are rescaled only when a maximum has risen by more than a factor of 2^8 (rare behind a row's first tiles), so that nobody
//                         waits for the product in between
//   1 warp                says which unit is next, brings the query rows, looks through value tiles that not all rows see for infinities and NaNs, and clears
//                         what lies behind a sequence's last cell
//   2 warps               TMA, keys and values: runs of cells that lie together in a block (as many as divide both the block and the tile) into the 128-byte swizzled rows that the
//                         tensor core reads; a ring of key and value tiles that runs ahead over units
//   1 warp                issues tcgen05.mma: scores = Q K^T (both from shared memory), values += P V (P in TMEM, V as it lies, d contiguous)
// With two query tiles one's softmax runs beside the other's products; with one, scores have two buffers and the next tile's are formed ahead.
// What bounds it: for each key and row 4 head_dim flop, one exponential (16 a clock and SM) and some five other instructions of a lane; the
// products of a 128 x 128 tile of heads of 128 take 1024 cycles, its exponentials as long.  Keys and values come at 2850 cycles a tile where
// they are read once.
#include "fq_attention.cuh"

#include <atomic>
#include <numeric>

#include "fq_rowtypes.cuh"
#include "fq_umma.cuh"

namespace fq {
namespace {

template <int DP, int NQ>
struct TcShape {
    static constexpr int kRows = 128 * NQ;
    static constexpr int kKeys = DP == 256 ? 64 : 128;
    static constexpr int kBufs = NQ == 1 ? 2 : 1;                            // tiles of scores of a query tile: they share 512 columns with the values
    static constexpr int kSoftmax = 4 * NQ;                                  // warps
    static constexpr int kWarps = kSoftmax + 4;
    static constexpr int kThreads = kWarps * 32;
    static constexpr int kEnds = 512 / kKeys;                                // key tiles' time that a unit's ends take
    static constexpr int kQBytes = 128 * DP * 2;                             // of a query tile
    static constexpr int kSlotBytes = kKeys * DP * 2;
    static constexpr int kSlots = (224 * 1024 - NQ * kQBytes) / kSlotBytes < 10 ? (224 * 1024 - NQ * kQBytes) / kSlotBytes : 10;
    static constexpr int oRing = NQ * kQBytes;
    static constexpr int oBars = oRing + kSlots * kSlotBytes;
    // full[slots] empty[slots] raw[slots] q_full q_empty s_full[4] p_full[4] pv_done[2] unit_full[2] unit_empty[2]
    static constexpr int kBars = 3 * kSlots + 16;
    static constexpr int oSums = oBars + kBars * 8;
    // Units whose noted cells are kept: the warp that notes them is no more than two ahead of those that give them back.
    static constexpr int kOddUnits = 4;
    static constexpr int oMisc = oSums + (kWarps + 3) * 8;                   // TMEM address, abort flag, spoilt[kOddUnits]
    static constexpr int oUnits = (oMisc + 8 + kOddUnits * 4 + 15) / 16 * 16;             // Unit [2]
    static constexpr int oOdd = oUnits + 2 * 64;                             // bits [kOddUnits][kOddWords]
    static constexpr int kTotal = oOdd + kOddUnits * kOddWords * 4 + 1024;   // (tiles start at a multiple of 1024)
    static constexpr int kTmemS = 0;                                         // scores of the query tiles, then their values
    static constexpr int kTmemO = kBufs * NQ * kKeys;
    static_assert(kTmemO + NQ * DP <= 512, "TMEM columns");
    static_assert(kTotal <= 232448, "shared memory over the per-CTA limit");
};

// What the softmax warps and the one that issues products know of a unit.  One warp works it out ahead of time: between units that takes some 4000
// cycles, while the tensor core idled.  (Prompts of up to 2048: 128 us, 136 where each warp did it for itself; trees of 60 over 40000 cells 220 and 236.)
struct Unit {
    int there, whole;                            // 0: no more units
    int t0, t1, end[2];                          // key tiles of the part; up to where the rows of a query tile see any
    int b, tile, head;
    int row0, fresh, len, ctx;                   // of the sequence
    int pad[3];
};
static_assert(sizeof(Unit) == 64, "TcShape::oUnits");

__device__ __forceinline__ void to_async_proxy() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// 32 columns of this warp's lanes, a lane a thread; and 64 that have arrived only behind tmem_ld_wait, which names them so that nothing uses them before.
__device__ __forceinline__ void tmem_ld32(uint32_t addr, float (&v)[32])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {"
        "%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, "
        "%28, %29, %30, %31"
        "}, [%32];\n\ttcgen05.wait::ld.sync.aligned;"
        :
          "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]), "=f"(v[10]),
          "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]), "=f"(v[16]), "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]),
          "=f"(v[21]), "=f"(v[22]), "=f"(v[23]), "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]),
          "=f"(v[31])
        : "r"(addr) : "memory");
}
__device__ __forceinline__ void tmem_ld64(uint32_t addr, float (&v)[64])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x64.b32 {"
        "%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, "
        "%28, %29, %30, %31, %32, %33, %34, %35, %36, %37, %38, %39, %40, %41, %42, %43, %44, %45, %46, %47, %48, %49, %50, %51, %52, %53, "
        "%54, %55, %56, %57, %58, %59, %60, %61, %62, %63"
        "}, [%64];"
        :
          "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]), "=f"(v[10]),
          "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]), "=f"(v[16]), "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]),
          "=f"(v[21]), "=f"(v[22]), "=f"(v[23]), "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]),
          "=f"(v[31]), "=f"(v[32]), "=f"(v[33]), "=f"(v[34]), "=f"(v[35]), "=f"(v[36]), "=f"(v[37]), "=f"(v[38]), "=f"(v[39]), "=f"(v[40]),
          "=f"(v[41]), "=f"(v[42]), "=f"(v[43]), "=f"(v[44]), "=f"(v[45]), "=f"(v[46]), "=f"(v[47]), "=f"(v[48]), "=f"(v[49]), "=f"(v[50]),
          "=f"(v[51]), "=f"(v[52]), "=f"(v[53]), "=f"(v[54]), "=f"(v[55]), "=f"(v[56]), "=f"(v[57]), "=f"(v[58]), "=f"(v[59]), "=f"(v[60]),
          "=f"(v[61]), "=f"(v[62]), "=f"(v[63])
        : "r"(addr) : "memory");
}
__device__ __forceinline__ void tmem_ld_wait(float (&v)[64])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
        :
          "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]), "+f"(v[8]), "+f"(v[9]), "+f"(v[10]),
          "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15]), "+f"(v[16]), "+f"(v[17]), "+f"(v[18]), "+f"(v[19]), "+f"(v[20]),
          "+f"(v[21]), "+f"(v[22]), "+f"(v[23]), "+f"(v[24]), "+f"(v[25]), "+f"(v[26]), "+f"(v[27]), "+f"(v[28]), "+f"(v[29]), "+f"(v[30]),
          "+f"(v[31]), "+f"(v[32]), "+f"(v[33]), "+f"(v[34]), "+f"(v[35]), "+f"(v[36]), "+f"(v[37]), "+f"(v[38]), "+f"(v[39]), "+f"(v[40]),
          "+f"(v[41]), "+f"(v[42]), "+f"(v[43]), "+f"(v[44]), "+f"(v[45]), "+f"(v[46]), "+f"(v[47]), "+f"(v[48]), "+f"(v[49]), "+f"(v[50]),
          "+f"(v[51]), "+f"(v[52]), "+f"(v[53]), "+f"(v[54]), "+f"(v[55]), "+f"(v[56]), "+f"(v[57]), "+f"(v[58]), "+f"(v[59]), "+f"(v[60]),
          "+f"(v[61]), "+f"(v[62]), "+f"(v[63])
        :: "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t addr, const float (&v)[32])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {"
        "%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, "
        "%28, %29, %30, %31, %32"
        "};"
        :: "r"(addr),
           "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]), "f"(v[8]), "f"(v[9]), "f"(v[10]), "f"(v[11]),
           "f"(v[12]), "f"(v[13]), "f"(v[14]), "f"(v[15]), "f"(v[16]), "f"(v[17]), "f"(v[18]), "f"(v[19]), "f"(v[20]), "f"(v[21]), "f"(v[22]),
           "f"(v[23]), "f"(v[24]), "f"(v[25]), "f"(v[26]), "f"(v[27]), "f"(v[28]), "f"(v[29]), "f"(v[30]), "f"(v[31]) : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t addr, const uint32_t (&v)[32])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {"
        "%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, "
        "%28, %29, %30, %31, %32"
        "};"
        :: "r"(addr),
           "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]),
           "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]), "r"(v[20]), "r"(v[21]), "r"(v[22]),
           "r"(v[23]), "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]), "r"(v[29]), "r"(v[30]), "r"(v[31]) : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// D (+)= A * B, both in shared memory; or A in TMEM.
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)accumulate) : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                 ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"((uint32_t)accumulate) : "memory");
}
// fp16 or bf16 operands, fp32 sums, 128 x n outputs; B with its outputs contiguous (values) or its inner dimension (keys).
template <class T>
__device__ __forceinline__ uint32_t idesc_of(int n, bool b_outputs_contiguous)
{
    const uint32_t type = std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;
    return 1u << 4 | type << 7 | type << 10 | (b_outputs_contiguous ? 1u << 16 : 0u) | (uint32_t)(n >> 3) << 17 | 8u << 24;
}
// A tile of values as it lies: rows of cells, 64 values (128 bytes, swizzled) wide, eight cells 1024 bytes apart; the next 64 values `chunk` bytes further.
__device__ __forceinline__ uint64_t desc_values(uint32_t addr, uint32_t chunk)
{
    return umma_desc_sw128(addr) & ~((uint64_t)0x3fff << 16) | (uint64_t)(chunk >> 4) << 16;
}

// The largest absolute value of many, two at a time; a NaN stays.
template <class T> struct Pair;
template <> struct Pair<__nv_bfloat16> {
    using Type = __nv_bfloat162;
    static __device__ __forceinline__ Type zero() { return __float2bfloat162_rn(0.0f); }
    static __device__ __forceinline__ void take(Type& m, const uint4& v) { Group<__nv_bfloat16>::take_abs(m, v); }
    static __device__ __forceinline__ bool finite(Type m) { return finite16<__nv_bfloat16>(*reinterpret_cast<const uint32_t*>(&m)); }
};
template <> struct Pair<__half> {
    using Type = __half2;
    static __device__ __forceinline__ Type zero() { return __float2half2_rn(0.0f); }
    static __device__ __forceinline__ void take(Type& m, const uint4& v) { Group<__half>::take_abs(m, v); }
    static __device__ __forceinline__ bool finite(Type m) { return finite16<__half>(*reinterpret_cast<const uint32_t*>(&m)); }
};

__device__ __forceinline__ float max3(float a, float b, float c)
{
    float y;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
    return y;
}

// A place in the ring.
template <int SLOTS>
struct Place {
    int slot = 0;
    uint32_t phase = 0;
    __device__ __forceinline__ void next()
    {
        if (++slot == SLOTS) slot = 0, phase ^= 1;
    }
};

// Key tiles [t0, t1) of the part, of which the rows of query tile q see those below.
template <int NQ, int KEYS, class Work>
__device__ __forceinline__ int tiles_end(const AttnArgs& a, const Work& w, int q)
{
    if (w.s.fresh * a.share <= (w.tile * NQ + q) * 128) return w.t0();           // no rows
    return max(w.t0(), min(w.t1(), key_tiles<128, KEYS>(a, w.s, w.tile * NQ + q)));
}

// Cells lie in a cache as [block][key head][cell of the block][value], whatever their strides.
__device__ __forceinline__ void tma_cells(uint32_t dst, const CUtensorMap* map, int value, int cell, int head, int block, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
                 ::"r"(dst), "l"(map), "r"(value), "r"(cell), "r"(head), "r"(block), "r"(bar) : "memory");
}

//   run : cells of a TMA box;  q_map: query rows of [token][key head][head of its group][value], if rows_by_tma
template <class T, int DP, int NQ>
__global__ void __launch_bounds__(TcShape<DP, NQ>::kThreads, 1)
attention_tc_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map,
                    const __grid_constant__ CUtensorMap q_map, int run)
{
    using S = TcShape<DP, NQ>;
    using Work = Deal<S::kRows, S::kKeys, S::kEnds, S::kThreads>;
    constexpr int kUnits = DP / 8;               // 16-byte pieces of a row
    extern __shared__ char smem_raw[];
    char* smem = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
    const uint32_t base = smem_u32(smem), ring = base + S::oRing, bars = base + S::oBars;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const auto full = [&](int slot) { return bars + slot * 8; };
    const auto empty = [&](int slot) { return bars + (S::kSlots + slot) * 8; };
    const auto raw = [&](int slot) { return bars + (2 * S::kSlots + slot) * 8; };
    const uint32_t q_full = bars + 3 * S::kSlots * 8, q_empty = q_full + 8, s_full = q_full + 16, p_full = q_full + 48, pv_done = q_full + 80;
    const uint32_t unit_full = q_full + 96, unit_empty = q_full + 112;
    uint32_t* tmem_at = reinterpret_cast<uint32_t*>(smem + S::oMisc);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + S::oMisc + 4);
    volatile int* spoilt = reinterpret_cast<volatile int*>(smem + S::oMisc + 8);
    Unit* units = reinterpret_cast<Unit*>(smem + S::oUnits);
    const auto odd_cells = [&](int unit) { return reinterpret_cast<uint32_t*>(smem + S::oOdd) + unit % S::kOddUnits * kOddWords; };
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");              // (the joining kernel waits for this one's end)
    if (tid == 0) {
        AttnJoin none{};
        a.joins[blockIdx.x] = none;
        *abort_flag = 0;
        for (int i = 0; i < S::kOddUnits; i++) spoilt[i] = -1;
        for (int i = 0; i < S::kSlots; i++) {
            mbar_init(full(i), 1);
            mbar_init(empty(i), 1);
            mbar_init(raw(i), 1);
        }
        mbar_init(q_full, 1);
        mbar_init(q_empty, 1);
        for (int i = 0; i < 4; i++) {
            mbar_init(s_full + 8 * i, 1);
            mbar_init(p_full + 8 * i, 4);
        }
        for (int i = 0; i < 2; i++) {
            mbar_init(pv_done + 8 * i, 1);
            mbar_init(unit_full + 8 * i, 1);
            mbar_init(unit_empty + 8 * i, S::kSoftmax + 1);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == S::kWarps - 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(base + S::oMisc) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    Work w;
    const bool some = w.begin(a, reinterpret_cast<long long*>(smem + S::oSums));
    tc_before();
    __syncthreads();
    tc_after();
    const uint32_t tmem = *tmem_at;
    const auto gave_up = [&]() {
        atomicCAS(a.status, 0, FQ_ERR_TIMEOUT);
        *abort_flag = 1;
    };
    bool ok = true;                              // (of this warp: every wait has a limit)
    const auto wait = [&](uint32_t bar, uint32_t parity) {
        if (ok && !g_wait(bar, parity, abort_flag)) {
            gave_up();
            ok = false;
        }
        return ok = __all_sync(0xffffffffu, ok);
    };

    // The nth unit, for the softmax warps and the one that issues products.  Nobody is more than two units ahead of another.
    const auto take_unit = [&](int nth, Unit& u) {
        if (!wait(unit_full + 8 * (nth & 1), nth >> 1 & 1)) return false;
        u = units[nth & 1];
        __syncwarp();
        if (lane == 0) mbar_arrive(unit_empty + 8 * (nth & 1));
        return u.there != 0;
    };

    // With two query tiles a softmax thread holds 128 scores and needs more registers than the 168 that all got; the last four warps give theirs
    // up: 8 x 32 x 208 + 4 x 32 x 88 = 12 x 32 x 168.
    if constexpr (NQ == 2) {
        static_assert(S::kThreads == 384, "the split of registers");
        if (warp < S::kSoftmax) asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
        else asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    }

    if (some && warp < S::kSoftmax) {
        // ------------------------------------------------------------------------------------------------ softmax
        const int q = warp / 4, r = (warp & 3) * 32 + lane;                      // query tile, row of it
        const uint32_t lanes = tmem + ((uint32_t)(warp & 3) << 21);              // (32 lanes a warp, in the address's upper half)
        const uint32_t o_at = lanes + S::kTmemO + q * DP;
        unsigned n_tiles = 0;                                                    // of this query tile so far
        uint32_t o_turn = 0;
        int unit = 0;                                                            // (those that have key tiles)
        Unit u;
        for (int nth = 0; take_unit(nth, u); nth++) {
            Seq s;
            s.row0 = u.row0; s.fresh = u.fresh; s.len = u.len; s.ctx = u.ctx;
            const int n = u.tile * S::kRows + q * 128 + r, rows = s.fresh * a.share;
            const bool real = n < rows, idle = n - lane >= rows;                 // idle: the warp has no row at all
            const int t = min(n, rows - 1) / a.share, row = s.row0 + t;
            const int t0 = u.t0, t1 = q == 0 ? u.end[0] : u.end[1];
            // cells before this one are seen by all rows of the tile
            const int all_see = a.mask ? s.ctx : s.ctx + (u.tile * S::kRows + q * 128) / a.share + 1;
            float m = -INFINITY, l = 0.0f;                                       // m: of the raw scores
            for (int tile = t0; tile < t1; tile++, n_tiles++) {
                const uint32_t buf = S::kBufs == 2 ? n_tiles & 1 : (uint32_t)q, phase = (S::kBufs == 2 ? n_tiles >> 1 : n_tiles) & 1;
                if (!wait(s_full + 8 * buf, phase)) break;
                if (idle) {                      // (whatever stands for weights there: no row has anything from another)
                    if (S::kBufs == 2 && tile > t0 && !wait(pv_done + 8 * q, (n_tiles - 1) & 1)) break;
                    if (lane == 0) mbar_arrive(p_full + 8 * buf);
                    continue;
                }
                tc_after();
                const uint32_t s_at = lanes + S::kTmemS + buf * S::kKeys;
                const int cell0 = tile * S::kKeys;
                const bool partial = cell0 + S::kKeys > all_see;
                // 64 scores at a time: the next ones are on their way while the maximum of these is formed
                constexpr int kHalves = S::kKeys / 64;
                float v[kHalves][64];
                tmem_ld64(s_at, v[0]);
                float x[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int c = 0; c < kHalves; c++) {
                    tmem_ld_wait(v[c]);
                    if (c + 1 < kHalves) tmem_ld64(s_at + 64 * (c + 1), v[c + 1]);
                    if (partial) {
#pragma unroll
                        for (int b = 0; b < 64; b += 32) {
                            const uint32_t in = seen32(a, s, t, row, cell0 + 64 * c + b);
#pragma unroll
                            for (int j = 0; j < 32; j++) v[c][b + j] = in >> j & 1 ? v[c][b + j] : -INFINITY;
                        }
                    }
#pragma unroll
                    for (int j = 0; j < 64; j += 2) x[j / 2 & 3] = max3(x[j / 2 & 3], v[c][j], v[c][j + 1]);
                }
                const float top = max3(max3(x[0], x[1], x[2]), x[3], x[3]);
                // the maximum in use follows only when it is far behind
                const bool far = (top - m) * a.scale > 8.0f || (m == -INFINITY && top > -INFINITY);
                float rise = 1.0f;
                if (far) {
                    rise = exp2_fast((m - top) * a.scale);
                    m = top;
                    l *= rise;
                }
                const bool late = tile > t0 && __any_sync(0xffffffffu, far);
                if (late) {
                    if (S::kBufs == 2 && !wait(pv_done + 8 * q, (n_tiles - 1) & 1)) break;
                    tc_after();
#pragma unroll 1
                    for (int c = 0; c < DP; c += 32) {
                        float v[32];
                        tmem_ld32(o_at + c, v);
#pragma unroll
                        for (int j = 0; j < 32; j++) v[j] *= rise;
                        tmem_st32(o_at + c, v);
                    }
                }
                const float less = m == -INFINITY ? 0.0f : m * a.scale;
                const float2 by = make_float2(a.scale, a.scale), minus = make_float2(-less, -less);
                float2 sum[2] = {};
#pragma unroll
                for (int c = 0; c < kHalves; c++) {
                    uint32_t p[32];
#pragma unroll
                    for (int j = 0; j < 64; j += 2) {
                        const float2 e = fma2(make_float2(v[c][j], v[c][j + 1]), by, minus);
                        const float2 w2 = make_float2(exp2_fast(e.x), exp2_fast(e.y));
                        sum[j / 2 & 1] = add2(sum[j / 2 & 1], w2);
                        p[j / 2] = pack2<T>(w2.x, w2.y);                     // (the product takes 16-bit weights: half a step of each, as much as an output's own rounding)
                    }
                    tmem_st32(s_at + 32 * c, p); // (columns whose scores have been read)
                }
                l += (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
                tmem_st_wait();
                // (every product's end is waited for in its turn: a parity tells it from the one before it only.  With one buffer these scores were
                // issued behind that product, and what tells of them tells of it.)
                if (S::kBufs == 2 && tile > t0 && !late && !wait(pv_done + 8 * q, (n_tiles - 1) & 1)) break;
                tc_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(p_full + 8 * buf);
            }
            if (!ok) break;
            // ---- the part's end
            if (t1 > t0) {
                if (!wait(pv_done + 8 * q, S::kBufs == 2 ? (n_tiles - 1) & 1 : o_turn)) break;
                o_turn ^= 1;
                tc_after();
            }
            const bool whole = u.whole, odd = spoilt[unit % S::kOddUnits] == unit;
            const float by = whole ? (l == 0.0f ? 0.0f : 1.0f / l) : 1.0f;
            const int h = u.head * a.share + n % a.share;
            T* out = static_cast<T*>(a.out) + row * a.out_token + h * a.out_head;
            float* part = a.parts + (long long)(blockIdx.x * 2 + (t0 == 0)) * S::kRows * (DP + 2);
#pragma unroll 1
            for (int c = 0; c < (idle ? 0 : DP); c += 32) {
                float v[32];
                if (t1 > t0) {
                    tmem_ld32(o_at + c, v);
                } else {
#pragma unroll
                    for (int j = 0; j < 32; j++) v[j] = 0.0f;
                }
                if (real && whole) {
#pragma unroll
                    for (int j = 0; j < 32; j += 8)
                        if (c + j < a.head_dim)
                            *reinterpret_cast<uint4*>(out + c + j) = make_uint4(pack2<T>(v[j] * by, v[j + 1] * by), pack2<T>(v[j + 2] * by, v[j + 3] * by),
                                                                                pack2<T>(v[j + 4] * by, v[j + 5] * by), pack2<T>(v[j + 6] * by, v[j + 7] * by));
                } else if (real) {
#pragma unroll
                    for (int j = 0; j < 32; j += 4)
                        *reinterpret_cast<float4*>(part + ((c + j) / 4 * S::kRows + q * 128 + r) * 4) = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
                }
                __syncwarp();                    // (the next load is the whole warp's)
            }
            if (__any_sync(0xffffffffu, odd)) {
                const int first = a.mask ? s.ctx : s.ctx + u.tile * S::kRows / a.share + 1;          // (of the unit, not of its query tile)
                give_back<T>(a, s, u.b, u.head, t, real, first, odd_cells(unit), [&](int d, float x) {
                    if (whole) out[d] = (T)((float)out[d] + x);              // (cells that all rows see may have left an infinity there)
                    else part[(d / 4 * S::kRows + q * 128 + r) * 4 + d % 4] += x;
                });
            }
            const float top = m * a.scale;       // (-inf stays)
            if (!whole) {
                part[S::kRows * DP + q * 128 + r] = top;
                part[S::kRows * (DP + 1) + q * 128 + r] = l;
            } else if (real && a.lse) {
                a.lse[(long long)row * (a.kv_heads * a.share) + h] = l == 0.0f ? -INFINITY : (top + log2f(l)) * 0.69314718055994531f;
            }
            if (u.t1 > t0) unit++;
            tc_before();
        }
    } else if (some && warp == S::kSoftmax) {
        // ------------------------------------------------------------------------------------------------ queries, values that not all see
        const int pieces = a.head_dim / 8;
        int pos = 0, unit = 0;                   // tiles of the ring so far
        uint32_t raw_phase = 0;                  // a bit a slot
        int nth = 0;
        for (bool more = true; ok; more = w.next(a)) {
            if (more && !w.any()) continue;
            if (!wait(unit_empty + 8 * (nth & 1), (nth >> 1 & 1) ^ 1)) break;
            const int t0 = w.t0(), t1 = w.t1();
            if (lane == 0) {
                Unit u{};
                u.there = more;
                if (more) {
                    u.whole = w.whole();
                    u.t0 = t0; u.t1 = t1;
#pragma unroll
                    for (int q = 0; q < NQ; q++) u.end[q] = tiles_end<NQ, S::kKeys>(a, w, q);
                    u.b = w.b; u.tile = w.tile; u.head = w.head;
                    u.row0 = w.s.row0; u.fresh = w.s.fresh; u.len = w.s.len; u.ctx = w.s.ctx;
                }
                units[nth & 1] = u;
                mbar_arrive(unit_full + 8 * (nth & 1));
                if (more && !u.whole && t0 == 0)
                    a.joins[blockIdx.x] = AttnJoin{w.s.row0, w.tile * S::kRows, w.head, w.others(), min(w.s.fresh * a.share - w.tile * S::kRows, S::kRows),
                                                   (int)blockIdx.x * 2 + 1, {0, 0}};
            }
            __syncwarp();
            if (!more) break;
            nth++;
            if (t1 <= t0) continue;
            // once the unit before has formed its last scores
            if (!wait(q_empty, (unit & 1) ^ 1)) break;
            if (a.rows_by_tma) {
                if (lane == 0) mbar_expect_tx(q_full, NQ * S::kQBytes);
                __syncwarp();
                const int token = w.s.row0 + w.tile * (S::kRows / a.share);      // (rows of other sequences, or none, behind the last token: nobody uses them)
                if (elect_one()) {
#pragma unroll
                    for (int q = 0; q < NQ; q++)
#pragma unroll
                        for (int d = 0; d < DP / 64; d++)
                            tma_cells(base + q * S::kQBytes + d * (128 * 128), &q_map, d * 64, 0, w.head, token + q * (128 / a.share), q_full);
                }
                __syncwarp();
            } else {
#pragma unroll 1
                for (int r0 = 0; r0 < S::kRows; r0 += 32) {
                    const int rn = w.tile * S::kRows + r0 + lane, tok = rn / a.share;
                    const long long mine = tok < w.s.fresh ? (long long)(w.s.row0 + tok) * a.q_token + (w.head * a.share + rn - tok * a.share) * a.q_head : -1;
#pragma unroll 8
                    for (int i = 0; i < kUnits; i++) {
                        const int n = i * 32 + lane, r = n / kUnits, u = n % kUnits, rr = r0 + r;
                        const long long from = __shfl_sync(0xffffffffu, mine, r);
                        const bool there = from >= 0 && u < pieces;
                        copy16(base + (rr >> 7) * S::kQBytes + (u >> 3) * (128 * 128) + (rr & 127) * 128 + ((u ^ rr) & 7) * 16,
                               static_cast<const T*>(a.q) + (there ? from + u * 8 : 0), there);
                    }
                }
                copies_commit();
                copies_wait<0>();
                to_async_proxy();
                __syncwarp();
                if (lane == 0) mbar_arrive(q_full);
            }
            const int all_see = a.mask ? w.s.ctx : w.s.ctx + w.tile * S::kRows / a.share + 1;
            odd_cells(unit)[lane] = 0;
            __syncwarp();
            for (int tile = max(t0, all_see / S::kKeys); tile < t1; tile++) {
                const int slot = (pos + 2 * (tile - t0) + 1) % S::kSlots;
                if (!wait(raw(slot), raw_phase >> slot & 1)) break;
                raw_phase ^= 1u << slot;
                const auto piece = [&](int r, int u) { return ring + slot * S::kSlotBytes + (u >> 3) * (S::kKeys * 128) + r * 128 + ((u ^ r) & 7) * 16; };
                // Cells that all rows see need no look.  Those behind the sequence's last one are nobody's, whatever lies there; behind its last box zeros were read.
                const int from = max(0, all_see - tile * S::kKeys), there = min(S::kKeys, w.s.len - tile * S::kKeys);
                const int read = min(S::kKeys, (w.s.len + run - 1) / run * run - tile * S::kKeys);
                for (int n = there * kUnits + lane; n < read * kUnits; n += 32) sts128(piece(n / kUnits, n % kUnits), make_uint4(0, 0, 0, 0));
                bool odd = false;
                for (int r0 = from; r0 < there; r0 += 8 * 32 / kUnits) {
                    uint4 v[8];
                    typename Pair<T>::Type most = Pair<T>::zero();
#pragma unroll
                    for (int i = 0; i < 8; i++) {
                        const int n = i * 32 + lane;
                        v[i] = lds128(piece(min(r0 + n / kUnits, there - 1), n % kUnits));
                    }
#pragma unroll
                    for (int i = 0; i < 8; i++) Pair<T>::take(most, v[i]);
                    if (__all_sync(0xffffffffu, Pair<T>::finite(most))) continue;
                    odd = true;
#pragma unroll 1
                    for (int i = 0; i < 8; i++) {
                        const int n = i * 32 + lane, r = min(r0 + n / kUnits, there - 1);
                        const uint32_t at = piece(r, n % kUnits);
                        uint4 y = lds128(at);
                        const bool mine = take_out<T>(y);
                        if (mine) sts128(at, y);
                        note_odd<kUnits>(odd_cells(unit), mine, tile * S::kKeys + r - all_see);
                    }
                }
                if (odd) spoilt[unit % S::kOddUnits] = unit;
                to_async_proxy();
                __syncwarp();
                if (lane == 0) mbar_arrive(full(slot));
            }
            pos = (pos + 2 * (t1 - t0)) % (2 * S::kSlots);
            unit++;
        }
    } else if (some && warp < S::kSoftmax + 3) {
        // ------------------------------------------------------------------------------------------------ fetching
        const bool values = warp == S::kSoftmax + 2;
        const CUtensorMap* map = values ? &v_map : &k_map;
        Place<S::kSlots> at;                     // keys and values take slots in turn
        if (values) at.next();
        const int boxes = S::kKeys / run;
        for (bool more = true; more && ok; more = w.next(a)) {
            const int t0 = w.t0(), t1 = w.t1();
            if (t1 <= t0) continue;
            const int all_see = a.mask ? w.s.ctx : w.s.ctx + w.tile * S::kRows / a.share + 1;
            // a block behind the cache reads as zeros: for cells that are not there, and numbers that cannot be
            const auto entry = [&](int cell) { return cell < w.s.len ? a.table[w.b * a.ld + cell / a.block_size] : a.blocks; };
            const auto block_of = [&](int block, int cell) {                     // (looked at only when it is needed: the load is on its way until then)
                const bool good = (unsigned)block < (unsigned)a.blocks;
                if (!good && cell < w.s.len) atomicCAS(a.status, 0, FQ_ERR_INDEX);
                return good ? block : a.blocks;
            };
            const auto looked_up = [&](int cell) { return block_of(entry(cell), cell); };
            int ahead = lane < boxes ? entry(t0 * S::kKeys + lane * run) : a.blocks;
            for (int tile = t0; tile < t1; tile++) {
                const int now = block_of(ahead, lane < boxes ? tile * S::kKeys + lane * run : w.s.len);
                if (tile + 1 < t1 && lane < boxes) ahead = entry((tile + 1) * S::kKeys + lane * run);            // (on its way meanwhile)
                if (!wait(empty(at.slot), at.phase ^ 1)) break;
                const bool look = values && (tile + 1) * S::kKeys > all_see;
                int in_block = tile * S::kKeys % a.block_size;
                const uint32_t to = ring + at.slot * S::kSlotBytes, bar = look ? raw(at.slot) : full(at.slot);
                if (lane == 0) mbar_expect_tx(bar, S::kSlotBytes);
                __syncwarp();
                // (block numbers first, then one lane issues eight boxes without a pause)
                for (int i0 = 0; i0 < boxes; i0 += 8) {
                    int in[8], cell[8];
#pragma unroll
                    for (int i = 0; i < 8; i++) {
                        in[i] = i0 < 32 ? __shfl_sync(0xffffffffu, now, i0 + i) : i0 + i < boxes ? looked_up(tile * S::kKeys + (i0 + i) * run) : 0;
                        cell[i] = in_block;
                        in_block += run;
                        if (in_block >= a.block_size) in_block = 0;
                    }
                    if (elect_one()) {
#pragma unroll
                        for (int i = 0; i < 8; i++)
                            if (i0 + i < boxes)
#pragma unroll
                                for (int d = 0; d < DP / 64; d++)
                                    tma_cells(to + d * (S::kKeys * 128) + (i0 + i) * run * 128, map, d * 64, cell[i], w.head, in[i], bar);
                    }
                }
                __syncwarp();
                at.next();
                at.next();
            }
        }
    } else if (some) {
        // ------------------------------------------------------------------------------------------------ products
        const uint32_t id_s = idesc_of<T>(S::kKeys, false), id_o = idesc_of<T>(DP, true);
        Place<S::kSlots> k_at, v_at;
        v_at.next();
        unsigned n_tiles[2] = {0, 0};
        int unit = 0;
        // (All that follows one wait is issued by one lane in one go: entering and leaving such a stretch takes some 300 cycles, whatever it issues.)
        const auto scores = [&](int q, uint32_t buf) {
            const uint32_t k_tile = ring + k_at.slot * S::kSlotBytes, q_tile = base + q * S::kQBytes;
#pragma unroll
            for (int k = 0; k < DP / 16; k++) {
                const uint32_t in = (k & 3) * 32;                                // bytes within a 128-byte row
                mma_ss(tmem + S::kTmemS + buf * S::kKeys, umma_desc_sw128(q_tile + (k >> 2) * (128 * 128) + in),
                       umma_desc_sw128(k_tile + (k >> 2) * (S::kKeys * 128) + in), id_s, k > 0);
            }
            umma_commit(s_full + 8 * buf);
        };
        const auto values = [&](int q, uint32_t buf, bool accumulate, bool last) {
            const uint32_t v_tile = ring + v_at.slot * S::kSlotBytes;
#pragma unroll
            for (int k = 0; k < S::kKeys / 16; k++)
                mma_ts(tmem + S::kTmemO + q * DP, tmem + S::kTmemS + buf * S::kKeys + k * 8, desc_values(v_tile + k * 2048, S::kKeys * 128), id_o,
                       accumulate || k > 0);
            if (S::kBufs == 2 || last) umma_commit(pv_done + 8 * q);
        };
        const auto buffer = [](int q, unsigned n) { return S::kBufs == 2 ? n & 1 : (uint32_t)q; };
        const auto two_on = [](Place<S::kSlots>& p) { p.next(); p.next(); };
        Unit u;
        for (int nth = 0; take_unit(nth, u); nth++) {
            const int t0 = u.t0, t1 = u.t1;
            if (t1 <= t0) continue;
            const int end[2] = {u.end[0], u.end[1]};
            if (!wait(full(k_at.slot), k_at.phase) || !wait(q_full, unit & 1)) break;
            tc_after();
            if (elect_one()) {
#pragma unroll
                for (int q = 0; q < NQ; q++)
                    if (end[q] > t0) scores(q, buffer(q, n_tiles[q]));
                umma_commit(empty(k_at.slot));
                if (t1 - t0 == 1) umma_commit(q_empty);
            }
            __syncwarp();
            two_on(k_at);
            for (int tile = t0; tile < t1 && ok; tile++) {
                const bool ahead = tile + 1 < t1;
                if (ahead && !wait(full(k_at.slot), k_at.phase)) break;
                if constexpr (S::kBufs == 2) {
                    if (ahead) {                 // the next scores, into the buffer whose weights have had their product issued
                        tc_after();
                        if (elect_one()) {
                            scores(0, buffer(0, n_tiles[0] + 1));
                            umma_commit(empty(k_at.slot));
                            if (tile + 2 == t1) umma_commit(q_empty);
                        }
                        __syncwarp();
                    }
                }
                if (!wait(full(v_at.slot), v_at.phase)) break;
#pragma unroll
                for (int q = 0; q < NQ; q++) {
                    const bool mine = tile < end[q], last = q == NQ - 1;
                    const uint32_t buf = buffer(q, n_tiles[q]), phase = (S::kBufs == 2 ? n_tiles[q] >> 1 : n_tiles[q]) & 1;
                    if (mine && !wait(p_full + 8 * buf, phase)) break;
                    tc_after();
                    if (elect_one()) {
                        if (mine) values(q, buf, tile > t0, tile + 1 == end[q]);
                        if (S::kBufs == 1 && tile + 1 < end[q]) scores(q, buf);  // (behind the product that reads the weights there)
                        if (last) {
                            umma_commit(empty(v_at.slot));
                            if (S::kBufs == 1 && ahead) {
                                umma_commit(empty(k_at.slot));
                                if (tile + 2 == t1) umma_commit(q_empty);
                            }
                        }
                    }
                    __syncwarp();
                    n_tiles[q] += mine;
                }
                two_on(v_at);
                if (ahead) two_on(k_at);
            }
            unit++;
        }
    }
    if (!ok) let_copies_land();
    tc_before();
    __syncthreads();
    tc_after();
    if (warp == S::kWarps - 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
}

// Keys or values as a tensor of [block][key head][cell][value]; box: 64 values (a swizzle span) of `run` cells.  Bits are only copied: any 16-bit type
// serves.  What lies beyond head_dim, or beyond the last block, reads as zeros.
int cells_map(CUtensorMap* map, const void* base, const AttnArgs& a, int run)
{
    PFN_cuTensorMapEncodeTiled_v12000 enc = tensor_map_encoder();
    if (!enc) return FQ_ERR_CUDA;
    const cuuint64_t dims[4] = {(cuuint64_t)a.head_dim, (cuuint64_t)a.block_size, (cuuint64_t)a.kv_heads, (cuuint64_t)a.blocks};
    const auto stride = [&](long long s) { return (cuuint64_t)(s > 0 ? s * 2 : (a.head_dim * 2 + 15) / 16 * 16); };      // (0: there is one of them)
    const cuuint64_t strides[3] = {stride(a.cell_stride), stride(a.head_stride), stride(a.block_stride)};
    const cuuint32_t box[4] = {64u, (cuuint32_t)run, 1u, 1u}, one[4] = {1, 1, 1, 1};
    const CUresult r = enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT16, 4, const_cast<void*>(base), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                           CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? FQ_OK : FQ_ERR_CUDA;
}

int rows_map(CUtensorMap* map, const AttnArgs& a)
{
    PFN_cuTensorMapEncodeTiled_v12000 enc = tensor_map_encoder();
    if (!enc) return FQ_ERR_CUDA;
    const cuuint64_t dims[4] = {(cuuint64_t)a.head_dim, (cuuint64_t)a.share, (cuuint64_t)a.kv_heads, (cuuint64_t)a.tokens};
    const auto stride = [&](long long s) { return (cuuint64_t)(s > 0 ? s * 2 : (a.head_dim * 2 + 15) / 16 * 16); };      // (0: there is one of them)
    const cuuint64_t strides[3] = {stride(a.q_head), stride(a.q_head * a.share), stride(a.q_token)};
    const cuuint32_t box[4] = {64u, (cuuint32_t)a.share, 1u, (cuuint32_t)(128 / a.share)}, one[4] = {1, 1, 1, 1};
    const CUresult r = enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT16, 4, const_cast<void*>(a.q), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                           CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? FQ_OK : FQ_ERR_CUDA;
}

template <class T, int DP, int NQ>
int launch(const fq_ctx* ctx, const AttnArgs& a, cudaStream_t st)
{
    using S = TcShape<DP, NQ>;
    static std::atomic<bool> ready[64];
    if (ctx->device >= 64) return FQ_ERR_ARG;
    if (!ready[ctx->device].load(std::memory_order_acquire)) {
        if (cudaFuncSetAttribute(attention_tc_kernel<T, DP, NQ>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kTotal) != cudaSuccess) return FQ_ERR_CUDA;
        ready[ctx->device].store(true, std::memory_order_release);
    }
    const int run = std::gcd(a.block_size, S::kKeys);
    CUtensorMap k_map, v_map, q_map{};
    if (a.rows_by_tma && rows_map(&q_map, a) != FQ_OK) return FQ_ERR_CUDA;
    if (cells_map(&k_map, a.k, a, run) != FQ_OK || cells_map(&v_map, a.v, a, run) != FQ_OK) return FQ_ERR_CUDA;
    attention_tc_kernel<T, DP, NQ><<<ctx->sm_count, S::kThreads, S::kTotal, st>>>(a, k_map, v_map, q_map, run);
    return cudaGetLastError() == cudaSuccess ? FQ_OK : FQ_ERR_CUDA;
}

template <class T>
int launch_typed(const fq_ctx* ctx, const AttnArgs& a, int rows, int dp, cudaStream_t st)
{
    if (dp == 64) return rows > 128 ? launch<T, 64, 2>(ctx, a, st) : launch<T, 64, 1>(ctx, a, st);
    if (dp == 128) return rows > 128 ? launch<T, 128, 2>(ctx, a, st) : launch<T, 128, 1>(ctx, a, st);
    return launch<T, 256, 1>(ctx, a, st);
}

}  // namespace

int launch_attention_tc(const fq_ctx* ctx, const AttnArgs& a, int dtype, int rows, int dp, cudaStream_t st)
{
    return dtype == FQ_DT_F16 ? launch_typed<__half>(ctx, a, rows, dp, st) : launch_typed<__nv_bfloat16>(ctx, a, rows, dp, st);
}

}  // namespace fq
