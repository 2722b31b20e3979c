// Attention of a sequence's last tokens over its paged cache, up to 16 query rows a tile (single tokens, small trees): bound by reading keys and values.
//
// One CTA an SM, every warp by itself: a tile of keys is 16 cells for each warp, fetched by its own asynchronous copies into its own ring (192 KB an SM, of
// which two thirds are on their way), so that no warp waits for another until the unit's end.  The online softmax is kept per warp;
// at the end the warps' maxima, sums and values are joined through shared memory.  Scores and values are formed by mma.m16n8k16: at 16 rows the bytes of
// a key take ten times as long to arrive as its products take.
#include "fq_attention.cuh"

#include <atomic>
#include <cmath>

#include "fq_rowtypes.cuh"

namespace fq {
namespace {

constexpr int kRows = 16;
constexpr int kChunk = 16;                       // cells of a warp's share of a key tile

template <int DP>
struct Shape {                                   // DP: head_dim, rounded up to 64, 128 or 256
    static constexpr int kWarps = DP == 256 ? 4 : 8;
    static constexpr int kThreads = kWarps * 32;
    static constexpr int kKeys = kWarps * kChunk;
    static constexpr int kStageBytes = 2 * kChunk * DP * 2;                  // of a warp: keys, then values
    static constexpr int kStages = 196608 / (kWarps * kStageBytes);
    static constexpr int kSets = kWarps / 2;                                 // sets of values that meet at a unit's end
    static constexpr int oSets = kWarps * kStages * kStageBytes;
    static constexpr int oMl = oSets + kSets * kRows * DP * 4;       // float2 [warps][rows]
    static constexpr int oSums = oMl + kWarps * kRows * 8;                   // long long [warps + 4]
    static constexpr int oSpoilt = oSums + (kWarps + 4) * 8;
    static constexpr int kTotal = oSpoilt + 16;
    static_assert(kTotal <= 232448, "shared memory over the per-CTA limit");
};

__device__ __forceinline__ void ldm4(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldm4t(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
template <class T>
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    if constexpr (std::is_same<T, __half>::value)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <class T, int DP>
__global__ void __launch_bounds__(Shape<DP>::kThreads, 1) attention_kernel(const __grid_constant__ AttnArgs a)
{
    using S = Shape<DP>;
    using Work = Deal<kRows, S::kKeys, 3, S::kThreads>;
    constexpr int kUnits = DP / 8;               // 16-byte pieces of a row
    constexpr int kSteps = DP / 16;
    extern __shared__ __align__(1024) char smem[];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, c = lane & 3;
    const uint32_t ring = smem_u32(smem) + warp * S::kStages * S::kStageBytes;
    float* sets = reinterpret_cast<float*>(smem + S::oSets);
    float2* ml = reinterpret_cast<float2*>(smem + S::oMl);
    volatile int* spoilt = reinterpret_cast<volatile int*>(smem + S::oSpoilt);
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");              // (the joining kernel waits for this one's end)
    if (tid == 0) {
        AttnJoin none{};
        a.joins[blockIdx.x] = none;
        spoilt[0] = spoilt[1] = 0;
    }
    Work w;
    if (!w.begin(a, reinterpret_cast<long long*>(smem + S::oSums))) return;
    const int pieces = a.head_dim / 8;

    // ---- fetching runs ahead of computing, over the ends of units
    Work f = w;
    int f_tile = f.t0(), f_stage = 0, f_block = -1;
    bool f_more = true;
    const auto settle = [&]() {                  // f at a unit with key tiles, and its next tile's block on the way
        while (f_more && f_tile >= f.t1()) {
            f_more = f.next(a);
            f_tile = f_more ? f.t0() : 0;
        }
        f_block = -1;
        if (f_more) {
            const int cell = f_tile * S::kKeys + warp * kChunk + (lane & 15);
            if (cell < f.s.len) f_block = a.table[f.b * a.ld + cell / a.block_size];
        }
    };
    const auto fetch = [&]() {
        if (f_more) {
            const int cell = f_tile * S::kKeys + warp * kChunk + (lane & 15);
            long long place = -1;
            if (cell < f.s.len) {
                if ((unsigned)f_block < (unsigned)a.blocks) place = f_block * a.block_stride + cell % a.block_size * a.cell_stride + f.head * a.head_stride;
                else if (lane < 16) atomicCAS(a.status, 0, FQ_ERR_INDEX);
            }
            const uint32_t to = ring + f_stage * S::kStageBytes;
#pragma unroll
            for (int i = 0; i < kChunk * kUnits / 32; i++) {
                const int n = i * 32 + lane, row = n / kUnits, unit = n % kUnits;
                const long long at = __shfl_sync(0xffffffffu, place, row);
                const bool there = at >= 0 && unit < pieces;
                const long long from = there ? at + unit * 8 : 0;
                const uint32_t dst = to + (uint32_t)(row * kUnits + (unit ^ (row & 7))) * 16;
                copy16(dst, static_cast<const T*>(a.k) + from, there);
                copy16(dst + kChunk * DP * 2, static_cast<const T*>(a.v) + from, there);
            }
            f_tile++;
            settle();
        }
        f_stage = f_stage + 1 == S::kStages ? 0 : f_stage + 1;
        copies_commit();
    };
    settle();
#pragma unroll 1
    for (int i = 0; i < S::kStages - 1; i++) fetch();

    int stage = 0, turn = 0;
    for (bool more = true; more; more = w.next(a)) {
        if (!w.any()) continue;
        const int rows = w.s.fresh * a.share - w.tile * kRows;                   // of the unit, from this tile on
        int t[2], row[2];                                                        // this lane's two rows: new token, row of the batch
#pragma unroll
        for (int h = 0; h < 2; h++) {
            t[h] = min(w.tile * kRows + g + 8 * h, w.s.fresh * a.share - 1) / a.share;
            row[h] = w.s.row0 + t[h];
        }
        uint32_t qf[kSteps][4];
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const int r = min(w.tile * kRows + g + 8 * h, w.s.fresh * a.share - 1);
            const T* q = static_cast<const T*>(a.q) + row[h] * a.q_token + (w.head * a.share + r % a.share) * a.q_head;
#pragma unroll
            for (int k = 0; k < kSteps; k++)
#pragma unroll
                for (int e = 0; e < 2; e++) {
                    const int d = k * 16 + e * 8 + 2 * c;
                    qf[k][h + 2 * e] = d < a.head_dim ? *reinterpret_cast<const uint32_t*>(q + d) : 0u;
                }
        }
        float o[DP / 8][4];
#pragma unroll
        for (int n = 0; n < DP / 8; n++)
#pragma unroll
            for (int i = 0; i < 4; i++) o[n][i] = 0.0f;
        float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.0f, 0.0f};
        // cells before this one are seen by all rows of the tile
        const int all_see = a.mask ? w.s.ctx : w.s.ctx + w.tile * kRows / a.share + 1;
        const int t1 = w.t1();
        for (int tile = w.t0(); tile < t1; tile++) {
            copies_wait<S::kStages - 2>();
            __syncwarp();
            fetch();
            const uint32_t ks = ring + stage * S::kStageBytes, vs = ks + kChunk * DP * 2;
            stage = stage + 1 == S::kStages ? 0 : stage + 1;
            const int cell0 = tile * S::kKeys + warp * kChunk;
            if (cell0 >= w.s.len) continue;
            float sc[2][4];
#pragma unroll
            for (int n = 0; n < 2; n++)
#pragma unroll
                for (int i = 0; i < 4; i++) sc[n][i] = 0.0f;
            const int krow = (lane >> 4) * 8 + (lane & 7), kunit = (lane >> 3) & 1;
#pragma unroll
            for (int k = 0; k < kSteps; k++) {
                uint32_t b[4];
                ldm4(b, ks + (uint32_t)(krow * kUnits + ((k * 2 + kunit) ^ (krow & 7))) * 16);
                mma16816<T>(sc[0], qf[k], b[0], b[1]);
                mma16816<T>(sc[1], qf[k], b[2], b[3]);
            }
#pragma unroll
            for (int n = 0; n < 2; n++)
#pragma unroll
                for (int i = 0; i < 4; i++) sc[n][i] *= a.scale;
            if (cell0 + kChunk > all_see) {
#pragma unroll
                for (int n = 0; n < 2; n++)
#pragma unroll
                    for (int i = 0; i < 4; i++)
                        if (!sees(a, w.s, t[i >> 1], row[i >> 1], cell0 + n * 8 + 2 * c + (i & 1))) sc[n][i] = -INFINITY;
                // values that not all rows see: none may be infinite or NaN in the product
                bool odd = false;
#pragma unroll
                for (int i = 0; i < kChunk * kUnits / 32; i++) {
                    const uint32_t at = vs + (uint32_t)(i * 32 + lane) * 16;
                    const uint4 v = lds128(at);
                    if (finite16<T>(v.x) && finite16<T>(v.y) && finite16<T>(v.z) && finite16<T>(v.w)) continue;
                    odd = true;
                    const uint32_t in[4] = {v.x, v.y, v.z, v.w};
                    uint32_t out[4];
#pragma unroll
                    for (int j = 0; j < 4; j++) out[j] = (finite16<T>(in[j] & 0xffffu) ? in[j] & 0xffffu : 0u) | (finite16<T>(in[j] & 0xffff0000u) ? in[j] & 0xffff0000u : 0u);
                    sts128(at, make_uint4(out[0], out[1], out[2], out[3]));
                }
                if (odd) spoilt[turn] = 1;
                __syncwarp();
            }
            // online softmax: a row is four lanes'
            float p[2][4], rise[2];
#pragma unroll
            for (int h = 0; h < 2; h++) {
                float top = fmaxf(fmaxf(sc[0][2 * h], sc[0][2 * h + 1]), fmaxf(sc[1][2 * h], sc[1][2 * h + 1]));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                top = fmaxf(top, m[h]);
                const float base = top == -INFINITY ? 0.0f : top;
                rise[h] = exp2_fast(m[h] - base);
                m[h] = top;
#pragma unroll
                for (int n = 0; n < 2; n++)
#pragma unroll
                    for (int e = 0; e < 2; e++) p[n][2 * h + e] = exp2_fast(sc[n][2 * h + e] - base);
                l[h] = l[h] * rise[h] + ((p[0][2 * h] + p[0][2 * h + 1]) + (p[1][2 * h] + p[1][2 * h + 1]));
            }
            const uint32_t pf[4] = {pack2<T>(p[0][0], p[0][1]), pack2<T>(p[0][2], p[0][3]), pack2<T>(p[1][0], p[1][1]), pack2<T>(p[1][2], p[1][3])};
            const int vrow = ((lane >> 3) & 1) * 8 + (lane & 7), vunit = lane >> 4;
            const bool risen = rise[0] != 1.0f || rise[1] != 1.0f;
            if (__any_sync(0xffffffffu, risen)) {
#pragma unroll
                for (int n = 0; n < DP / 8; n++) {
                    o[n][0] *= rise[0]; o[n][1] *= rise[0];
                    o[n][2] *= rise[1]; o[n][3] *= rise[1];
                }
            }
#pragma unroll
            for (int n = 0; n < DP / 16; n++) {
                uint32_t b[4];
                ldm4t(b, vs + (uint32_t)(vrow * kUnits + ((n * 2 + vunit) ^ (vrow & 7))) * 16);
                mma16816<T>(o[2 * n], pf, b[0], b[1]);
                mma16816<T>(o[2 * n + 1], pf, b[2], b[3]);
            }
        }
        // ---- the warps' parts are joined
#pragma unroll
        for (int h = 0; h < 2; h++) {
            l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
            l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
            if (c == 0) ml[warp * kRows + g + 8 * h] = make_float2(m[h], l[h]);
        }
        __syncthreads();
#pragma unroll
        for (int h = 0; h < 2; h++) {
            float top = -INFINITY;
#pragma unroll
            for (int i = 0; i < S::kWarps; i++) top = fmaxf(top, ml[i * kRows + g + 8 * h].x);
            const float by = exp2_fast(m[h] - (top == -INFINITY ? 0.0f : top));
#pragma unroll
            for (int n = 0; n < DP / 8; n++) { o[n][2 * h] *= by; o[n][2 * h + 1] *= by; }
        }
        // (eight values of a row move within it by the row's number, so that the four rows of a half-warp's access lie in different banks)
        float* mine = sets + ((warp % S::kSets) * kRows + g) * DP + 2 * c;
        if (warp < S::kSets) {
#pragma unroll
            for (int n = 0; n < DP / 8; n++) {
                *reinterpret_cast<float2*>(mine + (n ^ (g & 3)) * 8) = make_float2(o[n][0], o[n][1]);
                *reinterpret_cast<float2*>(mine + 8 * DP + (n ^ (g & 3)) * 8) = make_float2(o[n][2], o[n][3]);
            }
        }
        __syncthreads();
        if (warp >= S::kSets) {
#pragma unroll
            for (int n = 0; n < DP / 8; n++) {
                float2* x = reinterpret_cast<float2*>(mine + (n ^ (g & 3)) * 8);
                float2* y = reinterpret_cast<float2*>(mine + 8 * DP + (n ^ (g & 3)) * 8);
                *x = make_float2(x->x + o[n][0], x->y + o[n][1]);
                *y = make_float2(y->x + o[n][2], y->y + o[n][3]);
            }
        }
        __syncthreads();
        const bool whole = w.whole(), odd = spoilt[turn];
        const int k0 = w.t0() * S::kKeys, k1 = t1 * S::kKeys;
        float* part = a.parts + (long long)(blockIdx.x * 2 + (w.t0() == 0)) * kRows * (DP + 2);
        for (int i = tid; i < kRows * kUnits; i += S::kThreads) {
            const int r = i / kUnits, d = i % kUnits * 8;
            float top = -INFINITY, sum = 0.0f;
#pragma unroll
            for (int j = 0; j < S::kWarps; j++) top = fmaxf(top, ml[j * kRows + r].x);
#pragma unroll
            for (int j = 0; j < S::kWarps; j++) {
                const float2 x = ml[j * kRows + r];
                sum += x.y * exp2_fast(x.x - (top == -INFINITY ? 0.0f : top));
            }
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; e++) v[e] = 0.0f;
#pragma unroll
            for (int j = 0; j < S::kSets; j++) {
                const float4* x = reinterpret_cast<const float4*>(sets + (j * kRows + r) * DP + (d ^ (r & 3) * 8));
                const float4 x0 = x[0], x1 = x[1];
                v[0] += x0.x; v[1] += x0.y; v[2] += x0.z; v[3] += x0.w;
                v[4] += x1.x; v[5] += x1.y; v[6] += x1.z; v[7] += x1.w;
            }
            const int n = w.tile * kRows + r, tok = n / a.share;
            if (odd && r < rows && d < a.head_dim)
#pragma unroll 1
                for (int e = 0; e < 8; e++) {
                    const float more_of = unseen_spoils<T>(a, w.s, w.b, w.head, tok, w.s.row0 + tok, d + e, k0, k1);
#pragma unroll
                    for (int x = 0; x < 8; x++) v[x] += x == e ? more_of : 0.0f;
                }
            if (!whole) {
                *reinterpret_cast<float4*>(part + r * DP + d) = make_float4(v[0], v[1], v[2], v[3]);
                *reinterpret_cast<float4*>(part + r * DP + d + 4) = make_float4(v[4], v[5], v[6], v[7]);
                if (d == 0) {
                    part[kRows * DP + r] = top;
                    part[kRows * DP + kRows + r] = sum;
                }
                continue;
            }
            if (r >= rows || d >= a.head_dim) continue;
            const float by = sum == 0.0f ? 0.0f : 1.0f / sum;
            const int h = w.head * a.share + n % a.share;
            const long long at = w.s.row0 + tok;
            *reinterpret_cast<uint4*>(static_cast<T*>(a.out) + at * a.out_token + h * a.out_head + d) =
                make_uint4(pack2<T>(v[0] * by, v[1] * by), pack2<T>(v[2] * by, v[3] * by), pack2<T>(v[4] * by, v[5] * by), pack2<T>(v[6] * by, v[7] * by));
            if (a.lse && d == 0) a.lse[at * (a.kv_heads * a.share) + h] = sum == 0.0f ? -INFINITY : (top + log2f(sum)) * 0.69314718055994531f;
        }
        if (tid == 0 && !whole && w.t0() == 0) a.joins[blockIdx.x] = AttnJoin{w.b, w.tile * kRows, w.head, w.others(), min(rows, kRows), {0, 0, 0}};
        turn ^= 1;
        if (tid == 0) spoilt[turn] = 0;          // (the next unit's; the last to read it did so before that unit's last barrier)
        __syncthreads();
    }
    copies_wait<0>();
}

// Joins the parts of units that were cut: CTAs x take those of the unit that begins in CTA x of the kernel before, each y a share of its values.
//   rows_of_tile : rows of a part;  by_piece : a part lies as [dp / 4][rows][4], else as [rows][dp];  behind that the rows' maxima and sums
constexpr int kJoinThreads = 256, kJoinPieces = 1024;
template <class T>
__global__ void __launch_bounds__(kJoinThreads) attention_join_kernel(const __grid_constant__ AttnArgs a, int rows_of_tile, int dp, int by_piece)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const AttnJoin j = a.joins[blockIdx.x];
    if (j.others == 0) return;
    const int s0 = a.starts[j.seq], per_row = dp / 4, end = min(rows_of_tile * per_row, ((int)blockIdx.y + 1) * kJoinPieces);
    const long long slot = (long long)rows_of_tile * (dp + 2);
    // the first part is the second slot of its CTA, the others are the first slots of those behind it
    const float* first = a.parts + (blockIdx.x * 2 + 1) * slot;
    const float* rest = a.parts + (blockIdx.x + 1) * 2 * slot;
    for (int i = blockIdx.y * kJoinPieces + threadIdx.x; i < end; i += kJoinThreads) {
        const int r = by_piece ? i % rows_of_tile : i / per_row, d = (by_piece ? i / rows_of_tile : i % per_row) * 4;
        if (r >= j.rows || d >= a.head_dim) continue;
        const long long om = (long long)rows_of_tile * dp + r, ol = om + rows_of_tile;
        float top = __ldcg(first + om);
#pragma unroll 4
        for (int x = 0; x < j.others; x++) top = fmaxf(top, __ldcg(rest + x * 2 * slot + om));
        const float base = top == -INFINITY ? 0.0f : top;
        float by = exp2_fast(__ldcg(first + om) - base), sum = __ldcg(first + ol) * by;
        float4 v = __ldcg(reinterpret_cast<const float4*>(first) + i);
        v = make_float4(v.x * by, v.y * by, v.z * by, v.w * by);
#pragma unroll 4
        for (int x = 0; x < j.others; x++) {
            const float* p = rest + x * 2 * slot;
            by = exp2_fast(__ldcg(p + om) - base);
            sum += __ldcg(p + ol) * by;
            const float4 u = __ldcg(reinterpret_cast<const float4*>(p) + i);
            v.x += u.x * by; v.y += u.y * by; v.z += u.z * by; v.w += u.w * by;
        }
        by = sum == 0.0f ? 0.0f : 1.0f / sum;
        const int n = j.row0 + r, h = j.head * a.share + n % a.share;
        const long long at = s0 + n / a.share;
        *reinterpret_cast<uint2*>(static_cast<T*>(a.out) + at * a.out_token + h * a.out_head + d) = make_uint2(pack2<T>(v.x * by, v.y * by), pack2<T>(v.z * by, v.w * by));
        if (a.lse && d == 0) a.lse[at * (a.kv_heads * a.share) + h] = sum == 0.0f ? -INFINITY : (top + log2f(sum)) * 0.69314718055994531f;
    }
}

template <class T, int DP>
int launch_attention(const fq_ctx* ctx, const AttnArgs& a, cudaStream_t st)
{
    using S = Shape<DP>;
    static std::atomic<bool> ready[64];
    if (ctx->device >= 64) return FQ_ERR_ARG;
    if (!ready[ctx->device].load(std::memory_order_acquire)) {
        if (cudaFuncSetAttribute(attention_kernel<T, DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kTotal) != cudaSuccess) return FQ_ERR_CUDA;
        ready[ctx->device].store(true, std::memory_order_release);
    }
    attention_kernel<T, DP><<<ctx->sm_count, S::kThreads, S::kTotal, st>>>(a);
    return cudaGetLastError() == cudaSuccess ? FQ_OK : FQ_ERR_CUDA;
}

int padded_dim(int head_dim) { return head_dim <= 64 ? 64 : head_dim <= 128 ? 128 : 256; }

// Query rows of a unit.  Up to 16 rows to a key head go to the kernel of this file, whose work grows with every 16 rows; more to the tensor cores',
// whose does with every 128, two tiles of them side by side where there are as many.
int unit_rows(int new_tokens, int share, int dp)
{
    const long long rows = (long long)new_tokens * share;
    return rows <= kRows ? kRows : rows <= 128 || dp == 256 ? 128 : 256;
}

template <class T>
int launch_typed(const fq_ctx* ctx, const AttnArgs& a, int rows, int dp, cudaStream_t st)
{
    int rc;
    if (rows > kRows) rc = launch_attention_tc(ctx, a, std::is_same<T, __half>::value ? FQ_DT_F16 : FQ_DT_BF16, rows, dp, st);
    else if (dp == 64) rc = launch_attention<T, 64>(ctx, a, st);
    else if (dp == 128) rc = launch_attention<T, 128>(ctx, a, st);
    else rc = launch_attention<T, 256>(ctx, a, st);
    if (rc != FQ_OK) return rc;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)ctx->sm_count, (unsigned)((rows * dp / 4 + kJoinPieces - 1) / kJoinPieces)); cfg.blockDim = dim3(kJoinThreads);
    cfg.stream = st; cfg.attrs = &attr; cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, attention_join_kernel<T>, a, rows, dp, rows > kRows ? 1 : 0) == cudaSuccess ? FQ_OK : FQ_ERR_CUDA;
}

bool good_sizes(const fq_ctx* ctx, int n_seqs, int tokens, int q_heads, int cache_heads, int head_dim, int new_tokens)
{
    return n_seqs >= 1 && n_seqs <= FQ_MAX_SEQS && tokens >= 1 && tokens <= FQ_MAX_ROWS && cache_heads >= 1 && q_heads >= cache_heads && q_heads <= 1024 &&
           q_heads % cache_heads == 0 && head_dim >= 8 && head_dim <= 256 && head_dim % 8 == 0 && new_tokens >= 1;
}

size_t join_bytes(const fq_ctx* ctx) { return ((size_t)ctx->sm_count * sizeof(AttnJoin) + 127) / 128 * 128; }

}  // namespace
}  // namespace fq

using namespace fq;

extern "C" {

size_t fq_tree_attention_scratch(const fq_ctx* ctx, int n_seqs, int tokens, int q_heads, int cache_heads, int head_dim, int new_tokens)
{
    if (!ctx || !good_sizes(ctx, n_seqs, tokens, q_heads, cache_heads, head_dim, new_tokens)) return 0;
    const int dp = padded_dim(head_dim), rows = unit_rows(new_tokens, q_heads / cache_heads, dp);
    return join_bytes(ctx) + (size_t)ctx->sm_count * 2 * rows * (dp + 2) * sizeof(float);
}

int fq_tree_attention(fq_ctx* ctx, const fq_heads* q, const fq_heads* out, const fq_cache* cache, int dtype, int head_dim, int tokens, int n_seqs,
                      const int* starts_dev, const int* lens_dev, const int* table_dev, long long ld, int max_blocks, const uint64_t* mask_dev, int words,
                      int new_tokens, float scale, float* lse_dev, void* scratch_dev, size_t scratch_bytes, void* stream)
{
    if (!ctx || !q || !out || !cache || !q->dev || !out->dev || !starts_dev || !lens_dev || !scratch_dev) return FQ_ERR_ARG;
    if ((dtype != FQ_DT_F16 && dtype != FQ_DT_BF16) || !(scale > 0.0f) || !std::isfinite(scale)) return FQ_ERR_ARG;
    if (!good_sizes(ctx, n_seqs, tokens, q->heads, cache->heads, head_dim, new_tokens) || out->heads != q->heads) return FQ_ERR_SHAPE;
    if (mask_dev && (words < 1 || words > FQ_MAX_TREE_WORDS)) return FQ_ERR_SHAPE;
    int rc = check_heads(out, dtype, tokens, head_dim);
    if (rc == FQ_OK) rc = check_cache(cache, dtype, head_dim);
    if (rc == FQ_OK) rc = check_table(table_dev, ld, n_seqs, max_blocks, cache->block_size);
    if (rc != FQ_OK) return rc;
    if (q->head_stride < 0 || q->token_stride < 0) return FQ_ERR_SHAPE;
    const bool many = tokens > 1, wide = q->heads > 1;
    if (!aligned(q->dev, 16) || !aligned(out->dev, 16) || !aligned(scratch_dev, 16) || !aligned(starts_dev, 4) || !aligned(lens_dev, 4) ||
        !aligned(mask_dev, 8) || !aligned(lse_dev, 4) || (many && (q->token_stride % 8 || out->token_stride % 8)) ||
        (wide && (q->head_stride % 8 || out->head_stride % 8)))
        return FQ_ERR_ALIGN;
    if (scratch_bytes < fq_tree_attention_scratch(ctx, n_seqs, tokens, q->heads, cache->heads, head_dim, new_tokens)) return FQ_ERR_SCRATCH;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return FQ_ERR_CUDA;
    AttnArgs a{};
    a.q = q->dev; a.out = out->dev;
    a.q_token = many ? q->token_stride : 0; a.q_head = wide ? q->head_stride : 0;
    a.out_token = many ? out->token_stride : 0; a.out_head = wide ? out->head_stride : 0;
    a.k = cache->k_dev; a.v = cache->v_dev;
    a.block_stride = cache->blocks > 1 ? cache->block_stride : 0; a.cell_stride = cache->block_size > 1 ? cache->token_stride : 0;
    a.head_stride = cache->heads > 1 ? cache->head_stride : 0;
    a.blocks = cache->blocks; a.block_size = cache->block_size;
    a.tokens = tokens; a.n_seqs = n_seqs; a.kv_heads = cache->heads; a.share = q->heads / cache->heads; a.head_dim = head_dim;
    a.starts = starts_dev; a.lens = lens_dev; a.table = table_dev; a.ld = ld; a.max_blocks = max_blocks; a.mask = mask_dev; a.words = words;
    a.scale = (float)((double)scale * 1.4426950408889634);
    a.lse = lse_dev;
    a.joins = static_cast<AttnJoin*>(scratch_dev);
    a.parts = reinterpret_cast<float*>(static_cast<char*>(scratch_dev) + join_bytes(ctx));
    a.status = ctx->status_dev;
    const cudaStream_t st = (cudaStream_t)stream;
    const int dp = padded_dim(head_dim), rows = unit_rows(new_tokens, a.share, dp);
    return dtype == FQ_DT_F16 ? launch_typed<__half>(ctx, a, rows, dp, st) : launch_typed<__nv_bfloat16>(ctx, a, rows, dp, st);
}

}  // extern "C"
