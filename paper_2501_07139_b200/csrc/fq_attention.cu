// Attention of a sequence's last tokens over its paged cache, up to 16 query rows to a key head (single tokens, small trees) and heads of up to 128: bound by
// reading keys and values.
//
// Every warp is a worker: it has a share of the batch's work of its own, which it fetches by its own asynchronous copies, 16 cells at a time, into its own
// ring (192 KB an SM, of which two thirds are on their way), so that nobody waits for another before the end of the kernel; there the warps join
// what they have of the same units.  (With a unit's keys dealt to all warps of a CTA, and their parts joined at its end, a unit's ends took 4 us of the
// CTA: 48 tokens of a ragged batch, 40 heads, 391 us.)  Scores and values are formed by mma.m16n8k16: at 16 rows the bytes
// of a key take ten times as long to arrive as its products take.
#include "fq_attention.cuh"

#include <atomic>
#include <cmath>

#include "fq_rowtypes.cuh"

namespace fq {
namespace {

constexpr int kRows = 16;
constexpr int kChunk = 16;                       // cells of a warp's share of a key tile

constexpr int kWorkers = 8;                      // warps of a CTA
template <int DP>
struct Shape {                                   // DP: head_dim, rounded up to 64 or 128
    static constexpr int kWarps = kWorkers;
    static constexpr int kThreads = kWarps * 32;
    static constexpr int kStageBytes = 2 * kChunk * DP * 2;                  // of a warp: keys, then values
    static constexpr int kStages = 196608 / (kWarps * kStageBytes);
    static constexpr int kSlot = kRows * (DP + 2);                           // floats of a part: [rows][DP], maxima, sums
    // A unit's ends (the queries' way here, the results' way out) take the time of two chunks; a worker gets no less than four.
    using Work = Deal<kRows, kChunk, 2, kThreads, kWarps, 4>;
    static constexpr int oSums = kWarps * kStages * kStageBytes;             // long long [Work::kSums]
    static constexpr int oLeft = oSums + Work::kSums * 8;                    // Left [warps]
    static constexpr int oOdd = oLeft + kWarps * 32;                         // bits [warps][kOddWords]
    static constexpr int kTotal = oOdd + kWarps * kOddWords * 4;
    static_assert(kTotal <= 232448, "shared memory over the per-CTA limit");
};
// What a warp leaves: a part of the unit that it continues, whether that ends here, a part of a unit that ends elsewhere; rows of the first, and the
// second: its rows, first row of its sequence in the batch, row tile, key head.
enum { kContinues = 1, kEnds = 2, kBegins = 4 };
struct Left { int flag, lead_rows, rows, seq_row0, tile, head, pad[2]; };
static_assert(sizeof(Left) == 32, "Shape::oLeft");

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
// Parts 0 .. n - 1 of row r become one: their values d .. d + 3 (at offset `at`), the row's maximum (at `om`) and sum (at `ol`).  part(x): where part x is.
struct Joined { float4 v; float top, sum; };
template <class Part>
__device__ __forceinline__ Joined join_parts(Part part, int n, int at, int om, int ol)
{
    Joined j{make_float4(0.0f, 0.0f, 0.0f, 0.0f), -INFINITY, 0.0f};
    // (eight at a time: their loads are on their way together)
    for (int x0 = 0; x0 < n; x0 += 8) {
        float m[8], l[8];
        float4 v[8];
#pragma unroll
        for (int i = 0; i < 8; i++) {
            m[i] = -INFINITY;
            l[i] = 0.0f;
            v[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (x0 + i < n) {
                const float* p = part(x0 + i);
                m[i] = p[om];
                l[i] = p[ol];
                v[i] = *reinterpret_cast<const float4*>(p + at);
            }
        }
        float top = j.top;
#pragma unroll
        for (int i = 0; i < 8; i++) top = fmaxf(top, m[i]);
        const float base = top == -INFINITY ? 0.0f : top;
        float by = exp2_fast(j.top - base);
        j.top = top;
        j.sum *= by;
        j.v = make_float4(j.v.x * by, j.v.y * by, j.v.z * by, j.v.w * by);
#pragma unroll
        for (int i = 0; i < 8; i++) {
            by = exp2_fast(m[i] - base);
            j.sum += l[i] * by;
            j.v.x += v[i].x * by; j.v.y += v[i].y * by; j.v.z += v[i].z * by; j.v.w += v[i].w * by;
        }
    }
    return j;
}
// Row r of a unit, values d .. d + 3.
template <class T>
__device__ __forceinline__ void write_out(const AttnArgs& a, int row0, int n, int head, int d, const Joined& j)
{
    const float by = j.sum == 0.0f ? 0.0f : 1.0f / j.sum;
    const int t = n / a.share, h = head * a.share + n - t * a.share;
    const long long at = row0 + t;
    *reinterpret_cast<uint2*>(static_cast<T*>(a.out) + at * a.out_token + h * a.out_head + d) =
        make_uint2(pack2<T>(j.v.x * by, j.v.y * by), pack2<T>(j.v.z * by, j.v.w * by));
    if (a.lse && d == 0) a.lse[at * (a.kv_heads * a.share) + h] = j.sum == 0.0f ? -INFINITY : (j.top + log2f(j.sum)) * 0.69314718055994531f;
}

template <class T, int DP>
__global__ void __launch_bounds__(Shape<DP>::kThreads, 1) attention_kernel(const __grid_constant__ AttnArgs a)
{
    using S = Shape<DP>;
    using Work = typename S::Work;
    constexpr int kUnits = DP / 8;               // 16-byte pieces of a row
    constexpr int kSteps = DP / 16;
    extern __shared__ __align__(1024) char smem[];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, c = lane & 3;
    const uint32_t ring = smem_u32(smem) + warp * S::kStages * S::kStageBytes;
    volatile Left* left = reinterpret_cast<volatile Left*>(smem + S::oLeft);
    uint32_t* odd_cells = reinterpret_cast<uint32_t*>(smem + S::oOdd) + warp * kOddWords;
    odd_cells[lane] = 0;                         // (begin() has a barrier)
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");              // (the joining kernel waits for this one's end)
    if (tid == 0) {
        AttnJoin none{};
        a.joins[blockIdx.x] = none;
    }
    Work w;
    const bool some = w.begin(a, reinterpret_cast<long long*>(smem + S::oSums));
    const int pieces = a.head_dim / 8;
    float* parts = a.parts + (long long)(blockIdx.x * S::kWarps + warp) * 2 * S::kSlot;

    // ---- fetching runs ahead of computing, over the ends of units
    Work f = w;
    int f_tile = 0, f_stage = 0, f_block = -1;
    bool f_more = some;
    const auto settle = [&]() {                  // f at a unit with key tiles, and its next tile's block on the way
        while (f_more && f_tile >= f.t1()) {
            f_more = f.next(a);
            f_tile = f_more ? f.t0() : 0;
        }
        f_block = -1;
        if (f_more) {
            const int cell = f_tile * kChunk + (lane & 15);
            if (cell < f.s.len) f_block = a.table[f.b * a.ld + cell / a.block_size];
        }
    };
    const auto fetch = [&]() {
        if (f_more) {
            const int cell = f_tile * kChunk + (lane & 15);
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
    if (some) {
        f_tile = f.t0();
        settle();
    }
#pragma unroll 1
    for (int i = 0; i < S::kStages - 1; i++) fetch();

    int stage = 0, flag = 0, lead_rows = 0;
    for (bool more = some; more;) {
        if (!w.any()) {
            more = w.next(a);
            continue;
        }
        const int rows = min(w.s.fresh * a.share - w.tile * kRows, kRows);       // of the unit
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
            const T* q = static_cast<const T*>(a.q) + row[h] * a.q_token + (w.head * a.share + r - t[h] * a.share) * a.q_head;
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
        const int t0 = w.t0(), t1 = w.t1();
        bool odd = false;                        // infinities or NaNs among values that not all rows see
        for (int tile = t0; tile < t1; tile++) {
            copies_wait<S::kStages - 2>();
            __syncwarp();
            fetch();
            const uint32_t ks = ring + stage * S::kStageBytes, vs = ks + kChunk * DP * 2;
            stage = stage + 1 == S::kStages ? 0 : stage + 1;
            const int cell0 = tile * kChunk;
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
                // values that not all rows see: none may be infinite or NaN in the product.  (Those of the cells before stay as they are.)
#pragma unroll 1
                for (int i = 0; i < kChunk * kUnits / 32; i++) {
                    const int cell = cell0 + (i * 32 + lane) / kUnits;
                    const uint32_t at = vs + (uint32_t)(i * 32 + lane) * 16;
                    uint4 v = lds128(at);
                    const bool mine = cell >= all_see && take_out<T>(v);
                    if (mine) sts128(at, v);
                    odd |= note_odd<kUnits>(odd_cells, mine, cell - all_see);
                }
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
            // (the product takes 16-bit weights: half a step of each, as much as an output's own rounding; the sum above has them in full)
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
        // ---- the unit's end, or this worker's
        const bool whole = w.whole();
        // A part that does not end its share goes to scratch, else to this warp's ring, which nobody needs any more.
        const bool last = !whole && t1 < w.tiles;
        if (last) {
            copies_wait<0>();
            __syncwarp();
        }
        float* part = last ? reinterpret_cast<float*>(smem + warp * S::kStages * S::kStageBytes) : parts;
#pragma unroll
        for (int h = 0; h < 2; h++) {
            l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
            l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
            const int r = g + 8 * h;
            if (r >= rows) continue;
            if (whole) {
                const float by = l[h] == 0.0f ? 0.0f : 1.0f / l[h];
                const int head = w.head * a.share + w.tile * kRows + r - t[h] * a.share;
                T* out = static_cast<T*>(a.out) + row[h] * a.out_token + head * a.out_head;
#pragma unroll
                for (int n = 0; n < DP / 8; n++)
                    if (n < pieces) *reinterpret_cast<uint32_t*>(out + n * 8 + 2 * c) = pack2<T>(o[n][2 * h] * by, o[n][2 * h + 1] * by);
                if (a.lse && c == 0) a.lse[(long long)row[h] * (a.kv_heads * a.share) + head] = l[h] == 0.0f ? -INFINITY : (m[h] + log2f(l[h])) * 0.69314718055994531f;
            } else {
#pragma unroll
                for (int n = 0; n < DP / 8; n++) *reinterpret_cast<float2*>(part + r * DP + n * 8 + 2 * c) = make_float2(o[n][2 * h], o[n][2 * h + 1]);
                if (c == 0) {
                    part[kRows * DP + r] = m[h];
                    part[kRows * (DP + 1) + r] = l[h];
                }
            }
        }
        if (odd) {
            __syncwarp();
            const int r = min(lane, rows - 1), n = w.tile * kRows + r, tok = n / a.share;
            T* out = static_cast<T*>(a.out) + (long long)(w.s.row0 + tok) * a.out_token + (w.head * a.share + n - tok * a.share) * a.out_head;
            give_back<T>(a, w.s, w.b, w.head, tok, lane < rows, all_see, odd_cells, [&](int d, float x) {
                if (whole) out[d] = (T)((float)out[d] + x);                  // (cells that all rows see may have left an infinity there)
                else part[r * DP + d] += x;
            });
            __syncwarp();
            odd_cells[lane] = 0;
            __syncwarp();
        }
        if (!whole && t0 > 0) {
            flag |= t1 == w.tiles ? kContinues | kEnds : kContinues;
            lead_rows = rows;
        }
        if (!whole && t0 == 0) {
            flag |= kBegins;                     // (the share's last unit: w stays at it)
            break;
        }
        more = w.next(a);
    }
    copies_wait<0>();

    // ---- what the warps have of the same units, joined by all of them
    const bool begins = flag & kBegins;
    if (lane == 0) {
        left[warp].flag = flag;
        left[warp].lead_rows = lead_rows;
        if (begins) {
            left[warp].rows = min(w.s.fresh * a.share - w.tile * kRows, kRows);
            left[warp].seq_row0 = w.s.row0; left[warp].tile = w.tile; left[warp].head = w.head;
        }
    }
    __syncthreads();
    // Unit by unit: the one that this CTA continues (f = -1), then those that begin in a warp and end elsewhere.
    for (int f = -1; f < w.per_cta; f++) {
        const int first = max(f, 0);
        if (f < 0 ? (left[0].flag & (kContinues | kEnds)) != kContinues : !(left[f].flag & kBegins)) continue;   // (one that ends in the first warp is in scratch already)
        int n = 1;
        bool ends = false;
        while (!ends && first + n < w.per_cta && (left[first + n].flag & kContinues)) {
            ends = left[first + n].flag & kEnds;
            n++;
        }
        const bool out = f >= 0 && ends;         // all of the unit is here; else it goes to scratch for the other kernel
        const int rows = f < 0 ? left[0].lead_rows : left[f].rows;
        const float* last = a.parts + (long long)(blockIdx.x * S::kWarps + first + n - 1) * 2 * S::kSlot;
        const auto part = [&](int x) -> const float* {
            return ends && x == n - 1 ? last : reinterpret_cast<const float*>(smem + (first + x) * S::kStages * S::kStageBytes);
        };
        float* to = a.parts + ((long long)(blockIdx.x * S::kWarps + first) * 2 + (f >= 0)) * S::kSlot;
        for (int i = tid; i < rows * (DP / 4); i += S::kThreads) {
            const int r = i / (DP / 4), d = i % (DP / 4) * 4;
            if (d >= a.head_dim) continue;
            const Joined j = join_parts(part, n, r * DP + d, kRows * DP + r, kRows * (DP + 1) + r);
            if (out) {
                write_out<T>(a, left[f].seq_row0, left[f].tile * kRows + r, left[f].head, d, j);
                continue;
            }
            *reinterpret_cast<float4*>(to + r * DP + d) = j.v;
            if (d == 0) {
                to[kRows * DP + r] = j.top;
                to[kRows * (DP + 1) + r] = j.sum;
            }
        }
        if (f >= 0 && !ends && warp == f && lane == 0)
            a.joins[blockIdx.x] = AttnJoin{w.s.row0, w.tile * kRows, w.head, w.others(), rows, (int)(blockIdx.x * S::kWarps + f) * 2 + 1, {0, 0}};
    }
}

// Joins the parts of units that were cut between CTAs: CTAs x take those of the unit that begins in CTA x of the kernel before, each y a share of its values.
//   rows_of_tile : rows of a part;  by_piece : a part lies as [dp / 4][rows][4], else as [rows][dp];  behind that the rows' maxima and sums
//   workers : of a CTA, each with two slots
constexpr int kJoinThreads = 256, kJoinPieces = 1024;
template <class T>
__global__ void __launch_bounds__(kJoinThreads) attention_join_kernel(const __grid_constant__ AttnArgs a, int rows_of_tile, int dp, int by_piece, int workers)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const AttnJoin j = a.joins[blockIdx.x];
    if (j.others == 0) return;
    const int per_row = dp / 4, end = min(rows_of_tile * per_row, ((int)blockIdx.y + 1) * kJoinPieces);
    const long long slot = (long long)rows_of_tile * (dp + 2);
    const float* first = a.parts + j.slot * slot;
    const float* rest = a.parts + (blockIdx.x + 1) * 2 * workers * slot;         // (of what a CTA continues, its first worker has all)
    for (int i = blockIdx.y * kJoinPieces + threadIdx.x; i < end; i += kJoinThreads) {
        const int r = by_piece ? i % rows_of_tile : i / per_row, d = (by_piece ? i / rows_of_tile : i % per_row) * 4;
        if (r >= j.rows || d >= a.head_dim) continue;
        const int om = rows_of_tile * dp + r;
        const auto part = [&](int x) { return x == 0 ? first : rest + (x - 1) * 2 * workers * slot; };
        write_out<T>(a, j.seq_row0, j.row0 + r, j.head, d, join_parts(part, j.others + 1, i * 4, om, om + rows_of_tile));
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

// Query rows of a unit, by how many a key head has.  (Measured, us; "warps" is this file's kernel.)
//   Up to 16, heads of up to 128: warps.  48 sequences of 4096, 40 heads, 1 row: 339, tensor cores 411; 64 of 1000, 8 heads, 8 rows: 37 and 59, 16 rows 44 and 59; one
//   of 4000, 32 heads, 1 row: 20.5 and 28.5, 8 heads, 16 rows: 22 and 25.  Larger heads: tensor cores (16 sequences of 4000, 8 heads of 256, 1 row: 77, warps 82; 8 rows of 32 x 2000: 74 and 94).
//   Up to 256: one tile of 128 query rows at a time.  16 sequences of 16000, 8 heads, 32 rows: 114, two tiles 134; 256 rows of 16 x 4000: 55 and 65; 240 rows of 5 x
//   40000: 153 and 144.  More: two tiles side by side, which read keys once for both.  480 rows of 5 x 40000: 222, one tile at a time 293; 320 rows: 200 and 238; four
//   prompts of up to 2048: 129 and 151; 300 rows of 2 x 8000 cells, 32 heads: 101 and 109.
int unit_rows(int new_tokens, int share, int dp)
{
    const long long rows = (long long)new_tokens * share;
    if (dp == 256) return 128;
    return rows <= kRows ? kRows : rows <= 256 ? 128 : 256;
}
int workers_of(int rows) { return rows > kRows ? 1 : kWorkers; }

template <class T>
int launch_typed(const fq_ctx* ctx, const AttnArgs& a, int rows, int dp, cudaStream_t st)
{
    int rc;
    if (rows > kRows) rc = launch_attention_tc(ctx, a, std::is_same<T, __half>::value ? FQ_DT_F16 : FQ_DT_BF16, rows, dp, st);
    else if (dp == 64) rc = launch_attention<T, 64>(ctx, a, st);
    else rc = launch_attention<T, 128>(ctx, a, st);
    if (rc != FQ_OK) return rc;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)ctx->sm_count, (unsigned)((rows * dp / 4 + kJoinPieces - 1) / kJoinPieces)); cfg.blockDim = dim3(kJoinThreads);
    cfg.stream = st; cfg.attrs = &attr; cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, attention_join_kernel<T>, a, rows, dp, rows > kRows ? 1 : 0, workers_of(rows)) == cudaSuccess ? FQ_OK : FQ_ERR_CUDA;
}

bool good_sizes(int n_seqs, int tokens, int q_heads, int cache_heads, int head_dim, int new_tokens)
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
    if (!ctx || !good_sizes(n_seqs, tokens, q_heads, cache_heads, head_dim, new_tokens)) return 0;
    const int dp = padded_dim(head_dim), rows = unit_rows(new_tokens, q_heads / cache_heads, dp);
    return join_bytes(ctx) + (size_t)ctx->sm_count * workers_of(rows) * 2 * rows * (dp + 2) * sizeof(float);
}

int fq_tree_attention(fq_ctx* ctx, const fq_attention_args* args, void* stream)
{
    if (!ctx || !args) return FQ_ERR_ARG;
    const fq_attention_args& x = *args;
    const fq_heads &q = x.q, &out = x.out;
    const fq_cache& cache = x.cache;
    if (!q.dev || !out.dev || !x.starts_dev || !x.lens_dev || !x.scratch_dev) return FQ_ERR_ARG;
    if ((x.dtype != FQ_DT_F16 && x.dtype != FQ_DT_BF16) || !(x.scale > 0.0f) || !std::isfinite(x.scale)) return FQ_ERR_ARG;
    if (!good_sizes(x.n_seqs, x.tokens, q.heads, cache.heads, x.head_dim, x.new_tokens) || out.heads != q.heads) return FQ_ERR_SHAPE;
    if (x.mask_dev && (x.words < 1 || x.words > FQ_MAX_TREE_WORDS)) return FQ_ERR_SHAPE;
    int rc = check_heads(&out, x.dtype, x.tokens, x.head_dim);
    if (rc == FQ_OK) rc = check_cache(&cache, x.dtype, x.head_dim);
    if (rc == FQ_OK) rc = check_table(x.table_dev, x.ld, x.n_seqs, x.max_blocks, cache.block_size);
    if (rc != FQ_OK) return rc;
    if (q.head_stride < 0 || q.token_stride < 0) return FQ_ERR_SHAPE;
    const bool many = x.tokens > 1, wide = q.heads > 1;
    if (!aligned(q.dev, 16) || !aligned(out.dev, 16) || !aligned(x.scratch_dev, 16) || !aligned(x.starts_dev, 4) || !aligned(x.lens_dev, 4) ||
        !aligned(x.mask_dev, 8) || !aligned(x.lse_dev, 4) || (many && (q.token_stride % 8 || out.token_stride % 8)) ||
        (wide && (q.head_stride % 8 || out.head_stride % 8)))
        return FQ_ERR_ALIGN;
    if (out.dev == q.dev) return FQ_ERR_ARG;     // (several CTAs read a unit's queries)
    if (x.scratch_bytes < fq_tree_attention_scratch(ctx, x.n_seqs, x.tokens, q.heads, cache.heads, x.head_dim, x.new_tokens)) return FQ_ERR_SCRATCH;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return FQ_ERR_CUDA;
    AttnArgs a{};
    a.q = q.dev; a.out = out.dev;
    a.q_token = many ? q.token_stride : 0; a.q_head = wide ? q.head_stride : 0;
    a.out_token = many ? out.token_stride : 0; a.out_head = wide ? out.head_stride : 0;
    a.rows_by_tma = 128 % (q.heads / cache.heads) == 0 && (!many || q.token_stride > 0) && (!wide || q.head_stride > 0);
    a.k = cache.k_dev; a.v = cache.v_dev;
    a.block_stride = cache.blocks > 1 ? cache.block_stride : 0; a.cell_stride = cache.block_size > 1 ? cache.token_stride : 0;
    a.head_stride = cache.heads > 1 ? cache.head_stride : 0;
    a.blocks = cache.blocks; a.block_size = cache.block_size;
    a.tokens = x.tokens; a.n_seqs = x.n_seqs; a.kv_heads = cache.heads; a.share = q.heads / cache.heads; a.head_dim = x.head_dim;
    a.starts = x.starts_dev; a.lens = x.lens_dev; a.table = x.table_dev; a.ld = x.ld; a.max_blocks = x.max_blocks; a.mask = x.mask_dev; a.words = x.words;
    a.scale = (float)((double)x.scale * 1.4426950408889634);
    a.lse = x.lse_dev;
    a.joins = static_cast<AttnJoin*>(x.scratch_dev);
    a.parts = reinterpret_cast<float*>(static_cast<char*>(x.scratch_dev) + join_bytes(ctx));
    a.status = ctx->status_dev;
    const cudaStream_t st = (cudaStream_t)stream;
    const int dp = padded_dim(x.head_dim), rows = unit_rows(x.new_tokens, a.share, dp);
    return x.dtype == FQ_DT_F16 ? launch_typed<__half>(ctx, a, rows, dp, st) : launch_typed<__nv_bfloat16>(ctx, a, rows, dp, st);
}

}  // extern "C"
