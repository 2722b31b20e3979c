// What the attention kernels share: their arguments, how the work of a batch is dealt, and what a row sees.
//
// Work.  A unit is one key head of one sequence and a tile of its query rows: the query heads that share the key head, for all new tokens, are rows
// r = token * share + head, so that keys and values are read once for all of them.  A unit costs the key tiles that its rows see and
// some more for its ends.  The host does not know the lengths, so every CTA adds the costs up for itself; a worker (a CTA, or a warp) takes an equal
// share of the sum.  Units of long sequences are cut: each part leaves (maximum, sum, values) in scratch, and they are joined by the CTA whose
// warps have them all, or by a second small kernel.  The parts and their order depend on the lengths alone.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cmath>
#include <type_traits>

#include "fq_internal.cuh"
#include "fq_ptx.cuh"

namespace fq {

struct AttnArgs {
    const void* q;
    void* out;
    long long q_token, q_head, out_token, out_head;
    bool rows_by_tma;                            // a tile of 128 query rows is a whole number of tokens, and no stride is 0
    const void* k;
    const void* v;
    long long block_stride, cell_stride, head_stride;
    int blocks, block_size;
    int tokens, n_seqs, kv_heads, share;         // share: query heads of a key head
    int head_dim;
    const int* starts;
    const int* lens;
    const int* table;
    long long ld;
    int max_blocks;
    const uint64_t* mask;                        // null: a token sees those before it
    int words;
    float scale;                                 // times log2 e
    float* lse;
    float* parts;                                // two slots a worker, rows x (head_dim + 2): of the unit it continues, of the one it leaves unfinished
    struct AttnJoin* joins;                      // one a CTA
    int* status;
};

// A unit that begins in this CTA and ends in another.
struct AttnJoin {
    int seq_row0, row0, head;                    // first rows of the sequence in the batch and of the unit in the sequence
    int others;                                  // CTAs behind this one that hold parts (0: nothing to join)
    int rows;                                    // rows of the unit
    int slot;                                    // where its first part is
    int pad[2];
};

struct Seq {
    int row0, fresh, len, ctx;                   // first row in the batch, new tokens, cells, cells before the new ones
    // Numbers that cannot be never lead outside the arrays.
    __device__ __forceinline__ Seq(const AttnArgs& a, int b)
    {
        row0 = a.starts[b];
        const int end = a.starts[b + 1];
        len = a.lens[b];
        fresh = end - row0;
        if (row0 < 0 || fresh < 0 || end > a.tokens || len < fresh || len > (long long)a.max_blocks * a.block_size) {
            if (row0 < 0 || fresh < 0 || end > a.tokens) row0 = fresh = 0;
            len = 0;
            atomicCAS(a.status, 0, FQ_ERR_INDEX);
        }
        ctx = max(0, len - fresh);
    }
    __device__ __forceinline__ Seq() {}
};

// Key tiles of KEYS cells that a tile of ROWS query rows sees (rows r0 .. of a sequence).
template <int ROWS, int KEYS>
__device__ __forceinline__ int key_tiles(const AttnArgs& a, const Seq& s, int row_tile)
{
    int last = s.len;                            // with a tree's bits any row may see any new token
    if (!a.mask) last = min(last, s.ctx + ((row_tile + 1) * ROWS - 1) / a.share + 1);
    return (last + KEYS - 1) / KEYS;
}
template <int ROWS>
__device__ __forceinline__ int row_tiles(const AttnArgs& a, const Seq& s) { return (s.fresh * a.share + ROWS - 1) / ROWS; }

// Cost of one key head of a sequence.  ENDS: key tiles that a unit's beginning and end take the time of.
template <int ROWS, int KEYS, int ENDS>
__device__ __forceinline__ long long head_cost(const AttnArgs& a, const Seq& s)
{
    const int n = row_tiles<ROWS>(a, s);
    if (a.mask || n <= 1) return (long long)n * (ENDS + key_tiles<ROWS, KEYS>(a, s, n - 1));
    long long c = 0;
    for (int r = 0; r < n; r++) c += ENDS + key_tiles<ROWS, KEYS>(a, s, r);
    return c;
}

// A worker's parts of units, one after the other.
//   WARPS : workers of a CTA: its warps, or 1: the CTA is one;  LEAST : a worker's share, at least, in key tiles
template <int ROWS, int KEYS, int ENDS, int THREADS, int WARPS = 1, int LEAST = 1>
struct Deal {
    long long at, end, total;                    // cost position, of the share's end, of all work
    int b, head, tile;                           // sequence, key head, row tile
    Seq s;
    int tiles;                                   // key tiles of the unit
    long long unit;                              // where the unit begins
    int per_cta;                                 // workers of a CTA that have work: fewer where there is little of it

    static constexpr int kSums = THREADS / 32 + 3 * WARPS;       // long longs of shared memory that begin() needs

    // (total < 2^51: cells of a sequence < 2^30, rows of the batch <= 2^30.)
    __device__ __forceinline__ unsigned workers() const { return (unsigned)min((long long)gridDim.x * per_cta, total); }
    __device__ __forceinline__ long long share_of(unsigned worker) const
    {
        const unsigned n = workers();
        if (worker >= n) return total;
        if (total < 1 << 20) return (unsigned)total * worker / n;                // (n < 2^12; dividing 64 bits takes five times as long)
        return (long long)((unsigned long long)total * worker / n);
    }

    // All threads of the CTA.  False: nothing to do for this worker.
    __device__ __forceinline__ bool begin(const AttnArgs& a, long long* sums)
    {
        constexpr int W = THREADS / 32;
        const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
        long long base = 0;
        total = 0;
        per_cta = 1;
        const auto found = [&](long long excl, long long c, int seq) {           // of the sequence at [excl, excl + c): the workers that begin in it
            for (int j = 0; j < per_cta; j++) {
                const long long from = sums[W + 2 * WARPS + j];
                if (from >= excl && from < excl + c) {
                    sums[W + 2 * j] = seq;
                    sums[W + 2 * j + 1] = excl;
                }
            }
        };
        const auto known = [&](long long all) {
            total = all;
            per_cta = (int)min((long long)WARPS, max(1ll, all / ((long long)LEAST * gridDim.x)));
            if (tid < per_cta) sums[W + 2 * WARPS + tid] = share_of(blockIdx.x * per_cta + tid);
            __syncthreads();
        };
        for (int pass = 0; pass < 2; pass++) {
            base = 0;
            for (int b0 = 0; b0 < a.n_seqs; b0 += THREADS) {
                long long c = 0;
                if (b0 + tid < a.n_seqs) {
                    const Seq q(a, b0 + tid);
                    c = q.fresh > 0 ? a.kv_heads * head_cost<ROWS, KEYS, ENDS>(a, q) : 0;
                }
                long long in = c;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const long long up = __shfl_up_sync(0xffffffffu, in, o);
                    if (lane >= o) in += up;
                }
                __syncthreads();
                if (lane == 31) sums[warp] = in;
                __syncthreads();
                long long before = 0, all = 0;
#pragma unroll
                for (int w = 0; w < W; w++) {
                    if (w < warp) before += sums[w];
                    all += sums[w];
                }
                if (a.n_seqs <= THREADS) {       // one look is enough
                    known(all);
                    pass = 1;
                }
                if (pass == 1 && c > 0) found(base + before + in - c, c, b0 + tid);
                base += all;
            }
            if (pass == 0) known(base);
        }
        __syncthreads();
        const int mine = WARPS > 1 ? warp : 0;
        if (mine >= per_cta) return false;
        at = sums[W + 2 * WARPS + mine];
        end = share_of(blockIdx.x * per_cta + mine + 1);
        if (at >= end) return false;
        b = (int)sums[W + 2 * mine];
        s = Seq(a, b);
        unit = sums[W + 2 * mine + 1];
        const long long hc = head_cost<ROWS, KEYS, ENDS>(a, s);
        head = (int)((at - unit) / hc);
        unit += head * hc;
        tile = 0;
        tiles = key_tiles<ROWS, KEYS>(a, s, 0);
        while (at >= unit + ENDS + tiles) {
            unit += ENDS + tiles;
            tile++;
            tiles = key_tiles<ROWS, KEYS>(a, s, tile);
        }
        return true;
    }
    // Key tiles [t0, t1) of the unit are this worker's.  Its outputs are, if `whole`; else a part is left in scratch.
    __device__ __forceinline__ int t0() const { return (int)max(0ll, at - unit - ENDS); }
    __device__ __forceinline__ int t1() const { return (int)max(0ll, min(end - unit, (long long)ENDS + tiles) - ENDS); }
    __device__ __forceinline__ bool any() const { return t1() > t0() || (tiles == 0 && at == unit); }
    __device__ __forceinline__ bool whole() const { return t0() == 0 && t1() == tiles; }
    // CTAs behind this one that hold the unit's other parts
    __device__ __forceinline__ int others() const
    {
        const long long last = unit + ENDS + tiles - 1;     // the last cost position of the unit
        // the worker whose share holds it: share_of(c) <= last < share_of(c + 1)
        long long c = (long long)((double)last * workers() / (double)total);
        while (share_of((unsigned)c + 1) <= last) c++;
        while (share_of((unsigned)c) > last) c--;
        return (int)c / per_cta - (int)blockIdx.x;
    }
    __device__ __forceinline__ bool next(const AttnArgs& a)
    {
        unit += ENDS + tiles;
        at = unit;
        if (at >= end) return false;
        if (++tile >= row_tiles<ROWS>(a, s)) {
            tile = 0;
            if (++head >= a.kv_heads) {
                head = 0;
                do {
                    if (++b >= a.n_seqs) return false;
                    s = Seq(a, b);
                } while (s.fresh <= 0);
            }
        }
        tiles = key_tiles<ROWS, KEYS>(a, s, tile);
        return true;
    }
};

__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool there)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

template <class T>
__device__ __forceinline__ uint32_t pack2(float x, float y)
{
    if constexpr (std::is_same<T, __half>::value) {
        const __half2 h = __floats2half2_rn(x, y);
        return *reinterpret_cast<const uint32_t*>(&h);
    } else {
        const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
}
__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Does new token `t` (its row of bits: `row` of the batch) see cell `cell` of its sequence?
__device__ __forceinline__ bool sees(const AttnArgs& a, const Seq& s, int t, int row, int cell)
{
    if (cell >= s.len) return false;
    const int nth = cell - s.ctx;
    if (nth < 0) return true;
    if (!a.mask) return nth <= t;
    return (nth >> 6) < a.words && (a.mask[(long long)row * a.words + (nth >> 6)] >> (nth & 63) & 1);
}

// Which of the cells cell0 .. + 31 a new token sees.
__device__ __forceinline__ uint32_t seen32(const AttnArgs& a, const Seq& s, int t, int row, int cell0)
{
    const int left = s.len - cell0;
    uint32_t in = left >= 32 ? 0xffffffffu : left <= 0 ? 0u : (1u << left) - 1;
    const int nth = cell0 - s.ctx;               // new token of the first
    if (nth <= -32) return in;
    if (!a.mask) {
        const int n = t + 1 - nth;               // cells seen from the first on
        return in & (n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1);
    }
    const uint64_t* bits = a.mask + (long long)row * a.words;
    const int from = max(nth, 0), w = from >> 6, shift = from & 63;
    uint64_t v = w < a.words ? bits[w] >> shift : 0;
    if (shift > 32 && w + 1 < a.words) v |= bits[w + 1] << (64 - shift);
    uint32_t b = (uint32_t)v;
    if (nth < 0) b = b << -nth | ((1u << -nth) - 1);
    return in & b;
}

// Offset (in values) of a cell's row in the cache, or -1 (recorded) where its block is not one.
__device__ __forceinline__ long long cell_place(const AttnArgs& a, int b, int cell)
{
    const int nth = cell / a.block_size, block = a.table[b * a.ld + nth];
    if ((unsigned)block >= (unsigned)a.blocks) {
        atomicCAS(a.status, 0, FQ_ERR_INDEX);
        return -1;
    }
    return block * a.block_stride + (cell - nth * a.block_size) * a.cell_stride;
}

template <class T> __device__ __forceinline__ bool finite16(uint32_t two);       // both of two 16-bit values
template <> __device__ __forceinline__ bool finite16<__nv_bfloat16>(uint32_t v) { return (v & 0x7f80u) != 0x7f80u && (v & 0x7f800000u) != 0x7f800000u; }
template <> __device__ __forceinline__ bool finite16<__half>(uint32_t v) { return (v & 0x7c00u) != 0x7c00u && (v & 0x7c000000u) != 0x7c000000u; }

// Infinities and NaNs among values that not all rows of a unit see are taken out before the product, where a weight of 0 would spread them to rows that do
// not see them.  The cells that had any are noted, a bit each, from the first cell on that not all rows see; once a unit's values are written, a row gets
// back what is in those that it sees.  (Tree bits reach kOddCells new tokens; without them a unit ends, with its last row and key tile, well before
// that.  Looking through all new cells instead took 10 ms for one infinity among 2000 new tokens of 4 heads, which take 43 us without it.)
constexpr int kOddWords = 2 * FQ_MAX_TREE_WORDS, kOddCells = 32 * kOddWords;
static_assert(kOddWords == 32, "a word a lane clears them");

// Zeros in place of infinities and NaNs; true if there were any.
template <class T>
__device__ __forceinline__ bool take_out(uint4& v)
{
    uint32_t w[4] = {v.x, v.y, v.z, v.w};
    bool any = false;
#pragma unroll
    for (int j = 0; j < 4; j++) {
        any |= !finite16<T>(w[j]);
        w[j] = (finite16<T>(w[j] & 0xffffu) ? w[j] & 0xffffu : 0u) | (finite16<T>(w[j] & 0xffff0000u) ? w[j] & 0xffff0000u : 0u);
    }
    v = make_uint4(w[0], w[1], w[2], w[3]);
    return any;
}
// All lanes: `mine`: this lane's piece had some.  UNITS lanes in a row hold a cell's pieces: cell `nth` from the first one that is noted on.
template <int UNITS>
__device__ __forceinline__ bool note_odd(uint32_t* words, bool mine, int nth)
{
    const uint32_t who = __ballot_sync(0xffffffffu, mine), lane = threadIdx.x & 31;
    if (lane % UNITS == 0 && (who >> lane & (UNITS == 32 ? 0xffffffffu : (1u << (UNITS & 31)) - 1)) && nth < kOddCells) atomicOr(words + (nth >> 5), 1u << (nth & 31));
    return who != 0;
}
// What the noted cells, from cell `first` on, add to the values of new token t, a lane's row (`real`: it has one): add(d, infinity or NaN).  A lane looks
// through 32 values of a cell and hands what it finds to the lanes whose row sees that cell, so that 32 cells are on their way at a time.  (Each lane by itself, cell after cell: prompts
// of up to 2048 tokens of which one value in each head is infinite took 6.8 ms, those of NaNs 1.4.)
template <class T, class Add>
__device__ __forceinline__ void give_back(const AttnArgs& a, const Seq& s, int b, int head, int t, bool real, int first, const volatile uint32_t* words, Add add)
{
    const int lane = threadIdx.x & 31;
#pragma unroll 1
    for (int d0 = 0; d0 < a.head_dim; d0 += 32) {
        const int there = min(32, a.head_dim - d0);
        const uint32_t all = there == 32 ? 0xffffffffu : (1u << there) - 1;
        uint32_t up = 0, down = 0;               // +inf or NaN, -inf or NaN: both are a NaN, which nothing changes any more
#pragma unroll 1
        for (int i = 0; i < kOddWords; i++) {
            const uint32_t noted = __shfl_sync(0xffffffffu, words[i], 0);
            if (!noted) continue;
            const uint32_t seen = real && (up & down) != all ? noted & seen32(a, s, t, s.row0 + t, first + i * 32) : 0;
            if (!__any_sync(0xffffffffu, seen != 0)) continue;
            uint32_t here_up = 0, here_down = 0;
            const long long place = noted >> lane & 1 ? cell_place(a, b, first + i * 32 + lane) : -1;
            if (place >= 0) {
                const T* v = static_cast<const T*>(a.v) + place + head * a.head_stride + d0;
                uint4 x[4];
#pragma unroll
                for (int u = 0; u < 4; u++) x[u] = 8 * u < there ? *reinterpret_cast<const uint4*>(v + 8 * u) : make_uint4(0, 0, 0, 0);
#pragma unroll
                for (int u = 0; u < 4; u++) {
                    const uint32_t w[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
#pragma unroll
                    for (int e = 0; e < 8; e++) {
                        const uint32_t h = w[e / 2] >> 16 * (e & 1) & 0xffffu;
                        const bool odd = !finite16<T>(h), nan = h & (std::is_same<T, __half>::value ? 0x3ffu : 0x7fu), minus = h & 0x8000u;
                        here_up |= (uint32_t)(odd && (nan || !minus)) << (8 * u + e);
                        here_down |= (uint32_t)(odd && (nan || minus)) << (8 * u + e);
                    }
                }
            }
            for (uint32_t left = __ballot_sync(0xffffffffu, here_up | here_down); left; left &= left - 1) {
                const int j = __ffs((int)left) - 1;
                const uint32_t u = __shfl_sync(0xffffffffu, here_up, j), n = __shfl_sync(0xffffffffu, here_down, j);
                if (seen >> j & 1) {
                    up |= u;
                    down |= n;
                }
            }
        }
        for (uint32_t left = up | down; left; left &= left - 1) {
            const int d = __ffs((int)left) - 1;
            add(d0 + d, (up & down) >> d & 1 ? NAN : up >> d & 1 ? INFINITY : -INFINITY);
        }
        __syncwarp();
    }
}

// rows: 128 or 256 to a unit; dp: head_dim rounded up to 64, 128 or 256 (128 rows alone)
int launch_attention_tc(const fq_ctx* ctx, const AttnArgs& a, int dtype, int rows, int dp, cudaStream_t st);

}  // namespace fq
