// The bookkeeping of paged caches on the GPU: blocks go back to and come from a free list, every new token gets a slot, a position and, in a
// drafted tree, the bits of what it sees; and the accepted branch of a tree is moved together.
//
// fq_cache_step is a chain of short phases that depend on one another through exclusive sums over the sequences, so its time is latency.  One cluster does
// it: every CTA forms the sums for itself, each phase's writes are dealt to all of them, and a cluster barrier stands between phases.  The rows of
// a large batch, which depend on nothing but the new tables, are a kernel of their own over all SMs (150 thousand rows, 300 sequences: 41 us by the
// cluster).
#include <algorithm>
#include <functional>
#include <memory>
#include <new>

#include "fq_cluster.cuh"
#include "fq_internal.cuh"
#include "fq_rowtypes.cuh"

namespace fq {
namespace {

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxCluster = 8;

struct StepArgs {
    int n_seqs, max_blocks, block_size;
    int* lens;
    const int* keep;
    const int* fresh;
    int* table;
    long long ld;
    int* free_blocks;
    int free_room;
    int* free_count;
    const int* parents;
    int tokens;
    int* starts;
    long long* slots;
    int* positions;
    uint64_t* mask;
    int words;
    int n_cta;
    int rows_here;                               // the cluster writes the rows too
    int* status;
};

struct Three { int back, take, rows; };
__device__ __forceinline__ Three operator+(Three a, Three b) { return {a.back + b.back, a.take + b.take, a.rows + b.rows}; }

// Exclusive sums over the CTA's threads; `all` gets the whole CTA's.
__device__ __forceinline__ Three block_sums(Three v, Three& all, Three* warp_sums)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    Three in = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const Three up{__shfl_up_sync(0xffffffffu, in.back, o), __shfl_up_sync(0xffffffffu, in.take, o), __shfl_up_sync(0xffffffffu, in.rows, o)};
        if (lane >= o) in = in + up;
    }
    __syncthreads();
    if (lane == 31) warp_sums[warp] = in;
    __syncthreads();
    Three before{0, 0, 0};
    all = {0, 0, 0};
#pragma unroll
    for (int w = 0; w < kWarps; w++) {
        const Three s = warp_sums[w];
        if (w < warp) before = before + s;
        all = all + s;
    }
    return {before.back + in.back - v.back, before.take + in.take - v.take, before.rows + in.rows - v.rows};
}

__device__ __forceinline__ void phase_end(int n_cta)
{
    if (n_cta > 1) {
        cluster_arrive();
        cluster_wait();
    } else {
        __syncthreads();
    }
}

// Row t of the batch: slot, position, and in a drafted tree what it sees.  starts[n_seqs]: first rows of the sequences;  rows: of all new tokens.  What
// was kept of a sequence is told from its new length: `keep` may be the array of the lengths, which has these by now.
__device__ __forceinline__ void token_row(const StepArgs& a, const int* starts, int t, int rows)
{
    uint64_t* bits = a.parents ? a.mask + (long long)t * a.words : nullptr;
    if (t >= rows) {
        a.slots[t] = -1;
        a.positions[t] = 0;
        if (bits)
            for (int w = 0; w < a.words; w++) bits[w] = 0;
        return;
    }
    int lo = 0, hi = a.n_seqs - 1;               // the last sequence that starts at or before this row
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (starts[mid] <= t) lo = mid;
        else hi = mid - 1;
    }
    const int keep = __ldcg(a.lens + lo) - ((lo + 1 < a.n_seqs ? starts[lo + 1] : rows) - starts[lo]);
    const int i = t - starts[lo], cell = keep + i, block = cell / a.block_size;
    a.slots[t] = (long long)__ldcg(a.table + lo * a.ld + block) * a.block_size + (cell - block * a.block_size);
    if (!bits) {
        a.positions[t] = cell;
        return;
    }
    // up the branch: token numbers fall, so the words are finished one after the other
    const int* parents = a.parents + starts[lo];
    int at = i, above = 0, word = a.words - 1;
    uint64_t w = 0;
    for (;;) {
        for (; word > at / 64; word--, w = 0) bits[word] = w;
        w |= 1ull << (at & 63);
        const int p = parents[at];
        if (p >= at || p < -1) atomicCAS(a.status, 0, FQ_ERR_INDEX);
        if (p >= at || p < 0) break;
        at = p;
        above++;
    }
    for (; word >= 0; word--, w = 0) bits[word] = w;
    a.positions[t] = keep + above;
}

__global__ void __launch_bounds__(kThreads) cache_step_kernel(const StepArgs a)
{
    extern __shared__ int sums[];                // [3][n_seqs]: returned blocks, taken blocks, rows of the sequences before
    int* s_back = sums;
    int* s_take = sums + a.n_seqs;
    int* s_rows = sums + 2 * a.n_seqs;
    __shared__ Three warp_sums[kWarps];
    __shared__ int bad;                          // the call is refused, and why
    if (!a.rows_here) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");        // (the rows' kernel waits for this one's end)
    const int tid = threadIdx.x, cta = a.n_cta > 1 ? (int)cluster_rank() : 0;
    const int worker = cta * kThreads + tid, workers = a.n_cta * kThreads;
    if (tid == 0) bad = 0;
    __syncthreads();
    const int count = *a.free_count;
    long long back = 0, take = 0, rows = 0;
    for (int b0 = 0; b0 < a.n_seqs; b0 += kThreads) {
        const int b = b0 + tid;
        Three v{0, 0, 0};
        if (b < a.n_seqs) {
            const int len = a.lens[b], keep = a.keep[b], fresh = a.fresh[b];
            const long long room = (long long)a.max_blocks * a.block_size;
            int why = 0;
            if (len < 0 || keep < 0 || keep > len || fresh < 0 || len > room || (a.parents && fresh > 64 * a.words)) why = FQ_ERR_INDEX;
            else if ((long long)keep + fresh > room || fresh > a.tokens) why = FQ_ERR_BLOCKS;
            if (why) {
                atomicMin(&bad, why);
            } else {
                const int left = (keep + a.block_size - 1) / a.block_size;
                v = {(len + a.block_size - 1) / a.block_size - left, (int)(((long long)keep + fresh + a.block_size - 1) / a.block_size) - left, fresh};
            }
        }
        Three all;
        const Three before = block_sums(v, all, warp_sums);      // (512 values of at most 2^20)
        if (b < a.n_seqs) {
            s_back[b] = (int)back + before.back;
            s_take[b] = (int)take + before.take;
            s_rows[b] = (int)rows + before.rows;
        }
        back += all.back; take += all.take; rows += all.rows;
    }
    if (tid == 0) {
        if (count < 0 || count > a.free_room || count + back > a.free_room) atomicMin(&bad, FQ_ERR_INDEX);
        if (count + back - take < 0 || rows > a.tokens) atomicMin(&bad, FQ_ERR_BLOCKS);
    }
    phase_end(a.n_cta);                          // all have read the lengths, and this CTA's `bad` is known
    if (bad) {
        if (worker == 0) atomicCAS(a.status, 0, bad);
        for (int b = worker; b <= a.n_seqs; b += workers) a.starts[b] = 0;
        if (a.rows_here)
            for (int t = worker; t < a.tokens; t += workers) token_row(a, s_rows, t, 0);
        return;
    }
    const int lane = tid & 31, warps = workers / 32;
    const auto upto = [&](const int* s, long long all, int b) { return b + 1 < a.n_seqs ? s[b + 1] : (int)all; };
    // blocks go back
    for (int b = worker / 32; b < a.n_seqs; b += warps) {
        const int n = upto(s_back, back, b) - s_back[b];
        if (n == 0) continue;
        const int left = (a.keep[b] + a.block_size - 1) / a.block_size;
        for (int j = lane; j < n; j += 32) a.free_blocks[count + s_back[b] + j] = a.table[b * a.ld + left + j];
    }
    phase_end(a.n_cta);
    // blocks are taken
    const int end = count + (int)back;
    for (int b = worker / 32; b < a.n_seqs; b += warps) {
        const int gone = upto(s_back, back, b) - s_back[b], n = upto(s_take, take, b) - s_take[b];
        const int keep = a.keep[b], left = (keep + a.block_size - 1) / a.block_size;
        for (int j = lane; j < max(gone, n); j += 32) a.table[b * a.ld + left + j] = j < n ? __ldcg(a.free_blocks + end - 1 - s_take[b] - j) : -1;
        __syncwarp();                            // (`keep` may be the lengths themselves)
        if (lane == 0) {
            a.lens[b] = keep + upto(s_rows, rows, b) - s_rows[b];
            a.starts[b] = s_rows[b];
        }
    }
    if (worker == 0) {
        a.starts[a.n_seqs] = (int)rows;
        *a.free_count = end - (int)take;
    }
    if (!a.rows_here) return;
    phase_end(a.n_cta);
    for (int t = worker; t < a.tokens; t += workers) token_row(a, s_rows, t, (int)rows);
}

// The rows of a large batch, by all SMs, from what the kernel before left.
__global__ void __launch_bounds__(kThreads) cache_rows_kernel(const StepArgs a)
{
    extern __shared__ int starts[];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    for (int b = threadIdx.x; b < a.n_seqs; b += kThreads) starts[b] = a.starts[b];
    const int rows = a.starts[a.n_seqs];
    __syncthreads();
    for (int t = blockIdx.x * kThreads + threadIdx.x; t < a.tokens; t += gridDim.x * kThreads) token_row(a, starts, t, rows);
}

// ------------------------------------------------------------------------------------------------ the accepted branch
constexpr int kMoveThreads = 128;
constexpr int kMoveCaches = 128;                 // caches of a launch
constexpr int kMaxKept = 1024;

struct MoveArgs {
    void* cache[kMoveCaches];
    int n_caches;
    long long block_bytes, token_bytes, head_bytes;
    int blocks, block_size;
    int pieces, per_head;                        // 16-byte pieces of a cell, and of a head
    int n_seqs, max_blocks;
    const int* table;
    long long ld;
    const int* starts;
    const int* lens;
    const int* kept;
    long long ld_kept;
    int max_kept;
    const int* n_kept;
    int* keep;
    int* status;
};

// A thread owns one piece of a cell in one cache and moves it for token after token: cell before + i only ever takes from cells at or behind it, so what a
// thread has yet to read is never what it has written.  Eight loads at a time.  90 sequences, 64 caches, 8 heads of 128, 105 MB moved: 46 us (HBM floor 33; several
// pieces a thread, so that a CTA looks its cells up once for them: 51).
__global__ void __launch_bounds__(kMoveThreads) cache_move_kernel(const __grid_constant__ MoveArgs a)
{
    __shared__ long long from[kMaxKept], to[kMaxKept];
    __shared__ int bad;
    const int b = blockIdx.y, tid = threadIdx.x;
    if (tid == 0) bad = 0;
    __syncthreads();
    const long long rows = (long long)a.starts[b + 1] - a.starts[b], cells = a.lens[b];
    const int len = (int)cells, fresh = (int)max(0ll, min(rows, cells)), before = max(0, len - fresh);
    const int n = a.n_kept[b];
    const int* kept = a.kept + b * a.ld_kept;
    if (rows != fresh || len < 0 || len > (long long)a.max_blocks * a.block_size || n < 0 || n > a.max_kept || n > fresh) {
        if (tid == 0) {
            atomicCAS(a.status, 0, FQ_ERR_INDEX);
            if (a.keep && blockIdx.x == 0) a.keep[b] = before;
        }
        return;
    }
    const auto place = [&](int cell) -> long long {
        const int block = a.table[b * a.ld + cell / a.block_size];
        if (block < 0 || block >= a.blocks) return -1;
        return block * a.block_bytes + cell % a.block_size * a.token_bytes;
    };
    for (int i = tid; i < n; i += kMoveThreads) {
        const int k = kept[i];
        if (k < i || k >= fresh || (i > 0 && kept[i - 1] >= k)) {
            bad = 1;
        } else {
            from[i] = place(before + k);
            to[i] = k == i ? -2 : place(before + i);     // (-2: stays)
            if (from[i] < 0 || to[i] == -1) bad = 1;
        }
    }
    __syncthreads();
    if (bad && tid == 0) atomicCAS(a.status, 0, FQ_ERR_INDEX);
    if (tid == 0 && a.keep && blockIdx.x == 0) a.keep[b] = before + (bad ? 0 : n);
    if (bad) return;
    const int p = blockIdx.x * kMoveThreads + tid;
    if (p >= a.n_caches * a.pieces) return;
    const int c = p / a.pieces, piece = p - c * a.pieces, head = piece / a.per_head;
    char* base = static_cast<char*>(a.cache[c]) + head * a.head_bytes + (piece - head * a.per_head) * 16;
    for (int i0 = 0; i0 < n; i0 += 8) {
        uint4 v[8];
#pragma unroll
        for (int j = 0; j < 8; j++)
            if (i0 + j < n && to[i0 + j] >= 0) v[j] = *reinterpret_cast<const uint4*>(base + from[i0 + j]);
#pragma unroll
        for (int j = 0; j < 8; j++)
            if (i0 + j < n && to[i0 + j] >= 0) *reinterpret_cast<uint4*>(base + to[i0 + j]) = v[j];
    }
}

// Is an address among them twice?  -1: no memory to find out.  (64 of them: under a microsecond.)
int any_twice(void* const* p, int n)
{
    constexpr int kHere = 256;
    const void* here[kHere];
    std::unique_ptr<const void*[]> more(n > kHere ? new (std::nothrow) const void*[n] : nullptr);
    if (n > kHere && !more) return -1;
    const void** all = n > kHere ? more.get() : here;
    std::copy(p, p + n, all);
    std::sort(all, all + n, std::less<const void*>());
    return std::adjacent_find(all, all + n) != all + n;
}

}  // namespace

int check_table(const int* table, long long ld, int n_seqs, int max_blocks, int block_size)
{
    if (!table) return FQ_ERR_ARG;
    if (n_seqs < 1 || n_seqs > FQ_MAX_SEQS || max_blocks < 1 || max_blocks > (1 << 20) || ld < max_blocks || block_size < 1 || block_size > (1 << 16) ||
        (long long)max_blocks * block_size >= (1ll << 30))
        return FQ_ERR_SHAPE;
    return aligned(table, 4) ? FQ_OK : FQ_ERR_ALIGN;
}

}  // namespace fq

using namespace fq;

extern "C" {

int fq_cache_step(fq_ctx* ctx, const fq_cache_step_args* args, void* stream)
{
    if (!ctx || !args) return FQ_ERR_ARG;
    const fq_cache_step_args& x = *args;
    if (!x.lens_dev || !x.keep_dev || !x.new_dev || !x.free_dev || !x.free_count_dev || !x.starts_dev || !x.slots_dev || !x.positions_dev) return FQ_ERR_ARG;
    if (x.parents_dev && !x.mask_dev) return FQ_ERR_ARG;
    const int rc = check_table(x.table_dev, x.ld, x.n_seqs, x.max_blocks, x.block_size);
    if (rc != FQ_OK) return rc;
    if (x.tokens < 1 || x.tokens > FQ_MAX_ROWS || x.free_room < 1 || (x.parents_dev && (x.words < 1 || x.words > FQ_MAX_TREE_WORDS))) return FQ_ERR_SHAPE;
    if (!aligned(x.lens_dev, 4) || !aligned(x.keep_dev, 4) || !aligned(x.new_dev, 4) || !aligned(x.free_dev, 4) || !aligned(x.free_count_dev, 4) ||
        !aligned(x.parents_dev, 4) || !aligned(x.starts_dev, 4) || !aligned(x.slots_dev, 8) || !aligned(x.positions_dev, 4) || !aligned(x.mask_dev, 8))
        return FQ_ERR_ALIGN;
    const int n_seqs = x.n_seqs, tokens = x.tokens;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return FQ_ERR_CUDA;
    StepArgs a{n_seqs, x.max_blocks, x.block_size, x.lens_dev, x.keep_dev, x.new_dev, x.table_dev, x.ld, x.free_dev, x.free_room, x.free_count_dev,
               x.parents_dev, tokens, x.starts_dev, x.slots_dev, x.positions_dev, x.mask_dev, x.words, 1, tokens <= 4096, ctx->status_dev};
    if (n_seqs > 64 || tokens > 512) a.n_cta = kMaxCluster;
    const size_t smem = 3 * sizeof(int) * (size_t)n_seqs;
    if (smem > 47 * 1024) {                      // (48 KB without asking, of which the kernel's own variables take a part)
        // (a setting of the kernel on this device; asking for it again costs a microsecond, and only very large batches do)
        if (cudaFuncSetAttribute(cache_step_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 3 * (int)sizeof(int) * FQ_MAX_SEQS) != cudaSuccess ||
            cudaFuncSetAttribute(cache_rows_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(int) * FQ_MAX_SEQS) != cudaSuccess)
            return FQ_ERR_CUDA;
    }
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = (unsigned)a.n_cta; attr.val.clusterDim.y = 1; attr.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)a.n_cta); cfg.blockDim = dim3(kThreads); cfg.dynamicSmemBytes = smem; cfg.stream = (cudaStream_t)stream;
    if (a.n_cta > 1) { cfg.attrs = &attr; cfg.numAttrs = 1; }
    if (cudaLaunchKernelEx(&cfg, cache_step_kernel, a) != cudaSuccess) return FQ_ERR_CUDA;
    if (a.rows_here) return FQ_OK;
    const int ctas = (tokens + kThreads - 1) / kThreads, most = 4 * ctx->sm_count;
    cudaLaunchAttribute early{};
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3((unsigned)(ctas < most ? ctas : most)); cfg.dynamicSmemBytes = sizeof(int) * (size_t)n_seqs;
    cfg.attrs = &early; cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, cache_rows_kernel, a) == cudaSuccess ? FQ_OK : FQ_ERR_CUDA;
}

int fq_cache_move(fq_ctx* ctx, const fq_cache_move_args* args, void* stream)
{
    if (!ctx || !args) return FQ_ERR_ARG;
    const fq_cache_move_args& x = *args;
    const int size = type_size(x.dtype), n_caches = x.n_caches;
    if (!x.caches_host || !x.starts_dev || !x.lens_dev || !x.kept_dev || !x.n_kept_dev || !x.keep_dev || !size) return FQ_ERR_ARG;
    if (n_caches < 1 || n_caches > (1 << 16) || x.head_dim < 1 || x.head_dim > 1024 || x.max_kept < 1 || x.max_kept > kMaxKept || x.ld_kept < x.max_kept)
        return FQ_ERR_SHAPE;
    int rc = check_table(x.table_dev, x.ld, x.n_seqs, x.max_blocks, x.layout.block_size);
    for (int i = 0; i < n_caches && rc == FQ_OK; i++) {
        fq_cache c = x.layout;
        c.k_dev = c.v_dev = x.caches_host[i];
        rc = check_cache(&c, x.dtype, x.head_dim);
    }
    if (rc != FQ_OK) return rc;
    if (!aligned(x.starts_dev, 4) || !aligned(x.lens_dev, 4) || !aligned(x.kept_dev, 4) || !aligned(x.n_kept_dev, 4) || !aligned(x.keep_dev, 4))
        return FQ_ERR_ALIGN;
    for (const int* read : {x.starts_dev, x.lens_dev, x.kept_dev, x.n_kept_dev, x.table_dev})    // (while other CTAs write keep)
        if (read == x.keep_dev) return FQ_ERR_ARG;
    const int twice = any_twice(x.caches_host, n_caches);
    if (twice) return twice < 0 ? FQ_ERR_CUDA : FQ_ERR_ARG;
    const fq_cache* layout = &x.layout;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return FQ_ERR_CUDA;
    MoveArgs a{};
    a.block_bytes = layout->blocks > 1 ? layout->block_stride * size : 0;
    a.token_bytes = layout->block_size > 1 ? layout->token_stride * size : 0;
    a.head_bytes = layout->heads > 1 ? layout->head_stride * size : 0;
    a.blocks = layout->blocks; a.block_size = layout->block_size;
    a.per_head = x.head_dim * size / 16; a.pieces = a.per_head * layout->heads;
    a.n_seqs = x.n_seqs; a.max_blocks = x.max_blocks; a.table = x.table_dev; a.ld = x.ld; a.starts = x.starts_dev; a.lens = x.lens_dev;
    a.kept = x.kept_dev; a.ld_kept = x.ld_kept; a.max_kept = x.max_kept; a.n_kept = x.n_kept_dev; a.status = ctx->status_dev;
    for (int c0 = 0; c0 < n_caches; c0 += kMoveCaches) {
        a.n_caches = n_caches - c0 < kMoveCaches ? n_caches - c0 : kMoveCaches;
        for (int i = 0; i < a.n_caches; i++) a.cache[i] = x.caches_host[c0 + i];
        a.keep = c0 == 0 ? x.keep_dev : nullptr;
        // (at most 128 caches x 1024 heads x 256 pieces)
        const dim3 grid((unsigned)((a.n_caches * a.pieces + kMoveThreads - 1) / kMoveThreads), (unsigned)x.n_seqs);
        cache_move_kernel<<<grid, kMoveThreads, 0, (cudaStream_t)stream>>>(a);
        if (cudaGetLastError() != cudaSuccess) return FQ_ERR_CUDA;
    }
    return FQ_OK;
}

}  // extern "C"
