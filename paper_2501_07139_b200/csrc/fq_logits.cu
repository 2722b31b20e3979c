// What a model answers, row by row of its logits: log probabilities of given tokens with entropy and top alternatives, and
// distillation from a teacher's top logits (value and gradient).
//
// With m = max z, d_i = (z_i - m) / T and S = sum exp d_i a row needs m, S and sum exp(d_i) d_i, then a second look at a few of its entries
// for the alternatives, or at all of them for the gradient q_i = exp(d_i) / S.  What has to move is the row once in (and once out).
// Log probabilities and the loss alone read it into registers, once; value and gradient together keep it in shared memory, where the
// gradient takes its place.  Rows that are few, or too long for an SM, are cut into slices for the CTAs of a cluster (up to 8), which
// exchange (m, S, ...) and their largest entries through distributed shared memory.
//
// Rows may start anywhere.  Slices keep the alignment that the row has in global memory: 16-byte groups inside the slice are moved
// whole, the elements before the first and behind the last of them one by one, and the rest of those two groups counts as -inf,
// which no maximum and no sum sees.
//
// What bounds it: passes without alternatives and the gradient alone HBM.  Alternatives, and value and gradient, add phases that other CTAs of the
// SM cover in part: no pipe is full (exponentials 53 - 66 %, issue slots 55 - 60 % of 16-bit rows, HBM 50 - 60 %).  4094 x 32000 bf16: m, S and
// entropy 50 us, with 32 alternatives 66 us, the loss alone 48 us (a pass that only reads: 47 us); value and gradient 95 us, the
// gradient alone 79 us (a copy: 82 us).  fp32, half as many logits: 47, 57, 46, 104 and 79 us.
#include <algorithm>
#include <atomic>
#include <cmath>

#include "fq_cluster.cuh"
#include "fq_internal.cuh"
#include "fq_ptx.cuh"
#include "fq_rowtypes.cuh"

namespace fq {
namespace {

constexpr int kMaxTop = FQ_MAX_TOP;
constexpr int kCandidates = 512;
constexpr int kBatchBits = 2, kBatch = 1 << kBatchBits;       // 16-byte groups that a thread reads at a time
constexpr int kSlots = 8;                 // pieces of a thread's groups whose largest entries are kept apart
constexpr int kFewTop = 64;               // up to here 128 threads have maxima enough to bound the alternatives closely
constexpr int kBinBits = 7, kBins = 1 << kBinBits;
constexpr int kMaxCluster = 8;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kNegInf = -INFINITY;

// ------------------------------------------------------------------------------- arithmetic
__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// log2 of exp(d): the difference first, so that a row of the type's lowest values, or one far from 0, loses nothing.
__device__ __forceinline__ float2 scaled2(float2 z, float m, float c2) { return mul2(add2(z, make_float2(-m, -m)), make_float2(c2, c2)); }

// Order-preserving map of a float (with -0 as +0) onto unsigned integers, and back.
__device__ __forceinline__ uint32_t key_of(float v)
{
    const uint32_t u = __float_as_uint(v + 0.0f);
    return u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float of_key(uint32_t k) { return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xffffffffu)); }

__device__ __forceinline__ long long load_id(const void* ids, int wide, long long i)
{
    return wide ? static_cast<const long long*>(ids)[i] : (long long)static_cast<const int*>(ids)[i];
}

// ------------------------------------------------------------------------------- a slice on chip
struct RowArgs {
    const void* z;
    long long ld;
    int vocab;
    int slice;                   // entries of a CTA's slice (a multiple of a group's); CTA r of the row holds [r * slice, ...)
    int n_cta;                   // CTAs of a row
    float c2;                    // log2(e) / T
    float t;
    int* status;
    unsigned long long wait_ns;
};

struct Slice {
    int first, n;                // entries [first, first + n) of the row
    int shift;                   // entry j is element shift + j of the buffer
    int groups;                  // 16-byte groups of the buffer that hold entries
};

// The part of a row that is copied in whole groups, in elements of the buffer: [lo, hi).
template <class T>
__device__ __forceinline__ void whole_groups(const Slice& s, int& lo, int& hi)
{
    constexpr int N = Group<T>::N;
    lo = s.shift > 0 ? N : 0;
    hi = (s.shift + s.n) / N * N;
    if (hi < lo) hi = lo;
}

template <class T>
__device__ __forceinline__ Slice slice_of(const RowArgs& a, const T* row, int rank)
{
    constexpr int N = Group<T>::N;
    Slice s;
    s.first = rank * a.slice;
    s.n = a.vocab - s.first < a.slice ? a.vocab - s.first : a.slice;
    if (s.n < 0) s.n = 0;
    s.shift = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));          // the same for all slices of a row
    s.groups = s.n > 0 ? (s.shift + s.n + N - 1) / N : 0;
    return s;
}

// Starts the copies and fills the ends.  The caller synchronises the CTA, then waits for `bar`.  (A barrier for every 16 KB, so that
// sums start with the first, gains nothing.)
template <class T>
__device__ __forceinline__ void fetch_slice(const T* row, const Slice& s, uint4* buf, uint32_t bar)
{
    constexpr int N = Group<T>::N;
    constexpr int kPart = 32768;
    int lo, hi;
    whole_groups<T>(s, lo, hi);
    const T* src = row + s.first - s.shift;                              // element 0 of the buffer (a multiple of 16 bytes)
    if (threadIdx.x == 0) {
        mbar_init(bar, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        const int bytes = (hi - lo) * (int)sizeof(T);
        mbar_expect_tx(bar, (uint32_t)bytes);
        for (int b = 0; b < bytes; b += kPart)
            bulk_g2s(smem_u32(buf) + (uint32_t)(lo * (int)sizeof(T) + b), reinterpret_cast<const char*>(src + lo) + b,
                     (uint32_t)(bytes - b < kPart ? bytes - b : kPart), bar);
    }
    // the first and the last group, where they are not whole
    T* el = reinterpret_cast<T*>(buf);
    const int t = threadIdx.x - 32, end = s.shift + s.n;
    if (t >= 0 && t < 2 * N && s.n > 0) {
        const int e = t < N ? t : (end / N) * N + (t - N);
        const bool loose = t < N ? s.shift > 0 : (end % N != 0 && !(s.shift > 0 && end < N));
        if (loose) el[e] = e >= s.shift && e < end ? src[e] : Group<T>::from_f(kNegInf);
    }
}

__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

struct RowSums { float m, s, s1; };       // maximum, sum of exp(d), sum of exp(d) * log2(exp(d)); of a slice, then of the row

struct RowShared {
    unsigned long long bar;
    RowSums sums;                         // of this CTA's slice, read by the others
    float4 warp[16];                      // the warps' sums, and the least of their threads' keys
    int failed;
};

// `part`, which is against its own maximum, added to `r` against `r.m`, the larger one.
__device__ __forceinline__ void add_part(RowSums& r, const RowSums& part, float c2)
{
    if (part.s == 0.0f) return;                                  // nothing but -inf (NaN goes on)
    const float t = part.m == r.m ? 0.0f : (part.m - r.m) * c2, f = ex2(t);
    r.s += f * part.s;
    if (f > 0.0f) r.s1 += f * (part.s1 + part.s * t);
}

// Sums of the slice, from its first THREADS threads, in every thread; `least` is the smallest of the threads' keys (of those that have an entry).
template <int THREADS, bool ENTROPY>
__device__ __forceinline__ RowSums slice_sums(const RowSums& mine, uint32_t my_key, float c2, RowShared& sh, uint32_t& least)
{
    // (a thread without entries, or whose entries are all NaN, has m = -inf; its sum, 0 or NaN, counts as it is)
    const uint32_t key = __reduce_max_sync(0xffffffffu, my_key);
    RowSums w{key ? of_key(key) : kNegInf, 0.0f, 0.0f};
    add_part(w, mine, c2);
    w.s = warp_sum(w.s);
    if (ENTROPY) w.s1 = warp_sum(w.s1);
    const uint32_t low = __reduce_min_sync(0xffffffffu, my_key ? my_key : 0xffffffffu);
    if ((threadIdx.x & 31) == 0 && threadIdx.x < THREADS) sh.warp[threadIdx.x >> 5] = make_float4(w.m, w.s, w.s1, __uint_as_float(low));
    __syncthreads();
    // every warp adds the warps' up, one to a lane
    const int lane = threadIdx.x & ((THREADS / 32) - 1);
    const float4 v = sh.warp[lane];
    RowSums r{v.x, 0.0f, 0.0f};
    least = __float_as_uint(v.w);
#pragma unroll
    for (int o = 1; o < (THREADS / 32); o <<= 1) {
        r.m = fmaxf(r.m, __shfl_xor_sync(0xffffffffu, r.m, o));
        least = min(least, __shfl_xor_sync(0xffffffffu, least, o));
    }
    add_part(r, RowSums{v.x, v.y, v.z}, c2);
#pragma unroll
    for (int o = 1; o < (THREADS / 32); o <<= 1) {
        r.s += __shfl_xor_sync(0xffffffffu, r.s, o);
        if (ENTROPY) r.s1 += __shfl_xor_sync(0xffffffffu, r.s1, o);
    }
    return r;
}

// Sums of the row from those of its slices.  All threads of all CTAs; every CTA's `sums` is written before.
__device__ __forceinline__ RowSums join(const RowShared& sh, int n_cta, float c2)
{
    const uint32_t at = smem_u32(&sh.sums);
    RowSums part[kMaxCluster], r{kNegInf, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < kMaxCluster; i++)
        if (i < n_cta) {
            const uint32_t there = cluster_map(at, (uint32_t)i);
            part[i] = RowSums{cluster_ld_f32(there), cluster_ld_f32(there + 4), cluster_ld_f32(there + 8)};
            r.m = fmaxf(r.m, part[i].m);
        }
#pragma unroll
    for (int i = 0; i < kMaxCluster; i++)
        if (i < n_cta) add_part(r, part[i], c2);
    return r;
}

// Waits for the slice; a wait that runs out is noted, the kernel then works on whatever the buffer holds.  (A limit below the time of
// any copy gets one look at the barrier: try_wait may stay suspended for longer.)
__device__ __forceinline__ void await_slice(RowShared& sh, const RowArgs& a)
{
    const uint32_t bar = smem_u32(&sh.bar);
    if (!(a.wait_ns < 200ull ? mbar_test_wait(bar, 0) != 0u : mbar_wait(bar, 0, a.wait_ns))) {
        atomicCAS(a.status, 0, FQ_ERR_TIMEOUT);
        sh.failed = 1;
    }
}

// ------------------------------------------------------------------------------- a slice that only passes through
// Where the entries are needed once, or a few of them again, they go from global memory into registers: without a slice in shared
// memory more CTAs fit on an SM, and those that search their rows' largest entries are hidden behind those that read.

template <class T>
__device__ __forceinline__ uint4 load_group(const T* p)
{
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}

template <class T>
struct Stream {
    const T* src;                // element 0: the 16-byte group in which the slice begins
    Slice s;
    int lo, hi;                  // whole groups [lo, hi); of the others there are at most two, one at either end
    __device__ __forceinline__ Stream(const T* row, const Slice& slice) : src(row + slice.first - slice.shift), s(slice)
    {
        whole_groups<T>(slice, lo, hi);
        lo /= Group<T>::N;
        hi /= Group<T>::N;
    }
    __device__ __forceinline__ uint4 whole(int group) const { return load_group(src + (long long)group * Group<T>::N); }
    // Group `group` if it is one of those at the ends, -inf for what is not the slice's.
    __device__ __noinline__ uint4 end(int group) const
    {
        constexpr int N = Group<T>::N;
        uint4 v;
        T* el = reinterpret_cast<T*>(&v);
        for (int i = 0; i < N; i++) {
            const int e = group * N + i;
            el[i] = e >= s.shift && e < s.shift + s.n ? src[e] : Group<T>::from_f(kNegInf);
        }
        return v;
    }
    __device__ __forceinline__ bool is_whole(int group) const { return group >= lo && group < hi; }
    __device__ __forceinline__ uint4 any(int group) const { return is_whole(group) ? whole(group) : end(group); }
};

// Running sums of a thread.
template <class T, bool ENTROPY>
struct Running {
    float m = kNegInf;
    float2 s = {0.0f, 0.0f}, s1 = {0.0f, 0.0f};

    // Returns the largest of these entries.
    template <int G>
    __device__ __forceinline__ float take(const uint4 (&v)[G], float c2)
    {
        typename Group<T>::Max best = Group<T>::lowest();
#pragma unroll
        for (int g = 0; g < G; g++) Group<T>::take_max(best, v[g]);
        const float here = Group<T>::of_max(best), higher = fmaxf(m, here);
        if (higher > m) {                                        // the sums so far are put on the new maximum
            const float t = (m - higher) * c2, f = ex2(t);       // (m = -inf: factor 0; the sums are 0 or NaN)
            if (ENTROPY) {
                if (f > 0.0f) s1 = fma2(s, make_float2(t, t), s1);
                s1 = mul2(s1, make_float2(f, f));
            }
            s = mul2(s, make_float2(f, f));
            m = higher;
        }
        const float mm = m == kNegInf ? 0.0f : m;
        // exp(d) d of a masked entry would be 0 * -inf.  Entries of two to a register are kept above a floor whose exponential is 0
        // all the same, at half the cost of doing so with the scaled differences.
        if constexpr (ENTROPY && Group<T>::N == 8) {
            const float floor2 = (Group<T>::kFloor - mm) * c2;
            if (floor2 < -160.0f && floor2 > -1e37f) {
                uint4 w[G];
#pragma unroll
                for (int g = 0; g < G; g++) w[g] = Group<T>::above_floor(v[g]);
                add<false>(w, mm, c2);
                return here;
            }
        }
        add<ENTROPY>(v, mm, c2);
        return here;
    }
    // A batch is added up before it is added to the sums: a long row takes a thread vocab / 2048 (fp32) or vocab / 4096 additions to them
    // instead of vocab / 256, which round alike where terms are (393216 equal ones: a log probability off by 13 of 2^-24 instead of 371).
    // (Pairwise within the batch: 4094 x 32000 fp16 96.0 us instead of 95.4 us, the loss alone 47.8 us instead of 47.1 us.)
    template <bool CLAMP, int G>
    __device__ __forceinline__ void add(const uint4 (&v)[G], float mm, float c2)
    {
        float2 batch, batch1;
#pragma unroll
        for (int g = 0; g < G; g++) {
            float2 f[Group<T>::N / 2];
            Group<T>::unpack(v[g], f);
#pragma unroll
            for (int p = 0; p < Group<T>::N / 2; p++) {
                float2 t = scaled2(f[p], mm, c2);
                if (CLAMP) {                                     // (exp(-160 ln 2) is 0 in 32 bits)
                    t.x = max_nan(t.x, -160.0f);
                    t.y = max_nan(t.y, -160.0f);
                }
                const float2 e = make_float2(ex2(t.x), ex2(t.y));
                batch = g + p == 0 ? e : add2(batch, e);
                if (ENTROPY) batch1 = g + p == 0 ? mul2(e, t) : fma2(e, t, batch1);
            }
        }
        s = add2(s, batch);
        if (ENTROPY) s1 = add2(s1, batch1);
    }
    __device__ __forceinline__ RowSums sums() const { return RowSums{m, s.x + s.y, ENTROPY ? s1.x + s1.y : 0.0f}; }
};

// Sums of this thread's groups of a slice on chip.
template <class T, int THREADS>
__device__ __forceinline__ RowSums kept_sums(const uint4* buf, int groups, float c2)
{
    constexpr int U = kBatch;
    Running<T, false> run;
    int i = threadIdx.x;
    for (; i + (U - 1) * THREADS < groups; i += U * THREADS) {
        uint4 v[U];
#pragma unroll
        for (int g = 0; g < U; g++) v[g] = buf[i + g * THREADS];
        run.take(v, c2);
    }
    for (; i < groups; i += THREADS) {
        const uint4 one[1] = {buf[i]};
        run.take(one, c2);
    }
    return run.sums();
}

// Sums of this thread's groups lo + thread, + THREADS ..., kBatch of them at a time; those at the ends are the first threads' of two
// warps.  largest (or NULL): [kSlots][THREADS], -inf before; gets the largest entry of the thread's batches b, b + kSlots, ... in [b].
template <class T, int THREADS, bool ENTROPY>
__device__ __forceinline__ RowSums stream_sums(const Stream<T>& x, float c2, float* largest)
{
    constexpr int U = kBatch;
    Running<T, ENTROPY> run;
    const T* at = x.src + (long long)(x.lo + (int)threadIdx.x) * Group<T>::N;
    int left = x.hi - x.lo - (int)threadIdx.x;                   // > g THREADS: there is a group g rounds on
    int slot = threadIdx.x;
    const auto keep = [&](float here) {
        if (!largest) return;
        largest[slot] = fmaxf(largest[slot], here);
        slot = slot + THREADS < kSlots * THREADS ? slot + THREADS : (int)threadIdx.x;
    };
    for (; left > (U - 1) * THREADS; left -= U * THREADS, at += U * THREADS * Group<T>::N) {
        uint4 v[U];
#pragma unroll
        for (int g = 0; g < U; g++) v[g] = load_group(at + g * THREADS * Group<T>::N);
        keep(run.take(v, c2));
    }
    uint4 v[U - 1];
#pragma unroll
    for (int g = 0; g < U - 1; g++) {
        v[g] = Group<T>::fill();
        if (left > g * THREADS) v[g] = load_group(at + g * THREADS * Group<T>::N);
    }
    if (left > (U / 2) * THREADS) {
        keep(run.take(v, c2));
    } else if (left > 0) {
        uint4 half[U / 2];
#pragma unroll
        for (int g = 0; g < U / 2; g++) half[g] = v[g];
        keep(run.take(half, c2));
    }
    const int end = threadIdx.x == 0 && x.s.groups > 0 && !x.is_whole(0) ? 0 : threadIdx.x == 32 && x.hi > 0 && x.hi < x.s.groups ? x.hi : -1;
    if (end >= 0) {
        const uint4 one[1] = {x.end(end)};
        run.take(one, c2);
    }
    return run.sums();
}

// ------------------------------------------------------------------------------- the largest entries of a slice
template <int THREADS>
struct TopShared {
    unsigned long long cand[kCandidates];     // (key, ~index): larger is earlier
    unsigned long long top[kMaxTop];
    union {
        struct {
            float largest[kSlots * THREADS];          // of some batches of a thread each; -inf before
            unsigned short piece[kSlots * THREADS];   // those that may hold a candidate
        };
        unsigned long long lists[kMaxCluster * kMaxTop];      // of all CTAs, in the first one
    };
    int bins[256];                            // the first kBins zeroed before
    int n_pieces, n_cand;                     // zeroed before
    float reach;
    int warp[THREADS / 32];
};

__device__ __forceinline__ unsigned long long entry_word(uint32_t key, int index) { return (unsigned long long)key << 32 | (0xffffffffu - (uint32_t)index); }
// Where a bin lies: those of a lane (some in a row, from the top) in different banks from the other lanes'.
__device__ __forceinline__ int bin_at(int bin) { return bin % (kBins / 32) * 32 + bin / (kBins / 32); }

// Of bins 0 .. 32 B - 1 (at(bin) says where they lie) the highest one so that it and those above it hold k, or -1; `above` gets what
// those above it hold.  A whole warp.
template <int B, class At>
__device__ __forceinline__ int bin_of_kth(const int* bins, int k, At&& at, int& above)
{
    const int lane = threadIdx.x & 31;
    int sum = 0, in_bin[B];                                            // from the top, B to a lane
#pragma unroll
    for (int i = 0; i < B; i++) {
        in_bin[i] = bins[at(32 * B - 1 - (lane * B + i))];
        sum += in_bin[i];
    }
    int upto = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += v;
    }
    const unsigned enough = __ballot_sync(0xffffffffu, upto >= k);
    if (!enough) return -1;
    int before = upto - sum, bin = 0, over = 0;
#pragma unroll
    for (int i = 0; i < B; i++) {
        if (before < k) { bin = 32 * B - 1 - (lane * B + i); over = before; }
        before += in_bin[i];
    }
    const int who = __ffs((int)enough) - 1;
    above = __shfl_sync(0xffffffffu, over, who);
    return __shfl_sync(0xffffffffu, bin, who);
}

// Too many entries reach the bound (a row of equal logits): the k-th largest key is found digit by digit, a pass over the slice each,
// then its first bearers in order of their indices.  Leaves exactly k candidates.  Needs as many finite entries as k.
template <class T, int THREADS>
__device__ __noinline__ void exact_candidates(const Stream<T>& x, int k, TopShared<THREADS>& sh)
{
    constexpr int N = Group<T>::N, U = 4;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const auto each_group = [&](auto&& fn) {                           // (some loads on their way at a time)
        for (int i = threadIdx.x; i < x.s.groups; i += U * THREADS) {
            uint4 v[U];
#pragma unroll
            for (int u = 0; u < U; u++) v[u] = i + u * THREADS < x.s.groups ? x.any(i + u * THREADS) : Group<T>::fill();
#pragma unroll 1
            for (int u = 0; u < U; u++) {
                fn(i + u * THREADS, v[0]);
                v[0] = v[1]; v[1] = v[2]; v[2] = v[3];
            }
        }
    };
    uint32_t kth = 0;
    int need = k;                                                      // of the entries whose upper digits are those of kth
    for (int d = 24; d >= 0; d -= 8) {
        if (d + 8 <= 32 - Group<T>::kKeyBits) {                        // digits that all keys of a sign share
            kth |= kth >> 31 ? 0u : 255u << d;
            continue;
        }
        __syncthreads();
        for (int i = threadIdx.x; i < 256; i += THREADS) sh.bins[i] = 0;
        __syncthreads();
        int digit = 0, run = 0;                                        // alike entries in a row are counted before they are added
        each_group([&](int, const uint4& v) {
            float2 f[N / 2];
            Group<T>::unpack(v, f);
#pragma unroll
            for (int e = 0; e < N; e++) {
                const float z = e & 1 ? f[e / 2].y : f[e / 2].x;
                const uint32_t key = key_of(z);
                if (!(z > kNegInf) || (d < 24 && (key ^ kth) >> (d + 8))) continue;
                const int now = (int)(key >> d & 255u);
                if (now != digit && run) { atomicAdd(&sh.bins[digit], run); run = 0; }
                digit = now;
                run++;
            }
        });
        if (run) atomicAdd(&sh.bins[digit], run);
        __syncthreads();
        int above = 0;
        const int bin = bin_of_kth<8>(sh.bins, need, [](int b) { return b; }, above);      // (every warp)
        kth |= (uint32_t)(bin < 0 ? 0 : bin) << d;
        need -= above;
    }
    __syncthreads();
    if (threadIdx.x == 0) sh.n_cand = 0;
    __syncthreads();
    const auto add = [&](uint32_t key, int group, int e) {
        const int at = atomicAdd(&sh.n_cand, 1);
        if (at < kCandidates) sh.cand[at] = entry_word(key, x.s.first + group * N + e - x.s.shift);
    };
    // those above it, fewer than k, in any order
    if (need < k)
        each_group([&](int group, const uint4& v) {
            float2 f[N / 2];
            Group<T>::unpack(v, f);
#pragma unroll
            for (int e = 0; e < N; e++) {
                const float z = e & 1 ? f[e / 2].y : f[e / 2].x;
                if (z > kNegInf && key_of(z) > kth) add(key_of(z), group, e);
            }
        });
    // its bearers, in order, until there are enough
    for (int i0 = 0, taken = 0; i0 < x.s.groups && taken < need; i0 += THREADS) {
        const int i = i0 + threadIdx.x;
        unsigned bearers = 0;
        if (i < x.s.groups) {
            float2 f[N / 2];
            Group<T>::unpack(x.any(i), f);
#pragma unroll
            for (int e = 0; e < N; e++) {
                const float z = e & 1 ? f[e / 2].y : f[e / 2].x;
                if (z > kNegInf && key_of(z) == kth) bearers |= 1u << e;
            }
        }
        int upto = __popc(bearers);
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int n = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += n;
        }
        if (lane == 31) sh.warp[warp] = upto;
        __syncthreads();
        int before = taken, all = 0;
        for (int w = 0; w < THREADS / 32; w++) {
            if (w < warp) before += sh.warp[w];
            all += sh.warp[w];
        }
        before += upto - __popc(bearers);
        for (; bearers; bearers &= bearers - 1, before++)
            if (before < need) add(kth, i, __ffs((int)bearers) - 1);
        taken += all;
        __syncthreads();
    }
    __syncthreads();
}

// Calls place(rank, word) for the k largest entries, once each, and returns how many there are (fewer than k if the slice has no more).
//   The threads' own maxima bound the k-th largest entry from below, k of them being entries.  A histogram of them over
//   [least, most] gives a bound within 1/128 of that range; what reaches it, usually a few more entries than k, is found in two steps
//   that each deal the little there is to do to all threads: the batches whose maximum does, then the entries of their groups (read
//   once more, from the L2 as a rule).  Then they are ordered by counting.
template <class T, int THREADS, class Fn>
__device__ __forceinline__ int slice_top(const Stream<T>& x, int k, uint32_t my_key, uint32_t least, uint32_t most, TopShared<THREADS>& sh, Fn&& place)
{
    constexpr int N = Group<T>::N;
    const int span = 32 - __clz((int)(most - least)), shift = span > kBinBits ? span - kBinBits : 0;
    if (my_key) atomicAdd(&sh.bins[bin_at((int)((my_key - least) >> shift))], 1);
    __syncthreads();
    if (threadIdx.x < 32) {
        int above;
        const int bin = bin_of_kth<kBins / 32>(sh.bins, k, [](int b) { return bin_at(b); }, above);
        // (fewer than k threads have an entry: the lowest finite value)
        if (threadIdx.x == 0) sh.reach = of_key(bin < 0 ? 0x00800000u : least + ((uint32_t)bin << shift));
    }
    __syncthreads();
    const float reach = sh.reach;                                      // (compared as a number, not met by -inf or NaN)
#pragma unroll
    for (int i = 0; i < kSlots; i++)
        if (sh.largest[i * THREADS + threadIdx.x] >= reach) sh.piece[atomicAdd(&sh.n_pieces, 1)] = (unsigned short)(i * THREADS + threadIdx.x);
    __syncthreads();
    // a piece is up to 2^bits groups: kBatch of every kSlots-th batch
    const int rounds = (x.hi - x.lo + THREADS - 1) / THREADS, turns = (rounds + kSlots * kBatch - 1) / (kSlots * kBatch);
    const int bits = kBatchBits + (turns > 1 ? 32 - __clz(turns - 1) : 0), items = sh.n_pieces << bits;
    for (int i = threadIdx.x; i < items + 2; i += THREADS) {           // and the two groups at the ends
        if (*const_cast<volatile int*>(&sh.n_cand) > kCandidates) break;
        int group;
        if (i < items) {
            const int piece = sh.piece[i >> bits], part = i & ((1 << bits) - 1);
            group = x.lo + piece % THREADS + ((part >> kBatchBits) * kSlots + piece / THREADS) * kBatch * THREADS + (part & (kBatch - 1)) * THREADS;
            if (group >= x.hi) continue;
        } else {
            group = i == items ? 0 : x.s.groups - 1;
            if (x.s.groups == 0 || x.is_whole(group) || (i > items && group == 0)) continue;
        }
        const uint4 v = i < items ? x.whole(group) : x.end(group);
        float2 f[N / 2];
        Group<T>::unpack(v, f);
        unsigned found = 0;
#pragma unroll
        for (int e = 0; e < N; e++) found |= (e & 1 ? f[e / 2].y : f[e / 2].x) >= reach ? 1u << e : 0u;
        for (; found; found &= found - 1) {
            const int e = __ffs((int)found) - 1, at = atomicAdd(&sh.n_cand, 1);
            float z = f[0].x;
#pragma unroll
            for (int j = 1; j < N; j++) z = j == e ? (j & 1 ? f[j / 2].y : f[j / 2].x) : z;
            if (at < kCandidates) sh.cand[at] = entry_word(key_of(z), x.s.first + group * N + e - x.s.shift);
        }
    }
    __syncthreads();
    int n = sh.n_cand;
    if (n > kCandidates) {
        exact_candidates<T, THREADS>(x, k, sh);
        n = sh.n_cand;
    }
    for (int c = threadIdx.x; c < n; c += THREADS) {
        const unsigned long long w = sh.cand[c];
        int rank = 0;
#pragma unroll 8
        for (int j = 0; j < n; j++) rank += sh.cand[j] > w;
        if (rank < k) place(rank, w);
    }
    return n < k ? n : k;
}

// ------------------------------------------------------------------------------- log probabilities
struct LogprobArgs {
    const void* tokens;
    int wide;
    float* logprob;
    float* entropy;
    int n_top;
    int* top_ids;
    float* top_logprobs;
};

template <int THREADS>
__device__ __forceinline__ int block_sum(int mine, int* words)
{
    const int w = __reduce_add_sync(0xffffffffu, mine);
    if ((threadIdx.x & 31) == 0) words[threadIdx.x >> 5] = w;
    __syncthreads();
    int all = 0;
#pragma unroll
    for (int i = 0; i < THREADS / 32; i++) all += words[i];
    return all;
}

// What a row's sums make of its entries.
struct RowAnswer {
    float zm, log_s, t;
    bool nan;
    __device__ __forceinline__ RowAnswer(const RowSums& sum, float temperature)
        : zm(sum.m == kNegInf ? 0.0f : sum.m), log_s(sum.s == 0.0f ? 0.0f : logf(sum.s)), t(temperature), nan(sum.s != sum.s) {}
    __device__ __forceinline__ float logprob(float z) const { return (z - zm) / t - log_s; }
    __device__ __forceinline__ void put(const LogprobArgs& o, long long r, int vocab, long long token, float z, const RowSums& sum) const
    {
        o.logprob[r] = token < 0 ? 0.0f : token >= vocab || nan ? NAN : logprob(z);
        o.entropy[r] = sum.s == 0.0f ? 0.0f : log_s - kLn2 * (sum.s1 / sum.s);
    }
    __device__ __forceinline__ void put_top(const LogprobArgs& o, long long r, int place, unsigned long long w) const
    {
        if (nan) return put_none(o, r, place);
        o.top_ids[r * o.n_top + place] = (int)(0xffffffffu - (uint32_t)w);
        o.top_logprobs[r * o.n_top + place] = logprob(of_key((uint32_t)(w >> 32)));
    }
    __device__ __forceinline__ void put_none(const LogprobArgs& o, long long r, int place) const
    {
        o.top_ids[r * o.n_top + place] = -1;
        o.top_logprobs[r * o.n_top + place] = nan ? NAN : kNegInf;
    }
};

// A CTA to a row, or to a slice of one.  128 threads a row: with 256, and their barriers, 4094 x 32000 bf16 takes 73 us instead of 66 us; more than 64
// alternatives need the closer bound of 256 threads' maxima.  One row of 32000 and 20 alternatives: 7.6 us, a chain of launch, loads, seven barriers
// and the exchange between four CTAs.
template <class T, int THREADS>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) token_logprobs_kernel(const RowArgs a, const LogprobArgs o)
{
    __shared__ RowShared sh;
    __shared__ TopShared<THREADS> top;
    const int rank = a.n_cta > 1 ? (int)cluster_rank() : 0;
    const long long r = blockIdx.x / a.n_cta;
    const T* row = static_cast<const T*>(a.z) + r * a.ld;
    const Stream<T> x(row, slice_of<T>(a, row, rank));
    // the last warp asks for the token, and for its logit at the end
    const bool scalar = rank == 0 && threadIdx.x == THREADS - 32;
    const long long token = scalar ? load_id(o.tokens, o.wide, r) : -1;
    for (int i = threadIdx.x; i < kBins; i += THREADS) top.bins[i] = 0;
    if (threadIdx.x == THREADS - 1) top.n_pieces = top.n_cand = 0;
    if (o.n_top > 0)
#pragma unroll
        for (int i = 0; i < kSlots; i++) top.largest[i * THREADS + threadIdx.x] = kNegInf;
    const RowSums mine = stream_sums<T, THREADS, true>(x, a.c2, o.n_top > 0 ? top.largest : nullptr);
    const float z_token = token >= 0 && token < a.vocab ? Group<T>::to_f(row[token]) : 0.0f;
    const uint32_t my_key = mine.m > kNegInf ? key_of(mine.m) : 0u;
    uint32_t least;
    RowSums sum = slice_sums<THREADS, true>(mine, my_key, a.c2, sh, least);
    const uint32_t most = sum.m > kNegInf ? key_of(sum.m) : 0u;
    if (least > most) least = most;                              // (no thread has an entry)
    if (a.n_cta == 1) {
        const RowAnswer ans(sum, a.t);
        if (scalar) ans.put(o, r, a.vocab, token, z_token, sum);
        if (o.n_top > 0) {
            const int n = slice_top<T, THREADS>(x, o.n_top, my_key, least, most, top, [&](int place, unsigned long long w) { ans.put_top(o, r, place, w); });
            for (int j = n + threadIdx.x; j < o.n_top; j += THREADS) ans.put_none(o, r, j);
        }
        return;
    }
    const int k = o.n_top;
    if (k > 0) {                                                 // (0 where there are fewer: smaller than any entry's word)
        const int n = slice_top<T, THREADS>(x, k, my_key, least, most, top, [&](int place, unsigned long long w) { top.top[place] = w; });
        for (int j = n + threadIdx.x; j < k; j += THREADS) top.top[j] = 0ull;
    }
    if (threadIdx.x == 0) sh.sums = sum;
    cluster_arrive();
    cluster_wait();
    if (rank == 0) {
        sum = join(sh, a.n_cta, a.c2);
        const RowAnswer ans(sum, a.t);
        if (scalar) ans.put(o, r, a.vocab, token, z_token, sum);
        // the CTAs' lists, merged: an entry's place is its own place in its list and what is larger in each of the others
        if (k > 0) {
            const uint32_t at = smem_u32(top.top);
            for (int i = threadIdx.x; i < a.n_cta * k; i += THREADS) top.lists[i] = cluster_ld_u64(cluster_map(at, (uint32_t)(i / k)) + (uint32_t)(i % k) * 8);
            __syncthreads();
            int mine_of = 0;
            for (int i = threadIdx.x; i < a.n_cta * k; i += THREADS) {
                const unsigned long long w = top.lists[i];
                if (w == 0) continue;
                mine_of++;
                int larger[kMaxCluster] = {};                    // of every list, found bit by bit, all lists side by side
#pragma unroll
                for (int step = kMaxTop; step > 0; step >>= 1) {
                    if (step > k) continue;
#pragma unroll
                    for (int d = 0; d < kMaxCluster; d++) {
                        const int to = larger[d] + step;
                        if (d < a.n_cta && to <= k && top.lists[d * k + to - 1] > w) larger[d] = to;
                    }
                }
                int place = 0;                                   // (of its own list that is its place there)
#pragma unroll
                for (int d = 0; d < kMaxCluster; d++) place += larger[d];
                if (place < k) ans.put_top(o, r, place, w);
            }
            const int total = block_sum<THREADS>(mine_of, top.warp);
            for (int j = total + threadIdx.x; j < k; j += THREADS) ans.put_none(o, r, j);
        }
    }
    cluster_arrive();                                                    // nobody's shared memory is read any more
    cluster_wait();
}

// ------------------------------------------------------------------------------- distillation
struct DistillArgs {
    const void* ids;
    int wide;
    const float* teacher;
    int k;
    const float* grad_loss;
    float* loss;
    float2* stats;               // (m, log S) of every row
    void* grad;
    long long ldg;
};

struct __align__(16) TeacherShared {
    int id[kMaxTop];                      // -1: none
    float p[kMaxTop];
    float all[kMaxTop];                   // the probability of the slot's token, in all of its slots
    int at[kMaxTop];                      // where the token is in the buffer; -1: not there, or the token of an earlier slot
    int any, bad;
    volatile int seen;
};

// The teacher's distribution over the warp's slots, kMaxTop / 32 to a lane: from logits (-inf: empty) to log probabilities, and probabilities.
// Returns whether there is one (a NaN is).
__device__ __forceinline__ bool teacher_softmax(float (&p)[kMaxTop / 32], float (&lp)[kMaxTop / 32], float c2, float t)
{
    float m = kNegInf, s = 0.0f;
#pragma unroll
    for (int i = 0; i < kMaxTop / 32; i++) m = max_nan(m, lp[i]);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
    const float mm = m == kNegInf ? 0.0f : m;
#pragma unroll
    for (int i = 0; i < kMaxTop / 32; i++) {
        p[i] = ex2((lp[i] - mm) * c2);
        s += p[i];
    }
    s = warp_sum(s);
    const float inv = s == 0.0f ? 0.0f : 1.0f / s, log_s = s == 0.0f ? 0.0f : logf(s);
#pragma unroll
    for (int i = 0; i < kMaxTop / 32; i++) {
        p[i] *= inv;
        lp[i] = (lp[i] - mm) / t - log_s;
    }
    return s != 0.0f;
}

// A warp's slots, kMaxTop / 32 to a lane: ids, the teacher's logits (-inf: empty) and, if `row` is not NULL, the student's at the ids.  Those are on
// their way when the function returns: nothing waits for them before they are used.  (They are read before any gradient may overwrite them.)
template <class T>
__device__ __forceinline__ void load_slots(const DistillArgs& o, long long r, const T* row, int vocab, long long (&id)[kMaxTop / 32], float (&u)[kMaxTop / 32],
                                           T (&z)[kMaxTop / 32], bool& bad)
{
    const int lane = threadIdx.x & 31;
    bad = false;
#pragma unroll
    for (int i = 0; i < kMaxTop / 32; i++) {
        const int j = lane + 32 * i;
        id[i] = j < o.k ? load_id(o.ids, o.wide, r * o.k + j) : -1;
        u[i] = j < o.k ? o.teacher[r * o.k + j] : kNegInf;
    }
#pragma unroll
    for (int i = 0; i < kMaxTop / 32; i++) {
        z[i] = row && id[i] >= 0 && id[i] < vocab ? row[id[i]] : Group<T>::from_f(kNegInf);
        if (id[i] < 0) u[i] = kNegInf;
        bad |= id[i] >= vocab && u[i] != kNegInf;                // (an empty slot may have any id)
    }
    bad = __any_sync(0xffffffffu, bad);
}

// p (log p - log q); p times a distance that 32 bits do not hold may well be one that they do.
__device__ __forceinline__ float loss_term(float p, float lp, float z_id, float zm, float log_s, float t)
{
    return p == 0.0f ? 0.0f : p * (lp + log_s) - p * (z_id - zm) / t;
}

// The value alone: the logits pass through once (4094 x 32000 bf16 48 us, 255 x 32000 7.3 us: with 128 threads and clusters of four 10.2 us).
template <class T, int THREADS>
__global__ void __launch_bounds__(THREADS + 32, 1024 / THREADS) distill_loss_kernel(const RowArgs a, const DistillArgs o)
{
    __shared__ RowShared sh;
    constexpr int kPer = kMaxTop / 32;
    const int rank = a.n_cta > 1 ? (int)cluster_rank() : 0, lane = threadIdx.x & 31;
    const long long r = blockIdx.x / a.n_cta;
    const T* row = static_cast<const T*>(a.z) + r * a.ld;
    const bool teaches = rank == 0 && threadIdx.x >= THREADS;    // one warp more than those that see to the logits
    RowSums mine{kNegInf, 0.0f, 0.0f};
    float p[kPer], lp[kPer];
    T z_id[kPer];
    bool bad = false;
    if (teaches) {
        long long id[kPer];
        load_slots<T>(o, r, row, a.vocab, id, lp, z_id, bad);
        teacher_softmax(p, lp, a.c2, a.t);
    } else if (threadIdx.x < THREADS) {
        mine = stream_sums<T, THREADS, false>(Stream<T>(row, slice_of<T>(a, row, rank)), a.c2, nullptr);
    }
    uint32_t least;
    RowSums sum = slice_sums<THREADS, false>(mine, mine.m > kNegInf ? key_of(mine.m) : 0u, a.c2, sh, least);
    if (a.n_cta > 1) {
        if (threadIdx.x == 0) sh.sums = sum;
        cluster_arrive();
        cluster_wait();
        if (rank == 0) sum = join(sh, a.n_cta, a.c2);
        cluster_arrive();                                        // nobody's sums are read any more
    }
    if (teaches) {
        const float log_s = sum.s == 0.0f ? 0.0f : logf(sum.s), zm = sum.m == kNegInf ? 0.0f : sum.m;
        float loss = 0.0f;
#pragma unroll
        for (int i = 0; i < kPer; i++) loss += loss_term(p[i], lp[i], Group<T>::to_f(z_id[i]), zm, log_s, a.t);
        loss = warp_sum(loss);
        if (lane == 0) {
            o.loss[r] = bad ? NAN : loss;
            o.stats[r] = make_float2(sum.m, sum.s != sum.s ? NAN : log_s);
        }
    }
    if (a.n_cta > 1) cluster_wait();
}

// GIVEN: the gradient alone, from the (m, log S) that an earlier call kept; slices then need nothing from one another.
//   THREADS threads see to the logits.  One warp more sees to the teacher: its distribution, the student's logits at its tokens (two loads, one after the
// other, and a chain of dependent arithmetic that would hold the others up, 7 % of the time), and at the end the loss.  The gradient
// leaves in pieces while the next ones are formed.  Three CTAs with slices of up to 68 KB fill an SM; smaller ones in clusters lose more in the exchange than they win.
template <class T, int THREADS, bool GIVEN>
__global__ void __launch_bounds__(THREADS + 32, 1024 / THREADS) distill_kernel(const RowArgs a, const DistillArgs o)
{
    extern __shared__ __align__(16) uint4 buf[];
    __shared__ RowShared sh;
    __shared__ TeacherShared te;
    constexpr int N = Group<T>::N, kPer = kMaxTop / 32;
    const int rank = (int)(blockIdx.x % a.n_cta), warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const long long r = blockIdx.x / a.n_cta;
    const T* row = static_cast<const T*>(a.z) + r * a.ld;
    const Slice s = slice_of<T>(a, row, rank);
    const bool teaches = warp == THREADS / 32;
    if (threadIdx.x == 0) sh.failed = 0;
    fetch_slice<T>(row, s, buf, smem_u32(&sh.bar));
    const float g = o.grad_loss[r];
    const float2 given = GIVEN ? o.stats[r] : make_float2(0.0f, 0.0f);
    __syncthreads();
    RowSums mine{kNegInf, 0.0f, 0.0f};
    float p[kPer], lp[kPer];                                     // of the last warp: slots lane, lane + 32, ...
    T z_id[kPer];
    if (teaches) {
        bool bad;
        long long id[kPer];
        load_slots<T>(o, r, rank == 0 && !GIVEN ? row : nullptr, a.vocab, id, lp, z_id, bad);
        const bool some = teacher_softmax(p, lp, a.c2, a.t);
        // a token's probabilities, added up once for all of its slots
#pragma unroll
        for (int i = 0; i < kPer; i++) {
            te.id[lane + 32 * i] = id[i] >= 0 && id[i] < a.vocab ? (int)id[i] : -1;
            te.p[lane + 32 * i] = p[i];
        }
        __syncwarp();
#pragma unroll
        for (int i = 0; i < kPer; i++) {
            const int j = lane + 32 * i;
            const bool here = id[i] >= s.first && id[i] < s.first + s.n;
            int at = here ? s.shift + (int)(id[i] - s.first) : -1;
            float all = 0.0f;
            if (__any_sync(0xffffffffu, here)) {
                const int mine = here ? (int)id[i] : -2;
                for (int l = 0; l < o.k; l += 4) {
                    const int4 v = *reinterpret_cast<const int4*>(te.id + l);
                    const float4 q = *reinterpret_cast<const float4*>(te.p + l);
                    if (v.x == mine) { all += q.x; if (l < j) at = -1; }
                    if (v.y == mine) { all += q.y; if (l + 1 < j) at = -1; }
                    if (v.z == mine) { all += q.z; if (l + 2 < j) at = -1; }
                    if (v.w == mine) { all += q.w; if (l + 3 < j) at = -1; }
                }
            }
            te.at[j] = at;
            te.all[j] = all;
        }
        if (lane == 0) {
            te.any = some;
            te.bad = bad;
        }
        if (o.grad == a.z) {
            // in place: these logits have arrived before any warp's gradient leaves
            bool seen = false;
#pragma unroll
            for (int i = 0; i < kPer; i++) seen |= Group<T>::to_f(z_id[i]) > 0.0f;
            te.seen = __any_sync(0xffffffffu, seen);
        }
    } else {
        await_slice(sh, a);
        if (!GIVEN) mine = kept_sums<T, THREADS>(buf, s.groups, a.c2);
    }
    RowSums sum;
    float log_s;
    if (GIVEN) {
        sum = RowSums{given.x, 0.0f, 0.0f};
        log_s = given.y;
        __syncthreads();
    } else {
        uint32_t least;
        sum = slice_sums<THREADS, false>(mine, mine.m > kNegInf ? key_of(mine.m) : 0u, a.c2, sh, least);
        if (a.n_cta > 1) {
            if (threadIdx.x == 0) sh.sums = sum;
            cluster_arrive();
            cluster_wait();
            sum = join(sh, a.n_cta, a.c2);
            cluster_arrive();                                // this CTA has read the others' sums
        }
        log_s = sum.s == 0.0f ? 0.0f : logf(sum.s);
    }
    const float zm = sum.m == kNegInf ? 0.0f : sum.m;
    if (teaches) {
        if (!GIVEN && rank == 0) {
            float loss = 0.0f;
#pragma unroll
            for (int i = 0; i < kPer; i++) loss += loss_term(p[i], lp[i], Group<T>::to_f(z_id[i]), zm, log_s, a.t);
            loss = warp_sum(loss);
            if (lane == 0) {
                o.loss[r] = te.bad ? NAN : loss;
                o.stats[r] = make_float2(sum.m, sum.s != sum.s ? NAN : log_s);
            }
        }
    } else {
        // g (q_i - p_i) / T, formed where the logits are.  A row without a teacher, or whose upstream gradient is 0, gets zeros
        // whatever it holds.
        const bool bad = te.bad, zero = g == 0.0f || (!te.any && !bad);
        const float w = bad ? NAN : g / a.t;
        const float off = log_s * kLog2e;                    // q = 2^(t - off)
        T* dst = static_cast<T*>(o.grad) + r * o.ldg + s.first - s.shift;      // element 0 of the buffer
        const bool alike = ((reinterpret_cast<uintptr_t>(dst) ^ reinterpret_cast<uintptr_t>(row + s.first - s.shift)) & 15) == 0;
        T* el = reinterpret_cast<T*>(buf);
        int lo, hi, at[kPer];
        whole_groups<T>(s, lo, hi);
        const int end = s.shift + s.n;
#pragma unroll
        for (int i = 0; i < kPer; i++) at[i] = !zero && lane + 32 * i < o.k ? te.at[lane + 32 * i] : -1;
        // q w = +-2^(z c2 - shift).  16-bit gradients are formed like that, in one step, where the shift and its largest part are small: with
        // four roundings of at most 2^-18 it puts q off by 1.1e-5, where the gradient's own rounding is one of 2^-11 or 2^-8.
        const float reach = zm * a.c2, shift = reach + off - log2f(fabsf(w));
        const bool quick = N == 8 && fabsf(reach) < 64.0f && fabsf(shift) < 64.0f && !zero;      // (not if w is NaN or an infinity)
        const uint32_t sign = w < 0.0f ? 0x80008000u : 0u;
        // A warp takes 4 KB at a time, which leave as soon as they are done: what has been stored and what is still being formed overlap.
        constexpr int kBlock = 256;
        for (int b = warp * kBlock; b < s.groups; b += (THREADS / 32) * kBlock) {
            const int b0 = b * N, b1 = (b + kBlock) * N, e0 = max(lo, b0), e1 = min(hi, b1);
            float z[kPer];
#pragma unroll
            for (int i = 0; i < kPer; i++)
                if (32 * i < o.k) z[i] = at[i] >= b0 && at[i] < b1 ? Group<T>::to_f(el[at[i]]) : 0.0f;
            __syncwarp();
            if (quick) {
                const float2 c2 = make_float2(a.c2, a.c2), minus = make_float2(-shift, -shift);
                const auto one = [&](int group) {
                    float2 f[N / 2];
                    Group<T>::unpack(buf[group], f);
#pragma unroll
                    for (int h = 0; h < N / 2; h++) {
                        const float2 t = fma2(f[h], c2, minus);
                        f[h] = make_float2(ex2(t.x), ex2(t.y));
                    }
                    uint4 v = Group<T>::pack(f);
                    if (sign) { v.x ^= sign; v.y ^= sign; v.z ^= sign; v.w ^= sign; }
                    buf[group] = v;
                };
                if (b + kBlock <= s.groups) {
#pragma unroll 4
                    for (int i = 0; i < kBlock / 32; i++) one(b + i * 32 + lane);
                } else {
                    for (int group = b + lane; group < s.groups; group += 32) one(group);
                }
            } else {
                for (int group = b + lane; group < min(b + kBlock, s.groups); group += 32) {
                    float2 f[N / 2];
                    Group<T>::unpack(buf[group], f);
#pragma unroll
                    for (int h = 0; h < N / 2; h++) {
                        const float2 t = fma2(add2(f[h], make_float2(-zm, -zm)), make_float2(a.c2, a.c2), make_float2(-off, -off));
                        f[h] = mul2(make_float2(ex2(t.x), ex2(t.y)), make_float2(w, w));
                    }
                    buf[group] = zero ? make_uint4(0u, 0u, 0u, 0u) : Group<T>::pack(f);
                }
            }
            __syncwarp();
#pragma unroll
            for (int i = 0; i < kPer; i++)
                if (32 * i < o.k && at[i] >= b0 && at[i] < b1)
                    el[at[i]] = Group<T>::from_f((ex2((z[i] - zm) * a.c2 - off) - te.all[lane + 32 * i]) * w);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (!alike) {
                for (int e = max(b0, s.shift) + lane; e < min(b1, end); e += 32) dst[e] = el[e];
                continue;
            }
            if (lane == 0 && e1 > e0) {
                asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;"
                             ::"l"(dst + e0), "r"(smem_u32(el + e0)), "r"((e1 - e0) * (int)sizeof(T)) : "memory");
                asm volatile("cp.async.bulk.commit_group;" ::: "memory");
            }
            // the ends of the slice, where its groups are not whole
            if (b == 0 && s.shift + lane < min(lo, end)) dst[s.shift + lane] = el[s.shift + lane];
            if (hi >= b0 && hi < b1 && hi + lane < end) dst[hi + lane] = el[hi + lane];
        }
        if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
    }
    if (!GIVEN && a.n_cta > 1) cluster_wait();                   // nobody's sums are read any more
    if (sh.failed) let_copies_land();
}

// ------------------------------------------------------------------------------- host side
// How rows that stay on chip are cut.  A slice of up to 68 KB leaves room for three CTAs on an SM, so that one computes while the copies
// of the others are on their way.  Where the CTAs of a row need nothing from one another, slices of up to 36 KB leave room for four (their registers)
// and cost no exchange: the gradient alone of 4094 x 32000 bf16 takes 79.4 us against 80.5 us.  In clusters of two, value and gradient take 114 us
// against 95 us.  With few rows a row is spread over more SMs, down to slices of 8 KB.
struct Cut { int n_cta, slice; size_t smem; };
Cut cut_rows(int rows, int vocab, int size, int sm_count, bool cluster)
{
    constexpr int kLeastBytes = 8 * 1024;
    const int slice_bytes = (cluster ? 68 : 36) * 1024;
    const int n = 16 / size;
    Cut c{};
    const auto per = [&](int ctas) { return ((vocab + ctas - 1) / ctas + n - 1) / n * n; };
    c.n_cta = 1;
    while ((c.n_cta < kMaxCluster || !cluster) && per(c.n_cta) * size > slice_bytes) c.n_cta *= 2;
    while (c.n_cta < kMaxCluster && (long long)rows * c.n_cta * 2 <= sm_count && per(2 * c.n_cta) * size >= kLeastBytes) c.n_cta *= 2;
    c.slice = per(c.n_cta);
    c.smem = (size_t)c.slice * size + 32;
    return c;
}

// Threads of a CTA whose rows pass through: 128, the fewest barriers and sums for each row, as long as the rows fill the SMs with them; more where they are few.
int stream_threads(int rows, int sm_count)
{
    int t = 128;
    while (t < 512 && (long long)rows * t * 2 <= 1024ll * sm_count) t *= 2;
    return t;
}

// Rows that pass through are cut only where they are few: until the SMs have all the CTAs that they hold, down to slices of 8 KB.
Cut cut_streams(int rows, int vocab, int size, int sm_count, int threads)
{
    constexpr int kLeastBytes = 8 * 1024;
    const int n = 16 / size;
    const auto per = [&](int ctas) { return ((vocab + ctas - 1) / ctas + n - 1) / n * n; };
    Cut c{};
    c.n_cta = 1;
    while (c.n_cta < kMaxCluster && (long long)rows * c.n_cta * 2 <= 1024 / threads * sm_count && per(2 * c.n_cta) * size >= kLeastBytes) c.n_cta *= 2;
    c.slice = per(c.n_cta);
    return c;
}

// ready: of the kernels with slices on chip, for which devices they may have as much shared memory as they ask for.
template <class... Args>
int launch_rows(void (*kernel)(Args...), int threads, std::atomic<bool>* ready, const Ctx* ctx, int rows, const Cut& c, bool cluster, cudaStream_t st,
                Args... args)
{
    if (ready && ctx->device >= 64) return FQ_ERR_ARG;
    if (ready && !ready[ctx->device].load(std::memory_order_acquire)) {
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 208 * 1024) != cudaSuccess) return FQ_ERR_CUDA;
        ready[ctx->device].store(true, std::memory_order_release);
    }
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = (unsigned)c.n_cta; attr.val.clusterDim.y = 1; attr.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)rows * (unsigned)c.n_cta); cfg.blockDim = dim3((unsigned)threads); cfg.dynamicSmemBytes = c.smem;
    cfg.stream = st;
    if (cluster && c.n_cta > 1) { cfg.attrs = &attr; cfg.numAttrs = 1; }
    return cudaLaunchKernelEx(&cfg, kernel, args...) == cudaSuccess ? FQ_OK : FQ_ERR_CUDA;
}

int check_rows(const fq_ctx* ctx, const void* logits, int dtype, int rows, int vocab, long long ld, float temperature, int n_top, int id_bytes)
{
    const int size = type_size(dtype);
    if (!ctx || !logits || !size || (id_bytes != 4 && id_bytes != 8)) return FQ_ERR_ARG;
    if (!(temperature >= 1e-30f && temperature <= 1e30f)) return FQ_ERR_ARG;
    if (rows < 1 || rows > FQ_MAX_ROWS || vocab < 1 || vocab > FQ_MAX_VOCAB || ld < vocab || n_top < 0 || n_top > FQ_MAX_TOP) return FQ_ERR_SHAPE;
    if (!aligned(logits, (size_t)size)) return FQ_ERR_ALIGN;
    return FQ_OK;
}

// A gradient in place of the logits has to have their pitch: one row's gradient would overwrite another's logits.
bool other_pitch(const void* logits, long long ld, const void* grad, long long ldg, int rows) { return grad == logits && ldg != ld && rows > 1; }

RowArgs row_args(const Ctx* ctx, const void* logits, int vocab, long long ld, float temperature, const Cut& c)
{
    RowArgs a{};
    a.z = logits; a.ld = ld; a.vocab = vocab; a.slice = c.slice; a.n_cta = c.n_cta;
    a.c2 = (float)(1.4426950408889634 / (double)temperature); a.t = temperature;
    a.status = ctx->status_dev; a.wait_ns = ctx->wait_limit_ns;
    return a;
}

template <class T>
int logprobs_typed(const Ctx* ctx, int threads, int rows, const Cut& c, const RowArgs& a, const LogprobArgs& o, cudaStream_t st)
{
    if (threads == 128) return launch_rows(token_logprobs_kernel<T, 128>, 128, nullptr, ctx, rows, c, true, st, a, o);
    return launch_rows(token_logprobs_kernel<T, 256>, 256, nullptr, ctx, rows, c, true, st, a, o);
}

template <class T>
int loss_typed(const Ctx* ctx, int threads, int rows, const Cut& c, const RowArgs& a, const DistillArgs& o, cudaStream_t st)
{
    if (threads == 128) return launch_rows(distill_loss_kernel<T, 128>, 128 + 32, nullptr, ctx, rows, c, true, st, a, o);
    if (threads == 256) return launch_rows(distill_loss_kernel<T, 256>, 256 + 32, nullptr, ctx, rows, c, true, st, a, o);
    return launch_rows(distill_loss_kernel<T, 512>, 512 + 32, nullptr, ctx, rows, c, true, st, a, o);
}

template <class T, bool GIVEN>
int distill_typed(const Ctx* ctx, int rows, const Cut& c, const RowArgs& a, const DistillArgs& o, cudaStream_t st)
{
    static std::atomic<bool> ready[2][64];
    // (rows of up to 36 KB: five CTAs to an SM and more, if they have half the threads)
    if constexpr (!GIVEN) {
        if (c.smem <= 36 * 1024) return launch_rows(distill_kernel<T, 128, false>, 128 + 32, ready[0], ctx, rows, c, true, st, a, o);
    }
    return launch_rows(distill_kernel<T, 256, GIVEN>, 256 + 32, ready[1], ctx, rows, c, !GIVEN, st, a, o);
}

template <bool GIVEN>
int distill_any(const fq_ctx* ctx, int dtype, int rows, int vocab, long long ld, const void* logits, float temperature, const DistillArgs& o,
                cudaStream_t st)
{
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return FQ_ERR_CUDA;
    if (!o.grad) {
        const int threads = stream_threads(rows, ctx->sm_count);
        const Cut c = cut_streams(rows, vocab, type_size(dtype), ctx->sm_count, threads);
        const RowArgs a = row_args(ctx, logits, vocab, ld, temperature, c);
        if (dtype == FQ_DT_F32) return loss_typed<float>(ctx, threads, rows, c, a, o, st);
        if (dtype == FQ_DT_F16) return loss_typed<__half>(ctx, threads, rows, c, a, o, st);
        return loss_typed<__nv_bfloat16>(ctx, threads, rows, c, a, o, st);
    }
    const Cut c = cut_rows(rows, vocab, type_size(dtype), ctx->sm_count, !GIVEN);
    const RowArgs a = row_args(ctx, logits, vocab, ld, temperature, c);
    if (dtype == FQ_DT_F32) return distill_typed<float, GIVEN>(ctx, rows, c, a, o, st);
    if (dtype == FQ_DT_F16) return distill_typed<__half, GIVEN>(ctx, rows, c, a, o, st);
    return distill_typed<__nv_bfloat16, GIVEN>(ctx, rows, c, a, o, st);
}

}  // namespace
}  // namespace fq

using namespace fq;

extern "C" {

int fq_token_logprobs(fq_ctx* ctx, const void* logits_dev, int dtype, int rows, int vocab, long long ld, const void* tokens_dev, int id_bytes,
                      float temperature, float* logprob_dev, float* entropy_dev, int n_top, int* top_ids_dev, float* top_logprobs_dev, void* stream)
{
    const int rc = check_rows(ctx, logits_dev, dtype, rows, vocab, ld, temperature, n_top, id_bytes);
    if (rc != FQ_OK) return rc;
    if (!tokens_dev || !logprob_dev || !entropy_dev || (n_top > 0 && (!top_ids_dev || !top_logprobs_dev))) return FQ_ERR_ARG;
    if (!aligned(tokens_dev, (size_t)id_bytes) || !aligned(logprob_dev, 4) || !aligned(entropy_dev, 4) || !aligned(top_ids_dev, 4) ||
        !aligned(top_logprobs_dev, 4))
        return FQ_ERR_ALIGN;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return FQ_ERR_CUDA;
    const int threads = n_top <= kFewTop ? 128 : 256;
    const Cut c = cut_streams(rows, vocab, type_size(dtype), ctx->sm_count, threads);
    const RowArgs a = row_args(ctx, logits_dev, vocab, ld, temperature, c);
    const LogprobArgs o{tokens_dev, id_bytes == 8, logprob_dev, entropy_dev, n_top, top_ids_dev, top_logprobs_dev};
    const cudaStream_t st = (cudaStream_t)stream;
    if (dtype == FQ_DT_F32) return logprobs_typed<float>(ctx, threads, rows, c, a, o, st);
    if (dtype == FQ_DT_F16) return logprobs_typed<__half>(ctx, threads, rows, c, a, o, st);
    return logprobs_typed<__nv_bfloat16>(ctx, threads, rows, c, a, o, st);
}

int fq_distill_topk(fq_ctx* ctx, const void* logits_dev, int dtype, int rows, int vocab, long long ld, const void* ids_dev, int id_bytes,
                    const float* teacher_dev, int n_top, float temperature, const float* grad_loss_dev, float* loss_dev, float* lse_dev,
                    void* grad_dev, long long ldg, void* stream)
{
    const int rc = check_rows(ctx, logits_dev, dtype, rows, vocab, ld, temperature, n_top, id_bytes);
    if (rc != FQ_OK) return rc;
    if (!ids_dev || !teacher_dev || !loss_dev || !lse_dev || (grad_dev && !grad_loss_dev)) return FQ_ERR_ARG;
    if (n_top < 1 || (grad_dev && ldg < vocab)) return FQ_ERR_SHAPE;
    if (other_pitch(logits_dev, ld, grad_dev, ldg, rows)) return FQ_ERR_ARG;
    if (!aligned(ids_dev, (size_t)id_bytes) || !aligned(teacher_dev, 4) || !aligned(grad_loss_dev, 4) || !aligned(loss_dev, 4) ||
        !aligned(lse_dev, 8) || !aligned(grad_dev, (size_t)type_size(dtype)))
        return FQ_ERR_ALIGN;
    const DistillArgs o{ids_dev, id_bytes == 8, teacher_dev, n_top, grad_loss_dev, loss_dev, reinterpret_cast<float2*>(lse_dev), grad_dev, ldg};
    return distill_any<false>(ctx, dtype, rows, vocab, ld, logits_dev, temperature, o, (cudaStream_t)stream);
}

int fq_distill_topk_grad(fq_ctx* ctx, const void* logits_dev, int dtype, int rows, int vocab, long long ld, const void* ids_dev, int id_bytes,
                         const float* teacher_dev, int n_top, float temperature, const float* grad_loss_dev, const float* lse_dev,
                         void* grad_dev, long long ldg, void* stream)
{
    const int rc = check_rows(ctx, logits_dev, dtype, rows, vocab, ld, temperature, n_top, id_bytes);
    if (rc != FQ_OK) return rc;
    if (!ids_dev || !teacher_dev || !grad_loss_dev || !lse_dev || !grad_dev) return FQ_ERR_ARG;
    if (n_top < 1 || ldg < vocab) return FQ_ERR_SHAPE;
    if (other_pitch(logits_dev, ld, grad_dev, ldg, rows)) return FQ_ERR_ARG;
    if (!aligned(ids_dev, (size_t)id_bytes) || !aligned(teacher_dev, 4) || !aligned(grad_loss_dev, 4) || !aligned(lse_dev, 8) ||
        !aligned(grad_dev, (size_t)type_size(dtype)))
        return FQ_ERR_ALIGN;
    const DistillArgs o{ids_dev, id_bytes == 8, teacher_dev, n_top, grad_loss_dev, nullptr, reinterpret_cast<float2*>(const_cast<float*>(lse_dev)),
                        grad_dev, ldg};
    return distill_any<true>(ctx, dtype, rows, vocab, ld, logits_dev, temperature, o, (cudaStream_t)stream);
}

}  // extern "C"
