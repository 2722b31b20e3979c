// What a model answers, row by row of its logits: log probabilities of given tokens with entropy and top alternatives, and
// distillation from a teacher's top logits (value and gradient).
//
// With m = max z, d_i = (z_i - m) / T and S = sum exp d_i a row needs m, S and sum exp(d_i) d_i, then a second look at its entries
// for the alternatives or the gradient q_i = exp(d_i) / S.  So a row comes on chip once: a cluster of 1..8 CTAs holds it in shared
// memory, a slice each, fetched with bulk copies; the passes over it read shared memory, the CTAs exchange (m, S, ...) through
// distributed shared memory, and a gradient is formed where the logits were and leaves by a bulk copy.  What it has to move is the
// row once in (and once out).
//
// Slices keep the alignment that the row has in global memory, whatever it is: the 16-byte groups inside the slice are copied, the
// elements before the first and behind the last group are loaded one by one, and the rest of those two groups is filled with -inf,
// which no maximum and no sum sees: every pass runs over whole groups without masks.
#include <atomic>
#include <cmath>

#include "fq_cluster.cuh"
#include "fq_internal.cuh"
#include "fq_ptx.cuh"
#include "fq_rowtypes.cuh"

namespace fq {
namespace {

constexpr int kRowThreads = 512;
constexpr int kRowWarps = kRowThreads / 32;
constexpr int kMaxTop = FQ_MAX_TOP;
constexpr int kCandidates = 512;
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
__device__ __forceinline__ unsigned long long two(float2 v)
{
    unsigned long long r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(v.x), "f"(v.y));
    return r;
}
__device__ __forceinline__ float2 apart(unsigned long long v)
{
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
    return r;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b)
{
    unsigned long long r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(two(a)), "l"(two(b)));
    return apart(r);
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b)
{
    unsigned long long r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(two(a)), "l"(two(b)));
    return apart(r);
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    unsigned long long r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(two(a)), "l"(two(b)), "l"(two(c)));
    return apart(r);
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

// Starts the copies and fills the ends.  The caller synchronises the CTA, then waits for `bar`.
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

__device__ __forceinline__ float warp_max(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
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
    float red[2][kRowWarps];
    int failed;
};

// Maximum of the slice; `mine` is that of this thread's entries.
template <class T>
__device__ __forceinline__ float slice_max(const uint4* buf, int groups, RowShared& sh, float& mine)
{
    float m = kNegInf;
    for (int i = threadIdx.x; i < groups; i += kRowThreads) m = fmaxf(m, Group<T>::max_of(buf[i]));
    mine = m;
    m = warp_max(m);
    if ((threadIdx.x & 31) == 0) sh.red[0][threadIdx.x >> 5] = m;
    __syncthreads();
    m = sh.red[0][0];
#pragma unroll
    for (int w = 1; w < kRowWarps; w++) m = fmaxf(m, sh.red[0][w]);
    return m;
}

// Sums of the slice against its own maximum (0 if that is -inf); every thread gets them.
template <class T, bool ENTROPY>
__device__ __forceinline__ RowSums slice_sums(const uint4* buf, int groups, float m, float c2, RowShared& sh)
{
    constexpr int P = Group<T>::N / 2;
    const float mm = m == kNegInf ? 0.0f : m;
    float2 s = make_float2(0.0f, 0.0f), s1 = make_float2(0.0f, 0.0f);
    for (int i = threadIdx.x; i < groups; i += kRowThreads) {
        float2 f[P];
        Group<T>::unpack(buf[i], f);
#pragma unroll
        for (int p = 0; p < P; p++) {
            float2 t = scaled2(f[p], mm, c2);
            if (ENTROPY) {                                       // exp(-160 ln 2) is 0 in 32 bits; 0 * -inf would be NaN
                t.x = max_nan(t.x, -160.0f);
                t.y = max_nan(t.y, -160.0f);
            }
            const float2 e = make_float2(ex2(t.x), ex2(t.y));
            s = add2(s, e);
            if (ENTROPY) s1 = fma2(e, t, s1);
        }
    }
    const float a = warp_sum(s.x + s.y), b = ENTROPY ? warp_sum(s1.x + s1.y) : 0.0f;
    __syncthreads();                                             // slice_max's words have been read
    if ((threadIdx.x & 31) == 0) {
        sh.red[0][threadIdx.x >> 5] = a;
        sh.red[1][threadIdx.x >> 5] = b;
    }
    __syncthreads();
    RowSums r{m, 0.0f, 0.0f};
#pragma unroll
    for (int w = 0; w < kRowWarps; w++) {
        r.s += sh.red[0][w];
        if (ENTROPY) r.s1 += sh.red[1][w];
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
        if (i < n_cta && part[i].s != 0.0f) {                    // (a slice of nothing but -inf has none)
            const float t = part[i].m == r.m ? 0.0f : (part[i].m - r.m) * c2, f = ex2(t);
            r.s += f * part[i].s;
            if (f > 0.0f || part[i].s != part[i].s) r.s1 += f * (part[i].s1 + part[i].s * t);
        }
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

// ------------------------------------------------------------------------------- the largest entries of a slice
struct TopShared {
    unsigned long long cand[kCandidates];     // (key, ~index): larger is earlier
    unsigned long long top[kMaxTop];
    int n, n_top;
    int count[32 + 32];
};

template <class T, class Fn>
__device__ __forceinline__ void each_entry(const uint4* buf, const Slice& s, Fn&& fn)
{
    constexpr int N = Group<T>::N;
    for (int i = threadIdx.x; i < s.groups; i += kRowThreads) {
        float2 f[N / 2];
        Group<T>::unpack(buf[i], f);
#pragma unroll
        for (int e = 0; e < N; e++) {
            const float v = e & 1 ? f[e / 2].y : f[e / 2].x;
            if (v > kNegInf) fn(v, s.first + i * N + e - s.shift);        // not -inf, not NaN
        }
    }
}
__device__ __forceinline__ int block_count(int mine, int& word)
{
    const int c = __reduce_add_sync(0xffffffffu, mine);
    if ((threadIdx.x & 31) == 0 && c) atomicAdd(&word, c);
    __syncthreads();
    return word;
}
__device__ __forceinline__ unsigned long long entry_word(uint32_t key, int index) { return (unsigned long long)key << 32 | (0xffffffffu - (uint32_t)index); }

// Leaves the k largest entries, in order, in sh.top and their number in sh.n_top.
//   The threads' own maxima bound the k-th largest entry from below (k of them are entries): the k-th largest of them, cut to its
//   upper 16 bits, is found by halving, with one vote of the CTA per bit.  What reaches it is collected, usually a few
//   more than k, and ordered by counting.  Entries that are alike in great number (a row of equal logits) overflow the list: then
//   the k-th largest key, and among its bearers the last index that belongs to the k, are found by halving over all entries.
template <class T>
__device__ void slice_top(const uint4* buf, const Slice& s, int k, float mine, TopShared& sh)
{
    for (int i = threadIdx.x; i < 64; i += kRowThreads) sh.count[i] = 0;
    if (threadIdx.x == 0) sh.n = 0;
    const uint32_t my = mine > kNegInf ? key_of(mine) >> 16 : 0u;
    uint32_t least = 0;
    for (int b = 15; b >= 0; b--) {
        const uint32_t q = least | 1u << b;
        if (__syncthreads_count(my >= q) >= k) least = q;
    }
    if (my >= least && my > 0)
        each_entry<T>(buf, s, [&](float v, int index) {
            const uint32_t key = key_of(v);
            if (key >> 16 >= least) {
                const int at = atomicAdd(&sh.n, 1);
                if (at < kCandidates) sh.cand[at] = entry_word(key, index);
            }
        });
    __syncthreads();
    int n = sh.n;
    if (n > kCandidates) {
        uint32_t kth = 0;
        for (int b = 31; b >= 0; b--) {
            const uint32_t q = kth | 1u << b;
            int c = 0;
            each_entry<T>(buf, s, [&](float v, int) { c += key_of(v) >= q; });
            if (block_count(c, sh.count[b]) >= k) kth = q;
        }
        int c = 0;
        each_entry<T>(buf, s, [&](float v, int) { c += key_of(v) > kth; });
        const int above = block_count(c, sh.count[32]);                    // fewer than k
        int before = 0;                                                    // the bearers of `kth` below this index are too few ...
        for (int b = 30; b >= 0; b--) {
            if ((1 << b) > s.first + s.n) continue;
            const int q = before | 1 << b;
            c = 0;
            each_entry<T>(buf, s, [&](float v, int index) { c += key_of(v) == kth && index < q; });
            if (block_count(c, sh.count[33 + b]) < k - above) before = q;  // ... so that the last that counts is at it
        }
        if (threadIdx.x == 0) sh.n = 0;
        __syncthreads();
        each_entry<T>(buf, s, [&](float v, int index) {
            const uint32_t key = key_of(v);
            if (key > kth || (key == kth && index <= before)) {
                const int at = atomicAdd(&sh.n, 1);
                if (at < kCandidates) sh.cand[at] = entry_word(key, index);
            }
        });
        __syncthreads();
        n = sh.n;
    }
    for (int i = threadIdx.x; i < n; i += kRowThreads) {
        const unsigned long long w = sh.cand[i];
        int rank = 0;
        for (int j = 0; j < n; j++) rank += sh.cand[j] > w;
        if (rank < k) sh.top[rank] = w;
    }
    if (threadIdx.x == 0) sh.n_top = n < k ? n : k;
    __syncthreads();
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

template <class T>
__global__ void __launch_bounds__(kRowThreads, 2) token_logprobs_kernel(const RowArgs a, const LogprobArgs o)
{
    extern __shared__ __align__(16) uint4 buf[];
    __shared__ RowShared sh;
    __shared__ TopShared top;
    const int rank = a.n_cta > 1 ? (int)cluster_cta() : 0;
    const long long r = blockIdx.x / a.n_cta;
    const T* row = static_cast<const T*>(a.z) + r * a.ld;
    const Slice s = slice_of<T>(a, row, rank);
    if (threadIdx.x == 0) sh.failed = 0;
    fetch_slice<T>(row, s, buf, smem_u32(&sh.bar));
    long long token = -1;
    float z_token = 0.0f;
    if (rank == 0 && threadIdx.x == 0) {
        token = load_id(o.tokens, o.wide, r);
        if (token >= 0 && token < a.vocab) z_token = Group<T>::to_f(row[token]);
    }
    __syncthreads();
    await_slice(sh, a);
    float mine;
    const float m = slice_max<T>(buf, s.groups, sh, mine);
    RowSums sum = slice_sums<T, true>(buf, s.groups, m, a.c2, sh);
    if (o.n_top > 0) slice_top<T>(buf, s, o.n_top, mine, top);
    int n_top = o.n_top > 0 ? top.n_top : 0;
    const unsigned long long* best = top.top;
    if (a.n_cta > 1) {
        if (threadIdx.x == 0) sh.sums = sum;
        __syncthreads();
        cluster_arrive();
        cluster_wait();
        if (rank == 0) {
            sum = join(sh, a.n_cta, a.c2);
            // the CTAs' lists, merged: an entry's place is its own place in its list and what is larger in each of the others
            if (o.n_top > 0) {
                unsigned long long* lists = reinterpret_cast<unsigned long long*>(buf);
                int* lens = top.count;
                const uint32_t at = smem_u32(top.top), at_n = smem_u32(&top.n_top);
                if (threadIdx.x < a.n_cta) {
                    const uint32_t there = cluster_map(at_n, threadIdx.x);
                    int n;
                    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(n) : "r"(there) : "memory");
                    lens[threadIdx.x] = n;
                }
                __syncthreads();
                for (int i = threadIdx.x; i < a.n_cta * kMaxTop; i += kRowThreads) {
                    const int c = i / kMaxTop, j = i % kMaxTop;
                    if (j < lens[c]) lists[i] = cluster_ld_u64(cluster_map(at, (uint32_t)c) + (uint32_t)j * 8);
                }
                __syncthreads();
                int total = 0;
                for (int c = 0; c < a.n_cta; c++) total += lens[c];
                n_top = total < o.n_top ? total : o.n_top;
                for (int i = threadIdx.x; i < a.n_cta * kMaxTop; i += kRowThreads) {
                    const int c = i / kMaxTop, j = i % kMaxTop;
                    if (j >= lens[c]) continue;
                    const unsigned long long w = lists[i];
                    int place = j;
                    for (int d = 0; d < a.n_cta; d++) {
                        if (d == c) continue;
                        int lo = 0, hi = lens[d];                           // entries of list d that are larger than w
                        while (lo < hi) {
                            const int mid = (lo + hi) >> 1;
                            if (lists[d * kMaxTop + mid] > w) lo = mid + 1; else hi = mid;
                        }
                        place += lo;
                    }
                    if (place < o.n_top) top.cand[place] = w;
                }
                best = top.cand;
                __syncthreads();
            }
        }
        cluster_arrive();                                                    // nobody's shared memory is read any more
        cluster_wait();
    }
    if (rank == 0) {
        const float zm = sum.m == kNegInf ? 0.0f : sum.m;
        const float log_s = sum.s == 0.0f ? 0.0f : logf(sum.s);
        const bool nan = sum.s != sum.s;
        if (threadIdx.x == 0) {
            float lp = 0.0f;
            if (token >= a.vocab) lp = NAN;
            else if (token >= 0) lp = nan ? NAN : (z_token - zm) / a.t - log_s;
            o.logprob[r] = lp;
            o.entropy[r] = sum.s == 0.0f ? 0.0f : log_s - kLn2 * (sum.s1 / sum.s);
        }
        if (threadIdx.x < o.n_top) {
            const int j = threadIdx.x;
            const bool there = j < n_top && !nan;
            const unsigned long long w = there ? best[j] : 0ull;
            o.top_ids[r * o.n_top + j] = there ? (int)(0xffffffffu - (uint32_t)w) : -1;
            o.top_logprobs[r * o.n_top + j] = there ? (of_key((uint32_t)(w >> 32)) - zm) / a.t - log_s : (nan ? NAN : kNegInf);
        }
    }
    if (sh.failed) let_copies_land();
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

struct TeacherShared {
    long long id[kMaxTop];
    float p[kMaxTop], lp[kMaxTop];        // probability, its logarithm (first: the logits)
    float part[kMaxTop / 32];
    int any, bad;
};

// The teacher's distribution over its slots (threads 0..31 after the slots are written).
__device__ __forceinline__ void teacher_softmax(TeacherShared& sh, int k, float c2, float t)
{
    const int lane = threadIdx.x;
    float u[kMaxTop / 32], m = kNegInf, s = 0.0f;
#pragma unroll
    for (int i = 0; i < kMaxTop / 32; i++) {
        u[i] = lane + 32 * i < k ? sh.lp[lane + 32 * i] : kNegInf;
        m = max_nan(m, u[i]);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
    const float mm = m == kNegInf ? 0.0f : m;
    float e[kMaxTop / 32];
#pragma unroll
    for (int i = 0; i < kMaxTop / 32; i++) {
        e[i] = ex2((u[i] - mm) * c2);
        s += e[i];
    }
    s = warp_sum(s);
    const float inv = s == 0.0f ? 0.0f : 1.0f / s, log_s = s == 0.0f ? 0.0f : logf(s);
#pragma unroll
    for (int i = 0; i < kMaxTop / 32; i++)
        if (lane + 32 * i < k) {
            sh.p[lane + 32 * i] = e[i] * inv;
            sh.lp[lane + 32 * i] = (u[i] - mm) / t - log_s;
        }
    if (lane == 0) sh.any = s != 0.0f;                                       // (NaN: true)
}

// GIVEN: the gradient alone, from the (m, log S) that an earlier call kept; slices then need nothing from one another.
template <class T, bool GIVEN>
__global__ void __launch_bounds__(kRowThreads, 2) distill_kernel(const RowArgs a, const DistillArgs o)
{
    extern __shared__ __align__(16) uint4 buf[];
    __shared__ RowShared sh;
    __shared__ TeacherShared te;
    constexpr int N = Group<T>::N;
    const int rank = (int)(blockIdx.x % a.n_cta);
    const long long r = blockIdx.x / a.n_cta;
    const T* row = static_cast<const T*>(a.z) + r * a.ld;
    const Slice s = slice_of<T>(a, row, rank);
    if (threadIdx.x == 0) {
        sh.failed = 0;
        te.bad = 0;
    }
    fetch_slice<T>(row, s, buf, smem_u32(&sh.bar));
    __syncthreads();
    // slot j is thread j's: its id, and the student's logit there (read before any gradient may overwrite it)
    long long id = -1;
    float z_id = kNegInf;
    if (threadIdx.x < o.k) {
        id = load_id(o.ids, o.wide, r * o.k + threadIdx.x);
        const float u = o.teacher[r * o.k + threadIdx.x];
        if (id >= a.vocab) te.bad = 1;
        const bool in_reach = GIVEN ? id >= s.first && id < s.first + s.n : id >= 0 && id < a.vocab;
        if (in_reach) z_id = Group<T>::to_f(row[id]);
        te.id[threadIdx.x] = id;
        te.lp[threadIdx.x] = id >= 0 ? u : kNegInf;
    }
    __syncthreads();
    if (threadIdx.x < 32) teacher_softmax(te, o.k, a.c2, a.t);
    await_slice(sh, a);
    RowSums sum;
    float log_s;
    if (GIVEN) {
        const float2 st = o.stats[r];
        sum = RowSums{st.x, 0.0f, 0.0f};
        log_s = st.y;
        __syncthreads();
    } else {
        float mine;
        const float m = slice_max<T>(buf, s.groups, sh, mine);
        sum = slice_sums<T, false>(buf, s.groups, m, a.c2, sh);
        if (a.n_cta > 1) {
            if (threadIdx.x == 0) sh.sums = sum;
            __syncthreads();
            cluster_arrive();
            cluster_wait();
            sum = join(sh, a.n_cta, a.c2);
        }
        log_s = sum.s == 0.0f ? 0.0f : logf(sum.s);
    }
    const float zm = sum.m == kNegInf ? 0.0f : sum.m;
    if (!GIVEN && rank == 0) {
        float term = 0.0f;
        if (threadIdx.x < o.k) {
            const float p = te.p[threadIdx.x];
            // p (log p - log q); p times a distance that 32 bits do not hold may well be one that they do
            if (!(p == 0.0f)) term = p * (te.lp[threadIdx.x] + log_s) - p * (z_id - zm) / a.t;
        }
        if (threadIdx.x < kMaxTop) {
            term = warp_sum(term);
            if ((threadIdx.x & 31) == 0) te.part[threadIdx.x >> 5] = term;
        }
        __syncthreads();
        if (threadIdx.x == 0) {
            float loss = 0.0f;
            for (int i = 0; i < kMaxTop / 32; i++) loss += te.part[i];
            o.loss[r] = te.bad ? NAN : loss;
            o.stats[r] = make_float2(sum.m, sum.s != sum.s ? NAN : log_s);
        }
    }
    if (o.grad) {
        // g (q_i - p_i) / T, formed where the logits are.  A row without a teacher, or whose upstream gradient is 0, gets zeros
        // whatever it holds.
        const float g = o.grad_loss[r];
        const bool zero = g == 0.0f || (!te.any && !te.bad);
        const float w = te.bad ? NAN : g / a.t;
        const float off = log_s * kLog2e;                        // q = 2^(t - off)
        T* out_row = static_cast<T*>(o.grad) + r * o.ldg;
        T* el = reinterpret_cast<T*>(buf);
        for (int i = threadIdx.x; i < s.groups; i += kRowThreads) {
            float2 f[N / 2];
            Group<T>::unpack(buf[i], f);
#pragma unroll
            for (int p = 0; p < N / 2; p++) {
                const float2 t = add2(scaled2(f[p], zm, a.c2), make_float2(-off, -off));
                const float2 q = mul2(make_float2(ex2(t.x), ex2(t.y)), make_float2(w, w));
                f[p] = zero ? make_float2(0.0f, 0.0f) : q;
            }
            buf[i] = Group<T>::pack(f);
        }
        __syncthreads();
        if (threadIdx.x < o.k && !zero && id >= s.first && id < s.first + s.n) {
            float p = 0.0f;
            bool first = true;
            for (int j = 0; j < o.k; j++)
                if (te.id[j] == id) {
                    if (j < (int)threadIdx.x) first = false;
                    p += te.p[j];
                }
            const float t = (z_id - zm) * a.c2 - off;
            if (first) el[s.shift + (int)(id - s.first)] = Group<T>::from_f((ex2(t) - p) * w);
        }
        const bool alike = ((reinterpret_cast<uintptr_t>(out_row) ^ reinterpret_cast<uintptr_t>(row)) & 15) == 0;
        T* dst = out_row + s.first - s.shift;                    // element 0 of the buffer
        int lo, hi;
        whole_groups<T>(s, lo, hi);
        if (alike) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncthreads();
        const int end = s.shift + s.n;
        if (alike) {
            if (threadIdx.x == 0 && hi > lo) {
                asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;"
                             ::"l"(dst + lo), "r"(smem_u32(el + lo)), "r"((hi - lo) * (int)sizeof(T)) : "memory");
                asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
            }
            const int t = threadIdx.x - 32;
            if (t >= 0 && t < 2 * N) {
                const int e = t < N ? s.shift + t : hi + (t - N);
                if (t < N ? e < lo && e < end : e < end) dst[e] = el[e];
            }
        } else {
            for (int e = s.shift + threadIdx.x; e < end; e += kRowThreads) dst[e] = el[e];
        }
    }
    if (!GIVEN && a.n_cta > 1) {                                 // nobody's sums are read any more
        cluster_arrive();
        cluster_wait();
    }
    if (sh.failed) let_copies_land();
}

// ------------------------------------------------------------------------------- host side
// How the rows are cut.  A slice of up to 68 KB leaves room for three CTAs on an SM, so that one computes while the copies of the
// others are on their way.  With few rows a row is spread over more SMs, down to slices of 8 KB.
struct Cut { int n_cta, slice; size_t smem; };
Cut cut_rows(int rows, int vocab, int size, int sm_count)
{
    constexpr int kSliceBytes = 68 * 1024, kLeastBytes = 8 * 1024;
    const int n = 16 / size;
    Cut c{};
    const auto per = [&](int ctas) { return ((vocab + ctas - 1) / ctas + n - 1) / n * n; };
    c.n_cta = 1;
    while (c.n_cta < kMaxCluster && per(c.n_cta) * size > kSliceBytes) c.n_cta *= 2;
    while (c.n_cta < kMaxCluster && (long long)rows * c.n_cta * 2 <= sm_count && per(2 * c.n_cta) * size >= kLeastBytes) c.n_cta *= 2;
    c.slice = per(c.n_cta);
    c.smem = (size_t)c.slice * size + 32;
    const size_t lists = c.n_cta > 1 ? (size_t)c.n_cta * kMaxTop * 8 : 0;
    if (c.smem < lists) c.smem = lists;
    return c;
}

template <class... Args>
int launch_rows(void (*kernel)(Args...), std::atomic<bool>* ready, const Ctx* ctx, int rows, const Cut& c, bool cluster, cudaStream_t st,
                Args... args)
{
    if (ctx->device >= 64) return FQ_ERR_ARG;
    if (!ready[ctx->device].load(std::memory_order_acquire)) {
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 208 * 1024) != cudaSuccess) return FQ_ERR_CUDA;
        ready[ctx->device].store(true, std::memory_order_release);
    }
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = (unsigned)c.n_cta; attr.val.clusterDim.y = 1; attr.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)rows * (unsigned)c.n_cta); cfg.blockDim = dim3(kRowThreads); cfg.dynamicSmemBytes = c.smem;
    cfg.stream = st;
    if (cluster && c.n_cta > 1) { cfg.attrs = &attr; cfg.numAttrs = 1; }
    return cudaLaunchKernelEx(&cfg, kernel, args...) == cudaSuccess ? FQ_OK : FQ_ERR_CUDA;
}

int check_rows(const fq_ctx* ctx, const void* logits, int dtype, int rows, int vocab, long long ld, float temperature, int n_top, int id_bytes)
{
    const int size = type_size(dtype);
    if (!ctx || !logits || !size || (id_bytes != 4 && id_bytes != 8)) return FQ_ERR_ARG;
    if (!(temperature > 0.0f) || std::isinf(temperature)) return FQ_ERR_ARG;
    if (rows < 1 || rows > FQ_MAX_ROWS || vocab < 1 || vocab > FQ_MAX_VOCAB || ld < vocab || n_top < 0 || n_top > FQ_MAX_TOP) return FQ_ERR_SHAPE;
    if (!aligned(logits, (size_t)size)) return FQ_ERR_ALIGN;
    return FQ_OK;
}

RowArgs row_args(const Ctx* ctx, const void* logits, int vocab, long long ld, float temperature, const Cut& c)
{
    RowArgs a{};
    a.z = logits; a.ld = ld; a.vocab = vocab; a.slice = c.slice; a.n_cta = c.n_cta;
    a.c2 = (float)(1.4426950408889634 / (double)temperature); a.t = temperature;
    a.status = ctx->status_dev; a.wait_ns = ctx->wait_limit_ns;
    return a;
}

template <class T>
int logprobs_typed(const Ctx* ctx, int rows, const Cut& c, const RowArgs& a, const LogprobArgs& o, cudaStream_t st)
{
    static std::atomic<bool> ready[64];
    return launch_rows(token_logprobs_kernel<T>, ready, ctx, rows, c, true, st, a, o);
}

template <class T, bool GIVEN>
int distill_typed(const Ctx* ctx, int rows, const Cut& c, const RowArgs& a, const DistillArgs& o, cudaStream_t st)
{
    static std::atomic<bool> ready[64];
    return launch_rows(distill_kernel<T, GIVEN>, ready, ctx, rows, c, !GIVEN, st, a, o);
}

template <bool GIVEN>
int distill_any(const fq_ctx* ctx, int dtype, int rows, int vocab, long long ld, const void* logits, float temperature, const DistillArgs& o,
                cudaStream_t st)
{
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return FQ_ERR_CUDA;
    const Cut c = cut_rows(rows, vocab, type_size(dtype), ctx->sm_count);
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
    const Cut c = cut_rows(rows, vocab, type_size(dtype), ctx->sm_count);
    const RowArgs a = row_args(ctx, logits_dev, vocab, ld, temperature, c);
    const LogprobArgs o{tokens_dev, id_bytes == 8, logprob_dev, entropy_dev, n_top, top_ids_dev, top_logprobs_dev};
    const cudaStream_t st = (cudaStream_t)stream;
    if (dtype == FQ_DT_F32) return logprobs_typed<float>(ctx, rows, c, a, o, st);
    if (dtype == FQ_DT_F16) return logprobs_typed<__half>(ctx, rows, c, a, o, st);
    return logprobs_typed<__nv_bfloat16>(ctx, rows, c, a, o, st);
}

int fq_distill_topk(fq_ctx* ctx, const void* logits_dev, int dtype, int rows, int vocab, long long ld, const void* ids_dev, int id_bytes,
                    const float* teacher_dev, int n_top, float temperature, const float* grad_loss_dev, float* loss_dev, float* lse_dev,
                    void* grad_dev, long long ldg, void* stream)
{
    const int rc = check_rows(ctx, logits_dev, dtype, rows, vocab, ld, temperature, n_top, id_bytes);
    if (rc != FQ_OK) return rc;
    if (!ids_dev || !teacher_dev || !loss_dev || !lse_dev || (grad_dev && !grad_loss_dev)) return FQ_ERR_ARG;
    if (n_top < 1 || (grad_dev && ldg < vocab)) return FQ_ERR_SHAPE;
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
    if (!aligned(ids_dev, (size_t)id_bytes) || !aligned(teacher_dev, 4) || !aligned(grad_loss_dev, 4) || !aligned(lse_dev, 8) ||
        !aligned(grad_dev, (size_t)type_size(dtype)))
        return FQ_ERR_ALIGN;
    const DistillArgs o{ids_dev, id_bytes == 8, teacher_dev, n_top, grad_loss_dev, nullptr, reinterpret_cast<float2*>(const_cast<float*>(lse_dev)),
                        grad_dev, ldg};
    return distill_any<true>(ctx, dtype, rows, vocab, ld, logits_dev, temperature, o, (cudaStream_t)stream);
}

}  // extern "C"
