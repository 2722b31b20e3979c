// Rotary positions: pairs of a head's values are turned by angles that grow with the token's position; keys and values may go straight to a
// layer's cache.
//
// Angles.  A pair's angle is position * f, of which only the part beyond whole turns counts.  In fp32 that part is lost far out (at a million, 2^-24 of the
// product is 0.06 radians), so frequencies come as 64-bit fixed-point fractions of a turn: position * fraction modulo 2^64 is the angle exactly, two
// integer multiplications, and its upper 32 bits as a float are an argument of sincospi within 2^-25 of half a turn.
#include <cmath>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "fq_internal.cuh"
#include "fq_rowtypes.cuh"

namespace fq {
namespace {

constexpr int kMaxTensors = 3;
constexpr int kThreads = 256;
constexpr int kMaxRot = 1024;

struct Tensor {
    const void* src;
    void* dst;                           // null: the layer's cache
    long long src_token, src_head, dst_token, dst_head;
    int heads;
    int rot;                             // values turned (0: copied)
    int pieces;                          // pieces of a head: turned ones, then copied ones (none in place)
};
struct RotaryArgs {
    Tensor t[kMaxTensors];
    int n, items;                        // pieces of a token, all tensors
    int head_dim, half;                  // half: rot_dim / 2
    const void* positions;
    int wide_positions;
    const uint64_t* turns;
    float magnitude, side;               // side: -1 turns the other way
    const long long* slots;              // null: nothing goes to a cache
    void* cache[2];
    long long block_stride, token_stride;
    long long n_slots;
    int block_size;
    int* status;
};

// N values of a row in registers, as they lie in memory: one access.
template <class T, int N>
struct Piece {
    static constexpr int kBytes = N * (int)sizeof(T);
    static_assert(kBytes == 16 || kBytes == 8 || N == 1, "one access");
    alignas(16) T raw[N];
    __device__ __forceinline__ void load(const T* p)
    {
        if constexpr (kBytes == 16) *reinterpret_cast<uint4*>(raw) = *reinterpret_cast<const uint4*>(p);
        else if constexpr (kBytes == 8) *reinterpret_cast<uint2*>(raw) = *reinterpret_cast<const uint2*>(p);
        else raw[0] = p[0];
    }
    __device__ __forceinline__ void store(T* p) const
    {
        if constexpr (kBytes == 16) *reinterpret_cast<uint4*>(p) = *reinterpret_cast<const uint4*>(raw);
        else if constexpr (kBytes == 8) *reinterpret_cast<uint2*>(p) = *reinterpret_cast<const uint2*>(raw);
        else p[0] = raw[0];
    }
    __device__ __forceinline__ float at(int i) const { return Group<T>::to_f(raw[i]); }
    __device__ __forceinline__ void set(int i, float v) { raw[i] = Group<T>::from_f(v); }
};

// A CTA has an item a thread of one token: with several (fewer CTAs form a token's angles then) 777 tokens of 64 heads took 10.5 us instead of 8.5, and
// 8192 of 80 as long.  The loads go out before the angles are formed.  8192 tokens, 80 heads of 128 in fp32, 671 MB: 123 us (HBM floor 104).
//   N : values of a piece.  A turned item is a piece of the lower and one of the upper half, or with INTERLEAVED one piece of pairs (two single values
//       where N is 1)
template <class T, int N, bool INTERLEAVED>
__global__ void __launch_bounds__(kThreads, 4) rotary_kernel(const __grid_constant__ RotaryArgs a)
{
    __shared__ float2 angle[kMaxRot / 2];        // (cos, sin) * magnitude
    __shared__ long long place;                  // offset of the token's cell in the cache, or -1
    const int token = blockIdx.x;
    constexpr int kStep = INTERLEAVED && N == 1 ? 2 : N;        // values of a row that a turned item's first piece stands for
    constexpr bool kTwo = !(INTERLEAVED && N > 1);
    Piece<T, N> lo, hi;
    T* out = nullptr;
    int pair = -1, apart = 0;                    // first pair (-1: copied), distance of the second piece
    bool stored = false;                         // goes to the cache
    int i = blockIdx.y * kThreads + (int)threadIdx.x;
    if (i < a.items) {
        int which = 0;
        while (i >= a.t[which].heads * a.t[which].pieces) i -= a.t[which].heads * a.t[which].pieces, which++;
        const Tensor& t = a.t[which];
        const int head = i / t.pieces, piece = i - head * t.pieces;
        const int turned = INTERLEAVED ? t.rot / kStep : t.rot / 2 / N;
        int at = t.rot + (piece - turned) * N;
        if (piece < turned) {
            at = piece * kStep;
            pair = INTERLEAVED ? at / 2 : at;
            apart = INTERLEAVED ? 1 : t.rot / 2;
        }
        const T* src = static_cast<const T*>(t.src) + token * t.src_token + head * t.src_head + at;
        stored = !t.dst;
        out = (stored ? static_cast<T*>(a.cache[which == 2]) : static_cast<T*>(t.dst) + token * t.dst_token) + head * t.dst_head + at;
        lo.load(src);
        if (kTwo && pair >= 0) hi.load(src + apart);
    }
    const long long position = a.wide_positions ? static_cast<const long long*>(a.positions)[token] : static_cast<const int*>(a.positions)[token];
    for (int p = threadIdx.x; p < a.half; p += kThreads) {
        const uint64_t turn = (uint64_t)position * a.turns[p];
        float s, c;
        sincospif((float)(int)(turn >> 32) * 0x1p-31f, &s, &c);
        angle[p] = make_float2(c * a.magnitude, s * a.magnitude * a.side);
    }
    if (threadIdx.x == 0 && a.slots) {
        const long long slot = a.slots[token];
        place = -1;
        if (slot >= a.n_slots) atomicCAS(a.status, 0, FQ_ERR_INDEX);
        else if (slot >= 0) place = slot / a.block_size * a.block_stride + slot % a.block_size * a.token_stride;
    }
    __syncthreads();
    if (!out || (stored && place < 0)) return;
    T* y = stored ? out + place : out;
    if (pair < 0) {
        lo.store(y);
        return;
    }
    if constexpr (!kTwo) {
#pragma unroll
        for (int e = 0; e < N; e += 2) {
            const float2 w = angle[pair + e / 2];
            const float x0 = lo.at(e), x1 = lo.at(e + 1);
            lo.set(e, fmaf(x0, w.x, -(x1 * w.y)));               // (written out: the same roundings in every variant)
            lo.set(e + 1, fmaf(x0, w.y, x1 * w.x));
        }
        lo.store(y);
    } else {
#pragma unroll
        for (int e = 0; e < N; e++) {
            const float2 w = angle[pair + e];
            const float x0 = lo.at(e), x1 = hi.at(e);
            lo.set(e, fmaf(x0, w.x, -(x1 * w.y)));
            hi.set(e, fmaf(x0, w.y, x1 * w.x));
        }
        lo.store(y);
        hi.store(y + apart);
    }
}

template <class T, int N, bool INTERLEAVED>
int launch_pieces(RotaryArgs& a, int tokens, cudaStream_t st)
{
    constexpr int kStep = INTERLEAVED && N == 1 ? 2 : N;
    a.items = 0;
    for (int i = 0; i < a.n; i++) {
        Tensor& t = a.t[i];
        const int turned = INTERLEAVED ? t.rot / kStep : t.rot / 2 / N;
        t.pieces = turned + (t.dst == t.src ? 0 : (a.head_dim - t.rot) / N);
        a.items += t.heads * t.pieces;
    }
    rotary_kernel<T, N, INTERLEAVED><<<dim3((unsigned)tokens, (unsigned)((a.items + kThreads - 1) / kThreads)), kThreads, 0, st>>>(a);
    return cudaGetLastError() == cudaSuccess ? FQ_OK : FQ_ERR_CUDA;
}

template <class T>
int launch_typed(RotaryArgs& a, int tokens, int interleaved, size_t align, cudaStream_t st)
{
    constexpr int kFull = 16 / (int)sizeof(T), kHalf = 8 / (int)sizeof(T);
    if (interleaved) {
        if (align >= 16) return launch_pieces<T, kFull, true>(a, tokens, st);
        if (align >= 8) return launch_pieces<T, kHalf, true>(a, tokens, st);
        return launch_pieces<T, 1, true>(a, tokens, st);
    }
    if (align >= 16) return launch_pieces<T, kFull, false>(a, tokens, st);
    if (align >= 8) return launch_pieces<T, kHalf, false>(a, tokens, st);
    return launch_pieces<T, 1, false>(a, tokens, st);
}

// The largest power of two, up to 16, that divides every address and distance (in bytes).
struct Common {
    unsigned long long bits = 16;
    void take(unsigned long long v) { bits |= v; }
    size_t bytes() const { return (size_t)(bits & (~bits + 1)); }
};

int launch_rotary(const fq_ctx* ctx, RotaryArgs& a, int dtype, int tokens, int rot, int interleaved, cudaStream_t st)
{
    const int size = type_size(dtype);
    Common c;
    c.take((unsigned long long)(interleaved ? rot : rot / 2) * size);
    for (int i = 0; i < a.n; i++) {
        const Tensor& t = a.t[i];
        c.take(reinterpret_cast<uintptr_t>(t.src));
        c.take((unsigned long long)t.src_token * size);
        c.take((unsigned long long)t.src_head * size);
        c.take((unsigned long long)t.dst_token * size);
        c.take((unsigned long long)t.dst_head * size);
        c.take(reinterpret_cast<uintptr_t>(t.dst));
        if (t.dst != t.src) c.take((unsigned long long)(a.head_dim - t.rot) * size);
    }                                    // (a cache's cells are 16-byte aligned)
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return FQ_ERR_CUDA;
    if (dtype == FQ_DT_F32) return launch_typed<float>(a, tokens, interleaved, c.bytes(), st);
    if (dtype == FQ_DT_F16) return launch_typed<__half>(a, tokens, interleaved, c.bytes(), st);
    return launch_typed<__nv_bfloat16>(a, tokens, interleaved, c.bytes(), st);
}

int check_rotary(const fq_ctx* ctx, int dtype, int tokens, int head_dim, int rot_dim, const void* positions, int id_bytes, const uint64_t* turns,
                 float magnitude)
{
    if (!ctx || !positions || !turns || !type_size(dtype) || (id_bytes != 4 && id_bytes != 8) || !std::isfinite(magnitude)) return FQ_ERR_ARG;
    if (tokens < 1 || tokens > FQ_MAX_ROWS || head_dim < 2 || head_dim > kMaxRot || rot_dim < 2 || rot_dim > head_dim || rot_dim % 2) return FQ_ERR_SHAPE;
    if (!aligned(positions, (size_t)id_bytes) || !aligned(turns, 8)) return FQ_ERR_ALIGN;
    return FQ_OK;
}


// A source may be read again and again (a stride of 0).
int check_source(const fq_heads* x, int dtype)
{
    if (!x || !x->dev) return FQ_ERR_ARG;
    if (x->heads < 1 || x->heads > 1024 || x->head_stride < 0 || x->token_stride < 0) return FQ_ERR_SHAPE;
    return aligned(x->dev, (size_t)type_size(dtype)) ? FQ_OK : FQ_ERR_ALIGN;
}

int check_pair(const fq_heads* x, const fq_heads* y, int dtype, int tokens, int head_dim)
{
    int rc = check_source(x, dtype);
    if (rc == FQ_OK) rc = check_heads(y, dtype, tokens, head_dim);
    if (rc != FQ_OK) return rc;
    if (x->heads != y->heads) return FQ_ERR_SHAPE;
    // in place: cell for cell
    if (x->dev == y->dev && ((x->heads > 1 && x->head_stride != y->head_stride) || (tokens > 1 && x->token_stride != y->token_stride))) return FQ_ERR_ARG;
    return FQ_OK;
}

Tensor tensor(const fq_heads* x, const fq_heads* y, int tokens, int rot)
{
    Tensor t{};
    t.src = x->dev; t.dst = y->dev; t.heads = x->heads; t.rot = rot;
    // (a stride that is never taken says nothing about alignment)
    t.src_token = tokens > 1 ? x->token_stride : 0; t.src_head = x->heads > 1 ? x->head_stride : 0;
    t.dst_token = tokens > 1 ? y->token_stride : 0; t.dst_head = x->heads > 1 ? y->head_stride : 0;
    return t;
}

Tensor to_cache(const fq_heads* x, const fq_cache* cache, int tokens, int rot)
{
    Tensor t{};
    t.src = x->dev; t.heads = x->heads; t.rot = rot;
    t.src_token = tokens > 1 ? x->token_stride : 0; t.src_head = x->heads > 1 ? x->head_stride : 0;
    t.dst_head = x->heads > 1 ? cache->head_stride : 0;
    return t;
}

}  // namespace

// Rows of an output may not overlap: heads within a token's stride, or tokens within a head's.
int check_heads(const fq_heads* x, int dtype, int tokens, int head_dim)
{
    if (!x || !x->dev) return FQ_ERR_ARG;
    if (x->heads < 1 || x->heads > 1024 || x->head_stride < 0 || x->token_stride < 0) return FQ_ERR_SHAPE;
    const long long heads = (x->heads - 1) * x->head_stride + head_dim, rows = (tokens - 1) * x->token_stride + head_dim;
    if ((x->heads > 1 && x->head_stride < head_dim) || (tokens > 1 && x->token_stride < head_dim)) return FQ_ERR_SHAPE;
    if (x->heads > 1 && tokens > 1 && x->token_stride < heads && x->head_stride < rows) return FQ_ERR_SHAPE;
    return aligned(x->dev, (size_t)type_size(dtype)) ? FQ_OK : FQ_ERR_ALIGN;
}

int check_cache(const fq_cache* c, int dtype, int head_dim)
{
    if (!c || !c->k_dev || !c->v_dev) return FQ_ERR_ARG;
    const long long size = type_size(dtype);
    if (c->blocks < 1 || c->block_size < 1 || c->block_size > (1 << 16) || c->heads < 1 || c->heads > 1024) return FQ_ERR_SHAPE;
    if ((c->blocks > 1 && c->block_stride < head_dim) || (c->block_size > 1 && c->token_stride < head_dim) || (c->heads > 1 && c->head_stride < head_dim))
        return FQ_ERR_SHAPE;
    if (head_dim * size % 16 || c->block_stride < 0 || c->token_stride < 0 || c->head_stride < 0) return FQ_ERR_SHAPE;
    if (!aligned(c->k_dev, 16) || !aligned(c->v_dev, 16)) return FQ_ERR_ALIGN;
    if ((c->blocks > 1 && c->block_stride * size % 16) || (c->block_size > 1 && c->token_stride * size % 16) || (c->heads > 1 && c->head_stride * size % 16))
        return FQ_ERR_ALIGN;
    return FQ_OK;
}

}  // namespace fq

using namespace fq;

extern "C" {

int fq_rotary_table(int rot_dim, double base, double factor, int context, double low, double high, uint64_t* turns_host)
{
    if (!turns_host) return FQ_ERR_ARG;
    if (rot_dim < 2 || rot_dim > kMaxRot || rot_dim % 2) return FQ_ERR_SHAPE;
    if (!(base > 1.0) || !(factor >= 1.0) || !std::isfinite(base) || !std::isfinite(factor) || context < 0 || !(low >= 0.0) || !(high > low) || !std::isfinite(high))
        return FQ_ERR_ARG;
    const long double turn = 2.0L * acosl(-1.0L);
    for (int i = 0; i < rot_dim / 2; i++) {
        const long double f = powl((long double)base, -2.0L * i / rot_dim) / turn;       // turns a position
        long double kept = 0.0L;
        if (context > 0) kept = fminl(1.0L, fmaxl(0.0L, ((long double)context * f - low) / ((long double)high - low)));
        const long double scaled = kept * f + (1.0L - kept) * f / factor;                // at most 1 / (2 pi)
        turns_host[i] = (uint64_t)rintl(ldexpl(scaled, 64));
    }
    return FQ_OK;
}

int fq_rotary(fq_ctx* ctx, const fq_rotary_args* args, void* stream)
{
    if (!args) return FQ_ERR_ARG;
    const fq_rotary_args& x = *args;
    int rc = check_rotary(ctx, x.dtype, x.tokens, x.head_dim, x.rot_dim, x.positions_dev, x.id_bytes, x.turns_dev, x.magnitude);
    if (rc != FQ_OK) return rc;
    if (x.n < 1 || x.n > 2) return FQ_ERR_SHAPE;
    RotaryArgs a{};
    for (int i = 0; i < x.n; i++) {
        rc = check_pair(x.x + i, x.y + i, x.dtype, x.tokens, x.head_dim);
        if (rc != FQ_OK) return rc;
        a.t[i] = tensor(x.x + i, x.y + i, x.tokens, x.rot_dim);
    }
    // one tensor's output is neither the other's output nor its source
    if (x.n == 2 && (x.y[0].dev == x.y[1].dev || x.y[0].dev == x.x[1].dev || x.y[1].dev == x.x[0].dev)) return FQ_ERR_ARG;
    a.n = x.n; a.head_dim = x.head_dim; a.half = x.rot_dim / 2;
    a.positions = x.positions_dev; a.wide_positions = x.id_bytes == 8; a.turns = x.turns_dev;
    a.magnitude = x.magnitude; a.side = x.inverse ? -1.0f : 1.0f; a.status = ctx->status_dev;
    return launch_rotary(ctx, a, x.dtype, x.tokens, x.rot_dim, x.interleaved, (cudaStream_t)stream);
}

int fq_rotary_cache(fq_ctx* ctx, const fq_rotary_cache_args* args, void* stream)
{
    if (!args) return FQ_ERR_ARG;
    const fq_rotary_cache_args& x = *args;
    int rc = check_rotary(ctx, x.dtype, x.tokens, x.head_dim, x.rot_dim, x.positions_dev, x.id_bytes, x.turns_dev, x.magnitude);
    if (rc == FQ_OK) rc = check_pair(&x.q, &x.q_out, x.dtype, x.tokens, x.head_dim);
    if (rc == FQ_OK) rc = check_source(&x.k, x.dtype);
    if (rc == FQ_OK) rc = check_source(&x.v, x.dtype);
    if (rc == FQ_OK) rc = check_cache(&x.cache, x.dtype, x.head_dim);
    if (rc != FQ_OK) return rc;
    if (!x.slots_dev) return FQ_ERR_ARG;
    if (x.k.heads != x.cache.heads || x.v.heads != x.cache.heads) return FQ_ERR_SHAPE;
    if (!aligned(x.slots_dev, 8)) return FQ_ERR_ALIGN;
    if (x.q_out.dev == x.k.dev || x.q_out.dev == x.v.dev || x.cache.k_dev == x.cache.v_dev) return FQ_ERR_ARG;
    RotaryArgs a{};
    a.t[0] = tensor(&x.q, &x.q_out, x.tokens, x.rot_dim);
    a.t[1] = to_cache(&x.k, &x.cache, x.tokens, x.rot_dim);
    a.t[2] = to_cache(&x.v, &x.cache, x.tokens, 0);
    a.n = 3; a.head_dim = x.head_dim; a.half = x.rot_dim / 2;
    a.positions = x.positions_dev; a.wide_positions = x.id_bytes == 8; a.turns = x.turns_dev;
    a.magnitude = x.magnitude; a.side = 1.0f; a.status = ctx->status_dev;
    a.slots = x.slots_dev; a.cache[0] = x.cache.k_dev; a.cache[1] = x.cache.v_dev;
    a.block_stride = x.cache.block_stride; a.token_stride = x.cache.token_stride; a.block_size = x.cache.block_size;
    a.n_slots = (long long)x.cache.blocks * x.cache.block_size;
    return launch_rotary(ctx, a, x.dtype, x.tokens, x.rot_dim, x.interleaved, (cudaStream_t)stream);
}

}  // extern "C"
