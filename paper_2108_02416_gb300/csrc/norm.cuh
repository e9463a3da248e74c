// Sums of squares over many tensors: what the norm's own kernel and those that take the norm on
// their way share.
//
// Squares are added in fp32 over the eight 16-byte vectors that a thread holds (at
// most 19 roundings in a row), and these sums as pairs of fp32 numbers, whose lower
// one holds the rounding errors of the upper one: 48 bits without the fp64 units, which are few on
// this chip (with fp64 sums the norm of a ResNet-18's 62 tensors took 27 us, with these 21).  Where the sum over a thread's vectors
// leaves [1e-30, 1e24], outside of which fp32 squares or their sum might vanish or overflow, the
// vectors are read again (from L2) and squared and added in fp64; all-zero vectors, most of an
// embedding's gradient, are told apart before that.
#pragma once

#include <math.h>

#include "optim.cuh"

namespace aspis {

constexpr int kVecs = 8;                          // 16-byte vectors in flight per thread
constexpr int kMostPolls = 1 << 22;               // of a wait for the other blocks
constexpr uint32_t kWide = 1u << 16;              // in the count of blocks that are done: one had an fp64 sum

// a + b exactly, as a rounded sum and its error
struct Pair {
    float hi, lo;

    __device__ __forceinline__ Pair(float h = 0, float l = 0) : hi(h), lo(l) {}

    __device__ __forceinline__ void add(float x)
    {
        const float s = __fadd_rn(hi, x), y = __fsub_rn(s, hi);
        lo = __fadd_rn(lo, __fadd_rn(__fsub_rn(hi, __fsub_rn(s, y)), __fsub_rn(x, y)));
        hi = s;
    }
    __device__ __forceinline__ void add(const Pair &p)
    {
        add(p.hi);
        lo = __fadd_rn(lo, p.lo);
    }
    __device__ __forceinline__ double value() const { return (double)hi + lo; }
};

// what a thread has added: in pairs, and what needed fp64
struct Sum {
    Pair p;
    double wide = 0;
};

__device__ __forceinline__ bool in_range(float s) { return s >= 1e-30f && s <= 1e24f; }

__device__ __forceinline__ void add_square(Sum &sum, float x)
{
    const float s = x * x;
    if (in_range(s))
        sum.p.add(s);
    else if (x != 0.0f)
        sum.wide += (double)x * x;
}

// sums over groups of LANES threads, in each group's first
template <int LANES>
__device__ __forceinline__ Pair group_sum(Pair x)
{
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) {
        Pair y;
        y.hi = __shfl_down_sync(0xFFFFFFFFu, x.hi, o, LANES);
        y.lo = __shfl_down_sync(0xFFFFFFFFu, x.lo, o, LANES);
        x.add(y);
    }
    return x;
}

template <int LANES>
__device__ __forceinline__ double group_sum(double x)
{
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) x += __shfl_down_sync(0xFFFFFFFFu, x, o, LANES);
    return x;
}

// the block's sum, in thread 0
template <class T>
__device__ __forceinline__ T block_sum(T x, T *sh)
{
    x = group_sum<32>(x);
    if (threadIdx.x % 32 == 0) sh[threadIdx.x / 32] = x;
    __syncthreads();
    if (threadIdx.x < 32) x = group_sum<kWarps>(sh[threadIdx.x % kWarps]);
    return x;
}

template <int TYPE>
__device__ __forceinline__ float2 pair(uint32_t w)
{
    return unpack(w, TYPE == ASPIS_BF16);
}

// a vector's squares added to four sums
template <int TYPE>
__device__ __forceinline__ void add_squares(float (&s)[4], const uint4 &v)
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (TYPE == ASPIS_F32) {
            const float x = __uint_as_float(w[i]);
            s[i] = fmaf(x, x, s[i]);
        } else {
            const float2 x = pair<TYPE>(w[i]);
            s[i] = fmaf(x.x, x.x, s[i]);
            s[i] = fmaf(x.y, x.y, s[i]);
        }
    }
}

template <int TYPE>
__device__ __forceinline__ double exact_squares(const uint4 &v)
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    double s = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (TYPE == ASPIS_F32) {
            const double x = __uint_as_float(w[i]);
            s = fma(x, x, s);
        } else {
            const float2 x = pair<TYPE>(w[i]);
            s = fma((double)x.x, (double)x.x, s);
            s = fma((double)x.y, (double)x.y, s);
        }
    }
    return s;
}

// How gradients are read: plainly (a cooperative kernel may write what it has summed), or with L2's
// policy for them.
struct PlainLoad {
    __device__ __forceinline__ uint4 operator()(const uint4 *p) const { return *p; }
};

struct PolicyLoad {
    uint64_t policy;

    __device__ __forceinline__ uint4 operator()(const uint4 *p) const
    {
        uint4 v;
        asm volatile("ld.global.L2::cache_hint.v4.u32 {%0,%1,%2,%3}, [%4], %5;"
                     : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                     : "l"(p), "l"(policy));
        return v;
    }
};

// The squares of the eight vectors v, v + TEAM, ... (those before b) of a tensor (base: 16-byte aligned),
// which stay in r (zeros beyond b).
template <int TYPE, int TEAM, class L>
__device__ __forceinline__ void sum_batch(Sum &sum, const uint4 *base, int64_t v, int64_t b, L load, uint4 (&r)[kVecs])
{
    if (v + (kVecs - 1) * TEAM < b) {
#pragma unroll
        for (int u = 0; u < kVecs; ++u) r[u] = load(base + v + u * TEAM);
    } else {
#pragma unroll
        for (int u = 0; u < kVecs; ++u) r[u] = v + u * TEAM < b ? load(base + v + u * TEAM) : make_uint4(0, 0, 0, 0);
    }
    float q[4] = {};
#pragma unroll
    for (int u = 0; u < kVecs; ++u) add_squares<TYPE>(q, r[u]);
    const float s = (q[0] + q[1]) + (q[2] + q[3]);
    // fp16 squares lie between 3.6e-15 and 4.3e9
    if (TYPE == ASPIS_F16 ? s <= 1e24f : in_range(s)) {
        sum.p.add(s);
        return;
    }
    uint32_t any = 0;
#pragma unroll
    for (int u = 0; u < kVecs; ++u) any |= (r[u].x | r[u].y) | (r[u].z | r[u].w);
    if ((any & (TYPE == ASPIS_F32 ? 0x7FFFFFFFu : 0x7FFF7FFFu)) == 0) return;
#pragma unroll 1
    for (int u = 0; u < kVecs && v + u * TEAM < b; ++u) sum.wide += exact_squares<TYPE>(base[v + u * TEAM]);
}

// A tensor's vectors are counted from a 16-byte boundary h elements before its first one: the last such
// boundary, or the 32-byte one (h up to 7), where clipping counts groups of eight fp32 values from that.
template <int TYPE>
struct Vectors {
    static constexpr int size = type_bytes(TYPE), per = 16 / size;
    const void *p;
    int64_t numel;
    int h;
    int first;                    // the first vector that begins inside the tensor
    int64_t full;                 // vectors before this one end inside the tensor

    __device__ __forceinline__ Vectors(const void *q, int64_t n, int before)
        : p(q), numel(n), h(before), first((h + per - 1) / per), full((h + n) / per)
    {
    }
    __device__ __forceinline__ const uint4 *base() const
    {
        return reinterpret_cast<const uint4 *>((uintptr_t)p - h * size);
    }
    // f of each element of [a, b) in a vector that the tensor fills only in part, at either end
    template <class F>
    __device__ __forceinline__ void ends(int64_t a, int64_t b, int rank, F f) const
    {
        if (rank >= 8) return;
        const int64_t head = min((int64_t)(first * per - h), numel);
        const int64_t i = rank, j = max(full * per - h, head) + rank;
        if (a == 0 && i < head) f(i);
        if (a <= full && full < b && j < numel) f(j);
    }
};

// h: the boundary at or before the first element
struct VectorOrigin {
    template <int TYPE>
    __device__ __forceinline__ static int of(const GradEntry &e)
    {
        return (int)((uintptr_t)e.in % 16) / type_bytes(TYPE);
    }
};

// One thread's share (rank of TEAM) of the vectors [a, b) of a tensor.
template <int TYPE, int TEAM, class L>
__device__ __forceinline__ void sum_range(Sum &sum, const Vectors<TYPE> &t, int64_t a, int64_t b, int rank, L load)
{
    const int64_t end = min(b, t.full);
    for (int64_t v = max(a, (int64_t)t.first) + rank; v < end; v += kVecs * TEAM) {
        uint4 r[kVecs];
        sum_batch<TYPE, TEAM>(sum, t.base(), v, end, load, r);
    }
    t.ends(a, b, rank, [&](int64_t i) { add_square(sum, load_one<t.size>(t.p, i, TYPE == ASPIS_BF16)); });
}

template <int TEAM, class O = VectorOrigin, class L = PlainLoad>
__device__ __forceinline__ void sum_range(Sum &sum, const GradEntry &e, int64_t a, int64_t b, int rank, L load = L())
{
    if (e.type() == ASPIS_F32)
        sum_range<ASPIS_F32, TEAM>(sum, Vectors<ASPIS_F32>(e.in, e.numel(), O::template of<ASPIS_F32>(e)), a, b, rank, load);
    else if (e.type() == ASPIS_BF16)
        sum_range<ASPIS_BF16, TEAM>(sum, Vectors<ASPIS_BF16>(e.in, e.numel(), O::template of<ASPIS_BF16>(e)), a, b, rank, load);
    else
        sum_range<ASPIS_F16, TEAM>(sum, Vectors<ASPIS_F16>(e.in, e.numel(), O::template of<ASPIS_F16>(e)), a, b, rank, load);
}

// The block's sum, in thread 0; true (in every thread) where something needed fp64.
struct BlockSums {
    Pair pairs[kWarps];
    double wides[kWarps];
};

__device__ __forceinline__ bool reduce(Sum &sum, BlockSums &sh)
{
    const bool wide = __syncthreads_or(!(sum.wide == 0));
    sum.p = block_sum(sum.p, sh.pairs);
    if (wide) sum.wide = block_sum(sum.wide, sh.wides);
    return wide;
}

// The sum of the blocks' partial sums, in thread 0: loaded all before the first is added.
__device__ __forceinline__ void collect(Sum &sum, const NormWork *work, uint32_t grid, bool wide, BlockSums &sh)
{
    constexpr int most = kMaxGrid / kOptThreads;
    float2 x[most];
#pragma unroll
    for (int i = 0; i < most; ++i) {
        const uint32_t q = threadIdx.x + i * kOptThreads;
        x[i] = q < grid ? __ldcg(&work->pair[q]) : make_float2(0, 0);
    }
    sum = Sum();
#pragma unroll
    for (int i = 0; i < most; ++i) sum.p.add(Pair(x[i].x, x[i].y));
    if (wide)
        for (uint32_t q = threadIdx.x; q < grid; q += kOptThreads) sum.wide += __ldcg(&work->wide[q]);
    reduce(sum, sh);
}

// scale * sqrt(sum)
__device__ __forceinline__ float root(const Sum &sum, bool wide, float scale)
{
    if (wide) return (float)(sqrt(sum.p.value() + sum.wide) * scale);
    return sqrtf(sum.p.hi + sum.p.lo) * scale;
}

// The norm inside a cooperative kernel: every block brings its sum and leaves with the norm of all,
// which every block adds up by itself, in the same order.  The wait is bounded (seconds); false
// where it ran out, and then the norm is NaN and the block has nothing more to do.
__device__ __forceinline__ bool meet(Sum &sum, float scale, NormWork *work, float &norm)
{
    __shared__ BlockSums sh;
    __shared__ float result;
    __shared__ uint32_t done;
    const uint32_t grid = gridDim.x, b = blockIdx.x;
    bool wide = reduce(sum, sh);
    if (grid > 1) {
        if (threadIdx.x == 0) {
            work->pair[b] = make_float2(sum.p.hi, sum.p.lo);
            work->wide[b] = wide ? sum.wide : 0.0;
            asm volatile("red.release.gpu.global.add.u32 [%0], %1;" ::"l"(&work->done), "r"(wide ? kWide + 1 : 1u)
                         : "memory");
            uint32_t seen = 0;
            for (int i = 0; i < kMostPolls; ++i) {
                asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(seen) : "l"(&work->done) : "memory");
                if (seen % kWide == grid) break;
            }
            done = seen;
        }
        __syncthreads();
        if (done % kWide != grid) {
            norm = __int_as_float(0x7FFFFFFF);
            return false;
        }
        wide = done >= kWide;
        collect(sum, work, grid, wide, sh);
    }
    if (threadIdx.x == 0) {
        result = root(sum, wide, scale);
        // the last block to have seen the count clears it for the next call
        if (grid > 1 && atomicAdd(&work->left, 1u) == grid - 1) {
            work->done = 0;
            work->left = 0;
        }
    }
    __syncthreads();
    norm = result;
    return true;
}

}  // namespace aspis
