// aspis_grad_norm: the global norm of many tensors.
//
// One kernel reads every element once.  A block takes a contiguous run of units,
// adds the squares of each tensor that it meets and leaves one partial sum per
// block, or, where the tensors' own norms are wanted, per (block, tensor).  The
// pairs that occur form a staircase (a later block starts no earlier than at the
// earlier one's last tensor), so block + tensor numbers them without collision.  The
// last block to finish adds the partial sums in their order: the result depends on
// the lengths and the grid alone, not on which block finished first.
//
// Squares are added in fp32 over the eight 16-byte vectors that a thread holds (at
// most 19 roundings in a row), and these sums as pairs of fp32 numbers, whose lower
// one holds the rounding errors of the upper one: 48 bits without the fp64 units, of which
// a multiprocessor has two (a warp's fp64 addition takes 16 cycles; with fp64 sums the norm of a
// ResNet-18's 62 tensors took 27 us).  Where the sum over a thread's vectors
// leaves [1e-30, 1e24], outside of which fp32 squares or their sum might vanish or overflow, the
// vectors are read again (from L2) and squared and added in fp64; all-zero vectors, most of an
// embedding's gradient, are told apart before that.
#include <math.h>

#include "optim.cuh"

namespace aspis {

namespace {

constexpr int kWarps = kOptThreads / 32;
constexpr int kVecs = 8;                          // 16-byte vectors in flight per thread
constexpr uint32_t kWide = 1u << 16;              // in the count of blocks that are done: one had an fp64 sum

// a + b exactly, as a rounded sum and its error
struct Pair {
    float hi = 0, lo = 0;

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

__device__ __forceinline__ Pair warp_sum(Pair x)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        Pair y;
        y.hi = __shfl_down_sync(0xFFFFFFFFu, x.hi, o);
        y.lo = __shfl_down_sync(0xFFFFFFFFu, x.lo, o);
        x.add(y);
    }
    return x;
}

__device__ __forceinline__ double warp_sum(double x)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_down_sync(0xFFFFFFFFu, x, o);
    return x;
}

// the block's sum, in thread 0
template <class T>
__device__ __forceinline__ T block_sum(T x, T *sh)
{
    x = warp_sum(x);
    __syncthreads();                              // sh free again
    if (threadIdx.x % 32 == 0) sh[threadIdx.x / 32] = x;
    __syncthreads();
    if (threadIdx.x < 32) {
        T y = threadIdx.x < kWarps ? sh[threadIdx.x] : T();
        x = warp_sum(y);
    }
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

// One thread's share of the vectors [a, b) of a tensor (base: 16-byte aligned).
template <int TYPE>
__device__ __forceinline__ void sum_vectors(Sum &sum, const uint4 *base, int64_t a, int64_t b)
{
    for (int64_t v = a + threadIdx.x; v < b; v += kVecs * kOptThreads) {
        uint4 r[kVecs];
        if (v + (kVecs - 1) * kOptThreads < b) {
#pragma unroll
            for (int u = 0; u < kVecs; ++u) r[u] = __ldg(base + v + u * kOptThreads);
        } else {
#pragma unroll
            for (int u = 0; u < kVecs; ++u)
                r[u] = v + u * kOptThreads < b ? __ldg(base + v + u * kOptThreads) : make_uint4(0, 0, 0, 0);
        }
        float q[4] = {};
#pragma unroll
        for (int u = 0; u < kVecs; ++u) add_squares<TYPE>(q, r[u]);
        const float s = (q[0] + q[1]) + (q[2] + q[3]);
        // fp16 squares lie between 3.6e-15 and 4.3e9
        if (TYPE == ASPIS_F16 ? s <= 1e24f : in_range(s)) {
            sum.p.add(s);
            continue;
        }
        uint32_t any = 0;
#pragma unroll
        for (int u = 0; u < kVecs; ++u) any |= (r[u].x | r[u].y) | (r[u].z | r[u].w);
        if ((any & (TYPE == ASPIS_F32 ? 0x7FFFFFFFu : 0x7FFF7FFFu)) == 0) continue;
#pragma unroll 1
        for (int u = 0; u < kVecs && v + u * kOptThreads < b; ++u)
            sum.wide += exact_squares<TYPE>(__ldg(base + v + u * kOptThreads));
    }
}

// One thread's share of units [ua, ub) of a tensor.  Vectors are counted from the 16-byte
// boundary at or before its first element; those that it fills only in part, at either end, are
// read element by element.
template <int TYPE>
__device__ __forceinline__ void sum_units(Sum &sum, const void *p, int64_t numel, uint32_t ua, uint32_t ub)
{
    constexpr int per = 16 / type_bytes(TYPE);
    const int h = (int)((uintptr_t)p % 16) / type_bytes(TYPE);
    const uint4 *base = reinterpret_cast<const uint4 *>((uintptr_t)p - h * type_bytes(TYPE));
    const int64_t full = (h + numel) / per;                  // vectors before this one end inside the tensor
    const int64_t a = (int64_t)ua * kOptThreads, b = (int64_t)ub * kOptThreads;
    sum_vectors<TYPE>(sum, base, max(a, (int64_t)(h > 0)), min(b, full));
    const int64_t head = h > 0 ? min((int64_t)(per - h), numel) : 0;
    if (threadIdx.x < 8) {
        const int64_t i = threadIdx.x, j = max(full * per - h, head) + threadIdx.x;
        if (ua == 0 && i < head) add_square(sum, load_one<type_bytes(TYPE)>(p, i, TYPE == ASPIS_BF16));
        if (a <= full && full < b && j < numel) add_square(sum, load_one<type_bytes(TYPE)>(p, j, TYPE == ASPIS_BF16));
    }
}

// The block's sum, in every thread of its first warp (the fp64 one in thread 0): true where something needed fp64.
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

// scale * sqrt(sum)
__device__ __forceinline__ float root(const Sum &sum, bool wide, float scale)
{
    if (wide) return (float)(sqrt(sum.p.value() + sum.wide) * scale);
    return sqrtf(sum.p.hi + sum.p.lo) * scale;
}

template <int N>
__global__ void __launch_bounds__(kOptThreads)
norm_kernel(const __grid_constant__ Table<GradEntry, N> t, float scale, float *norm, float *tensor_norms,
            NormWork *work, bool chained, uint32_t stretch)
{
    __shared__ BlockSums sh;
    __shared__ float2 parts[kMaxGrid + N];
    __shared__ uint16_t met[2][N];                // the first and the last block that met a tensor
    __shared__ uint32_t done;
    if (chained) chain();
    const uint32_t grid = gridDim.x, b = blockIdx.x;
    Sum sum;
    bool wide = false;
    // a partial sum: a pair, and in fp64 where that was needed (read only if a block says so)
    auto leave = [&](uint32_t slot) {
        wide |= reduce(sum, sh);
        if (threadIdx.x == 0) {
            work->pair[slot] = make_float2(sum.p.hi, sum.p.lo);
            work->wide[slot] = wide ? sum.wide : 0.0;
        }
        sum = Sum();
    };
    // stretch 0: one run of units for each block, else runs of so many units dealt in turn
    uint32_t u = stretch ? b * stretch : run_begin(t.units, b, grid);
    while (u < t.units) {
        const uint32_t end = stretch ? min(u + stretch, t.units) : run_begin(t.units, b + 1, grid);
        for (int k = entry_of(t, u); u < end; ++k) {
            const GradEntry &e = t.e[k];
            const uint32_t stop = min(end, e.end), ua = u - e.begin, ub = stop - e.begin;
            if (e.type() == ASPIS_F32)
                sum_units<ASPIS_F32>(sum, e.in, e.numel(), ua, ub);
            else if (e.type() == ASPIS_BF16)
                sum_units<ASPIS_BF16>(sum, e.in, e.numel(), ua, ub);
            else
                sum_units<ASPIS_F16>(sum, e.in, e.numel(), ua, ub);
            if (tensor_norms) {
                leave(b + k);
                if (threadIdx.x == 0) {
                    if (u == e.begin) work->first[k] = (uint16_t)b;
                    if (stop == e.end) work->last[k] = (uint16_t)b;
                }
            }
            u = stop;
        }
        if (!stretch) break;
        u += (grid - 1) * stretch;
    }
    if (!tensor_norms) leave(b);
    // the last block adds up
    if (threadIdx.x == 0) {
        __threadfence();
        done = atomicAdd(&work->done, wide ? kWide + 1 : 1u) + (wide ? kWide + 1 : 1u);
    }
    __syncthreads();
    if (done % kWide != grid) return;
    wide = done >= kWide;
    __threadfence();
    auto take = [&](Sum &to, uint32_t slot, float2 p) {
        Pair x;
        x.hi = p.x;
        x.lo = p.y;
        to.p.add(x);
        if (wide) to.wide += __ldcg(&work->wide[slot]);
    };
    if (!tensor_norms) {
        for (uint32_t q = threadIdx.x; q < grid; q += kOptThreads) take(sum, q, __ldcg(&work->pair[q]));
    } else {
        for (uint32_t q = threadIdx.x; q < grid + t.n; q += kOptThreads) parts[q] = __ldcg(&work->pair[q]);
        for (int k = threadIdx.x; k < t.n; k += kOptThreads) {
            met[0][k] = __ldcg(&work->first[k]);
            met[1][k] = __ldcg(&work->last[k]);
        }
        __syncthreads();
        // a thread per tensor that few blocks met, a warp per tensor that many did
        for (int pass = 0; pass < 2; ++pass) {
            const int lanes = pass ? 32 : 1, lane = threadIdx.x % lanes;
            for (int k = threadIdx.x / lanes; k < t.n; k += kOptThreads / lanes) {
                const int b0 = met[0][k], b1 = met[1][k];
                if ((b1 - b0 >= 16) != (pass == 1)) continue;
                Sum x;
                for (int q = b0 + lane; q <= b1; q += lanes) take(x, q + k, parts[q + k]);
                if (pass) {
                    x.p = warp_sum(x.p);
                    if (wide) x.wide = warp_sum(x.wide);
                }
                if (lane == 0) {
                    tensor_norms[t.first + k] = root(x, wide, scale);
                    sum.p.add(x.p);
                    sum.wide += x.wide;
                }
            }
        }
    }
    reduce(sum, sh);
    if (threadIdx.x == 0) {
        work->done = 0;
        if (!t.first && t.last) {
            *norm = root(sum, wide, scale);
        } else {                                  // one of several tables
            double all = sum.p.value() + sum.wide;
            if (t.first) all += work->before;
            work->before = all;
            if (t.last) *norm = (float)(sqrt(all) * scale);
        }
    }
}

template <int N>
cudaError_t launch(const GradTable &t, float scale, float *norm, float *tensor_norms, void *work,
                   cudaStream_t stream)
{
    int64_t grid = (int64_t)sm_count() * 4;
    if (grid > kMaxGrid) grid = kMaxGrid;
    if (grid > t.units) grid = t.units ? t.units : 1;
    bool chained = t.first > 0;
    uint32_t stretch = !tensor_norms && t.units >= 64 * (uint64_t)grid ? kVecs : 0;
    void *args[] = {(void *)&t, &scale, &norm, &tensor_norms, &work, &chained, &stretch};
    return launch_table((const void *)norm_kernel<N>, grid, args, chained, stream);
}

}  // namespace

cudaError_t launch_table(const void *kernel, int64_t grid, void **args, bool chained, cudaStream_t stream)
{
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3(kOptThreads);
    cfg.stream = stream;
    cfg.attrs = at;
    cfg.numAttrs = chained ? 1 : 0;
    return cudaLaunchKernelExC(&cfg, kernel, args);
}

cudaError_t launch_grad_norm(const std::vector<std::unique_ptr<GradTable>> &tables, float scale, float *norm,
                             float *tensor_norms, void *work, cudaStream_t stream)
{
    for (const auto &t : tables) {
        const cudaError_t e = t->n <= kGradsSmall ? launch<kGradsSmall>(*t, scale, norm, tensor_norms, work, stream)
                              : t->n <= kGradsMid ? launch<kGradsMid>(*t, scale, norm, tensor_norms, work, stream)
                                                  : launch<kGrads>(*t, scale, norm, tensor_norms, work, stream);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace aspis

using namespace aspis;

extern "C" aspis_status aspis_grad_norm(const aspis_tensors *grads, float scale, float *norm, float *tensor_norms,
                                        void *work, void *stream)
{
    if (!grads || !norm || !work || !(scale > 0.0f) || isinf(scale)) return ASPIS_E_INVAL;
    if ((uintptr_t)work % 16 != 0 || (uintptr_t)norm % 4 != 0 || (uintptr_t)tensor_norms % 4 != 0) return ASPIS_E_ALIGN;
    return launch_grad_norm(grads->tables, scale, norm, tensor_norms, work, (cudaStream_t)stream) == cudaSuccess
               ? ASPIS_OK
               : ASPIS_E_CUDA;
}
