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
// most 19 roundings in a row) and from there on in fp64: one fp64 addition per 32 or
// 64 elements, which the few fp64 units keep up with.  Where such a sum leaves the
// range in which fp32 squares are exact enough, the vectors are read again (from L2)
// and squared in fp64; all-zero vectors, most of an embedding's gradient, are told
// apart before that.
#include <math.h>

#include "optim.cuh"

namespace aspis {

namespace {

constexpr int kWarps = kOptThreads / 32;
constexpr int kVecs = 8;                          // 16-byte vectors in flight per thread

__device__ __forceinline__ double warp_sum(double x)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_down_sync(0xFFFFFFFFu, x, o);
    return x;
}

// the block's sum, in thread 0
__device__ __forceinline__ double block_sum(double x, double *sh)
{
    x = warp_sum(x);
    __syncthreads();                              // sh free again
    if (threadIdx.x % 32 == 0) sh[threadIdx.x / 32] = x;
    __syncthreads();
    if (threadIdx.x == 0)
        for (int w = 1; w < kWarps; ++w) x += sh[w];
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
__device__ __forceinline__ double sum_vectors(const uint4 *base, int64_t a, int64_t b)
{
    double acc = 0;
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
        float s[4] = {};
#pragma unroll
        for (int u = 0; u < kVecs; ++u) add_squares<TYPE>(s, r[u]);
        const float sum = (s[0] + s[1]) + (s[2] + s[3]);
        // fp16 squares lie between 3.6e-15 and 4.3e9
        if (TYPE == ASPIS_F16 || (sum >= 1e-30f && sum <= 3e38f)) {
            acc += sum;
            continue;
        }
        uint32_t any = 0;
#pragma unroll
        for (int u = 0; u < kVecs; ++u) any |= (r[u].x | r[u].y) | (r[u].z | r[u].w);
        if ((any & (TYPE == ASPIS_F32 ? 0x7FFFFFFFu : 0x7FFF7FFFu)) == 0) continue;
#pragma unroll 1
        for (int u = 0; u < kVecs && v + u * kOptThreads < b; ++u)
            acc += exact_squares<TYPE>(__ldg(base + v + u * kOptThreads));
    }
    return acc;
}

// One thread's share of units [ua, ub) of a tensor.  Vectors are counted from the 16-byte
// boundary at or before its first element; those that it fills only in part, at either end, are
// read element by element.
template <int TYPE>
__device__ __forceinline__ double sum_units(const void *p, int64_t numel, uint32_t ua, uint32_t ub)
{
    constexpr int per = 16 / type_bytes(TYPE);
    const int h = (int)((uintptr_t)p % 16) / type_bytes(TYPE);
    const uint4 *base = reinterpret_cast<const uint4 *>((uintptr_t)p - h * type_bytes(TYPE));
    const int64_t full = (h + numel) / per;                  // vectors before this one end inside the tensor
    const int64_t a = (int64_t)ua * kOptThreads, b = (int64_t)ub * kOptThreads;
    double acc = sum_vectors<TYPE>(base, max(a, (int64_t)(h > 0)), min(b, full));
    const int64_t head = h > 0 ? min((int64_t)(per - h), numel) : 0;
    if (threadIdx.x < 8) {
        const int64_t i = threadIdx.x, j = max(full * per - h, head) + threadIdx.x;
        if (ua == 0 && i < head) {
            const double x = load_one<type_bytes(TYPE)>(p, i, TYPE == ASPIS_BF16);
            acc += x * x;
        }
        if (a <= full && full < b && j < numel) {
            const double x = load_one<type_bytes(TYPE)>(p, j, TYPE == ASPIS_BF16);
            acc += x * x;
        }
    }
    return acc;
}

template <int N>
__global__ void __launch_bounds__(kOptThreads)
norm_kernel(const __grid_constant__ Table<GradEntry, N> t, float scale, float *norm, float *tensor_norms,
            NormWork *work, bool chained, uint32_t stretch)
{
    __shared__ double sh[kWarps];
    __shared__ double parts[kMaxGrid + N];
    __shared__ bool last;
    if (chained) chain();
    const uint32_t grid = gridDim.x, b = blockIdx.x;
    double acc = 0;
    // stretch 0: one run of units for each block, else runs of so many units dealt in turn
    uint32_t u = stretch ? b * stretch : run_begin(t.units, b, grid);
    while (u < t.units) {
        const uint32_t end = stretch ? min(u + stretch, t.units) : run_begin(t.units, b + 1, grid);
        for (int k = entry_of(t, u); u < end; ++k) {
            const GradEntry &e = t.e[k];
            const uint32_t stop = min(end, e.end), ua = u - e.begin, ub = stop - e.begin;
            acc += e.type() == ASPIS_F32    ? sum_units<ASPIS_F32>(e.in, e.numel(), ua, ub)
                   : e.type() == ASPIS_BF16 ? sum_units<ASPIS_BF16>(e.in, e.numel(), ua, ub)
                                            : sum_units<ASPIS_F16>(e.in, e.numel(), ua, ub);
            if (tensor_norms) {
                acc = block_sum(acc, sh);
                if (threadIdx.x == 0) {
                    work->part[b + k] = acc;
                    if (u == e.begin) work->first[k] = (uint16_t)b;
                    if (stop == e.end) work->last[k] = (uint16_t)b;
                }
                acc = 0;
            }
            u = stop;
        }
        if (!stretch) break;
        u += (grid - 1) * stretch;
    }
    if (!tensor_norms) {
        acc = block_sum(acc, sh);
        if (threadIdx.x == 0) work->part[b] = acc;
    }
    // the last block adds up
    if (threadIdx.x == 0) {
        __threadfence();
        last = atomicAdd(&work->done, 1u) == grid - 1;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    double sum = 0;
    if (!tensor_norms) {
        for (uint32_t q = threadIdx.x; q < grid; q += kOptThreads) sum += __ldcg(&work->part[q]);
    } else {
        for (uint32_t q = threadIdx.x; q < grid + t.n; q += kOptThreads) parts[q] = __ldcg(&work->part[q]);
        __syncthreads();
        // a thread per tensor that few blocks met, a warp per tensor that many did
        for (int pass = 0; pass < 2; ++pass) {
            const int lanes = pass ? 32 : 1, lane = threadIdx.x % lanes;
            for (int k = threadIdx.x / lanes; k < t.n; k += kOptThreads / lanes) {
                const int b0 = __ldcg(&work->first[k]), b1 = __ldcg(&work->last[k]);
                if ((b1 - b0 >= 16) != (pass == 1)) continue;
                double x = 0;
                for (int q = b0 + lane; q <= b1; q += lanes) x += parts[q + k];
                if (pass) x = warp_sum(x);
                if (lane == 0) {
                    tensor_norms[t.first + k] = (float)(sqrt(x) * scale);
                    sum += x;
                }
            }
        }
    }
    sum = block_sum(sum, sh);
    if (threadIdx.x == 0) {
        if (t.first) sum += work->before;
        work->before = sum;
        work->done = 0;
        if (t.last) *norm = (float)(sqrt(sum) * scale);
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
