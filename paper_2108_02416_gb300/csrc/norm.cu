// aspis_grad_norm: the global norm of many tensors.
//
// One kernel reads every element once.  A block takes a contiguous run of units,
// adds the squares of each tensor that it meets and leaves one partial sum per
// (block, tensor).  The pairs that occur form a staircase (a later block starts
// no earlier than at the earlier one's last tensor), so block + tensor numbers
// them without gaps that collide, and the last block to finish adds the partial
// sums of every tensor in the order of the blocks: the result depends on the
// lengths and the grid alone, not on which block finished first.
#include <math.h>

#include "optim.cuh"

namespace aspis {

namespace {

constexpr int kWarps = kOptThreads / 32;

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

template <int N>
__global__ void __launch_bounds__(kOptThreads)
norm_kernel(const __grid_constant__ Table<GradEntry, N> t, float scale, float *norm, float *tensor_norms,
            NormWork *work)
{
    __shared__ double sh[kWarps];
    __shared__ bool last;
    chain();
    const uint32_t grid = gridDim.x, b = blockIdx.x;
    uint32_t u = run_begin(t.units, b, grid);
    const uint32_t end = run_begin(t.units, b + 1, grid);
    for (int k = u < end ? entry_of(t, u) : 0; u < end; ++k) {
        const GradEntry &e = t.e[k];
        const uint32_t before = k ? t.e[k - 1].unit_end : 0, stop = min(end, e.unit_end);
        if (stop <= u) continue;                  // an empty tensor
        const int unit = grad_unit(e.type);
        const int64_t i1 = min((int64_t)(stop - before) * unit, e.numel);
        double acc = 0;
        for (int64_t i = (int64_t)(u - before) * unit + threadIdx.x; i < i1; i += kOptThreads) {
            const double x = load_as_float(e.in, i, e.type);
            acc += x * x;
        }
        acc = block_sum(acc, sh);
        if (threadIdx.x == 0) work->part[b + k] = acc;
        u = stop;
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
    for (int k = threadIdx.x; k < t.n; k += kOptThreads) {
        const uint32_t u0 = k ? t.e[k - 1].unit_end : 0, u1 = t.e[k].unit_end;
        double x = 0;
        if (u1 > u0) {
            const uint32_t b0 = (uint32_t)(((uint64_t)(u0 + 1) * grid - 1) / t.units);
            const uint32_t b1 = (uint32_t)(((uint64_t)u1 * grid - 1) / t.units);
            for (uint32_t q = b0; q <= b1; ++q) x += __ldcg(&work->part[q + k]);
        }
        if (tensor_norms) tensor_norms[t.first + k] = (float)(sqrt(x) * scale);
        sum += x;
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
    void *args[] = {(void *)&t, &scale, &norm, &tensor_norms, &work};   // the kernel's table is a prefix of t
    return cudaLaunchKernel((const void *)norm_kernel<N>, dim3((unsigned)grid), dim3(kOptThreads), args, 0, stream);
}

}  // namespace

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
