// aspis_clip_grads: the norm (norm.cu), then every gradient times s * c.
#include <math.h>

#include "optim.cuh"

using namespace aspis;

namespace {

template <int N>
__global__ void __launch_bounds__(kOptThreads)
scale_kernel(const __grid_constant__ Table<GradEntry, N> t, float max_norm, float scale, const float *norm)
{
    chain();
    const float c = scale * clip_coef(*norm, max_norm);
    uint32_t u = run_begin(t.units, blockIdx.x, gridDim.x);
    const uint32_t end = run_begin(t.units, blockIdx.x + 1, gridDim.x);
    for (int k = u < end ? entry_of(t, u) : 0; u < end; ++k) {
        const GradEntry &e = t.e[k];
        const uint32_t before = k ? t.e[k - 1].unit_end : 0, stop = min(end, e.unit_end);
        if (stop <= u) continue;
        const int unit = grad_unit(e.type);
        const int64_t i1 = min((int64_t)(stop - before) * unit, e.numel);
        if (c != 1.0f || e.in != e.out)
            for (int64_t i = (int64_t)(u - before) * unit + threadIdx.x; i < i1; i += kOptThreads)
                store_rounded(e.out, i, e.out_type, load_as_float(e.in, i, e.type) * c);
        u = stop;
    }
}

template <int N>
cudaError_t launch(const GradTable &t, float max_norm, float scale, const float *norm, cudaStream_t stream)
{
    int64_t grid = (int64_t)sm_count() * 8;
    if (grid > t.units) grid = t.units;
    if (grid == 0) return cudaSuccess;
    void *args[] = {(void *)&t, &max_norm, &scale, &norm};
    return cudaLaunchKernel((const void *)scale_kernel<N>, dim3((unsigned)grid), dim3(kOptThreads), args, 0, stream);
}

}  // namespace

extern "C" aspis_status aspis_clip_grads(const aspis_tensors *grads, float max_norm, float scale, float *norm,
                                         void *work, void *stream)
{
    if (!grads || !norm || !(scale > 0.0f) || isinf(scale) || !(max_norm >= 0.0f) || !grads->apart)
        return ASPIS_E_INVAL;
    if ((uintptr_t)work % 16 != 0 || (uintptr_t)norm % 4 != 0) return ASPIS_E_ALIGN;
    const cudaStream_t st = (cudaStream_t)stream;
    cudaError_t e = work ? launch_grad_norm(grads->tables, scale, norm, nullptr, work, st) : cudaSuccess;
    for (const auto &t : grads->tables) {
        if (e != cudaSuccess) break;
        e = t->n <= kGradsSmall ? launch<kGradsSmall>(*t, max_norm, scale, norm, st)
            : t->n <= kGradsMid ? launch<kGradsMid>(*t, max_norm, scale, norm, st)
                                : launch<kGrads>(*t, max_norm, scale, norm, st);
    }
    return e == cudaSuccess ? ASPIS_OK : ASPIS_E_CUDA;
}
