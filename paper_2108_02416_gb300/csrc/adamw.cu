// aspis_adamw: the norm (norm.cu), then one AdamW step on every tensor with the
// gradient read through the clipping coefficient.
#include <math.h>

#include "optim.cuh"

using namespace aspis;

namespace {

struct Step {
    float beta1, one_beta1, beta2, one_beta2;
    float lr;
    float rate;                   // lr / (1 - beta1^step)
    float root;                   // 1 / sqrt(1 - beta2^step)
    float eps;
    float max_norm, scale;
    const float *norm;            // or NULL
    int skip;
};

template <int N>
__global__ void __launch_bounds__(kOptThreads)
adamw_kernel(const __grid_constant__ Table<ParamEntry, N> t, const __grid_constant__ Step s, int param_type,
             int grad_type)
{
    chain();
    float c = s.scale;
    if (s.norm) {
        const float norm = *s.norm;
        if (s.skip && !isfinite(norm)) return;
        c *= clip_coef(norm, s.max_norm);
    }
    uint32_t u = run_begin(t.units, blockIdx.x, gridDim.x);
    const uint32_t end = run_begin(t.units, blockIdx.x + 1, gridDim.x);
    for (int k = u < end ? entry_of(t, u) : 0; u < end; ++k) {
        const ParamEntry &e = t.e[k];
        const uint32_t before = k ? t.e[k - 1].unit_end : 0, stop = min(end, e.unit_end);
        if (stop <= u) continue;
        const int64_t i1 = min((int64_t)(stop - before) * kParamUnit, e.numel);
        const float decay = s.lr * e.decay;
        for (int64_t i = (int64_t)(u - before) * kParamUnit + threadIdx.x; i < i1; i += kOptThreads) {
            const float h = load_as_float(e.grad, i, grad_type) * c;
            const float m = fmaf(s.beta1, e.m[i], s.one_beta1 * h);
            const float v = fmaf(s.beta2, e.v[i], s.one_beta2 * h * h);
            float x = e.master ? e.master[i] : load_as_float(e.param, i, param_type);
            x -= fmaf(decay, x, s.rate * (m / fmaf(sqrtf(v), s.root, s.eps)));
            e.m[i] = m;
            e.v[i] = v;
            if (e.master) e.master[i] = x;
            store_rounded(e.param, i, param_type, x);
        }
        u = stop;
    }
}

template <int N>
cudaError_t launch(const ParamTable &t, Step s, int param_type, int grad_type, cudaStream_t stream)
{
    int64_t grid = (int64_t)sm_count() * 8;
    if (grid > t.units) grid = t.units;
    if (grid == 0) return cudaSuccess;
    void *args[] = {(void *)&t, &s, &param_type, &grad_type};
    return cudaLaunchKernel((const void *)adamw_kernel<N>, dim3((unsigned)grid), dim3(kOptThreads), args, 0, stream);
}

}  // namespace

extern "C" aspis_status aspis_adamw(const aspis_params *params, const aspis_adamw_args *a, float *norm, void *work,
                                    void *stream)
{
    if (!params || !a || !isfinite(a->lr) || !(a->beta1 >= 0 && a->beta1 < 1) || !(a->beta2 >= 0 && a->beta2 < 1) ||
        !(a->eps >= 0) || isinf(a->eps) || a->step < 1 || isnan(a->max_norm) || !(a->scale > 0) || isinf(a->scale) ||
        a->reserved != 0)
        return ASPIS_E_INVAL;
    const bool normed = a->max_norm >= 0;
    if (normed ? !norm : (work || a->skip_nonfinite)) return ASPIS_E_INVAL;
    if ((uintptr_t)work % 16 != 0 || (uintptr_t)norm % 4 != 0) return ASPIS_E_ALIGN;
    Step s;
    s.beta1 = (float)a->beta1;
    s.one_beta1 = (float)(1 - a->beta1);
    s.beta2 = (float)a->beta2;
    s.one_beta2 = (float)(1 - a->beta2);
    s.lr = (float)a->lr;
    s.rate = (float)(a->lr / (1 - pow(a->beta1, (double)a->step)));
    s.root = (float)(1 / sqrt(1 - pow(a->beta2, (double)a->step)));
    s.eps = (float)a->eps;
    s.max_norm = a->max_norm;
    s.scale = a->scale;
    s.norm = normed ? norm : nullptr;
    s.skip = a->skip_nonfinite;
    const cudaStream_t st = (cudaStream_t)stream;
    cudaError_t err = normed && work ? launch_grad_norm(params->grads.tables, a->scale, norm, nullptr, work, st)
                                     : cudaSuccess;
    for (const auto &g : params->groups)
        for (const auto &t : g.tables) {
            if (err != cudaSuccess) return ASPIS_E_CUDA;
            err = t->n <= kParamsSmall ? launch<kParamsSmall>(*t, s, g.param_type, g.grad_type, st)
                                       : launch<kParams>(*t, s, g.param_type, g.grad_type, st);
        }
    return err == cudaSuccess ? ASPIS_OK : ASPIS_E_CUDA;
}
