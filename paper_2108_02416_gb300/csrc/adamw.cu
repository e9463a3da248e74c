// aspis_adamw: the norm (norm.cu), then one AdamW step on every tensor with the
// gradient read through the clipping coefficient.  The step streams every array once, eight
// elements per thread and access, and is bound by HBM.
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

__device__ __forceinline__ void step_one(const Step &s, float c, float decay, float g, float &x, float &m, float &v)
{
    const float h = g * c;
    m = fmaf(s.beta1, m, s.one_beta1 * h);
    v = fmaf(s.beta2, v, s.one_beta2 * h * h);
    x -= fmaf(decay, x, s.rate * (m / fmaf(sqrtf(v), s.root, s.eps)));
}

// Element i alone.
template <int BP, int BG, bool MASTER>
__device__ __forceinline__ void step_element(const ParamEntry &e, const Step &s, float c, float decay, int64_t i, bool bp,
                                             bool bg)
{
    float x = MASTER ? e.master[i] : load_one<BP>(e.param, i, bp), m = e.m[i], v = e.v[i];
    step_one(s, c, decay, load_one<BG>(e.grad, i, bg), x, m, v);
    e.m[i] = m;
    e.v[i] = v;
    if (MASTER) e.master[i] = x;
    store_one<BP>(e.param, i, x, bp);
}

// Units [ua, ub) of a tensor: groups of eight elements, one per thread, counted from the group
// boundary at or before the first moment's first element.  The gradient may lie behind that boundary by
// any number of elements (a view of a flat aggregate); arrays that are written and do not share
// it are taken element by element.
template <int BP, int BG, bool MASTER>
__device__ __forceinline__ void step_units(const ParamEntry &e, const Step &s, float c, uint32_t ua, uint32_t ub, bool bp,
                                           bool bg)
{
    const float decay = s.lr * e.decay;
    const int h = behind<4>(e.m);
    const int64_t first = (int64_t)ua * kParamUnit, last = (int64_t)ub * kParamUnit;
    if (behind<4>(e.v) != h || behind<BP>(e.param) != h || (MASTER && behind<4>(e.master) != h)) {
        for (int64_t i = first + threadIdx.x; i < min(last, e.numel); i += kOptThreads)
            step_element<BP, BG, MASTER>(e, s, c, decay, i, bp, bg);
        return;
    }
    const char *grad = static_cast<const char *>(e.grad);
    char *param = static_cast<char *>(e.param);
    const int shift = behind<BG>(grad - h * BG);
    const int64_t end = min(last / 8, (e.numel + h + 7) / 8);
    for (int64_t q = first / 8 + threadIdx.x; q < end; q += kOptThreads) {
        const int64_t i = q * 8 - h;
        if (i >= shift && i + (shift ? 16 - shift : 8) <= e.numel) {
            float g[8], x[8], m[8], v[8];
            const Raw<4> rm = load_raw(e.m + i, (Raw<4> *)nullptr), rv = load_raw(e.v + i, (Raw<4> *)nullptr);
            if constexpr (MASTER)
                to_floats(load_raw(e.master + i, (Raw<4> *)nullptr), false, x);
            else
                to_floats(load_raw(param + i * BP, (Raw<BP> *)nullptr), bp, x);
            if (shift == 0)
                to_floats(load_raw(grad + i * BG, (Raw<BG> *)nullptr), bg, g);
            else
                to_floats(load_shifted<BG>(grad + (i - shift) * BG, shift), bg, g);
            to_floats(rm, false, m);
            to_floats(rv, false, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) step_one(s, c, decay, g[j], x[j], m[j], v[j]);
            store_floats<4>(e.m + i, m, false);
            store_floats<4>(e.v + i, v, false);
            if constexpr (MASTER) store_floats<4>(e.master + i, x, false);
            store_floats<BP>(param + i * BP, x, bp);
        } else {
            for (int64_t j = max(i, (int64_t)0); j < min(i + 8, e.numel); ++j)
                step_element<BP, BG, MASTER>(e, s, c, decay, j, bp, bg);
        }
    }
}

template <int BP, int BG, bool MASTER, int N>
__global__ void __launch_bounds__(kOptThreads, 4)
adamw_kernel(const __grid_constant__ Table<ParamEntry, N> t, const __grid_constant__ Step s, bool bp, bool bg, bool chained)
{
    if (chained) chain();
    float c = s.scale;
    if (s.norm) {
        const float norm = *s.norm;
        if (s.skip && !isfinite(norm)) return;
        c *= clip_coef(norm, s.max_norm);
    }
    const uint32_t u = gridDim.x - 1 - blockIdx.x;        // backwards: L2 still holds what the norm read last
    const ParamEntry &e = t.e[entry_of(t, u)];
    step_units<BP, BG, MASTER>(e, s, c, u - e.begin, u - e.begin + 1, bp, bg);
}

template <int BP, int BG, bool MASTER>
cudaError_t launch(const ParamTable &t, Step s, bool bp, bool bg, bool chained, cudaStream_t stream)
{
    void *args[] = {(void *)&t, &s, &bp, &bg, &chained};
    return launch_table(t.n <= kParamsSmall ? (const void *)adamw_kernel<BP, BG, MASTER, kParamsSmall>
                                            : (const void *)adamw_kernel<BP, BG, MASTER, kParams>,
                        t.units, args, chained, stream);
}

cudaError_t launch(const aspis_params::Group &g, const ParamTable &t, const Step &s, bool chained, cudaStream_t stream)
{
    const bool bp = g.param_type == ASPIS_BF16, bg = g.grad_type == ASPIS_BF16, wide = g.grad_type == ASPIS_F32;
    if (g.param_type == ASPIS_F32)
        return wide ? launch<4, 4, false>(t, s, bp, bg, chained, stream) : launch<4, 2, false>(t, s, bp, bg, chained, stream);
    if (g.master)
        return wide ? launch<2, 4, true>(t, s, bp, bg, chained, stream) : launch<2, 2, true>(t, s, bp, bg, chained, stream);
    return wide ? launch<2, 4, false>(t, s, bp, bg, chained, stream) : launch<2, 2, false>(t, s, bp, bg, chained, stream);
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
    bool chained = normed && work;
    for (auto g = params->groups.rbegin(); g != params->groups.rend(); ++g)
        for (auto t = g->tables.rbegin(); t != g->tables.rend(); ++t) {
            if (err != cudaSuccess) return ASPIS_E_CUDA;
            err = launch(*g, **t, s, chained, st);
            chained = true;
        }
    return err == cudaSuccess ? ASPIS_OK : ASPIS_E_CUDA;
}
