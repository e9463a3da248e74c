// aspis_adamw: the norm (norm.cu), then one AdamW step on every tensor with the gradient read through the
// clipping coefficient.
//
//     h = s c g;  m <- b1 m + (1 - b1) h;  v <- b2 v + (1 - b2) h^2
//     x <- x - ( lr wd x + lr / (1 - b1^t) * m / ( sqrt(v) / sqrt(1 - b2^t) + eps ) )
//
// The step streams every array once and is bound by HBM: 28 bytes per parameter in fp32, or in 16 bits with master
// weights; 1.1 billion of the latter take 4.81 ms with the norm in front of them (31.9 + 2.3 GB: 7.1 TB/s).  A
// warp takes 256 parameters, eight per thread, with its four or five loads in flight, and a block eight
// such units: blocks that the hardware deals out in the order of the addresses stream faster than
// resident ones that walk runs of their own (234 million parameters: 1,031 us, and 1,136 with four blocks per
// multiprocessor).  Moments and masters are held in fp32; a 16-bit parameter is rounded to nearest once a step.
#include <math.h>

#include "optim.cuh"

using namespace aspis;

namespace {

template <int P, int G, bool M>
struct Types {
    static constexpr int param = P, grad = G;
    static constexpr bool master = M;
};

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

// A warp's unit of a tensor: groups of eight elements, one per thread, counted from the group
// boundary at or before the first moment's first element.  A 16-bit gradient may lie behind that
// boundary by any number of elements (it is shifted: 408 us for 100 million parameters with master weights, 425 taken
// element by element).  Where an fp32 gradient (a view of a flat aggregate) or an array that is written does not
// share it, neighbouring threads take neighbouring elements: 404 us for 100 million fp32 parameters, 401 aligned, 423 with
// the gradient shifted.
template <int BP, int BG, bool MASTER>
__device__ __forceinline__ void step_unit(const ParamEntry &e, const Step &s, float c, uint32_t unit, bool bp, bool bg)
{
    const float decay = s.lr * e.decay;
    const int lane = threadIdx.x % 32, h = behind<4>(e.m);
    const int64_t first = (int64_t)unit * kParamUnit;
    const char *grad = static_cast<const char *>(e.grad);
    const int shift = behind<BG>(grad - h * BG);
    if ((BG == 4 && shift) || behind<4>(e.v) != h || behind<BP>(e.param) != h || (MASTER && behind<4>(e.master) != h)) {
        if (first + kParamUnit <= e.numel) {
            float g[8], x[8], m[8], v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int64_t i = first + lane + 32 * j;
                g[j] = load_one<BG>(e.grad, i, bg);
                x[j] = MASTER ? e.master[i] : load_one<BP>(e.param, i, bp);
                m[j] = e.m[i];
                v[j] = e.v[i];
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int64_t i = first + lane + 32 * j;
                step_one(s, c, decay, g[j], x[j], m[j], v[j]);
                e.m[i] = m[j];
                e.v[i] = v[j];
                if (MASTER) e.master[i] = x[j];
                store_one<BP>(e.param, i, x[j], bp);
            }
            return;
        }
        for (int64_t i = first + lane; i < e.numel; i += 32) step_element<BP, BG, MASTER>(e, s, c, decay, i, bp, bg);
        return;
    }
    char *param = static_cast<char *>(e.param);
    const int64_t i = first + 8 * lane - h;       // the group's first element
    if (i >= shift && i + (shift ? 16 - shift : 8) <= e.numel) {
        float g[8], x[8], m[8], v[8];
        const Raw<4> rm = load_raw(e.m + i, (Raw<4> *)nullptr), rv = load_raw(e.v + i, (Raw<4> *)nullptr);
        if constexpr (MASTER)
            to_floats(load_raw(e.master + i, (Raw<4> *)nullptr), false, x);
        else
            to_floats(load_raw(param + i * BP, (Raw<BP> *)nullptr), bp, x);
        if (BG == 4 || shift == 0)
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
    // from the end backwards: L2 still holds what the norm read last
    const uint32_t u = (gridDim.x - 1 - blockIdx.x) * kWarps + threadIdx.x / 32;
    if (u >= t.units) return;
    const ParamEntry &e = t.e[entry_of(t, u)];
    step_unit<BP, BG, MASTER>(e, s, c, u - e.begin, bp, bg);
}

template <int BP, int BG, bool MASTER>
cudaError_t launch(const ParamTable &t, Step s, bool bp, bool bg, bool chained, cudaStream_t stream)
{
    void *args[] = {(void *)&t, &s, &bp, &bg, &chained};
    return launch_table(t.n <= kParamsSmall ? (const void *)adamw_kernel<BP, BG, MASTER, kParamsSmall>
                                            : (const void *)adamw_kernel<BP, BG, MASTER, kParams>,
                        ((int64_t)t.units + kWarps - 1) / kWarps, args, chained, stream);
}

// calls f with the sizes of a group's types as template arguments
template <class F>
auto by_types(const aspis_params::Group &g, F f)
{
    const bool wide = g.grad_type == ASPIS_F32;
    if (g.param_type == ASPIS_F32) return wide ? f(Types<4, 4, false>()) : f(Types<4, 2, false>());
    if (g.master) return wide ? f(Types<2, 4, true>()) : f(Types<2, 2, true>());
    return wide ? f(Types<2, 4, false>()) : f(Types<2, 2, false>());
}

}  // namespace

extern "C" aspis_status aspis_adamw(const aspis_params *params, const aspis_adamw_args *a, float *norm, void *work,
                                    void *stream)
{
    if (!params || !a || !isfinite((float)a->lr) || !(a->beta1 >= 0 && a->beta1 < 1) || !(a->beta2 >= 0 && a->beta2 < 1) ||
        !(a->eps >= 0) || isinf((float)a->eps) || a->step < 1 || isnan(a->max_norm) || !(a->scale > 0) || isinf(a->scale) ||
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
    cudaError_t err = normed && work ? launch_grad_norm(params->grads.tables, a->scale, norm, nullptr, work, true, st)
                                     : cudaSuccess;
    bool chained = normed && work;
    for (auto g = params->groups.rbegin(); g != params->groups.rend(); ++g)
        for (auto t = g->tables.rbegin(); t != g->tables.rend(); ++t) {
            if (err != cudaSuccess) return ASPIS_E_CUDA;
            err = by_types(*g, [&](auto k) {
                return launch<k.param, k.grad, k.master>(**t, s, g->param_type == ASPIS_BF16, g->grad_type == ASPIS_BF16,
                                                         chained, st);
            });
            chained = true;
        }
    return err == cudaSuccess ? ASPIS_OK : ASPIS_E_CUDA;
}
