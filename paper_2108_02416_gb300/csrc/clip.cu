// aspis_clip_grads: the norm (norm.cu), then every gradient times s * c.
//
// The second kernel reads and writes eight elements per thread and access, aligned to
// the output.  Blocks take their runs from the end of the list backwards, as what the norm
// has read last is what L2 still holds.
#include "norm.cuh"

using namespace aspis;

namespace {

constexpr int kDepth = 2;         // groups of eight elements that a thread loads before it stores
constexpr int kRun = 8;           // units that a block takes at a time
constexpr int kBlocks = 8;        // per multiprocessor
constexpr int kTogether = 3;      // blocks of the cooperative kernel per multiprocessor
constexpr int64_t kMostTogether = 16384;          // units

// Units [ua, ub) of a tensor: groups of eight elements counted from the group boundary at or
// before the output's first element.
template <int BI, int BO>
__device__ __forceinline__ void scale_units(const GradEntry &e, uint32_t ua, uint32_t ub, float c)
{
    const bool bi = e.type() == ASPIS_BF16, bo = e.out_type() == ASPIS_BF16;
    const int64_t numel = e.numel();
    const int h = behind<BO>(e.out);
    const char *in = static_cast<const char *>(e.in);
    char *out = static_cast<char *>(e.out);
    const int shift = behind<BI>(in - h * BI);    // of the input's groups against the output's
    constexpr int per = kOptThreads * 2 / BI;     // groups per unit
    const int64_t end = min((int64_t)ub * per, (numel + h + 7) / 8);
    // groups that can be taken whole: [lo, hi)
    const int64_t lo = (h + shift + 7) / 8, hi = (numel + h - (shift ? 8 - shift : 0)) / 8;
    for (int64_t q = (int64_t)ua * per + threadIdx.x; q < end; q += kDepth * kOptThreads) {
        if (q >= lo && q + (kDepth - 1) * kOptThreads < min(hi, end)) {
            Raw<BI> r[kDepth];
#pragma unroll
            for (int d = 0; d < kDepth; ++d) {
                const char *p = in + ((q + d * kOptThreads) * 8 - h - shift) * BI;
                r[d] = shift ? load_shifted<BI>(p, shift) : load_raw(p, (Raw<BI> *)nullptr);
            }
#pragma unroll
            for (int d = 0; d < kDepth; ++d) {
                float f[8];
                to_floats(r[d], bi, f);
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] *= c;
                store_floats<BO>(out + ((q + d * kOptThreads) * 8 - h) * BO, f, bo);
            }
        } else {
            for (int64_t p = q; p < min(end, q + kDepth * kOptThreads); p += kOptThreads) {
                const int64_t i = p * 8 - h;      // the group's first element
                if (p >= lo && p < hi) {
                    float f[8];
                    const char *at = in + (i - shift) * BI;
                    to_floats(shift ? load_shifted<BI>(at, shift) : load_raw(at, (Raw<BI> *)nullptr), bi, f);
#pragma unroll
                    for (int j = 0; j < 8; ++j) f[j] *= c;
                    store_floats<BO>(out + i * BO, f, bo);
                } else {
                    for (int64_t j = max(i, (int64_t)0); j < min(i + 8, numel); ++j)
                        store_one<BO>(out, j, load_one<BI>(in, j, bi) * c, bo);
                }
            }
        }
    }
}

__device__ __forceinline__ void scale_units(const GradEntry &e, uint32_t ua, uint32_t ub, float c)
{
    if (c == 1.0f && e.in == e.out) return;
    if (e.type() == ASPIS_F32) {
        if (e.out_type() == ASPIS_F32)
            scale_units<4, 4>(e, ua, ub, c);
        else
            scale_units<4, 2>(e, ua, ub, c);
    } else {
        if (e.out_type() == ASPIS_F32)
            scale_units<2, 4>(e, ua, ub, c);
        else
            scale_units<2, 2>(e, ua, ub, c);
    }
}

template <int N>
__global__ void __launch_bounds__(kOptThreads, 6)
scale_kernel(const __grid_constant__ Table<GradEntry, N> t, float max_norm, float scale, const float *norm, bool chained)
{
    if (chained) chain();
    const float c = scale * clip_coef(*norm, max_norm);
    if (c == 1.0f && t.in_place) return;
    const uint32_t runs = (t.units + kRun - 1) / kRun;
    for (uint32_t r = blockIdx.x; r < runs; r += gridDim.x) {
        uint32_t u = (runs - 1 - r) * kRun;
        const uint32_t end = min(u + kRun, t.units);
        for (int k = entry_of(t, u); u < end; ++k) {
            const GradEntry &e = t.e[k];
            const uint32_t stop = min(end, e.end);
            scale_units(e, u - e.begin, stop - e.begin, c);
            u = stop;
        }
    }
}

// Norm and clipping in one cooperative kernel: every block sums a run of units, waits for the others, and
// scales the same run.
template <int N>
__global__ void __launch_bounds__(kOptThreads, kTogether)
clip_kernel(const __grid_constant__ Table<GradEntry, N> t, float max_norm, float scale, float *norm, NormWork *work)
{
    const uint32_t begin = run_begin(t.units, blockIdx.x, gridDim.x), end = run_begin(t.units, blockIdx.x + 1, gridDim.x);
    const int first = entry_of(t, begin);
    Sum sum;
    uint32_t u = begin;
    for (int k = first; u < end; ++k) {
        const GradEntry &e = t.e[k];
        const uint32_t stop = min(end, e.end);
        sum_units(sum, e.in, e.numel(), e.type(), u - e.begin, stop - e.begin);
        u = stop;
    }
    float all;
    const bool met = meet(sum, scale, work, all);
    if (blockIdx.x == 0 && threadIdx.x == 0) *norm = all;
    if (!met) return;
    const float c = scale * clip_coef(all, max_norm);
    u = begin;
    for (int k = first; u < end; ++k) {
        const GradEntry &e = t.e[k];
        const uint32_t stop = min(end, e.end);
        scale_units(e, u - e.begin, stop - e.begin, c);
        u = stop;
    }
}

template <int N>
cudaError_t launch(const GradTable &t, float max_norm, float scale, const float *norm, bool chained,
                   cudaStream_t stream)
{
    const int64_t runs = ((int64_t)t.units + kRun - 1) / kRun;
    const int64_t most = t.in_place ? (int64_t)sm_count() * kBlocks : runs;
    const int64_t grid = runs < most ? runs : most;
    if (grid == 0) return cudaSuccess;
    void *args[] = {(void *)&t, &max_norm, &scale, &norm, &chained};
    return launch_table((const void *)scale_kernel<N>, grid, args, chained, stream);
}

template <int N>
bool launch_clip(cudaError_t &err, const GradTable &t, float max_norm, float scale, float *norm, void *work,
                 cudaStream_t stream)
{
    const int64_t most = (int64_t)sm_count() * kTogether;
    void *args[] = {(void *)&t, &max_norm, &scale, &norm, &work};
    return launch_together(err, (const void *)clip_kernel<N>, t.units < most ? t.units : most, args, stream);
}

}  // namespace

extern "C" aspis_status aspis_clip_grads(const aspis_tensors *grads, float max_norm, float scale, float *norm,
                                         void *work, void *stream)
{
    if (!grads || !norm || !(scale > 0.0f) || isinf(scale) || !(max_norm >= 0.0f) || !grads->apart)
        return ASPIS_E_INVAL;
    if ((uintptr_t)work % 16 != 0 || (uintptr_t)norm % 4 != 0) return ASPIS_E_ALIGN;
    const cudaStream_t st = (cudaStream_t)stream;
    cudaError_t e = cudaSuccess;
    if (const GradTable &t = *grads->tables[0]; work && t.last && t.units > 0 && t.units <= kMostTogether) {
        if (t.n <= kGradsSmall ? launch_clip<kGradsSmall>(e, t, max_norm, scale, norm, work, st)
            : t.n <= kGradsMid ? launch_clip<kGradsMid>(e, t, max_norm, scale, norm, work, st)
                               : launch_clip<kGrads>(e, t, max_norm, scale, norm, work, st))
            return e == cudaSuccess ? ASPIS_OK : ASPIS_E_CUDA;
    }
    e = work ? launch_grad_norm(grads->tables, scale, norm, nullptr, work, st) : cudaSuccess;
    bool chained = work != nullptr;
    for (auto it = grads->tables.rbegin(); it != grads->tables.rend() && e == cudaSuccess; ++it) {
        const GradTable &t = **it;
        e = t.n <= kGradsSmall ? launch<kGradsSmall>(t, max_norm, scale, norm, chained, st)
            : t.n <= kGradsMid ? launch<kGradsMid>(t, max_norm, scale, norm, chained, st)
                               : launch<kGrads>(t, max_norm, scale, norm, chained, st);
        chained = chained || t.units;
    }
    return e == cudaSuccess ? ASPIS_OK : ASPIS_E_CUDA;
}
