// aspis_clip_grads: the norm, then every gradient times s * c, c = min(1, max_norm / (norm + eps)).
//
// The factor depends on every gradient, so what does not fit the chip crosses HBM twice: n bytes for
// the norm (norm.cu), n read again and n_out written by scale_kernel, which is bound by HBM.  It
// goes through the list from its end backwards, as what the norm has read last is what L2 still holds: 234
// million bf16 into fp32 take 280 us (468 + 468 + 936 MB: 6.7 TB/s).  Below the bound a list in place is only
// read: 936 MB in 136 us (6.9 TB/s).
//
// Up to 64 MB of gradients one cooperative kernel does both: a warp's first unit waits in registers for the
// norm (12.4 us for 8.4 million bf16 values in 256 tensors, 14.3 read again), the others come from L1 or L2.  60
// thousand bf16 values take 7.5 us (two kernels 8.2), 200 thousand 8.2 (10.3), a ResNet-18's 11 million fp32
// 22.8 (26.6), 17 million bf16 18.7 (18.6); from 75 MB on the two kernels are as fast (33 us) or faster (301 ragged
// fp16 tensors, 164 MB: 94 and 78).
#include "norm.cuh"

using namespace aspis;

namespace {

// That a thread loads before it stores.  Of 234 million bf16 into fp32 285 us, with 64 bytes 287, with 32 291; of 301
// ragged fp16 tensors at odd addresses 83, 86 and 86.
constexpr int kDepthBytes = 128;
// Blocks per multiprocessor where the call may turn out to write nothing (else a block per eight units).  The whole
// call on 234 million fp32 in place takes 401 us clipped (2.8 GB: 7.0 TB/s; scaling alone, with a given norm, 274) and
// 139 below the bound; with 8 blocks 416 and 137, with a block per eight units 390 and 166.
constexpr int kBlocks = 16;
constexpr int kTogether = 3;                      // blocks of the cooperative kernel per multiprocessor
constexpr int64_t kMostTogether = 16384;          // units that it takes

// A warp's unit of a tensor: groups of eight elements counted from the group boundary at or before
// the output's first element.
template <int BI, int BO>
__device__ __forceinline__ void scale_unit(const GradEntry &e, uint32_t unit, float c)
{
    const bool bi = e.type() == ASPIS_BF16, bo = e.out_type() == ASPIS_BF16;
    const int64_t numel = e.numel();
    const int h = behind<BO>(e.out);
    const char *in = static_cast<const char *>(e.in);
    char *out = static_cast<char *>(e.out);
    const int shift = behind<BI>(in - h * BI);    // of the input's groups against the output's
    constexpr int per = kUnitVecs * 2 / BI;       // groups per unit
    const int64_t end = min(((int64_t)unit + 1) * per, (numel + h + 7) / 8);
    // groups that can be taken whole: [lo, hi)
    const int64_t lo = (h + shift + 7) / 8, hi = (numel + h - (shift ? 8 - shift : 0)) / 8;
    constexpr int depth = kDepthBytes / (8 * BI);
    const int lane = threadIdx.x % 32;
    for (int64_t row = (int64_t)unit * per; row < end; row += depth * 32) {
        const int64_t q = row + lane;
        if (row >= lo && row + depth * 32 <= min(hi, end)) {
            Raw<BI> r[depth];
            const char *p = in + (row * 8 - h - shift) * BI;
            if (shift)
                load_shifted_rows(r, p, shift);
            else
#pragma unroll
                for (int d = 0; d < depth; ++d) r[d] = load_raw(p + (d * 32 + lane) * 8 * BI, (Raw<BI> *)nullptr);
#pragma unroll
            for (int d = 0; d < depth; ++d) {
                float f[8];
                to_floats(r[d], bi, f);
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] *= c;
                store_floats<BO>(out + ((q + d * 32) * 8 - h) * BO, f, bo);
            }
        } else {
            for (int64_t p = q; p < min(end, row + depth * 32); p += 32) {
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

__device__ __forceinline__ void scale_unit(const GradEntry &e, uint32_t unit, float c)
{
    if (c == 1.0f && e.in == e.out) return;
    if (e.type() == ASPIS_F32) {
        if (e.out_type() == ASPIS_F32)
            scale_unit<4, 4>(e, unit, c);
        else
            scale_unit<4, 2>(e, unit, c);
    } else {
        if (e.out_type() == ASPIS_F32)
            scale_unit<2, 4>(e, unit, c);
        else
            scale_unit<2, 2>(e, unit, c);
    }
}

template <int N>
__global__ void __launch_bounds__(kOptThreads, 4)
scale_kernel(const __grid_constant__ Table<GradEntry, N> t, float max_norm, float scale, const float *norm, bool chained)
{
    if (chained) chain();
    const float c = scale * clip_coef(*norm, max_norm);
    if (c == 1.0f && t.in_place) return;
    for (uint32_t r = blockIdx.x * kWarps + threadIdx.x / 32; r < t.units; r += gridDim.x * kWarps) {
        const uint32_t u = t.units - 1 - r;
        const GradEntry &e = t.e[entry_of(t, u)];
        scale_unit(e, u - e.begin, c);
    }
}

// How the cooperative kernel counts a tensor's units.  Where the output's elements have the input's size and
// lie at the same place within 16 bytes, both from the boundary of the output's groups, as scale_unit does: a
// unit that waits in registers then has the elements that scale_unit would take, and its neighbours may be
// left to either.  (fp32 groups are 32 bytes: units counted from the 16-byte boundary instead would begin four
// elements away from scale_unit's for every second such address.)  Else the sum counts from the input's vectors,
// and scale_unit alone stores.
__device__ __forceinline__ bool stays_held(const GradEntry &e)
{
    return type_bytes(e.type()) == type_bytes(e.out_type()) && ((uintptr_t)e.in - (uintptr_t)e.out) % 16 == 0;
}

struct GroupOrigin {              // 16-bit groups are one vector
    template <int TYPE>
    __device__ __forceinline__ static int of(const GradEntry &e)
    {
        return TYPE == ASPIS_F32 && stays_held(e) ? behind<4>(e.out) : VectorOrigin::of<TYPE>(e);
    }
};

// A warp's unit whose vectors stay in registers from the sum to the store.
template <int TYPE>
__device__ __forceinline__ void sum_held(Sum &sum, const GradEntry &e, uint32_t unit, uint4 (&r)[kVecs])
{
    const int lane = threadIdx.x % 32;
    const Vectors<TYPE> t(e.in, e.numel(), GroupOrigin::of<TYPE>(e));
    const int64_t a = (int64_t)unit * kUnitVecs, b = a + kUnitVecs;
    sum_batch<TYPE, 32>(sum, t.base(), max(a, (int64_t)t.first) + lane, min(b, t.full), PlainLoad(), r);
    t.ends(a, b, lane, [&](int64_t i) { add_square(sum, load_one<t.size>(e.in, i, TYPE == ASPIS_BF16)); });
}

template <int TYPE>
__device__ __forceinline__ void store_held(const GradEntry &e, uint32_t unit, const uint4 (&r)[kVecs], float c)
{
    constexpr int size = type_bytes(TYPE);
    const int lane = threadIdx.x % 32;
    const bool bi = TYPE == ASPIS_BF16, bo = e.out_type() == ASPIS_BF16;
    const Vectors<TYPE> t(e.in, e.numel(), GroupOrigin::of<TYPE>(e));
    const int64_t a = (int64_t)unit * kUnitVecs, b = a + kUnitVecs, end = min(b, t.full);
    uint4 *out = reinterpret_cast<uint4 *>((uintptr_t)e.out - t.h * size);
    const int64_t v = max(a, (int64_t)t.first) + lane;
#pragma unroll
    for (int u = 0; u < kVecs; ++u) {
        if (v + u * 32 >= end) break;
        uint32_t w[4] = {r[u].x, r[u].y, r[u].z, r[u].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (size == 4) {
                w[i] = __float_as_uint(__uint_as_float(w[i]) * c);
            } else {
                const float2 f = unpack(w[i], bi);
                w[i] = pack(f.x * c, f.y * c, bo);
            }
        }
        __stcs(out + v + u * 32, make_uint4(w[0], w[1], w[2], w[3]));
    }
    t.ends(a, b, lane, [&](int64_t i) { store_one<size>(e.out, i, load_one<size>(e.in, i, bi) * c, bo); });
}

// Norm and clipping in one cooperative kernel: every block sums a run of units, waits for the others, and
// scales the same run: a warp's first unit from registers, the others from what L1 or L2 still holds.
template <int N>
__global__ void __launch_bounds__(kOptThreads, kTogether)
clip_kernel(const __grid_constant__ Table<GradEntry, N> t, float max_norm, float scale, float *norm, NormWork *work)
{
    const uint32_t begin = run_begin(t.units, blockIdx.x, gridDim.x) + threadIdx.x / 32;
    const uint32_t end = run_begin(t.units, blockIdx.x + 1, gridDim.x);
    const int first = begin < end ? entry_of(t, begin) : 0;
    Sum sum;
    uint4 held[kVecs];
    if (begin < end) {
        const GradEntry &e = t.e[first];
        if (e.type() == ASPIS_F32)
            sum_held<ASPIS_F32>(sum, e, begin - e.begin, held);
        else if (e.type() == ASPIS_BF16)
            sum_held<ASPIS_BF16>(sum, e, begin - e.begin, held);
        else
            sum_held<ASPIS_F16>(sum, e, begin - e.begin, held);
    }
    for (uint32_t u = begin + kWarps; u < end; u += kWarps) {
        const GradEntry &e = t.e[entry_of(t, u)];
        const int64_t a = (int64_t)(u - e.begin) * kUnitVecs;
        sum_range<32, GroupOrigin>(sum, e, a, a + kUnitVecs, threadIdx.x % 32);
    }
    float all;
    const bool met = meet(sum, scale, work, all);
    if (blockIdx.x == 0 && threadIdx.x == 0) *norm = all;
    if (!met) return;
    const float c = scale * clip_coef(all, max_norm);
    if (begin < end) {
        const GradEntry &e = t.e[first];
        if (stays_held(e)) {
            if (c == 1.0f && e.in == e.out) {
            } else if (e.type() == ASPIS_F32)
                store_held<ASPIS_F32>(e, begin - e.begin, held, c);
            else if (e.type() == ASPIS_BF16)
                store_held<ASPIS_BF16>(e, begin - e.begin, held, c);
            else
                store_held<ASPIS_F16>(e, begin - e.begin, held, c);
        } else {
            scale_unit(e, begin - e.begin, c);
        }
    }
    for (uint32_t u = begin + kWarps; u < end; u += kWarps) {
        const GradEntry &e = t.e[entry_of(t, u)];
        scale_unit(e, u - e.begin, c);
    }
}

template <int N>
cudaError_t launch(const GradTable &t, float max_norm, float scale, const float *norm, bool chained,
                   cudaStream_t stream)
{
    const int64_t all = ((int64_t)t.units + kWarps - 1) / kWarps;
    const int64_t most = t.in_place ? (int64_t)sm_count() * kBlocks : all;
    const int64_t grid = all < most ? all : most;
    if (grid == 0) return cudaSuccess;
    void *args[] = {(void *)&t, &max_norm, &scale, &norm, &chained};
    return launch_table((const void *)scale_kernel<N>, grid, args, chained, stream);
}

template <int N>
bool launch_clip(cudaError_t &err, const GradTable &t, float max_norm, float scale, float *norm, void *work,
                 cudaStream_t stream)
{
    const int64_t all = ((int64_t)t.units + kWarps - 1) / kWarps, most = (int64_t)sm_count() * kTogether;
    void *args[] = {(void *)&t, &max_norm, &scale, &norm, &work};
    return launch_together(err, (const void *)clip_kernel<N>, all < most ? all : most, args, stream);
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
    e = work ? launch_grad_norm(grads->tables, scale, norm, nullptr, work, !grads->tables.back()->in_place, st) : cudaSuccess;
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
