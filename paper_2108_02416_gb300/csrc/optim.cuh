// Tables of many tensors, shared by the norm, clipping and AdamW.
//
// A launch takes its tensors' addresses and lengths as a kernel argument: the
// table lies in the constant bank, needs no device memory, no copy and no
// lifetime beyond the call, and can be captured.  A table is a prefix of the
// largest one, and kernels exist for a few capacities, because the launch's cost
// grows with the argument: stream of launches 2.06 us up to 8 KB, 2.4 at 16 KB,
// 3.2 at 32 KB, and 3 us more between events at 32 KB.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <memory>
#include <vector>

#include "aspis_internal.cuh"
#include "aspis_optim.h"

namespace aspis {

// Work is dealt in units of consecutive elements of one tensor, which a warp takes; every tensor,
// an empty one too, has a unit at least.  (With units for whole blocks a list's smallest tensors, a few
// elements each, took a block's full latency one after the other: the norm of 301 tensors of 0 to 4
// million fp16 values ran at 4.4 TB/s.)
struct GradEntry {
    const void *in;
    void *out;                    // in place: in
    uint64_t length_types;        // elements, and the types from bit 48 and 56
    uint32_t begin, end;          // units of the table that are this tensor's

    __host__ __device__ int64_t numel() const { return (int64_t)(length_types & 0xFFFFFFFFFFFFull); }
    __host__ __device__ int type() const { return (int)(length_types >> 48) & 0xFF; }
    __host__ __device__ int out_type() const { return (int)(length_types >> 56); }
};

struct ParamEntry {
    void *param;
    float *master;
    const void *grad;
    float *m, *v;
    int64_t numel;
    uint32_t begin, end;
    float decay;
    uint32_t pad;
};

// hint[u >> shift] is the tensor of the first unit with that quotient: what the constant bank
// has to deliver before the first element can be read is the hint, its successor, few steps of a bisection
// between them (none inside a large tensor) and the entry.
constexpr int kHints = 64;

template <class E, int N>
struct Table {
    int32_t n;
    uint32_t units;
    int32_t first;                // of the list's tensors, the one that entry 0 is
    int32_t last;                 // 1: the last table of its list
    uint32_t shift;
    int32_t in_place;             // 1: every tensor is clipped in place
    uint16_t hint[kHints + 2];
    E e[N];
};

constexpr int kGradsSmall = 120, kGradsMid = 500, kGrads = 1000;
constexpr int kParamsSmall = 60, kParams = 500;
using GradTable = Table<GradEntry, kGrads>;
using ParamTable = Table<ParamEntry, kParams>;
static_assert(sizeof(GradTable) <= 32700 && sizeof(ParamTable) <= 32600, "a kernel's arguments have 32,764 bytes");

constexpr int kOptThreads = 256;
constexpr int kMaxGrid = 1024;    // of the norm

constexpr int kWarps = kOptThreads / 32;

__host__ __device__ constexpr int type_bytes(int type) { return type == ASPIS_F32 ? 4 : 2; }
// 4 KB of gradient: eight vectors of 16 bytes per thread of a warp
constexpr int kUnitVecs = 256;
__host__ __device__ constexpr int grad_unit(int type) { return kUnitVecs * 16 / type_bytes(type); }
// eight elements per thread of a warp
constexpr int kParamUnit = 256;

// the tensor that unit u of the table belongs to
template <class T>
__device__ __forceinline__ int entry_of(const T &t, uint32_t u)
{
    int lo = t.hint[u >> t.shift], hi = t.hint[(u >> t.shift) + 1];
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (t.e[mid].begin <= u)
            lo = mid;
        else
            hi = mid - 1;
    }
    return lo;
}

__device__ __forceinline__ uint32_t run_begin(uint32_t units, uint32_t b, uint32_t grid)
{
    return (uint32_t)((uint64_t)units * b / grid);
}

// ---- eight elements at a time: one 32-byte access of fp32, one of 16 bytes of a 16-bit type

template <int B>
struct Raw {                      // eight elements of B bytes
    uint32_t w[2 * B];
};

// Streams are read past L1 and leave L2 first, so that gradients which the norm has just read stay there.
__device__ __forceinline__ Raw<4> load_raw(const void *p, Raw<4> *)
{
    Raw<4> r;
    asm volatile("ld.global.L1::no_allocate.L2::evict_first.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(r.w[0]), "=r"(r.w[1]), "=r"(r.w[2]), "=r"(r.w[3]), "=r"(r.w[4]), "=r"(r.w[5]), "=r"(r.w[6]),
                   "=r"(r.w[7])
                 : "l"(p));
    return r;
}

__device__ __forceinline__ Raw<2> load_raw(const void *p, Raw<2> *)
{
    const uint4 v = __ldcs(static_cast<const uint4 *>(p));
    return Raw<2>{{v.x, v.y, v.z, v.w}};
}

__device__ __forceinline__ void store_raw(void *p, const Raw<4> &r)
{
    asm volatile("st.global.L1::no_allocate.L2::evict_first.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(r.w[0]),
                 "r"(r.w[1]), "r"(r.w[2]), "r"(r.w[3]), "r"(r.w[4]), "r"(r.w[5]), "r"(r.w[6]), "r"(r.w[7])
                 : "memory");
}

__device__ __forceinline__ void store_raw(void *p, const Raw<2> &r)
{
    __stcs(static_cast<uint4 *>(p), make_uint4(r.w[0], r.w[1], r.w[2], r.w[3]));
}

// the elements of the groups x, y from number `shift` (0 to 7) on
template <int B>
__device__ __forceinline__ Raw<B> shifted(const Raw<B> &x, const Raw<B> &y, int shift)
{
    constexpr int n = 2 * B, four = B;            // words of a group, and of four elements
    uint32_t w[2 * n];
#pragma unroll
    for (int i = 0; i < n; ++i) w[i] = x.w[i], w[n + i] = y.w[i];
    if (shift & 4)
#pragma unroll
        for (int i = 0; i < 2 * n - four; ++i) w[i] = w[i + four];
    if (shift & 2)
#pragma unroll
        for (int i = 0; i < 2 * n - four - four / 2; ++i) w[i] = w[i + four / 2];
    if (shift & 1) {
#pragma unroll
        for (int i = 0; i < n; ++i) w[i] = B == 4 ? w[i + 1] : __funnelshift_r(w[i], w[i + 1], 16);
    }
    Raw<B> r;
#pragma unroll
    for (int i = 0; i < n; ++i) r.w[i] = w[i];
    return r;
}

// Eight elements from any element-aligned address: the two aligned groups that hold them (p: the
// first), the second of which is the next thread's first and comes from L1.
template <int B>
__device__ __forceinline__ Raw<B> load_shifted(const char *p, int shift)
{
    Raw<B> x[2];
#pragma unroll
    for (int h = 0; h < B; ++h) {
        const uint4 v = __ldg(reinterpret_cast<const uint4 *>(p) + h);
        uint32_t *w = x[h / (B / 2)].w + 4 * (h % (B / 2));
        w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
    }
    return shifted(x[0], x[1], shift);
}

// The same for a warp's D rows of 32 consecutive groups (p: the first thread's first group): each thread loads
// its own, and gets the next one from its neighbour; thread 0 loads the one after the last row.
template <int B, int D>
__device__ __forceinline__ void load_shifted_rows(Raw<B> (&r)[D], const char *p, int shift)
{
    const int lane = threadIdx.x % 32;
    Raw<B> after = {};
#pragma unroll
    for (int d = 0; d < D; ++d) r[d] = load_raw(p + (d * 32 + lane) * 8 * B, (Raw<B> *)nullptr);
    if (lane == 0) after = load_raw(p + D * 32 * 8 * B, (Raw<B> *)nullptr);
#pragma unroll
    for (int d = 0; d < D; ++d) {
        Raw<B> next;
#pragma unroll
        for (int i = 0; i < 2 * B; ++i) {
            const uint32_t given = lane ? r[d].w[i] : d + 1 < D ? r[d + 1 < D ? d + 1 : d].w[i] : after.w[i];
            next.w[i] = __shfl_sync(0xFFFFFFFFu, given, (lane + 1) % 32);
        }
        r[d] = shifted(r[d], next, shift);
    }
}

// bf16 or fp16 pair -> two floats, and back (round to nearest even)
__device__ __forceinline__ float2 unpack(uint32_t w, bool bf16)
{
    if (bf16) return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
    return __half22float2(*reinterpret_cast<const __half2 *>(&w));
}

__device__ __forceinline__ uint32_t pack(float lo, float hi, bool bf16)
{
    uint32_t w;
    if (bf16) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
        w = *reinterpret_cast<const uint32_t *>(&v);
    } else {
        const __half2 v = __floats2half2_rn(lo, hi);
        w = *reinterpret_cast<const uint32_t *>(&v);
    }
    return w;
}

__device__ __forceinline__ void to_floats(const Raw<4> &r, bool, float (&f)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(r.w[i]);
}

__device__ __forceinline__ void to_floats(const Raw<2> &r, bool bf16, float (&f)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 v = unpack(r.w[i], bf16);
        f[2 * i] = v.x;
        f[2 * i + 1] = v.y;
    }
}

template <int B>
__device__ __forceinline__ void store_floats(void *p, const float (&f)[8], bool bf16)
{
    Raw<B> r;
    if constexpr (B == 4) {
#pragma unroll
        for (int i = 0; i < 8; ++i) r.w[i] = __float_as_uint(f[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) r.w[i] = pack(f[2 * i], f[2 * i + 1], bf16);
    }
    store_raw(p, r);
}

// one element
template <int B>
__device__ __forceinline__ float load_one(const void *p, int64_t i, bool bf16)
{
    if constexpr (B == 4) return static_cast<const float *>(p)[i];
    const uint32_t w = static_cast<const uint16_t *>(p)[i];
    return unpack(w, bf16).x;
}

template <int B>
__device__ __forceinline__ void store_one(void *p, int64_t i, float x, bool bf16)
{
    if constexpr (B == 4)
        static_cast<float *>(p)[i] = x;
    else
        static_cast<uint16_t *>(p)[i] = (uint16_t)(pack(x, 0.0f, bf16) & 0xFFFFu);
}

// Elements that an address lies behind the group boundary before it.
template <int B>
__device__ __forceinline__ int behind(const void *p)
{
    return (int)((uintptr_t)p % (8 * B)) / B;
}

// min(1, max_norm / (norm + eps)), where NaN stays NaN; 1 for an infinite bound, whatever the norm (the
// quotient would be NaN where that is infinite too)
__device__ __forceinline__ float clip_coef(float norm, float max_norm)
{
    if (isinf(max_norm)) return 1.0f;
    const float c = max_norm / (norm + ASPIS_CLIP_EPS);
    return c > 1.0f ? 1.0f : c;
}

// Workspace of the norm: the counts of blocks that are done and that have seen the others done, the sum of
// the tables before this one, the blocks that met each tensor, and the partial sums.
struct NormWork {
    uint32_t done, left;
    double before;
    uint16_t first[kGrads], last[kGrads];
    float2 pair[kMaxGrid + kGrads];
    double wide[kMaxGrid + kGrads];
};
static_assert(offsetof(NormWork, first) % 16 == 0 && offsetof(NormWork, last) % 16 == 0 &&
                  offsetof(NormWork, pair) % 16 == 0 && kGrads % 8 == 0, "fetched in steps of 16 bytes");
static_assert(sizeof(NormWork) <= ASPIS_NORM_WORKSPACE_BYTES, "workspace");

// Launches a kernel whose first argument is a prefix of the table; chained: as a dependent of the kernel before it, which
// belongs to the same call (chain()).
cudaError_t launch_table(const void *kernel, int64_t grid, void **args, bool chained, cudaStream_t stream);

// The same as a cooperative kernel; false (and nothing enqueued) where its blocks do not fit the device at once.
bool launch_together(cudaError_t &err, const void *kernel, int64_t grid, void **args, cudaStream_t stream);

// The norm of the list's gradients; norm (and tensor_norms) written by the last block.  again: the call reads them
// all once more, from the end of the list backwards.
cudaError_t launch_grad_norm(const std::vector<std::unique_ptr<GradTable>> &tables, float scale, float *norm,
                             float *tensor_norms, void *work, bool again, cudaStream_t stream);

}  // namespace aspis

struct aspis_tensors {
    int64_t n = 0;
    bool apart = true;            // no range that clipping writes overlaps another
    std::vector<std::unique_ptr<aspis::GradTable>> tables;   // one at least
};

struct aspis_params {
    struct Group {                // tensors of the same types, which one kernel takes
        int param_type, grad_type;
        bool master;
        std::vector<std::unique_ptr<aspis::ParamTable>> tables;
    };
    int64_t n = 0;
    aspis_tensors grads;          // the same gradients, for the norm
    std::vector<Group> groups;
};
