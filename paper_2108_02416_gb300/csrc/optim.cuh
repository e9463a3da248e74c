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

// Work is dealt in units of consecutive elements of one tensor; a block takes a
// contiguous run of units, found once by bisection.
struct GradEntry {
    const void *in;
    void *out;                    // in place: in
    int64_t numel;
    uint32_t unit_end;            // units of this table's tensors up to and with this one
    uint8_t type, out_type;
    uint16_t pad;
};

struct ParamEntry {
    void *param;
    float *master;
    const void *grad;
    float *m, *v;
    int64_t numel;
    uint32_t unit_end;
    float decay;
};

template <class E, int N>
struct Table {
    int32_t n;
    uint32_t units;
    int32_t first;                // of the list's tensors, the one that entry 0 is
    int32_t last;                 // 1: the last table of its list
    E e[N];
};

constexpr int kGradsSmall = 120, kGradsMid = 500, kGrads = 1000;
constexpr int kParamsSmall = 72, kParams = 576;
using GradTable = Table<GradEntry, kGrads>;
using ParamTable = Table<ParamEntry, kParams>;
static_assert(sizeof(GradTable) <= 32764 && sizeof(ParamTable) <= 32764, "a kernel argument's limit");

constexpr int kOptThreads = 256;
constexpr int kMaxGrid = 2048;    // of the norm: one partial sum per block and tensor that it meets
static_assert(64 + 8 * (kMaxGrid + kGrads) <= ASPIS_NORM_WORKSPACE_BYTES, "workspace");

__host__ __device__ constexpr int type_bytes(int type) { return type == ASPIS_F32 ? 4 : 2; }
// 4 KB of gradient; one vector of 16 bytes per thread
__host__ __device__ constexpr int grad_unit(int type) { return kOptThreads * 16 / type_bytes(type); }
constexpr int kParamUnit = 2048;

// the tensor that unit u of the table belongs to
template <class T>
__device__ __forceinline__ int entry_of(const T &t, uint32_t u)
{
    int lo = 0, hi = t.n - 1;
    while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (t.e[mid].unit_end > u)
            hi = mid;
        else
            lo = mid + 1;
    }
    return lo;
}

__device__ __forceinline__ uint32_t run_begin(uint32_t units, uint32_t b, uint32_t grid)
{
    return (uint32_t)((uint64_t)units * b / grid);
}

__device__ __forceinline__ float load_as_float(const void *p, int64_t i, int type)
{
    if (type == ASPIS_F32) return static_cast<const float *>(p)[i];
    if (type == ASPIS_BF16) return __bfloat162float(static_cast<const __nv_bfloat16 *>(p)[i]);
    return __half2float(static_cast<const __half *>(p)[i]);
}

__device__ __forceinline__ void store_rounded(void *p, int64_t i, int type, float x)
{
    if (type == ASPIS_F32)
        static_cast<float *>(p)[i] = x;
    else if (type == ASPIS_BF16)
        static_cast<__nv_bfloat16 *>(p)[i] = __float2bfloat16_rn(x);
    else
        static_cast<__half *>(p)[i] = __float2half_rn(x);
}

// min(1, max_norm / (norm + eps)); NaN stays NaN
__device__ __forceinline__ float clip_coef(float norm, float max_norm)
{
    const float c = max_norm / (norm + ASPIS_CLIP_EPS);
    return c > 1.0f ? 1.0f : c;
}

// Workspace of the norm: the count of blocks that are done, the sum of the
// tables before this one, and the partial sums.
struct NormWork {
    uint32_t done;
    uint32_t pad;
    double before;
    double pad2[6];
    double part[1];
};

// The norm of the list's gradients; norm (and tensor_norms) written by the last block.
cudaError_t launch_grad_norm(const std::vector<std::unique_ptr<GradTable>> &tables, float scale, float *norm,
                             float *tensor_norms, void *work, cudaStream_t stream);

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
