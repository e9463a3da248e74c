// aspis_grad_norm: the global norm of many tensors, sqrt of the sum of all squares.
//
// One kernel reads every element once and is bound by HBM (1.1 billion bf16 values in 146 tensors, with each
// one's own norm, 314 us: 7.2 TB/s) or, in small lists, by latency (six tensors 6.2 us, 62 of a
// ResNet-18 16.8).  Its last block to finish adds up the partial sums in their order: the result depends
// on the lengths, the addresses modulo 16 and the grid, not on which block finished first.  Units are dealt to warps in turn, and a
// block leaves one partial sum.  Where the tensors' own norms are wanted, a block takes a
// contiguous run of units and leaves one per tensor that it meets.  The (block, tensor) pairs that occur
// then form a staircase (a later block starts no earlier than at the earlier one's last tensor), so
// block + tensor numbers them without collision.
#include "norm.cuh"

namespace aspis {

namespace {

// Of gradients that the next kernel reads again, from the end backwards, L2 is told to keep the last
// 60 MB and to let the others go first.  Clipping 234 million bf16 into fp32 287 us without, 280 with 48 to 80 MB;
// AdamW of 234 million parameters 1,010 and 994 us.  Lists that fit L2 are better off without (56 us and 57).  The
// second kernel reads what was kept with the priority to go first; what it leaves behind cost 4 to 6 us in the next reads
// of 88 MB that fit L2 themselves.
constexpr uint32_t kKept = 15000;                 // units

__device__ __forceinline__ uint64_t l2_policy(bool some, bool keep)
{
    uint64_t normal, first, last;
    asm("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(normal));
    asm("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(first));
    asm("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(last));
    return !some ? normal : keep ? last : first;
}

// Units of a tensor in a block's run from which on all warps take it together: 601 tensors of up
// to 3 million bf16 values 49 us with 2 to 5, 54 with 8, 62 where every tensor was taken by all.
constexpr uint32_t kApart = 4;
// Of the last block: a thread adds up a tensor that fewer blocks than kFew met, else kLanes threads.  With
// 8 threads for each 12.3 us for 256 small tensors (now 10.3), with one for each 33 for a ResNet-18's 62 (now 16.7).
constexpr int kLanes = 8, kFew = 6;
constexpr int kBlocks = 3;                        // per multiprocessor, each with 32 KB of gradient in flight (4: as fast or slower)

// bytes from L2 into shared memory, in steps of 16
__device__ __forceinline__ void fetch(void *to, const void *from, uint32_t bytes)
{
    const uint32_t at = (uint32_t)__cvta_generic_to_shared(to);
#pragma unroll 1
    for (uint32_t o = 16 * threadIdx.x; o < bytes; o += 16 * kOptThreads)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at + o), "l"(static_cast<const char *>(from) + o)
                     : "memory");
}

template <int N>
__global__ void __launch_bounds__(kOptThreads, kBlocks)
norm_kernel(const __grid_constant__ Table<GradEntry, N> t, float scale, float *norm, float *tensor_norms,
            NormWork *work, bool chained, uint32_t kept)
{
    __shared__ BlockSums sh;
    __shared__ __align__(16) float2 parts[kMaxGrid + N];
    __shared__ __align__(16) uint16_t met_first[(N + 7) / 8 * 8], met_last[(N + 7) / 8 * 8];
    __shared__ uint32_t done;
    __shared__ uint32_t warp_wide;
    if (threadIdx.x == 0) warp_wide = 0;
    __syncthreads();
    if (chained) chain();
    const uint32_t grid = gridDim.x, b = blockIdx.x;
    Sum sum;
    bool wide = false;
    // a partial sum: a pair, and in fp64 where that was needed (read only if a block says so)
    auto leave = [&](uint32_t slot) {
        wide |= reduce(sum, sh);
        if (threadIdx.x == 0) {
            work->pair[slot] = make_float2(sum.p.hi, sum.p.lo);
            work->wide[slot] = wide ? sum.wide : 0.0;
        }
        sum = Sum();
    };
    if (!tensor_norms) {
        // units dealt to the grid's warps in turn
        for (uint32_t u = b * kWarps + threadIdx.x / 32; u < t.units; u += grid * kWarps) {
            const GradEntry &e = t.e[entry_of(t, u)];
            const int64_t a = (int64_t)(u - e.begin) * kUnitVecs;
            sum_range<32>(sum, e, a, a + kUnitVecs, threadIdx.x % 32, PolicyLoad{l2_policy(kept, u + kept >= t.units)});
        }
        leave(b);
    } else {
        // one run of units for each block, which leaves a partial sum for each tensor in it: of the
        // long ones by all of its warps, of the others by one
        uint32_t u = run_begin(t.units, b, grid);
        const uint32_t end = run_begin(t.units, b + 1, grid);
        int turn = 0;
        for (int k = u < end ? entry_of(t, u) : 0; u < end; ++k) {
            const GradEntry &e = t.e[k];
            const uint32_t stop = min(end, e.end);
            const int64_t a = (int64_t)(u - e.begin) * kUnitVecs, z = (int64_t)(stop - e.begin) * kUnitVecs;
            if (stop - u >= kApart) {
                sum_range<kOptThreads>(sum, e, a, z, threadIdx.x);
                leave(b + k);
            } else if (turn++ % kWarps == threadIdx.x / 32) {
                Sum x;
                sum_range<32>(x, e, a, z, threadIdx.x % 32);
                const bool w = __any_sync(0xFFFFFFFFu, !(x.wide == 0));
                x.p = group_sum<32>(x.p);
                if (w) x.wide = group_sum<32>(x.wide);
                if (threadIdx.x % 32 == 0) {
                    work->pair[b + k] = make_float2(x.p.hi, x.p.lo);
                    work->wide[b + k] = x.wide;
                    if (w) warp_wide = 1;
                }
            }
            if (threadIdx.x == 0) {
                if (u == e.begin) work->first[k] = (uint16_t)b;
                if (stop == e.end) work->last[k] = (uint16_t)b;
            }
            u = stop;
        }
        __syncthreads();
        wide |= warp_wide != 0;
    }
    // the last block adds up
    if (threadIdx.x == 0) {
        __threadfence();
        done = atomicAdd(&work->done, wide ? kWide + 1 : 1u) + (wide ? kWide + 1 : 1u);
    }
    __syncthreads();
    if (done % kWide != grid) return;
    wide = done >= kWide;
    __threadfence();
    if (!tensor_norms) {
        collect(sum, work, grid, wide, sh);
    } else {
        // what this block runs now nobody has run before: short loops, as their code comes from memory too
        fetch(parts, work->pair, (grid + t.n) * sizeof(float2));
        fetch(met_first, work->first, t.n * sizeof(uint16_t));
        fetch(met_last, work->last, t.n * sizeof(uint16_t));
        asm volatile("cp.async.wait_all;" ::: "memory");
        __syncthreads();
        auto note = [&](int k, const Sum &x) {
            tensor_norms[t.first + k] = root(x, wide, scale);
            sum.p.add(x.p);
            sum.wide += x.wide;
        };
        // a thread per tensor that few blocks met, kLanes threads per tensor that more did
#pragma unroll 1
        for (int k = threadIdx.x; k < t.n; k += kOptThreads) {
            if (met_last[k] - met_first[k] >= kFew) continue;
            Sum x;
#pragma unroll 1
            for (int q = met_first[k] + k; q <= met_last[k] + k; ++q) {
                x.p.add(Pair(parts[q].x, parts[q].y));
                if (wide) x.wide += __ldcg(&work->wide[q]);
            }
            note(k, x);
        }
        const int lane = threadIdx.x % kLanes;
#pragma unroll 1
        for (int k0 = 0; k0 < t.n; k0 += kOptThreads / kLanes) {
            const int k = k0 + threadIdx.x / kLanes;
            const bool more = k < t.n && met_last[k] - met_first[k] >= kFew;
            if (!__any_sync(0xFFFFFFFFu, more)) continue;
            Sum x;
            const int q0 = more ? met_first[k] + k : 0, q1 = more ? met_last[k] + k : -1;
#pragma unroll 2
            for (int q = q0 + lane; q <= q1; q += kLanes) x.p.add(Pair(parts[q].x, parts[q].y));
            if (wide)
#pragma unroll 1
                for (int q = q0 + lane; q <= q1; q += kLanes) x.wide += __ldcg(&work->wide[q]);
            x.p = group_sum<kLanes>(x.p);
            if (wide) x.wide = group_sum<kLanes>(x.wide);
            if (more && lane == 0) note(k, x);
        }
        reduce(sum, sh);
    }
    if (threadIdx.x == 0) {
        work->done = 0;
        if (!t.first && t.last) {
            *norm = root(sum, wide, scale);
        } else {                                  // one of several tables
            double all = sum.p.value() + sum.wide;
            if (t.first) all += work->before;
            work->before = all;
            if (t.last) *norm = (float)(sqrt(all) * scale);
        }
    }
}

template <int N>
cudaError_t launch(const GradTable &t, float scale, float *norm, float *tensor_norms, void *work, bool again,
                   cudaStream_t stream)
{
    const int per = tensor_norms ? 2 : kWarps;    // units, where there are few
    const int64_t all = ((int64_t)t.units + per - 1) / per;
    int64_t grid = (int64_t)sm_count() * kBlocks;
    if (grid > kMaxGrid) grid = kMaxGrid;
    if (grid > all) grid = all ? all : 1;
    bool chained = t.first > 0;
    uint32_t kept = again && t.last && t.units > kKept ? kKept : 0;
    void *args[] = {(void *)&t, &scale, &norm, &tensor_norms, &work, &chained, &kept};
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
    const cudaError_t e = cudaLaunchKernelExC(&cfg, kernel, args);
    if (e != cudaSuccess) cudaGetLastError();     // the status says it; nobody else's call shall
    return e;
}

bool launch_together(cudaError_t &err, const void *kernel, int64_t grid, void **args, cudaStream_t stream)
{
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeCooperative;
    at[0].val.cooperative = 1;
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3(kOptThreads);
    cfg.stream = stream;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    err = cudaLaunchKernelExC(&cfg, kernel, args);
    if (err != cudaSuccess) cudaGetLastError();
    return err != cudaErrorCooperativeLaunchTooLarge;
}

cudaError_t launch_grad_norm(const std::vector<std::unique_ptr<GradTable>> &tables, float scale, float *norm,
                             float *tensor_norms, void *work, bool again, cudaStream_t stream)
{
    for (const auto &t : tables) {
        const cudaError_t e = t->n <= kGradsSmall ? launch<kGradsSmall>(*t, scale, norm, tensor_norms, work, again, stream)
                              : t->n <= kGradsMid ? launch<kGradsMid>(*t, scale, norm, tensor_norms, work, again, stream)
                                                  : launch<kGrads>(*t, scale, norm, tensor_norms, work, again, stream);
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
    return launch_grad_norm(grads->tables, scale, norm, tensor_norms, work, false, (cudaStream_t)stream) == cudaSuccess
               ? ASPIS_OK
               : ASPIS_E_CUDA;
}
