// What the embedding, dropout and the policy loss share: the dropout mask, elements of
// the three types, checks of matrices.
#pragma once

#include "aspis_worker.h"
#include "columns.h"
#include "optim.cuh"

namespace aspis {

constexpr int kRowThreads = 256, kRowWarps = kRowThreads / 32;
constexpr int kSMs = 152;

// ---- the dropout mask (aspis_drop)

struct Mask {
    uint32_t key[20];             // of the ten rounds
    uint32_t threshold;           // 0: no mask; 65536: nothing stays
    uint32_t high;                // threshold * 65536, what a word's upper half is compared with in place
    float up;                     // of what stays; 0 where nothing does
    uint64_t stream, first;
    const uint64_t *step;
};

inline aspis_status make_mask(const aspis_drop *drop, Mask &m)
{
    m = Mask{};
    m.up = 1.0f;
    if (!drop) return ASPIS_OK;
    if (!(drop->p >= 0.0 && drop->p <= 1.0)) return ASPIS_E_INVAL;
    if ((uintptr_t)drop->step % 8) return ASPIS_E_ALIGN;
    m.threshold = (uint32_t)(drop->p * 65536.0 + 0.5);
    m.up = m.threshold < 65536 ? (float)(65536.0 / (65536 - m.threshold)) : 0.0f;
    m.high = m.threshold << 16;
    for (int i = 0; i < 10; ++i) {
        m.key[2 * i] = (uint32_t)drop->seed + (uint32_t)i * 0x9E3779B9u;
        m.key[2 * i + 1] = (uint32_t)(drop->seed >> 32) + (uint32_t)i * 0xBB67AE85u;
    }
    m.stream = drop->stream;
    m.first = drop->first;
    m.step = drop->step;
    return ASPIS_OK;
}

// scale times what stays is multiplied by: one fp32 number.  Where that product is infinite a value of 0 would become NaN, and where
// it is below the normal numbers few of its bits are left: ASPIS_E_RANGE.
inline aspis_status make_factor(float scale, const Mask &m, float &factor)
{
    factor = scale * m.up;
    return m.threshold == 0 || factor == 0.0f || isnormal(factor) ? ASPIS_OK : ASPIS_E_RANGE;
}

// Philox 4x32 with ten rounds of (counter = block, stream; key): 128 bits, 16 for each of eight elements.  With 32
// bits an element, two such calls, dropout is bound by its multiplications: 268 million bf16 values 228 us, with 16
// bits 156, as long as a copy takes.
__device__ __forceinline__ void philox(uint32_t (&w)[4], const Mask &m, uint64_t block, uint64_t stream)
{
    uint32_t c0 = (uint32_t)block, c1 = (uint32_t)(block >> 32), c2 = (uint32_t)stream, c3 = (uint32_t)(stream >> 32);
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ m.key[2 * i];
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ m.key[2 * i + 1];
        c3 = (uint32_t)a;
    }
    w[0] = c0, w[1] = c1, w[2] = c2, w[3] = c3;
}

// whether element k of a block's eight stays
__device__ __forceinline__ bool stays(const uint32_t (&w)[4], int k, uint32_t high) { return (k & 1 ? w[k / 2] : w[k / 2] << 16) >= high; }

// f[k] * factor where the k-th of eight 16-bit words says that it stays, else 0
__device__ __forceinline__ void mask8(float (&f)[8], const Mask &m, const uint32_t (&w)[4], float factor)
{
    if (m.threshold == 65536)
#pragma unroll
        for (int k = 0; k < 8; ++k) f[k] = 0.0f;
#pragma unroll
    for (int k = 0; k < 8; ++k) f[k] = stays(w, k, m.high) ? f[k] * factor : 0.0f;
}

// the same without a factor
__device__ __forceinline__ void mask8(float (&f)[8], const Mask &m, const uint32_t (&w)[4])
{
    if (m.threshold == 65536)
#pragma unroll
        for (int k = 0; k < 8; ++k) f[k] = 0.0f;
#pragma unroll
    for (int k = 0; k < 8; ++k) f[k] = stays(w, k, m.high) ? f[k] : 0.0f;
}

__device__ __forceinline__ uint64_t mask_stream(const Mask &m)
{
    return m.threshold && m.step ? m.stream + *m.step : m.stream;
}

// ---- elements of a type known at compile time

template <int TYPE>
constexpr int kBytes = TYPE == ASPIS_F32 ? 4 : 2;

// eight elements that stay in L2 (rows of a table that are met again)
template <int TYPE>
__device__ __forceinline__ Raw<kBytes<TYPE>> load8(const void *p)
{
    Raw<kBytes<TYPE>> r;
    if constexpr (TYPE == ASPIS_F32) {
        asm volatile("ld.global.L1::no_allocate.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                     : "=r"(r.w[0]), "=r"(r.w[1]), "=r"(r.w[2]), "=r"(r.w[3]), "=r"(r.w[4]), "=r"(r.w[5]), "=r"(r.w[6]),
                       "=r"(r.w[7])
                     : "l"(p));
    } else {
        const uint4 v = __ldcg(static_cast<const uint4 *>(p));
        r.w[0] = v.x, r.w[1] = v.y, r.w[2] = v.z, r.w[3] = v.w;
    }
    return r;
}

template <int TYPE>
__device__ __forceinline__ float load_elem(const void *p, int64_t i)
{
    return load_one<kBytes<TYPE>>(p, i, TYPE == ASPIS_BF16);
}

template <int TYPE>
__device__ __forceinline__ void store_elem(void *p, int64_t i, float x)
{
    store_one<kBytes<TYPE>>(p, i, x, TYPE == ASPIS_BF16);
}

// eight elements; KEEP: they stay in L2
template <int TYPE, bool KEEP>
__device__ __forceinline__ Raw<kBytes<TYPE>> load_group(const char *p)
{
    if constexpr (KEEP)
        return load8<TYPE>(p);
    else
        return load_raw(p, (Raw<kBytes<TYPE>> *)nullptr);
}

// Elements [c, c + 8) of a row, those outside lo .. hi - 1 as zeros.
template <int TYPE>
__device__ __forceinline__ void load_edge(float (&f)[8], const char *row, int c, int lo, int hi)
{
#pragma unroll
    for (int k = 0; k < 8; ++k) f[k] = c + k >= lo && c + k < hi ? load_elem<TYPE>(row, c + k) : 0.0f;
}

template <int TYPE>
__device__ __forceinline__ void store_edge(char *row, int c, int lo, int hi, const float (&f)[8])
{
#pragma unroll
    for (int k = 0; k < 8; ++k)
        if (c + k >= lo && c + k < hi) store_elem<TYPE>(row, c + k, f[k]);
}

// The group that element c of a row lies in, `shift` behind the group's begin, or the columns of it that the row has, and zeros.
template <int TYPE, bool KEEP>
__device__ __forceinline__ Raw<kBytes<TYPE>> load_around(const char *row, int c, int shift, Columns columns, bool end)
{
    constexpr int B = kBytes<TYPE>;
    Raw<B> r = {};
    c -= shift;
    if (load_nothing(c, columns)) return r;
    if (load_whole(c, columns, end)) return load_group<TYPE, KEEP>(row + (int64_t)c * B);
    float f[8];
    load_edge<TYPE>(f, row, c, columns.lo, columns.hi);
#pragma unroll
    for (int i = 0; i < 2 * B; ++i) {
        if constexpr (B == 4)
            r.w[i] = __float_as_uint(f[i]);
        else
            r.w[i] = pack(f[2 * i], f[2 * i + 1], TYPE == ASPIS_BF16);
    }
    return r;
}

// Of this lane's group and the next lane's, the eight elements from number shift on.
template <int B>
__device__ __forceinline__ Raw<B> with_next(const Raw<B> &r, int shift)
{
    if (shift == 0) return r;
    Raw<B> next;
#pragma unroll
    for (int i = 0; i < 2 * B; ++i) next.w[i] = __shfl_down_sync(0xFFFFFFFFu, r.w[i], 1);
    return shifted(r, next, shift);
}

// token i, or -1 where it is outside the vocabulary
__device__ __forceinline__ int64_t load_token(const void *tokens, int wide, int64_t i, int64_t V)
{
    const int64_t v = wide ? static_cast<const int64_t *>(tokens)[i] : static_cast<const int32_t *>(tokens)[i];
    return v < 0 || v >= V ? -1 : v;
}

// A block's shared memory is there for the others of its cluster only once it has begun, and being scheduled together does not
// say that it has.  cluster_begin() tells the others; cluster_begun(), which comes before the first access, waits for them.  What
// lies between them hides the barrier.  All threads of all blocks of the cluster call both, or neither.
__device__ __forceinline__ void cluster_begin() { asm volatile("barrier.cluster.arrive.relaxed;\n"); }
__device__ __forceinline__ void cluster_begun() { asm volatile("barrier.cluster.wait;\n" ::: "memory"); }

// ---- on the host

// What a launch that failed leaves is not for the next call to find: the status says it.
inline aspis_status status_of(cudaError_t e)
{
    if (e == cudaSuccess) return ASPIS_OK;
    cudaGetLastError();
    return ASPIS_E_CUDA;
}

inline bool type_ok(int type) { return type == ASPIS_F32 || type == ASPIS_BF16 || type == ASPIS_F16; }

// Rows in memory.  check() refuses what no matrix is; bytes() is the range's length.
struct Rows {
    const void *p;
    int64_t rows, cols, ld;
    int type;

    aspis_status check() const
    {
        if (!type_ok(type) || ld < cols) return ASPIS_E_INVAL;
        if (rows == 0 || cols == 0) return ASPIS_OK;
        if (!p) return ASPIS_E_INVAL;
        if ((uintptr_t)p % type_bytes(type)) return ASPIS_E_ALIGN;
        if (ld > (INT64_C(1) << 58) / type_bytes(type) / rows) return ASPIS_E_RANGE;
        return ASPIS_OK;
    }
    int64_t bytes() const { return rows && cols ? ((rows - 1) * ld + cols) * type_bytes(type) : 0; }
    // groups of eight elements, from every row's first on, begin at multiples of their size
    bool by_eights() const { return (uintptr_t)p % (8 * type_bytes(type)) == 0 && (rows <= 1 || ld % 8 == 0); }
};

inline bool ranges_meet(const void *a, int64_t n, const void *b, int64_t m)
{
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return a && b && n > 0 && m > 0 && (x < y ? y - x < (uint64_t)n : x - y < (uint64_t)m);
}

// true where rows of a and b meet, or may
inline bool rows_meet(const Rows &a, const Rows &b)
{
    if (!ranges_meet(a.p, a.bytes(), b.p, b.bytes())) return false;
    const int64_t ld = a.ld * type_bytes(a.type);
    if (ld != b.ld * type_bytes(b.type)) return true;
    int64_t off = (int64_t)((uintptr_t)b.p - (uintptr_t)a.p) % ld;
    if (off < 0) off += ld;
    return off < a.cols * type_bytes(a.type) || ld - off < b.cols * type_bytes(b.type);
}

// true where the number that a mask's stream is counted up by lies in a row of what is written
inline bool step_in(const Mask &m, const Rows &a)
{
    if (!m.threshold || !ranges_meet(m.step, 8, a.p, a.bytes())) return false;
    const int64_t ld = a.ld * type_bytes(a.type);
    int64_t off = (int64_t)((uintptr_t)m.step - (uintptr_t)a.p) % ld;
    if (off < 0) off += ld;
    return off < a.cols * type_bytes(a.type) || off + 8 > ld;
}

inline bool same_rows(const Rows &a, const Rows &b)
{
    return a.p == b.p && a.type == b.type && (a.ld == b.ld || a.rows <= 1);
}

}  // namespace aspis
