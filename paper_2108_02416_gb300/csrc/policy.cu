// aspis_token_logp and aspis_policy_loss: log-probabilities of tokens from rows of logits, the clipped policy
// loss with a KL term, and its gradient.
//
//     m = max_j z_j,  s = sum_j exp(a (z_j - m)),  lp = a (z_y - m) - log s
//     rho = exp(lp - old),  L = max(-A rho, -A clip(rho)),  k = exp(ref - lp) - (ref - lp) - 1
//     dz_j = c ( [j = y] - exp(a (z_j - m)) / s ),  c = grad_scale scale w a s_i
//
// Bound by HBM: logits are read once and their gradient written once.  A row is held in registers by a warp, a block or a
// cluster, from the one reading to the gradient; longer ones are read twice, the second time from L2.
// 8192 x 131,072 bf16 with the gradient 650 us (6.3 TB/s), 2047 x 50,001 fp16 at odd addresses 78.6 (4.7 TB/s: 13 waves of
// clusters, and what each waits for its token and weight and for its sums), log-probabilities of 8192 x 32,000 bf16 83 (6.3 TB/s).
// The terms of the sums go to the workspace row by row and are added by one more kernel in a fixed order.
#include <cooperative_groups.h>
#include <limits.h>
#include <math.h>

#include "worker.cuh"

using namespace aspis;

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kScore = 0, kLoss = 1, kGrad = 2;   // what a kernel gives

struct Args {
    const void *logits, *tokens;
    void *grad;
    const float *old, *ref, *advantage, *weight;
    float *logp;
    float4 *terms;                                // w (L + beta k), w L, w k, w [clipped] of a row
    int64_t T, V, ld, ld_grad;
    float a, low, high, beta, scale, factor;      // low, high: the bounds of the ratio; factor: grad_scale scale a
    int32_t wide_tokens;
    int32_t blocks, share;                        // that have a row: a cluster; groups of each (rows of any alignment)
    int32_t ahead;                                // rows whose blocks run at the same time
};

__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// The maximum of some elements, and the sum of 2^(k z - c) over them.  c is the rounded product k m: what matters is that it is
// the same number in all of them, so each exponent is one fused multiply-add with one rounding.  Where it is beyond
// 2^30 (masks of a type's lowest value, and nothing else in the row), neighbouring logits lie further than 2^64 apart: only those that
// equal m count, and the product may overflow (`far`).  Nothing but -infinity: c = 0 and a sum of 0.
struct Part {
    float m, s;
};

struct Base {
    float c;
    bool far;

    __device__ Base(float m, float k)
    {
        c = m == -INFINITY ? 0.0f : __fmul_rn(m, k);
        far = !(fabsf(c) < 0x1p30f);
    }
};

// a far row's: 1 for the maximum; NaN where an element, or the maximum, is none of the numbers
__device__ __forceinline__ float far_weight(float z, float m) { return z == m ? (isinf(m) ? NAN : 1.0f) : z != z ? NAN : 0.0f; }

__device__ __forceinline__ float weight(float z, float m, Base b, float k)
{
    return b.far ? far_weight(z, m) : exp2_fast(fmaf(z, k, -b.c));
}

// what a sum with maximum `from` is multiplied by where the maximum is `to`
__device__ __forceinline__ float scale_to(float from, float to, float k)
{
    const Base x(from, k), y(to, k);
    return from == to ? 1.0f : x.far || y.far || from == -INFINITY ? 0.0f : exp2_fast(x.c - y.c);
}

__device__ __forceinline__ float max_of_lanes(float x)
{
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
    return r;
}

// the parts of `size` neighbouring lanes (a power of two) in one; all lanes have it, if those of other groups have the same
__device__ __forceinline__ Part join_lanes(Part p, int size, float k)
{
    const float m = max_of_lanes(p.m);
    float s = p.s * scale_to(p.m, m, k);
    for (int o = size / 2; o > 0; o /= 2) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
    return {m, s};
}

// A row's elements: `head` before the first group of eight at a multiple of its size, groups, and the rest.
template <class T>
struct Cut {
    T head, groups, tail;                         // tail: its first element

    __device__ Cut(const void *row, T V, int bytes)
    {
        const int h = (int)((uintptr_t)row % (8 * bytes)) / bytes;
        head = min((T)(h ? 8 - h : 0), V);
        groups = (T)((V - head) / 8);
        tail = head + 8 * groups;
    }
    // the element outside the groups that thread t has, or -1
    __device__ T edge(int t, T V) const
    {
        if (t < 8) return t < head ? t : -1;
        return t < 16 && tail + t - 8 < V ? tail + t - 8 : -1;
    }
};

// two elements in one word of a group, or one
template <int TYPE>
constexpr uint32_t kNothing = TYPE == ASPIS_F32 ? 0xFF800000u : TYPE == ASPIS_BF16 ? 0xFF80FF80u : 0xFC00FC00u;

// the largest elements of two words; a NaN yields to a number
template <int TYPE>
__device__ __forceinline__ uint32_t max_words(uint32_t x, uint32_t y)
{
    uint32_t r;
    if constexpr (TYPE == ASPIS_F32)
        r = __float_as_uint(fmaxf(__uint_as_float(x), __uint_as_float(y)));
    else if constexpr (TYPE == ASPIS_BF16)
        asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(x), "r"(y));
    else
        asm("max.f16x2 %0, %1, %2;" : "=r"(r) : "r"(x), "r"(y));
    return r;
}

// What a row's loss needs besides its log-probability, fetched before that is known.
struct Given {
    float advantage, old, ref;

    __device__ Given(const Args &a, int64_t i) : advantage(a.advantage[i]), old(a.old ? a.old[i] : 0.0f), ref(a.ref ? a.ref[i] : 0.0f) {}
    __device__ Given() : advantage(0.0f), old(0.0f), ref(0.0f) {}
};

// Its loss, and its slope (d loss / d lp, of one token)
struct Loss {
    float loss, kl, clipped, slope;
};

__device__ __forceinline__ Loss row_loss(const Args &a, const Given &g, float lp)
{
    Loss r;
    const float adv = g.advantage, ratio = a.old ? expf(lp - g.old) : 1.0f + 0.0f * lp;
    const float free = -adv * ratio, bound = -adv * fminf(fmaxf(ratio, a.low), a.high);
    const bool clipped = bound > free;
    r.loss = adv == 0.0f ? 0.0f : clipped ? bound : free;
    r.slope = adv == 0.0f || clipped ? 0.0f : free;
    r.clipped = clipped ? 1.0f : 0.0f;
    r.kl = 0.0f;
    if (a.ref) {
        const float d = g.ref - lp, e = expm1f(d);
        r.kl = e - d;
        if (a.beta > 0.0f) r.slope -= a.beta * e;
    }
    return r;
}

struct Row {
    const char *in;
    char *out;
    int64_t i, y;                                 // y < 0: the row does not count
    float w;
};

template <int TYPE, int MODE>
__device__ __forceinline__ Row make_row(const Args &a, int64_t i)
{
    Row r;
    r.i = i;
    r.in = static_cast<const char *>(a.logits) + i * a.ld * kBytes<TYPE>;
    r.out = static_cast<char *>(a.grad) + i * a.ld_grad * kBytes<TYPE>;
    r.y = load_token(a.tokens, a.wide_tokens, i, a.V);
    r.w = MODE != kScore && a.weight ? a.weight[i] : 1.0f;
    if (r.w == 0.0f) r.y = -1;
    return r;
}

// What is written of a row that does not count, by `size` threads.
template <int TYPE, int MODE>
__device__ __forceinline__ void skip_row(const Args &a, const Row &r, int64_t t, int64_t size)
{
    if (t == 0) {
        if (a.logp) a.logp[r.i] = 0.0f;
        if (MODE != kScore) a.terms[r.i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    }
    if constexpr (MODE == kGrad) {
        const Cut<int64_t> cut(r.out, a.V, kBytes<TYPE>);
        const float zero[8] = {};
        for (int64_t g = t; g < cut.groups; g += size)
            store_floats<kBytes<TYPE>>(r.out + (cut.head + 8 * g) * kBytes<TYPE>, zero, TYPE == ASPIS_BF16);
        const int64_t e = t < 16 ? cut.edge((int)t, a.V) : -1;
        if (e >= 0) store_elem<TYPE>(r.out, e, 0.0f);
    }
}

// What the row's elements become in the gradient: 2^(k z - c) * minus, and the token's own.
struct Slope {
    float minus, own;
};

// The row's log-probability and its terms, and its gradient's factors.
template <int MODE>
__device__ __forceinline__ Slope finish_row(const Args &a, const Row &r, const Given &given, const Part &p, float zy, bool first)
{
    const float k = a.a * kLog2e;
    const Base base(p.m, k);
    // from the difference to the maximum, which loses least (logits of 16 bits: nothing); the maximum's own exponent is what
    // rounding left of k m - c.  Where it has more than half of the sum, the rest is taken by itself: nothing beside the
    // maximum makes exactly 0, as 2^(k m - c) is the same number in the sum and here.
    float lp;
    if (!base.far) {
        const float left = fmaf(p.m, k, -base.c), top = exp2_fast(left), rest = p.s - top;
        float share = kLn2 * (left - log2f(p.s)); // the maximum's log-probability
        if (rest < top) share = -log1pf(rest / top);
        lp = fmaf(a.a, zy - p.m, share);
    } else {
        lp = isinf(p.m) ? NAN : (zy == p.m ? 0.0f : a.a * (zy - p.m)) - logf(p.s);
    }
    lp = lp > 0.0f ? 0.0f : lp;                   // (roundings; a NaN stays)
    if (MODE == kScore) {
        if (first) a.logp[r.i] = lp;
        return {0.0f, 0.0f};
    }
    const Loss l = row_loss(a, given, lp);
    if (first) {
        if (a.logp) a.logp[r.i] = lp;
        a.terms[r.i] = make_float4(r.w * (a.beta > 0.0f && a.ref ? l.loss + a.beta * l.kl : l.loss), r.w * l.loss,
                                   r.w * l.kl, r.w * l.clipped);
    }
    if (MODE != kGrad) return {0.0f, 0.0f};
    const float c = a.factor * r.w * l.slope, part = 1.0f / p.s;
    return {-c * part, c * ((p.s - weight(zy, p.m, base, k)) * part)};
}

// The kernel that adds the rows' terms may be scheduled while this one runs; it waits for its end.
__device__ __forceinline__ void next_may_start() { asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory"); }

// ---- rows that threads hold in registers

// A row belongs to a warp (KIND kWarp: four rows a block), a block or a cluster of up to eight; each thread holds up to 128 bytes of
// it in registers (GROUPS groups of eight) from the one reading to the gradient.
// What a row has but one of (its loss, the quotient) is left to a block's first warp: in every warp it was a third of all
// instructions.  While a row is worked on, the one that its block's successor will have is fetched into L2.
constexpr int kWarp = 0, kBlock = 1, kCluster = 2;

template <int TYPE, int MODE, int THREADS, int GROUPS, int KIND>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS)
hold_kernel(const __grid_constant__ Args a)
{
    namespace cg = cooperative_groups;
    constexpr int B = kBytes<TYPE>, size = KIND == kWarp ? 32 : THREADS;         // threads of a block that share a row
    __shared__ Part parts[THREADS / 32], ranks[8];
    __shared__ float given[3];                    // m, and what finish_row gives
    const int t = threadIdx.x % size, warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    next_may_start();
    int rank = 0, count = 1;
    int64_t i = KIND == kWarp ? (int64_t)blockIdx.x * (THREADS / 32) + warp : blockIdx.x;
    if constexpr (KIND == kCluster) {
        uint32_t cluster;
        asm("mov.u32 %0, %%clusterid.x;" : "=r"(cluster));
        rank = (int)cg::this_cluster().block_rank();
        count = a.blocks;
        i = cluster;
    }
    if (KIND == kWarp && i >= a.T) return;
    const int V = (int)a.V;
    const Row r = make_row<TYPE, MODE>(a, i);
    if (r.y < 0) {
        skip_row<TYPE, MODE>(a, r, rank * size + t, count * size);
        return;                                   // (in all blocks of a cluster)
    }
    if constexpr (KIND == kCluster) cluster_begin();
    const float k = a.a * kLog2e;
    const Cut<int> cut(r.in, V, B);
    const int share = KIND == kCluster ? a.share : cut.groups, from = rank * share;
    const int mine = min(share, cut.groups - from);               // groups of this block, 0 or less: none
    if (KIND != kWarp && threadIdx.x == THREADS - 1 && i + a.ahead < a.T) {
        const Row next = make_row<TYPE, MODE>(a, i + a.ahead);
        const Cut<int> c(next.in, V, B);
        const int bytes = KIND == kCluster ? min(share, c.groups - from) * 8 * B : c.groups * 8 * B;
        if (next.y >= 0 && bytes > 0)
            asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(next.in + (c.head + 8 * from) * B), "r"(bytes) : "memory");
    }
    // a warp's lanes go through the same slots; all but the last one are full
    const int left = mine - (t - lane);
    const char *at = r.in + ((int64_t)cut.head + 8 * (from + t)) * B;
    constexpr int step = size * 8 * B;
    Raw<B> v[GROUPS];
#pragma unroll
    for (int n = 0; n < GROUPS; ++n) {
        if (left - n * size >= 32) {
            v[n] = load_raw(at + n * step, (Raw<B> *)nullptr);
        } else {
#pragma unroll
            for (int j = 0; j < 2 * B; ++j) v[n].w[j] = kNothing<TYPE>;
            if (lane < left - n * size) v[n] = load_raw(at + n * step, (Raw<B> *)nullptr);
        }
    }
    int edge = -1;
    float ze = -INFINITY, zy = 0.0f;
    Given known;
    if (t < 32) {
        if constexpr (MODE != kScore) known = Given(a, i);
        if (rank == 0) edge = cut.edge(t, V);
        if (edge >= 0) ze = load_elem<TYPE>(r.in, edge);
        zy = load_elem<TYPE>(r.in, r.y);
    }
    if constexpr (KIND == kCluster) cluster_begun();              // (while the loads are on their way)

    uint32_t top = kNothing<TYPE>;
#pragma unroll
    for (int n = 0; n < GROUPS; ++n) {
        if (left <= n * size) break;
#pragma unroll
        for (int j = 0; j < 2 * B; ++j) top = max_words<TYPE>(top, v[n].w[j]);
    }
    Part p;
    if constexpr (B == 4) {
        p.m = fmaxf(__uint_as_float(top), ze);
    } else {
        const float2 m = unpack(top, TYPE == ASPIS_BF16);
        p.m = fmaxf(fmaxf(m.x, m.y), ze);
    }
    p.m = max_of_lanes(p.m);
    const Base own(p.m, k);
    if (!own.far) {
        float2 s = {t < 32 ? exp2_fast(fmaf(ze, k, -own.c)) : 0.0f, 0.0f};
        const float2 kk = {k, k}, cc = {-own.c, -own.c};
#pragma unroll
        for (int n = 0; n < GROUPS; ++n) {
            if (left <= n * size) break;
            float z[8];
            to_floats(v[n], TYPE == ASPIS_BF16, z);
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                const float2 x = __ffma2_rn(make_float2(z[j], z[j + 1]), kk, cc);
                s = __fadd2_rn(s, make_float2(exp2_fast(x.x), exp2_fast(x.y)));
            }
        }
        p.s = s.x + s.y;
    } else {
        p.s = far_weight(ze, p.m);
#pragma unroll
        for (int n = 0; n < GROUPS; ++n) {
            float z[8];
            to_floats(v[n], TYPE == ASPIS_BF16, z);
#pragma unroll
            for (int j = 0; j < 8; ++j) p.s += far_weight(z[j], p.m);
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o /= 2) p.s += __shfl_xor_sync(0xFFFFFFFFu, p.s, o);
    const Part nothing = {-INFINITY, 0.0f};
    if constexpr (KIND != kWarp) {
        if (lane == 0) parts[warp] = p;
        __syncthreads();
        if (warp == 0) p = join_lanes(lane < size / 32 ? parts[lane] : nothing, 32, k);
    }
    if constexpr (KIND == kCluster) {
        auto cluster = cg::this_cluster();
        if (threadIdx.x < count) *cluster.map_shared_rank(&ranks[rank], threadIdx.x) = p;
        cluster.sync();
        if (warp == 0) p = join_lanes(lane < count ? ranks[lane] : nothing, 32, k);
    }
    __syncwarp();                                 // the token's element is read everywhere before one is overwritten
    Slope slope = {};
    if (t < 32) slope = finish_row<MODE>(a, r, known, p, zy, rank == 0 && t == 0);
    if constexpr (MODE == kGrad) {
        if constexpr (KIND != kWarp) {
            if (t == 0) given[0] = p.m, given[1] = slope.minus, given[2] = slope.own;
            __syncthreads();
            p.m = given[0], slope.minus = given[1], slope.own = given[2];
        }
        const float minus = slope.minus;
        const Base base(p.m, k);
        const float2 kk = {k, k}, cc = {-base.c, -base.c}, mm = {minus, minus};
        char *out = r.out + ((int64_t)cut.head + 8 * (from + t)) * B;
        const bool aligned = (uintptr_t)out % (8 * B) == 0;
#pragma unroll
        for (int n = 0; n < GROUPS; ++n) {
            if (lane >= left - n * size) break;
#pragma unroll
            for (int j = 0; j < 2 * B; ++j) asm volatile("" : "+r"(v[n].w[j]));      // nothing kept of the first exponents
            float z[8];
            to_floats(v[n], TYPE == ASPIS_BF16, z);
            if (!base.far) {
#pragma unroll
                for (int j = 0; j < 8; j += 2) {
                    const float2 x = __ffma2_rn(make_float2(z[j], z[j + 1]), kk, cc);
                    const float2 y = __fmul2_rn(make_float2(exp2_fast(x.x), exp2_fast(x.y)), mm);
                    z[j] = y.x, z[j + 1] = y.y;
                }
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) z[j] = far_weight(z[j], p.m) * minus;
            }
            if (aligned)
                store_floats<B>(out + n * step, z, TYPE == ASPIS_BF16);
            else
#pragma unroll
                for (int j = 0; j < 8; ++j) store_elem<TYPE>(out + n * step, j, z[j]);
        }
        if (edge >= 0) store_elem<TYPE>(r.out, edge, weight(ze, p.m, base, k) * minus);
        // the token's own element, by the thread that has just written the others of its group
        const int y = (int)r.y, g = y < cut.head || y >= cut.tail ? -1 : (y - cut.head) / 8 - from;
        if (edge == y || (g >= 0 && g < mine && g % size == t)) store_elem<TYPE>(r.out, y, slope.own);
    }
}

// ---- rows of any length: read twice, the second time from L2

template <int TYPE, int MODE>
__global__ void __launch_bounds__(1024)
long_kernel(const __grid_constant__ Args a)
{
    constexpr int B = kBytes<TYPE>, kThreads = 1024, kUnroll = 4;
    __shared__ Part parts[kThreads / 32];
    const int t = threadIdx.x;
    next_may_start();
    const Row r = make_row<TYPE, MODE>(a, blockIdx.x);
    if (r.y < 0) {
        skip_row<TYPE, MODE>(a, r, t, kThreads);
        return;
    }
    const float k = a.a * kLog2e;
    const Cut<int64_t> cut(r.in, a.V, B);
    const int64_t edge = cut.edge(t, a.V);
    const float ze = edge >= 0 ? load_elem<TYPE>(r.in, edge) : -INFINITY, zy = load_elem<TYPE>(r.in, r.y);
    Given known;
    if constexpr (MODE != kScore) known = Given(a, r.i);
    // groups that stay in L2, and are no read-only loads: the gradient may take their place
    auto group = [&](int64_t g, float (&z)[8]) {
        Raw<B> v;
#pragma unroll
        for (int h = 0; h < B / 2; ++h) {
            const uint4 x = *reinterpret_cast<const uint4 *>(r.in + (cut.head + 8 * g) * B + 16 * h);
            v.w[4 * h] = x.x, v.w[4 * h + 1] = x.y, v.w[4 * h + 2] = x.z, v.w[4 * h + 3] = x.w;
        }
        to_floats(v, TYPE == ASPIS_BF16, z);
    };
    Part p = {ze, weight(ze, ze, Base(ze, k), k)};
    auto add_group = [&](const float (&z)[8]) {
        float top = z[0];
#pragma unroll
        for (int j = 1; j < 8; ++j) top = fmaxf(top, z[j]);
        if (top > p.m) {
            p.s *= scale_to(p.m, top, k);
            p.m = top;
        }
        const Base b(p.m, k);
        float s = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) s += weight(z[j], p.m, b, k);
        p.s += s;
    };
    int64_t g = t;
    for (; g + (kUnroll - 1) * kThreads < cut.groups; g += kUnroll * kThreads) {
        float z[kUnroll][8];
#pragma unroll
        for (int n = 0; n < kUnroll; ++n) group(g + n * kThreads, z[n]);
#pragma unroll
        for (int n = 0; n < kUnroll; ++n) add_group(z[n]);
    }
    for (; g < cut.groups; g += kThreads) {
        float z[8];
        group(g, z);
        add_group(z);
    }
    p = join_lanes(p, 32, k);
    if (t % 32 == 0) parts[t / 32] = p;
    __syncthreads();
    p = join_lanes(parts[t % 32], 32, k);
    const Slope slope = finish_row<MODE>(a, r, known, p, zy, t == 0);
    if constexpr (MODE == kGrad) {
        const float minus = slope.minus;
        const Base base(p.m, k);
        char *out = r.out + cut.head * B;
        const bool aligned = (uintptr_t)out % (8 * B) == 0;
        for (g = t; g < cut.groups; g += kThreads) {
            float z[8];
            group(g, z);
#pragma unroll
            for (int j = 0; j < 8; ++j) z[j] = weight(z[j], p.m, base, k) * minus;
            if (aligned)
                store_floats<B>(out + g * 8 * B, z, TYPE == ASPIS_BF16);
            else
#pragma unroll
                for (int j = 0; j < 8; ++j) store_elem<TYPE>(out, g * 8 + j, z[j]);
        }
        if (edge >= 0) store_elem<TYPE>(r.out, edge, weight(ze, p.m, base, k) * minus);
        const bool inside = r.y >= cut.head && r.y < cut.tail;
        if (edge == r.y || (inside && (r.y - cut.head) / 8 % kThreads == t))
            store_elem<TYPE>(r.out, r.y, slope.own);
    }
}

// ---- the sums

// A sum as a pair of fp32 numbers, hi the rounded sum and lo what is missing (48 bits).  Where hi is not finite lo means
// nothing, and is left out of what follows: infinite terms make an infinite sum.
struct Two {
    float hi, lo;
};

__device__ __forceinline__ Two add(Two x, Two y)
{
    const float s = x.hi + y.hi, b = s - x.hi;
    const float missing = ((x.hi - (s - b)) + (y.hi - b)) + (x.lo + y.lo), e = isfinite(s) ? missing : 0.0f;
    const float hi = s + e;
    return {hi, e - (hi - s)};
}

constexpr int kSumThreads = 1024, kSumRows = 16384, kMostSums = 256;

// Adds n rows' terms: block b its share, thread t rows t, t + 1024, ..., then threads in a tree.  One block: into
// sums[], times scale; several: their pairs into `blocks`, which another launch adds in the same way.
__global__ void __launch_bounds__(kSumThreads)
sums_kernel(const float4 *terms, const Two *pairs, int64_t n, Two *blocks, float scale, float *sums, bool chained)
{
    __shared__ Two share[kSumThreads / 32][4];
    const int t = threadIdx.x, lane = t % 32;
    if (chained) chain();
    const int64_t per_block = (n + gridDim.x - 1) / gridDim.x, from = blockIdx.x * per_block, end = min(from + per_block, n);
    Two s[4] = {};
    if (pairs) {
        if (from + t < end)
#pragma unroll
            for (int j = 0; j < 4; ++j) s[j] = pairs[4 * (from + t) + j];
    } else {
#pragma unroll 8
        for (int64_t i = from + t; i < end; i += kSumThreads) {
            const float4 x = terms[i];
            s[0] = add(s[0], {x.x, 0.0f}), s[1] = add(s[1], {x.y, 0.0f});
            s[2] = add(s[2], {x.z, 0.0f}), s[3] = add(s[3], {x.w, 0.0f});
        }
    }
    auto tree = [&](int width) {
        for (int o = width / 2; o > 0; o /= 2)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                s[j] = add(s[j], {__shfl_xor_sync(0xFFFFFFFFu, s[j].hi, o), __shfl_xor_sync(0xFFFFFFFFu, s[j].lo, o)});
    };
    tree(32);
    if (lane == 0)
#pragma unroll
        for (int j = 0; j < 4; ++j) share[t / 32][j] = s[j];
    __syncthreads();
    if (t >= 32) return;
#pragma unroll
    for (int j = 0; j < 4; ++j) s[j] = share[lane % (kSumThreads / 32)][j];
    tree(kSumThreads / 32);
    if (lane >= 4) return;
    const Two x = lane == 0 ? s[0] : lane == 1 ? s[1] : lane == 2 ? s[2] : s[3];
    if (gridDim.x > 1)
        blocks[4 * blockIdx.x + lane] = x;
    else
        sums[lane] = isfinite(x.hi) ? fmaf(x.hi, scale, x.lo * scale) : x.hi * scale;
}

template <int TYPE, int MODE, int THREADS, int KIND>
cudaError_t launch_hold(Args a, int blocks, cudaStream_t stream)
{
    constexpr int kGroups = 16 / kBytes<TYPE>;
    a.blocks = blocks;
    a.share = (int32_t)((a.V / 8 + blocks - 1) / blocks);
    a.ahead = kSMs * (1024 / THREADS) / blocks;
    if constexpr (KIND != kCluster) {
        constexpr int kRows = KIND == kWarp ? THREADS / 32 : 1;
        hold_kernel<TYPE, MODE, THREADS, kGroups, KIND><<<(unsigned)((a.T + kRows - 1) / kRows), THREADS, 0, stream>>>(a);
        return cudaGetLastError();
    }
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = (unsigned)blocks, at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.gridDim = dim3((unsigned)a.T * (unsigned)blocks);
    cfg.blockDim = dim3(THREADS);
    cfg.stream = stream;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, hold_kernel<TYPE, MODE, THREADS, kGroups, kCluster>, a);
}

// Blocks of a row, of 16 or 10 warps, by what a multiprocessor's two or three blocks hold together (more blocks, which wait for
// one another, have to hold a tenth more: 25,000 bf16 logits took 73 us in one block, 131 in seven of two warps); 0: eight
// are too few.  4096 x 40,000 fp16 117 us in two of 10, 136 in two of 16; 2048 x 200,000 bf16 308 in seven, 322 in eight.
struct Blocks {
    int blocks, warps;
};

inline Blocks cluster_of(int64_t groups, int held)
{
    Blocks best = {0, 0};
    int64_t most = 0;
    for (int blocks = 2; blocks <= 8; ++blocks)
        for (int warps : {16, 10}) {
            const int64_t share = (groups + blocks - 1) / blocks, together = 32 / warps * share;
            if (share <= (int64_t)warps * held && together * 10 > most * 11) best = {blocks, warps}, most = together;
        }
    return best;
}

template <int TYPE, int MODE>
cudaError_t launch_rows(const Args &a, cudaStream_t stream)
{
    constexpr int kHeld = 32 * 16 / kBytes<TYPE>;                                // a warp's groups
    const int64_t groups = a.V / 8, warps = (groups + kHeld - 1) / kHeld;        // at most; that hold a row
    // as few warps as hold the row, for what they do not hold is not in flight: 9000 x 3000 bf16 28.0 us in two warps, 32.7 in
    // four; x 10,000 62.8 in five, 69.4 in eight (inputs in turn)
    if (warps <= 1) return launch_hold<TYPE, MODE, 128, kWarp>(a, 1, stream);
    if (warps <= 2) return launch_hold<TYPE, MODE, 64, kBlock>(a, 1, stream);
    if (warps <= 4) return launch_hold<TYPE, MODE, 128, kBlock>(a, 1, stream);
    if (warps <= 5) return launch_hold<TYPE, MODE, 160, kBlock>(a, 1, stream);
    if (warps <= 8) return launch_hold<TYPE, MODE, 256, kBlock>(a, 1, stream);
    if (warps <= 10) return launch_hold<TYPE, MODE, 320, kBlock>(a, 1, stream);
    if (warps <= 16) return launch_hold<TYPE, MODE, 512, kBlock>(a, 1, stream);
    if (a.T <= INT32_MAX >> 3) {
        const Blocks c = cluster_of(groups, kHeld);
        if (c.warps == 16) return launch_hold<TYPE, MODE, 512, kCluster>(a, c.blocks, stream);
        if (c.warps == 10) return launch_hold<TYPE, MODE, 320, kCluster>(a, c.blocks, stream);
        // a multiprocessor for each block: one row of 200,000 fp32 logits 31.5 us in long_kernel, 8.7 so
        if (warps <= 8 * 32) return launch_hold<TYPE, MODE, 1024, kCluster>(a, 8, stream);
    }
    long_kernel<TYPE, MODE><<<(unsigned)a.T, 1024, 0, stream>>>(a);
    return cudaGetLastError();
}

template <int MODE>
cudaError_t launch_types(const Args &a, int type, cudaStream_t stream)
{
    if (type == ASPIS_F32) return launch_rows<ASPIS_F32, MODE>(a, stream);
    return type == ASPIS_BF16 ? launch_rows<ASPIS_BF16, MODE>(a, stream) : launch_rows<ASPIS_F16, MODE>(a, stream);
}

int64_t sum_blocks(int64_t T)
{
    const int64_t n = (T + kSumRows - 1) / kSumRows;
    return n < 1 ? 1 : n < kMostSums ? n : kMostSums;
}

aspis_status check_rows(const Rows &logits, const void *tokens, int token_type, float logit_scale)
{
    if (logits.rows < 0 || logits.cols < 1 || (token_type != ASPIS_I32 && token_type != ASPIS_I64) ||
        !(logit_scale > 0) || isinf(logit_scale))
        return ASPIS_E_INVAL;
    const aspis_status s = logits.check();
    if (s != ASPIS_OK || logits.rows == 0) return s;
    if (!tokens) return ASPIS_E_INVAL;
    if ((uintptr_t)tokens % (token_type == ASPIS_I64 ? 8 : 4)) return ASPIS_E_ALIGN;
    return logits.rows > INT32_MAX ? ASPIS_E_RANGE : ASPIS_OK;
}

}  // namespace

extern "C" aspis_status aspis_token_logp(const void *logits, int type, int64_t ld, const void *tokens, int token_type,
                                         int64_t T, int64_t V, float logit_scale, float *logp, void *stream)
{
    const Rows in{logits, T, V, ld, type};
    const aspis_status s = check_rows(in, tokens, token_type, logit_scale);
    if (s != ASPIS_OK || T == 0) return s;
    if (!logp) return ASPIS_E_INVAL;
    if ((uintptr_t)logp % 4) return ASPIS_E_ALIGN;
    if (ranges_meet(logp, 4 * T, logits, in.bytes()) || ranges_meet(logp, 4 * T, tokens, T * (token_type == ASPIS_I64 ? 8 : 4)))
        return ASPIS_E_INVAL;
    Args a{};
    a.logits = logits, a.tokens = tokens, a.logp = logp;
    a.T = T, a.V = V, a.ld = ld, a.a = logit_scale;
    a.wide_tokens = token_type == ASPIS_I64;
    return status_of(launch_types<kScore>(a, type, (cudaStream_t)stream));
}

extern "C" size_t aspis_policy_workspace_bytes(int64_t T)
{
    return T < 0 || T > INT32_MAX ? 0 : (size_t)T * sizeof(float4) + 4 * kMostSums * sizeof(Two);
}

extern "C" aspis_status aspis_policy_loss(const aspis_policy_args *p, void *stream)
{
    if (!p || !(p->clip_low >= 0 && p->clip_low <= 1) || !(p->clip_high >= 0) || !(p->kl_coef >= 0) || isinf(p->kl_coef) ||
        !isfinite(p->scale) || !isfinite(p->grad_scale))
        return ASPIS_E_INVAL;
    const Rows in{p->logits, p->T, p->V, p->ld, p->type}, out{p->grad, p->T, p->V, p->ld_grad, p->type};
    aspis_status s = check_rows(in, p->tokens, p->token_type, p->logit_scale);
    if (s == ASPIS_OK && p->grad) s = out.check();
    if (s != ASPIS_OK) return s;
    // infinite, it would make NaN of a slope of 0; below the normal numbers it would have few bits
    const float factor = (float)((double)p->grad_scale * p->scale * p->logit_scale);
    if (p->grad && !isnormal(factor) && p->grad_scale != 0.0f && p->scale != 0.0f) return ASPIS_E_RANGE;
    const int64_t T = p->T, work = (int64_t)aspis_policy_workspace_bytes(T);
    if (!p->sums || (T > 0 && (!p->advantages || !p->work))) return ASPIS_E_INVAL;
    const float *const rows[] = {p->old_logp, p->ref_logp, p->advantages, p->weights, p->logp, p->sums};
    for (const float *r : rows)
        if ((uintptr_t)r % 4) return ASPIS_E_ALIGN;
    if ((uintptr_t)p->work % 16) return ASPIS_E_ALIGN;
    if (T > 0 && p->work_bytes < (size_t)work) return ASPIS_E_RANGE;
    // what is written meets nothing else
    const struct {
        const void *p;
        int64_t n;
    } written[] = {{p->sums, 16}, {p->logp, 4 * T}, {p->work, T ? work : 0}, {p->grad, out.bytes()}},
      read[] = {{p->tokens, T * (p->token_type == ASPIS_I64 ? 8 : 4)}, {p->old_logp, 4 * T}, {p->ref_logp, 4 * T},
                {p->advantages, 4 * T}, {p->weights, 4 * T}, {p->logits, in.bytes()}};
    for (int i = 0; i < 4; ++i) {
        for (int j = 0; j < i; ++j)
            if (ranges_meet(written[i].p, written[i].n, written[j].p, written[j].n)) return ASPIS_E_INVAL;
        for (int j = 0; j < 6; ++j)
            if (!(i == 3 && j == 5) && ranges_meet(written[i].p, written[i].n, read[j].p, read[j].n)) return ASPIS_E_INVAL;
    }
    if (p->grad && rows_meet(in, out) && !same_rows(in, out)) return ASPIS_E_INVAL;
    Args a{};
    a.logits = p->logits, a.tokens = p->tokens, a.grad = p->grad;
    a.old = p->old_logp, a.ref = p->ref_logp, a.advantage = p->advantages, a.weight = p->weights;
    a.logp = p->logp;
    a.terms = static_cast<float4 *>(p->work);
    a.T = T, a.V = p->V, a.ld = p->ld, a.ld_grad = p->ld_grad;
    a.a = p->logit_scale, a.low = 1.0f - p->clip_low, a.high = 1.0f + p->clip_high;
    a.beta = p->kl_coef, a.scale = p->scale, a.factor = factor;
    a.wide_tokens = p->token_type == ASPIS_I64;
    const cudaStream_t st = (cudaStream_t)stream;
    if (T == 0) {
        sums_kernel<<<1, kSumThreads, 0, st>>>(nullptr, nullptr, 0, nullptr, a.scale, p->sums, false);
        return status_of(cudaGetLastError());
    }
    cudaError_t e = a.grad ? launch_types<kGrad>(a, p->type, st) : launch_types<kLoss>(a, p->type, st);
    const int64_t blocks = sum_blocks(T);
    Two *const pairs = reinterpret_cast<Two *>(a.terms + T);
    if (e == cudaSuccess)
        e = launch_chained(sums_kernel, blocks, kSumThreads, 0, st, (const float4 *)a.terms, (const Two *)nullptr, T, pairs,
                           a.scale, p->sums, true);
    if (e == cudaSuccess && blocks > 1)
        e = launch_chained(sums_kernel, 1, kSumThreads, 0, st, (const float4 *)nullptr, (const Two *)pairs, blocks,
                           (Two *)nullptr, a.scale, p->sums, true);
    return status_of(e);
}
