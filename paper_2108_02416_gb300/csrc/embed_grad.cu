// aspis_embed_grad: the gradient of a table of embeddings, by sorted tokens.
//
//     dtable[v] (+)= scale * sum over i with token_i = v of drop( dy[i] )
//
// A sum of atomics would have an order of its own in every run.  Here tokens are sorted stably by counting, nine
// bits at a time, and the sums run over the sorted positions: a block has 256 of them (64 where there are few) and
// 256 columns, each of its warps an eighth.  A token whose run stays inside a warp's piece is written at once; runs that
// pass from piece to piece are joined in shared memory, those that pass from block to block in
// the workspace.  So long runs (a text's commonest token is a tenth of it) and tokens that occur once cost
// the same, and the order of a sum depends on the tokens and the sizes alone.
// Bound by HBM where T is large: 131,072 tokens x 2048 bf16 added to fp32 201 us, 172 of it the sums (6.2 TB/s), the
// rest the sort in three launches and the joins.  Not where they go through a mask (x 1024 133 us, 90 without; x 1001 223 and 130): a
// row's words are drawn after the row has arrived, so that both times add up; nor where rows are narrow (x 16 39 us: the sort).  8192 x 1024 with a mask into 32,000 rows 33 us (131 MB of it zeros and sums
// written: 19), half of which is the latency of two launches and of the sums' last joins.
#include <cooperative_groups.h>
#include <limits.h>
#include <math.h>

#include "worker.cuh"

using namespace aspis;

namespace {

constexpr int kSortThreads = 512, kSortWarps = kSortThreads / 32;
constexpr int kRounds = 4, kSubTile = kSortThreads * kRounds;
constexpr int kDigits = 512;
constexpr int kMostTiles = 256;
constexpr int kTile = 256;                        // a lane's eight columns, 32 times
// a block's columns: where rows begin anywhere, the last lane only helps its neighbour
template <bool EIGHTS>
constexpr int kCols = EIGHTS ? 256 : 248;
constexpr int kPiece = 32, kChunk = kPiece * kRowWarps;          // sorted positions of a warp, of a block
constexpr int kJoinWarps = 2;
constexpr int kFewPiece = 8, kFewBlocks = 2 * kSMs;    // where that makes few blocks
constexpr int kFewTokens = 8 * kSubTile, kOneTokens = 1024;      // sorted by a cluster of eight blocks, by one block

static_assert(kOneTokens <= kSubTile, "a block's pairs in shared memory");
static_assert(kSortThreads == kDigits && kDigits == 4 * 128 && sizeof(uint2) * kSubTile >= 2 * sizeof(uint4) * kSortThreads, "scatter_kernel's sums");

struct Plan {
    int64_t T, V, width;
    int bits, passes;                             // of a digit; over the tokens
    uint32_t tiles, tile;                         // blocks of the sort, and their tokens
    uint32_t chunks;
    bool few, fine;                               // sorted by one cluster; chunks of kFewPiece positions a warp
    int64_t columns;
    size_t tables, pairs[2], arrived, parts, bytes;
};

bool make_plan(int64_t T, int64_t V, int64_t width, Plan &p)
{
    if (T < 0 || V < 1 || width < 0 || T > INT32_MAX || V > INT32_MAX) return false;
    p = Plan{};
    p.T = T, p.V = V, p.width = width;
    int need = 1;
    while (need < 32 && V >> need) ++need;        // of the keys 0 .. V, V being padding
    p.passes = (need + 8) / 9;
    p.bits = (need + p.passes - 1) / p.passes;
    p.few = T <= kFewTokens;
    p.tiles = (uint32_t)((T + kSubTile - 1) / kSubTile);
    if (p.tiles > kMostTiles) p.tiles = kMostTiles;
    if (p.tiles == 0) p.tiles = 1;
    p.tile = (uint32_t)((T + p.tiles - 1) / p.tiles);
    p.columns = (width + kCols<false> - 1) / kCols<false>;        // at most
    const int64_t coarse = (T + kChunk - 1) / kChunk, most = 4 * kFewBlocks;
    if (width > (INT64_C(1) << 50) / (coarse + 1)) return false;
    p.fine = coarse * p.columns < kFewBlocks;
    p.chunks = (uint32_t)(p.fine ? (T + kFewPiece * kRowWarps - 1) / (kFewPiece * kRowWarps) : coarse);
    size_t at = 0;
    auto take = [&](size_t n) {
        const size_t here = at;
        at += (n + 255) / 256 * 256;
        return here;
    };
    p.tables = take((size_t)p.passes * p.tiles * kDigits * 4);
    for (int i = 0; i < 2; ++i) p.pairs[i] = take((size_t)T * sizeof(uint2));
    // (for more tokens or a wider table never less, though their chunks are longer)
    p.arrived = take((size_t)most * 4);
    const size_t parts = (size_t)coarse * 2 * (size_t)p.columns * kTile * 4, fine = (size_t)most * 2 * kTile * 4;
    p.parts = take(T == 0 ? 0 : parts < fine ? fine : parts);
    p.bytes = at;
    return true;
}

// ---- the sort

// a pair is a token's key (V for padding) and its position
struct SortArgs {
    const void *tokens;                           // of the first pass, or NULL
    const uint2 *pairs;
    uint2 *out;
    uint32_t *table, *next;                       // [tiles][kDigits] of this pass, and of the one after it or NULL
    uint32_t T, V, tiles, tile;
    int32_t wide_tokens, shift, bits;
    uint32_t clear;                               // words behind `next` that the count clears
    uint32_t *arrived;                            // and other words
    int64_t arrived_size;
};

__device__ __forceinline__ uint2 sort_pair(const SortArgs &a, uint32_t i)
{
    if (!a.tokens) return a.pairs[i];
    const int64_t v = load_token(a.tokens, a.wide_tokens, i, a.V);
    return make_uint2(v < 0 ? a.V : (uint32_t)v, i);
}

// The sum of the values of all threads before this one.
__device__ __forceinline__ uint32_t sum_before(uint32_t x, uint32_t (&sums)[kSortWarps])
{
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    uint32_t scan = x;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
        const uint32_t v = __shfl_up_sync(0xFFFFFFFFu, scan, o);
        if (lane >= o) scan += v;
    }
    __syncthreads();                              // the last call's sums have been read
    if (lane == 31) sums[warp] = scan;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kSortWarps; ++w) scan += w < warp ? sums[w] : 0;
    return scan - x;
}

// The lanes whose digit is this lane's, of those that have one (in), by a ballot a bit.
template <int BITS>
__device__ __forceinline__ uint32_t same_digit(uint32_t digit, bool in)
{
    uint32_t same = __ballot_sync(0xFFFFFFFFu, in);
#pragma unroll
    for (int b = 0; b < BITS; ++b) {
        const bool set = digit >> b & 1;
        const uint32_t with = __ballot_sync(0xFFFFFFFFu, set);
        same &= set ? with : ~with;
    }
    return same;
}

// the first pass's digits by tiles; the other passes' are counted by the pass before
__global__ void __launch_bounds__(kSortThreads)
count_kernel(const __grid_constant__ SortArgs a)
{
    __shared__ uint32_t n[kDigits];
    n[threadIdx.x] = 0;
    for (uint32_t i = blockIdx.x * kSortThreads + threadIdx.x; i < a.clear; i += gridDim.x * kSortThreads) a.next[i] = 0;
    for (int64_t i = blockIdx.x * kSortThreads + threadIdx.x; i < a.arrived_size; i += gridDim.x * kSortThreads) a.arrived[i] = 0;
    __syncthreads();
    const uint32_t begin = blockIdx.x * a.tile, end = min(begin + a.tile, a.T), mask = (1u << a.bits) - 1;
    for (uint32_t i = begin + threadIdx.x; i < end; i += kSortThreads) atomicAdd(&n[sort_pair(a, i).x & mask], 1u);
    __syncthreads();
    a.table[blockIdx.x * kDigits + threadIdx.x] = n[threadIdx.x];
}

// A pass over a block's tile, 2048 pairs at a time: they are sorted in shared memory first, so that neighbours are
// written together (a store to 32 places takes a multiprocessor 32 times as long as one to neighbouring words).
__global__ void __launch_bounds__(kSortThreads)
scatter_kernel(const __grid_constant__ SortArgs a)
{
    __shared__ __align__(16) uint2 stage[kSubTile];
    __shared__ __align__(4) uint16_t place[kSortWarps][kDigits];   // (cleared by words)
    __shared__ uint32_t sums[kSortWarps], shift_of[kDigits];      // from the place in `stage` to that in `out`
    const int t = threadIdx.x, lane = t % 32, warp = t / 32;
    const uint32_t mask = (1u << a.bits) - 1;
    chain();
    // where this tile's first element of digit t goes: behind all smaller digits, and the tiles before.  A quarter of the
    // threads each go through a quarter of the tiles, four digits at a time.
    uint4 all4 = {}, before4 = {};
    const uint32_t quarter = (a.tiles + 3) / 4, last = min((t / 128 + 1) * quarter, a.tiles);
    for (uint32_t i = t / 128 * quarter; i < last; i += 8) {
        uint4 n[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            n[j] = i + j < last ? *reinterpret_cast<const uint4 *>(a.table + (i + j) * kDigits + t % 128 * 4) : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            all4.x += n[j].x, all4.y += n[j].y, all4.z += n[j].z, all4.w += n[j].w;
            if (i + j < blockIdx.x) before4.x += n[j].x, before4.y += n[j].y, before4.z += n[j].z, before4.w += n[j].w;
        }
    }
    uint4 *const share = reinterpret_cast<uint4 *>(stage);        // [2][4][128]
    share[t] = all4;
    share[kSortThreads + t] = before4;
    __syncthreads();
    uint32_t all = 0, before = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        all += reinterpret_cast<const uint32_t *>(share)[q * kDigits + t];
        before += reinterpret_cast<const uint32_t *>(share + kSortThreads)[q * kDigits + t];
    }
    uint32_t base = before + sum_before(all, sums);
    const uint32_t begin = blockIdx.x * a.tile, end = min(begin + a.tile, a.T);
    for (uint32_t sub = begin; sub < end; sub += kSubTile) {
        uint2 pair[kRounds];
        uint32_t rank[kRounds];
        const uint32_t i0 = sub + warp * (32 * kRounds) + lane, size = min(end - sub, (uint32_t)kSubTile);
#pragma unroll
        for (int r = 0; r < kRounds; ++r) pair[r] = i0 + 32 * r < end ? sort_pair(a, i0 + 32 * r) : make_uint2(0, 0);
#pragma unroll
        for (int i = 0; i < kDigits / 64; ++i) reinterpret_cast<uint32_t *>(place[warp])[32 * i + lane] = 0;
        __syncwarp();
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
            const bool in = i0 + 32 * r < end;
            const uint32_t digit = pair[r].x >> a.shift & mask;
            const uint32_t same = same_digit<9>(digit, in), below = __popc(same & ((1u << lane) - 1));
            const uint32_t so_far = place[warp][digit];
            rank[r] = so_far + below;
            __syncwarp();
            if (in && below == 0) place[warp][digit] = (uint16_t)(so_far + __popc(same));
            __syncwarp();
        }
        __syncthreads();
        uint32_t n[kSortWarps], count = 0;
#pragma unroll
        for (int w = 0; w < kSortWarps; ++w) count += n[w] = place[w][t];
        uint32_t first = sum_before(count, sums);
        shift_of[t] = base - first;
        base += count;
#pragma unroll
        for (int w = 0; w < kSortWarps; ++w) {
            place[w][t] = (uint16_t)first;
            first += n[w];
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kRounds; ++r)
            if (i0 + 32 * r < end) stage[place[warp][pair[r].x >> a.shift & mask] + rank[r]] = pair[r];
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
            const uint32_t i = t + r * kSortThreads;
            if (i >= size) break;
            const uint2 x = stage[i];
            const uint32_t to = shift_of[x.x >> a.shift & mask] + i;
            a.out[to] = x;
            if (a.next) atomicAdd(&a.next[to / a.tile * kDigits + (x.x >> (a.shift + a.bits) & mask)], 1u);
        }
        __syncthreads();
    }
}

// The sort of at most 16,384 tokens in one launch, by a block or a cluster of eight: a block has a tile of pairs in shared
// memory, the blocks exchange how many of each digit they have, and write each pair into the block whose tile it goes to.
// One block's sort of 8192 tokens was bound by its instructions (16 us).  The launch's other
// blocks write zeros meanwhile (FILL), to the first rows, where no token names them.
struct FewArgs {
    const void *tokens;
    uint2 *pairs;
    uint32_t *arrived;
    char *out;
    int64_t row_bytes, ld_bytes, arrived_size;
    uint32_t T, V, fill, rows, group;             // rows that zeros are written to where no token names them; of a block, of a warp
    int32_t wide_tokens, bits, passes, tile_bits; // a tile has 2^tile_bits pairs
};

// Zeros to `bytes` of each row whose bit is set, by a warp, in pieces of 32 bytes (shorter at a row's ends): of several
// rows at a time where they are narrow.  Addresses are multiples of two.
__device__ __forceinline__ void zero_rows(char *first, int64_t ld_bytes, int64_t bytes, uint32_t rows)
{
    const int64_t pieces = (bytes + 30 + 31) / 32;                // of a row at any address, at most
    const int width = pieces < 32 ? (int)pieces : 32, together = 32 / width, mine = threadIdx.x % 32 / width;
    const Raw<4> none = {};
    while (rows) {
        uint32_t left = rows;
        for (int i = 0; i < together; ++i) {
            if (i < mine) left &= left - 1;       // this lane's row is the mine-th of those to come
            rows &= rows - 1;
        }
        if (!left || mine >= together) continue;
        char *row = first + (__ffs(left) - 1) * ld_bytes, *end = row + bytes;
        for (char *p = row - (uintptr_t)row % 32 + threadIdx.x % 32 % width * 32; p < end; p += width * 32) {
            if (p >= row && p + 32 <= end) {
                store_raw(p, none);
            } else {
                char *q = p < row ? row : p, *const to = p + 32 < end ? p + 32 : end;
                if ((uintptr_t)q % 4 && q < to) *reinterpret_cast<uint16_t *>(q) = 0, q += 2;
                for (; q + 4 <= to; q += 4) *reinterpret_cast<uint32_t *>(q) = 0;
                if (q < to) *reinterpret_cast<uint16_t *>(q) = 0;
            }
        }
    }
}

constexpr int kFillBlocks = 2 * kSMs - 1, kFillRows = 32768;
static_assert(kFillRows <= 64 * kSubTile, "their bits where the pairs are");
constexpr int64_t kFillBytes = 48 << 20;          // what is written while the cluster sorts

template <bool FILL, bool CLUSTER>
__global__ void __launch_bounds__(kSortThreads)
few_kernel(const __grid_constant__ FewArgs a)
{
    namespace cg = cooperative_groups;
    constexpr int kRanks = CLUSTER ? 8 : 1;
    __shared__ uint2 tile[kSubTile];
    __shared__ __align__(4) uint16_t place[kSortWarps][kDigits], digits[kRanks][kDigits];
    __shared__ uint32_t sums[kSortWarps];
    const int t = threadIdx.x, lane = t % 32, warp = t / 32;
    asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
    if (FILL && blockIdx.x >= kRanks) {
        // the tokens' bits of this block's rows
        uint32_t *bits = reinterpret_cast<uint32_t *>(tile);
        const uint32_t first = (blockIdx.x - kRanks) * a.rows;
        if (first >= a.fill) return;
        const uint32_t rows = min(a.rows, a.fill - first);
        for (uint32_t i = t; i < (rows + 31) / 32; i += kSortThreads) bits[i] = 0;
        __syncthreads();
        for (uint32_t i = t; i < a.T; i += kSortThreads) {
            const int64_t v = load_token(a.tokens, a.wide_tokens, i, a.V) - first;
            if (v >= 0 && v < rows) atomicOr(&bits[v / 32], 1u << (v % 32));
        }
        __syncthreads();
        // (a.group, the rows of a warp at a time, divides 32)
        for (uint32_t v = warp * a.group; v < rows; v += kSortWarps * a.group) {
            const uint32_t size = min(a.group, rows - v), empty = ~(bits[v / 32] >> (v % 32)) & (0xFFFFFFFFu >> (32 - size));
            zero_rows(a.out + (int64_t)(first + v) * a.ld_bytes, a.ld_bytes, a.row_bytes, empty);
        }
        return;
    }
    if constexpr (CLUSTER) cluster_begin();       // (the blocks above are whole clusters)
    const uint32_t rank = CLUSTER ? blockIdx.x : 0, mask = (1u << a.bits) - 1;
    const uint32_t begin = rank << a.tile_bits, size = begin < a.T ? min(1u << a.tile_bits, a.T - begin) : 0;
    // a warp has 32 * rounds neighbouring pairs
    const int rounds = ((1 << a.tile_bits) + kSortThreads - 1) / kSortThreads;
    const uint32_t i0 = warp * 32 * rounds + lane;
    for (int pass = 0; pass < a.passes; ++pass) {
        const int shift = pass * a.bits;
        uint2 pair[kRounds];
        uint32_t rank_of[kRounds];
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
            const uint32_t i = i0 + 32 * r;
            pair[r] = make_uint2(0, 0);
            if (r >= rounds || i >= size) continue;
            if (pass > 0) {
                pair[r] = tile[i];
            } else {
                const int64_t v = load_token(a.tokens, a.wide_tokens, begin + i, a.V);
                pair[r] = make_uint2(v < 0 ? a.V : (uint32_t)v, begin + i);
            }
        }
#pragma unroll
        for (int i = 0; i < kDigits / 64; ++i) reinterpret_cast<uint32_t *>(place[warp])[32 * i + lane] = 0;
        __syncwarp();
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
            if (r >= rounds) break;
            const bool in = i0 + 32 * r < size;
            const uint32_t digit = pair[r].x >> shift & mask;
            const uint32_t same = same_digit<9>(digit, in), below = __popc(same & ((1u << lane) - 1));
            const uint32_t so_far = place[warp][digit];
            rank_of[r] = so_far + below;
            __syncwarp();
            if (in && below == 0) place[warp][digit] = (uint16_t)(so_far + __popc(same));
            __syncwarp();
        }
        __syncthreads();
        uint32_t n[kSortWarps], count = 0, before = 0;
#pragma unroll
        for (int w = 0; w < kSortWarps; ++w) count += n[w] = place[w][t];
        if constexpr (CLUSTER) {
            auto cluster = cg::this_cluster();
            if (pass == 0) cluster_begun();
#pragma unroll
            for (int b = 0; b < kRanks; ++b) cluster.map_shared_rank(digits[rank], b)[t] = (uint16_t)count;
            cluster.sync();                       // and all have their pairs in registers
            count = 0;
#pragma unroll
            for (int b = 0; b < kRanks; ++b) {
                const uint32_t m = digits[b][t];
                count += m;
                before += b < rank ? m : 0;
            }
        }
        uint32_t first = before + sum_before(count, sums);
#pragma unroll
        for (int w = 0; w < kSortWarps; ++w) {
            place[w][t] = (uint16_t)first;
            first += n[w];
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
            if (r >= rounds || i0 + 32 * r >= size) continue;
            const uint32_t to = place[warp][pair[r].x >> shift & mask] + rank_of[r];
            if constexpr (CLUSTER)
                *cg::this_cluster().map_shared_rank(&tile[to & ((1u << a.tile_bits) - 1)], to >> a.tile_bits) = pair[r];
            else
                tile[to] = pair[r];
        }
        if constexpr (CLUSTER)
            cg::this_cluster().sync();
        else
            __syncthreads();
    }
    for (uint32_t i = t; i < size; i += kSortThreads) a.pairs[begin + i] = tile[i];
    // (last: the clusters' barriers wait for what has been written)
    for (int64_t i = rank * kSortThreads + t; i < a.arrived_size; i += kRanks * kSortThreads) a.arrived[i] = 0;
}

// ---- the sums

struct SumArgs {
    const void *grad;
    void *out;
    const uint2 *pairs;                           // sorted
    uint32_t *arrived;                            // [chunks][columns]: parts of the run that begins in a chunk
    float *parts;                                 // [chunks][2][columns][kTile]: of the run that began before the chunk; of the
                                                  // one that begins in it and goes on behind it
    int64_t ld, ldo, width;
    uint32_t T, V, chunks, columns;               // blocks of kCols of them
    uint32_t blocks;                              // (chunk, column); the launch's others write zeros
    uint32_t fill_from, fill_rows;                // to this row and those behind it, where no token names them; of a warp
    float factor;
    int32_t fine;                                 // chunks of kFewPiece positions a warp
    Mask mask;
};

// A lane's eight neighbouring columns of a row of the gradient, as they were loaded: where rows begin anywhere, the group that
// the first lies in (the next lane's group is the next one).
template <int TYPE, bool EIGHTS>
struct Cells {
    Raw<kBytes<TYPE>> r;
    int shift;

    // columns c0 .. c0 + n - 1 of row i
    __device__ __forceinline__ void load(const SumArgs &a, uint32_t i, int64_t c0, int n)
    {
        const int lane = threadIdx.x % 32;
        const char *p = static_cast<const char *>(a.grad) + ((int64_t)i * a.ld + c0) * kBytes<TYPE>;
        if constexpr (EIGHTS) {
            r = {};
            if (8 * lane < n) r = load_group<TYPE, false>(p + 8 * lane * kBytes<TYPE>);
        } else {
            shift = behind<kBytes<TYPE>>(p);
            r = load_around<TYPE, false>(p, 8 * lane, shift, columns_from(c0, a.width, 512), i == 0 || i + 1 == a.T || a.ld < 8);
        }
    }
    __device__ __forceinline__ void get(float (&f)[8]) const
    {
        if constexpr (EIGHTS)
            to_floats(r, TYPE == ASPIS_BF16, f);
        else
            to_floats(with_next(r, shift), TYPE == ASPIS_BF16, f);
    }
};

// The same of a row of the table: whole, or where rows begin anywhere column 32 k + lane in place k.
template <int TYPE, bool EIGHTS>
struct TableCells {
    Raw<kBytes<TYPE>> r;
    __device__ __forceinline__ void load(const SumArgs &a, uint32_t v, int64_t c0, int n)
    {
        const int c = 8 * (threadIdx.x % 32);
        r = {};
        if (c < n) r = load_group<TYPE, false>(static_cast<const char *>(a.out) + ((int64_t)v * a.ldo + c0 + c) * kBytes<TYPE>);
    }
    __device__ __forceinline__ void get(float (&f)[8]) const { to_floats(r, TYPE == ASPIS_BF16, f); }
};

template <int TYPE>
struct TableCells<TYPE, false> {
    float f[8];
    __device__ __forceinline__ void load(const SumArgs &a, uint32_t v, int64_t c0, int n)
    {
        const char *row = static_cast<const char *>(a.out) + ((int64_t)v * a.ldo + c0) * kBytes<TYPE>;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int c = 32 * k + threadIdx.x % 32;
            f[k] = c < n ? load_elem<TYPE>(row, c) : 0.0f;
        }
    }
    __device__ __forceinline__ void get(float (&g)[8]) const
    {
#pragma unroll
        for (int k = 0; k < 8; ++k) g[k] = f[k];
    }
};

// A row's sum, times the factor, to the table, or added to what was there.  Where rows begin anywhere it changes places
// through shared memory (a warp's own), so that neighbouring lanes write neighbouring elements.
template <int OUT, bool EIGHTS, bool ADD>
__device__ __forceinline__ void put(const SumArgs &a, uint32_t v, int64_t c0, int n, const float (&sum)[8],
                                    const TableCells<OUT, EIGHTS> &old, float *tile)
{
    const int lane = threadIdx.x % 32;
    char *row = static_cast<char *>(a.out) + ((int64_t)v * a.ldo + c0) * kBytes<OUT>;
    float f[8], s[8];
    if constexpr (!EIGHTS) {
        __syncwarp();
        reinterpret_cast<float4 *>(tile)[2 * lane] = make_float4(sum[0], sum[1], sum[2], sum[3]);
        reinterpret_cast<float4 *>(tile)[2 * lane + 1] = make_float4(sum[4], sum[5], sum[6], sum[7]);
        __syncwarp();
    }
    if constexpr (ADD) old.get(f);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        s[k] = EIGHTS ? sum[k] : tile[32 * k + lane];
        f[k] = ADD ? fmaf(s[k], a.factor, f[k]) : s[k] * a.factor;
    }
    if constexpr (EIGHTS) {
        if (8 * lane < n) store_floats<kBytes<OUT>>(row + 8 * lane * kBytes<OUT>, f, OUT == ASPIS_BF16);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (32 * k + lane < n) store_elem<OUT>(row, 32 * k + lane, f[k]);
    }
}

template <int OUT, bool EIGHTS, bool ADD>
__device__ __forceinline__ void emit(const SumArgs &a, uint32_t v, int64_t c0, int n, const float (&sum)[8], float *tile)
{
    TableCells<OUT, EIGHTS> old;
    if constexpr (ADD) old.load(a, v, c0, n);
    put<OUT, EIGHTS, ADD>(a, v, c0, n, sum, old, tile);
}

// A part of a run's sum in the workspace: a chunk's first (slot 0) or last one, a tile for each block of columns.
__device__ __forceinline__ float *part_of(const SumArgs &a, uint32_t chunk, int slot, uint32_t column)
{
    return a.parts + (((size_t)chunk * 2 + slot) * a.columns + column) * kTile + 8 * (threadIdx.x % 32);
}

__device__ __forceinline__ void store_part(float *p, const float (&f)[8])
{
    reinterpret_cast<float4 *>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
    reinterpret_cast<float4 *>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
}

// (past L1: another multiprocessor may just have written it)
__device__ __forceinline__ void load_part(const float *p, float (&f)[8])
{
    const float4 x = __ldcg(reinterpret_cast<const float4 *>(p)), y = __ldcg(reinterpret_cast<const float4 *>(p) + 1);
    f[0] = x.x, f[1] = x.y, f[2] = x.z, f[3] = x.w, f[4] = y.x, f[5] = y.y, f[6] = y.z, f[7] = y.w;
}

// The first position whose key is not below v, by a warp: 32 places at a time.
__device__ __forceinline__ uint32_t first_of(const uint2 *pairs, uint32_t T, uint32_t v)
{
    uint32_t lo = 0, n = T;                       // it is one of lo .. lo + n
    while (n > 0) {
        const uint32_t end = lo + n, step = (n + 31) / 32;
        const uint64_t at = (uint64_t)lo + (uint64_t)(threadIdx.x % 32) * step + step - 1;
        lo += step * __popc(__ballot_sync(0xFFFFFFFFu, at < end && pairs[at].x < v));
        lo = min(lo, end);
        n = min(step - 1, end - lo);
    }
    return lo;
}

// bit i: a token is v + i, for i < 32; by a warp.  Where 32 pairs do not reach to v + 31, each lane looks for its own.
__device__ __forceinline__ uint32_t named_rows(const uint2 *pairs, uint32_t T, uint32_t v)
{
    const int lane = threadIdx.x % 32;
    const uint32_t first = first_of(pairs, T, v);
    const uint32_t key = (uint64_t)first + lane < T ? pairs[first + lane].x : 0xFFFFFFFFu, off = key - v;
    uint32_t named = __reduce_or_sync(0xFFFFFFFFu, off < 32 ? 1u << off : 0u);
    if (__shfl_sync(0xFFFFFFFFu, off, 31) >= 31) return named;
    uint32_t lo = first + 32, n = T - lo;         // (the 32 pairs are there)
    while (n > 0) {
        const uint32_t half = n / 2;
        if (pairs[lo + half].x < v + lane)
            lo += half + 1, n -= half + 1;
        else
            n = half;
    }
    return named | __ballot_sync(0xFFFFFFFFu, lo < T && pairs[lo].x == v + lane);
}

// How many chunks before and behind `chunk` a run of v comes from and goes on into; by a warp, half of it each way.
template <int CHUNK>
__device__ __forceinline__ void neighbours_of(const SumArgs &a, uint32_t v, uint32_t chunk, bool head, uint32_t &before, uint32_t &behind)
{
    const int lane = threadIdx.x % 32;
    bool back = head, on = true;                  // ways that have not come to an end
    before = behind = 0;
    while (back || on) {
        // (a chunk's first position and the one before it are v's)
        const int64_t k = lane < 16 ? (int64_t)chunk - before - lane : (int64_t)chunk + 1 + behind + lane - 16, at = k * CHUNK;
        const bool in = at > 0 && at < a.T && a.pairs[at].x == v && a.pairs[at - 1].x == v;
        const uint32_t ends = ~__ballot_sync(0xFFFFFFFFu, in);
        const uint32_t left = __ffs(ends & 0xFFFFu | 0x10000u) - 1, right = __ffs(ends >> 16 | 0x10000u) - 1;
        if (back) before += left;
        if (on) behind += right;
        back = back && left == 16;
        on = on && right == 16;
    }
}

// Leaves a block's part of a run that has others, for join_kernel (ALONE), or for the last of them to come, which adds all in
// their order, whoever that is.  The latter saves a launch (8192 tokens x 1024 41 us, 35 so), but keeps blocks waiting for their
// stores: 131,072 tokens x 2048 took 2.5 % longer so than with the launch.
template <int OUT, bool EIGHTS, bool ADD, int PIECE>
__device__ __forceinline__ void hand_in(const SumArgs &a, uint32_t v, uint32_t chunk, bool head, uint32_t column, int n,
                                        float (&sum)[8], float *tile)
{
    const int lane = threadIdx.x % 32;
    store_part(part_of(a, chunk, !head, column), sum);
    if constexpr (PIECE == kPiece) return;
    uint32_t before, behind;
    neighbours_of<PIECE * kRowWarps>(a, v, chunk, head, before, behind);
    const uint32_t from = chunk - before, parts = before + 1 + behind;
    __threadfence();
    __syncwarp();
    uint32_t others = 0;
    if (lane == 0) others = atomicAdd(&a.arrived[(size_t)from * a.columns + column], 1u);
    if (__shfl_sync(0xFFFFFFFFu, others, 0) + 1 < parts) return;
    __threadfence();
    const int64_t c0 = (int64_t)column * kCols<EIGHTS>;
    TableCells<OUT, EIGHTS> old;
    if constexpr (ADD) old.load(a, v, c0, n);
#pragma unroll
    for (int k = 0; k < 8; ++k) sum[k] = 0.0f;
    for (uint32_t i = 0; i < parts; i += 4) {
        float f[4][8];
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (i + j < parts) load_part(part_of(a, from + i + j, i + j == 0, column), f[j]);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (i + j < parts)
#pragma unroll
                for (int k = 0; k < 8; ++k) sum[k] += f[j][k];
    }
    put<OUT, EIGHTS, ADD>(a, v, c0, n, sum, old, tile);
}

// The sums, and zeros to the rows that no token names.  Four blocks a multiprocessor (131,072 x 2048 into 131,072 rows 255 us, 272
// with three); three where rows are added to the table's, which are in flight too (200 us; 199 with four and half of them in flight).
template <int IN, int OUT, bool EIGHTS, bool ADD, int PIECE>
__global__ void __launch_bounds__(kRowThreads, ADD ? 3 : 4)
sum_kernel(const __grid_constant__ SumArgs a)
{
    // rows in flight: as many as 48 registers hold, with the rows of the table that they are added to
    constexpr int kHeld = 2 * kBytes<IN> + (!ADD ? 0 : EIGHTS ? 2 * kBytes<OUT> : 8);
    constexpr int kBatch = kHeld <= 4 ? 8 : kHeld <= 12 ? 4 : 2;
    __shared__ float heads[kRowWarps][kTile];     // of the run that began before a warp's piece
    __shared__ __align__(16) float tiles[EIGHTS ? 1 : kRowWarps][kTile];
    __shared__ uint8_t goes_on[kRowWarps];        // that run fills the piece, and the next position too
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    chain();
    // blocks that write zeros alternate with the others, so that both are at work from the start on
    const uint32_t pairs = min(a.blocks, gridDim.x - a.blocks);
    const bool fills = blockIdx.x < 2 * pairs ? blockIdx.x % 2 : pairs == a.blocks;
    const uint32_t block = blockIdx.x < 2 * pairs ? blockIdx.x / 2 : blockIdx.x - pairs;
    if (fills) {
        // rows without a token become zeros
        const uint64_t v = a.fill_from + (uint64_t)a.fill_rows * ((uint64_t)block * kRowWarps + warp);
        if (ADD || v >= a.V) return;
        const uint32_t size = (uint32_t)min((uint64_t)a.fill_rows, a.V - v);
        const uint32_t empty = ~named_rows(a.pairs, a.T, (uint32_t)v) & (0xFFFFFFFFu >> (32 - size));
        zero_rows(static_cast<char *>(a.out) + (int64_t)v * a.ldo * kBytes<OUT>, a.ldo * kBytes<OUT>, a.width * kBytes<OUT>, empty);
        return;
    }
    const uint32_t chunk = block / a.columns, column = block % a.columns;
    const int64_t c0 = (int64_t)column * kCols<EIGHTS>;
    const int n = (int)min((int64_t)kCols<EIGHTS>, a.width - c0);
    const uint32_t first = (chunk * kRowWarps + warp) * PIECE, left = first < a.T ? min((uint32_t)PIECE, a.T - first) : 0;
    float *const tile = tiles[EIGHTS ? 0 : warp];
    const uint64_t stream = mask_stream(a.mask);
    uint32_t key = a.V, index = 0, next = a.V;
    bool head = false;
    if (lane < left) {
        const uint32_t p = first + lane;
        const uint2 x = a.pairs[p];
        key = x.x, index = x.y;
        next = p + 1 < a.T ? a.pairs[p + 1].x : 0xFFFFFFFFu;
        if (lane == 0) head = p > 0 && a.pairs[p - 1].x == key;
    }
    const uint32_t real = __ballot_sync(0xFFFFFFFFu, key != a.V), ends = __ballot_sync(0xFFFFFFFFu, key != next) & real;
    head = __shfl_sync(0xFFFFFFFFu, head, 0) && real;
    const int head_end = head ? __ffs(ends) - 1 : -1;              // the position where the run from before ends, if it does
    float sum[8] = {};
#pragma unroll 1
    for (int b = 0; b < PIECE && real >> b; b += kBatch) {
        Cells<IN, EIGHTS> x[kBatch];
        TableCells<OUT, EIGHTS> old[ADD ? kBatch : 1];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            const uint32_t i = __shfl_sync(0xFFFFFFFFu, index, b + j);
            if (real >> (b + j) & 1) x[j].load(a, i, c0, n);
            if constexpr (ADD) {
                const uint32_t v = __shfl_sync(0xFFFFFFFFu, key, b + j);
                if (ends >> (b + j) & 1 && b + j != head_end) old[j].load(a, v, c0, n);
            }
        }
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            if (!(real >> (b + j) & 1)) continue;
            float f[8];
            x[j].get(f);
            if (a.mask.threshold) {
                const uint64_t at = a.mask.first + (uint64_t)__shfl_sync(0xFFFFFFFFu, index, b + j) * (uint64_t)a.width + c0;
                Raw<2> words;
                philox(words.w, a.mask, (at + 8 * lane) >> 3, stream);
                if constexpr (!EIGHTS) words = with_next(words, (int)(at & 7));
                mask8(f, a.mask, words.w);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) sum[k] += f[k];
            if (!(ends >> (b + j) & 1)) continue;
            if (b + j == head_end) {
#pragma unroll
                for (int k = 0; k < 8; ++k) heads[warp][32 * k + lane] = sum[k];
            } else {
                put<OUT, EIGHTS, ADD>(a, __shfl_sync(0xFFFFFFFFu, key, b + j), c0, n, sum, old[ADD ? j : 0], tile);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) sum[k] = 0.0f;
        }
    }
    const bool open = left > 0 && (real & ~ends) >> (left - 1) & 1, through = open && head && head_end < 0;
    if (through)
#pragma unroll
        for (int k = 0; k < 8; ++k) heads[warp][32 * k + lane] = sum[k];
    if (lane == 0) goes_on[warp] = through;
    __syncthreads();
    // the run that begins in this piece and goes on; the one that began before this block
#pragma unroll 1
    for (int before = 0; before < 2; ++before) {
        if (before ? !(warp == 0 && head) : !open || through) continue;
        if (before)
#pragma unroll
            for (int k = 0; k < 8; ++k) sum[k] = 0.0f;
        bool on = true;                           // joined with the pieces that it goes on in
#pragma unroll 1
        for (int w = before ? 0 : warp + 1; on && w < kRowWarps; ++w) {
#pragma unroll
            for (int k = 0; k < 8; ++k) sum[k] += heads[w][32 * k + lane];
            on = goes_on[w];
        }
        const uint32_t v = __shfl_sync(0xFFFFFFFFu, key, before ? 0 : left - 1);
        if (before || on)
            hand_in<OUT, EIGHTS, ADD, PIECE>(a, v, chunk, before, column, n, sum, tile);
        else
            emit<OUT, EIGHTS, ADD>(a, v, c0, n, sum, tile);
    }
}

// A block for the run that begins in a chunk and goes on behind it, and 256 columns: two warps take
// neighbouring parts.  Most blocks find no such run: small ones are all resident at once (with eight warps each 131,072
// tokens x 2048 took 205 us).
template <int OUT, bool EIGHTS, bool ADD>
__global__ void __launch_bounds__(32 * kJoinWarps)
join_kernel(const __grid_constant__ SumArgs a)
{
    __shared__ __align__(16) float share[kJoinWarps][kTile];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const uint32_t chunk = blockIdx.x / a.columns, column = blockIdx.x % a.columns;
    const int64_t c0 = (int64_t)column * kCols<EIGHTS>;
    const int n = (int)min((int64_t)kCols<EIGHTS>, a.width - c0);
    chain();
    const uint32_t end = (chunk + 1) * kChunk;    // (the last chunk has no block)
    const uint32_t v = a.pairs[end].x;
    if (v == a.V || a.pairs[end - 1].x != v) return;
    const uint32_t begin = chunk * kChunk;
    if (begin > 0 && a.pairs[begin - 1].x == v) return;       // began before
    uint32_t parts = 2;                           // chunks that have the run: their first key says it
    for (uint32_t more = 32; more == 32; parts += more) {
        const uint64_t at = (uint64_t)(chunk + parts + lane) * kChunk;
        more = __ffs(~__ballot_sync(0xFFFFFFFFu, at < a.T && a.pairs[at].x == v));
        more = more ? more - 1 : 32;
    }
    const uint32_t each = (parts + kJoinWarps - 1) / kJoinWarps;
    float sum[8] = {};
    const uint32_t to = min((warp + 1) * each, parts);
    for (uint32_t i = warp * each; i < to; i += 4) {
        float f[4][8];
#pragma unroll
        for (int b = 0; b < 4; ++b)
            if (i + b < to) load_part(part_of(a, chunk + i + b, i + b == 0, column), f[b]);
#pragma unroll
        for (int b = 0; b < 4; ++b)
            if (i + b < to)
#pragma unroll
                for (int k = 0; k < 8; ++k) sum[k] += f[b][k];
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) share[warp][32 * k + lane] = sum[k];
    __syncthreads();
    if (warp != 0) return;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        sum[k] = 0.0f;
#pragma unroll
        for (int w = 0; w < kJoinWarps; ++w) sum[k] += share[w][32 * k + lane];
    }
    emit<OUT, EIGHTS, ADD>(a, v, c0, n, sum, share[0]);
}

template <int IN, int OUT, bool EIGHTS, bool ADD, int PIECE>
cudaError_t launch_sum(const SumArgs &a, cudaStream_t stream)
{
    const int64_t grid = (int64_t)a.blocks + ((int64_t)a.V - a.fill_from + a.fill_rows * kRowWarps - 1) / (a.fill_rows * kRowWarps);
    if (a.T > 0) return launch_chained(sum_kernel<IN, OUT, EIGHTS, ADD, PIECE>, grid, kRowThreads, 0, stream, a);
    sum_kernel<IN, OUT, EIGHTS, ADD, PIECE><<<(unsigned)grid, kRowThreads, 0, stream>>>(a);
    return cudaGetLastError();
}

template <int IN, int OUT, bool EIGHTS, bool ADD>
cudaError_t launch_sums(const SumArgs &a, cudaStream_t stream)
{
    if (a.fine) return launch_sum<IN, OUT, EIGHTS, ADD, kFewPiece>(a, stream);
    const cudaError_t e = launch_sum<IN, OUT, EIGHTS, ADD, kPiece>(a, stream);
    if (e != cudaSuccess || a.chunks <= 1) return e;
    return launch_chained(join_kernel<OUT, EIGHTS, ADD>, (int64_t)(a.chunks - 1) * a.columns, 32 * kJoinWarps, 0, stream, a);
}

template <int IN, int OUT>
cudaError_t launch_types(const SumArgs &a, bool eights, bool add, cudaStream_t stream)
{
    if (eights) return add ? launch_sums<IN, OUT, true, true>(a, stream) : launch_sums<IN, OUT, true, false>(a, stream);
    return add ? launch_sums<IN, OUT, false, true>(a, stream) : launch_sums<IN, OUT, false, false>(a, stream);
}

template <bool FILL, bool CLUSTER>
cudaError_t launch_few(const FewArgs &a, unsigned grid, cudaStream_t stream)
{
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = 8, at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(kSortThreads);
    cfg.stream = stream;
    cfg.attrs = at;
    cfg.numAttrs = CLUSTER ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, few_kernel<FILL, CLUSTER>, a);
}

}  // namespace

extern "C" size_t aspis_embed_workspace_bytes(int64_t T, int64_t V, int64_t width)
{
    Plan p;
    return make_plan(T, V, width, p) ? p.bytes : 0;
}

extern "C" aspis_status aspis_embed_grad(const void *grad, int grad_type, int64_t ld_grad, const void *tokens,
                                         int token_type, int64_t T, int64_t V, int64_t width, float scale,
                                         const aspis_drop *drop, int accumulate, void *table_grad, int table_type,
                                         int64_t ld_table, void *work, size_t work_bytes, void *stream)
{
    if (T < 0 || V < 1 || width < 0 || (token_type != ASPIS_I32 && token_type != ASPIS_I64) || !isfinite(scale) ||
        (accumulate != 0 && accumulate != 1))
        return ASPIS_E_INVAL;
    Rows in{grad, T, width, ld_grad, grad_type}, out{table_grad, V, width, ld_table, table_type};
    SumArgs a{};
    Plan p;
    aspis_status s = make_mask(drop, a.mask);
    if (s == ASPIS_OK) s = make_factor(scale, a.mask, a.factor);
    if (s == ASPIS_OK) s = in.check();
    if (s == ASPIS_OK) s = out.check();
    if (s != ASPIS_OK) return s;
    if (!make_plan(T, V, width, p)) return ASPIS_E_RANGE;
    if (width == 0) return ASPIS_OK;
    const int token_bytes = token_type == ASPIS_I64 ? 8 : 4;
    if (T > 0) {
        if (!tokens || !work || step_in(a.mask, out)) return ASPIS_E_INVAL;
        if ((uintptr_t)tokens % token_bytes || (uintptr_t)work % 16) return ASPIS_E_ALIGN;
        if (work_bytes < p.bytes) return ASPIS_E_RANGE;
        if (rows_meet(in, out) || ranges_meet(tokens, T * token_bytes, table_grad, out.bytes()) ||
            ranges_meet(work, (int64_t)p.bytes, table_grad, out.bytes()) || ranges_meet(work, (int64_t)p.bytes, grad, in.bytes()) ||
            ranges_meet(work, (int64_t)p.bytes, tokens, T * token_bytes) ||
            (a.mask.threshold && ranges_meet(work, (int64_t)p.bytes, a.mask.step, 8)))
            return ASPIS_E_INVAL;
    } else if (accumulate) {
        return ASPIS_OK;
    }
    const cudaStream_t st = (cudaStream_t)stream;
    char *w = static_cast<char *>(work);
    uint2 *const pairs[2] = {(uint2 *)(w + p.pairs[0]), (uint2 *)(w + p.pairs[1])};
    uint32_t *const tables = (uint32_t *)(w + p.tables);
    const uint32_t step = p.tiles * kDigits;
    uint32_t filled = 0;                          // rows that the sort's launch writes zeros to
    const int64_t columns = p.columns;
    if (columns > INT32_MAX / (p.chunks + 1)) return ASPIS_E_RANGE;
    a.arrived = (uint32_t *)(w + p.arrived);
    // rows that a warp writes zeros to at a time: some 12 KB of them, a power of two up to 32, and work for 16 warps a multiprocessor
    uint32_t group = 1;
    while (group < 32 && 2 * group * width * type_bytes(table_type) <= 12288 && (int64_t)group * 2 * 16 * kSMs <= V) group *= 2;
    if (T > 0 && p.few) {
        FewArgs o{};
        o.tokens = tokens;
        o.pairs = pairs[0];
        o.arrived = a.arrived, o.arrived_size = p.fine ? p.chunks * columns : 0;
        o.T = (uint32_t)T, o.V = (uint32_t)V;
        o.wide_tokens = token_type == ASPIS_I64;
        o.bits = p.bits, o.passes = p.passes;
        const bool one = T <= kOneTokens;
        for (o.tile_bits = one ? 10 : 8; (one ? 1 : 8) << o.tile_bits < T;) ++o.tile_bits;
        if (!accumulate) {
            o.out = static_cast<char *>(table_grad);
            o.row_bytes = width * type_bytes(table_type), o.ld_bytes = ld_table * type_bytes(table_type);
            int64_t fit = kFillBytes / o.row_bytes + kSortWarps;
            if (fit > (int64_t)kFillBlocks * kFillRows) fit = (int64_t)kFillBlocks * kFillRows;
            filled = (uint32_t)(fit < V ? fit : V);
            const uint32_t rows = (filled + kFillBlocks - 1) / kFillBlocks;
            o.rows = rows < kSortWarps * group ? kSortWarps * group : rows;
            o.fill = filled;
            o.group = group;
        }
        const unsigned blocks = accumulate ? 0 : (filled + o.rows - 1) / o.rows;
        const cudaError_t e = one ? (accumulate ? launch_few<false, false>(o, 1, st) : launch_few<true, false>(o, 1 + blocks, st))
                                  : (accumulate ? launch_few<false, true>(o, 8, st)
                                                : launch_few<true, true>(o, 8 + (blocks + 7) / 8 * 8, st));
        if (e != cudaSuccess) return status_of(e);
        a.pairs = pairs[0];
    } else if (T > 0) {
        SortArgs o{};
        o.tokens = tokens;
        o.T = (uint32_t)T, o.V = (uint32_t)V, o.tiles = p.tiles, o.tile = p.tile;
        o.wide_tokens = token_type == ASPIS_I64;
        o.bits = p.bits;
        o.table = tables, o.next = tables + step;
        o.clear = (uint32_t)(p.passes - 1) * step;
        o.arrived = a.arrived, o.arrived_size = p.fine ? p.chunks * columns : 0;
        count_kernel<<<p.tiles, kSortThreads, 0, st>>>(o);
        if (cudaGetLastError() != cudaSuccess) return ASPIS_E_CUDA;
        for (int i = 0; i < p.passes; ++i) {
            o.tokens = i == 0 ? tokens : nullptr;
            o.pairs = pairs[(i + 1) % 2], o.out = pairs[i % 2];
            o.table = tables + i * step;
            o.next = i + 1 < p.passes ? o.table + step : nullptr;
            o.shift = i * p.bits;
            const cudaError_t e = launch_chained(scatter_kernel, p.tiles, kSortThreads, 0, st, o);
            if (e != cudaSuccess) return status_of(e);
        }
        a.pairs = o.out;
    }
    a.grad = grad, a.out = table_grad;
    a.parts = (float *)(w + p.parts);
    a.ld = ld_grad, a.ldo = ld_table, a.width = width;
    a.T = (uint32_t)T, a.V = (uint32_t)V, a.chunks = p.chunks, a.fine = p.fine;
    const bool eights = width % 8 == 0 && in.by_eights() && out.by_eights() && (!a.mask.threshold || a.mask.first % 8 == 0);
    a.columns = (uint32_t)(eights ? (width + kCols<true> - 1) / kCols<true> : columns);
    a.blocks = p.chunks * a.columns;
    a.fill_from = accumulate ? a.V : filled;
    a.fill_rows = group;
    cudaError_t e;
    switch (grad_type * 3 + table_type) {
        case 0: e = launch_types<0, 0>(a, eights, accumulate, st); break;
        case 1: e = launch_types<0, 1>(a, eights, accumulate, st); break;
        case 2: e = launch_types<0, 2>(a, eights, accumulate, st); break;
        case 3: e = launch_types<1, 0>(a, eights, accumulate, st); break;
        case 4: e = launch_types<1, 1>(a, eights, accumulate, st); break;
        case 5: e = launch_types<1, 2>(a, eights, accumulate, st); break;
        case 6: e = launch_types<2, 0>(a, eights, accumulate, st); break;
        case 7: e = launch_types<2, 1>(a, eights, accumulate, st); break;
        default: e = launch_types<2, 2>(a, eights, accumulate, st); break;
    }
    return status_of(e);
}
