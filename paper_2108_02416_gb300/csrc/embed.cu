// aspis_dropout and aspis_embed: rows of one matrix, or of a table by their tokens, scaled and masked into another.
//
// Each element is read and written once, which HBM bounds where the mask does not: Philox's ten rounds take 76 cycles of a
// scheduler for a warp's 256 elements, whichever way its 32 by 32 bit products are written, and the selection about as
// much.  A lane has eight neighbouring elements that begin at a multiple of their size in the output.
// Where the input's groups and the mask's blocks begin there too (EIGHTS), that is one load, one block of random bits and
// one store.  Else it takes what its neighbour loaded and drew as well: groups and blocks overlap those of
// the output by the same number of elements in the whole row.
// 16,384 x 4096 bf16 with a residual 64.4 us (6.2 TB/s).  16,384 tokens x 2048 fp32 to bf16 take 26.9 with a mask and 24.5 without one
// (4.6 and 5.0 TB/s of what they cannot do without), 20,001 unaligned rows of 1001 fp16 to fp32 28.7 (4.2 TB/s): neither HBM (35 and
// 28 % of its time) nor the issue slots (64 %) are full there, as a warp loads first and computes then, and a multiprocessor's
// warps overlap the two in part.
#include <limits.h>

#include "worker.cuh"

using namespace aspis;

namespace {

constexpr int kDrop = 0, kResidual = 1, kEmbed = 2;
constexpr int kNarrow = 512;                      // columns of cells_kernel's rows

struct RowsArgs {
    const void *x, *residual;
    void *out;
    const void *tokens;
    int64_t ldx, ldr, ldo, rows, cols, V;
    uint32_t units, chunks, pieces;               // warps' shares of the call; of a row; pieces of a share
    float factor;
    int32_t wide_tokens;
    Mask mask;
};

// 256 elements of a row (248 where neighbours overlap), at most as many times as 32 registers hold
template <int IN, int OUT, int KIND>
constexpr int kPieces = 32 / (2 * kBytes<IN> + (KIND == kResidual ? 2 * kBytes<OUT> : 0));

template <int IN, int OUT, int KIND, bool EIGHTS>
__global__ void __launch_bounds__(kRowThreads, 3)
rows_kernel(const __grid_constant__ RowsArgs a)
{
    constexpr int P = EIGHTS && kPieces<IN, OUT, KIND> > 4 ? 4 : kPieces<IN, OUT, KIND>, kWidth = EIGHTS ? 256 : 248, BI = kBytes<IN>, BO = kBytes<OUT>;
    const uint32_t u = blockIdx.x * kRowWarps + threadIdx.x / 32;
    if (u >= a.units) return;
    const int lane = threadIdx.x % 32;
    const int64_t row = u / a.chunks;
    const int64_t from = KIND == kEmbed ? load_token(a.tokens, a.wide_tokens, row, a.V) : row;
    const char *x = static_cast<const char *>(a.x) + from * a.ldx * BI;
    const char *res = static_cast<const char *>(a.residual) + row * a.ldr * BO;
    char *out = static_cast<char *>(a.out) + row * a.ldo * BO;
    const uint64_t number = a.mask.first + (uint64_t)row * (uint64_t)a.cols, stream = mask_stream(a.mask);
    int64_t c0 = (int64_t)(u % a.chunks) * (a.pieces * kWidth) + 8 * lane;

    if constexpr (EIGHTS) {
        Raw<BI> v[P];
        Raw<KIND == kResidual ? BO : BI> w[KIND == kResidual ? P : 1];
        const uint64_t block = (number + c0) >> 3;
        const bool real = KIND != kEmbed || from >= 0, masked = a.mask.threshold != 0;
        // groups of the row from this lane's first on; the last one may be short where the row is the only one
        const int n = (int)min((a.cols - c0 + 7) >> 3, (int64_t)32 * a.pieces), full = (int)min((a.cols - c0) >> 3, (int64_t)32 * a.pieces);
        x += c0 * BI, res += c0 * BO, out += c0 * BO;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            if (32 * i >= full) break;
            if (real) v[i] = load_group<IN, KIND == kEmbed>(x + i * kWidth * BI);
            if constexpr (KIND == kResidual) w[i] = load_group<OUT, false>(res + i * kWidth * BO);
        }
        auto finish = [&](int i, float (&f)[8], const float (&g)[8]) {
            if (!real)
#pragma unroll
                for (int k = 0; k < 8; ++k) f[k] = 0.0f;
            else if (masked) {
                uint32_t words[4];
                philox(words, a.mask, (block + 32 * i) & (~UINT64_C(0) >> 3), stream);
                mask8(f, a.mask, words, a.factor);
            } else
#pragma unroll
                for (int k = 0; k < 8; ++k) f[k] *= a.factor;
            if constexpr (KIND == kResidual)
#pragma unroll
                for (int k = 0; k < 8; ++k) f[k] += g[k];
        };
#pragma unroll
        for (int i = 0; i < P; ++i) {
            if (32 * i >= full) break;
            float f[8], g[8];
            to_floats(v[i], IN == ASPIS_BF16, f);
            if constexpr (KIND == kResidual) to_floats(w[i], OUT == ASPIS_BF16, g);
            finish(i, f, g);
            store_floats<BO>(out + i * kWidth * BO, f, OUT == ASPIS_BF16);
        }
        if (full >= 0 && full < n && full % 32 == 0) {         // this lane's next group is the short one
            const int i = full / 32, cols = (int)((a.cols - c0) & 7);
            float f[8], g[8];
            load_edge<IN>(f, x + i * kWidth * BI, 0, 0, cols);
            if constexpr (KIND == kResidual) load_edge<OUT>(g, res + i * kWidth * BO, 0, 0, cols);
            finish(i, f, g);
            store_edge<OUT>(out + i * kWidth * BO, 0, 0, cols, f);
        }
    } else {
        c0 -= behind<BO>(out);                    // a multiple of eight elements in memory
        const int64_t first = c0 - 8 * lane;      // the share's; columns are counted from it
        const Columns columns = columns_from(first, a.cols, 1 << 20);
        const int lo = columns.lo, hi = columns.hi;
        const uint64_t block = (number + c0) >> 3;
        const int pieces = min((int)a.pieces, (hi + kWidth - 1) / kWidth);
        const int sx = behind<BI>(x + c0 * BI), sr = KIND == kResidual ? behind<BO>(res + c0 * BO) : 0, off = (int)((number + c0) & 7);
        // (rows that are closer than a group: the second is as near to the matrix's begin as the first)
        const bool res_end = row == 0 || row + 1 == a.rows || a.ldr < 8;
        const bool x_end = KIND == kEmbed ? from <= 0 || from + 1 >= a.V || a.ldx < 8 : row == 0 || row + 1 == a.rows || a.ldx < 8;
        x += first * BI, res += first * BO, out += first * BO;
        Raw<BI> v[P];
        Raw<KIND == kResidual ? BO : BI> w[KIND == kResidual ? P : 1];
#pragma unroll
        for (int i = 0; i < P; ++i) {
            if (i >= pieces) break;
            const int c = 8 * lane + i * kWidth;
            v[i] = {};
            if (KIND != kEmbed || from >= 0) v[i] = load_around<IN, KIND == kEmbed>(x, c, sx, columns, x_end);
            if constexpr (KIND == kResidual) w[i] = load_around<OUT, false>(res, c, sr, columns, res_end);
        }
#pragma unroll
        for (int i = 0; i < P; ++i) {
            if (i >= pieces) break;
            const int c = 8 * lane + i * kWidth;
            float f[8] = {};
            if (KIND != kEmbed || from >= 0) {
                to_floats(with_next(v[i], sx), IN == ASPIS_BF16, f);
                if (a.mask.threshold) {
                    Raw<2> words;
                    philox(words.w, a.mask, (block + (kWidth / 8) * i) & (~UINT64_C(0) >> 3), stream);
                    mask8(f, a.mask, with_next(words, off).w, a.factor);
                } else
#pragma unroll
                    for (int k = 0; k < 8; ++k) f[k] *= a.factor;
            }
            if constexpr (KIND == kResidual) {
                float g[8];
                to_floats(with_next(w[i], sr), OUT == ASPIS_BF16, g);
#pragma unroll
                for (int k = 0; k < 8; ++k) f[k] += g[k];
            }
            if (lane == 31) continue;             // only its neighbour's helper
            if (c >= lo && c + 8 <= hi)
                store_floats<BO>(out + c * BO, f, OUT == ASPIS_BF16);
            else
                store_edge<OUT>(out, c, lo, hi, f);
        }
    }
}

// Narrow rows: a thread has eight neighbouring elements of a row, of which `cells` are enough for one at any offset.  Where
// groups or blocks overlap the output's it loads and draws both itself: with a warp for each row of 16 to 200 columns most lanes
// had nothing to do.  Dropout of 40,000 bf16 rows in wider ones (inputs in turn), 16 columns 3.0 us (11.2 with a warp a row), 33: 4.8 (19.3),
// 255: 17.3 (28.7), 256: 10.8 (13.2), 512: 17.7 (19.1), 1001: 51.2 (51.9); with the lookup 512: 19.1 either way.
template <int IN, int OUT, int KIND, bool EIGHTS>
__global__ void __launch_bounds__(kRowThreads)
cells_kernel(const __grid_constant__ RowsArgs a)
{
    constexpr int BI = kBytes<IN>, BO = kBytes<OUT>, P = EIGHTS ? 4 : 2;
    const uint32_t all = (uint32_t)a.rows * a.chunks;             // (a.chunks: cells of a row)
    const uint64_t stream = mask_stream(a.mask);
    const int cols = (int)a.cols;
    const Columns columns = {0, cols};
    uint32_t row[P];
    int64_t from[P];
    int c[P];
#pragma unroll
    for (int i = 0; i < P; ++i) {
        const uint32_t q = (blockIdx.x * P + i) * kRowThreads + threadIdx.x;
        row[i] = q / a.chunks;
        c[i] = q < all ? (int)(q - row[i] * a.chunks) * 8 : cols;
        from[i] = KIND == kEmbed ? q < all ? load_token(a.tokens, a.wide_tokens, row[i], a.V) : -1 : row[i];
        if (!EIGHTS && q < all) c[i] -= behind<BO>(static_cast<char *>(a.out) + row[i] * a.ldo * BO);
    }
    Raw<BI> v[P][EIGHTS ? 1 : 2];
    Raw<KIND == kResidual ? BO : BI> w[KIND == kResidual ? P : 1][EIGHTS ? 1 : 2];
#pragma unroll
    for (int i = 0; i < P; ++i) {
        if (c[i] >= cols) continue;
        const char *x = static_cast<const char *>(a.x) + from[i] * a.ldx * BI;
        const char *res = static_cast<const char *>(a.residual) + row[i] * a.ldr * BO;
        const bool real = KIND != kEmbed || from[i] >= 0;
        if constexpr (EIGHTS) {
            if (real) v[i][0] = load_group<IN, KIND == kEmbed>(x + c[i] * BI);
            if constexpr (KIND == kResidual) w[i][0] = load_group<OUT, false>(res + c[i] * BO);
        } else {
            const bool end = row[i] == 0 || row[i] + 1 == a.rows;
            const int sx = behind<BI>(x + c[i] * BI);
            v[i][0] = v[i][1] = {};
            if (real) {
                const bool x_end = a.ldx < 8 || (KIND == kEmbed ? from[i] <= 0 || from[i] + 1 >= a.V : end);
                v[i][0] = load_around<IN, KIND == kEmbed>(x, c[i], sx, columns, x_end);
                if (sx) v[i][1] = load_around<IN, KIND == kEmbed>(x, c[i] + 8, sx, columns, x_end);
            }
            if constexpr (KIND == kResidual) {
                const int sr = behind<BO>(res + c[i] * BO);
                w[i][0] = load_around<OUT, false>(res, c[i], sr, columns, end || a.ldr < 8);
                if (sr) w[i][1] = load_around<OUT, false>(res, c[i] + 8, sr, columns, end || a.ldr < 8);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < P; ++i) {
        if (c[i] >= cols) continue;
        const char *x = static_cast<const char *>(a.x) + from[i] * a.ldx * BI;
        const char *res = static_cast<const char *>(a.residual) + row[i] * a.ldr * BO;
        char *out = static_cast<char *>(a.out) + row[i] * a.ldo * BO;
        float f[8] = {};
        if (KIND != kEmbed || from[i] >= 0) {
            if constexpr (EIGHTS) {
                to_floats(v[i][0], IN == ASPIS_BF16, f);
            } else {
                const int sx = behind<BI>(x + c[i] * BI);
                to_floats(sx ? shifted(v[i][0], v[i][1], sx) : v[i][0], IN == ASPIS_BF16, f);
            }
            if (a.mask.threshold) {
                const uint64_t at = a.mask.first + (uint64_t)row[i] * (uint64_t)a.cols + (int64_t)c[i];
                Raw<2> words;
                philox(words.w, a.mask, at >> 3, stream);
                if (!EIGHTS && at & 7) {
                    Raw<2> next;
                    philox(next.w, a.mask, (at + 8) >> 3, stream);
                    words = shifted(words, next, (int)(at & 7));
                }
                mask8(f, a.mask, words.w, a.factor);
            } else
#pragma unroll
                for (int k = 0; k < 8; ++k) f[k] *= a.factor;
        }
        if constexpr (KIND == kResidual) {
            float g[8];
            if constexpr (EIGHTS) {
                to_floats(w[i][0], OUT == ASPIS_BF16, g);
            } else {
                const int sr = behind<BO>(res + c[i] * BO);
                to_floats(sr ? shifted(w[i][0], w[i][1], sr) : w[i][0], OUT == ASPIS_BF16, g);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) f[k] += g[k];
        }
        if (EIGHTS || (c[i] >= 0 && c[i] + 8 <= cols))
            store_floats<BO>(out + c[i] * BO, f, OUT == ASPIS_BF16);
        else
            store_edge<OUT>(out, c[i], 0, cols, f);
    }
}

template <int IN, int OUT, int KIND>
cudaError_t launch_kind(RowsArgs &a, int64_t rows, bool eights, cudaStream_t stream)
{
    const int64_t width = eights ? 256 : 248, pieces = (a.cols + (eights ? 0 : 7) + width - 1) / width;
    const int64_t most = eights && kPieces<IN, OUT, KIND> > 4 ? 4 : kPieces<IN, OUT, KIND>;
    const int64_t chunks = (pieces + most - 1) / most;
    a.chunks = (uint32_t)chunks;
    a.pieces = (uint32_t)((pieces + chunks - 1) / chunks);
    a.units = (uint32_t)(rows * chunks);
    const int64_t cells = eights ? a.cols / 8 : (a.cols + 14) / 8;
    if (rows > 1 && a.cols < kNarrow && (!eights || a.cols % 8 == 0) && rows * cells <= INT32_MAX) {
        constexpr int kEach = kRowThreads * 4;
        a.chunks = (uint32_t)cells;
        if (eights)
            cells_kernel<IN, OUT, KIND, true><<<(unsigned)((rows * cells + kEach - 1) / kEach), kRowThreads, 0, stream>>>(a);
        else
            cells_kernel<IN, OUT, KIND, false><<<(unsigned)((rows * cells + kEach / 2 - 1) / (kEach / 2)), kRowThreads, 0, stream>>>(a);
        return cudaGetLastError();
    }
    const unsigned grid = (a.units + kRowWarps - 1) / kRowWarps;
    if (eights)
        rows_kernel<IN, OUT, KIND, true><<<grid, kRowThreads, 0, stream>>>(a);
    else
        rows_kernel<IN, OUT, KIND, false><<<grid, kRowThreads, 0, stream>>>(a);
    return cudaGetLastError();
}

template <int IN, int OUT>
cudaError_t launch_types(RowsArgs &a, int64_t rows, bool eights, cudaStream_t stream)
{
    if (a.tokens) return launch_kind<IN, OUT, kEmbed>(a, rows, eights, stream);
    return a.residual ? launch_kind<IN, OUT, kResidual>(a, rows, eights, stream) : launch_kind<IN, OUT, kDrop>(a, rows, eights, stream);
}

aspis_status launch_rows(RowsArgs &a, const Rows &in, const Rows &res, const Rows &out, cudaStream_t stream)
{
    const bool eights = in.by_eights() && out.by_eights() && (!res.p || res.by_eights()) &&
                        (!a.mask.threshold || (a.mask.first % 8 == 0 && (out.cols % 8 == 0 || out.rows == 1)));
    a.x = in.p, a.residual = res.p, a.out = const_cast<void *>(out.p);
    a.ldx = in.ld, a.ldr = res.ld, a.ldo = out.ld, a.rows = out.rows, a.cols = out.cols;
    const int64_t chunks = (out.cols + 7 + 247) / 248;            // at most
    if (chunks > (INT64_C(1) << 31) / out.rows) return ASPIS_E_RANGE;
    cudaError_t e;
    switch (in.type * 3 + out.type) {
        case 0: e = launch_types<0, 0>(a, out.rows, eights, stream); break;
        case 1: e = launch_types<0, 1>(a, out.rows, eights, stream); break;
        case 2: e = launch_types<0, 2>(a, out.rows, eights, stream); break;
        case 3: e = launch_types<1, 0>(a, out.rows, eights, stream); break;
        case 4: e = launch_types<1, 1>(a, out.rows, eights, stream); break;
        case 5: e = launch_types<1, 2>(a, out.rows, eights, stream); break;
        case 6: e = launch_types<2, 0>(a, out.rows, eights, stream); break;
        case 7: e = launch_types<2, 1>(a, out.rows, eights, stream); break;
        default: e = launch_types<2, 2>(a, out.rows, eights, stream); break;
    }
    return status_of(e);
}

}  // namespace

extern "C" aspis_status aspis_dropout(const void *x, int x_type, int64_t ldx, const void *residual, int64_t ldr,
                                      void *out, int out_type, int64_t ldo, int64_t rows, int64_t cols,
                                      const aspis_drop *drop, void *stream)
{
    if (rows < 0 || cols < 0 || !drop) return ASPIS_E_INVAL;
    Rows in{x, rows, cols, ldx, x_type}, to{out, rows, cols, ldo, out_type};
    Rows res{residual, rows, cols, residual ? ldr : cols, out_type};
    RowsArgs a{};
    aspis_status s = make_mask(drop, a.mask);
    if (s == ASPIS_OK) s = in.check();
    if (s == ASPIS_OK) s = to.check();
    if (s == ASPIS_OK && residual) s = res.check();
    if (s != ASPIS_OK) return s;
    if (rows == 0 || cols == 0) return ASPIS_OK;
    if (step_in(a.mask, to)) return ASPIS_E_INVAL;
    if (rows_meet(in, to) && !same_rows(in, to)) return ASPIS_E_INVAL;
    if (residual && rows_meet(res, to) && !same_rows(res, to)) return ASPIS_E_INVAL;
    // rows without gaps are one row: their elements' numbers go on from row to row
    if ((ldx == cols && ldo == cols && (!residual || ldr == cols)) || rows == 1) {
        in.cols = to.cols = res.cols = in.ld = to.ld = res.ld = rows * cols;
        in.rows = to.rows = res.rows = 1;
    }
    a.factor = a.mask.up;
    return launch_rows(a, in, res, to, (cudaStream_t)stream);
}

extern "C" aspis_status aspis_embed(const void *table, int table_type, int64_t ld_table, int64_t V, const void *tokens,
                                    int token_type, int64_t T, int64_t width, float scale, const aspis_drop *drop,
                                    void *out, int out_type, int64_t ld_out, void *stream)
{
    if (T < 0 || V < 1 || width < 0 || (token_type != ASPIS_I32 && token_type != ASPIS_I64) || !(fabsf(scale) <= 3.4028235e38f))
        return ASPIS_E_INVAL;
    Rows in{table, V, width, ld_table, table_type}, to{out, T, width, ld_out, out_type}, none{};
    RowsArgs a{};
    aspis_status s = make_mask(drop, a.mask);
    if (s == ASPIS_OK) s = make_factor(scale, a.mask, a.factor);
    if (s == ASPIS_OK) s = in.check();
    if (s == ASPIS_OK) s = to.check();
    if (s != ASPIS_OK) return s;
    if (T == 0 || width == 0) return ASPIS_OK;
    if (step_in(a.mask, to)) return ASPIS_E_INVAL;
    const int token_bytes = token_type == ASPIS_I64 ? 8 : 4;
    if (!tokens) return ASPIS_E_INVAL;
    if ((uintptr_t)tokens % token_bytes) return ASPIS_E_ALIGN;
    if (rows_meet(in, to) || ranges_meet(tokens, T * token_bytes, out, to.bytes())) return ASPIS_E_INVAL;
    a.tokens = tokens, a.V = V;
    a.wide_tokens = token_type == ASPIS_I64;
    return launch_rows(a, in, none, to, (cudaStream_t)stream);
}
