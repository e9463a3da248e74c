"""csrc/columns.h on the CPU: what the lanes of dropout, the embedding and its gradient load stays inside their matrix, and holds
all that they need."""
import os
import shutil
import subprocess

import pytest

from conftest import ROOT

PROGRAM = r"""
#include <algorithm>
#include <cstdio>
#include <vector>
#include "columns.h"

using namespace aspis;
using std::max;
using std::min;

// A lane's load at columns c .. c + 7 of the row, counted from `first`: every element of the matrix that it touches.  Rows lie
// `ld` apart; the matrix has elements 0 .. size - 1.
static bool touch(std::vector<char> &seen, int64_t row_at, int64_t first, int c, Columns columns, bool end, int64_t size)
{
    if (load_nothing(c, columns)) return true;
    const bool whole = load_whole(c, columns, end);
    for (int k = 0; k < 8; ++k) {
        if (!whole && (c + k < columns.lo || c + k >= columns.hi)) continue;
        const int64_t at = row_at + first + c + k;
        if (at < 0 || at >= size) return false;
        seen[at] = 1;
    }
    return true;
}

static bool row_seen(const std::vector<char> &seen, int64_t row_at, int64_t cols)
{
    for (int64_t j = 0; j < cols; ++j)
        if (!seen[row_at + j]) return false;
    return true;
}

int main()
{
    const int64_t widths[] = {1, 7, 8, 9, 240, 241, 247, 248, 249, 255, 256, 257, 496, 503, 511, 512, 600, 745, 2049};
    const int kWidth = 248;
    for (int64_t cols : widths)
        for (int rows = 1; rows <= 3; ++rows)
            for (int pad = 0; pad <= 9; pad += 3)
                for (int x_place = 0; x_place < 8; ++x_place)            // the matrices' places behind a group's boundary
                    for (int out_place = 0; out_place < 8; ++out_place)
                        for (int pieces = 1; pieces <= 4; ++pieces) {
                            const int64_t ld = cols + pad, ldo = cols, size = (rows - 1) * ld + cols;
                            for (int row = 0; row < rows; ++row) {
                                const int64_t row_at = row * ld;
                                const bool end = row == 0 || row + 1 == rows || ld < 8;
                                const int behind_out = (int)((out_place + row * ldo) % 8);
                                std::vector<char> seen(size, 0);
                                // rows of one warp a share, as in rows_kernel: a group of the output each lane, the input's around it
                                const int64_t all = (cols + 7 + kWidth - 1) / kWidth, chunks = (all + pieces - 1) / pieces;
                                for (int64_t chunk = 0; chunk < chunks; ++chunk) {
                                    const int64_t first = chunk * pieces * kWidth - behind_out;
                                    const Columns columns = columns_from(first, cols, 1 << 20);
                                    const int shift = (int)(((x_place + row_at + first) % 8 + 8) % 8);
                                    for (int i = 0; i < min(pieces, (columns.hi + kWidth - 1) / kWidth); ++i)
                                        for (int lane = 0; lane < 32; ++lane)
                                            if (!touch(seen, row_at, first, 8 * lane + i * kWidth - shift, columns, end, size))
                                                return printf("rows: %ld columns, row %d of %d, pad %d, places %d %d\n", (long)cols, row, rows, pad, x_place, out_place), 1;
                                }
                                if (!row_seen(seen, row_at, cols)) return printf("rows: %ld columns not all loaded\n", (long)cols), 1;
                                // blocks of columns, as in sum_kernel
                                std::fill(seen.begin(), seen.end(), 0);
                                for (int64_t c0 = 0; c0 < cols; c0 += kWidth) {
                                    const Columns columns = columns_from(c0, cols, 512);
                                    const int shift = (int)((x_place + row_at + c0) % 8);
                                    for (int lane = 0; lane < 32; ++lane)
                                        if (!touch(seen, row_at, c0, 8 * lane - shift, columns, end, size))
                                            return printf("blocks: %ld columns, row %d of %d, pad %d, place %d\n", (long)cols, row, rows, pad, x_place), 1;
                                }
                                if (!row_seen(seen, row_at, cols)) return printf("blocks: %ld columns not all loaded\n", (long)cols), 1;
                                // two groups a thread, as in cells_kernel
                                std::fill(seen.begin(), seen.end(), 0);
                                const Columns whole = columns_from(0, cols, 1 << 20);
                                for (int cell = 0; cell < (cols + 14) / 8; ++cell) {
                                    const int c = 8 * cell - behind_out, shift = (int)(((x_place + row_at + c) % 8 + 8) % 8);
                                    if (c >= cols) continue;
                                    if (!touch(seen, row_at, 0, c - shift, whole, end, size) ||
                                        (shift && !touch(seen, row_at, 0, c + 8 - shift, whole, end, size)))
                                        return printf("cells: %ld columns, row %d of %d, pad %d, places %d %d\n", (long)cols, row, rows, pad, x_place, out_place), 1;
                                }
                                if (!row_seen(seen, row_at, cols)) return printf("cells: %ld columns not all loaded\n", (long)cols), 1;
                            }
                        }
    return 0;
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="no C++ compiler")
def test_loads_stay_inside_the_matrix(tmp_path):
    source, program = tmp_path / "columns.cpp", tmp_path / "columns"
    source.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O2", "-I", os.path.join(ROOT, "paper_2108_02416_gb300", "csrc"), str(source), "-o", str(program)],
                   check=True)
    p = subprocess.run([str(program)], capture_output=True, text=True, timeout=300)
    assert p.returncode == 0, p.stdout
