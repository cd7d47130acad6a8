"""Reads of a gapless matrix in octets and their 16-byte pieces stay inside it, and
leave out no value, at widths and row counts where rows end inside an octet: the
rules of clip.cuh, compiled for the host, as the join's copies (the last of a
thread's rows, which are a multiple of eight apart, is clipped) and the balance
loss's loads (whole octets of rows that are followed) use them."""

import subprocess

from paper_1601_04033_gb300 import build

SRC = r"""
#include <cstdio>
#include "clip.cuh"
using namespace fasgd;
int main() {
    int bad = 0;
    for (int64_t cols = 1; cols <= 23; ++cols)
        for (int64_t rows = 1; rows <= 70; ++rows)
            for (int per = 4; per <= 8; per += 4)                 // of fp32, of 16-bit types
                for (int64_t step = 8; step <= 72; step += 8)
                    for (int64_t r = 0; r < rows; ++r) {
                        // The copies: a thread's last row is clipped, the others are not.
                        const bool last = r + step >= rows;
                        const int32_t behind = last ? values_behind(rows, cols, r) : -1;
                        const int shift = (int)(r * cols % 8);
                        for (int32_t col = -shift; col < cols; col += per) {
                            if (col + per <= 0) continue;
                            const int n = values_there(col, (int32_t)cols, behind, per);
                            const int64_t from = r * cols + col, to = from + n;
                            const bool all = col + n >= cols || n == per;
                            if (from < 0 || n < 1 || n > per || to > rows * cols || !all) {
                                if (bad++ < 10)
                                    std::printf("copy: %lld x %lld, row %lld: %lld .. %lld\n", (long long)rows,
                                                (long long)cols, (long long)r, (long long)from, (long long)to);
                            }
                        }
                        // The loads: whole octets.
                        if (step > 8 || per > 4) continue;
                        for (int32_t c0 = -shift; c0 < cols; c0 += 8)
                            if ((c0 + 8 <= cols || r < rows_followed(rows, cols)) && r * cols + c0 + 8 > rows * cols)
                                if (bad++ < 10)
                                    std::printf("load: %lld x %lld, row %lld\n", (long long)rows, (long long)cols, (long long)r);
                    }
    return bad != 0;
}
"""


def test_reads_end_with_the_matrix(tmp_path):
    src, exe = tmp_path / "clip.cu", tmp_path / "clip"
    src.write_text(SRC)
    r = subprocess.run([build.nvcc(), *build.ARCH, "-std=c++17", "-O1", f"-I{build.CSRC}", str(src), "-o", str(exe)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout
