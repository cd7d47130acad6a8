// Which of a row's octets may be read whole: they are cut at multiples of eight
// values of a gapless matrix of any width (octet.cuh), so a row's last octet takes
// up to kBehind values that lie behind the row, and the matrix may end among them --
// with the row itself or, where rows are short, a few rows later.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

namespace fasgd {

constexpr int kBehind = 7;

// The matrix's values behind row r, or -1 where there are kBehind of them or more.
// Of rows eight or more apart only the last can have fewer.
__host__ __device__ __forceinline__ int32_t values_behind(int64_t rows, int64_t cols, int64_t r) {
    const int64_t n = (rows - 1 - r) * cols;
    return n < kBehind ? (int32_t)n : -1;
}
// Of `per` values from column `col` (one of the row's, or before them) on, those that
// may be read, behind the row what `behind` (values_behind) says.
__host__ __device__ __forceinline__ int32_t values_there(int32_t col, int32_t cols, int32_t behind, int32_t per) {
    const int32_t left = cols + behind - col;
    return behind < 0 || left > per ? per : left;
}
// Rows, from the first on, that have kBehind values behind them for certain.
__host__ __device__ __forceinline__ int64_t rows_followed(int64_t rows, int64_t cols) {
    return rows - (cols >= kBehind ? 1 : kBehind);
}

}  // namespace fasgd
