// What the client operators' entry points share: errors, checks of arguments, and what
// a launch asks of the device.
#pragma once

#include <cuda_runtime.h>

#include <cstdarg>
#include <cstdint>
#include <cstdio>

#include "fasgd.h"

namespace fasgd {
void set_handleless_error(const char* msg);  // defined in runtime.cu
}

namespace {

constexpr int64_t kRowsMax = (int64_t)1 << 40;

[[maybe_unused]] int fail(int code, const char* fmt, ...) noexcept {
    char buf[256];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    try {
        fasgd::set_handleless_error(buf);
    } catch (...) {       // out of memory for the text: the code says enough
    }
    return code;
}
[[maybe_unused]] int cuda_status(cudaError_t st, const char* call) {
    return st == cudaSuccess ? FASGD_OK : fail(FASGD_ECUDA, "%s: %s", call, cudaGetErrorString(st));
}

[[maybe_unused]] bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
[[maybe_unused]] int64_t dtype_size(int32_t dtype) { return dtype == FASGD_F32 ? 4 : 2; }

// An argument's memory: `rows` rows of `width` bytes, `step` bytes apart.
struct Region {
    const char* name;
    const void* p;
    int64_t rows, width, step;
    bool output;
};
[[maybe_unused]] Region block(const char* name, const void* p, int64_t bytes, bool output) {
    return {name, p, 1, bytes, bytes, output};
}
[[maybe_unused]] bool share(const Region& a, const Region& b) {
    if (a.p == nullptr || b.p == nullptr || a.rows == 0 || b.rows == 0 || a.width == 0 || b.width == 0)
        return false;
    const uintptr_t pa = (uintptr_t)a.p, pb = (uintptr_t)b.p;
    const uintptr_t ea = pa + (uintptr_t)((a.rows - 1) * a.step + a.width);
    const uintptr_t eb = pb + (uintptr_t)((b.rows - 1) * b.step + b.width);
    if (ea <= pb || eb <= pa) return false;
    if (a.rows > 1 && b.rows > 1 && a.step == b.step) {   // columns of one wider matrix
        const uintptr_t off = (pa < pb ? pb - pa : pa - pb) % (uintptr_t)a.step;
        const int64_t first = pa < pb ? a.width : b.width, second = pa < pb ? b.width : a.width;
        if ((int64_t)off >= first && (int64_t)off + second <= a.step) return false;
    }
    return true;
}
// EINVAL where an output shares memory with another argument.
[[maybe_unused]] int check_shared(const char* call, const Region* r, int n) {
    for (int i = 0; i < n; ++i)
        for (int j = 0; j < i; ++j)
            if ((r[i].output || r[j].output) && share(r[i], r[j]))
                return fail(FASGD_EINVAL, "%s: %s and %s share memory", call, r[j].name, r[i].name);
    return FASGD_OK;
}

[[maybe_unused]] int check_shape(const char* call, int64_t rows, int64_t cols, int64_t cols_max, int32_t dtype) {
    if (rows < 0 || rows > kRowsMax || cols < 1 || cols > cols_max)
        return fail(FASGD_EINVAL, "%s: rows must be in [0, 2^40], cols in [1, %lld]", call, (long long)cols_max);
    if (dtype != FASGD_F32 && dtype != FASGD_BF16 && dtype != FASGD_F16)
        return fail(FASGD_EINVAL, "%s: dtype %d is not an fasgd_dtype", call, dtype);
    return FASGD_OK;
}
// A matrix argument: pointer, alignment of its type, row step.  ld is set to cols
// where there is no second row to step to.
[[maybe_unused]] int check_matrix(const char* call, const char* name, const void* p, int64_t& ld, int64_t rows, int64_t cols,
                 int64_t size) {
    if (p == nullptr) return fail(FASGD_EINVAL, "%s: %s is NULL", call, name);
    if (!aligned(p, (uintptr_t)size)) return fail(FASGD_EINVAL, "%s: %s is not aligned to its type", call, name);
    if (rows < 2) ld = cols;
    if (ld < cols || ld > kRowsMax || (__int128)ld * rows * size > ((__int128)1 << 62))
        return fail(FASGD_EINVAL, "%s: the rows of %s are %lld values apart, fewer than cols or too many", call,
                    name, (long long)ld);
    return FASGD_OK;
}

[[maybe_unused]] cudaError_t sm_count(int& sms) {
    int dev = 0;
    const cudaError_t st = cudaGetDevice(&dev);
    return st != cudaSuccess ? st : cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
}

[[maybe_unused]] int64_t up16(int64_t n) { return (n + 15) / 16 * 16; }

}  // namespace
