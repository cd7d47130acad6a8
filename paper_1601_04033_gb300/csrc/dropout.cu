// fasgd_dropout: out = residual + m x scale, the mask drawn where it is used.

#include "client.cuh"
#include "pdl.cuh"

namespace fasgd {
namespace {

constexpr int kThreads = 256;

template <class T>
__device__ __forceinline__ T drop_one(T x, bool keep, float scale, bool residual, T res) {
    const float v = keep ? to_f32(x) * scale : 0.f;
    return from_f32<T>(residual ? v + to_f32(res) : v);
}

// Any strides and alignments: a thread takes an octet of the matrix's elements,
// which may end in a later row than it began in.
template <class T>
__global__ void __launch_bounds__(kThreads) dropout_any_kernel(const __grid_constant__ DropoutArgs a) {
    pdl_wait();
    pdl_trigger();
    const T* x = static_cast<const T*>(a.x);
    const T* res = static_cast<const T*>(a.residual);
    T* out = static_cast<T*>(a.out);
    const int64_t count = a.rows * a.cols, octets = (count + 7) >> 3;
    const int64_t stride = (int64_t)gridDim.x * kThreads;
    for (int64_t q = (int64_t)blockIdx.x * kThreads + threadIdx.x; q < octets; q += stride) {
        const Philox4 r = draw_octet(a.drop, q);
        int64_t row = (q << 3) / a.cols, col = (q << 3) - row * a.cols;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (row >= a.rows) break;
            out[row * a.ld_out + col] =
                drop_one<T>(x[row * a.ld_x + col], kept(r, i, a.drop.cut), a.drop.scale,
                            res != nullptr, res != nullptr ? res[row * a.ld_residual + col] : T());
            if (++col == a.cols) {
                col = 0;
                ++row;
            }
        }
    }
}

template <class T>
cudaError_t launch(const DropoutArgs& a, int num_sms, cudaStream_t stream) {
    const int64_t octets = (a.rows * a.cols + 7) >> 3;
    int64_t grid = (octets + kThreads - 1) / kThreads;
    if (grid > (int64_t)num_sms * 16) grid = (int64_t)num_sms * 16;
    return launch_pdl(dropout_any_kernel<T>, (unsigned)grid, kThreads, 0, stream, a);
}

}  // namespace

cudaError_t launch_dropout(const DropoutArgs& a, int dtype, int num_sms, cudaStream_t stream) {
    if (a.rows == 0) return cudaSuccess;
    if (dtype == FASGD_F32) return launch<float>(a, num_sms, stream);
    if (dtype == FASGD_BF16) return launch<__nv_bfloat16>(a, num_sms, stream);
    return launch<__half>(a, num_sms, stream);
}

}  // namespace fasgd
