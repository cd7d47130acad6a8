// fasgd_join: t = N(y), u = dropout(t), h = carry x + branch gate u, z = N(h).

#include "join.cuh"
#include "pdl.cuh"

namespace fasgd {
namespace {

constexpr int kThreads = 256;

// Any width, stride and alignment: a block takes a row at a time and reads it
// again for every statistic (out of L2, where a row fits).
template <class T>
__global__ void __launch_bounds__(kThreads) join_any_kernel(const __grid_constant__ JoinArgs a) {
    __shared__ float smem[kThreads / 32];
    constexpr int kWarps = kThreads / 32;
    pdl_wait();
    pdl_trigger();
    const T* x = static_cast<const T*>(a.x);
    const T* y = static_cast<const T*>(a.y);
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const int64_t group = r / a.group_rows;
        float4 st = {0.f, 1.f, 0.f, 1.f};
        float s[1];
        if (a.post != nullptr) {
            if (a.layer) {
                s[0] = 0.f;
                for (int64_t c = threadIdx.x; c < a.cols; c += kThreads) s[0] += to_f32(y[r * a.ld_y + c]);
                block_sums(s, smem, kWarps);
                st.x = s[0] * a.inv_cols;
            }
            s[0] = 0.f;
            for (int64_t c = threadIdx.x; c < a.cols; c += kThreads) {
                const float d = to_f32(y[r * a.ld_y + c]) - st.x;
                s[0] += d * d;
            }
            block_sums(s, smem, kWarps);
            st.y = 1.f / sqrtf(s[0] * a.inv_cols + a.eps);
        }
        const auto value = [&](int64_t c) {
            const float v = to_f32(x[r * a.ld_x + c]);
            if (y == nullptr) return v;
            return a.carry * v + a.branch * gate_at<T>(a, group, c) * branch_at<T>(a, r, c, st.x, st.y).u;
        };
        s[0] = 0.f;
        for (int64_t c = threadIdx.x; c < a.cols; c += kThreads) {
            const float v = value(c);
            if (y != nullptr) static_cast<T*>(a.h)[r * a.ld_h + c] = from_f32<T>(v);
            s[0] += a.layer ? v : v * v;
        }
        if (a.pre != nullptr) {
            block_sums(s, smem, kWarps);
            if (a.layer) {
                st.z = s[0] * a.inv_cols;
                s[0] = 0.f;
                for (int64_t c = threadIdx.x; c < a.cols; c += kThreads) {
                    const float d = value(c) - st.z;
                    s[0] += d * d;
                }
                block_sums(s, smem, kWarps);
            }
            st.w = 1.f / sqrtf(s[0] * a.inv_cols + a.eps);
            for (int64_t c = threadIdx.x; c < a.cols; c += kThreads) {
                float z = (value(c) - st.z) * st.w * a.pre[c];
                if (a.pre_bias != nullptr) z += a.pre_bias[c];
                static_cast<T*>(a.z)[r * a.ld_z + c] = from_f32<T>(z);
            }
        }
        if (a.stats != nullptr && threadIdx.x == 0) a.stats[r] = st;
    }
}

template <class T>
cudaError_t launch(const JoinArgs& a, int num_sms, cudaStream_t stream) {
    const int64_t grid = a.rows < (int64_t)num_sms * 8 ? a.rows : (int64_t)num_sms * 8;
    return launch_pdl(join_any_kernel<T>, (unsigned)grid, kThreads, 0, stream, a);
}

}  // namespace

cudaError_t launch_join(const JoinArgs& a, int dtype, int num_sms, cudaStream_t stream) {
    if (a.rows == 0) return cudaSuccess;
    if (dtype == FASGD_F32) return launch<float>(a, num_sms, stream);
    if (dtype == FASGD_BF16) return launch<__nv_bfloat16>(a, num_sms, stream);
    return launch<__half>(a, num_sms, stream);
}

}  // namespace fasgd
