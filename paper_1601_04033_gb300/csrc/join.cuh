// Shared by the forward and gradient kernels of the residual join.
#pragma once

#include "client.cuh"

namespace fasgd {
namespace {

// Sums of N values over the block, every thread ending with them; `smem` holds
// N * warps floats and is free again after the call's second barrier.
template <int N>
__device__ __forceinline__ void block_sums(float (&v)[N], float* smem, int warps) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = warp_sum(v[i]);
    if ((threadIdx.x & 31) == 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) smem[i * warps + (threadIdx.x >> 5)] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        float s = 0.f;
        for (int w = 0; w < warps; ++w) s += smem[i * warps + w];
        v[i] = s;
    }
    __syncthreads();
}

template <class T>
__device__ __forceinline__ float gate_at(const JoinArgs& a, int64_t group, int64_t c) {
    if (a.gate == nullptr) return 1.f;
    const int64_t i = group * a.cols + c;
    return a.gate_f32 ? static_cast<const float*>(a.gate)[i] : to_f32(static_cast<const T*>(a.gate)[i]);
}

// One element of the branch: yhat, t's draw applied (u), and whether it is kept.
struct Branch {
    float yhat, u;
    bool keep;
};
template <class T>
__device__ __forceinline__ Branch branch_at(const JoinArgs& a, int64_t r, int64_t c, float mean, float rstd) {
    Branch b;
    b.yhat = (to_f32(static_cast<const T*>(a.y)[r * a.ld_y + c]) - mean) * rstd;
    float t = b.yhat;
    if (a.post != nullptr) t *= a.post[c];
    if (a.post_bias != nullptr) t += a.post_bias[c];
    b.keep = a.drop.cut == 0 || kept_at(a.drop, r * a.cols + c);
    b.u = b.keep ? t * a.drop.scale : 0.f;
    return b;
}

}  // namespace
}  // namespace fasgd
