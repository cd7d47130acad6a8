// Internal interface of the client operators (client.cu checks the arguments and
// launches; join.cu, join_grad.cu, dropout.cu and balance.cu hold the kernels).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "eq9.cuh"
#include "fasgd.h"

namespace fasgd {

// The draws of one dropout call: 16-bit halves of Philox words, eight elements
// (an octet) per counter.  One octet costs about 80 operations whatever is made
// of it; 32-bit draws, four to a counter, would make the generator and not the
// memory the bound of 16-bit activations.
struct DropArgs {
    uint32_t round_key0[10], round_key1[10];
    uint32_t client_word, n_lo, n_hi;
    uint32_t cut;       // dropped iff half < cut; 0: nothing is, 65536: everything is
    uint32_t last;      // (cut << 16) - 1, or 0 for cut = 0 (octet.cuh)
    float scale;        // 65536 / (65536 - cut)
};

struct DropoutArgs {
    const void* x;
    const void* residual;    // may be null
    void* out;
    int64_t rows, cols, ld_x, ld_residual, ld_out;
    DropArgs drop;
};

// fasgd_join and fasgd_join_grad as the kernels take them.
struct JoinArgs {
    const void *x, *y;
    void *h, *z;
    const float *post, *post_bias, *pre, *pre_bias;
    const void* gate;
    float4* stats;           // per row: mean y, 1/sqrt y, mean h, 1/sqrt h
    int64_t rows, cols, groups, group_rows;
    int64_t ld_x, ld_y, ld_h, ld_z;
    bool layer, gate_f32;
    float eps, carry, branch, inv_cols;
    DropArgs drop;
    // gradient
    const void *dh, *dz;
    void *dx, *dy;
    int64_t ld_dh, ld_dz, ld_dx, ld_dy;
    float2* row_means;       // per row: mean q hhat, mean q (the plain form only)
    float* params;           // partial sums [parts][5][cols]: post, post_bias, pre, pre_bias, a single gate
    float* gates;            // partial sums [groups * splits][cols] of the groups' gates (splits > 1)
    int64_t parts, splits;   // splits: units that each group's rows fall into; parts: blocks that take the units
    float* out_param[4];     // final gradients, each may be null
    void* out_gate;
};

struct BalanceArgs {
    const void* logits;
    const int32_t* chosen;
    const uint8_t* valid;
    const float* upstream;
    void* dlogits;
    int32_t* counts;
    float* loss;
    int64_t rows, cols, groups, group_rows, top;
    int64_t ld_logits, ld_dlogits;
    float balance_scale, z_scale;
    int32_t* part_valid;     // [groups * splits] a split's valid rows
    int32_t* part_counts;    // [groups * splits][cols] a split's counts (splits > 1; else counts itself)
    float2* part_loss;       // [kBalanceParts] the blocks' sums of the two losses
    uint32_t* ticket;        // blocks that have left theirs (set to 0 by the counting kernel)
    int64_t splits;          // parts of each group's rows in the counting
};

cudaError_t launch_dropout(const DropoutArgs& a, int dtype, int num_sms, cudaStream_t stream);
cudaError_t launch_join(const JoinArgs& a, int dtype, int num_sms, cudaStream_t stream);
cudaError_t launch_join_grad(const JoinArgs& a, int dtype, int num_sms, cudaStream_t stream);
// parts, splits and row_means' length of a gradient call.
struct JoinPlan {
    int64_t parts, splits, row_means;
};
JoinPlan join_grad_plan(const JoinArgs& a, int dtype, int num_sms);
cudaError_t launch_balance(const BalanceArgs& a, int dtype, int num_sms, cudaStream_t stream);
int64_t balance_splits(int64_t rows, int64_t groups, int64_t top);
constexpr int64_t kBalanceParts = 2048;     // sums the blocks of the loss leave at most

// ---- device side ----------------------------------------------------------

template <class T>
__device__ __forceinline__ float to_f32(T v);
template <>
__device__ __forceinline__ float to_f32(float v) { return v; }
template <>
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
template <>
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }

template <class T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32(float v) { return __float2bfloat16_rn(v); }
template <>
__device__ __forceinline__ __half from_f32(float v) { return __float2half_rn(v); }

__device__ __forceinline__ Philox4 draw_octet(const DropArgs& d, int64_t q) {
    return philox4x32_10((uint32_t)q, d.client_word, d.n_lo,
                         d.n_hi + ((uint32_t)((uint64_t)q >> 32) << 16), d.round_key0, d.round_key1);
}
// Element i of an octet: whether it is kept.
__device__ __forceinline__ bool kept(const Philox4& r, int i, uint32_t cut) {
    const uint32_t w = r.x[i >> 1];
    return ((i & 1) ? w >> 16 : w & 0xffffu) >= cut;
}
// The factor of one element by its index (a whole octet's draws for it alone).
__device__ __forceinline__ bool kept_at(const DropArgs& d, int64_t index) {
    const Philox4 r = draw_octet(d, index >> 3);
    const int i = (int)(index & 7);
    const uint32_t w = i < 4 ? (i < 2 ? r.x[0] : r.x[1]) : (i < 6 ? r.x[2] : r.x[3]);
    return ((i & 1) ? w >> 16 : w & 0xffffu) >= d.cut;
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
    return v;
}

}  // namespace fasgd
