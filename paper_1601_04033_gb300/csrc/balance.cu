// fasgd_balance.  With f[g,e] = counts[g,e] / (top N_g), which `chosen` alone
// fixes, and dot_t = sum_e f[g,e] p_te,
//   balance = cols / G' sum_g 1/N_g sum_t dot_t,   z = 1/N sum_t lse_t^2,
//   dlogits_te = up p_te (s (f[g,e] - dot_t) + 2 z_scale / N lse_t),  s = balance_scale cols / (G' N_g).
// So once the assignments are counted, the losses and the gradient take one pass
// over the logits, and a row leaves two numbers, not cols probabilities, to sum.

#include "client.cuh"
#include "pdl.cuh"

namespace fasgd {
namespace {

constexpr int kCountThreads = 512;
constexpr int kThreads = 256;

// Counts of one split of one group's rows, in shared memory (integers: the order
// of the additions does not show).
__global__ void __launch_bounds__(kCountThreads) balance_count_kernel(const __grid_constant__ BalanceArgs a) {
    __shared__ int32_t hist[FASGD_EXPERTS_MAX];
    __shared__ int32_t rows_valid;
    pdl_wait();
    pdl_trigger();
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.ticket = 0;
    const int64_t per = (a.group_rows + a.splits - 1) / a.splits;
    const int cols = (int)a.cols;
    const uint32_t top = (uint32_t)a.top;
    for (int64_t unit = blockIdx.x; unit < a.groups * a.splits; unit += gridDim.x) {
        const int64_t group = unit / a.splits, split = unit - group * a.splits;
        const int64_t from = split * per < a.group_rows ? split * per : a.group_rows;
        const int64_t to = from + per < a.group_rows ? from + per : a.group_rows;
        const int64_t r0 = group * a.group_rows + from, r1 = group * a.group_rows + to;
        for (int e = threadIdx.x; e < cols; e += kCountThreads) hist[e] = 0;
        if (threadIdx.x == 0) rows_valid = 0;
        __syncthreads();
        if (a.valid != nullptr) {
            int32_t v = 0;
            for (int64_t r = r0 + threadIdx.x; r < r1; r += kCountThreads) v += a.valid[r] != 0;
            v = __reduce_add_sync(0xffffffffu, v);
            if ((threadIdx.x & 31) == 0 && v != 0) atomicAdd(&rows_valid, v);
        }
        const uint32_t i1 = (uint32_t)(r1 * a.top);
        for (uint32_t i = (uint32_t)(r0 * a.top) + threadIdx.x; i < i1; i += kCountThreads) {
            const int32_t e = a.chosen[i];
            if ((uint32_t)e < (uint32_t)cols && (a.valid == nullptr || a.valid[i / top] != 0))
                atomicAdd(&hist[e], 1);
        }
        __syncthreads();
        int32_t* out = a.splits > 1 ? a.part_counts + unit * cols : a.counts + group * cols;
        for (int e = threadIdx.x; e < cols; e += kCountThreads) out[e] = hist[e];
        if (threadIdx.x == 0) a.part_valid[unit] = a.valid != nullptr ? rows_valid : (int32_t)(r1 - r0);
        __syncthreads();
    }
}

// Sum of one value over the block, every thread ending with it.
__device__ __forceinline__ float block_sum(float v, float* smem) {
    v = warp_sum(v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) smem[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) v += smem[w];
    return v;
}

// A unit is `unit_rows` consecutive rows of one group; a block takes every
// gridDim-th unit, a warp a row at a time.
template <class T>
__global__ void __launch_bounds__(kThreads)
    balance_any_kernel(const __grid_constant__ BalanceArgs a, int64_t unit_rows) {
    __shared__ float f[FASGD_EXPERTS_MAX];
    __shared__ float smem[kThreads / 32];
    __shared__ bool last;
    constexpr int kWarps = kThreads / 32;
    pdl_wait();
    pdl_trigger();
    const int cols = (int)a.cols, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    // N and G'.
    float live = (float)a.groups, rows_all = (float)a.rows;
    if (a.valid != nullptr) {
        float n = 0.f, g1 = 0.f;
        for (int64_t g = threadIdx.x; g < a.groups; g += kThreads) {
            int32_t v = 0;
            for (int64_t s = 0; s < a.splits; ++s) v += a.part_valid[g * a.splits + s];
            n += (float)v;
            g1 += v > 0 ? 1.f : 0.f;
        }
        rows_all = block_sum(n, smem);
        live = block_sum(g1, smem);
    }
    const float up = a.upstream != nullptr ? *a.upstream : 1.f;
    const float zscale = rows_all > 0.f ? 2.f * a.z_scale / rows_all : 0.f;
    const int64_t units_per_group = (a.group_rows + unit_rows - 1) / unit_rows;
    float sum_dot = 0.f, sum_z = 0.f;
    for (int64_t unit = blockIdx.x; unit < a.groups * units_per_group; unit += gridDim.x) {
        const int64_t group = unit / units_per_group, part = unit - group * units_per_group;
        int32_t n = 0;
        for (int64_t s = 0; s < a.splits; ++s) n += a.part_valid[group * a.splits + s];
        const float inv_n = n > 0 ? 1.f / (float)n : 0.f;
        __syncthreads();
        for (int e = threadIdx.x; e < cols; e += kThreads) {
            int32_t c = 0;
            if (a.splits > 1) {
                for (int64_t s = 0; s < a.splits; ++s) c += a.part_counts[(group * a.splits + s) * cols + e];
                if (part == 0) a.counts[group * cols + e] = c;
            } else {
                c = a.counts[group * cols + e];
            }
            f[e] = (float)c * (inv_n / (float)a.top);
        }
        __syncthreads();
        const float scale = live > 0.f ? a.balance_scale * (float)cols / live * inv_n : 0.f;
        const int64_t end = (part + 1) * unit_rows < a.group_rows ? (part + 1) * unit_rows : a.group_rows;
        float unit_dot = 0.f;
        for (int64_t i = part * unit_rows + warp; i < end; i += kWarps) {
            const int64_t r = group * a.group_rows + i;
            const T* x = static_cast<const T*>(a.logits) + r * a.ld_logits;
            T* d = static_cast<T*>(a.dlogits) + r * a.ld_dlogits;
            if (a.valid != nullptr && a.valid[r] == 0) {
                if (a.dlogits != nullptr)
                    for (int e = lane; e < cols; e += 32) d[e] = from_f32<T>(0.f);
                continue;
            }
            float top = -INFINITY;
            for (int e = lane; e < cols; e += 32) top = fmaxf(top, to_f32(x[e]));
#pragma unroll
            for (int off = 16; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
            float sum = 0.f, dot = 0.f;
            for (int e = lane; e < cols; e += 32) {
                const float p = expf(to_f32(x[e]) - top);
                sum += p;
                dot += f[e] * p;
            }
            sum = warp_sum(sum);
            dot = warp_sum(dot);
            bool nan_row = false;
            for (int e = lane; e < cols; e += 32) nan_row |= isnan(to_f32(x[e]));
            nan_row = __any_sync(0xffffffffu, nan_row);
            const bool empty = top == -INFINITY && !nan_row;   // no expert is open to this row
            const float inv = empty ? 0.f : 1.f / sum, lse = empty ? 0.f : top + logf(sum);
            dot = empty ? 0.f : dot * inv;
            unit_dot += dot;
            sum_z += lse * lse;
            if (a.dlogits != nullptr)
                for (int e = lane; e < cols; e += 32) {
                    const float p = empty ? 0.f : expf(to_f32(x[e]) - top) * inv;
                    d[e] = from_f32<T>(up * p * (scale * (f[e] - dot) + zscale * lse));
                }
        }
        sum_dot += unit_dot * inv_n;
    }
    if (a.loss == nullptr) return;
    // The warps' sums (equal in all lanes), then the blocks', in order.
    __syncthreads();
    if (lane == 0) smem[warp] = sum_dot;
    __syncthreads();
    float dot = 0.f, z = 0.f;
    if (threadIdx.x == 0)
        for (int w = 0; w < kWarps; ++w) dot += smem[w];
    __syncthreads();
    if (lane == 0) smem[warp] = sum_z;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 0; w < kWarps; ++w) z += smem[w];
        a.part_loss[blockIdx.x] = make_float2(dot, z);
        __threadfence();
        last = atomicAdd(a.ticket, 1u) == gridDim.x - 1;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    dot = z = 0.f;
    for (int b = threadIdx.x; b < (int)gridDim.x; b += kThreads) {
        const float2 v = __ldcg(&a.part_loss[b]);
        dot += v.x;
        z += v.y;
    }
    dot = block_sum(dot, smem);
    z = block_sum(z, smem);
    if (threadIdx.x == 0) {
        const float balance = live > 0.f ? (float)cols / live * dot : 0.f;
        z = rows_all > 0.f ? z / rows_all : 0.f;
        a.loss[0] = a.balance_scale * balance + a.z_scale * z;
        a.loss[1] = balance;
        a.loss[2] = z;
    }
}

__global__ void balance_nothing_kernel(const __grid_constant__ BalanceArgs a) {
    pdl_wait();
    pdl_trigger();
    const int64_t stride = (int64_t)gridDim.x * blockDim.x;
    const int64_t t = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    for (int64_t i = t; i < a.groups * a.cols; i += stride) a.counts[i] = 0;
    if (t < 3 && a.loss != nullptr) a.loss[t] = 0.f;
}

template <class T>
cudaError_t launch(const BalanceArgs& a, int num_sms, cudaStream_t stream) {
    const int64_t cap = (int64_t)num_sms * 8 < kBalanceParts ? (int64_t)num_sms * 8 : kBalanceParts;
    int64_t unit_rows = (a.rows + cap - 1) / cap;
    unit_rows = (unit_rows + 7) / 8 * 8;
    if (unit_rows > a.group_rows) unit_rows = a.group_rows;
    const int64_t units = a.groups * ((a.group_rows + unit_rows - 1) / unit_rows);
    return launch_pdl(balance_any_kernel<T>, (unsigned)(units < cap ? units : cap), kThreads, 0, stream, a,
                      unit_rows);
}

}  // namespace

// Parts of each group in the counting: 32,768 assignments each, 64 at most (every
// block of the pass adds up its group's).
int64_t balance_splits(int64_t rows, int64_t groups, int64_t top) {
    if (groups < 1) return 1;
    const int64_t n = rows / groups * top, s = (n + 32767) / 32768;
    return s < 1 ? 1 : s > 64 ? 64 : s;
}

cudaError_t launch_balance(const BalanceArgs& a, int dtype, int num_sms, cudaStream_t stream) {
    if (a.rows == 0) return launch_pdl(balance_nothing_kernel, 32, kThreads, 0, stream, a);
    const int64_t units = a.groups * a.splits, cap = (int64_t)num_sms * 4;
    const cudaError_t st = launch_pdl(balance_count_kernel, (unsigned)(units < cap ? units : cap),
                                      kCountThreads, 0, stream, a);
    if (st != cudaSuccess) return st;
    if (dtype == FASGD_F32) return launch<float>(a, num_sms, stream);
    if (dtype == FASGD_BF16) return launch<__nv_bfloat16>(a, num_sms, stream);
    return launch<__half>(a, num_sms, stream);
}

}  // namespace fasgd
