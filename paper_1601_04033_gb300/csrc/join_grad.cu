// fasgd_join_grad.  With hats the normalised values and r the 1/sqrt of a row,
//   q  = dz pre,  dH = dh + r_h (q - mean q - hhat mean(q hhat))   (rms: no mean q)
//   dx = carry dH,  dgate += branch dH u,  dt = m scale branch gate dH
//   q2 = dt post,  dy = r_y (q2 - mean q2 - yhat mean(q2 yhat))
//   dpre += dz hhat, dpre_bias += dz, dpost += dt yhat, dpost_bias += dt.
// hhat comes from h formed again out of x and y, which costs the bytes that
// reading h would and keeps h's rounding out of the parameters' gradients.

#include "join.cuh"
#include "pdl.cuh"

namespace fasgd {
namespace {

constexpr int kThreads = 256;

// What both sweeps of the plain form need of element (r, c).
struct Point {
    Branch b;
    float hhat, dz, q, dh;
};
template <class T>
__device__ __forceinline__ Point point_at(const JoinArgs& a, int64_t r, int64_t c, const float4& st, float gate) {
    Point p;
    p.b = {0.f, 0.f, true};
    float h = to_f32(static_cast<const T*>(a.x)[r * a.ld_x + c]);
    if (a.y != nullptr) {
        p.b = branch_at<T>(a, r, c, st.x, st.y);
        h = a.carry * h + a.branch * gate * p.b.u;
    }
    p.hhat = (h - st.z) * st.w;
    p.dz = p.q = 0.f;
    if (a.pre != nullptr) {
        p.dz = to_f32(static_cast<const T*>(a.dz)[r * a.ld_dz + c]);
        p.q = p.dz * a.pre[c];
    }
    p.dh = a.dh != nullptr ? to_f32(static_cast<const T*>(a.dh)[r * a.ld_dh + c]) : 0.f;
    return p;
}
// dH of that element, given the row's means m = (mean q hhat, mean q).
__device__ __forceinline__ float d_stream(const JoinArgs& a, const Point& p, const float4& st, float2 m) {
    return a.pre != nullptr ? p.dh + st.w * (p.q - m.y - p.hhat * m.x) : p.dh;
}

template <class T>
__device__ __forceinline__ void store_gate(const JoinArgs& a, int64_t i, float v) {
    if (a.gate_f32)
        static_cast<float*>(a.out_gate)[i] = v;
    else
        static_cast<T*>(a.out_gate)[i] = from_f32<T>(v);
}

// dx, dy and the row's means: a block per row, any width, stride and alignment.
template <class T>
__global__ void __launch_bounds__(kThreads) grad_rows_any_kernel(const __grid_constant__ JoinArgs a) {
    constexpr int kWarps = kThreads / 32;
    __shared__ float smem[2 * kWarps];
    pdl_wait();
    pdl_trigger();
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const int64_t group = r / a.group_rows;
        const float4 st = a.stats[r];
        float s[2] = {0.f, 0.f};
        float2 m = {0.f, 0.f};
        if (a.pre != nullptr) {
            for (int64_t c = threadIdx.x; c < a.cols; c += kThreads) {
                const Point p = point_at<T>(a, r, c, st, gate_at<T>(a, group, c));
                s[0] += p.q * p.hhat;
                s[1] += p.q;
            }
            block_sums(s, smem, kWarps);
            m.x = s[0] * a.inv_cols;
            m.y = a.layer ? s[1] * a.inv_cols : 0.f;
        }
        if (threadIdx.x == 0) a.row_means[r] = m;
        s[0] = s[1] = 0.f;
        for (int64_t c = threadIdx.x; c < a.cols; c += kThreads) {
            const float gate = gate_at<T>(a, group, c);
            const Point p = point_at<T>(a, r, c, st, gate);
            const float d = d_stream(a, p, st, m);
            static_cast<T*>(a.dx)[r * a.ld_dx + c] = from_f32<T>(a.y != nullptr ? a.carry * d : d);
            if (a.y == nullptr) continue;
            const float dt = p.b.keep ? a.branch * gate * d * a.drop.scale : 0.f;
            if (a.post == nullptr) {
                static_cast<T*>(a.dy)[r * a.ld_dy + c] = from_f32<T>(dt);
            } else {
                const float q2 = dt * a.post[c];
                s[0] += q2 * p.b.yhat;
                s[1] += q2;
            }
        }
        if (a.post != nullptr) {
            block_sums(s, smem, kWarps);
            const float m1 = s[0] * a.inv_cols, m0 = a.layer ? s[1] * a.inv_cols : 0.f;
            for (int64_t c = threadIdx.x; c < a.cols; c += kThreads) {
                const float gate = gate_at<T>(a, group, c);
                const Point p = point_at<T>(a, r, c, st, gate);
                const float d = d_stream(a, p, st, m);
                const float dt = p.b.keep ? a.branch * gate * d * a.drop.scale : 0.f;
                static_cast<T*>(a.dy)[r * a.ld_dy + c] =
                    from_f32<T>(st.y * (dt * a.post[c] - m0 - p.b.yhat * m1));
            }
        }
    }
}

// The parameters' gradients of the plain form.  A unit is every splits-th row of
// one group; block (column tile, part) takes every parts-th unit, and each thread
// sums its column: the gate's gradient unit by unit, the parameters' over all.
template <class T>
__global__ void __launch_bounds__(kThreads) grad_columns_any_kernel(const __grid_constant__ JoinArgs a) {
    pdl_wait();
    pdl_trigger();
    const int64_t tiles = (a.cols + kThreads - 1) / kThreads;
    for (int64_t block = blockIdx.x; block < tiles * a.parts; block += gridDim.x) {
        const int64_t part = block / tiles, c = (block - part * tiles) * kThreads + threadIdx.x;
        if (c >= a.cols) continue;
        float s[4] = {0.f, 0.f, 0.f, 0.f};
        for (int64_t unit = part; unit < a.groups * a.splits; unit += a.parts) {
            const int64_t group = unit / a.splits;
            const float gate = gate_at<T>(a, group, c);
            float g = 0.f;
            for (int64_t i = unit - group * a.splits; i < a.group_rows; i += a.splits) {
                const int64_t r = group * a.group_rows + i;
                const float4 st = a.stats[r];
                const Point p = point_at<T>(a, r, c, st, gate);
                const float d = d_stream(a, p, st, a.row_means[r]);
                g += a.branch * d * p.b.u;
                if (a.post != nullptr) {
                    const float dt = p.b.keep ? a.branch * gate * d * a.drop.scale : 0.f;
                    s[0] += dt * p.b.yhat;
                    s[1] += dt;
                }
                s[2] += p.dz * p.hhat;
                s[3] += p.dz;
            }
            if (a.out_gate == nullptr) continue;
            if (a.splits > 1)
                a.gates[unit * a.cols + c] = g;
            else
                store_gate<T>(a, group * a.cols + c, g);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (a.out_param[k] != nullptr) a.params[(part * 4 + k) * a.cols + c] = s[k];
    }
}

// The gate's gradients that grad_finish_kernel has to write: a unit that is a
// whole group has written its own.
__host__ __device__ __forceinline__ int64_t gates_left(const JoinArgs& a) {
    return a.out_gate != nullptr && (a.splits > 1 || a.rows == 0) ? a.groups : 0;
}

// Joins the partial sums: a block takes 32 columns of one vector (the four
// parameters' gradients, then the gate's, group by group); eight lanes of rows
// take every eighth partial sum, then are added in order.
template <class T>
__global__ void __launch_bounds__(kThreads) grad_finish_kernel(const __grid_constant__ JoinArgs a) {
    __shared__ float smem[kThreads];
    pdl_wait();
    pdl_trigger();
    const int64_t tiles = (a.cols + 31) / 32;
    const int64_t vectors = 4 + gates_left(a);
    const int lane = threadIdx.x & 31, slot = threadIdx.x >> 5;
    for (int64_t u = blockIdx.x; u < tiles * vectors; u += gridDim.x) {
        const int64_t vec = u / tiles, c = (u - vec * tiles) * 32 + lane;
        if (vec < 4 && a.out_param[vec] == nullptr) continue;
        const float* src = vec < 4 ? a.params + vec * a.cols : a.gates + (vec - 4) * a.splits * a.cols;
        const int64_t step = vec < 4 ? 4 * a.cols : a.cols, count = vec < 4 ? a.parts : a.rows > 0 ? a.splits : 0;
        float s = 0.f;
        if (c < a.cols)
            for (int64_t i = slot; i < count; i += kThreads / 32) s += src[i * step + c];
        smem[threadIdx.x] = s;
        __syncthreads();
        if (slot == 0 && c < a.cols) {
            s = 0.f;
#pragma unroll
            for (int k = 0; k < kThreads / 32; ++k) s += smem[k * 32 + lane];
            if (vec < 4)
                a.out_param[vec][c] = s;
            else
                store_gate<T>(a, (vec - 4) * a.cols + c, s);
        }
        __syncthreads();
    }
}

int64_t at_most(int64_t n, int64_t cap) { return n < cap ? (n < 1 ? 1 : n) : cap; }

template <class T>
cudaError_t launch(const JoinArgs& a, int num_sms, cudaStream_t stream) {
    cudaError_t st = cudaSuccess;
    if (a.rows > 0) {
        st = launch_pdl(grad_rows_any_kernel<T>, (unsigned)at_most(a.rows, (int64_t)num_sms * 8), kThreads, 0,
                        stream, a);
        const int64_t tiles = (a.cols + kThreads - 1) / kThreads;
        if (st == cudaSuccess)
            st = launch_pdl(grad_columns_any_kernel<T>, (unsigned)at_most(tiles * a.parts, (int64_t)num_sms * 16),
                            kThreads, 0, stream, a);
    }
    const int64_t vectors = 4 + gates_left(a);
    if (st == cudaSuccess)
        st = launch_pdl(grad_finish_kernel<T>,
                        (unsigned)at_most((a.cols + 31) / 32 * vectors, (int64_t)num_sms * 64), kThreads, 0,
                        stream, a);
    return st;
}

}  // namespace

JoinPlan join_grad_plan(const JoinArgs& a, int dtype, int num_sms) {
    (void)dtype;
    JoinPlan p;
    p.fast = false;
    p.splits = (2 * (int64_t)num_sms + a.groups - 1) / a.groups;
    if (p.splits > a.group_rows) p.splits = a.group_rows;
    if (p.splits < 1) p.splits = 1;
    p.parts = a.rows > 0 ? at_most(a.groups * p.splits, 2 * (int64_t)num_sms) : 0;
    p.row_means = a.rows;
    return p;
}

cudaError_t launch_join_grad(const JoinArgs& a, int dtype, int num_sms, cudaStream_t stream) {
    if (dtype == FASGD_F32) return launch<float>(a, num_sms, stream);
    if (dtype == FASGD_BF16) return launch<__nv_bfloat16>(a, num_sms, stream);
    return launch<__half>(a, num_sms, stream);
}

}  // namespace fasgd
