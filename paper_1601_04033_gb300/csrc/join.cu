// fasgd_join: t = N(y), u = dropout(t), h = carry x + branch gate u, z = N(h).

#include "join.cuh"
#include "octet.cuh"
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

// Rows in octets: TPR threads hold a row, NV octets each, between its statistics,
// so x and y are read once; blocks stay and take every gridDim-th row, the next
// STAGES - 1 of them on their way into shared memory.
template <class T, int TPR, int NV, int STAGES, bool LAYER>
__global__ void __launch_bounds__(TPR < 256 ? 256 : TPR) join_rows_kernel(const __grid_constant__ JoinArgs a) {
    constexpr int kBlock = TPR < 256 ? 256 : TPR, kSubs = kBlock / TPR;
    constexpr int kSlots = 2 * NV * kPieces<T>;      // 16-byte places of a stage, each kBlock wide
    extern __shared__ uint4 ring[];
    __shared__ __align__(16) float red[kSubs * 2 * (TPR < 32 ? 1 : TPR / 32)];
    const int sub = threadIdx.x / TPR, lane = threadIdx.x % TPR;
    const int32_t cols = (int32_t)a.cols;
    const int64_t step = (int64_t)gridDim.x * kSubs, first = (int64_t)blockIdx.x * kSubs + sub;
    // Where a warp holds several rows, it goes on until the first of them is past the end.
    const int64_t last = a.rows + (TPR < 32 ? sub % (32 / TPR) : 0);
    const int shift = (int)((first * a.cols) & 7);
    Columns c[NV] = {{lane, shift, cols}};
#pragma unroll
    for (int v = 1; v < NV; ++v) c[v] = Columns(lane + v * TPR, shift, cols);
    RowSums<TPR, 1> sums(red, sub);
    const T* x = static_cast<const T*>(a.x);
    const T* y = static_cast<const T*>(a.y);
    const bool has_y = y != nullptr, has_pre = a.pre != nullptr, has_post = a.post != nullptr;
    const int64_t end_x = (a.rows - 1) * a.ld_x + a.cols, end_y = (a.rows - 1) * a.ld_y + a.cols;
    pdl_wait();
    pdl_trigger();

    const auto fetch = [&](int64_t r, int stage) {
        if (r < a.rows) {
            uint4* slot = ring + stage * kSlots * kBlock + threadIdx.x;
#pragma unroll
            for (int v = 0; v < NV; ++v)
                if (c[v].any()) {
                    copy_octet<T>(slot + v * kPieces<T> * kBlock, kBlock, x + r * a.ld_x, c[v],
                                  end_x - r * a.ld_x - c[v].c0);
                    if (has_y)
                        copy_octet<T>(slot + (NV + v) * kPieces<T> * kBlock, kBlock, y + r * a.ld_y, c[v],
                                      end_y - r * a.ld_y - c[v].c0);
                }
        }
        copy_commit();
    };
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) fetch(first + s * step, s);

    Oct post[NV], post_bias[NV], gate[NV], pre[NV], pre_bias[NV];
    const bool gates = a.groups > 1;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        post[v] = load_vector(a.post, c[v], 1.f);
        if (LAYER) post_bias[v] = load_vector(a.post_bias, c[v], 0.f);
        if (!gates) {
            gate[v] = load_gate<T>(a, 0, c[v]);
#pragma unroll
            for (int i = 0; i < 4; ++i) gate[v].v[i] = mul2(gate[v].v[i], f2(a.branch));
        }
        pre[v] = load_vector(a.pre, c[v], 0.f);
        if (LAYER) pre_bias[v] = load_vector(a.pre_bias, c[v], 0.f);
    }

    int stage = 0;
    for (int64_t r = first; r < last; r += step) {
        const bool live = TPR >= 32 || r < a.rows;
        copy_wait<STAGES - 2>();
        const uint4* slot = ring + stage * kSlots * kBlock + threadIdx.x;
        Oct h[NV], t[NV];
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            h[v] = take_octet<T>(slot + v * kPieces<T> * kBlock, kBlock, c[v]);
            if (has_y) t[v] = take_octet<T>(slot + (NV + v) * kPieces<T> * kBlock, kBlock, c[v]);
        }
        fetch(r + (STAGES - 1) * step, stage == 0 ? STAGES - 1 : stage - 1);
        stage = stage == STAGES - 1 ? 0 : stage + 1;
        float4 st = {0.f, 1.f, 0.f, 1.f};
        float s[1];
        const auto centre = [&](Oct (&o)[NV]) {      // the row's mean, taken off; 0 where there is no column
            float2 p = f2(0.f);
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int i = 0; i < 4; ++i) p = add2(p, o[v].v[i]);
            s[0] = p.x + p.y;
            sums(s);
            const float mean = s[0] * a.inv_cols;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
#pragma unroll
                for (int i = 0; i < 4; ++i) o[v].v[i] = add2(o[v].v[i], f2(-mean));
                if (!c[v].any()) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[v].v[i] = f2(0.f);
                } else {
                    mask(o[v], c[v]);
                }
            }
            return mean;
        };
        const auto inverse = [&](const Oct (&o)[NV]) {
            float2 p = f2(0.f);
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int i = 0; i < 4; ++i) p = fma2(o[v].v[i], o[v].v[i], p);
            s[0] = p.x + p.y;
            sums(s);
            return rsqrtf(fmaf(s[0], a.inv_cols, a.eps));
        };
        if (has_y) {
            if (has_post) {
                if (LAYER) st.x = centre(t);
                st.y = inverse(t);
            }
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                if (gates) {
                    gate[v] = load_gate<T>(a, (live ? r : 0) / a.group_rows, c[v]);
#pragma unroll
                    for (int i = 0; i < 4; ++i) gate[v].v[i] = mul2(gate[v].v[i], f2(a.branch));
                }
                uint32_t bits = 0xffu;
                if (a.drop.cut != 0 && c[v].any()) bits = kept_bits(a.drop, (r * a.cols + c[v].c0) >> 3);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float2 u = mul2(mul2(t[v].v[i], f2(st.y)), post[v].v[i]);
                    if (LAYER) u = add2(u, post_bias[v].v[i]);
                    if (a.drop.cut != 0) u = select2(bits, i, mul2(u, f2(a.drop.scale)));
                    h[v].v[i] = fma2(gate[v].v[i], u, mul2(h[v].v[i], f2(a.carry)));
                }
                if (live) store_octet(static_cast<T*>(a.h) + r * a.ld_h, c[v], h[v]);
            }
        }
        if (has_pre) {
            if (LAYER) st.z = centre(h);
            st.w = inverse(h);
#pragma unroll
            for (int v = 0; v < NV; ++v) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    h[v].v[i] = mul2(mul2(h[v].v[i], f2(st.w)), pre[v].v[i]);
                    if (LAYER) h[v].v[i] = add2(h[v].v[i], pre_bias[v].v[i]);
                }
                if (live) store_octet(static_cast<T*>(a.z) + r * a.ld_z, c[v], h[v]);
            }
        }
        if (lane == 0 && live && a.stats != nullptr) a.stats[r] = st;
    }
}

template <class T, int TPR, int NV, int STAGES, bool LAYER>
cudaError_t launch_rows(const JoinArgs& a, int num_sms, int per_sm, cudaStream_t stream) {
    constexpr int kBlock = TPR < 256 ? 256 : TPR, kSubs = kBlock / TPR;
    constexpr size_t kSmem = (size_t)STAGES * 2 * NV * kPieces<T> * kBlock * 16;
    int64_t grid = (a.rows + kSubs - 1) / kSubs;
    // Past one row each, blocks step by a multiple of 8 rows (octet.cuh).
    const int64_t cap = (int64_t)num_sms * per_sm / 8 * 8;
    if (grid > cap) grid = cap;
    if (kSmem > 40 * 1024) {    // beyond 48 KB with the kernel's own: asked for
        const cudaError_t st = cudaFuncSetAttribute(join_rows_kernel<T, TPR, NV, STAGES, LAYER>,
                                                    cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem);
        if (st != cudaSuccess) return st;
    }
    return launch_pdl(join_rows_kernel<T, TPR, NV, STAGES, LAYER>, (unsigned)grid, kBlock, kSmem, stream, a);
}

template <class T, bool LAYER>
cudaError_t launch_octets(const JoinArgs& a, int num_sms, cudaStream_t stream) {
    const int64_t octets = row_octets(a.cols);
    if (octets <= 8) return launch_rows<T, 8, 1, 3, LAYER>(a, num_sms, 4, stream);
    if (octets <= 32) return launch_rows<T, 32, 1, 3, LAYER>(a, num_sms, 4, stream);
    if (octets <= 64) return launch_rows<T, 64, 1, 3, LAYER>(a, num_sms, 4, stream);
    if (octets <= 128) return launch_rows<T, 128, 1, 3, LAYER>(a, num_sms, 4, stream);
    if (octets <= 256) return launch_rows<T, 256, 1, 3, LAYER>(a, num_sms, 4, stream);
    if (octets <= 512) return launch_rows<T, 512, 1, 3, LAYER>(a, num_sms, 2, stream);
    return launch_rows<T, 1024, 1, 3, LAYER>(a, num_sms, 1, stream);
}

bool in_octets(const JoinArgs& a) {
    return row_octets(a.cols) <= 1024 && octet_matrix(a.x, a.ld_x, a.rows, a.cols) &&
           octet_matrix(a.y, a.ld_y, a.rows, a.cols) && octet_matrix(a.h, a.ld_h, a.rows, a.cols) &&
           octet_matrix(a.z, a.ld_z, a.rows, a.cols) &&
           (a.cols % 8 == 0 || a.rows < 2 ||
            (a.ld_x == a.cols && (a.y == nullptr || a.ld_y == a.cols) && (a.h == nullptr || a.ld_h == a.cols) &&
             (a.z == nullptr || a.ld_z == a.cols)));
}

template <class T>
cudaError_t launch(const JoinArgs& a, int num_sms, cudaStream_t stream) {
    if (in_octets(a))
        return a.layer ? launch_octets<T, true>(a, num_sms, stream) : launch_octets<T, false>(a, num_sms, stream);
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
