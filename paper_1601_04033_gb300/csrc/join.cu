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

// Rows in octets: TPR threads hold a row between its statistics, an octet each
// (or as many in each of the C blocks of a cluster), so x and y are read once;
// blocks stay and take every gridDim-th row, the next STAGES - 1 of them on their
// way into shared memory.
template <class T, int TPR, int C, int STAGES, bool LAYER>
__global__ void __launch_bounds__(TPR < 256 ? 256 : TPR, TPR <= 256 ? (LAYER ? 3 : 4) : TPR == 512 ? 2 : 1)
    join_rows_kernel(const __grid_constant__ JoinArgs a) {
    constexpr int kBlock = TPR < 256 ? 256 : TPR, kSubs = kBlock / TPR, kP = kPieces<T>;
    using Sums = RowSums<TPR, 1, C>;
    extern __shared__ uint4 ring[];                  // [STAGES][x, y][kP][kBlock]
    __shared__ __align__(16) float red[kSubs * Sums::kPlaces];
    const int sub = threadIdx.x / TPR, lane = threadIdx.x % TPR;
    const int64_t step = (int64_t)(gridDim.x / C) * kSubs, first = (int64_t)(blockIdx.x / C) * kSubs + sub;
    // Where a warp holds several rows, it goes on until the first of them is past the end.
    const int64_t end = a.rows + (TPR < 32 ? sub % (32 / TPR) : 0);
    const bool ragged = (a.cols & 7) != 0;
    const Columns c(lane + (C > 1 ? (int)cluster_rank() * TPR : 0), ragged ? (int)((first * a.cols) & 7) : 0,
                    (int32_t)a.cols);
    Sums sums(red, sub);
    const bool has_y = a.y != nullptr, has_pre = a.pre != nullptr, has_post = a.post != nullptr;
    pdl_wait();
    pdl_trigger();

    const T* x = static_cast<const T*>(a.x) + first * a.ld_x + c.c0;      // of the next row to fetch
    const T* y = static_cast<const T*>(a.y) + first * a.ld_y + c.c0;
    int64_t fetched = first, left = (a.rows - first) * a.cols - c.c0;       // (used where rows leave no gaps)
    const auto fetch = [&](uint4* slot) {
        if (fetched < a.rows && c.any()) {
            const bool whole = !ragged || left >= kOctet;
            copy_octet<T>(slot, kBlock, x, whole, left);
            if (has_y) copy_octet<T>(slot + kP * kBlock, kBlock, y, whole, left);
        }
        copy_commit();
        fetched += step;
        left -= step * a.cols;
        x += step * a.ld_x;
        y += step * a.ld_y;
    };
    constexpr int kStage = 2 * kP * kBlock;
    uint4* const mine = ring + threadIdx.x;
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) fetch(mine + s * kStage);

    // u = yhat (post scale) + post_bias scale.
    Oct post = load_vector(a.post, c, 1.f), post_bias, gate, pre = load_vector(a.pre, c, 0.f), pre_bias;
    const bool gates = a.groups > 1;
    if (LAYER) {
        post_bias = load_vector(a.post_bias, c, 0.f);
        pre_bias = load_vector(a.pre_bias, c, 0.f);
    }
    if (!gates) gate = load_gate<T>(a, 0, c);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        post.v[i] = mul2(post.v[i], f2(a.drop.scale));
        if (LAYER) post_bias.v[i] = mul2(post_bias.v[i], f2(a.drop.scale));
        if (!gates) gate.v[i] = mul2(gate.v[i], f2(a.branch));
    }
    T* hp = static_cast<T*>(a.h) + first * a.ld_h + c.c0;
    T* zp = static_cast<T*>(a.z) + first * a.ld_z + c.c0;

    const auto centre = [&](Oct& o) {      // the row's mean, taken off; 0 where there is no column
        const float2 p = add2(add2(o.v[0], o.v[1]), add2(o.v[2], o.v[3]));
        float s[1] = {p.x + p.y};
        sums(s);
        const float mean = s[0] * a.inv_cols;
#pragma unroll
        for (int i = 0; i < 4; ++i) o.v[i] = add2(o.v[i], f2(-mean));
        mask(o, c);
        return mean;
    };
    const auto inverse = [&](const Oct& o) {
        const float2 p = fma2(o.v[0], o.v[0], mul2(o.v[1], o.v[1]));
        const float2 q = fma2(o.v[2], o.v[2], mul2(o.v[3], o.v[3]));
        float s[1] = {(p.x + q.x) + (p.y + q.y)};
        sums(s);
        return rsqrtf(fmaf(s[0], a.inv_cols, a.eps));
    };

    int stage = 0;
    for (int64_t r = first; r < end; r += step) {
        const bool live = TPR >= 32 || r < a.rows;
        copy_wait<STAGES - 2>();
        const uint4* slot = mine + stage * kStage;
        Oct h = take_octet<T>(slot, kBlock, c), t = {};
        if (has_y) t = take_octet<T>(slot + kP * kBlock, kBlock, c);
        fetch(mine + (stage == 0 ? STAGES - 1 : stage - 1) * kStage);
        stage = stage == STAGES - 1 ? 0 : stage + 1;
        float4 st = {0.f, 1.f, 0.f, 1.f};
        if (has_y) {
            const Philox4 draws = octet_draws(a.drop, c.any(), (r * a.cols + c.c0) >> 3);
            if (gates) {
                gate = load_gate<T>(a, (live ? r : 0) / a.group_rows, c);
#pragma unroll
                for (int i = 0; i < 4; ++i) gate.v[i] = mul2(gate.v[i], f2(a.branch));
            }
            if (has_post) {
                if (LAYER) st.x = centre(t);
                st.y = inverse(t);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float2 u = mul2(t.v[i], f2(st.y));
                u = LAYER ? fma2(u, post.v[i], post_bias.v[i]) : mul2(u, post.v[i]);
                u = keep2(draws, i, a.drop.last, u);
                h.v[i] = fma2(gate.v[i], u, mul2(h.v[i], f2(a.carry)));
            }
            if (live) store_octet(hp, c, h);
        }
        if (has_pre) {
            if (LAYER) st.z = centre(h);
            st.w = inverse(h);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                h.v[i] = mul2(h.v[i], f2(st.w));
                h.v[i] = LAYER ? fma2(h.v[i], pre.v[i], pre_bias.v[i]) : mul2(h.v[i], pre.v[i]);
            }
            if (live) store_octet(zp, c, h);
        }
        if (lane == 0 && live && a.stats != nullptr && (C == 1 || cluster_rank() == 0)) a.stats[r] = st;
        hp += step * a.ld_h;
        zp += step * a.ld_z;
    }
}

template <class T, int TPR, int C, bool LAYER>
cudaError_t launch_rows(const JoinArgs& a, int num_sms, cudaStream_t stream) {
    constexpr int kBlock = TPR < 256 ? 256 : TPR, kSubs = kBlock / TPR, kStages = 3;
    const int per_sm = TPR <= 256 ? (LAYER ? 3 : 4) : TPR == 512 ? 2 : 1;
    constexpr size_t kSmem = (size_t)kStages * 2 * kPieces<T> * kBlock * 16;
    int64_t grid = (a.rows + kSubs - 1) / kSubs;
    // Past one row each, they step by a multiple of 8 rows (octet.cuh).
    const int64_t cap = (int64_t)num_sms * per_sm / C / 8 * 8;
    if (grid > cap) grid = cap;
    return launch_rows_kernel<C>(join_rows_kernel<T, TPR, C, kStages, LAYER>, grid * C, kBlock, kSmem, stream, a);
}

template <class T, bool LAYER>
cudaError_t launch_octets(const JoinArgs& a, int num_sms, cudaStream_t stream) {
    const int64_t octets = row_octets(a.cols);
    if (octets <= 8) return launch_rows<T, 8, 1, LAYER>(a, num_sms, stream);
    if (octets <= 32) return launch_rows<T, 32, 1, LAYER>(a, num_sms, stream);
    if (octets <= 64) return launch_rows<T, 64, 1, LAYER>(a, num_sms, stream);
    if (octets <= 128) return launch_rows<T, 128, 1, LAYER>(a, num_sms, stream);
    if (octets <= 256) return launch_rows<T, 256, 1, LAYER>(a, num_sms, stream);
    if (octets <= 512) return launch_rows<T, 512, 1, LAYER>(a, num_sms, stream);
    if (octets <= 1024) return launch_rows<T, 512, 2, LAYER>(a, num_sms, stream);
    if (octets <= 2048) return launch_rows<T, 512, 4, LAYER>(a, num_sms, stream);
    return launch_rows<T, 512, 8, LAYER>(a, num_sms, stream);
}

bool in_octets(const JoinArgs& a) {
    return row_octets(a.cols) <= 4096 && octet_matrix(a.x, a.ld_x, a.rows, a.cols) &&
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
