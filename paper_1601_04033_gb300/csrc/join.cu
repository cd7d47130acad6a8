// fasgd_join: t = N(y), u = dropout(t), h = carry x + branch gate u, z = N(h).

#include "join.cuh"
#include "octet.cuh"
#include "pdl.cuh"

namespace fasgd {
namespace {

constexpr int kThreads = 256;

// Rows too wide for the rest: a block takes a row at a time and reads it again for
// every statistic (out of L2, where a row fits).
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

// Rows in octets (octet.cuh): a row's threads hold it between its statistics, an
// octet each, so x and y are read once; blocks stay and take NR rows at a time, so
// that two rows share each barrier, the next STAGES - 1 turns' on their way into
// shared memory.
//
// 8 bytes an element (16-bit types), about 33 instructions with dropout, 20 without.
// 32768 x 4096 bf16 with dropout: 181 us, 5.9 TB/s, where the issue of the draws and
// the latency of two reductions a row bound it; 32768 x 2048 without: 82 us, 6.6 TB/s,
// memory.  Layer norms take four reductions: 32768 x 4096 with dropout 262 us.
// Joining the warps' moments (Chan) in one barrier instead of two costs more
// arithmetic than the barrier (143 -> 193 us at 32768 x 2048).  One row a turn at
// 64 registers and twice the blocks: 246 us against 210 for the kernel of that time.
// From one of a block's rows to the next: bytes in each matrix, octets of draws.
struct RowSteps {
    int64_t rows, x, y, h, z, octets;
    bool vectors;        // h and z can be written in octets
};
constexpr int kForwardStages = 3;
constexpr int kForwardThreads = 512;      // of an SM
// FULL: with y and both norms.
// LOOSE (RAGGED too): matrices of any alignment and step.
template <class T, int TPR, int NR, bool LAYER, bool RAGGED, bool DROP, bool FULL, bool LOOSE>
__global__ void __launch_bounds__(TPR == 8 ? 32 : NR == 1 ? 1024 : 512, TPR == 8 ? 16 : 1)
    join_rows_kernel(const __grid_constant__ JoinArgs a, const __grid_constant__ RowSteps s, int blocks) {
    constexpr int kP = kPieces<T>, STAGES = kForwardStages;
    extern __shared__ uint4 ring[];                  // [STAGES][warp][NR][x, y][kP][lane]
    __shared__ __align__(16) float red[RowSums<TPR, NR>::kPlaces];
    const RowThreads<TPR> th(blocks);
    constexpr int kRows = TPR == 8 ? kWarpRows : 1;
    const int64_t step = s.rows, ahead = (int64_t)(blockIdx.x / blocks) * kRows;
    const int64_t first = ahead + th.sub;
    // Rows first, first + step, ...: `rows` of them, in `turns` turns (a warp's as many).
    const int64_t rows = first < a.rows ? (a.rows - first + step - 1) / step : 0;
    const int64_t turns = ahead < a.rows ? ((a.rows - ahead + step - 1) / step + NR - 1) / NR : 0;
    const Columns c(th.octet(), RAGGED ? (int)((first * a.cols) & 7) : 0, (int32_t)a.cols);
    RowSums<TPR, NR> sums(th, red);
    const bool has_y = FULL || a.y != nullptr, has_pre = FULL || a.pre != nullptr, has_post = FULL || a.post != nullptr;
    constexpr int kPlace = LOOSE ? LooseRow<T>::kPlace : kP * kLane;
    constexpr int kSlots = 2 * NR * kPlace;          // of a warp's stage
    uint4* const mine = ring + (threadIdx.x >> 5) * kSlots;
    const int stage_size = kSlots * th.warps;
    if (!LOOSE && !c.any())
        for (int i = 0; i < STAGES; ++i) clear_octets<T>(mine + i * stage_size, 2 * NR);
    __syncwarp();
    pdl_wait();
    pdl_trigger();

    const CopyLane<T, TPR == 8 ? 8 : 32> lane(c, (int32_t)a.cols);
    const LooseRow<T> loose(c, (int32_t)a.cols);
    const T* x = static_cast<const T*>(a.x) + first * a.ld_x + (LOOSE ? 0 : lane.col);      // of the next row to fetch
    const T* y = static_cast<const T*>(a.y) + first * a.ld_y + (LOOSE ? 0 : lane.col);
    // Where the next row to take begins (LOOSE; the low bits of the address).
    uint32_t start_x = (uint32_t)reinterpret_cast<uintptr_t>(x + loose.col_lo);
    uint32_t start_y = (uint32_t)reinterpret_cast<uintptr_t>(y + loose.col_lo);
    int64_t unfetched = rows;
    const int32_t last_behind = RAGGED ? values_behind(a.rows, a.cols, first + (rows - 1) * step) : -1;
    const auto fetch = [&](uint4* slot) {
#pragma unroll
        for (int j = 0; j < NR; ++j) {
            if (LOOSE && unfetched > 0) {
                loose.copy(slot + 2 * j * kPlace, x, a.x);
                if (has_y) loose.copy(slot + (2 * j + 1) * kPlace, y, a.y);
            } else if (unfetched > 0) {
                const int32_t behind = RAGGED && unfetched == 1 ? last_behind : -1;
                lane.copy(slot + 2 * j * kPlace, x, behind);
                if (has_y) lane.copy(slot + (2 * j + 1) * kPlace, y, behind);
            }
            --unfetched;
            x = on(x, s.x);
            y = on(y, s.y);
        }
        copy_commit();
    };
#pragma unroll
    for (int k = 0; k < STAGES - 1; ++k) fetch(mine + k * stage_size);

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
        if (DROP) post.v[i] = mul2(post.v[i], f2(a.drop.scale));
        if (DROP && LAYER) post_bias.v[i] = mul2(post_bias.v[i], f2(a.drop.scale));
        if (!gates) gate.v[i] = mul2(gate.v[i], f2(a.branch));
    }
    T* hp = static_cast<T*>(a.h) + first * a.ld_h + c.c0;
    T* zp = static_cast<T*>(a.z) + first * a.ld_z + c.c0;

    const auto centre = [&](Oct (&o)[NR], float (&mean)[NR]) {      // the rows' means, taken off
        float v[NR];
#pragma unroll
        for (int j = 0; j < NR; ++j) {
            const float2 p = add2(add2(o[j].v[0], o[j].v[1]), add2(o[j].v[2], o[j].v[3]));
            v[j] = p.x + p.y;
        }
        sums(v);
#pragma unroll
        for (int j = 0; j < NR; ++j) {
            mean[j] = v[j] * a.inv_cols;
#pragma unroll
            for (int i = 0; i < 4; ++i) o[j].v[i] = add2(o[j].v[i], f2(-mean[j]));
            if (RAGGED) mask(o[j], c);           // 0 where there is no column
        }
    };
    const auto inverse = [&](const Oct (&o)[NR], float (&rstd)[NR]) {
        float v[NR];
#pragma unroll
        for (int j = 0; j < NR; ++j) {
            const float2 p = fma2(o[j].v[0], o[j].v[0], mul2(o[j].v[1], o[j].v[1]));
            const float2 q = fma2(o[j].v[2], o[j].v[2], mul2(o[j].v[3], o[j].v[3]));
            v[j] = (p.x + q.x) + (p.y + q.y);
            if (LAYER && !RAGGED && !c.any()) v[j] = 0.f;      // (a mean was taken off)
        }
        sums(v);
#pragma unroll
        for (int j = 0; j < NR; ++j) rstd[j] = rsqrtf(fmaf(v[j], a.inv_cols, a.eps));
    };

    int64_t q = (first * a.cols + c.c0) >> 3;         // the row's octet of draws
    int stage = 0;
    for (int64_t turn = 0, left = rows; turn < turns; ++turn, left -= NR) {
        copy_wait<STAGES - 2>();
        __syncwarp();
        const uint4* slot = mine + stage * stage_size;
        Oct h[NR], t[NR];
#pragma unroll
        for (int j = 0; j < NR; ++j) {
            if constexpr (LOOSE) {
                h[j] = loose.take(slot + 2 * j * kPlace, start_x, c);
                if (has_y) t[j] = loose.take(slot + (2 * j + 1) * kPlace, start_y, c);
                start_x += (uint32_t)s.x;
                start_y += (uint32_t)s.y;
            } else {
                h[j] = take_octet<T, RAGGED>(slot + 2 * j * kPlace, c);
                if (has_y) t[j] = take_octet<T, RAGGED>(slot + (2 * j + 1) * kPlace, c);
            }
        }
        fetch(mine + (stage == 0 ? STAGES - 1 : stage - 1) * stage_size);
        stage = stage == STAGES - 1 ? 0 : stage + 1;
        float mean_y[NR], rstd_y[NR], mean_h[NR], rstd_h[NR];
#pragma unroll
        for (int j = 0; j < NR; ++j) {
            mean_y[j] = mean_h[j] = 0.f;
            rstd_y[j] = rstd_h[j] = 1.f;
        }
        if (has_y) {
            Philox4 draws[NR];
#pragma unroll
            for (int j = 0; j < NR; ++j)
                if (DROP) draws[j] = draw_octet(a.drop, q + j * s.octets);
            if (has_post) {
                if (LAYER) centre(t, mean_y);
                inverse(t, rstd_y);
            }
#pragma unroll
            for (int j = 0; j < NR; ++j) {
                if (gates) {
                    const int64_t r = first + (turn * NR + j) * step;
                    gate = load_gate<T>(a, (left > j ? r : 0) / a.group_rows, c);
#pragma unroll
                    for (int i = 0; i < 4; ++i) gate.v[i] = mul2(gate.v[i], f2(a.branch));
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float2 u = mul2(t[j].v[i], f2(rstd_y[j]));
                    u = LAYER ? fma2(u, post.v[i], post_bias.v[i]) : mul2(u, post.v[i]);
                    if (DROP) u = keep2(draws[j], i, a.drop.last, u);
                    h[j].v[i] = fma2(gate.v[i], u, mul2(h[j].v[i], f2(a.carry)));
                }
                if (left > j) store_octet<T, RAGGED>(hp, c, h[j], !LOOSE || s.vectors);
                hp = on(hp, s.h);
            }
        }
        if (has_pre) {
            if (LAYER) centre(h, mean_h);
            inverse(h, rstd_h);
#pragma unroll
            for (int j = 0; j < NR; ++j) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    h[j].v[i] = mul2(h[j].v[i], f2(rstd_h[j]));
                    h[j].v[i] = LAYER ? fma2(h[j].v[i], pre.v[i], pre_bias.v[i]) : mul2(h[j].v[i], pre.v[i]);
                }
                if (left > j) store_octet<T, RAGGED>(zp, c, h[j], !LOOSE || s.vectors);
                zp = on(zp, s.z);
            }
        }
        if (th.octet() == 0 && a.stats != nullptr) {
#pragma unroll
            for (int j = 0; j < NR; ++j)
                if (left > j)
                    a.stats[first + (turn * NR + j) * step] = make_float4(mean_y[j], rstd_y[j], mean_h[j], rstd_h[j]);
        }
        q += NR * s.octets;
    }
}

template <class T, int TPR, int NR, bool LAYER, bool RAGGED, bool DROP, bool FULL, bool LOOSE>
cudaError_t launch_rows(const JoinArgs& a, const RowShape& s, int num_sms, cudaStream_t stream) {
    const size_t place = LOOSE ? LooseRow<T>::kPlace : kPieces<T> * kLane;
    const size_t smem = (size_t)kForwardStages * 2 * NR * place * (s.threads / 32) * 16;
    int64_t grid = (a.rows + s.rows - 1) / s.rows;
    // Past one row each, they step by a multiple of 8 rows (octet.cuh).
    const int64_t cap = (int64_t)num_sms * (NR == 1 ? 1 : kForwardThreads / s.threads) / s.blocks / 8 * 8;
    if (grid > cap) grid = cap;
    const int64_t rows = grid * s.rows, bytes = rows * (int64_t)sizeof(T);
    const RowSteps steps = {rows, bytes * a.ld_x, bytes * a.ld_y, bytes * a.ld_h, bytes * a.ld_z, rows * a.cols / 8,
                            octet_matrix(a.h, a.ld_h, a.rows, a.cols, sizeof(T)) && octet_matrix(a.z, a.ld_z, a.rows, a.cols, sizeof(T))};
    return launch_rows_kernel<join_rows_kernel<T, TPR, NR, LAYER, RAGGED, DROP, FULL, LOOSE>>(
        grid * s.blocks, s.threads, smem, s.blocks, stream, a, steps, s.blocks);
}
template <class T, bool LAYER, bool RAGGED, bool DROP>
cudaError_t launch_octets(const JoinArgs& a, const RowShape& s, int num_sms, cudaStream_t stream) {
    if (s.rows > 1) return launch_rows<T, 8, 2, LAYER, RAGGED, DROP, false, false>(a, s, num_sms, stream);
    // Two rows a turn, but where a row takes more threads than have the registers for it.
    if (s.threads > 512) return launch_rows<T, 0, 1, LAYER, RAGGED, DROP, false, false>(a, s, num_sms, stream);
    // FULL where it gains (32768 x 4096 bf16 with dropout 181 us, 210 without it) and
    // not where it costs (32768 x 2048 rms norm, nothing dropped: 91 us, 82 without it).
    if constexpr (LAYER || DROP)
        if (a.y != nullptr && a.post != nullptr && a.pre != nullptr)
            return launch_rows<T, 0, 2, LAYER, RAGGED, DROP, true, false>(a, s, num_sms, stream);
    return launch_rows<T, 0, 2, LAYER, RAGGED, DROP, false, false>(a, s, num_sms, stream);
}
template <class T, bool LAYER, bool DROP>
cudaError_t launch_loose(const JoinArgs& a, const RowShape& s, int num_sms, cudaStream_t stream) {
    if (s.threads > 512) return launch_rows<T, 0, 1, LAYER, true, DROP, false, true>(a, s, num_sms, stream);
    return launch_rows<T, 0, 2, LAYER, true, DROP, false, true>(a, s, num_sms, stream);
}
template <class T, bool LAYER>
cudaError_t launch_octets(const JoinArgs& a, const RowShape& s, bool loose, int num_sms, cudaStream_t stream) {
    const bool drop = a.drop.cut != 0;
    if (loose)
        return drop ? launch_loose<T, LAYER, true>(a, s, num_sms, stream) : launch_loose<T, LAYER, false>(a, s, num_sms, stream);
    if (a.cols % 8 == 0)
        return drop ? launch_octets<T, LAYER, false, true>(a, s, num_sms, stream)
                    : launch_octets<T, LAYER, false, false>(a, s, num_sms, stream);
    return drop ? launch_octets<T, LAYER, true, true>(a, s, num_sms, stream)
                : launch_octets<T, LAYER, true, false>(a, s, num_sms, stream);
}

bool in_octets(const JoinArgs& a, int size) {
    const void* p[] = {a.x, a.y, a.h, a.z};
    const int64_t ld[] = {a.ld_x, a.ld_y, a.ld_h, a.ld_z};
    for (int i = 0; i < 4; ++i)
        if (!octet_matrix(p[i], ld[i], a.rows, a.cols, size)) return false;
    return true;
}

template <class T>
cudaError_t launch(const JoinArgs& a, int num_sms, cudaStream_t stream) {
    // One block where 1,024 threads will do (16384 x 8192 bf16: 291 us; a cluster of two: 376).
    const int64_t octets = row_octets(a.cols);
    const bool loose = !in_octets(a, (int)sizeof(T));
    const RowShape s(octets, octets <= 1024 ? 1024 : 512, loose);
    if (s.fits())
        return a.layer ? launch_octets<T, true>(a, s, loose, num_sms, stream)
                       : launch_octets<T, false>(a, s, loose, num_sms, stream);
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
