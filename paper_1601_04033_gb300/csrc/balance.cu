// fasgd_balance.  With f[g,e] = counts[g,e] / (top N_g), which `chosen` alone
// fixes, and dot_t = sum_e f[g,e] p_te,
//   balance = cols / G' sum_g 1/N_g sum_t dot_t,   z = 1/N sum_t lse_t^2,
//   dlogits_te = up p_te (s (f[g,e] - dot_t) + 2 z_scale / N lse_t),  s = balance_scale cols / (G' N_g).
// So once the assignments are counted, the losses and the gradient take one pass
// over the logits, and a row leaves two numbers, not cols probabilities, to sum.

#include "octet.cuh"
#include "pdl.cuh"

namespace fasgd {
namespace {

constexpr int kCountThreads = 1024;     // of a block in a cluster; 256 of one alone
constexpr int64_t kCountAlone = 2048, kSplitsAlone = 16;    // entries a block counts alone, blocks of a group that do
constexpr int kCountCluster = 8;        // blocks that count one split together
constexpr int kThreads = 256;

// Adds the assignments of rows r0 .. r1 to `hist`, and the rows that take part to
// `rows_valid`, both in shared memory (integers: no order shows).  U entries a
// thread are asked for before the first is counted.
template <int U>
__device__ __forceinline__ void count_rows(const BalanceArgs& a, int64_t r0, int64_t r1, int32_t* hist,
                                           int32_t* rows_valid) {
    const uint32_t top = (uint32_t)a.top, cols = (uint32_t)a.cols, threads = blockDim.x;
    if (a.valid != nullptr) {
        int32_t v = 0;
        for (int64_t r = r0 + threadIdx.x; r < r1; r += threads) v += a.valid[r] != 0;
        v = __reduce_add_sync(0xffffffffu, v);
        if ((threadIdx.x & 31) == 0 && v != 0) atomicAdd(rows_valid, v);
    }
    const int32_t* chosen = a.chosen + r0 * a.top;
    const uint8_t* valid = a.valid + r0;
    const uint32_t count = (uint32_t)((r1 - r0) * a.top);
    for (uint32_t i = threadIdx.x; i < count; i += threads * U) {
        int32_t e[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t k = i + u * threads;
            e[u] = -1;
            if (k < count) {
                e[u] = chosen[k];
                if (a.valid != nullptr && valid[k / top] == 0) e[u] = -1;
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if ((uint32_t)e[u] < cols) atomicAdd(&hist[e[u]], 1);
    }
}

// Counts of one split of one group's rows: a block's, or (long splits) a cluster's,
// whose blocks add up their counts, a share of the experts each.
__global__ void __launch_bounds__(kCountThreads)
    balance_count_kernel(const __grid_constant__ BalanceArgs a, int blocks) {
    __shared__ int32_t hist[FASGD_EXPERTS_MAX + 1];      // and the rows that take part
    pdl_wait();
    pdl_trigger();
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.ticket = 0;
    const int cols = (int)a.cols, rank = blocks > 1 ? (int)cluster_rank() : 0;
    const int64_t pieces = a.splits * blocks, per = (a.group_rows + pieces - 1) / pieces;
    // Every block of a cluster takes as many turns.
    for (int64_t unit = blockIdx.x / blocks; unit < a.groups * a.splits; unit += gridDim.x / blocks) {
        const int64_t group = unit / a.splits, piece = (unit - group * a.splits) * blocks + rank;
        const int64_t from = piece * per < a.group_rows ? piece * per : a.group_rows;
        const int64_t to = from + per < a.group_rows ? from + per : a.group_rows;
        for (int e = threadIdx.x; e <= cols; e += blockDim.x) hist[e] = 0;
        __syncthreads();
        if (a.valid == nullptr && threadIdx.x == 0) hist[cols] = (int32_t)(to - from);
        count_rows<16>(a, group * a.group_rows + from, group * a.group_rows + to, hist, &hist[cols]);
        __syncthreads();
        int32_t* out = a.splits > 1 ? a.part_counts + unit * cols : a.counts + group * cols;
        if (blocks == 1) {
            for (int e = threadIdx.x; e <= cols; e += blockDim.x)
                *(e < cols ? out + e : a.part_valid + unit) = hist[e];
            __syncthreads();
            continue;
        }
        cluster_barrier();
        for (int e = rank * blockDim.x + threadIdx.x; e <= cols; e += blocks * blockDim.x) {
            int32_t s = 0, v[kCountCluster];
#pragma unroll
            for (int k = 0; k < kCountCluster; ++k) {
                uint32_t there;
                asm volatile("mapa.shared::cluster.u32 %0, %1, %2;"
                             : "=r"(there)
                             : "r"((uint32_t)__cvta_generic_to_shared(&hist[e])), "r"(k));
                asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v[k]) : "r"(there) : "memory");
            }
#pragma unroll
            for (int k = 0; k < kCountCluster; ++k) s += v[k];
            *(e < cols ? out + e : a.part_valid + unit) = s;
        }
        cluster_barrier();       // before a block's counts are cleared, or it ends
    }
}

// Sums of two values over the block, every thread ending with them.
__device__ __forceinline__ float2 block_sum2(float2 v, float2* smem) {
    v.x = warp_sum(v.x);
    v.y = warp_sum(v.y);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) smem[threadIdx.x >> 5] = v;
    __syncthreads();
    v = smem[0];
#pragma unroll
    for (int w = 1; w < kThreads / 32; ++w) v = add2(v, smem[w]);
    return v;
}

// exp(x) for x <= 0, to a few ulp; 0 where it would be subnormal.
__device__ __forceinline__ float exp2_of(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
constexpr float kLog2e = 1.4426950408889634f;

// What every block of the pass knows: N and G' (as floats), and the factors made
// of them.
struct Totals {
    float rows, live, zscale, up;
};
__device__ __forceinline__ Totals totals(const BalanceArgs& a, float2* smem) {
    Totals t;
    t.rows = (float)a.rows;
    t.live = (float)a.groups;
    if (a.valid != nullptr) {
        float n = 0.f, g1 = 0.f;
        for (int64_t g = threadIdx.x; g < a.groups; g += kThreads) {
            int32_t v = 0;
#pragma unroll 4
            for (int64_t s = 0; s < a.splits; ++s) v += a.part_valid[g * a.splits + s];
            n += (float)v;
            g1 += v > 0 ? 1.f : 0.f;
        }
        const float2 s = block_sum2(make_float2(n, g1), smem);
        t.rows = s.x;
        t.live = s.y;
    }
    t.up = a.upstream != nullptr ? *a.upstream : 1.f;
    t.zscale = t.rows > 0.f ? 2.f * a.z_scale / t.rows : 0.f;
    return t;
}
// The group's f = counts / (top N_g) in shared memory (and its counts, where it has
// to add them up and `write` says so); returns 1 / N_g, or 0.
__device__ __forceinline__ float group_shares(const BalanceArgs& a, int64_t group, bool write, float* f) {
    const int cols = (int)a.cols;
    int32_t n = (int32_t)a.group_rows;
    if (a.valid != nullptr) {
        n = 0;
#pragma unroll 4
        for (int64_t s = 0; s < a.splits; ++s) n += a.part_valid[group * a.splits + s];
    }
    const float inv_n = n > 0 ? 1.f / (float)n : 0.f;
    __syncthreads();
    for (int e = threadIdx.x; e < cols; e += kThreads) {
        int32_t c = 0;
        if (a.splits > 1) {
#pragma unroll 8
            for (int64_t s = 0; s < a.splits; ++s) c += a.part_counts[(group * a.splits + s) * cols + e];
            if (write) a.counts[group * cols + e] = c;
        } else {
            c = a.counts[group * cols + e];
        }
        f[e] = (float)c * (inv_n / (float)a.top);
    }
    __syncthreads();
    return inv_n;
}
// The losses of sums over all rows.
__device__ __forceinline__ void store_loss(const BalanceArgs& a, const Totals& t, float dot, float z) {
    const float balance = t.live > 0.f ? (float)a.cols / t.live * dot : 0.f;
    z = t.rows > 0.f ? z / t.rows : 0.f;
    a.loss[0] = a.balance_scale * balance + a.z_scale * z;
    a.loss[1] = balance;
    a.loss[2] = z;
}
// The losses of the blocks' sums: the block that leaves its own last adds them up,
// in the blocks' order.
__device__ __forceinline__ void join_loss(const BalanceArgs& a, const Totals& t, float dot, float z, float2* smem) {
    __shared__ bool last;
    float2 s = block_sum2(make_float2(dot, z), smem);
    if (gridDim.x == 1) {
        if (threadIdx.x == 0) store_loss(a, t, s.x, s.y);
        return;
    }
    if (threadIdx.x == 0) {
        a.part_loss[blockIdx.x] = s;
        uint32_t before;                // releases this sum, acquires the others'
        asm volatile("atom.add.acq_rel.gpu.global.u32 %0, [%1], 1;" : "=r"(before) : "l"(a.ticket) : "memory");
        last = before == gridDim.x - 1;
    }
    __syncthreads();
    if (!last) return;
    s = f2(0.f);
    for (int b = threadIdx.x; b < (int)gridDim.x; b += kThreads) s = add2(s, __ldcg(&a.part_loss[b]));
    s = block_sum2(s, smem);
    if (threadIdx.x == 0) store_loss(a, t, s.x, s.y);
}

// Any width, stride and alignment (and accurate logarithms and quotients, where rows in
// octets have fast ones: 262144 x 256 bf16 131 us, 53).  A unit is `unit_rows` consecutive rows of one
// group; a block takes every gridDim-th unit, a warp a row at a time.
template <class T>
__global__ void __launch_bounds__(kThreads)
    balance_any_kernel(const __grid_constant__ BalanceArgs a, int64_t unit_rows) {
    __shared__ float f[FASGD_EXPERTS_MAX];
    __shared__ float2 smem[kThreads / 32];
    constexpr int kWarps = kThreads / 32;
    pdl_wait();
    pdl_trigger();
    const int cols = (int)a.cols, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const Totals t = totals(a, smem);
    const int64_t units_per_group = (a.group_rows + unit_rows - 1) / unit_rows;
    float sum_dot = 0.f, sum_z = 0.f;
    for (int64_t unit = blockIdx.x; unit < a.groups * units_per_group; unit += gridDim.x) {
        const int64_t group = unit / units_per_group, part = unit - group * units_per_group;
        const float inv_n = group_shares(a, group, part == 0, f);
        const float scale = t.live > 0.f ? a.balance_scale * (float)cols / t.live * inv_n : 0.f;
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
            if (top == -INFINITY) top = 0.f;         // no expert is open to this row: sum = 0 (or NaN)
            float sum = 0.f, dot = 0.f;
            for (int e = lane; e < cols; e += 32) {
                const float p = exp2_of((to_f32(x[e]) - top) * kLog2e);
                sum += p;
                dot += f[e] * p;
            }
            sum = warp_sum(sum);
            dot = warp_sum(dot);
            const float inv = sum == 0.f ? 0.f : 1.f / sum, lse = sum == 0.f ? 0.f : top + logf(sum);
            dot *= inv;
            unit_dot += dot;
            sum_z += lse * lse;
            const float k = t.up * inv, c = t.zscale * lse - scale * dot;
            if (a.dlogits != nullptr)
                for (int e = lane; e < cols; e += 32)
                    d[e] = from_f32<T>(exp2_of((to_f32(x[e]) - top) * kLog2e) * k * fmaf(scale, f[e], c));
        }
        sum_dot += unit_dot * inv_n;
    }
    if (a.loss != nullptr) join_loss(a, t, lane == 0 ? sum_dot : 0.f, lane == 0 ? sum_z : 0.f, smem);
}

// 262144 x 256 bf16, top 8 (277 MB): 53 us, 5.2 TB/s, of which counting two million
// assignments takes 8 and this pass 45 (5.9 TB/s).  The pass: 11 instructions an
// element and too few warps for more (128 registers); shares in shared memory or
// logits through it cost more than the warps they buy (69 and 64 us for all), two
// octets a lane more shuffles (51 for the pass).  The counting: latency of its loads
// and two cluster barriers; neighbours' equal experts matched first, 82 us for all.
// 16 x 2047 x 60: 12.4 us, a chain of latencies.
//
// Rows in octets (octet.cuh): LPR lanes hold a row, NV octets each, from its one
// read to its gradient; 256 / LPR rows a block at a time (a multiple of 8), the
// next ones' logits asked for before this one's are used.  ONE: a single block,
// which counts for itself.
template <class T, int LPR, int NV, bool RAGGED, bool ONE>
__global__ void __launch_bounds__(kThreads, NV > 2 ? 2 : 3)
    balance_rows_kernel(const __grid_constant__ BalanceArgs a, int64_t unit_rows) {
    constexpr int kSlots = kThreads / LPR, kP = kPieces<T>;
    __shared__ __align__(16) float f[FASGD_EXPERTS_MAX];
    __shared__ float2 smem[kThreads / 32];
    const int slot = threadIdx.x / LPR, lane = threadIdx.x % LPR;
    const int32_t cols = (int32_t)a.cols;
    pdl_wait();
    pdl_trigger();
    const int64_t units_per_group = (a.group_rows + unit_rows - 1) / unit_rows;
    // The unit's rows base .. base + rows, and its logits on their way: asked for
    // before the counts that it takes to use them.
    int64_t base = 0;
    int32_t rows = 0;
    Columns c[NV];
    uint4 raw[NV][kP];
    const T* x = nullptr;
    const int64_t step_x = kSlots * a.ld_logits, step_d = kSlots * a.ld_dlogits;
    // The matrix may end inside a last octet: such a one is read value by value.
    const int64_t followed = rows_followed(a.rows, a.cols);
    const auto fetch = [&](int32_t i) {
        if (i < rows) {
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                if (!c[v].any()) continue;
                if (!RAGGED || c[v].c0 + kOctet <= cols || base + i < followed) {
                    load_pieces(x + v * (LPR * kOctet), raw[v]);
                } else {
                    Oct o = {};
#pragma unroll
                    for (int k = 0; k < kOctet; ++k)
                        if (c[v].in >> k & 1) element(o, k) = to_f32(x[v * (LPR * kOctet) + k]);
                    pack<T>(o, raw[v]);
                }
            }
        }
        x += step_x;
    };
    const auto begin = [&](int64_t unit) {
        const int64_t group = unit / units_per_group, part = unit - group * units_per_group;
        base = group * a.group_rows + part * unit_rows;
        rows = (int32_t)(a.group_rows - part * unit_rows < unit_rows ? a.group_rows - part * unit_rows : unit_rows);
        const int shift = RAGGED ? (int)(((base + slot) * a.cols) & 7) : 0;
#pragma unroll
        for (int v = 0; v < NV; ++v) c[v] = Columns(lane + v * LPR, shift, cols);
        x = static_cast<const T*>(a.logits) + (base + slot) * a.ld_logits + c[0].c0;
        fetch(slot);
    };
    begin(blockIdx.x);
    Totals t;
    if constexpr (ONE) {
        int32_t* hist = reinterpret_cast<int32_t*>(f);
        __shared__ int32_t rows_valid;
        for (int e = threadIdx.x; e < cols; e += kThreads) hist[e] = 0;
        if (threadIdx.x == 0) rows_valid = a.valid != nullptr ? 0 : (int32_t)a.rows;
        __syncthreads();
        count_rows<8>(a, 0, a.rows, hist, &rows_valid);
        __syncthreads();
        for (int e = threadIdx.x; e < cols; e += kThreads) {
            const int32_t c = hist[e];
            a.counts[e] = c;
            f[e] = rows_valid > 0 ? (float)c * (1.f / (float)rows_valid / (float)a.top) : 0.f;
        }
        t.rows = (float)rows_valid;
        t.live = rows_valid > 0 ? 1.f : 0.f;
        t.up = a.upstream != nullptr ? *a.upstream : 1.f;
        t.zscale = t.rows > 0.f ? 2.f * a.z_scale / t.rows : 0.f;
        __syncthreads();
    } else {
        t = totals(a, smem);
    }
    float sum_dot = 0.f, sum_z = 0.f;
    for (int64_t unit = blockIdx.x; unit < a.groups * units_per_group; unit += gridDim.x) {
        if (unit != blockIdx.x) begin(unit);
        const int64_t group = unit / units_per_group;
        const float inv_n = ONE ? (t.rows > 0.f ? 1.f / t.rows : 0.f)
                                : group_shares(a, group, unit == group * units_per_group, f);
        const float scale = t.live > 0.f ? a.balance_scale * (float)cols / t.live * inv_n : 0.f;
        Oct share[NV];
        T* d = static_cast<T*>(a.dlogits) + (base + slot) * a.ld_dlogits + c[0].c0;
#pragma unroll
        for (int v = 0; v < NV; ++v) share[v] = load_vector(f, c[v], 0.f);
        float unit_dot = 0.f;
        // A warp goes on until the first of its rows is past the end.
        for (int32_t i = slot, ahead = slot - slot % (32 / LPR); ahead < rows; i += kSlots, ahead += kSlots) {
            Oct e[NV];
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                e[v] = unpack<T>(raw[v]);
                if (RAGGED ? !c[v].whole() : !c[v].any()) {
#pragma unroll
                    for (int k = 0; k < kOctet; ++k)
                        if (!(c[v].in >> k & 1)) element(e[v], k) = -INFINITY;
                }
            }
            const bool live = i < rows && (a.valid == nullptr || a.valid[base + i] != 0);
            fetch(i + kSlots);
            if (!live) {                             // whatever it holds
#pragma unroll
                for (int v = 0; v < NV; ++v) e[v] = Oct{};
            }
            float top = -INFINITY;
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int k = 0; k < 4; ++k) top = fmaxf(top, fmaxf(e[v].v[k].x, e[v].v[k].y));
#pragma unroll
            for (int off = LPR / 2; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
            if (top == -INFINITY) top = 0.f;         // no expert is open to this row: sum = 0 (or NaN)
            float2 s2 = f2(0.f), d2 = f2(0.f);
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const Oct& w = share[v];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    float2& p = e[v].v[k];
                    p = mul2(add2(p, f2(-top)), f2(kLog2e));
                    p = make_float2(exp2_of(p.x), exp2_of(p.y));
                    s2 = add2(s2, p);
                    d2 = fma2(w.v[k], p, d2);
                }
            }
            float sum = s2.x + s2.y, dot = d2.x + d2.y;
#pragma unroll
            for (int off = LPR / 2; off > 0; off >>= 1) {
                sum += __shfl_xor_sync(0xffffffffu, sum, off);
                dot += __shfl_xor_sync(0xffffffffu, dot, off);
            }
            float inv = 0.f, lse = 0.f;
            if (live && sum != 0.f) {
                inv = __fdividef(1.f, sum);
                lse = top + __logf(sum);
            }
            dot *= inv;
            unit_dot += dot;
            sum_z += lse * lse;
            if (a.dlogits != nullptr) {
                const float k = live ? t.up * inv : 0.f;       // (up may be infinite)
                const float k1 = k * scale, k0 = k * (t.zscale * lse - scale * dot);
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    const Oct& w = share[v];
#pragma unroll
                    for (int m = 0; m < 4; ++m) e[v].v[m] = mul2(e[v].v[m], fma2(w.v[m], f2(k1), f2(k0)));
                    if (i < rows) store_octet<T, RAGGED>(d + v * (LPR * kOctet), c[v], e[v]);
                }
                d += step_d;
            }
        }
        sum_dot += unit_dot * inv_n;
    }
    if (a.loss != nullptr) join_loss(a, t, lane == 0 ? sum_dot : 0.f, lane == 0 ? sum_z : 0.f, smem);
}

__global__ void balance_nothing_kernel(const __grid_constant__ BalanceArgs a) {
    pdl_wait();
    pdl_trigger();
    const int64_t stride = (int64_t)gridDim.x * blockDim.x;
    const int64_t t = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    for (int64_t i = t; i < a.groups * a.cols; i += stride) a.counts[i] = 0;
    if (t < 3 && a.loss != nullptr) a.loss[t] = 0.f;
}

// Whether one block does it all, `slots` rows at a time, in one launch: four turns
// of one group, whose assignments it counts in as few.
bool balance_alone(const BalanceArgs& a, int slots) {
    return a.groups == 1 && a.rows <= 4 * slots && a.rows * a.top <= 4 * 8 * kThreads;
}
// `unit_rows` rows of a group to a unit: at most `cap` units where the groups allow it.
int64_t rows_of_units(const BalanceArgs& a, int64_t cap, int64_t multiple) {
    int64_t rows = (a.rows + cap - 1) / cap;
    rows = (rows + multiple - 1) / multiple * multiple;
    return rows < a.group_rows ? rows : a.group_rows;
}
template <class T, int LPR, int NV, bool RAGGED>
cudaError_t launch_rows(const BalanceArgs& a, int num_sms, cudaStream_t stream) {
    constexpr int kSlots = kThreads / LPR;
    if (balance_alone(a, kSlots))
        return launch_pdl(balance_rows_kernel<T, LPR, NV, RAGGED, true>, 1, kThreads, 0, stream, a, a.rows);
    const int64_t cap = (int64_t)num_sms * (NV > 2 ? 2 : 3);      // as many as are resident
    const int64_t unit_rows = rows_of_units(a, cap, kSlots);
    const int64_t units = a.groups * ((a.group_rows + unit_rows - 1) / unit_rows);
    return launch_pdl(balance_rows_kernel<T, LPR, NV, RAGGED, false>, (unsigned)(units < cap ? units : cap), kThreads,
                      0, stream, a, unit_rows);
}
template <class T, bool RAGGED>
cudaError_t launch_octets(const BalanceArgs& a, int64_t octets, int num_sms, cudaStream_t stream) {
    if (octets <= 1) return launch_rows<T, 1, 1, RAGGED>(a, num_sms, stream);
    if (octets <= 4) return launch_rows<T, 1, 4, RAGGED>(a, num_sms, stream);
    if (octets <= 8) return launch_rows<T, 2, 4, RAGGED>(a, num_sms, stream);
    if (octets <= 16) return launch_rows<T, 4, 4, RAGGED>(a, num_sms, stream);
    if (octets <= 32) return launch_rows<T, 8, 4, RAGGED>(a, num_sms, stream);
    if (octets <= 64) return launch_rows<T, 16, 4, RAGGED>(a, num_sms, stream);
    return launch_rows<T, 32, 4, RAGGED>(a, num_sms, stream);
}
constexpr int64_t kOctetsMost = 128;

int lanes_per_row(int64_t octets) {
    int lanes = 1;
    while (lanes * 4 < octets && lanes < 32) lanes *= 2;
    return lanes;
}
bool in_octets(const BalanceArgs& a, int size) {
    return row_octets(a.cols) <= kOctetsMost && octet_matrix(a.logits, a.ld_logits, a.rows, a.cols, size) &&
           octet_matrix(a.dlogits, a.ld_dlogits, a.rows, a.cols, size);
}

template <class T>
cudaError_t launch(const BalanceArgs& a, int num_sms, cudaStream_t stream) {
    const int64_t octets = row_octets(a.cols);
    const bool fast = in_octets(a, (int)sizeof(T));
    if (!(fast && balance_alone(a, kThreads / lanes_per_row(octets)))) {
        const bool cluster = a.group_rows * a.top > kCountAlone * kSplitsAlone;
        const int blocks = cluster ? kCountCluster : 1;
        const int64_t units = a.groups * a.splits, cap = (int64_t)num_sms * (cluster ? 2 : 8) / blocks;
        const cudaError_t st = launch_rows_kernel<balance_count_kernel>(
            (units < cap ? units : cap) * blocks, cluster ? kCountThreads : 256, 0, blocks, stream, a, blocks);
        if (st != cudaSuccess) return st;
    }
    if (fast)
        return a.cols % kOctet != 0 ? launch_octets<T, true>(a, octets, num_sms, stream)
                                    : launch_octets<T, false>(a, octets, num_sms, stream);
    const int64_t cap = (int64_t)num_sms * 8 < kBalanceParts ? (int64_t)num_sms * 8 : kBalanceParts;
    const int64_t unit_rows = rows_of_units(a, cap, 8);
    const int64_t units = a.groups * ((a.group_rows + unit_rows - 1) / unit_rows);
    return launch_pdl(balance_any_kernel<T>, (unsigned)(units < cap ? units : cap), kThreads, 0, stream, a,
                      unit_rows);
}

}  // namespace

// Splits of each group in the counting (every block of the pass adds up its
// group's): up to 16 blocks of 1,024 assignments or more; past 32,768 a cluster of
// eight blocks for each 65,536, 19 at most (they fill 152 SMs).
int64_t balance_splits(int64_t rows, int64_t groups, int64_t top) {
    if (groups < 1) return 1;
    const int64_t n = rows / groups * top;
    int64_t s = (n + 1023) / 1024;
    if (n > kCountAlone * kSplitsAlone) {
        s = (n + 65535) / 65536;
        return s > 19 ? 19 : s;
    }
    return s < 1 ? 1 : s > kSplitsAlone ? kSplitsAlone : s;
}

cudaError_t launch_balance(const BalanceArgs& a, int dtype, int num_sms, cudaStream_t stream) {
    if (a.rows == 0) return launch_pdl(balance_nothing_kernel, 32, kThreads, 0, stream, a);
    if (dtype == FASGD_F32) return launch<float>(a, num_sms, stream);
    if (dtype == FASGD_BF16) return launch<__nv_bfloat16>(a, num_sms, stream);
    return launch<__half>(a, num_sms, stream);
}

}  // namespace fasgd
