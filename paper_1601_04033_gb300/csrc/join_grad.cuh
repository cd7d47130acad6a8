// fasgd_join_grad.  With hats the normalised values and r the 1/sqrt of a row,
//   q  = dz pre,  dH = dh + r_h (q - mean q - hhat mean(q hhat))   (rms: no mean q)
//   dx = carry dH,  dgate += branch dH u,  dt = m scale branch gate dH
//   q2 = dt post,  dy = r_y (q2 - mean q2 - yhat mean(q2 yhat))
//   dpre += dz hhat, dpre_bias += dz, dpost += dt yhat, dpost_bias += dt.
// hhat comes from h formed again out of x and y, which costs the bytes that
// reading h would and keeps h's rounding out of the parameters' gradients.

#pragma once

#include "join.cuh"
#include "octet.cuh"
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
            const float dt = p.b.keep ? a.branch * gate * a.drop.scale * d : 0.f * d;
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
                const float dt = p.b.keep ? a.branch * gate * a.drop.scale * d : 0.f * d;
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
        float s[5] = {0.f, 0.f, 0.f, 0.f, 0.f};
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
                    const float dt = p.b.keep ? a.branch * gate * a.drop.scale * d : 0.f * d;
                    s[0] += dt * p.b.yhat;
                    s[1] += dt;
                }
                s[2] += p.dz * p.hhat;
                s[3] += p.dz;
            }
            s[4] += g;
            if (a.out_gate == nullptr || a.groups == 1) continue;
            if (a.splits > 1)
                a.gates[unit * a.cols + c] = g;
            else
                store_gate<T>(a, group * a.cols + c, g);
        }
#pragma unroll
        for (int k = 0; k < 5; ++k)
            if (k < 4 ? a.out_param[k] != nullptr : a.out_gate != nullptr && a.groups == 1) a.params[(part * 5 + k) * a.cols + c] = s[k];
    }
}

// The gate's gradients that grad_finish_kernel has to write: a unit that is a
// whole group has written its own.  A single gate is the fifth of the vectors.
__host__ __device__ __forceinline__ int64_t gates_left(const JoinArgs& a) {
    return a.out_gate != nullptr && a.groups > 1 && (a.splits > 1 || a.rows == 0) ? a.groups : 0;
}

// Rows in octets.  A row's threads hold an octet of it each; every thread keeps its
// columns' sums over the rows it takes in registers.  Under rms norms one reduction
// a row is enough: with e = m scale branch gate post (so q2 = e dH) and w = dh + r_h q,
//   sum q2 yhat = S(e yhat w) - r_h mean(q hhat) S(e yhat hhat),
// sums of what is known before mean(q hhat) is.  Under layer norms that takes
// eight sums, whose registers cost more than a second reduction of two
// (32768 x 4096 bf16, when chosen: 510 us, 450).  Units as in the plain form, for the threads of
// one row ("sub") at a time; where cols is no multiple of 8 a unit's rows agree
// modulo 8 (octet.cuh).
//
// It moves 12 bytes an element (16-bit types) and issues about 50 instructions for
// each, a fifth of them the draws: instructions bound it, not memory.  32768 x 4096
// bf16 with dropout: 281 us, 5.7 TB/s; without 5.3 to 6.3 TB/s.  Layer norm with
// dropout 381 us, 4.2 TB/s, and fp32 3.8 to 4.1 TB/s wait for shared memory (short
// scoreboard; fp32 for its copies and the memory pipe too).  512 threads an SM of 128
// registers hold the vectors and sums of 4,096 columns; wider rows take a cluster,
// whose barrier for every row shows: 16384 x 8192 543 us, 3.0 TB/s.
struct Unit {
    int64_t row, step, rows;     // first row, from row to row, one past the last
    __device__ Unit(const JoinArgs& a, int64_t unit) {
        if (a.groups == 1) {
            row = unit;
            rows = a.rows;
        } else {
            const int64_t group = unit / a.splits, start = group * a.group_rows;
            int64_t at = unit - group * a.splits;
            if (a.cols & 7) at = (at & ~(int64_t)7) + ((at - start) & 7);
            row = start + at;
            rows = start + a.group_rows;
        }
        step = a.splits;
    }
};

// From one of a unit's rows to the next: bytes in each matrix, octets of draws.
struct GradSteps {
    int64_t x, y, dh, dz, dx, dy, stats, octets;
    bool vectors;        // dx and dy can be written in octets
};
template <class T, bool LAYER>
constexpr int kGradStages = sizeof(T) == 2 ? 4 : LAYER ? 2 : 3;
// Vectors held in shared memory: what fits beside the ring of 512 threads.
template <class T, bool LAYER>
constexpr int kHeld = LAYER ? 3 : 0;
__device__ __forceinline__ void hold_octet(float4* p, const Oct& o) {
    p[0] = make_float4(o.v[0].x, o.v[0].y, o.v[1].x, o.v[1].y);
    p[kLane] = make_float4(o.v[2].x, o.v[2].y, o.v[3].x, o.v[3].y);
}
__device__ __forceinline__ Oct held_octet(const float4* p) {
    const float4 x = p[0], y = p[kLane];
    Oct o;
    o.v[0] = make_float2(x.x, x.y);
    o.v[1] = make_float2(x.z, x.w);
    o.v[2] = make_float2(y.x, y.y);
    o.v[3] = make_float2(y.z, y.w);
    return o;
}
// FULL: with y, both norms and dh, and one ld for what is read, one for what is written.
// LOOSE (RAGGED too): matrices of any alignment and step.
template <class T, int TPR, bool LAYER, bool RAGGED, bool DROP, bool FULL, bool LOOSE>
__global__ void __launch_bounds__(TPR == 8 ? 32 : 512, TPR == 8 ? 16 : 1)
    grad_rows_kernel(const __grid_constant__ JoinArgs a, const __grid_constant__ GradSteps s, int blocks) {
    constexpr int kP = kPieces<T>, kSums = LAYER ? 2 : 3, STAGES = kGradStages<T, LAYER>;
    extern __shared__ uint4 ring[];                  // [STAGES][warp][x, y, dh, dz][kP][lane], then [STAGES][warp][row of a warp]
    __shared__ __align__(16) float red[RowSums<TPR, kSums>::kPlaces];
    const RowThreads<TPR> th(blocks);
    constexpr int kRows = TPR == 8 ? kWarpRows : 1;
    const int width = blockDim.x;
    const int64_t units = a.groups * a.splits, subs = (int64_t)(gridDim.x / blocks) * kRows;
    const int64_t ahead = (int64_t)(blockIdx.x / blocks) * kRows, mine = ahead + th.sub;
    const bool has_y = FULL || a.y != nullptr, has_pre = FULL || a.pre != nullptr, has_post = FULL || a.post != nullptr;
    const bool has_dh = FULL || a.dh != nullptr, gates = a.groups > 1;
    RowSums<TPR, kSums> sums(th, red);
    // All rows that this sub takes begin at the same place in an octet.
    const Columns c(th.octet(), RAGGED && mine < units ? (int)((Unit(a, mine).row * a.cols) & 7) : 0,
                    (int32_t)a.cols);
    constexpr int kPlace = LOOSE ? LooseRow<T>::kPlace : kP * kLane;
    constexpr int kSlots = 4 * kPlace;               // of a warp's stage
    uint4* const own = ring + (threadIdx.x >> 5) * kSlots;
    const int stage_size = kSlots * th.warps;
    // The rows' statistics, copied ahead by one lane of theirs in each warp.
    uint4* const own_stats = ring + STAGES * stage_size + (threadIdx.x >> 5) * kWarpRows + (TPR == 8 ? th.sub : 0);
    const bool asks = (threadIdx.x & (TPR == 8 ? 7 : 31)) == 0;
    if (!LOOSE && !c.any())
        for (int i = 0; i < STAGES; ++i) clear_octets<T>(own + i * stage_size, 4);
    __syncwarp();
    const CopyLane<T, TPR == 8 ? 8 : 32> lane(c, (int32_t)a.cols);
    const LooseRow<T> loose(c, (int32_t)a.cols);
    pdl_wait();
    pdl_trigger();

    const float scale = a.drop.scale;
    // As the forward kernel has them, so that h comes out in the same bits.
    Oct post = load_vector(a.post, c, 1.f), pre = load_vector(a.pre, c, 0.f), post_bias, gate;
    if (LAYER) post_bias = load_vector(a.post_bias, c, 0.f);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (DROP) post.v[i] = mul2(post.v[i], f2(scale));
        if (DROP && LAYER) post_bias.v[i] = mul2(post_bias.v[i], f2(scale));
    }
    // With both biases the registers do not hold everything: these lie in shared
    // memory (a place of each lane's own, as the ring's).  Before a third stage of
    // fp32 rows, too: 16384 x 4096, when chosen, 430 us, 577 with the stage and spills.
    float4* const vectors = reinterpret_cast<float4*>(ring + STAGES * (stage_size + kWarpRows * th.warps)) +
                            (threadIdx.x >> 5) * (kHeld<T, LAYER> * 2 * kLane) + (threadIdx.x & 31);
    if (kHeld<T, LAYER> > 0) hold_octet(vectors, pre);
    if (kHeld<T, LAYER> > 1) hold_octet(vectors + 2 * kLane, post_bias);
    if (kHeld<T, LAYER> > 2) hold_octet(vectors + 4 * kLane, post);
    // Sums over the rows: those of the norm after the block without `scale`, the
    // gate's without `branch`.
    Oct d_post = {}, d_post_bias = {}, d_gate = {}, d_pre = {}, d_pre_bias = {};

    // Where a warp holds several rows, it goes on until the first of them is done.
    for (int64_t ahead_unit = ahead; ahead_unit < units; ahead_unit += subs) {
        const int64_t unit = ahead_unit + th.sub;
        Unit u(a, unit < units ? unit : 0);
        if (unit >= units) u.rows = 0;
        int32_t turns = u.row < u.rows ? (int32_t)((u.rows - u.row + u.step - 1) / u.step) : 0;
        const int32_t rows = turns;
        if constexpr (TPR == 8) {
#pragma unroll
            for (int off = 16; off >= 8; off >>= 1) {
                const int32_t other = __shfl_xor_sync(0xffffffffu, turns, off);
                turns = other > turns ? other : turns;
            }
        }
        if (gates || unit == mine) {
            gate = load_gate<T>(a, gates && unit < units ? unit / a.splits : 0, c);
#pragma unroll
            for (int i = 0; i < 4; ++i) gate.v[i] = mul2(gate.v[i], f2(a.branch));
        }
        if (gates) d_gate = Oct{};

        const int64_t r0 = u.row;
        const int32_t col = LOOSE ? 0 : lane.col;
        const T* x = static_cast<const T*>(a.x) + r0 * a.ld_x + col;            // of the next row to fetch
        const T* y = static_cast<const T*>(a.y) + r0 * a.ld_y + col;
        const T* dh = static_cast<const T*>(a.dh) + r0 * a.ld_dh + col;
        const T* dz = static_cast<const T*>(a.dz) + r0 * a.ld_dz + col;
        // Where the next row to take begins (LOOSE; the low bits of the address).
        uint32_t start[4] = {(uint32_t)reinterpret_cast<uintptr_t>(x + loose.col_lo),
                             (uint32_t)reinterpret_cast<uintptr_t>(y + loose.col_lo),
                             (uint32_t)reinterpret_cast<uintptr_t>(dh + loose.col_lo),
                             (uint32_t)reinterpret_cast<uintptr_t>(dz + loose.col_lo)};
        const float4* stats = a.stats + r0;
        // FULL: bytes into the matrices instead, which frees ten registers.
        int64_t in = (r0 * a.ld_x + lane.col) * (int64_t)sizeof(T), out = (r0 * a.ld_dx + c.c0) * (int64_t)sizeof(T);
        int32_t unfetched = rows;
        const int32_t last_behind = RAGGED ? values_behind(a.rows, a.cols, r0 + (rows - 1) * u.step) : -1;
        const auto fetch = [&](int stage) {
            uint4* slot = own + stage * stage_size;
            if (unfetched > 0) {
                const int32_t behind = RAGGED && unfetched == 1 ? last_behind : -1;
                if (asks) copy_async16(own_stats + stage * kWarpRows * th.warps, stats, 16);
                if constexpr (LOOSE) {
                    loose.copy(slot, x, a.x);
                    if (has_y) loose.copy(slot + kPlace, y, a.y);
                    if (has_dh) loose.copy(slot + 2 * kPlace, dh, a.dh);
                    if (has_pre) loose.copy(slot + 3 * kPlace, dz, a.dz);
                } else {
                    lane.copy(slot, FULL ? on(static_cast<const T*>(a.x), in) : x, behind);
                    if (has_y) lane.copy(slot + kP * kLane, FULL ? on(static_cast<const T*>(a.y), in) : y, behind);
                    if (has_dh) lane.copy(slot + 2 * kP * kLane, FULL ? on(static_cast<const T*>(a.dh), in) : dh, behind);
                    if (has_pre) lane.copy(slot + 3 * kP * kLane, FULL ? on(static_cast<const T*>(a.dz), in) : dz, behind);
                }
            }
            copy_commit();
            --unfetched;
            if (FULL) {
                in += s.x;
            } else {
                x = on(x, s.x);
                y = on(y, s.y);
                dh = on(dh, s.dh);
                dz = on(dz, s.dz);
            }
            stats = on(stats, s.stats);
        };
#pragma unroll
        for (int k = 0; k < STAGES - 1; ++k) fetch(k);
        T* dxp = static_cast<T*>(a.dx) + r0 * a.ld_dx + c.c0;
        T* dyp = static_cast<T*>(a.dy) + r0 * a.ld_dy + c.c0;
        int64_t oct = (r0 * a.cols + c.c0) >> 3;         // the row's octet of draws
        int stage = 0;
        for (int32_t turn = 0; turn < turns; ++turn) {
            const bool live = TPR != 8 || turn < rows;
            Philox4 draws;
            if (DROP) draws = draw_octet(a.drop, oct);
            oct += s.octets;
            copy_wait<STAGES - 2>();
            __syncwarp();
            float4 st = *reinterpret_cast<const float4*>(own_stats + stage * kWarpRows * th.warps);
            const uint4* slot = own + stage * stage_size;
            Oct hhat, yhat = {}, w = {}, q = {}, e, uu;
            if constexpr (LOOSE) {
                hhat = loose.take(slot, start[0], c);
                if (has_y) yhat = loose.take(slot + kPlace, start[1], c);
                if (has_dh) w = loose.take(slot + 2 * kPlace, start[2], c);
                if (has_pre) q = loose.take(slot + 3 * kPlace, start[3], c);
                start[0] += (uint32_t)s.x;
                start[1] += (uint32_t)s.y;
                start[2] += (uint32_t)s.dh;
                start[3] += (uint32_t)s.dz;
            } else {
                hhat = take_octet<T, RAGGED>(slot, c);
                if (has_y) yhat = take_octet<T, RAGGED>(slot + kP * kLane, c);
                if (has_dh) w = take_octet<T, RAGGED>(slot + 2 * kP * kLane, c);
                if (has_pre) q = take_octet<T, RAGGED>(slot + 3 * kP * kLane, c);
            }
            fetch(stage == 0 ? STAGES - 1 : stage - 1);
            stage = stage == STAGES - 1 ? 0 : stage + 1;
            if (!live) {         // a row past the end: nobody copied its statistics either
                hhat = yhat = w = q = Oct{};
                st = make_float4(0.f, 0.f, 0.f, 0.f);
            }
            if (kHeld<T, LAYER> > 1) post_bias = held_octet(vectors + 2 * kLane);
            if (kHeld<T, LAYER> > 2) post = held_octet(vectors + 4 * kLane);
            // u; e = what dH is multiplied by in dt / scale.
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (LAYER) yhat.v[i] = add2(yhat.v[i], f2(-st.x));
                yhat.v[i] = mul2(yhat.v[i], f2(st.y));
                uu.v[i] = LAYER ? fma2(yhat.v[i], post.v[i], post_bias.v[i]) : mul2(yhat.v[i], post.v[i]);
                e.v[i] = gate.v[i];
                if (DROP) {
                    uu.v[i] = keep2(draws, i, a.drop.last, uu.v[i]);
                    e.v[i] = keep2(draws, i, a.drop.last, e.v[i]);
                }
                hhat.v[i] = fma2(gate.v[i], uu.v[i], mul2(hhat.v[i], f2(a.carry)));
                hhat.v[i] = LAYER ? mul2(add2(hhat.v[i], f2(-st.z)), f2(st.w)) : mul2(hhat.v[i], f2(st.w));
            }
            if (!has_pre) hhat = Oct{};        // (h may be infinite)
            if (kHeld<T, LAYER> > 0) pre = held_octet(vectors);
            float2 s2[3] = {f2(0.f), f2(0.f), f2(0.f)};
            float v[kSums];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                d_pre.v[i] = fma2(q.v[i], hhat.v[i], d_pre.v[i]);
                if (LAYER) d_pre_bias.v[i] = add2(d_pre_bias.v[i], q.v[i]);
                q.v[i] = mul2(q.v[i], pre.v[i]);
                w.v[i] = fma2(q.v[i], f2(st.w), w.v[i]);
                s2[0] = fma2(q.v[i], hhat.v[i], s2[0]);
                if (LAYER) {
                    s2[1] = add2(s2[1], q.v[i]);
                } else {
                    const float2 ey = mul2(mul2(e.v[i], post.v[i]), yhat.v[i]);
                    s2[1] = fma2(ey, w.v[i], s2[1]);
                    s2[2] = fma2(ey, hhat.v[i], s2[2]);
                }
            }
#pragma unroll
            for (int k = 0; k < kSums; ++k) v[k] = s2[k].x + s2[k].y;
            sums(v);
            // r_h times the means of q hhat and (layer norm) of q; then dH.
            const float m1 = v[0] * a.inv_cols * st.w, m0 = LAYER ? v[1] * a.inv_cols * st.w : 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float2 d = fma2(hhat.v[i], f2(-m1), w.v[i]);
                if (LAYER) d = add2(d, f2(-m0));
                hhat.v[i] = mul2(d, f2(a.carry));
                d_gate.v[i] = fma2(d, uu.v[i], d_gate.v[i]);
                w.v[i] = mul2(e.v[i], d);
            }
            if (live) store_octet<T, RAGGED>(FULL ? on(static_cast<T*>(a.dx), out) : dxp, c, hhat, !LOOSE || s.vectors);
            if (has_post) {
                // The means of q2 yhat and (layer norm) of q2.
                float k1, k0 = 0.f;
                if constexpr (LAYER) {
                    s2[0] = s2[1] = f2(0.f);
                    if (kHeld<T, LAYER> > 2) post = held_octet(vectors + 4 * kLane);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        d_post.v[i] = fma2(w.v[i], yhat.v[i], d_post.v[i]);
                        d_post_bias.v[i] = add2(d_post_bias.v[i], w.v[i]);
                        w.v[i] = mul2(w.v[i], post.v[i]);
                        s2[0] = fma2(w.v[i], yhat.v[i], s2[0]);
                        s2[1] = add2(s2[1], w.v[i]);
                    }
                    v[0] = s2[0].x + s2[0].y;
                    v[1] = s2[1].x + s2[1].y;
                    sums(v);
                    k1 = v[0] * a.inv_cols;
                    k0 = v[1] * a.inv_cols;
                } else {
                    k1 = (v[1] - m1 * v[2]) * a.inv_cols;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        d_post.v[i] = fma2(w.v[i], yhat.v[i], d_post.v[i]);
                        w.v[i] = mul2(w.v[i], post.v[i]);
                    }
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (LAYER) w.v[i] = add2(w.v[i], f2(-k0));
                    w.v[i] = mul2(fma2(yhat.v[i], f2(-k1), w.v[i]), f2(st.y));
                }
            }
            if (DROP && !has_post) {
#pragma unroll
                for (int i = 0; i < 4; ++i) w.v[i] = mul2(w.v[i], f2(scale));
            }
            if (live && has_y) store_octet<T, RAGGED>(FULL ? on(static_cast<T*>(a.dy), out) : dyp, c, w, !LOOSE || s.vectors);
            if (FULL) {
                out += s.dx;
            } else {
                dxp = on(dxp, s.dx);
                dyp = on(dyp, s.dy);
            }
        }
        copy_wait<0>();
        if (gates && a.out_gate != nullptr && unit < units) {
            const int64_t at = a.splits > 1 ? unit * a.cols : unit / a.splits * a.cols;
#pragma unroll
            for (int i = 0; i < kOctet; ++i)
                if (c.in >> i & 1) {
                    const float g = a.branch * element(d_gate, i);
                    if (a.splits > 1)
                        a.gates[at + c.c0 + i] = g;
                    else
                        store_gate<T>(a, at + c.c0 + i, g);
                }
        }
    }

    // The block's sums: four rows' are joined in shared memory, in turn.
    float* joint = reinterpret_cast<float*>(ring);
#pragma unroll
    for (int k = 0; k < 5; ++k) {
        if (k == 4 ? gates || a.out_gate == nullptr : a.out_param[k] == nullptr) continue;
        Oct& o = k == 0 ? d_post : k == 1 ? d_post_bias : k == 2 ? d_pre : k == 3 ? d_pre_bias : d_gate;
        float* out = a.params + ((int64_t)(blockIdx.x / blocks) * 5 + k) * a.cols;
        const float factor = k == 4 ? a.branch : k < 2 ? a.drop.scale : 1.f;
        if constexpr (TPR == 0) {
#pragma unroll
            for (int i = 0; i < kOctet; ++i)
                if (c.in >> i & 1) out[c.c0 + i] = factor * element(o, i);
        } else {
            for (int row = 0; row < kRows; ++row) {
                __syncwarp();
                if (row == th.sub && mine < units) {
#pragma unroll
                    for (int i = 0; i < kOctet; ++i)
                        if (c.in >> i & 1)
                            joint[c.c0 + i] = row == 0 ? element(o, i) : joint[c.c0 + i] + element(o, i);
                }
            }
            __syncwarp();
            for (int i = threadIdx.x; i < (int)a.cols; i += width) out[i] = factor * joint[i];
        }
    }
}

// Joins the partial sums: a block takes 32 columns of one vector (the four
// parameters' gradients and a single gate's, then the groups' gates'); its eight
// warps take every eighth partial sum, then are added in order.  Latency bounds it
// (2 to 4 us); 32 warps a block gain nothing.
template <class T>
__global__ void __launch_bounds__(kThreads) grad_finish_kernel(const __grid_constant__ JoinArgs a) {
    __shared__ float smem[kThreads];
    pdl_wait();
    pdl_trigger();
    const int64_t tiles = (a.cols + 31) / 32;
    const int64_t vectors = 5 + gates_left(a);
    const int lane = threadIdx.x & 31, slot = threadIdx.x >> 5;
    for (int64_t u = blockIdx.x; u < tiles * vectors; u += gridDim.x) {
        const int64_t vec = u / tiles, c = (u - vec * tiles) * 32 + lane;
        if (vec < 4 ? a.out_param[vec] == nullptr : vec == 4 && (a.out_gate == nullptr || a.groups > 1)) continue;
        const float* src = vec < 5 ? a.params + vec * a.cols : a.gates + (vec - 5) * a.splits * a.cols;
        const int64_t step = vec < 5 ? 5 * a.cols : a.cols, count = vec < 5 ? a.parts : a.rows > 0 ? a.splits : 0;
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
                store_gate<T>(a, (vec == 4 ? 0 : vec - 5) * a.cols + c, s);
        }
        __syncthreads();
    }
}

int64_t at_most(int64_t n, int64_t cap) { return n < cap ? (n < 1 ? 1 : n) : cap; }

constexpr int kGradThreads = 512;       // of a row in one block, and in an SM (128 registers each)
RowForm form_of(const JoinArgs& a, int size) {
    // 32-bit counters of rows; a group's rows fall into eight classes where cols is
    // no multiple of 8: short groups would leave more sums than rows.
    if (a.rows >> 31 || (a.cols % 8 != 0 && a.groups > 1 && a.group_rows < 64)) return kValues;
    if (!RowShape(row_octets(a.cols), kGradThreads, true).fits()) return kValues;
    const void* p[] = {a.x, a.y, a.dh, a.dz, a.dx, a.dy};
    const int64_t ld[] = {a.ld_x, a.ld_y, a.ld_dh, a.ld_dz, a.ld_dx, a.ld_dy};
    for (int i = 0; i < 6; ++i)
        if (!octet_matrix(p[i], ld[i], a.rows, a.cols, size)) return kLoose;
    return kInOctets;
}

template <class T, int TPR, bool LAYER, bool RAGGED, bool DROP, bool FULL, bool LOOSE>
cudaError_t launch_rows(const JoinArgs& a, const RowShape& s, cudaStream_t stream) {
    const size_t place = LOOSE ? LooseRow<T>::kPlace : kPieces<T> * kLane, warps = s.threads / 32;
    const size_t smem = ((size_t)kGradStages<T, LAYER> * (4 * place + kWarpRows) * warps +
                         (size_t)kHeld<T, LAYER> * 2 * s.threads) * 16;
    const int64_t step = a.splits, bytes = step * (int64_t)sizeof(T);
    const GradSteps steps = {bytes * a.ld_x,  bytes * a.ld_y,  bytes * a.ld_dh, bytes * a.ld_dz,
                             bytes * a.ld_dx, bytes * a.ld_dy, step * 16,       step * a.cols / 8,
                             octet_matrix(a.dx, a.ld_dx, a.rows, a.cols, sizeof(T)) &&
                                 octet_matrix(a.dy, a.ld_dy, a.rows, a.cols, sizeof(T))};
    return launch_rows_kernel<grad_rows_kernel<T, TPR, LAYER, RAGGED, DROP, FULL, LOOSE>>(
        a.parts * s.blocks, s.threads, smem, s.blocks, stream, a, steps, s.blocks);
}
template <class T, bool LAYER, bool RAGGED, bool DROP>
cudaError_t launch_octets(const JoinArgs& a, const RowShape& s, cudaStream_t stream) {
    if (s.rows > 1) return launch_rows<T, 8, LAYER, RAGGED, DROP, false, false>(a, s, stream);
    if (a.y != nullptr && a.post != nullptr && a.pre != nullptr && a.dh != nullptr && a.ld_y == a.ld_x &&
        a.ld_dh == a.ld_x && a.ld_dz == a.ld_x && a.ld_dy == a.ld_dx)
        return launch_rows<T, 0, LAYER, RAGGED, DROP, true, false>(a, s, stream);
    return launch_rows<T, 0, LAYER, RAGGED, DROP, false, false>(a, s, stream);
}
template <class T, bool LAYER>
cudaError_t launch_octets(const JoinArgs& a, bool loose, cudaStream_t stream) {
    const RowShape s(row_octets(a.cols), kGradThreads, loose);
    const bool drop = a.drop.cut != 0;
    if (loose)
        return drop ? launch_rows<T, 0, LAYER, true, true, false, true>(a, s, stream)
                    : launch_rows<T, 0, LAYER, true, false, false, true>(a, s, stream);
    if (a.cols % 8 == 0)
        return drop ? launch_octets<T, LAYER, false, true>(a, s, stream) : launch_octets<T, LAYER, false, false>(a, s, stream);
    return drop ? launch_octets<T, LAYER, true, true>(a, s, stream) : launch_octets<T, LAYER, true, false>(a, s, stream);
}

template <class T>
cudaError_t launch(const JoinArgs& a, int num_sms, cudaStream_t stream) {
    cudaError_t st = cudaSuccess;
    const RowForm form = form_of(a, (int)sizeof(T));
    if (a.rows > 0 && form != kValues) {
        st = a.layer ? launch_octets<T, true>(a, form == kLoose, stream) : launch_octets<T, false>(a, form == kLoose, stream);
    } else if (a.rows > 0) {
        st = launch_pdl(grad_rows_any_kernel<T>, (unsigned)at_most(a.rows, (int64_t)num_sms * 8), kThreads, 0,
                        stream, a);
        const int64_t tiles = (a.cols + kThreads - 1) / kThreads;
        if (st == cudaSuccess)
            st = launch_pdl(grad_columns_any_kernel<T>, (unsigned)at_most(tiles * a.parts, (int64_t)num_sms * 16),
                            kThreads, 0, stream, a);
    }
    const int64_t vectors = 5 + gates_left(a);
    if (st == cudaSuccess)
        st = launch_pdl(grad_finish_kernel<T>,
                        (unsigned)at_most((a.cols + 31) / 32 * vectors, (int64_t)num_sms * 64), kThreads, 0,
                        stream, a);
    return st;
}

}  // namespace
}  // namespace fasgd
