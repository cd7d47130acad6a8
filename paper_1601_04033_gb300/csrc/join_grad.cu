// fasgd_join_grad.  With hats the normalised values and r the 1/sqrt of a row,
//   q  = dz pre,  dH = dh + r_h (q - mean q - hhat mean(q hhat))   (rms: no mean q)
//   dx = carry dH,  dgate += branch dH u,  dt = m scale branch gate dH
//   q2 = dt post,  dy = r_y (q2 - mean q2 - yhat mean(q2 yhat))
//   dpre += dz hhat, dpre_bias += dz, dpost += dt yhat, dpost_bias += dt.
// hhat comes from h formed again out of x and y, which costs the bytes that
// reading h would and keeps h's rounding out of the parameters' gradients.

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

// Rows in octets.  TPR threads hold a row, an octet each; every thread keeps its
// columns' sums over the rows it takes in registers.  One reduction a row is
// enough: with e = m scale branch gate post (so q2 = e dH) and w = dh + r_h q,
//   sum q2 yhat = S(e yhat w) - r_h (mean q S(e yhat) + mean(q hhat) S(e yhat hhat)),
// and the same without yhat for mean q2, so all sums are of what is known before
// mean q is.  Units as in the plain form, for the threads of one row ("sub") at a
// time; where cols is no multiple of 8 a unit's rows agree modulo 8 (octet.cuh).
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

template <class T, int TPR, int C, int STAGES, bool LAYER>
__global__ void __launch_bounds__(TPR < 256 ? 256 : TPR, TPR <= 256 ? 2 : 1)
    grad_rows_kernel(const __grid_constant__ JoinArgs a) {
    constexpr int kBlock = TPR < 256 ? 256 : TPR, kSubs = kBlock / TPR, kP = kPieces<T>;
    constexpr int kSums = LAYER ? 8 : 3;
    using Sums = RowSums<TPR, kSums, C>;
    extern __shared__ uint4 ring[];                  // [STAGES][x, y, dh, dz][kP][kBlock]
    __shared__ __align__(16) float red[kSubs * Sums::kPlaces];
    const int sub = threadIdx.x / TPR, lane = threadIdx.x % TPR;
    const int64_t units = a.groups * a.splits, subs = (int64_t)(gridDim.x / C) * kSubs;
    const int64_t mine = (int64_t)(blockIdx.x / C) * kSubs + sub;
    const bool has_y = a.y != nullptr, has_pre = a.pre != nullptr, has_post = a.post != nullptr;
    const bool has_dh = a.dh != nullptr, gates = a.groups > 1, ragged = (a.cols & 7) != 0;
    Sums sums(red, sub);
    pdl_wait();
    pdl_trigger();

    // All rows that this sub takes begin at the same place in an octet.
    const Columns c(lane + (C > 1 ? (int)cluster_rank() * TPR : 0),
                    ragged && mine < units ? (int)((Unit(a, mine).row * a.cols) & 7) : 0, (int32_t)a.cols);
    const float scale = a.drop.scale;
    // As the forward kernel has them, so that h comes out in the same bits.
    Oct post = load_vector(a.post, c, 1.f), post_bias, gate;
    const Oct pre = load_vector(a.pre, c, 0.f);
    if (LAYER) post_bias = load_vector(a.post_bias, c, 0.f);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        post.v[i] = mul2(post.v[i], f2(scale));
        if (LAYER) post_bias.v[i] = mul2(post_bias.v[i], f2(scale));
    }
    // Sums over the rows: those of the norm after the block without `scale`, the
    // gate's without `branch`.
    Oct d_post = {}, d_post_bias = {}, d_gate = {}, d_pre = {}, d_pre_bias = {};
    constexpr int kStage = 4 * kP * kBlock;
    uint4* const own = ring + threadIdx.x;

    // Where a warp holds several rows, it goes on until the first of them is done.
    const int64_t last_unit = units + (TPR < 32 ? sub % (32 / TPR) : 0);
    for (int64_t unit = mine; unit < last_unit; unit += subs) {
        Unit u(a, unit < units ? unit : 0);
        if (unit >= units) u.rows = 0;
        int64_t turns = u.row < u.rows ? (u.rows - u.row + u.step - 1) / u.step : 0;
        if constexpr (TPR < 32) {
#pragma unroll
            for (int off = 16; off >= TPR; off >>= 1) {
                const int64_t other = __shfl_xor_sync(0xffffffffu, turns, off);
                turns = other > turns ? other : turns;
            }
        }
        if (gates || unit == mine) {
            gate = load_gate<T>(a, gates && unit < units ? unit / a.splits : 0, c);
#pragma unroll
            for (int i = 0; i < 4; ++i) gate.v[i] = mul2(gate.v[i], f2(a.branch));
        }
        if (gates) d_gate = Oct{};

        int64_t r = u.row, fetched = r, left = (a.rows - r) * a.cols - c.c0;
        const T* x = static_cast<const T*>(a.x) + r * a.ld_x + c.c0;       // of the next row to fetch
        const T* y = static_cast<const T*>(a.y) + r * a.ld_y + c.c0;
        const T* dh = static_cast<const T*>(a.dh) + r * a.ld_dh + c.c0;
        const T* dz = static_cast<const T*>(a.dz) + r * a.ld_dz + c.c0;
        const auto fetch = [&](uint4* slot) {
            if (fetched < u.rows && c.any()) {
                const bool whole = !ragged || left >= kOctet;
                copy_octet<T>(slot, kBlock, x, whole, left);
                if (has_y) copy_octet<T>(slot + kP * kBlock, kBlock, y, whole, left);
                if (has_dh) copy_octet<T>(slot + 2 * kP * kBlock, kBlock, dh, whole, left);
                if (has_pre) copy_octet<T>(slot + 3 * kP * kBlock, kBlock, dz, whole, left);
            }
            copy_commit();
            fetched += u.step;
            left -= u.step * a.cols;
            x += u.step * a.ld_x;
            y += u.step * a.ld_y;
            dh += u.step * a.ld_dh;
            dz += u.step * a.ld_dz;
        };
#pragma unroll
        for (int s = 0; s < STAGES - 1; ++s) fetch(own + s * kStage);
        T* dxp = static_cast<T*>(a.dx) + r * a.ld_dx + c.c0;
        T* dyp = static_cast<T*>(a.dy) + r * a.ld_dy + c.c0;
        int stage = 0;
        float4 st = r < u.rows ? a.stats[r] : make_float4(0.f, 0.f, 0.f, 0.f);
        for (int64_t turn = 0; turn < turns; ++turn) {
            const bool live = TPR >= 32 || r < u.rows;
            // The next row's statistics, ahead of its turn.
            const float4 next = r + u.step < u.rows ? a.stats[r + u.step] : make_float4(0.f, 0.f, 0.f, 0.f);
            const Philox4 draws = octet_draws(a.drop, c.any(), (r * a.cols + c.c0) >> 3);
            copy_wait<STAGES - 2>();
            const uint4* slot = own + stage * kStage;
            Oct hhat = take_octet<T>(slot, kBlock, c), yhat = {}, w = {}, q = {}, e, uu;
            if (has_y) yhat = take_octet<T>(slot + kP * kBlock, kBlock, c);
            if (has_dh) w = take_octet<T>(slot + 2 * kP * kBlock, kBlock, c);
            if (has_pre) q = take_octet<T>(slot + 3 * kP * kBlock, kBlock, c);
            fetch(own + (stage == 0 ? STAGES - 1 : stage - 1) * kStage);
            stage = stage == STAGES - 1 ? 0 : stage + 1;
            if (TPR < 32 && !live) hhat = yhat = w = q = Oct{};      // a row past the end
            // u; e = what dH is multiplied by in dt / scale.
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (LAYER) yhat.v[i] = add2(yhat.v[i], f2(-st.x));
                yhat.v[i] = mul2(yhat.v[i], f2(st.y));
                uu.v[i] = LAYER ? fma2(yhat.v[i], post.v[i], post_bias.v[i]) : mul2(yhat.v[i], post.v[i]);
                uu.v[i] = keep2(draws, i, a.drop.last, uu.v[i]);
                e.v[i] = keep2(draws, i, a.drop.last, gate.v[i]);
                hhat.v[i] = fma2(gate.v[i], uu.v[i], mul2(hhat.v[i], f2(a.carry)));
                hhat.v[i] = LAYER ? mul2(add2(hhat.v[i], f2(-st.z)), f2(st.w)) : mul2(hhat.v[i], f2(st.w));
            }
            if (!has_pre) hhat = Oct{};        // (h may be infinite)
            float2 s2[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) s2[k] = f2(0.f);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                d_pre.v[i] = fma2(q.v[i], hhat.v[i], d_pre.v[i]);
                if (LAYER) d_pre_bias.v[i] = add2(d_pre_bias.v[i], q.v[i]);
                q.v[i] = mul2(q.v[i], pre.v[i]);
                w.v[i] = fma2(q.v[i], f2(st.w), w.v[i]);
                const float2 ep = mul2(e.v[i], post.v[i]), ey = mul2(ep, yhat.v[i]);
                s2[0] = fma2(q.v[i], hhat.v[i], s2[0]);
                s2[1] = fma2(ey, w.v[i], s2[1]);
                s2[2] = fma2(ey, hhat.v[i], s2[2]);
                if (LAYER) {
                    s2[3] = add2(s2[3], q.v[i]);
                    s2[4] = add2(s2[4], ey);
                    s2[5] = fma2(ep, w.v[i], s2[5]);
                    s2[6] = fma2(ep, hhat.v[i], s2[6]);
                    s2[7] = add2(s2[7], ep);
                }
            }
            float s[kSums];
#pragma unroll
            for (int k = 0; k < kSums; ++k) s[k] = s2[k].x + s2[k].y;
            sums(s);
            // r_h times the means of q hhat and of q; the means of q2 yhat and of q2.
            const float m1 = s[0] * a.inv_cols * st.w, m0 = LAYER ? s[3] * a.inv_cols * st.w : 0.f;
            const float k1 = (LAYER ? s[1] - m0 * s[4] - m1 * s[2] : s[1] - m1 * s[2]) * a.inv_cols;
            const float k0 = LAYER ? (s[5] - m0 * s[7] - m1 * s[6]) * a.inv_cols : 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float2 d = fma2(hhat.v[i], f2(-m1), w.v[i]);
                if (LAYER) d = add2(d, f2(-m0));
                hhat.v[i] = mul2(d, f2(a.carry));
                d_gate.v[i] = fma2(d, uu.v[i], d_gate.v[i]);
                w.v[i] = mul2(e.v[i], d);
            }
            if (has_post) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    d_post.v[i] = fma2(w.v[i], yhat.v[i], d_post.v[i]);
                    if (LAYER) d_post_bias.v[i] = add2(d_post_bias.v[i], w.v[i]);
                    w.v[i] = mul2(w.v[i], post.v[i]);
                    if (LAYER) w.v[i] = add2(w.v[i], f2(-k0));
                    w.v[i] = mul2(fma2(yhat.v[i], f2(-k1), w.v[i]), f2(st.y));
                }
            }
            if (!has_post) {
#pragma unroll
                for (int i = 0; i < 4; ++i) w.v[i] = mul2(w.v[i], f2(scale));
            }
            if (live) {
                store_octet(dxp, c, hhat);
                if (has_y) store_octet(dyp, c, w);
            }
            st = next;
            r += u.step;
            dxp += u.step * a.ld_dx;
            dyp += u.step * a.ld_dy;
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

    // The block's sums: its subs' in turn, joined in shared memory.
    float* joint = reinterpret_cast<float*>(ring);
#pragma unroll
    for (int k = 0; k < 5; ++k) {
        if (k == 4 ? gates || a.out_gate == nullptr : a.out_param[k] == nullptr) continue;
        Oct& o = k == 0 ? d_post : k == 1 ? d_post_bias : k == 2 ? d_pre : k == 3 ? d_pre_bias : d_gate;
        float* out = a.params + ((int64_t)(blockIdx.x / C) * 5 + k) * a.cols;
        const float factor = k == 4 ? a.branch : k < 2 ? a.drop.scale : 1.f;
        if constexpr (kSubs == 1) {
#pragma unroll
            for (int i = 0; i < kOctet; ++i)
                if (c.in >> i & 1) out[c.c0 + i] = factor * element(o, i);
        } else {
            for (int s = 0; s < kSubs; ++s) {
                __syncthreads();
                if (s == sub && mine < units) {
#pragma unroll
                    for (int i = 0; i < kOctet; ++i)
                        if (c.in >> i & 1)
                            joint[c.c0 + i] = s == 0 ? element(o, i) : joint[c.c0 + i] + element(o, i);
                }
            }
            __syncthreads();
            for (int i = threadIdx.x; i < (int)a.cols; i += kBlock) out[i] = factor * joint[i];
        }
    }
}

// Joins the partial sums: a block takes 32 columns of one vector (the four
// parameters' gradients and a single gate's, then the groups' gates'); eight lanes of rows
// take every eighth partial sum, then are added in order.
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

// The threads of a row of the fast kernels, in blocks of at most 512 (0: the plain form).
int threads_per_row(const JoinArgs& a) {
    const int64_t octets = row_octets(a.cols);
    const void* p[] = {a.x, a.y, a.dh, a.dz, a.dx, a.dy};
    const int64_t ld[] = {a.ld_x, a.ld_y, a.ld_dh, a.ld_dz, a.ld_dx, a.ld_dy};
    for (int i = 0; i < 6; ++i) {
        if (!octet_matrix(p[i], ld[i], a.rows, a.cols)) return 0;
        if (a.cols % 8 != 0 && a.rows > 1 && p[i] != nullptr && ld[i] != a.cols) return 0;
    }
    // A group's rows fall into eight classes where cols is no multiple of 8: short
    // groups would leave more sums than rows.
    if (a.cols % 8 != 0 && a.groups > 1 && a.group_rows < 64) return 0;
    for (int t : {8, 32, 64, 128, 256, 512, 1024, 2048, 4096})
        if (octets <= t) return t;
    return 0;
}
int blocks_per_sm(int threads) { return threads <= 256 ? 2 : 1; }

template <class T, int TPR, int C, bool LAYER>
cudaError_t launch_rows(const JoinArgs& a, cudaStream_t stream) {
    constexpr int kBlock = TPR < 256 ? 256 : TPR;
    constexpr int kStages = sizeof(T) == 4 ? 3 : 4;
    constexpr size_t kSmem = (size_t)kStages * 4 * kPieces<T> * kBlock * 16;
    return launch_rows_kernel<C>(grad_rows_kernel<T, TPR, C, kStages, LAYER>, a.parts * C, kBlock, kSmem, stream, a);
}
template <class T, bool LAYER>
cudaError_t launch_octets(const JoinArgs& a, int threads, cudaStream_t stream) {
    switch (threads) {
        case 8: return launch_rows<T, 8, 1, LAYER>(a, stream);
        case 32: return launch_rows<T, 32, 1, LAYER>(a, stream);
        case 64: return launch_rows<T, 64, 1, LAYER>(a, stream);
        case 128: return launch_rows<T, 128, 1, LAYER>(a, stream);
        case 256: return launch_rows<T, 256, 1, LAYER>(a, stream);
        case 512: return launch_rows<T, 512, 1, LAYER>(a, stream);
        case 1024: return launch_rows<T, 512, 2, LAYER>(a, stream);
        case 2048: return launch_rows<T, 512, 4, LAYER>(a, stream);
        default: return launch_rows<T, 512, 8, LAYER>(a, stream);
    }
}

template <class T>
cudaError_t launch(const JoinArgs& a, int num_sms, cudaStream_t stream) {
    cudaError_t st = cudaSuccess;
    if (const int threads = a.rows > 0 ? threads_per_row(a) : 0) {
        st = a.layer ? launch_octets<T, true>(a, threads, stream) : launch_octets<T, false>(a, threads, stream);
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

JoinPlan join_grad_plan(const JoinArgs& a, int dtype, int num_sms) {
    (void)dtype;
    JoinPlan p;
    p.parts = p.splits = p.row_means = 0;
    if (a.rows == 0) return p;
    if (const int threads = threads_per_row(a)) {
        const int block_subs = threads < 256 ? 256 / threads : 1;
        const int cluster = threads > 512 ? threads / 512 : 1;
        const int64_t most = (int64_t)num_sms * blocks_per_sm(threads) / cluster / 8 * 8 * block_subs;
        if (a.groups == 1) {
            p.splits = at_most(a.rows, most);
        } else {
            // Four units for each sub, but no fewer than eight rows to a unit: each
            // leaves a row's worth of fp32 sums.
            p.splits = at_most((4 * most + a.groups - 1) / a.groups, at_most(a.group_rows / 8, a.group_rows));
            if (a.cols % 8 != 0) p.splits = (p.splits + 7) / 8 * 8;
        }
        const int64_t units = a.groups * p.splits;
        p.parts = (at_most(units, most) + block_subs - 1) / block_subs;
        if (a.groups == 1) p.splits = p.parts * block_subs;
        return p;
    }
    const int64_t most = 2 * (int64_t)num_sms;
    p.splits = at_most((most + a.groups - 1) / a.groups, a.group_rows);
    p.parts = at_most(a.groups * p.splits, most);
    p.row_means = a.rows;
    return p;
}

cudaError_t launch_join_grad(const JoinArgs& a, int dtype, int num_sms, cudaStream_t stream) {
    if (dtype == FASGD_F32) return launch<float>(a, num_sms, stream);
    if (dtype == FASGD_BF16) return launch<__nv_bfloat16>(a, num_sms, stream);
    return launch<__half>(a, num_sms, stream);
}

}  // namespace fasgd
