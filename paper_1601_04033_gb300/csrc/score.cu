// fasgd_score: softmax cross entropy of rows against classes from the last product on.
//
// s = z w is formed twice and never kept.  The first time its tiles leave, for each row,
// their maximum m_j and sum_v exp(s - m_j); these give lse = M + log sum_j exp(m_j - M)
// sum_j.  The second time, a piece of the classes after the other, the tiles leave
// g = exp(s - lse) - [v = label], from which the piece's part of dz = g w^T and its rows of
// dw = z^T g follow.  A piece of g lies by classes ([v][row]), which makes it an operand of
// both products as it stands.  Keeping s in place of forming it again would cost 4 bytes
// a value written and read, and rounding it to 2 would show in dz and dw.
//
// g is held without upstream / N, so that its values are in [-1, 1] and no fp16 value is
// lost for N's size; for fp16 it is held times 2^14, so that probabilities down to 2^-28
// keep all their bits.  The products' results are multiplied by upstream / N, in fp32.
// Rows without a label are copied as zeros, behind the others where there are many, and have no tiles.
//
// 8,192 x 2,048 x 131,072 bf16, a tenth without labels: 9.8 ms, 2.2 of them the first sweep; all products
// together 1,620 TFLOP/s of the work that rows with labels need.

#include <algorithm>

#include "checks.cuh"
#include "client.cuh"
#include "product.cuh"
#include "shared_limit.cuh"

namespace {

using fasgd::Product;

struct Score {
    fasgd_score_args u;
    int64_t size, tile;
    bool grad;
    bool few;                    // few classes: no products
    float* few_sums;
    float* few_dw;
    bool planes;                 // fp32 by planes on the tensor cores
    int64_t plane_z, plane_w, plane_g;
    // Rows that have labels first, where the tensor cores take many rows: what has none costs nothing.
    bool first;
    int32_t *to_row, *row_at, *live;     // [rows] each row's place and back, [1] how many have labels
    int64_t* labels;                     // [rows] by place
    float* loss_at;                      // [rows] by place (lse too)
    // workspace
    void* z_copy;                // rows x ld_zc (null: z itself serves)
    int64_t ld_zc;
    void* w_copy;                // as w, rows ld_wc apart (null: w itself serves)
    int64_t ld_wc;
    float2* parts;               // [tiles][rows]
    float *at_label, *lse;       // [rows]
    float* row_scale;            // [rows] upstream / N, 0 without a label
    float* share;                // [1] upstream / N
    void* g;                     // [piece][ld_g]
    int64_t ld_g, piece;
    float* dz_sum;               // [dz_parts][rows][cols] (several pieces)
    int32_t dz_parts;
    float* sums;                 // room for the parts of a product's sums
    float factor;                // what g is held times
    const void *z, *w;           // what the products read
};

// lse and the row's loss from the tiles' parts: ROWS rows a block, 256 / ROWS threads each, every one
// four parts at a time (few rows have more threads: one row's 1,024 parts took 8 of them 23 us).
template <int ROWS>
__global__ void __launch_bounds__(256) lse_kernel(Score s) {
    constexpr int kEach = 256 / ROWS;
    __shared__ float2 shared[kEach][ROWS];
    const int64_t rows = s.u.rows, tiles = (s.u.classes + s.tile - 1) / s.tile, live = s.first ? *s.live : rows;
    const int x = threadIdx.x % ROWS, y = threadIdx.x / ROWS;
    const int64_t r = (int64_t)blockIdx.x * ROWS + x;
    float top = -INFINITY, sum = 0.0f;
    const auto join = [&](float2 p) {
        const float most = fmaxf(top, p.x);
        sum = (top == most ? sum : sum * expf(top - most)) + (p.x == most ? p.y : p.y * expf(p.x - most));
        top = most;
    };
    if (r < live)
        for (int64_t j = y; j < tiles; j += 4 * kEach) {
            float2 p[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                p[i] = j + i * kEach < tiles ? s.parts[(j + i * kEach) * rows + r] : make_float2(-INFINITY, 0.0f);
#pragma unroll
            for (int i = 0; i < 4; ++i) join(p[i]);
        }
    shared[y][x] = make_float2(top, sum);
#pragma unroll
    for (int half = kEach / 2; half > 0; half /= 2) {
        __syncthreads();
        if (y < half) {
            join(shared[y + half][x]);
            shared[y][x] = make_float2(top, sum);
        }
    }
    if (y == 0 && r < live) {
        const float log_sum = logf(sum), lse = top + log_sum;
        const int64_t label = (s.first ? s.labels : s.u.labels)[r];
        const float loss = label >= 0 && label < s.u.classes ? (top - s.at_label[r]) + log_sum : 0.0f;
        s.lse[r] = lse;
        if (s.first) {
            const int64_t at = s.row_at[r];
            s.loss_at[r] = loss;
            s.u.row_loss[at] = loss;
            if (s.u.lse != nullptr) s.u.lse[at] = lse;
        } else {
            s.u.row_loss[r] = loss;
        }
    }
}
template <int ROWS>
cudaError_t launch_lse(const Score& s, cudaStream_t stream) {
    lse_kernel<ROWS><<<(unsigned)((s.u.rows + ROWS - 1) / ROWS), 256, 0, stream>>>(s);
    return cudaGetLastError();
}

// The rows' places, those that have labels first, in their order: one block, whose rounds of 1,024 rows wait
// for each other (a million rows: 938 us, of 2,310 for their score of 64 x 64).  What rows without a label leave
// behind is written here, and what is known of the others goes to their places.
__global__ void __launch_bounds__(1024) first_kernel(fasgd_score_args u, Score s) {
    __shared__ int32_t counts[32];
    __shared__ int32_t total;
    const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;
    const auto has = [&](int64_t r) { return r < u.rows && u.labels[r] >= 0 && u.labels[r] < u.classes; };
    int32_t n = 0;
#pragma unroll 8
    for (int64_t r = threadIdx.x; r < u.rows; r += 1024) n += has(r);
    n = __reduce_add_sync(0xffffffffu, n);
    if (lane == 0) counts[warp] = n;
    __syncthreads();
    if (warp == 0) {
        n = __reduce_add_sync(0xffffffffu, counts[lane]);
        if (lane == 0) *s.live = total = n;
    }
    int32_t before = 0;                              // labels in earlier rounds
    int64_t next = threadIdx.x < u.rows ? u.labels[threadIdx.x] : -1;
    for (int64_t r0 = 0; r0 < u.rows; r0 += 1024) {
        const int64_t r = r0 + threadIdx.x, label = next;
        next = r + 1024 < u.rows ? u.labels[r + 1024] : -1;      // (read ahead of this round's barriers)
        const bool is = label >= 0 && label < u.classes;
        const uint32_t votes = __ballot_sync(0xffffffffu, is);
        __syncthreads();
        if (lane == 0) counts[warp] = __popc(votes);
        __syncthreads();
        const int32_t of = counts[lane];             // this round's warps
        const int32_t earlier = __reduce_add_sync(0xffffffffu, lane < warp ? of : 0), all = __reduce_add_sync(0xffffffffu, of);
        if (r < u.rows) {
            const int32_t rank = before + earlier + __popc(votes & ((1u << lane) - 1u));
            const int32_t to = is ? rank : total + (int32_t)(r - rank);
            s.to_row[r] = to;
            s.row_at[to] = (int32_t)r;
            s.labels[to] = is ? label : -1;
            if (u.known) {
                s.lse[to] = is ? u.lse[r] : 0.0f;
                s.loss_at[to] = is ? u.row_loss[r] : 0.0f;
            } else if (!is) {
                u.row_loss[r] = 0.0f;
                if (u.lse != nullptr) u.lse[r] = 0.0f;
            }
        }
        before += all;
    }
}

// The loss, upstream / N, and what each row's gradient is multiplied by: one block (a million rows: 350 us).
__global__ void __launch_bounds__(1024) loss_kernel(int64_t rows, const int64_t* labels, int64_t classes,
                                                    const float* row_loss, const float* upstream, float* loss,
                                                    float* share, float* row_scale) {
    __shared__ float sums[32];
    __shared__ int64_t counts[32];
    const auto has = [&](int64_t r) { return labels[r] >= 0 && labels[r] < classes; };
    float sum = 0.0f;
    int64_t count = 0;
#pragma unroll 8
    for (int64_t r = threadIdx.x; r < rows; r += 1024) {
        const float loss_of = row_loss[r];
        if (has(r)) {
            sum += loss_of;
            ++count;
        }
    }
    sum = fasgd::warp_sum(sum);
    for (int d = 16; d > 0; d >>= 1) count += __shfl_xor_sync(0xffffffffu, count, d);
    if (threadIdx.x % 32 == 0) {
        sums[threadIdx.x / 32] = sum;
        counts[threadIdx.x / 32] = count;
    }
    __syncthreads();
    sum = 0.0f;
    count = 0;
    for (int w = 0; w < 32; ++w) {
        sum += sums[w];
        count += counts[w];
    }
    const float up = count == 0 ? 0.0f : (upstream != nullptr ? *upstream : 1.0f) / (float)count;
    if (threadIdx.x == 0) {
        if (loss != nullptr) *loss = count == 0 ? 0.0f : sum / (float)count;
        if (share != nullptr) *share = up;
    }
    if (row_scale != nullptr)
        for (int64_t r = threadIdx.x; r < rows; r += 1024) row_scale[r] = has(r) ? up : 0.0f;
}

// ---- few classes ------------------------------------------------------------------------------
// A client's last product with, say, 10 classes: everything in one pass over the rows, fp32 on the
// ordinary cores, and a second launch for the sums over the rows.  w lies in shared memory as
// [class][col]; a warp takes a row: its lanes go along the columns and keep a sum for each class, so that
// every value of z and w is read once a row.  Blocks take the rows by turns and keep their share of dw in
// shared memory too, each thread its own columns of it; the shares are added up in the blocks' order.
// The bound is latency: 128 x 200 x 10 takes 17 us with the host; seven launches of the products' general
// forms took 68.  Many rows are bound by a warp's shared-memory reads, one for each multiply-add: bf16, with
// gradients, 1,024 rows of 384 x 32 take 49 us and of 384 x 33, by the tensor cores, 63; 4,096 rows 99 and 71; 262,144
// 3,886 and 936; 16,384 rows of 200 x 10 103 and of 200 x 33 93.
constexpr int kFewClasses = 32, kFewBlocks = 152;
constexpr int64_t kFewValues = 12 << 10;           // of w: 48 KB, and dw as much again
constexpr int kFewWarps = 8;

bool few_classes(const fasgd_score_args& u) {
    return u.classes <= kFewClasses && u.cols * u.classes <= kFewValues;
}
int64_t few_blocks(int64_t rows) { return std::max<int64_t>(1, std::min<int64_t>(kFewBlocks, (rows + kFewWarps - 1) / kFewWarps)); }

struct FewArgs {
    fasgd_score_args u;
    float* sums;        // [blocks] of the rows' losses
    float* dw;          // [blocks][classes][cols]
};
template <class T>
__global__ void __launch_bounds__(32 * kFewWarps) few_kernel(FewArgs a) {
    extern __shared__ float shared[];              // w, then dw, then g [warps][classes], then sums [warps]
    const fasgd_score_args& u = a.u;
    const int V = (int)u.classes, D = (int)u.cols, warp = threadIdx.x / 32, lane = threadIdx.x & 31;
    float *const w = shared, *const dw = w + V * D, *const g = dw + (u.dw != nullptr ? V * D : 0), *const part = g + kFewWarps * V;
    __shared__ long long total;
    if (threadIdx.x == 0) total = 0;
    __syncthreads();
    // N, by every block for itself.
    if (u.dz != nullptr) {
        long long n = 0;
        for (int64_t r = threadIdx.x; r < u.rows; r += blockDim.x) n += u.labels[r] >= 0 && u.labels[r] < V;
        for (int d = 16; d > 0; d >>= 1) n += __shfl_xor_sync(0xffffffffu, n, d);
        if (lane == 0) atomicAdd(reinterpret_cast<unsigned long long*>(&total), (unsigned long long)n);
    }
    const T* from = static_cast<const T*>(u.w);
    for (int i = threadIdx.x; i < V * D; i += blockDim.x) {
        const int v = u.w_flip ? i / D : i % V, d = u.w_flip ? i % D : i / V;
        w[v * D + d] = fasgd::to_f32(from[u.w_flip ? v * u.ld_w + d : d * u.ld_w + v]);
        if (u.dw != nullptr) dw[i] = 0.0f;
    }
    __syncthreads();
    const float share = total == 0 ? 0.0f : (u.upstream != nullptr ? *u.upstream : 1.0f) / (float)total;
    float loss = 0.0f;
    for (int64_t r0 = (int64_t)blockIdx.x * kFewWarps; r0 < u.rows; r0 += (int64_t)gridDim.x * kFewWarps) {
        const int64_t r = r0 + warp;
        const int64_t label = r < u.rows ? u.labels[r] : -1;
        const bool has = label >= 0 && label < V;
        const T* z = static_cast<const T*>(u.z) + r * u.ld_z;
        float p = 0.0f;                            // lane v: g of class v
        if (has) {
            float s = -INFINITY;                   // lane v: the value of class v
            for (int v0 = 0; v0 < V; v0 += 8) {
                float sum[8] = {};
                for (int d = lane; d < D; d += 32) {
                    const float x = fasgd::to_f32(z[d]);
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (v0 + j < V) sum[j] = fmaf(x, w[(v0 + j) * D + d], sum[j]);
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float all = fasgd::warp_sum(sum[j]);
                    if (lane == v0 + j && v0 + j < V) s = all;
                }
            }
            float top = s;
            for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
            const float log_sum = logf(fasgd::warp_sum(lane < V ? (s == top ? 1.0f : expf(s - top)) : 0.0f));
            const float own = __shfl_sync(0xffffffffu, s, (int)label), row_loss = (top - own) + log_sum;
            const float lse = u.known ? u.lse[r] : top + log_sum;
            loss += row_loss;
            if (lane == 0 && !u.known) {
                u.row_loss[r] = row_loss;
                if (u.lse != nullptr) u.lse[r] = lse;
            }
            p = lane >= V ? 0.0f : lane == label ? expm1f(u.known ? -u.row_loss[r] : -row_loss) : expf(s - lse);
        } else if (r < u.rows && lane == 0 && !u.known) {
            u.row_loss[r] = 0.0f;
            if (u.lse != nullptr) u.lse[r] = 0.0f;
        }
        if (u.dz == nullptr && u.dw == nullptr) continue;
        if (lane < V) g[warp * V + lane] = p;
        __syncwarp();
        if (u.dz != nullptr && r < u.rows) {
            T* dz = static_cast<T*>(u.dz) + r * u.ld_dz;
            for (int d = lane; d < D; d += 32) {
                float sum = 0.0f;
                for (int v = 0; has && v < V; ++v) sum = fmaf(g[warp * V + v], w[v * D + d], sum);
                dz[d] = fasgd::from_f32<T>(has ? sum * share : 0.0f);
            }
            __syncwarp();                          // a next row without a label writes g at once
        }
        if (u.dw != nullptr) {
            __syncthreads();                       // the rows of all warps
            const int rows = (int)min((int64_t)kFewWarps, u.rows - r0);
            for (int d = threadIdx.x; d < D; d += blockDim.x) {
                float x[kFewWarps];
#pragma unroll
                for (int i = 0; i < kFewWarps; ++i) {
                    const int64_t l = i < rows ? u.labels[r0 + i] : -1;
                    x[i] = l >= 0 && l < V ? fasgd::to_f32(static_cast<const T*>(u.z)[(r0 + i) * u.ld_z + d]) : 0.0f;
                }
                for (int v = 0; v < V; ++v) {
                    float sum = dw[v * D + d];
#pragma unroll
                    for (int i = 0; i < kFewWarps; ++i) sum = fmaf(g[i * V + v], x[i], sum);
                    dw[v * D + d] = sum;
                }
            }
            __syncthreads();
        }
    }
    if (lane == 0) part[warp] = loss;
    __syncthreads();
    if (threadIdx.x == 0) {
        float sum = 0.0f;
        for (int i = 0; i < kFewWarps; ++i) sum += part[i];
        a.sums[blockIdx.x] = sum;
    }
    if (u.dw != nullptr)
        for (int i = threadIdx.x; i < V * D; i += blockDim.x) a.dw[(int64_t)blockIdx.x * V * D + i] = dw[i];
}
// The blocks' shares of dw and of the loss.
template <class T>
__global__ void __launch_bounds__(256) few_sum_kernel(FewArgs a, int32_t blocks) {
    const fasgd_score_args& u = a.u;
    __shared__ unsigned long long total;
    if (threadIdx.x == 0) total = 0;
    __syncthreads();
    unsigned long long n = 0;
    for (int64_t r = threadIdx.x; r < u.rows; r += 256) n += u.labels[r] >= 0 && u.labels[r] < u.classes;
    for (int d = 16; d > 0; d >>= 1) n += __shfl_xor_sync(0xffffffffu, n, d);
    if ((threadIdx.x & 31) == 0) atomicAdd(&total, n);
    __syncthreads();
    const float count = (float)total;
    if (blockIdx.x == 0 && threadIdx.x == 0 && u.loss != nullptr) {
        float sum = 0.0f;
        for (int b = 0; b < blocks; ++b) sum += a.sums[b];
        *u.loss = total == 0 ? 0.0f : sum / count;
    }
    if (u.dw == nullptr) return;
    const float share = total == 0 ? 0.0f : (u.upstream != nullptr ? *u.upstream : 1.0f) / count;
    const int64_t values = u.classes * u.cols, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= values) return;
    float sum = 0.0f;
#pragma unroll 8
    for (int b = 0; b < blocks; ++b) sum += a.dw[b * values + i];
    const int64_t v = i / u.cols, d = i % u.cols;
    static_cast<T*>(u.dw)[u.dw_flip ? v * u.ld_dw + d : d * u.ld_dw + v] = fasgd::from_f32<T>(total == 0 ? 0.0f : sum * share);
}
template <class T>
cudaError_t run_few(const FewArgs& a, cudaStream_t stream) {
    static fasgd::SharedLimit limit;
    const fasgd_score_args& u = a.u;
    const int64_t blocks = few_blocks(u.rows), values = u.cols * u.classes;
    const int64_t bytes = 4 * (values * (u.dw != nullptr ? 2 : 1) + kFewWarps * u.classes + kFewWarps);
    int device = 0;
    cudaError_t st = cudaGetDevice(&device);
    if (st != cudaSuccess) return st;
    const int error = limit.ensure(device, bytes, 4 * (2 * kFewValues + kFewWarps * kFewClasses + kFewWarps), [](int64_t n) {
        return (int)cudaFuncSetAttribute(few_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)n);
    });
    if (error != 0) return (cudaError_t)error;
    few_kernel<T><<<(unsigned)blocks, 32 * kFewWarps, bytes, stream>>>(a);
    if ((st = cudaGetLastError()) != cudaSuccess) return st;
    const int64_t grid = u.dw != nullptr ? (values + 255) / 256 : 1;
    few_sum_kernel<T><<<(unsigned)grid, 256, 0, stream>>>(a, (int32_t)blocks);
    return cudaGetLastError();
}

int fill_score(const char* call, const fasgd_score_args& given, Score& s) {
    s = Score();
    s.u = given;
    fasgd_score_args& u = s.u;
    if (int rc = check_shape(call, u.rows, u.cols, FASGD_COLS_MAX, u.dtype)) return rc;
    if (u.rows >= (int64_t)1 << 31 || u.classes < 1 || u.classes > FASGD_CLASSES_MAX)
        return fail(FASGD_EINVAL, "%s: rows must be below 2^31, classes in [1, 2^24]", call);
    if ((u.w_flip | u.dw_flip) & ~1) return fail(FASGD_EINVAL, "%s: w_flip and dw_flip are 0 or 1", call);
    s.size = dtype_size(u.dtype);
    s.grad = u.dz != nullptr || u.dw != nullptr;
    if (int rc = check_matrix(call, "z", u.z, u.ld_z, u.rows, u.cols, s.size)) return rc;
    const auto shape = [&](bool flip) { return flip ? u.classes : u.cols; };
    const auto width = [&](bool flip) { return flip ? u.cols : u.classes; };
    if (int rc = check_matrix(call, "w", u.w, u.ld_w, shape(u.w_flip), width(u.w_flip), s.size)) return rc;
    if (u.dz != nullptr)
        if (int rc = check_matrix(call, "dz", u.dz, u.ld_dz, u.rows, u.cols, s.size)) return rc;
    if (u.dw != nullptr)
        if (int rc = check_matrix(call, "dw", u.dw, u.ld_dw, shape(u.dw_flip), width(u.dw_flip), s.size)) return rc;
    if (u.labels == nullptr || !aligned(u.labels, 8))
        return fail(FASGD_EINVAL, "%s: labels must not be NULL, and 8-byte aligned", call);
    if (u.known & ~1) return fail(FASGD_EINVAL, "%s: known is 0 or 1", call);
    if (u.row_loss == nullptr || (u.known ? u.lse == nullptr || !s.grad : u.loss == nullptr))
        return fail(FASGD_EINVAL, "%s: loss and row_loss must not be NULL; what is known: row_loss, lse, and dz or dw", call);
    if (u.known) u.loss = nullptr;
    if (!aligned(u.loss, 4) || !aligned(u.row_loss, 4) || !aligned(u.lse, 4) || !aligned(u.upstream, 4))
        return fail(FASGD_EINVAL, "%s: loss, row_loss, lse and upstream must be 4-byte aligned", call);
    return FASGD_OK;
}

// A piece of n classes' part of dz, and its rows (or columns) of dw; q.a.p or q.out are the piece's.
Product product_of_g(const Score& s) {
    Product q = {};
    q.dtype = s.u.rows == 0 ? FASGD_F32 : s.planes ? FASGD_BF16 : s.u.dtype;      // no rows: no operands to describe
    q.planes = q.exact = s.planes;
    q.ending = fasgd::kStore;
    q.factor = 1.0f / s.factor;
    q.out_dtype = s.u.dtype;
    return q;
}
Product product_dz(const Score& s, int64_t n) {
    const fasgd_score_args& u = s.u;
    Product q = product_of_g(s);
    q.a = {s.w, s.ld_wc, 0, u.w_flip, s.plane_w, 4};
    q.b = {s.g, s.ld_g, 0, 1, s.plane_g, 3};
    q.m = u.cols;
    q.n = u.rows;
    q.k = n;
    if (s.dz_sum != nullptr) {
        q.out = s.dz_sum;
        q.ld_out = u.cols;
        q.step_split = u.rows * u.cols;
        q.live = s.first ? s.live : nullptr;
        q.live_of = fasgd::kLiveN;
        q.out_dtype = FASGD_F32;
        q.factor = 1.0f;
        q.add = 1;      // (a plan for sums that are read again)
    } else {
        q.out = u.dz;
        q.ld_out = u.ld_dz;
        q.scale = s.row_scale;
        q.by_n = 1;
    }
    return q;
}
Product product_dw(const Score& s, int64_t n) {
    const fasgd_score_args& u = s.u;
    Product q = product_of_g(s);
    const fasgd::Side zs = {s.z, s.ld_zc, 0, 1, s.plane_z, 4}, gs = {s.g, s.ld_g, 0, 0, s.plane_g, 3};
    q.a = u.dw_flip ? zs : gs;
    q.b = u.dw_flip ? gs : zs;
    q.m = u.dw_flip ? u.cols : n;
    q.n = u.dw_flip ? n : u.cols;
    q.k = u.rows;
    q.live = s.first ? s.live : nullptr;
    q.live_of = fasgd::kLiveK;
    q.ld_out = u.ld_dw;
    q.scale = s.share;
    return q;
}

int64_t lay_out(Score& s, char* base) {
    const fasgd_score_args& u = s.u;
    int64_t at = 0;
    const auto take = [&](int64_t bytes) {
        char* p = base + at;
        at += (bytes + 255) / 256 * 256;
        return p;
    };
    s.few = few_classes(u);
    if (s.few) {
        s.few_sums = reinterpret_cast<float*>(take(4 * few_blocks(u.rows)));
        s.few_dw = reinterpret_cast<float*>(take(u.dw != nullptr ? 4 * few_blocks(u.rows) * u.classes * u.cols : 0));
        return at;
    }
    s.planes = u.dtype == FASGD_F32 && fasgd::by_planes(u.rows, u.classes, u.cols);
    s.tile = u.dtype == FASGD_F32 && !s.planes ? fasgd::kPlainN : fasgd::statistics_tile(u.rows, u.classes);
    const int64_t tiles = (u.classes + s.tile - 1) / s.tile;
    // (512 rows are two tiles; of fewer none would be saved)
    s.first = (u.dtype != FASGD_F32 || s.planes) && u.rows > 512;
    if (s.first) {
        s.to_row = reinterpret_cast<int32_t*>(take(4 * u.rows));
        s.row_at = reinterpret_cast<int32_t*>(take(4 * u.rows));
        s.live = reinterpret_cast<int32_t*>(take(4));
        s.labels = reinterpret_cast<int64_t*>(take(8 * u.rows));
        s.loss_at = reinterpret_cast<float*>(take(4 * u.rows));
    }
    if (!u.known) {
        s.parts = reinterpret_cast<float2*>(take(8 * tiles * u.rows));
        s.at_label = reinterpret_cast<float*>(take(4 * u.rows));
    }
    s.lse = u.lse != nullptr && !s.first ? u.lse : reinterpret_cast<float*>(take(4 * u.rows));
    // Gradients' sums over rows need zeros where there is no label; 16-bit products, rows that
    // start on 16 bytes.
    s.z_copy = s.w_copy = nullptr;
    s.ld_zc = u.ld_z;
    s.ld_wc = u.ld_w;
    const auto fits = [&](const void* p, int64_t ld) {
        return !s.planes && (u.dtype == FASGD_F32 || fasgd::tile_side({p, ld, 0, 0, 0, 0}, 1));
    };
    const auto copy = [&](int64_t values, int64_t& plane) {
        plane = values;
        return take(s.planes ? 8 * values : values * s.size);
    };
    if (s.grad || s.first || !fits(u.z, u.ld_z)) {
        s.ld_zc = (u.cols + 7) / 8 * 8;
        s.z_copy = copy(u.rows * s.ld_zc, s.plane_z);
    }
    if (!fits(u.w, u.ld_w)) {
        s.ld_wc = ((u.w_flip ? u.cols : u.classes) + 7) / 8 * 8;
        s.w_copy = copy((u.w_flip ? u.classes : u.cols) * s.ld_wc, s.plane_w);
    }
    s.z = s.z_copy != nullptr ? s.z_copy : u.z;
    s.w = s.w_copy != nullptr ? s.w_copy : u.w;
    if (!s.grad) return at;
    s.share = reinterpret_cast<float*>(take(4));
    s.row_scale = reinterpret_cast<float*>(take(4 * u.rows));
    s.ld_g = (u.rows + 63) / 64 * 64;      // (a stage of rows)
    const int64_t g_size = s.planes ? 6 : s.size;
    const int64_t most = std::max<int64_t>(64, FASGD_SCORE_PIECE / std::max<int64_t>(1, s.ld_g * g_size));
    const int64_t pieces = (u.classes + most - 1) / most;
    s.piece = (u.classes + pieces - 1) / pieces;
    if (pieces > 1) s.piece = std::min(s.piece / 64 * 64 + 64, most / 64 * 64);
    s.plane_g = s.piece * s.ld_g;
    s.g = take(g_size * s.plane_g);
    s.factor = u.dtype == FASGD_F16 ? 16384.0f : 1.0f;
    int64_t parts = 0;
    s.dz_sum = nullptr;
    s.dz_parts = 1;
    if (u.dz != nullptr && u.rows > 0) {
        if (s.piece < u.classes || s.first) {
            s.dz_sum = reinterpret_cast<float*>(16);      // (that there is one counts)
            const Product q = product_dz(s, s.piece);
            if (q.dtype != FASGD_F32) s.dz_parts = fasgd::plan_tiles(q).splits;
            s.dz_sum = reinterpret_cast<float*>(take(4 * s.dz_parts * u.rows * u.cols));
        } else {
            parts = fasgd::part_values(product_dz(s, u.classes));
        }
    }
    // (a last piece may be shorter than the others and split otherwise)
    if (u.dw != nullptr && u.rows > 0)
        parts = std::max({parts, fasgd::part_values(product_dw(s, s.piece)),
                          fasgd::part_values(product_dw(s, u.classes - (u.classes - 1) / s.piece * s.piece))});
    s.sums = reinterpret_cast<float*>(take(4 * parts));
    return at;
}

// The piece's part of an operand or result by classes.
const void* at_class(const void* p, int64_t ld, bool flip, int64_t v, int64_t size) {
    return static_cast<const char*>(p) + (flip ? v * ld : v) * size;
}

cudaError_t run(const Score& s, cudaStream_t stream) {
    const fasgd_score_args& u = s.u;
    cudaError_t st = cudaSuccess;
    if (s.few) {
        FewArgs a = {u, s.few_sums, s.few_dw};
        return u.dtype == FASGD_F32 ? run_few<float>(a, stream)
               : u.dtype == FASGD_BF16 ? run_few<__nv_bfloat16>(a, stream) : run_few<__half>(a, stream);
    }
    if (s.first) {
        first_kernel<<<1, 1024, 0, stream>>>(s.u, s);
        if ((st = cudaGetLastError()) != cudaSuccess) return st;
    }
    const void *z = s.z, *w_all = s.w;
    const int64_t ld_z = s.ld_zc, ld_w = s.ld_wc;
    fasgd::Pack c = {};
    c.groups = 1;
    c.dtype_from = c.dtype_to = u.dtype;
    if (s.w_copy != nullptr) {
        c.from = u.w;
        c.to = s.w_copy;
        c.rows = u.w_flip ? u.classes : u.cols;
        c.cols = u.w_flip ? u.cols : u.classes;
        c.ld_from = u.ld_w;
        c.ld_to = s.ld_wc;
        c.plane = s.planes ? s.plane_w : 0;
        if ((st = fasgd::launch_pack(c, stream)) != cudaSuccess) return st;
    }
    if (s.z_copy != nullptr) {
        c.from = u.z;
        c.to = s.z_copy;
        c.rows = u.rows;
        c.cols = u.cols;
        c.ld_from = u.ld_z;
        c.ld_to = s.ld_zc;
        c.plane = s.planes ? s.plane_z : 0;
        c.labels = u.labels;
        c.classes = u.classes;
        c.to_row = s.first ? s.to_row : nullptr;
        if ((st = fasgd::launch_pack(c, stream)) != cudaSuccess) return st;
    }
    Product p = {};
    p.a = {z, ld_z, 0, 0, s.plane_z, 4};
    p.b = {w_all, ld_w, 0, !u.w_flip, s.plane_w, 4};
    p.m = u.rows;
    p.n = u.classes;
    p.k = u.cols;
    const int32_t dtype = u.rows > 0 && s.planes ? FASGD_BF16 : u.rows > 0 ? u.dtype : FASGD_F32;      // no rows: no operands to describe
    p.dtype = dtype;
    p.planes = s.planes;
    p.ending = fasgd::kStatistics;
    // The log-sum-exps and losses are fp32.  A row's own g, which for a row that is nearly sure of its
    // label is a small difference, is taken from its loss, exp(-row_loss) - 1; in the others an s that is
    // off by 2^-16 of itself, as one accumulator of up to 2,048 columns leaves it, is lost in g's rounding to 16
    // bits while |s| is below some 30 (fp16) or 100 (bf16).  Rows of more columns go on in exact parts.
    p.exact = 1;
    p.live = s.first ? s.live : nullptr;
    p.live_of = fasgd::kLiveM;
    p.labels = s.first ? s.labels : u.labels;
    p.classes = u.classes;
    p.parts = s.parts;
    p.at_label = s.at_label;
    p.lse = s.lse;
    p.row_loss = s.first ? s.loss_at : u.row_loss;
    if (!u.known && u.rows > 0) {
        st = fasgd::launch_product(p, nullptr, stream);
        if (st != cudaSuccess) return st;
        const auto launch = u.rows >= 4096 ? launch_lse<32> : u.rows >= 64 ? launch_lse<8> : launch_lse<1>;
        st = launch(s, stream);
        if (st != cudaSuccess) return st;
    }
    loss_kernel<<<1, 1024, 0, stream>>>(u.rows, u.labels, u.classes, u.row_loss, u.upstream, u.loss, s.share, s.row_scale);
    if ((st = cudaGetLastError()) != cudaSuccess || !s.grad) return st;

    for (int64_t v = 0; v < u.classes; v += s.piece) {
        const int64_t n = std::min(s.piece, u.classes - v);
        const void* w = at_class(w_all, ld_w, u.w_flip, v, s.planes ? 2 : s.size);
        p.b.p = w;
        p.n = n;
        p.n0 = v;
        p.ending = fasgd::kResidual;
        p.step_plane = s.plane_g;
        p.out = s.g;
        p.ld_out = s.ld_g;
        p.out_dtype = u.dtype;
        p.factor = s.factor;
        st = fasgd::launch_product(p, nullptr, stream);
        if (st != cudaSuccess) return st;
        if (u.dz != nullptr && u.rows > 0) {
            Product q = product_dz(s, n);
            q.a.p = w;
            if (s.dz_sum == nullptr) {
                st = fasgd::launch_product(q, s.sums, stream);
            } else {      // every piece in as many parts
                q.add = v > 0;
                st = q.dtype == FASGD_F32 ? fasgd::launch_plain(q, 1, stream)
                                          : fasgd::launch_tiles(q, {fasgd::plan_tiles(q).pair, s.dz_parts}, stream);
            }
            if (st != cudaSuccess) return st;
        }
        if (u.dw != nullptr) {
            Product q = product_dw(s, n);
            q.dtype = dtype;
            q.out = const_cast<void*>(at_class(u.dw, u.ld_dw, u.dw_flip, v, s.size));
            st = fasgd::launch_product(q, s.sums, stream);
            if (st != cudaSuccess) return st;
        }
    }
    if (s.dz_sum != nullptr && u.rows > 0) {
        Product q = product_dz(s, s.piece);
        q.out = u.dz;
        q.ld_out = u.ld_dz;
        q.out_dtype = u.dtype;
        q.add = 0;
        q.scale = s.row_scale;
        q.by_n = 1;
        q.factor = 1.0f / s.factor;
        q.row_of = s.first ? s.to_row : nullptr;
        st = fasgd::launch_fold(q, s.dz_sum, u.rows * u.cols, s.dz_parts, stream);
    }
    return st;
}

}  // namespace

extern "C" {

int64_t fasgd_score_workspace(const fasgd_score_args* u) {
    const char* call = "fasgd_score_workspace";
    if (u == nullptr) {
        fail(FASGD_EINVAL, "%s: no arguments", call);
        return -1;
    }
    Score s;
    if (fill_score(call, *u, s) != FASGD_OK) return -1;
    return lay_out(s, nullptr);
}

int fasgd_score(const fasgd_score_args* u, void* stream) {
    const char* call = "fasgd_score";
    if (u == nullptr) return fail(FASGD_EINVAL, "%s: no arguments", call);
    Score s;
    if (int rc = fill_score(call, *u, s)) return rc;
    const int64_t need = lay_out(s, static_cast<char*>(u->workspace));
    if (need > 0 && (u->workspace == nullptr || !aligned(u->workspace, 256) || u->workspace_bytes < need))
        return fail(FASGD_EINVAL, "%s: workspace must be 256-byte aligned and hold %lld bytes", call, (long long)need);
    const auto classes = [&](const char* name, const void* p, bool flip, int64_t ld, bool output) {
        return Region{name, p, flip ? u->classes : u->cols, (flip ? u->cols : u->classes) * s.size, ld * s.size, output};
    };
    const Region r[] = {{"z", u->z, u->rows, u->cols * s.size, s.u.ld_z * s.size, false},
                        classes("w", u->w, u->w_flip, s.u.ld_w, false),
                        block("labels", u->labels, 8 * u->rows, false),
                        block("upstream", u->upstream, 4, false),
                        block("loss", s.u.loss, 4, true),
                        block("row_loss", u->row_loss, 4 * u->rows, !u->known),
                        block("lse", u->lse, 4 * u->rows, !u->known),
                        {"dz", u->dz, u->rows, u->cols * s.size, s.u.ld_dz * s.size, true},
                        classes("dw", u->dw, u->dw_flip, s.u.ld_dw, true),
                        block("workspace", u->workspace, u->workspace_bytes, true)};
    if (int rc = check_shared(call, r, sizeof r / sizeof r[0])) return rc;
    return cuda_status(run(s, static_cast<cudaStream_t>(stream)), call);
}

}  // extern "C"
