// Matrix products of the client operators (experts.cu and score.cu lay them out;
// product.cu and tile.cu hold the kernels).
//
//   D[m, n] = sum_k A[m, k] B[n, k]
//
// m is the index that is consecutive where the result is stored, so that the lanes of a
// warp, which hold consecutive m, write consecutive memory whatever the product.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace fasgd {

// One side of a product.  Element (i, k): i * ld + k, or (across) k * ld + i; group g of
// several is step values further on.
struct Side {
    const void* p;
    int64_t ld, step;
    int32_t across;
    int64_t plane;      // fp32 values in bf16 planes: from one of them to the next (launch_tiles)
    int32_t planes;     // how many: 4, or 3 of values that are finite or reach only results that are NaN
};

enum Ragged {
    kNotRagged,
    kRaggedN,    // n counts rows of all groups: group g has offsets[g] <= n < offsets[g + 1], B and D go by them, A by groups
    kRaggedK,    // so does k: A and B go by rows, D by groups
};
enum Live { kLiveM, kLiveN, kLiveK };
enum Ending {
    kStore,      // D, times scale where there is one, into out
    kStatistics, // of the values s = D over n: each tile's maximum and sum of exp(s - maximum), and s[m, label m]
    kResidual,   // exp(s - lse m), for n = label m exp(-row_loss m) - 1, 0 where m has no label, times `factor`, into out
};

struct Product {
    Side a, b;
    int64_t m, n, k;
    int32_t groups;              // ragged products
    const int32_t* offsets;      // int32[groups + 1] on the device
    int32_t ragged;              // enum Ragged
    int32_t dtype;               // of A and B (enum fasgd_dtype)
    int32_t ending;              // enum Ending
    // kStore, kResidual: element (m, n) of group g is out[g * step_out + n * ld_out + m]
    void* out;
    int64_t ld_out, step_out;
    int64_t step_split;          // launch_tiles: from one part of k's sums to the next
    int64_t step_plane;          // kResidual of planes: from one to the next
    int32_t planes;              // the sides are fp32 values in planes of dtype FASGD_BF16
    int32_t out_dtype;
    int32_t exact;               // sums to fp32's accuracy (launch_tiles: the tensor cores' additions cut bits off)
    int32_t add;                 // kStore, fp32: out += instead
    const float* scale;          // kStore: one value, or (by_n) one for each n, whose 0 makes its values 0
    int32_t by_n;
    float factor;                // kStore, kResidual: a power of two, on top
    // Where not all of m, n or k take part, how many do is known on the device (null: all).  What lies
    // behind them in the sides is 0 as far as a stage reaches.
    const int32_t* live;
    int32_t live_of;             // enum Live
    const int32_t* row_of;       // launch_fold: n's sums are those of row_of[n] (null: of n)
    // kStatistics, kResidual
    const int64_t* labels;       // [m]
    float2* parts;               // [n tiles][m]: kStatistics
    float* at_label;             // [m]: kStatistics
    const float *lse, *row_loss; // [m]: kResidual
    int64_t n0, classes;         // the first n of this piece, and how many there are of all pieces
};

// fp32 of any layout and size on the ordinary cores.  kPlainN: the n of a tile.
constexpr int kPlainN = 64;
cudaError_t launch_plain(const Product& p, int32_t splits, cudaStream_t stream);
// Parts of k that fill the SMs where there are few tiles: a stage of 32 k takes a block alone some 1.5 us
// of latency, however little there is to do (12 rows by 2,036 x 34: 100 us in one part).
int32_t plain_splits(const Product& p);

// 16-bit types on the tensor cores, for sides that start and step on 16 bytes.  kTileN: the n of a tile.
//
// fp32 values take part as three bf16 ones each (rounded, then what is left, twice: x = x0 + x1 + x2 to
// 2^-27), in the six products of them that reach 2^-26:
// x2 y0, x0 y2, x1 y1, x1 y0, x0 y1, x0 y0.
// An infinity is x0 alone, and may meet the other's largest part only: with the others, which are 0 or of either
// sign, it would make NaN of an infinite result.  So there is a fourth plane, x0 where it is finite and else 0,
// for the products with smaller parts.  (It is copied like the others, 8 bytes a value and not 6.)
constexpr int kTileN = 256;
constexpr int kPairs = 6;
constexpr double kPlanesFrom = 1 << 28;
// The planes of each pair, 4 bits a pair from the lowest on.
constexpr uint32_t planes_a(int32_t planes) { return planes == 4 ? 0x031132u : 0x001102u; }
constexpr uint32_t planes_b(int32_t planes) { return planes == 4 ? 0x013123u : 0x010120u; }
bool tile_side(const Side& s, int64_t groups);
// n of a tile of statistics.  A few rows' classes are one tile each of 152 SMs at a time: the width that
// takes the least rounds times width (131,072 classes: four of 256 or of 224).
inline int32_t statistics_tile(int64_t m, int64_t n) {
    int32_t best = kTileN;
    if (m <= 128)
        for (int32_t width = kTileN; width >= 192; width -= 16) {
            const auto cost = [&](int32_t w) { return ((n + w - 1) / w + 151) / 152 * w; };
            if (cost(width) < cost(best)) best = width;
        }
    return best;
}
// How a product falls to the SMs: blocks or pairs of them, parts of k's sums.
struct TilePlan {
    int32_t pair, splits;
};
TilePlan plan_tiles(const Product& p);      // by sizes alone
cudaError_t launch_tiles(const Product& p, const TilePlan& plan, cudaStream_t stream);
// ns without a copy after which a launch's waits give up, of launches from now on (10^9 before the first call).
void set_wait_limit(uint64_t ns);
// Waits for the stream; whether a launch's wait ran out on this device since the last call.
cudaError_t read_late(int32_t* late, cudaStream_t stream);
cudaError_t launch_expiry(cudaStream_t stream);      // a kernel whose waits run out
// out = the sum of `count` parts, `step` values apart, each [groups of ragged k][n][m], as p stores it.
cudaError_t launch_fold(const Product& p, const float* parts, int64_t step, int32_t count, cudaStream_t stream);
// The values of the parts that launch_product needs room for.
inline int64_t part_values(const Product& p) {
    if (p.ending != kStore) return 0;
    const int64_t splits = p.dtype == 0 ? plain_splits(p) : plan_tiles(p).splits;
    return splits > 1 ? splits * p.n * p.m * (p.ragged == kRaggedK ? p.groups : 1) : 0;
}
// Whether an fp32 product of m x n x k goes by planes: from where copies and launches of theirs are made
// up for.  Measured on both sides: y of 128 x 128 x 128 11 us plain and 13 by planes; of 1,024 rows by 512 x 512 in 4
// experts (2^28) 31 and 25, of 1,024 x 1,024 x 1,024 104 and 29, of 512 rows by 1,024 x 1,024 in 128 experts, where the
// copies are of 134 million values for 2^29 multiply-adds, 692 and 472; a score of 512 x 512 x 2,048 with gradients
// 244 and 110.
inline bool by_planes(int64_t m, int64_t n, int64_t k) {
    return (double)m * (double)n * (double)k >= kPlanesFrom;
}
// What is of fp32 still when it gets here takes the plain form; its callers copy sides of large fp32
// products to planes, and lay out 16-bit ones for the tensor cores.
// parts: room for part_values().
inline cudaError_t launch_product(const Product& p, float* parts, cudaStream_t stream) {
    const bool plain = p.dtype == 0;
    const TilePlan plan = plain ? TilePlan{1, plain_splits(p)} : plan_tiles(p);
    if (part_values(p) == 0)
        return plain ? launch_plain(p, 1, stream) : launch_tiles(p, {plan.pair, 1}, stream);
    Product q = p;
    q.out = parts;
    q.out_dtype = 0;
    q.ld_out = p.m;
    q.step_out = p.n * p.m;
    q.step_split = q.step_out * (p.ragged == kRaggedK ? p.groups : 1);
    q.scale = nullptr;
    q.by_n = 0;
    q.factor = 1.0f;
    const cudaError_t st = plain ? launch_plain(q, plan.splits, stream) : launch_tiles(q, plan, stream);
    return st != cudaSuccess ? st : launch_fold(p, parts, q.step_split, plan.splits, stream);
}

// A copy of a side with rows that lie as the fast kernels want them: `rows` rows of `cols`
// values (of group g: p + g * step) to rows ld_to apart (a multiple of 8, as step_to and plane; what is
// between the rows is overwritten), of the same type or rounded from fp32.  Groups without rows by
// offsets (null: there are none) are not read or written; the copy of a row without a label (labels
// null: all have one) is 0 whatever the row holds.
struct Pack {
    const void* from;
    void* to;
    int64_t rows, cols, ld_from, step_from, ld_to, step_to;
    int32_t groups, dtype_from, dtype_to;
    int64_t plane;               // fp32 to FASGD_BF16 in four planes this far apart; 0: one value each
    const int32_t* offsets;
    const int64_t* labels;
    int64_t classes;
    const int32_t* to_row;       // row r goes to row to_row[r] (null: r)
};
cudaError_t launch_pack(const Pack& p, cudaStream_t stream);

#ifdef __CUDACC__
// The three parts of an fp32 value.  A value that would round to infinity in bf16 is cut instead; what is
// not finite is its first part alone.
__device__ __forceinline__ void planes_of(float x, __nv_bfloat16 (&to)[3]) {
    const bool finite = fabsf(x) <= 3.4028234e38f;
    to[0] = __float2bfloat16_rn(fabsf(x) < 3.38e38f || !finite ? x : __uint_as_float(__float_as_uint(x) & 0xffff0000u));
    const float rest = finite ? x - __bfloat162float(to[0]) : 0.0f;
    to[1] = __float2bfloat16_rn(rest);
    to[2] = __float2bfloat16_rn(rest - __bfloat162float(to[1]));
}
#endif

// Group g's rows, cut to [0, n).
struct Bounds {
    int64_t lo, hi;
};
__device__ __forceinline__ Bounds group_bounds(const int32_t* offsets, int g, int64_t n) {
    const int64_t lo = min(max((int64_t)offsets[g], (int64_t)0), n);
    return {lo, min(max((int64_t)offsets[g + 1], lo), n)};
}

}  // namespace fasgd
