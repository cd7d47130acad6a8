// Rows in octets: the fast kernels of the client operators give every thread the
// same eight columns of all the rows it takes, and move them 16 bytes at a time.
//
// Octets are cut where memory and the draws cut them: at multiples of eight
// values of the (gapless) matrix.  Where cols is no multiple of 8, row r begins
// s = r * cols mod 8 values into its first octet, so a thread's columns would
// move from row to row; rows whose numbers agree modulo 8 share s, and a thread
// takes only such rows.  The octets at a row's ends then hold a neighbour's values
// too, which are loaded, set to zero and not stored.
#pragma once

#include "client.cuh"
#include "clip.cuh"
#include "shared_limit.cuh"

namespace fasgd {
namespace {

constexpr int kOctet = 8;

struct Oct {
    float2 v[4];
};
// 16-byte pieces of an octet.
template <class T>
constexpr int kPieces = (int)sizeof(T) / 2;

__device__ __forceinline__ float2 f2(float x) { return make_float2(x, x); }
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) { return __ffma2_rn(a, b, c); }
__device__ __forceinline__ float2 mul2(float2 a, float2 b) { return __fmul2_rn(a, b); }
__device__ __forceinline__ float2 add2(float2 a, float2 b) { return __fadd2_rn(a, b); }

__device__ __forceinline__ float2 unpack2(uint32_t w, __nv_bfloat16) {
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
__device__ __forceinline__ float2 unpack2(uint32_t w, __half) {
    return __half22float2(*reinterpret_cast<const __half2*>(&w));
}
template <class T>
__device__ __forceinline__ Oct unpack(const uint4 (&p)[kPieces<T>]) {
    Oct o;
    if constexpr (sizeof(T) == 4) {
        o.v[0] = make_float2(__uint_as_float(p[0].x), __uint_as_float(p[0].y));
        o.v[1] = make_float2(__uint_as_float(p[0].z), __uint_as_float(p[0].w));
        o.v[2] = make_float2(__uint_as_float(p[1].x), __uint_as_float(p[1].y));
        o.v[3] = make_float2(__uint_as_float(p[1].z), __uint_as_float(p[1].w));
    } else {
        o.v[0] = unpack2(p[0].x, T());
        o.v[1] = unpack2(p[0].y, T());
        o.v[2] = unpack2(p[0].z, T());
        o.v[3] = unpack2(p[0].w, T());
    }
    return o;
}
__device__ __forceinline__ uint32_t pack2(float2 v, __nv_bfloat16) {
    const __nv_bfloat162 h = __float22bfloat162_rn(v);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t pack2(float2 v, __half) {
    const __half2 h = __float22half2_rn(v);
    return *reinterpret_cast<const uint32_t*>(&h);
}
template <class T>
__device__ __forceinline__ void pack(const Oct& o, uint4 (&p)[kPieces<T>]) {
    if constexpr (sizeof(T) == 4) {
        p[0] = make_uint4(__float_as_uint(o.v[0].x), __float_as_uint(o.v[0].y), __float_as_uint(o.v[1].x),
                          __float_as_uint(o.v[1].y));
        p[1] = make_uint4(__float_as_uint(o.v[2].x), __float_as_uint(o.v[2].y), __float_as_uint(o.v[3].x),
                          __float_as_uint(o.v[3].y));
    } else {
        p[0] = make_uint4(pack2(o.v[0], T()), pack2(o.v[1], T()), pack2(o.v[2], T()), pack2(o.v[3], T()));
    }
}
__device__ __forceinline__ float& element(Oct& o, int i) { return (i & 1) ? o.v[i >> 1].y : o.v[i >> 1].x; }

// A thread's columns: c0 .. c0+7, of which bit i of `in` says that c0 + i is one.
struct Columns {
    int32_t c0;
    uint32_t in;
    Columns() = default;
    __device__ Columns(int octet, int shift, int32_t cols) {
        c0 = octet * kOctet - shift;
        in = 0;
        if (c0 < cols && c0 + kOctet > 0) {
            in = 0xffu;
            if (c0 < 0) in &= 0xffu << -c0;
            if (c0 + kOctet > cols) in &= 0xffu >> (c0 + kOctet - cols);
        }
    }
    __device__ bool any() const { return in != 0; }
    __device__ bool whole() const { return in == 0xffu; }
};
// Zeros in the places of a neighbour's values.
__device__ __forceinline__ void mask(Oct& o, const Columns& c) {
    if (c.whole()) return;
#pragma unroll
    for (int i = 0; i < kOctet; ++i)
        if (!(c.in >> i & 1)) element(o, i) = 0.f;
}

// Eight of a vector's values (none: `fill`), 0 where there is no column.
__device__ __forceinline__ Oct load_vector(const float* p, const Columns& c, float fill) {
    Oct o;
    if (p != nullptr && c.whole() && (reinterpret_cast<uintptr_t>(p + c.c0) & 15) == 0) {
        const float4 a = *reinterpret_cast<const float4*>(p + c.c0);
        const float4 b = *reinterpret_cast<const float4*>(p + c.c0 + 4);
        o.v[0] = make_float2(a.x, a.y);
        o.v[1] = make_float2(a.z, a.w);
        o.v[2] = make_float2(b.x, b.y);
        o.v[3] = make_float2(b.z, b.w);
        return o;
    }
#pragma unroll
    for (int i = 0; i < kOctet; ++i) {
        const bool in = c.in >> i & 1;
        element(o, i) = !in ? 0.f : p != nullptr ? p[c.c0 + i] : fill;
    }
    return o;
}
// Eight of the gate's values of one group (no gate: 1).
template <class T>
__device__ __forceinline__ Oct load_gate(const JoinArgs& a, int64_t group, const Columns& c) {
    if (a.gate == nullptr || a.gate_f32)
        return load_vector(a.gate == nullptr ? nullptr : static_cast<const float*>(a.gate) + group * a.cols, c, 1.f);
    const T* p = static_cast<const T*>(a.gate) + group * a.cols;
    if (c.whole() && (reinterpret_cast<uintptr_t>(p + c.c0) & 15) == 0) {
        uint4 raw[kPieces<T>];
#pragma unroll
        for (int k = 0; k < kPieces<T>; ++k) raw[k] = reinterpret_cast<const uint4*>(p + c.c0)[k];
        return unpack<T>(raw);
    }
    Oct o;
#pragma unroll
    for (int i = 0; i < kOctet; ++i) element(o, i) = (c.in >> i & 1) ? to_f32(p[c.c0 + i]) : 0.f;
    return o;
}

// Pair i of an octet, 0 where dropped.  A half is kept iff >= cut; shifted to the
// top of its word that is > last = (cut << 16) - 1 (cut 65536: never).
__device__ __forceinline__ float2 keep2(const Philox4& r, int i, uint32_t last, float2 v) {
    return make_float2((r.x[i] << 16) > last ? v.x : 0.f, r.x[i] > last ? v.y : 0.f);
}

// ---- loads into shared memory -------------------------------------------------
// A warp copies its own octets ahead, into places that it alone reads, so the
// pipeline needs no barrier of the block and no wait that could run out.  Of an
// fp32 octet's two pieces a lane copies those that make a warp's copies contiguous
// (each owner's own would touch every 32-byte sector twice); so a lane reads what
// others copied, after the wait and a __syncwarp.
constexpr int kLane = 32;          // 16-byte places of one piece of a warp's octets
__device__ __forceinline__ void copy_async16(void* smem, const void* global, int bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(smem)),
                 "l"(global), "r"(bytes)
                 : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
// The pieces that a lane copies of a row that W lanes of its warp hold, the first
// of them from column c0 on: from column col + k * kStep on, if bit k of `in`.
template <class T, int W>
struct CopyLane {
    static constexpr int kPer = 16 / (int)sizeof(T), kStep = W * kPer;
    int32_t col, cols;
    uint32_t in;
    int place;          // the lane
    CopyLane() = default;
    __device__ CopyLane(const Columns& c, int32_t cols_) : cols(cols_), in(0) {
        const int lane = threadIdx.x & 31, of_row = lane % W;
        col = __shfl_sync(0xffffffffu, c.c0, 0, W) + of_row * kPer;
        place = lane;
#pragma unroll
        for (int k = 0; k < kPieces<T>; ++k)
            if (col + k * kStep + kPer > 0 && col + k * kStep < cols) in |= 1u << k;
    }
    // Piece k * W + i of the row (i: this lane of it) belongs to the lane of octet
    // (k W + i) / 2; second pieces lie four places off, so that the copies of
    // eight neighbours fall into all banks.
    __device__ __forceinline__ int place_of(int k) const {
        if (kPieces<T> == 1) return place;
        const int i = place % W, piece = k * W + i, owner = place - i + (piece >> 1);
        return (piece & 1) * kLane + (owner ^ (4 * (piece & 1)));
    }
    // p: the row's first value, `col` on.  behind: what the matrix has behind the row
    // (clip.cuh); past its end nothing is read (zeros).
    __device__ __forceinline__ void copy(uint4* slot, const T* p, int32_t behind) const {
#pragma unroll
        for (int k = 0; k < kPieces<T>; ++k) {
            if (!(in >> k & 1)) continue;
            uint4* to = slot + place_of(k);
            copy_async16(to, p + k * kStep, values_there(col + k * kStep, cols, behind, kPer) * (int)sizeof(T));
        }
    }
};
// Matrices of any alignment and step ("loose"): a warp copies the 16-byte granules
// that hold its columns of a row, col_lo .. col_hi, and a lane reads its octet at
// whatever byte it begins.  Two granules lie free before the data, for the values
// before a row's first that an octet spans.  32768 x 1024 bf16 rows three values
// apart: 70 us forward, 130 us gradients; without gaps 42 and 76.
template <class T>
struct LooseRow {
    static constexpr int kPlace = kLane * kPieces<T> + 4;       // 16-byte places of a warp's matrix
    int32_t col_lo, col_hi;
    __device__ LooseRow(const Columns& c, int32_t cols) {
        const int32_t c0 = __shfl_sync(0xffffffffu, c.c0, 0);
        col_lo = c0 > 0 ? c0 : 0;
        col_hi = c0 + 32 * kOctet < cols ? c0 + 32 * kOctet : cols;
    }
    // row: the row's first value; base: the matrix's.  What lies before base or
    // behind col_hi is not read.
    __device__ __forceinline__ void copy(uint4* slot, const T* row, const void* base) const {
        if (col_lo >= col_hi) return;
        const uintptr_t from = reinterpret_cast<uintptr_t>(row + col_lo) & ~(uintptr_t)15;
        const uintptr_t end = reinterpret_cast<uintptr_t>(row + col_hi);
#pragma unroll
        for (int k = 0; k <= kPieces<T>; ++k) {
            const int g = k * 32 + (threadIdx.x & 31);
            const uintptr_t p = from + (uintptr_t)g * 16;
            if (g > 32 * kPieces<T> || p >= end) continue;
            if (p >= reinterpret_cast<uintptr_t>(base)) {
                copy_async16(slot + 2 + g, reinterpret_cast<const void*>(p), end - p < 16 ? (int)(end - p) : 16);
            } else {                       // the matrix begins inside this granule
                T* to = reinterpret_cast<T*>(slot + 2 + g);
                const T* v = reinterpret_cast<const T*>(p);
                for (int i = 0; i < 16 / (int)sizeof(T); ++i)
                    if (reinterpret_cast<uintptr_t>(v + i) >= reinterpret_cast<uintptr_t>(base) &&
                        reinterpret_cast<uintptr_t>(v + i) < end)
                        to[i] = v[i];
            }
        }
    }
    // start: the address of the row's column col_lo (its low bits).
    __device__ __forceinline__ Oct take(const uint4* slot, uint32_t start, const Columns& c) const {
        Oct o = {};
        if (!c.any()) return o;
        const int at = 32 + (int)(start & 15) + (c.c0 - col_lo) * (int)sizeof(T);
        const uint32_t* w = reinterpret_cast<const uint32_t*>(reinterpret_cast<const char*>(slot) + (at & ~3));
        uint4 raw[kPieces<T>];
        if constexpr (sizeof(T) == 4) {
            raw[0] = make_uint4(w[0], w[1], w[2], w[3]);
            raw[1] = make_uint4(w[4], w[5], w[6], w[7]);
        } else {
            const uint32_t v[5] = {w[0], w[1], w[2], w[3], w[4]};
            const int shift = (at & 2) * 8;
            raw[0] = make_uint4(__funnelshift_r(v[0], v[1], shift), __funnelshift_r(v[1], v[2], shift),
                                __funnelshift_r(v[2], v[3], shift), __funnelshift_r(v[3], v[4], shift));
        }
        o = unpack<T>(raw);
        mask(o, c);
        return o;
    }
};
// Zeros in the places of an octet that nobody copies, of `count` matrices.
template <class T>
__device__ __forceinline__ void clear_octets(uint4* slot, int count) {
    for (int i = 0; i < count * kPieces<T>; ++i)
        slot[i * kLane + ((threadIdx.x & 31) ^ (4 * (i % kPieces<T>)))] = make_uint4(0, 0, 0, 0);
}
// slot: the warp's place of a matrix.
template <class T, bool RAGGED>
__device__ __forceinline__ Oct take_octet(const uint4* slot, const Columns& c) {
    uint4 raw[kPieces<T>];
#pragma unroll
    for (int k = 0; k < kPieces<T>; ++k) raw[k] = slot[k * kLane + ((threadIdx.x & 31) ^ (4 * k))];
    Oct o = unpack<T>(raw);
    if (RAGGED) mask(o, c);
    return o;
}
// p, `bytes` on.
template <class T>
__device__ __forceinline__ T* on(T* p, int64_t bytes) {
    return reinterpret_cast<T*>(reinterpret_cast<uintptr_t>(p) + (uintptr_t)bytes);
}
// A whole octet in one instruction: an fp32 one as 32 bytes.
__device__ __forceinline__ void store_pieces(void* p, const uint4 (&r)[1]) { *static_cast<uint4*>(p) = r[0]; }
__device__ __forceinline__ void store_pieces(void* p, const uint4 (&r)[2]) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(r[0].x), "r"(r[0].y),
                 "r"(r[0].z), "r"(r[0].w), "r"(r[1].x), "r"(r[1].y), "r"(r[1].z), "r"(r[1].w)
                 : "memory");
}
__device__ __forceinline__ void load_pieces(const void* p, uint4 (&r)[1]) { r[0] = *static_cast<const uint4*>(p); }
__device__ __forceinline__ void load_pieces(const void* p, uint4 (&r)[2]) {
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0].x), "=r"(r[0].y), "=r"(r[0].z), "=r"(r[0].w), "=r"(r[1].x), "=r"(r[1].y), "=r"(r[1].z),
                   "=r"(r[1].w)
                 : "l"(p)
                 : "memory");
}
// An octet to p on (the place of its first column, which may not be one);
// vectors: p is aligned to an octet.
template <class T, bool RAGGED>
__device__ __forceinline__ void store_octet(T* p, const Columns& c, Oct& o, bool vectors = true) {
    if (RAGGED ? c.whole() && vectors : c.any()) {
        uint4 raw[kPieces<T>];
        pack<T>(o, raw);
        store_pieces(p, raw);
        return;
    }
    if (RAGGED) {
#pragma unroll
        for (int i = 0; i < kOctet; ++i)
            if (c.in >> i & 1) p[i] = from_f32<T>(element(o, i));
    }
}

// Sums of N values over the threads of a row, every thread ending with them.  In a warp the values are halved among the lanes
// as they are added (four values: 6 shuffles, not 20).  Warps meet at a barrier of
// the block, or the cluster, having left their sums in its blocks' `red`, which
// has two places that are used in turn: one barrier for each use is enough.
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void store_to_block(float* p, uint32_t rank, float v) {
    uint32_t there;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;"
                 : "=r"(there)
                 : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(there), "f"(v) : "memory");
}
__device__ __forceinline__ void cluster_barrier() {
    asm volatile("barrier.cluster.arrive.release;\n barrier.cluster.wait.acquire;" ::: "memory");
}
constexpr int pow2_above(int n) { return n <= 1 ? 1 : n <= 2 ? 2 : n <= 4 ? 4 : 8; }
constexpr int kRowWarps = 32;       // of a block, that hold a row; times a cluster's blocks
constexpr int kCluster = 8;

// The threads of a row: a block's (TPR = 0, whole warps), or those of each block
// of a cluster; or TPR = 8 of a block of one warp, which then holds four rows.
template <int TPR>
struct RowThreads {
    int warps, sub, lane;           // in this block: of a row, which row's, which of them
    int rank, blocks;               // in the row's cluster
    __device__ explicit RowThreads(int blocks_) : warps(1), sub(0), lane(threadIdx.x), rank(0), blocks(1) {
        if constexpr (TPR == 8) {
            sub = threadIdx.x >> 3;
            lane = threadIdx.x & 7;
        } else {
            warps = blockDim.x >> 5;
            blocks = blocks_;
            if (blocks > 1) rank = (int)cluster_rank();
        }
    }
    __device__ int octet() const { return rank * (int)blockDim.x + lane; }
};
constexpr int kWarpRows = 4;       // of TPR = 8

template <int TPR, int N>
struct RowSums {
    static constexpr int kN = pow2_above(N), kLanes = 32 / kN;     // lanes that end with one value
    // Floats of shared memory: two places for each warp of a cluster's blocks (of 16 at most).
    static constexpr int kPlaces = TPR ? 1 : 2 * kN * (kRowWarps / 2) * kCluster;
    const RowThreads<TPR>& th;
    float* red;
    int warps, turn;
    __device__ RowSums(const RowThreads<TPR>& th_, float* smem) : th(th_), red(smem), warps(th_.warps * th_.blocks), turn(0) {
        if (TPR == 0 && th.blocks > 1) cluster_barrier();      // every block of the cluster has begun
    }
    __device__ __forceinline__ void operator()(float (&in)[N]) {
        if constexpr (TPR == 8) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
#pragma unroll
                for (int off = 4; off > 0; off >>= 1) in[i] += __shfl_xor_sync(0xffffffffu, in[i], off);
            }
        } else {
            const int lane = threadIdx.x & 31;
            float v[kN];
#pragma unroll
            for (int i = 0; i < kN; ++i) v[i] = i < N ? in[i] : 0.f;
            // A lane keeps the half of the values that its bits name.
#pragma unroll
            for (int n = kN / 2, off = 16; off > 0; off >>= 1, n >>= 1) {
                if (n >= 1) {
                    const bool upper = lane & off;
#pragma unroll
                    for (int i = 0; i < (n >= 1 ? n : 1); ++i) {
                        const float mine = upper ? v[i + n] : v[i], other = upper ? v[i] : v[i + n];
                        v[i] = mine + __shfl_xor_sync(0xffffffffu, other, off);
                    }
                } else {
                    v[0] += __shfl_xor_sync(0xffffffffu, v[0], off);
                }
            }
            if (warps > 1) {
                float* at = red + turn * kN * warps;
                turn ^= 1;
                float* place = at + lane / kLanes * warps + th.rank * th.warps + (threadIdx.x >> 5);
                if (th.blocks == 1) {
                    if (lane % kLanes == 0) *place = v[0];
                    __syncthreads();
                } else {
                    if (lane % kLanes == 0)
                        for (int k = 0; k < th.blocks; ++k) store_to_block(place, k, v[0]);
                    __syncwarp();
                    cluster_barrier();
                }
                float s = 0.f;
                const float* from = at + lane / kLanes * warps;
                const int w = lane % kLanes;
                if (warps <= 2 * kLanes) {
                    if (w < warps) s = from[w];
                    if (w + kLanes < warps) s += from[w + kLanes];
                } else {
                    for (int i = w; i < warps; i += kLanes) s += from[i];
                }
#pragma unroll
                for (int off = kLanes / 2; off > 0; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
                v[0] = s;
            }
#pragma unroll
            for (int i = 0; i < N; ++i) in[i] = kN == 1 ? v[0] : __shfl_sync(0xffffffffu, v[0], i * kLanes);
        }
    }
};

// How rows of so many octets lie in threads: `threads` of a block, which holds
// `rows` rows, or its part of one that `blocks` blocks of a cluster hold.
struct RowShape {
    int threads, rows, blocks;
    RowShape(int64_t octets, int most, bool loose) : rows(1), blocks(1) {    // most: threads of a row in one block
        if (octets <= 8 && !loose) {
            threads = 32;
            rows = kWarpRows;
            return;
        }
        while ((octets + blocks - 1) / blocks > most) blocks *= 2;
        threads = (int)((octets + 32 * blocks - 1) / (32 * blocks) * 32);
    }
    bool fits() const { return blocks <= kCluster && threads <= 32 * kRowWarps; }
};

// Octets that a row of `cols` values touches at most.
inline int64_t row_octets(int64_t cols) {
    int64_t most = 0;              // the largest r * cols mod 8
    for (int r = 0; r < 8; ++r) most = r * cols % 8 > most ? r * cols % 8 : most;
    return (most + cols + 7) / 8;
}
// Dynamic shared memory that any of these kernels can have: 227 KB less their own
// (4 KB at most); the largest call takes 207 KB.
constexpr int64_t kSharedMost = 220 * 1024;
// Programmatic dependent launch (pdl.cuh), of clusters of `cluster` blocks.  With
// the kernel's own, shared memory beyond 48 KB is to be asked for: once a device.
template <auto Kernel, class... Args>
cudaError_t launch_rows_kernel(int64_t grid, int block, size_t smem, int cluster, cudaStream_t stream, Args... args) {
    if (smem > 32 * 1024) {
        static SharedLimit limit;
        int dev = 0;
        cudaError_t st = cudaGetDevice(&dev);
        if (st != cudaSuccess) return st;
        st = (cudaError_t)limit.ensure(dev, (int64_t)smem, kSharedMost, [](int64_t bytes) {
            return (int)cudaFuncSetAttribute(Kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
        });
        if (st != cudaSuccess) return st;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3((unsigned)block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, Kernel, args...);
}

// How a call's rows are taken: in octets; in octets, from matrices that are not
// laid out for it; or value by value.
enum RowForm { kInOctets, kLoose, kValues };
// Whether a matrix (an absent one: yes) can be moved in octets.
inline bool octet_matrix(const void* p, int64_t ld, int64_t rows, int64_t cols, int size) {
    if (p == nullptr) return true;
    if (reinterpret_cast<uintptr_t>(p) % (kOctet * size)) return false;
    return rows < 2 || (cols % 8 == 0 ? ld % 8 == 0 : ld == cols);
}

}  // namespace
}  // namespace fasgd
