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

// Which elements of octet q are kept, a bit each.  A half is kept iff >= cut;
// shifted to the top of its word that is > (cut << 16) - 1 (cut 65536: never).
__device__ __forceinline__ uint32_t kept_bits(const DropArgs& d, int64_t q) {
    const Philox4 r = draw_octet(d, q);
    const uint32_t last = (d.cut << 16) - 1u;
    uint32_t bits = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        bits |= (r.x[w] << 16) > last ? 1u << (2 * w) : 0u;
        bits |= r.x[w] > last ? 2u << (2 * w) : 0u;
    }
    return bits;
}
__device__ __forceinline__ float2 select2(uint32_t bits, int pair, float2 v) {
    return make_float2((bits >> (2 * pair) & 1) ? v.x : 0.f, (bits >> (2 * pair + 1) & 1) ? v.y : 0.f);
}

// ---- loads into shared memory -------------------------------------------------
// Each thread copies its own octets ahead, into places that it alone reads, so
// the pipeline needs no barrier and no wait that could run out.
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
// Octet c of a row that begins at `row`, of which the matrix holds `left` values
// from the octet's start on (what lies behind its end is not read; zeros).
template <class T>
__device__ __forceinline__ void copy_octet(uint4* slot, int stride, const T* row, const Columns& c, int64_t left) {
    const T* p = row + c.c0;
#pragma unroll
    for (int k = 0; k < kPieces<T>; ++k) {
        constexpr int kPer = 16 / (int)sizeof(T);
        const int64_t l = left - k * kPer;
        const int n = l >= kPer ? kPer : l > 0 ? (int)l : 0;
        copy_async16(slot + k * stride, n > 0 ? p + k * kPer : p, n * (int)sizeof(T));
    }
}
template <class T>
__device__ __forceinline__ Oct take_octet(const uint4* slot, int stride, const Columns& c) {
    uint4 raw[kPieces<T>];
#pragma unroll
    for (int k = 0; k < kPieces<T>; ++k) raw[k] = slot[k * stride];
    Oct o = unpack<T>(raw);
    mask(o, c);
    return o;
}
template <class T>
__device__ __forceinline__ void store_octet(T* row, const Columns& c, Oct& o) {
    if (c.whole()) {
        uint4 raw[kPieces<T>];
        pack<T>(o, raw);
#pragma unroll
        for (int k = 0; k < kPieces<T>; ++k) reinterpret_cast<uint4*>(row + c.c0)[k] = raw[k];
        return;
    }
#pragma unroll
    for (int i = 0; i < kOctet; ++i)
        if (c.in >> i & 1) row[c.c0 + i] = from_f32<T>(element(o, i));
}

// Sums of N values over the TPR threads of a row, every thread ending with them.
// Rows of more than a warp meet at a barrier of their own; `red` has two places
// that are used in turn, so that one barrier a sum is enough.
template <int TPR, int N>
struct RowSums {
    static constexpr int kWarps = TPR / 32;
    float* red;          // [2][N][kWarps] of this row's threads
    int barrier, turn;
    __device__ RowSums(float* smem, int sub) : red(smem + sub * 2 * N * kWarps), barrier(1 + sub), turn(0) {}
    template <int M>
    __device__ __forceinline__ void operator()(float (&v)[M]) {
        static_assert(M <= N, "places");
#pragma unroll
        for (int i = 0; i < M; ++i) {
#pragma unroll
            for (int off = (TPR < 32 ? TPR : 32) / 2; off > 0; off >>= 1)
                v[i] += __shfl_xor_sync(0xffffffffu, v[i], off);
        }
        if constexpr (TPR > 32) {
            float* at = red + turn * N * kWarps;
            turn ^= 1;
            const int warp = (threadIdx.x % TPR) >> 5;
            if ((threadIdx.x & 31) == 0) {
#pragma unroll
                for (int i = 0; i < M; ++i) at[i * kWarps + warp] = v[i];
            }
            asm volatile("bar.sync %0, %1;" ::"r"(barrier), "n"(TPR) : "memory");
#pragma unroll
            for (int i = 0; i < M; ++i) {
                float s = 0.f;
#pragma unroll
                for (int w = 0; w < kWarps; ++w) s += at[i * kWarps + w];
                v[i] = s;
            }
        }
    }
};

// Octets that a row of `cols` values touches at most.
inline int64_t row_octets(int64_t cols) {
    int64_t most = 0;              // the largest r * cols mod 8
    for (int r = 0; r < 8; ++r) most = r * cols % 8 > most ? r * cols % 8 : most;
    return (most + cols + 7) / 8;
}
// Whether a matrix (an absent one: yes) can be moved in octets.
inline bool octet_matrix(const void* p, int64_t ld, int64_t rows, int64_t cols) {
    if (p == nullptr) return true;
    if (reinterpret_cast<uintptr_t>(p) & 15) return false;
    return rows < 2 || ld == cols || (cols % 8 == 0 && ld % 8 == 0);
}

}  // namespace
}  // namespace fasgd
