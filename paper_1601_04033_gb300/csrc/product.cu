// Matrix products of fp32 values in their simple form: 64 x 64 tiles of D in registers, 32
// steps of k through shared memory at a time, the next 32 read meanwhile.  Right for every layout,
// alignment and size; for products too small for planes (by_planes) also the fastest here: 11 us for
// 128 x 128 x 128, where planes take 13; at 1,024 x 1,024 x 1,024 it is 104 us (21 TFLOP/s) to 29.  At 242 registers
// a thread one block fits on an SM, whose eight warps leave its loads' latency exposed at every stage.
//
// Also here: the copies that lay sides out for the tensor cores, and the sums of parts of k.

#include <algorithm>

#include "client.cuh"
#include "pdl.cuh"
#include "product.cuh"

namespace fasgd {
namespace {

constexpr int kM = 64, kN = kPlainN, kK = 32;
constexpr int kSum = 256;                // k of a sum
constexpr int kEach = kM * kK / 256;     // values of a stage that a thread reads

__device__ __forceinline__ float element(const Side& s, int64_t group, int64_t i, int64_t k) {
    const float* p = static_cast<const float*>(s.p) + group * s.step;
    return s.across ? p[k * s.ld + i] : p[i * s.ld + k];
}
// Elements [i0, i0 + 64) x [k0, k0 + 32) of a side, 0 beyond [.., i1) and [.., k1): into
// registers, and from there to shared memory.
__device__ __forceinline__ void read(float (&v)[kEach], const Side& s, int64_t group, int64_t i0, int64_t i1, int64_t k0,
                                     int64_t k1) {
#pragma unroll
    for (int r = 0; r < kEach; ++r) {
        const int j = threadIdx.x + r * 256;
        const int i = s.across ? j % kM : j / kK, k = s.across ? j / kM : j % kK;
        v[r] = i0 + i < i1 && k0 + k < k1 ? element(s, group, i0 + i, k0 + k) : 0.0f;
    }
}
__device__ __forceinline__ void stage(float (&to)[kK][kM + 1], const float (&v)[kEach], bool across) {
#pragma unroll
    for (int r = 0; r < kEach; ++r) {
        const int j = threadIdx.x + r * 256;
        if (across)
            to[j / kM][j % kM] = v[r];
        else
            to[j % kK][j / kK] = v[r];
    }
}

__device__ __forceinline__ void put(const Product& p, int64_t group, int64_t m, int64_t n, float v) {
    const int64_t at = group * p.step_out + n * p.ld_out + m;
    if (p.out_dtype == FASGD_F32) {
        float* out = static_cast<float*>(p.out) + at;
        *out = p.add ? *out + v : v;
    } else if (p.out_dtype == FASGD_BF16) {
        static_cast<__nv_bfloat16*>(p.out)[at] = from_f32<__nv_bfloat16>(v);
    } else {
        static_cast<__half*>(p.out)[at] = from_f32<__half>(v);
    }
}

// The group and first n of the block's tile; false: there is no such tile.
__device__ bool find_tile(const Product& p, int64_t tile, int64_t& group, Bounds& rows) {
    const int lane = threadIdx.x & 31;
    int64_t before = 0;
    for (int g0 = 0; g0 < p.groups; g0 += 32) {
        Bounds b = {0, 0};
        if (g0 + lane < p.groups) b = group_bounds(p.offsets, g0 + lane, p.n);
        const int64_t tiles = (b.hi - b.lo + kN - 1) / kN;
        int64_t s = tiles;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int64_t o = __shfl_up_sync(0xffffffffu, s, d);
            if (lane >= d) s += o;
        }
        const uint32_t has = __ballot_sync(0xffffffffu, tile < before + s);
        if (has != 0) {
            const int first = __ffs(has) - 1;
            const int64_t begin = before + __shfl_sync(0xffffffffu, s - tiles, first);
            group = g0 + first;
            rows = {__shfl_sync(0xffffffffu, b.lo, first) + (tile - begin) * kN, __shfl_sync(0xffffffffu, b.hi, first)};
            return true;
        }
        before += __shfl_sync(0xffffffffu, s, 31);
    }
    return false;
}

// Parts of k's sums into a product's result, four values of m a thread (one at a time, with a division
// each, 78 MB of sums took 90 us).
template <class T>
__device__ __forceinline__ void put_four(const Product& p, int64_t at, int most, bool wide, const float (&v)[4]) {
    T* out = static_cast<T*>(p.out) + at;
    if (wide) {
        struct alignas(4 * sizeof(T)) Four {
            T v[4];
        } four;
#pragma unroll
        for (int j = 0; j < 4; ++j) four.v[j] = from_f32<T>(v[j]);
        *reinterpret_cast<Four*>(out) = four;
        return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (j < most) out[j] = from_f32<T>(v[j]);
}
__global__ void __launch_bounds__(256) fold_kernel(Product p, const float* parts, int64_t step, int32_t count, bool wide) {
    const int64_t g = blockIdx.y, fours = (p.m + 3) / 4, all = p.n * fours;
    pdl_wait();
    pdl_trigger();
    Bounds rows = {0, p.n};
    if (p.ragged == kRaggedN) rows = {group_bounds(p.offsets, 0, p.n).lo, group_bounds(p.offsets, p.groups - 1, p.n).hi};
    const float* from = parts + g * p.n * p.m;
    const float one = p.scale != nullptr && !p.by_n ? *p.scale * p.factor : p.factor;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
        const int64_t n = all >> 31 ? i / fours : (int64_t)((uint32_t)i / (uint32_t)fours), m = (i - n * fours) * 4;
        const int64_t at = (p.row_of != nullptr ? (int64_t)p.row_of[n] : n) * p.m + m;
        const int most = (int)min((int64_t)4, p.m - m);
        float v[4] = {};
        if (n >= rows.lo && n < rows.hi)
            for (int s = 0; s < count; ++s) {
                float x[4];
                if (p.m % 4 == 0) {
                    *reinterpret_cast<float4*>(x) = *reinterpret_cast<const float4*>(from + s * step + at);
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[j] = j < most ? from[s * step + at + j] : 0.0f;
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] += x[j];
            }
        float scale = one;
        if (p.by_n) scale = p.scale[n] * p.factor;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = p.by_n && scale == 0.0f ? 0.0f : v[j] * scale;
        const int64_t to = g * p.step_out + n * p.ld_out + m;
        if (p.out_dtype == FASGD_F32)
            put_four<float>(p, to, most, wide, v);
        else if (p.out_dtype == FASGD_BF16)
            put_four<__nv_bfloat16>(p, to, most, wide, v);
        else
            put_four<__half>(p, to, most, wide, v);
    }
}

// splits: parts of k, each to its own result.
__global__ void __launch_bounds__(256) plain_kernel(Product p, int32_t splits) {
    __shared__ float as[kK][kM + 1], bs[kK][kN + 1];
    const uint32_t across = (uint32_t)((p.m + kM - 1) / kM), tile = blockIdx.x / across, tiles = gridDim.x / across;
    const int64_t m0 = (int64_t)(blockIdx.x % across) * kM;
    int64_t group = blockIdx.z / splits, n0 = (int64_t)tile * kN, n1 = p.n, k0 = 0, k1 = p.k;
    const int32_t split = blockIdx.z % splits;
    if (p.ragged == kRaggedN) {
        // Rows of no group, spread over the blocks; then the block's own tile.
        const int64_t lo = group_bounds(p.offsets, 0, p.n).lo, hi = group_bounds(p.offsets, p.groups - 1, p.n).hi;
        for (int64_t r = tile; splits == 1 && r < p.n - (hi - lo); r += tiles)      // (else the fold does)
            for (int64_t m = m0 + threadIdx.x; m < min(m0 + kM, p.m); m += blockDim.x)
                put(p, 0, m, r < lo ? r : hi + (r - lo), 0.0f);
        Bounds rows;
        if (!find_tile(p, tile, group, rows)) return;
        n0 = rows.lo;
        n1 = rows.hi;
    } else if (p.ragged == kRaggedK) {
        const Bounds b = group_bounds(p.offsets, (int)group, p.k);
        k0 = b.lo;
        k1 = b.hi;
    }
    if (splits > 1) {
        const int64_t stages = (k1 - k0 + kK - 1) / kK, first = k0;
        k0 = first + stages * split / splits * kK;
        k1 = min(k1, first + stages * (split + 1) / splits * kK);
    }
    const int64_t ga = p.ragged == kRaggedN ? group : 0;
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    // [m: tx + 16 i][n: ty + 16 j].  Sums of kSum k each are added up: all of k one after the other left dz of one row
    // over 220,561 classes, a part of 13,786 of them, 8e-6 off (3e-7 now; 3 % slower).
    float d[4][4] = {}, sums[4][4] = {};
    float a_next[kEach], b_next[kEach];
    read(a_next, p.a, ga, m0, p.m, k0, k1);
    read(b_next, p.b, 0, n0, n1, k0, k1);
    for (int64_t from = k0; from < k1; from += kSum) {
        for (int64_t k = from; k < min(k1, from + kSum); k += kK) {
            stage(as, a_next, p.a.across);
            stage(bs, b_next, p.b.across);
            __syncthreads();
            read(a_next, p.a, ga, m0, p.m, k + kK, k1);
            read(b_next, p.b, 0, n0, n1, k + kK, k1);
#pragma unroll
            for (int s = 0; s < kK; ++s) {
                float av[4], bv[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) av[i] = as[s][tx + 16 * i];
#pragma unroll
                for (int j = 0; j < 4; ++j) bv[j] = bs[s][ty + 16 * j];
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) d[i][j] = fmaf(av[i], bv[j], d[i][j]);
            }
            __syncthreads();
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                sums[i][j] += d[i][j];
                d[i][j] = 0.0f;
            }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) d[i][j] = sums[i][j];
    const int64_t go = p.ragged == kRaggedK ? group : 0;
    p.out = static_cast<char*>(p.out) + 4 * split * p.step_split;
    if (p.ending == kStore) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t n = n0 + ty + 16 * j;
            if (n >= n1) continue;
            float scale = p.factor;
            bool zero = false;
            if (p.scale != nullptr) {
                const float s = p.scale[p.by_n ? n : 0];
                zero = p.by_n && s == 0.0f;
                scale *= s;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int64_t m = m0 + tx + 16 * i;
                if (m < p.m) put(p, go, m, n, zero ? 0.0f : d[i][j] * scale);
            }
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t m = m0 + tx + 16 * i;
        const int64_t label = m < p.m ? p.labels[m] : -1;
        const bool has = label >= 0 && label < p.classes;
        if (p.ending == kResidual) {
            const float lse = has ? p.lse[m] : 0.0f, own = has ? expm1f(-p.row_loss[m]) : 0.0f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int64_t n = n0 + ty + 16 * j;
                if (m < p.m && n < n1)
                    put(p, 0, m, n, has ? p.factor * (p.n0 + n == label ? own : expf(d[i][j] - lse)) : 0.0f);
            }
            continue;
        }
        float top = -INFINITY;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t n = n0 + ty + 16 * j;
            if (n < n1) top = fmaxf(top, d[i][j]);
            if (n < n1 && has && p.n0 + n == label) p.at_label[m] = d[i][j];
        }
        as[ty][tx + 16 * i] = top;
        __syncthreads();
        for (int r = 0; r < 16; ++r) top = fmaxf(top, as[r][tx + 16 * i]);
        __syncthreads();
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (n0 + ty + 16 * j < n1) sum += d[i][j] == top ? 1.0f : expf(d[i][j] - top);
        as[ty][tx + 16 * i] = sum;
        __syncthreads();
        if (ty == 0 && m < p.m) {
            sum = 0.0f;
            for (int r = 0; r < 16; ++r) sum += as[r][tx + 16 * i];
            p.parts[(p.n0 / kN + tile) * p.m + m] = make_float2(top, sum);
        }
        __syncthreads();
    }
}

// Copies of a side, eight values a thread: 16-byte stores, and 16-byte loads where the side has them.
// PLANES: fp32 to four bf16 planes.
template <class F, class T, bool WIDE, bool PLANES>
__global__ void __launch_bounds__(256) pack_kernel(Pack p) {
    const int64_t g = blockIdx.y, octets = (p.cols + 7) / 8, all = p.rows * octets;
    pdl_wait();
    pdl_trigger();
    if (p.offsets != nullptr && p.offsets[g + 1] <= p.offsets[g]) return;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
        const int64_t r = all >> 31 ? i / octets : (int64_t)((uint32_t)i / (uint32_t)octets), c = (i - r * octets) * 8;
        const int64_t label = p.labels != nullptr ? p.labels[r] : 0;
        const bool has = p.labels == nullptr || (label >= 0 && label < p.classes);
        const F* from = static_cast<const F*>(p.from) + g * p.step_from + r * p.ld_from + c;
        const int most = (int)min((int64_t)8, p.cols - c);
        alignas(16) F v[8];
        if (WIDE && most == 8) {
            constexpr int kWords = 8 * sizeof(F) / 16;
#pragma unroll
            for (int j = 0; j < kWords; ++j) reinterpret_cast<uint4*>(v)[j] = reinterpret_cast<const uint4*>(from)[j];
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = j < most ? from[j] : from_f32<F>(0.0f);
        }
        T* to = static_cast<T*>(p.to) + g * p.step_to + (p.to_row != nullptr ? p.to_row[r] : r) * p.ld_to + c;
        alignas(16) T out[PLANES ? 4 : 1][8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float x = has ? to_f32(v[j]) : 0.0f;
            if constexpr (PLANES) {
                __nv_bfloat16 y[3];
                planes_of(x, y);
#pragma unroll
                for (int k = 0; k < 3; ++k) out[k][j] = y[k];
                out[3][j] = isfinite(x) ? y[0] : from_f32<T>(0.0f);
            } else {
                out[0][j] = from_f32<T>(x);
            }
        }
#pragma unroll
        for (int k = 0; k < (PLANES ? 4 : 1); ++k)
#pragma unroll
            for (int j = 0; j < (int)sizeof(T) / 2; ++j)
                reinterpret_cast<uint4*>(to + k * p.plane)[j] = reinterpret_cast<const uint4*>(out[k])[j];
    }
}
template <class F, class T, bool PLANES>
cudaError_t pack(const Pack& p, cudaStream_t stream) {
    const int64_t octets = (p.cols + 7) / 8, blocks = std::min<int64_t>((p.rows * octets + 255) / 256, 1 << 14);
    constexpr int kStep = 16 / sizeof(F);
    const bool wide = (reinterpret_cast<uintptr_t>(p.from) & 15) == 0 && p.ld_from % kStep == 0 &&
                      (p.groups < 2 || p.step_from % kStep == 0);
    const dim3 grid((unsigned)blocks, (unsigned)p.groups);
    return launch_pdl(wide ? pack_kernel<F, T, true, PLANES> : pack_kernel<F, T, false, PLANES>, grid, dim3(256), 0, stream, p);
}

}  // namespace

cudaError_t launch_pack(const Pack& p, cudaStream_t stream) {
    if (p.rows == 0) return cudaSuccess;
    if (p.plane != 0) return pack<float, __nv_bfloat16, true>(p, stream);
    if (p.dtype_from == p.dtype_to) {
        switch (p.dtype_to) {
            case FASGD_F32: return pack<float, float, false>(p, stream);
            case FASGD_BF16: return pack<__nv_bfloat16, __nv_bfloat16, false>(p, stream);
            default: return pack<__half, __half, false>(p, stream);
        }
    }
    return p.dtype_to == FASGD_BF16 ? pack<float, __nv_bfloat16, false>(p, stream) : pack<float, __half, false>(p, stream);
}

cudaError_t launch_fold(const Product& p, const float* parts, int64_t step, int32_t count, cudaStream_t stream) {
    if (p.n * p.m == 0) return cudaSuccess;
    const int64_t size = p.out_dtype == FASGD_F32 ? 4 : 2;
    const bool wide = p.m % 4 == 0 && reinterpret_cast<uintptr_t>(p.out) % (4 * size) == 0 && p.ld_out % 4 == 0 &&
                      p.step_out % 4 == 0;
    const dim3 grid((unsigned)std::min<int64_t>((p.n * ((p.m + 3) / 4) + 255) / 256, 1 << 14),
                    p.ragged == kRaggedK ? p.groups : 1);
    return launch_pdl(fold_kernel, grid, dim3(256), 0, stream, p, parts, step, count, wide);
}

int32_t plain_splits(const Product& p) {
    const bool rows = p.ragged == kRaggedN;
    const int64_t tiles = ((p.m + kM - 1) / kM) * ((p.n + kN - 1) / kN + (rows ? std::min<int64_t>(p.groups, p.n) : 0)) *
                          (p.ragged == kRaggedK ? p.groups : 1);
    const int64_t k = p.ragged == kRaggedK ? p.k / p.groups : p.k;
    return (int32_t)std::max<int64_t>(1, std::min<int64_t>({16, 304 / std::max<int64_t>(1, tiles), k / 128}));
}

cudaError_t launch_plain(const Product& p, int32_t splits, cudaStream_t stream) {
    const int64_t tiles = ((p.n + kN - 1) / kN + (p.ragged == kRaggedN ? p.groups : 0)) * ((p.m + kM - 1) / kM);
    if (tiles == 0) return cudaSuccess;
    if (tiles >= (int64_t)1 << 31) return cudaErrorInvalidConfiguration;
    const dim3 grid((unsigned)tiles, 1, (p.ragged == kRaggedK ? p.groups : 1) * splits);
    plain_kernel<<<grid, 256, 0, stream>>>(p, splits);
    return cudaGetLastError();
}

}  // namespace fasgd
