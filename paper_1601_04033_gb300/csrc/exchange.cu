// Between rows and places: fasgd_gather, fasgd_combine and fasgd_combine_grad.
//
// Nothing is computed to speak of: the bound is memory.  All three go by rows, so that a
// row is read once however many places it has (by places it would be read `top` times,
// from an L2 that the places' stream sweeps), and every place is touched once.  A place
// that no entry has is 0: entry a's thread looks at order[a], so row t clears those of
// the places t top ... t top + top - 1 that stand empty.
//
// 16,384 x 8 rows of 2,048 bf16: gather 92 us (6.6 TB/s), combine 102 (5.9), its gradients 173 (6.6).  Rows
// that allow no 16-byte packs go in pairs of values or single ones, four of them a thread.

#include <algorithm>

#include "client.cuh"
#include "route.cuh"

namespace fasgd {
namespace {

// N values that move together: 16 bytes, or one value where the layout allows no more.
template <class T, int N>
struct alignas(sizeof(T) * N) Pack {
    T v[N];
};
template <class T, int N>
__device__ __forceinline__ Pack<T, N> load(const void* base, int64_t at) {
    return *reinterpret_cast<const Pack<T, N>*>(static_cast<const T*>(base) + at);
}
template <class T, int N>
__device__ __forceinline__ void store(void* base, int64_t at, const Pack<T, N>& p) {
    *reinterpret_cast<Pack<T, N>*>(static_cast<T*>(base) + at) = p;
}
__device__ __forceinline__ bool there(int32_t i, int64_t n) { return i >= 0 && i < n; }

// A thread's row and its U packs of columns, c and `step` values further on.  U = 1: threads go along
// the rows; more: a warp takes 32 U packs of a row, so that the row's places are read once for U.
template <int N, int U>
__device__ __forceinline__ bool own(const ExchangeArgs& a, int64_t& t, int64_t& c) {
    const int64_t units = ((a.cols + N - 1) / N + (U > 1 ? 32 * U - 1 : 0)) / (U > 1 ? 32 * U : 1);
    int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (U > 1) i /= 32;
    if (i >= a.rows * units) return false;
    t = a.rows * units >> 31 ? i / units : (int64_t)((uint32_t)i / (uint32_t)units);
    c = (i - t * units) * N;
    if (U > 1) c = c * 32 * U + (threadIdx.x & 31) * N;
    return true;
}

template <class T, int N, int U>
__global__ void __launch_bounds__(256) gather_kernel(ExchangeArgs a) {
    int64_t t, c;
    if (!own<N, U>(a, t, c)) return;
    Pack<T, N> v[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (U == 1 || c + u * 32 * N < a.cols) v[u] = load<T, N>(a.row_values, t * a.ld_rows + c + u * 32 * N);
    const Pack<T, N> zero = {};
    // Eight entries at a time, so that their places are read together.
    for (int64_t k0 = t * a.top; k0 < (t + 1) * a.top; k0 += 8) {
        const int most = (int)min((int64_t)8, (t + 1) * a.top - k0);
        int32_t place[8];
        bool empty[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            place[k] = k < most ? __ldg(a.place + k0 + k) : -1;
            empty[k] = k < most && !there(__ldg(a.order + k0 + k), a.n);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k)
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t at = c + u * 32 * N;
                if (U > 1 && at >= a.cols) continue;
                if (there(place[k], a.n)) store(a.places, place[k] * a.ld_places + at, v[u]);
                if (empty[k]) store(a.places, (k0 + k) * a.ld_places + at, zero);
            }
    }
}

template <class T, int N, int U>
__global__ void __launch_bounds__(256) combine_kernel(ExchangeArgs a) {
    constexpr int kAtOnce = 8;
    int64_t t, c;
    if (!own<N, U>(a, t, c)) return;
    float sum[U][N] = {};
    for (int64_t k0 = t * a.top; k0 < (t + 1) * a.top; k0 += kAtOnce) {
        const int most = (int)min((int64_t)kAtOnce, (t + 1) * a.top - k0);
        Pack<T, N> v[kAtOnce][U];
        float w[kAtOnce];
        bool has[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            const int32_t i = k < most ? __ldg(a.place + k0 + k) : -1;
            has[k] = there(i, a.n);
            // (of an absent place the first one's values are read and left out: a load that has a
            // branch of its own waits for the one before)
#pragma unroll
            for (int u = 0; u < U; ++u)
                v[k][u] = load<T, N>(a.places, (has[k] ? i : 0) * a.ld_places + (U == 1 || c + u * 32 * N < a.cols ? c + u * 32 * N : 0));
            w[k] = a.weight != nullptr ? __ldg(a.weight + (has[k] ? k0 + k : 0)) : 1.0f;
        }
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k)
            if (has[k])
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int j = 0; j < N; ++j) sum[u][j] = fmaf(w[k], to_f32(v[k][u].v[j]), sum[u][j]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (U > 1 && c + u * 32 * N >= a.cols) continue;
        Pack<T, N> out;
#pragma unroll
        for (int j = 0; j < N; ++j) out.v[j] = from_f32<T>(sum[u][j]);
        store(a.row_values, t * a.ld_rows + c + u * 32 * N, out);
    }
}

// A team of `TEAM` threads for each row; the dot products of kAtOnce places at a time.
template <class T, int N, int TEAM>
__global__ void __launch_bounds__(256) combine_grad_kernel(ExchangeArgs a) {
    constexpr int kAtOnce = 8, kTeams = 256 / TEAM, kWarps = TEAM / 32;
    __shared__ float part[kTeams][kWarps][kAtOnce];
    const int team = threadIdx.x / TEAM, me = threadIdx.x % TEAM;
    const int64_t t = (int64_t)blockIdx.x * kTeams + team;
    const bool live = t < a.rows;
    const Pack<T, N> zero = {};
    for (int64_t k0 = 0; k0 < a.top; k0 += kAtOnce) {
        float dot[kAtOnce] = {};
        int32_t at[kAtOnce];
        float w[kAtOnce];
        bool empty[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            const int64_t e = t * a.top + k0 + k;
            const bool is = live && k0 + k < a.top;
            at[k] = is ? __ldg(a.place + e) : -1;
            if (!there(at[k], a.n)) at[k] = -1;
            w[k] = at[k] >= 0 ? __ldg(a.weight + e) : 0.0f;
            empty[k] = is && !there(__ldg(a.order + e), a.n);
        }
        for (int64_t c = (int64_t)me * N; live && c < a.cols; c += TEAM * N) {
            const Pack<T, N> d = load<T, N>(a.row_values, t * a.ld_rows + c);
            Pack<T, N> v[kAtOnce];
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k)
                v[k] = load<T, N>(a.places, max(at[k], 0) * a.ld_places + c);
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
                if (at[k] >= 0) {
                    Pack<T, N> out;
#pragma unroll
                    for (int j = 0; j < N; ++j) {
                        const float g = to_f32(d.v[j]);
                        out.v[j] = from_f32<T>(w[k] * g);
                        if (a.dweight != nullptr) dot[k] = fmaf(g, to_f32(v[k].v[j]), dot[k]);
                    }
                    store(a.dplaces, at[k] * a.ld_dplaces + c, out);
                }
                if (empty[k]) store(a.dplaces, (t * a.top + k0 + k) * a.ld_dplaces + c, zero);
            }
        }
        if (a.dweight == nullptr) continue;
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            dot[k] = warp_sum(dot[k]);
            if (kWarps > 1 && me % 32 == 0) part[team][me / 32][k] = dot[k];
        }
        if (kWarps > 1) {
            __syncthreads();
            if (me < kAtOnce) {
                float sum = 0.0f;
                for (int w8 = 0; w8 < kWarps; ++w8) sum += part[team][w8][me];
                if (live && k0 + me < a.top) a.dweight[t * a.top + k0 + me] = sum;
            }
            __syncthreads();
        } else if (me == 0) {
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k)
                if (live && k0 + k < a.top) a.dweight[t * a.top + k0 + k] = dot[k];
        }
    }
}

template <class T, int N, int U>
cudaError_t launch_rows(const ExchangeArgs& a, ExchangeKind kind, cudaStream_t stream) {
    const int64_t packs = (a.cols + N - 1) / N, threads = U > 1 ? (packs + 32 * U - 1) / (32 * U) * 32 : packs;
    const int64_t blocks = (a.rows * threads + 255) / 256;
    if (blocks >= (int64_t)1 << 31) return cudaErrorInvalidConfiguration;
    if (kind == kGather)
        gather_kernel<T, N, U><<<(unsigned)blocks, 256, 0, stream>>>(a);
    else
        combine_kernel<T, N, U><<<(unsigned)blocks, 256, 0, stream>>>(a);
    return cudaGetLastError();
}
template <class T, int N>
cudaError_t launch(const ExchangeArgs& a, ExchangeKind kind, cudaStream_t stream) {
    const int64_t packs = (a.cols + N - 1) / N;
    if (kind == kCombineGrad) {
        // A warp for each row needs no barriers; few and wide rows want more threads.
        if (packs <= 64 || a.rows >= 2048) {
            combine_grad_kernel<T, N, 32><<<(unsigned)((a.rows + 7) / 8), 256, 0, stream>>>(a);
        } else {
            combine_grad_kernel<T, N, 256><<<(unsigned)a.rows, 256, 0, stream>>>(a);
        }
        return cudaGetLastError();
    }
    // Narrow packs are bound by instructions: a thread has four of them where the row is long enough.
    if constexpr (N * sizeof(T) < 16)
        if (packs >= 128) return launch_rows<T, N, 4>(a, kind, stream);
    return launch_rows<T, N, 1>(a, kind, stream);
}

template <class T>
cudaError_t launch(const ExchangeArgs& a, ExchangeKind kind, cudaStream_t stream) {
    constexpr int N = 16 / sizeof(T);
    const auto whole = [&](int n) {
        const auto fits = [&](const void* p, int64_t ld, int64_t rows) {
            return (reinterpret_cast<uintptr_t>(p) & (n * sizeof(T) - 1)) == 0 && (rows < 2 || ld % n == 0);
        };
        return a.cols % n == 0 && fits(a.row_values, a.ld_rows, a.rows) && fits(a.places, a.ld_places, a.n) &&
               (kind != kCombineGrad || fits(a.dplaces, a.ld_dplaces, a.n));
    };
    return whole(N) ? launch<T, N>(a, kind, stream) : whole(2) ? launch<T, 2>(a, kind, stream) : launch<T, 1>(a, kind, stream);
}

}  // namespace

cudaError_t launch_exchange(const ExchangeArgs& a, ExchangeKind kind, int dtype, cudaStream_t stream) {
    switch (dtype) {
        case FASGD_F32: return launch<float>(a, kind, stream);
        case FASGD_BF16: return launch<__nv_bfloat16>(a, kind, stream);
        default: return launch<__half>(a, kind, stream);
    }
}

}  // namespace fasgd
