// fasgd_route: a stable counting sort of a router's choices by expert.
//
// The entries fall into chunks of consecutive ones, a block each, and a chunk into
// one piece for each of its warps, so (chunk, warp, step, lane) is the entries' own
// order.  A warp counts its piece 32 entries at a time, each lane adding one to the warp's
// counter of its entry's expert in shared memory.  Counters become first places by sums over
// experts, earlier chunks and earlier warps.  A second sweep hands the places out: lanes of one
// expert find each other by votes over the bits of its number, take the places behind its
// counter in their order, and the first of them moves the counter on.
//
// Short lists (128 rows of a minibatch) take one block and one launch.  Longer ones take
// two: each block of the second adds up the counters of all chunks itself, at most 64
// chunks (with 256 of them the sums took 40 of 65 us), which costs less than a third launch.
//
// Bound by latency: 524,288 entries of 256 experts take 15 us (6.3 MB would be 1), 256 entries 5 with the host.

#include <algorithm>

#include "pdl.cuh"
#include "route.cuh"

namespace fasgd {
namespace {

constexpr int kManyWarps = 32, kFewWarps = 8;
constexpr int kManyExperts = 320;        // experts that 32 warps have counters for in 40 KB
constexpr int64_t kChunk = 4096;         // entries of a block where there are several
constexpr int kChunks = 64;

int warps_of(int32_t experts) { return experts <= kManyExperts ? kManyWarps : kFewWarps; }

__device__ __forceinline__ bool goes(int32_t e, int32_t experts) { return (uint32_t)e < (uint32_t)experts; }

// Entries of this warp, kAhead steps read together.
constexpr int kAhead = 8;
template <class F>
__device__ __forceinline__ void sweep(const int32_t* chosen, int64_t begin, int64_t end, F step) {
    const int lane = threadIdx.x & 31;
    for (int64_t i0 = begin; i0 < end; i0 += 32 * kAhead) {
        int32_t e[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) e[j] = i0 + 32 * j + lane < end ? __ldg(chosen + i0 + 32 * j + lane) : -1;
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
            if (i0 + 32 * j < end) step(i0 + 32 * j + lane, e[j]);
    }
}
// Entries [begin, end) of this warp into its counters (whose order does not matter).
__device__ void count(const int32_t* chosen, int64_t begin, int64_t end, int32_t experts, int32_t* mine) {
    sweep(chosen, begin, end, [&](int64_t, int32_t e) {
        if (goes(e, experts)) atomicAdd(mine + e, 1);
    });
}
// The lanes whose entries go to the same expert as this one's: a vote for each bit of its number
// (the warp's own match of values takes a round for each different one, of which there are many).
__device__ __forceinline__ uint32_t same_as(int32_t e, bool goes_on, int bits) {
    uint32_t same = __ballot_sync(0xffffffffu, goes_on);
    for (int b = 0; b < bits; ++b) {
        const uint32_t ones = __ballot_sync(0xffffffffu, e >> b & 1);
        same &= e >> b & 1 ? ones : ~ones;
    }
    return same;
}
// The places of this warp's entries; mine: the next place of each expert.
__device__ void hand_out(const RouteArgs& a, int64_t begin, int64_t end, int32_t* mine) {
    const int lane = threadIdx.x & 31, bits = 32 - __clz(a.experts - 1);
    int32_t *const place = a.place, *const order = a.order;
    sweep(a.chosen, begin, end, [&](int64_t i, int32_t e) {
        const bool on = goes(e, a.experts);
        const uint32_t same = same_as(e, on, bits);
        int32_t at = -1;
        if (on) at = mine[e] + __popc(same & ((1u << lane) - 1u));
        __syncwarp();
        if (on && lane == __ffs(same) - 1) mine[e] = at + __popc(same);
        __syncwarp();
        if (i < end) place[i] = at;
        if (on) order[at] = (int32_t)i;
    });
}
// first[0..experts) from counts to their exclusive sums; the total is returned to all.
// By warp 0, 32 at a time.
__device__ int32_t scan(int32_t* first, int32_t experts, int32_t* total) {
    if (threadIdx.x < 32) {
        int32_t before = 0;
        for (int32_t e = threadIdx.x; e < (experts + 31) / 32 * 32; e += 32) {
            const int32_t v = e < experts ? first[e] : 0;
            int32_t s = v;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int32_t o = __shfl_up_sync(0xffffffffu, s, d);
                if (threadIdx.x >= d) s += o;
            }
            if (e < experts) first[e] = before + s - v;
            before += __shfl_sync(0xffffffffu, s, 31);
        }
        if (threadIdx.x == 0) *total = before;
    }
    __syncthreads();
    return *total;
}

// A warp's piece of its block's chunk.
__device__ __forceinline__ void piece(const RouteArgs& a, int64_t& begin, int64_t& end) {
    const int warps = blockDim.x / 32;
    const int64_t lo = (int64_t)blockIdx.x * a.chunk, hi = min(lo + a.chunk, a.n);
    const int64_t step = (a.chunk + warps * 32 - 1) / (warps * 32) * 32;
    begin = min(lo + (threadIdx.x / 32) * step, hi);
    end = min(begin + step, hi);
}
__device__ void clear(int32_t* counters, int32_t experts) {
    for (int i = threadIdx.x; i < (int)(blockDim.x / 32) * experts; i += blockDim.x) counters[i] = 0;
    __syncthreads();
}

__global__ void __launch_bounds__(1024) count_kernel(RouteArgs a) {
    extern __shared__ int32_t counters[];      // [warps][experts]
    const int warps = blockDim.x / 32;
    clear(counters, a.experts);
    int64_t begin, end;
    piece(a, begin, end);
    count(a.chosen, begin, end, a.experts, counters + (threadIdx.x / 32) * a.experts);
    __syncthreads();
    pdl_trigger();
    for (int e = threadIdx.x; e < a.experts; e += blockDim.x) {
        int32_t sum = 0;
        for (int w = 0; w < warps; ++w) sum += counters[w * a.experts + e];
        a.part_counts[(int64_t)blockIdx.x * a.experts + e] = sum;
    }
}

__global__ void __launch_bounds__(1024) place_kernel(RouteArgs a) {
    extern __shared__ int32_t counters[];      // [warps][experts], then first and before
    __shared__ int32_t total;
    const int warps = blockDim.x / 32;
    int32_t* first = counters + warps * a.experts;
    clear(counters, a.experts);
    int64_t begin, end;
    piece(a, begin, end);
    int32_t* mine = counters + (threadIdx.x / 32) * a.experts;
    count(a.chosen, begin, end, a.experts, mine);
    __syncthreads();
    if (a.chunks > 1) pdl_wait();
    // first[e]: all entries of e, then where e begins; before[e]: its entries of earlier chunks.
    int32_t* before = first + a.experts;
    for (int e = threadIdx.x; e < a.experts; e += blockDim.x) {
        int32_t sum = 0, mine_before = 0;
        if (a.chunks == 1) {
            for (int w = 0; w < warps; ++w) sum += counters[w * a.experts + e];
        } else {
#pragma unroll 16
            for (int c = 0; c < a.chunks; ++c) {
                const int32_t k = a.part_counts[(int64_t)c * a.experts + e];
                sum += k;
                mine_before += c < (int)blockIdx.x ? k : 0;
            }
        }
        first[e] = sum;
        before[e] = mine_before;
    }
    __syncthreads();
    const int32_t all = scan(first, a.experts, &total);
    for (int e = threadIdx.x; e < a.experts; e += blockDim.x) {
        int32_t at = first[e];
        if (blockIdx.x == 0) a.offsets[e] = at;
        at += before[e];
        for (int w = 0; w < warps; ++w) {
            const int32_t k = counters[w * a.experts + e];
            counters[w * a.experts + e] = at;
            at += k;
        }
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) a.offsets[a.experts] = all;
    __syncthreads();
    hand_out(a, begin, end, mine);
    const int64_t lo = (int64_t)blockIdx.x * a.chunk, hi = min(lo + a.chunk, a.n);
    for (int64_t i = max(lo, (int64_t)all) + threadIdx.x; i < hi; i += blockDim.x) a.order[i] = -1;
}

}  // namespace

void route_chunks(int64_t n, int32_t experts, int32_t& chunks, int64_t& chunk) {
    if (n <= (int64_t)warps_of(experts) * 32 * 16) {
        chunks = 1;
        chunk = n;
        return;
    }
    chunk = std::max(kChunk, (n + kChunks - 1) / kChunks);
    chunk = (chunk + 1023) / 1024 * 1024;
    chunks = (int32_t)((n + chunk - 1) / chunk);
}

cudaError_t launch_route(const RouteArgs& a, cudaStream_t stream) {
    const int warps = std::max(1, (int)std::min<int64_t>(warps_of(a.experts), (a.n + 31) / 32));
    const size_t smem = sizeof(int32_t) * warps * a.experts;
    if (a.chunks == 1) {
        place_kernel<<<1, warps * 32, smem + 2 * sizeof(int32_t) * a.experts, stream>>>(a);
        return cudaGetLastError();
    }
    count_kernel<<<a.chunks, warps * 32, smem, stream>>>(a);
    cudaError_t st = cudaGetLastError();
    if (st != cudaSuccess) return st;
    return launch_pdl(place_kernel, dim3(a.chunks), dim3(warps * 32), smem + 2 * sizeof(int32_t) * a.experts, stream, a);
}

}  // namespace fasgd
