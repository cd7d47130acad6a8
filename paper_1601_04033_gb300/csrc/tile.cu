// Matrix products of 16-bit values on the tensor cores (tcgen05), operands by TMA.
//
// A block, or a pair of blocks (cluster of 2) that shares its MMAs, computes tiles of
// 128 (256) m by up to 256 n, one after the other: warp 0 copies 64 steps of k of both
// sides at a time into a ring of stages in shared memory, warp 1 issues the MMAs into one
// of two accumulators in tensor memory, warps 4 to 11 empty the other one.  A side is
// copied as it lies in memory, k or its own index consecutive (128-byte swizzle either way; the
// MMA's descriptors say which), so no operand is ever transposed by a pass of its own.
//
// A pair exists for the copies: a tile of 256 x 256 moves 32 KB per block and 64 steps of
// k, half as much per MMA as one block's 128 x 128, and less than its 128 x 256 (48 KB,
// which at the tensor cores' full rate would be 96 bytes a cycle and SM out of L2).
//
// Ragged n (rows sorted by expert): a tile's n are one group's; what it copies beyond the
// group's last row is another's and not stored, and the MMA is only as wide as it needs to be.
// Ragged k (sums over a group's rows): the last copy's rows beyond the group are set to 0 in
// shared memory before the MMAs, in both sides, since another group's NaN times 0 is NaN.
//
// Bound: the tensor pipe, 80 to 90 % active in products of some thousands a side, at the clock that the power
// limit leaves: 1,550 to 1,930 TFLOP/s (bf16, 8,192 rows; 1,800 for 32,768 rows in 32 experts of 4,096 x
// 2,048).  Short products are bound by a launch's latency (6 us) and 0.3 us for each 64 of k.
//
// Every wait is bounded (wait_thread): one that runs out raises the block's flag, every
// role leaves, what was not computed is written as NaN, and the host learns of it (read_late).
//
// Kernels that add sums up in registers (Sums) spill 36 to 44 bytes at 216 of them.

#include <cuda.h>

#include <algorithm>
#include <atomic>

#include "client.cuh"
#include "pdl.cuh"
#include "product.cuh"
#include "shared_limit.cuh"
#include "wait.cuh"

namespace fasgd {
namespace {

constexpr int kK = 64;                              // steps of k in a stage: 128 bytes
constexpr int kBlockM = 128;                        // m of a block
constexpr int kEnds = 8;                            // warps that take results: two for each 32 lanes
constexpr int kThreads = 128 + 32 * kEnds;          // warps 0 to 3: copies, MMAs, groups' last rows, one at rest
constexpr int kExact = 256;                         // k of an accumulator where the sums are to be exact ones
// An accumulator's additions cut bits off, always toward zero: each of n terms of one sign up to 2^-24 of what is
// there, n / 2 2^-24 of the sum; measured is a quarter of that (16,384: 1.1e-4).  Up to kLongFrom that is at most the
// 2^-11 by which rounding to fp16 is off; where sums are longer they leave the accumulator every kLong k and
// go on in registers, 6e-5 at most (1.4e-5).  Going on like that from 2,048 on cost dw of 12,279 rows by 1,021 x 509
// in 7 experts 5 us (a kernel more to fetch), and 8,192 x 2,048 x 131,072's score 2 %.
constexpr int kLong = 2048, kLongFrom = 16384;
constexpr int kSideA = kBlockM * kK * 2;            // bytes of A in a stage
constexpr int kFew = 32;                             // rows of a box of a short tile
constexpr int kMaxGroups = FASGD_EXPERTS_MAX;
constexpr int kColumns = 512;                       // of tensor memory: two accumulators

template <int PAIR>
struct Shape {
    static constexpr int kSideB = kTileN / PAIR * kK * 2;
    static constexpr int kStage = kSideA + kSideB;
    static constexpr int kStages = PAIR == 2 ? 6 : 4;
    static constexpr int kBytes = kStages * kStage + 1024;     // and room to align to 1,024
};

struct TileArgs {
    CUtensorMap a, b, few;     // few: B in boxes of kFew rows, for groups' short tiles
    Product p;
    int32_t wide_a, wide_b;    // a side that is across, in boxes of several chunks
    int64_t m_tiles, items;    // items: of all groups, unless n is ragged
    int32_t splits;
    int32_t tile_n;            // of a tile
    uint64_t limit;            // ns: see wait_thread
    uint32_t planes_a, planes_b;      // the pairs'
};

// ---- PTX ------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t block_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
// The address of a shared variable of the pair's first block.
__device__ __forceinline__ uint32_t first_block(uint32_t addr) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(addr));
    return r;
}
// CLUSTER: what the pair's other block wrote before it arrived is seen too.  (That, and a release
// of the same width, cost some 2,000 cycles each: only where a block writes what its pair's MMA reads.)
template <bool CLUSTER>
__device__ __forceinline__ bool test(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    if (CLUSTER)
        asm volatile(
            "{\n .reg .pred p;\n mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n"
            " selp.u32 %0, 1, 0, p;\n}\n"
            : "=r"(ok)
            : "r"(bar), "r"(parity)
            : "memory");
    else
        asm volatile(
            "{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}\n"
            : "=r"(ok)
            : "r"(bar), "r"(parity)
            : "memory");
    return ok != 0;
}
template <bool CLUSTER = false>
__device__ __forceinline__ void arrive_first(uint64_t* bar) {
    const uint32_t at = first_block(smem_addr(bar));
    if (CLUSTER)
        asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(at) : "memory");
    else
        asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(at) : "memory");
}
__device__ __forceinline__ void arrive_expect(uint32_t bar, uint32_t bytes) {     // in either block
    asm volatile("mbarrier.arrive.expect_tx.shared::cluster.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// A box at (x, y, z, g) of a plane to shared memory; bar: an address in this block's or (PAIR 2) its pair's.
template <int PAIR>
__device__ __forceinline__ void copy_box(const CUtensorMap* map, uint32_t to, uint32_t bar, int32_t x, int32_t y, int32_t z,
                                         int32_t g, int32_t plane) {
    if (PAIR == 2)
        asm volatile(
            "cp.async.bulk.tensor.5d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, "
            "%5, %6, %7}], [%2];" ::"r"(to),
            "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z), "r"(g), "r"(plane)
            : "memory");
    else
        asm volatile(
            "cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6, "
            "%7}], [%2];" ::"r"(to),
            "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z), "r"(g), "r"(plane)
            : "memory");
}
template <int PAIR>
__device__ __forceinline__ void mma(uint32_t to, uint32_t a_low, uint32_t b_low, uint32_t a_high, uint32_t b_high, uint32_t shape,
                                    bool add) {
    if (PAIR == 2)
        asm volatile(
            "{\n .reg .pred p;\n .reg .b64 a, b;\n setp.ne.u32 p, %4, 0;\n mov.b64 a, {%1, %5};\n mov.b64 b, {%2, %6};\n"
            " tcgen05.mma.cta_group::2.kind::f16 [%0], a, b, %3, p;\n}\n" ::"r"(to),
            "r"(a_low), "r"(b_low), "r"(shape), "r"((uint32_t)add), "r"(a_high), "r"(b_high)
            : "memory");
    else
        asm volatile(
            "{\n .reg .pred p;\n .reg .b64 a, b;\n setp.ne.u32 p, %4, 0;\n mov.b64 a, {%1, %5};\n mov.b64 b, {%2, %6};\n"
            " tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n}\n" ::"r"(to),
            "r"(a_low), "r"(b_low), "r"(shape), "r"((uint32_t)add), "r"(a_high), "r"(b_high)
            : "memory");
}
// The barrier (of both blocks of a pair) is arrived at once all MMAs before this have ended.
template <int PAIR>
__device__ __forceinline__ void commit(uint64_t* bar) {
    if (PAIR == 2)
        asm volatile(
            "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(
                smem_addr(bar)),
            "h"((uint16_t)3)
            : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_addr(bar))
                     : "memory");
}
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
// 32 columns of the warp's 32 lanes of tensor memory, there after wait_columns().
__device__ __forceinline__ void load_columns(uint32_t from, float (&v)[32]) {
    uint32_t* r = reinterpret_cast<uint32_t*>(v);
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
        "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]),
          "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]),
          "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(from)
        : "memory");
}
__device__ __forceinline__ void load_half(uint32_t from, float (&v)[16]) {
    uint32_t* r = reinterpret_cast<uint32_t*>(v);
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(from)
        : "memory");
}
// One thread of a converged warp.
__device__ __forceinline__ bool elected() {
    uint32_t is;
    asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}\n" : "=r"(is));
    return is != 0;
}
__device__ __forceinline__ void wait_columns() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
constexpr float kLog2E = 1.4426950408889634f;

// A shared-memory matrix for the MMA: 128-byte swizzle; k consecutive (8 rows of 128 bytes
// are 1,024 apart), or across: chunks of 64 values by 64 steps of k, 8,192 bytes apart, whose
// groups of 8 steps are 1,024 apart.
__device__ __forceinline__ uint64_t matrix_of(uint32_t addr, bool across) {
    const uint64_t lead = across ? 8192 >> 4 : 1;
    return (uint64_t)((addr & 0x3ffff) >> 4) | lead << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}

// ---- tiles ------------------------------------------------------------------------------
struct Tile {
    int64_t m0, n0, n1, k0, k1;
    int32_t group, split;
    int64_t n_tile;
};
struct Shared {
    uint64_t full[6], empty[6], tail[6], ready[2], taken[2];
    float2 halves[2][kBlockM];          // statistics of the tile's odd columns' half, by tiles in turn
    uint32_t tmem;
    volatile int32_t late;
    volatile uint32_t rounds;           // of the ring that the block has issued copies of
    uint64_t limit;                     // ns without one after which a wait gives up
    int32_t first[kMaxGroups + 1];      // ragged n: the first n tile of each group
    int32_t lo[kMaxGroups], hi[kMaxGroups];      // ragged products: the groups' rows
};

// One thread waits for a phase; false (and s.late): it did not come.  It gives up where the block has issued no
// copies for s.limit ns, however long its launch takes: a wait for a group's last rows lasts through all tiles
// before them.  The barrier is then tested for a while more, so that time in which the GPU is another
// context's does not count.  The timer is read only after a while: that takes as long as the MMAs of some k.
constexpr uint32_t kAgain = 64;                     // times 256 tests
template <bool CLUSTER = false>
__device__ __forceinline__ bool wait_thread(uint64_t* barrier, uint32_t parity, Shared& s) {
    const uint32_t bar = smem_addr(barrier);
    uint64_t since = 0;
    uint32_t seen = 0, again = 0;
#pragma unroll 1
    for (uint32_t i = 1; i < (1u << 30); ++i) {
        if (test<CLUSTER>(bar, parity)) return true;
        if ((i & 255u) == 0) {
            const uint64_t now = global_ns();
            if (since == 0) {
                since = now;
                seen = s.rounds;
            }
            if (now - since > s.limit || s.late != 0) {
                const uint32_t rounds = s.rounds;
                if (s.late != 0 || (rounds == seen && ++again > kAgain)) break;
                if (rounds != seen) {
                    since = now;
                    seen = rounds;
                    again = i = 0;
                }
            }
        }
    }
    s.late = 1;
    return false;
}
// A whole warp.
__device__ __forceinline__ bool wait(uint64_t* barrier, uint32_t parity, Shared& s) {
    return __all_sync(0xffffffffu, wait_thread(barrier, parity, s));
}

// Whether a wait of a launch on this device ran out since the host last asked (read_late).
__device__ int32_t waits_ran_out;

// lo, hi and first[] of the groups, by the first warp.  Offsets that rise and fall may claim more rows than
// there are: numbers stay within 31 bits all the same.
__device__ void count_tiles(const Product& p, Shared& s) {
    if (threadIdx.x < 32) {
        int64_t before = 0;
        for (int g = threadIdx.x; g < (p.groups + 31) / 32 * 32; g += 32) {
            int64_t tiles = 0;
            if (g < p.groups) {
                const Bounds b = group_bounds(p.offsets, g, p.ragged == kRaggedN ? p.n : p.k);
                s.lo[g] = (int32_t)b.lo;
                s.hi[g] = (int32_t)b.hi;
                tiles = (b.hi - b.lo + kTileN - 1) / kTileN;
            }
            int64_t sum = tiles;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int64_t o = __shfl_up_sync(0xffffffffu, sum, d);
                if (threadIdx.x >= d) sum += o;
            }
            if (g < p.groups) s.first[g] = (int32_t)min(before + sum - tiles, (int64_t)INT32_MAX);
            before += __shfl_sync(0xffffffffu, sum, 31);
        }
        if (threadIdx.x == 0) s.first[p.groups] = (int32_t)min(before, (int64_t)INT32_MAX);
    }
}

// What takes part of n and k, and the tiles of it.
struct Sizes {
    int64_t n, k, m_tiles, items;
};
template <int PAIR>
__device__ __forceinline__ Sizes sizes_of(const TileArgs& t, const Shared& s) {
    const Product& p = t.p;
    Sizes z = {p.n, p.k, t.m_tiles, t.items};
    if (p.live != nullptr) {
        const int64_t live = *p.live;
        if (p.live_of == kLiveM) z.m_tiles = (min(p.m, live) + kBlockM * PAIR - 1) / (kBlockM * PAIR);
        if (p.live_of == kLiveN) z.n = min(p.n, live);
        if (p.live_of == kLiveK) z.k = min(p.k, live);
        z.items = z.m_tiles * ((z.n + t.tile_n - 1) / t.tile_n) * t.splits;
    }
    if (p.ragged == kRaggedN) z.items = (int64_t)s.first[p.groups] * t.m_tiles * t.splits;
    return z;
}
// Item i of the product; ragged n: i counts m tiles first, then the groups' n tiles.
template <int PAIR>
__device__ __forceinline__ Tile tile_of(const TileArgs& t, const Shared& s, const Sizes& z, int64_t i) {
    const Product& p = t.p;
    Tile w;
    w.split = 0;
    w.group = 0;
    w.k0 = 0;
    w.k1 = z.k;
    if (t.splits > 1) {
        w.split = (int32_t)(i % t.splits);
        i /= t.splits;
    }
    if (p.ragged == kRaggedN) {
        const int64_t j = i / t.m_tiles;
        w.m0 = (i - j * t.m_tiles) * (kBlockM * PAIR);
        int lo = 0, hi = p.groups;                  // first[lo] <= j < first[hi]
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (s.first[mid] <= j)
                lo = mid;
            else
                hi = mid;
        }
        w.group = lo;
        w.n_tile = j;
        w.n0 = s.lo[lo] + (j - s.first[lo]) * kTileN;
        w.n1 = min((int64_t)s.hi[lo], w.n0 + kTileN);
    } else {
        const int64_t n_tiles = (z.n + t.tile_n - 1) / t.tile_n;
        if (p.ragged == kRaggedK) {
            w.group = (int32_t)(i / (t.m_tiles * n_tiles));
            i -= (int64_t)w.group * t.m_tiles * n_tiles;
            w.k0 = s.lo[w.group];
            w.k1 = s.hi[w.group];
        }
        // Bands of up to 32 m tiles, by n: what runs at the same time shares its operands in L2.
        const int64_t band = i / (32 * n_tiles), m_first = band * 32, high = min((int64_t)32, z.m_tiles - m_first);
        i -= band * 32 * n_tiles;
        w.n_tile = i / high;
        w.m0 = (m_first + i - w.n_tile * high) * (kBlockM * PAIR);
        w.n0 = w.n_tile * t.tile_n;
        w.n1 = min(z.n, w.n0 + t.tile_n);
    }
    if (t.splits > 1) {
        const int64_t blocks = (w.k1 - w.k0 + kK - 1) / kK, k0 = w.k0;
        w.k0 = k0 + blocks * w.split / t.splits * kK;
        w.k1 = min(w.k1, k0 + blocks * (w.split + 1) / t.splits * kK);
    }
    return w;
}
// n of the MMA; the halves of a pair's side that is across begin with a chunk.
template <int PAIR>
__device__ __forceinline__ int width_of(const TileArgs& t, const Tile& w) {
    const int step = PAIR == 2 && t.p.b.across ? 128 : 16 * PAIR;
    return (int)(w.n1 - w.n0 + step - 1) / step * step;
}
// What a block copies of B in a stage: one box, or for a short tile of a group and for sides of
// odd widths several.
struct Boxes {
    int rows_b, boxes_b;
    bool few;
    uint32_t bytes;      // of A too
};
template <int PAIR>
__device__ __forceinline__ Boxes boxes_of(const TileArgs& t, const Tile& w) {
    Boxes x;
    x.rows_b = width_of<PAIR>(t, w) / PAIR;
    x.few = t.p.ragged == kRaggedN && x.rows_b <= 64 * (3 - PAIR);
    const int step = x.few ? kFew : t.p.b.across && !t.wide_b ? 64 : t.tile_n / PAIR;
    x.boxes_b = (x.rows_b + step - 1) / step;
    x.bytes = kSideA + x.boxes_b * step * kK * 2;
    return x;
}
// The copy at k holds rows of the next group.
__device__ __forceinline__ bool cut(const Product& p, const Tile& w, int64_t k) {
    return p.ragged == kRaggedK && w.k1 - k < kK;
}
// ---- what becomes of an accumulator -----------------------------------------------------
// What the stores need, in registers: read again from the kernel's parameters after each of
// them (which might alias, for all the compiler knows) it made 180 cycles a column.
struct Target {
    void* out;
    int64_t ld;
    const float* scale;
    float factor;
    int32_t by_n, dtype, add;
};
template <class T>
__device__ __forceinline__ void store_columns(const Target& g, int64_t at, int64_t n, int count, bool live, const float (&v)[32]) {
    if (!live) return;
    T* out = static_cast<T*>(g.out) + at;
    if (g.scale != nullptr && g.by_n) {
#pragma unroll
        for (int j = 0; j < 32; ++j)
            if (j < count) {
                const float scale = g.scale[n + j];
                *out = from_f32<T>(scale == 0.0f ? 0.0f : v[j] * (scale * g.factor));
                out += g.ld;
            }
        return;
    }
    const float scale = g.scale != nullptr ? *g.scale * g.factor : g.factor;
#pragma unroll
    for (int j = 0; j < 32; ++j)
        if (j < count) {
            *out = from_f32<T>(v[j] * scale);
            out += g.ld;
        }
}
__device__ __forceinline__ void add_columns(const Target& g, int64_t at, int count, bool live, const float (&v)[32]) {
    if (!live) return;
    float* const out = static_cast<float*>(g.out) + at;
    float old[32];
#pragma unroll
    for (int j = 0; j < 32; ++j) old[j] = j < count ? out[j * g.ld] : 0.0f;
#pragma unroll
    for (int j = 0; j < 32; ++j)
        if (j < count) out[j * g.ld] = old[j] + v[j] * g.factor;
}
__device__ __forceinline__ void store_any(const Target& g, int64_t at, int64_t n, int count, bool live, const float (&v)[32]) {
    if (g.dtype == FASGD_F32) {
        if (g.add)
            add_columns(g, at, count, live, v);
        else
            store_columns<float>(g, at, n, count, live, v);
    } else if (g.dtype == FASGD_BF16) {
        store_columns<__nv_bfloat16>(g, at, n, count, live, v);
    } else {
        store_columns<__half>(g, at, n, count, live, v);
    }
}

// Rows of y or dx that no group has.
__device__ void clear_rows(const Product& p, const Shared& s, int64_t block, int64_t blocks, int thread, int threads) {
    const int64_t lo = s.lo[0], hi = s.hi[p.groups - 1];
    for (int64_t r = block; r < p.n - (hi - lo); r += blocks) {
        const int64_t at = (r < lo ? r : hi + (r - lo)) * p.ld_out;
        for (int64_t m = thread; m < p.m; m += threads) {
            if (p.out_dtype == FASGD_F32)
                static_cast<float*>(p.out)[at + m] = 0.0f;
            else
                static_cast<uint16_t*>(p.out)[at + m] = 0;
        }
    }
}

// SUMS: kOne accumulator for all of k, or parts of k that are added up in registers: of kExact or kLong each.
// PLANES: results of kResidual are the planes of fp32 values.
enum Sums { kOne, kExactParts, kLongParts };
template <int PAIR, int ENDING, int SUMS, bool PLANES = false>
__global__ void __launch_bounds__(kThreads, 1) tile_kernel(const __grid_constant__ TileArgs t) {
    using S = Shape<PAIR>;
    constexpr bool EXACT = SUMS == kExactParts;
    // k of the parts, and of a tile's first one: for the residuals as long as the MMAs need to go on while the results of
    // the tile before leave (with 256 they waited, and a score of 4,096 x 4,096 x 32,768 took 8 % longer).
    constexpr int kPart = SUMS == kLongParts ? kLong : kExact, kFirst = ENDING == kResidual && !PLANES ? kLong : kPart;
    extern __shared__ char raw[];
    __shared__ Shared s;
    char* const ring = raw + ((1024 - (smem_addr(raw) & 1023)) & 1023);
    const Product& p = t.p;
    const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;
    const uint32_t rank = PAIR == 2 ? block_rank() : 0;

    if (threadIdx.x == 0) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&t.a) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&t.b) : "memory");
        if (p.ragged == kRaggedN) asm volatile("prefetch.tensormap [%0];" ::"l"(&t.few) : "memory");
        for (int i = 0; i < S::kStages; ++i) {
            mbar_init(&s.full[i], PAIR);
            mbar_init(&s.empty[i], 1);
            mbar_init(&s.tail[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&s.ready[i], 1);
            mbar_init(&s.taken[i], kEnds * PAIR);
        }
        s.late = 0;
        s.rounds = 0;
        s.limit = t.limit;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        if (PAIR == 2)
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&s.tmem)), "n"(kColumns)
                         : "memory");
        else
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&s.tmem)), "n"(kColumns)
                         : "memory");
    }
    // Nothing in global memory is touched before the kernels before this one have ended.
    pdl_wait();
    pdl_trigger();
    if (p.ragged != kNotRagged) count_tiles(p, s);
    fence_before();
    __syncthreads();
    if (PAIR == 2) {
        asm volatile("barrier.cluster.arrive.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
    }
    fence_after();
    const uint32_t tmem = *(volatile uint32_t*)&s.tmem;
    const uint32_t pairs = p.planes ? kPairs : 1;
    const Sizes sizes = sizes_of<PAIR>(t, s);
    const int64_t items = sizes.items, team = blockIdx.x / PAIR, teams = gridDim.x / PAIR;

    // 384 threads are launched with 168 registers; 128 x 56 + 256 x 216 are fewer.
    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        if (warp == 0) {
            // Copies, by one thread.
            if (elected()) {
                const uint32_t to = smem_addr(ring);
                const uint32_t full = PAIR == 2 ? first_block(smem_addr(&s.full[0])) : smem_addr(&s.full[0]);
                uint32_t stage = 0, phase = 0, rounds = 0;
                bool ok = true;
                for (int64_t i = team; i < items && ok; i += teams) {
                    const Tile w = tile_of<PAIR>(t, s, sizes, i);
                    const Boxes x = boxes_of<PAIR>(t, w);
                    const int32_t m0 = (int32_t)(w.m0 + rank * kBlockM), n0 = (int32_t)(w.n0 + (int64_t)rank * x.rows_b);
                    const int32_t ga = p.ragged == kRaggedN ? w.group : 0;
                    for (uint32_t pair = 0; pair < pairs && ok; ++pair) {
                        const int32_t pa = t.planes_a >> 4 * pair & 15u, pb = t.planes_b >> 4 * pair & 15u;      // (one pair: 0)
                        for (int64_t k64 = w.k0; k64 < w.k1; k64 += kK) {
                            const int32_t k = (int32_t)k64;
                            if (!(ok = wait_thread(&s.empty[stage], phase ^ 1, s))) break;
                            const uint32_t bar = cut(p, w, k64) ? smem_addr(&s.tail[stage]) : full + 8 * stage;
                            const uint32_t to_a = to + stage * S::kStage, to_b = to_a + kSideA;
                            arrive_expect(bar, x.bytes);
                            if (!p.a.across)
                                copy_box<PAIR>(&t.a, to_a, bar, k, m0, 0, ga, pa);
                            else if (t.wide_a)
                                copy_box<PAIR>(&t.a, to_a, bar, 0, k, m0 / 64, ga, pa);
                            else
                                for (int j = 0; j < kBlockM / 64; ++j)
                                    copy_box<PAIR>(&t.a, to_a + j * 8192, bar, m0 + j * 64, k, 0, ga, pa);
                            if (x.few)
                                for (int j = 0; j < x.boxes_b; ++j)
                                    copy_box<PAIR>(&t.few, to_b + j * kFew * kK * 2, bar, k, n0 + j * kFew, 0, 0, pb);
                            else if (!p.b.across)
                                copy_box<PAIR>(&t.b, to_b, bar, k, n0, 0, 0, pb);
                            else if (t.wide_b)
                                copy_box<PAIR>(&t.b, to_b, bar, 0, k, n0 / 64, 0, pb);
                            else
                                for (int j = 0; j < x.boxes_b; ++j)
                                    copy_box<PAIR>(&t.b, to_b + j * 8192, bar, n0 + j * 64, k, 0, 0, pb);
                            if (++stage == S::kStages) {
                                stage = 0;
                                phase ^= 1;
                                s.rounds = ++rounds;      // (with every stage it cost 1 %)
                            }
                        }
                    }
                }
                if (!ok) {      // copies in flight end within this
                    const uint64_t t0 = global_ns();
                    for (uint32_t i = 0; i < (1u << 24) && global_ns() - t0 < 2000000; ++i) {
                    }
                }
            }
            __syncwarp();
        } else if (warp == 2) {
            // Ragged k: in a group's last copy, rows of other groups become 0 (both sides are across: a
            // row is 128 bytes of each chunk).
            if (p.ragged == kRaggedK) {
                uint32_t copies = 0, used = 0;      // copies: modulo the stages
                bool ok = true;
                for (int64_t i = team; i < items && ok; i += teams) {
                    const Tile w = tile_of<PAIR>(t, s, sizes, i);
                    const int rows = (int)((w.k1 - w.k0) % kK);
                    for (uint32_t pair = 0; pair < pairs && w.k0 < w.k1 && ok; ++pair) {
                        copies = (uint32_t)((copies + (w.k1 - w.k0 + kK - 1) / kK) % S::kStages);
                        if (rows == 0) continue;
                        const uint32_t stage = (copies + S::kStages - 1) % S::kStages;
                        if (!(ok = wait(&s.tail[stage], used >> stage & 1, s))) break;
                        used ^= 1u << stage;
                        const int chunks = (int)(boxes_of<PAIR>(t, w).bytes / 8192);
                        char* const at = ring + stage * S::kStage;
                        for (int j = lane; j < chunks * (kK - rows) * 8; j += 32) {
                            const int c = j / ((kK - rows) * 8), r = j % ((kK - rows) * 8);
                            *reinterpret_cast<float4*>(at + c * 8192 + rows * 128 + r * 16) = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                        }
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                        __syncwarp();
                        if (lane == 0) {
                            if (PAIR == 2)
                                arrive_first<true>(&s.full[stage]);
                            else
                                mbar_arrive(&s.full[stage]);
                        }
                    }
                }
            }
        } else if (warp == 1) {
            // MMAs: one thread of the pair's first block issues them.  It is elected, so that the compiler
            // knows that it is one, and counts in 32 bits: by `lane == 0` and in 64 bits the tensor cores
            // waited for it (1,530 TFLOP/s for 1,760 at 8,192 of m, n and k).
            if (rank == 0 && elected()) {
                uint32_t stage = 0, phase = 0, tile = 0;
                const uint32_t kind = p.dtype == FASGD_BF16 ? 1u << 7 | 1u << 10 : 0u;
                const uint32_t base = 1u << 4 | kind | (uint32_t)(p.a.across != 0) << 15 | (uint32_t)(p.b.across != 0) << 16 |
                                      (uint32_t)(kBlockM * PAIR / 16) << 24;
                const uint32_t next_a = p.a.across ? 2048 >> 4 : 32 >> 4, next_b = p.b.across ? 2048 >> 4 : 32 >> 4;
                const uint64_t a0 = matrix_of(smem_addr(ring), p.a.across), b0 = matrix_of(smem_addr(ring) + kSideA, p.b.across);
                const uint32_t a_high = (uint32_t)(a0 >> 32), b_high = (uint32_t)(b0 >> 32);
                // The next tile with sums and the next accumulator are looked up while MMAs run.
                int64_t i = team - teams;
                int blocks = 0, last = 0;                 // of 64 k each, of every pair of planes; MMAs of the last one
                uint32_t shape = 0;
                bool zeroed = false, ok = true;           // zeroed: that holds rows set to 0
                const auto look = [&] {
                    blocks = 0;
                    while (blocks == 0 && (i += teams) < items) {
                        const Tile w = tile_of<PAIR>(t, s, sizes, i);
                        if (w.k0 >= w.k1) continue;
                        blocks = (int)((w.k1 - w.k0 + kK - 1) / kK);
                        last = (int)((w.k1 - w.k0 + 15) / 16) - (blocks - 1) * (kK / 16);
                        shape = base | (uint32_t)(width_of<PAIR>(t, w) / 8) << 17;
                        zeroed = p.ragged == kRaggedK && (w.k1 - w.k0) % kK != 0;
                    }
                };
                look();
                while (blocks > 0 && ok) {
                    const int each = blocks, all = each * (int)pairs, chunk = SUMS == kOne ? all : kPart / kK, mmas = last;
                    const uint32_t now = shape;
                    const bool cuts = zeroed;
                    int in = 0;                           // blocks of this pair of planes
                    const auto part = [&](int done) { return SUMS != kOne && kFirst != kPart && done == 0 ? kFirst / kK : chunk; };
                    for (int done = 0; done < all && ok; done += part(done)) {
                        const int until = min(done + part(done), all);
                        if (!(ok = wait_thread(&s.taken[tile & 1], (tile >> 1 & 1) ^ 1, s))) break;
                        fence_after();
                        const uint32_t to = tmem + (tile & 1) * kTileN;
                        uint32_t add = 0;
                        for (int k = done; k < until; ++k) {
                            const bool end = ++in == each;
                            ok = PAIR == 2 && cuts && end ? wait_thread<true>(&s.full[stage], phase, s)
                                                          : wait_thread(&s.full[stage], phase, s);
                            if (!ok) break;
                            fence_after();
                            const uint32_t a = (uint32_t)a0 + stage * (S::kStage >> 4), b = (uint32_t)b0 + stage * (S::kStage >> 4);
                            mma<PAIR>(to, a, b, a_high, b_high, now, add);
                            add = 1;
                            if (!end) {
#pragma unroll
                                for (int j = 1; j < 4; ++j) mma<PAIR>(to, a + j * next_a, b + j * next_b, a_high, b_high, now, true);
                            } else {
                                for (int j = 1; j < mmas; ++j) mma<PAIR>(to, a + j * next_a, b + j * next_b, a_high, b_high, now, true);
                                in = 0;
                            }
                            commit<PAIR>(&s.empty[stage]);
                            if (++stage == S::kStages) {
                                stage = 0;
                                phase ^= 1;
                            }
                        }
                        if (ok) commit<PAIR>(&s.ready[tile & 1]);
                        ++tile;
                        if (done == 0) look();
                    }
                }
            }
            __syncwarp();
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
        // Results.  The warp's lanes of tensor memory are those of its number modulo 4; two warps share
        // them, one with the even 32 columns, one with the odd ones.
        const int quarter = warp & 3, odd = (warp - 4) >> 2;
        const float more = log2f(p.factor);
        const Target target = {p.out, p.ld_out, p.scale, p.factor, p.by_n, p.out_dtype, p.add};
        if (p.ragged == kRaggedN) clear_rows(p, s, blockIdx.x, gridDim.x, threadIdx.x - 128, 32 * kEnds);
        uint32_t tile = 0, turn = 0;
        bool ok = true;
        for (int64_t i = team; i < items; i += teams, turn ^= 1) {
            const Tile w = tile_of<PAIR>(t, s, sizes, i);
            const int64_t m = w.m0 + rank * kBlockM + quarter * 32 + lane;
            const bool live = m < p.m;
            const int count = (int)(w.n1 - w.n0);
            const int64_t blocks = w.k0 < w.k1 ? (w.k1 - w.k0 + kK - 1) / kK * pairs : 0;
            const auto taken = [&](uint32_t buffer) {
                fence_before();
                __syncwarp();
                if (lane == 0) {
                    if (PAIR == 2)
                        arrive_first(&s.taken[buffer]);
                    else
                        mbar_arrive(&s.taken[buffer]);
                }
            };
            const auto columns_of = [&](uint32_t buffer) {
                return tmem + buffer * kTileN + ((uint32_t)(quarter * 32) << 16) + odd * 32;
            };
            // What the endings know of the row m, and of its label's column of this tile.
            const int64_t label = ENDING != kStore && live ? p.labels[m] : -1;
            const bool has = label >= 0 && label < p.classes;
            const int64_t in = label - p.n0 - w.n0;
            const int at = has && in >= 0 && in < count ? (int)in : -1;
            const bool mine = at >= 0 && (at >> 5 & 1) == odd;
            const float lse = ENDING == kResidual && has ? p.lse[m] : 0.0f;
            const float own = ENDING == kResidual && mine ? target.factor * expm1f(-p.row_loss[m]) : 0.0f;
            const int64_t base = (ENDING == kStore ? (p.ragged == kRaggedK ? w.group * p.step_out : 0) + w.split * p.step_split : 0) +
                                 w.n0 * target.ld + m;
            // Columns c ... c + 31 of the tile into out.
            const auto end_columns = [&](int c, const float (&x)[32]) {
                if (ENDING == kStore) {
                    if (EXACT && !target.add)
                        store_columns<float>(target, base + c * target.ld, w.n0 + c, min(32, count - c), live, x);
                    else if (EXACT)
                        add_columns(target, base + c * target.ld, min(32, count - c), live, x);
                    else
                        store_any(target, base + c * target.ld, w.n0 + c, min(32, count - c), live, x);
                    return;
                }
                if (!live) return;
                const int own_at = mine ? at - c : -1;
                if (PLANES) {
                    __nv_bfloat16* out = static_cast<__nv_bfloat16*>(target.out) + base + c * target.ld;
#pragma unroll
                    for (int j = 0; j < 32; ++j)
                        if (j < count - c) {
                            __nv_bfloat16 y[3];
                            planes_of(j == own_at ? own : has ? exp2_fast((x[j] - lse) * kLog2E) : 0.0f, y);
#pragma unroll
                            for (int i = 0; i < 3; ++i) out[i * p.step_plane] = y[i];
                            out += target.ld;
                        }
                    return;
                }
                const auto write = [&](auto* out) {
                    using T = std::remove_reference_t<decltype(*out)>;
                    out += base + c * target.ld;
#pragma unroll
                    for (int j = 0; j < 32; ++j)
                        if (j < count - c) {
                            *out = from_f32<T>(has ? exp2_fast(fmaf(x[j] - lse, kLog2E, more)) : 0.0f);
                            out += target.ld;
                        }
                    if ((uint32_t)own_at < 32u) out[(own_at - min(32, count - c)) * target.ld] = from_f32<T>(own);
                };
                if (target.dtype == FASGD_BF16)
                    write(static_cast<__nv_bfloat16*>(target.out));
                else
                    write(static_cast<__half*>(target.out));
            };
            if constexpr (SUMS == kOne) {
                // 32 columns after the other, out of tensor memory and on their way: a loop that stays in the
                // instruction cache (for all 128 at once the code outgrew it: 38,000 cycles a tile of g).
                const uint32_t buffer = tile & 1;
                if (blocks > 0) {
                    ok = ok && wait(&s.ready[buffer], tile >> 1 & 1, s);
                    ++tile;
                    fence_after();
                }
#pragma unroll 1
                for (int c = odd * 32; c < count; c += 64) {
                    float x[32];
                    if (blocks > 0 && ok) {
                        load_columns(columns_of(buffer) + (c - odd * 32), x);
                        wait_columns();
                    } else {
#pragma unroll
                        for (int j = 0; j < 32; ++j) x[j] = ok ? 0.0f : NAN;
                    }
                    if (c + 64 >= count && blocks > 0) taken(buffer);
                    end_columns(c, x);
                }
                if (odd * 32 >= count && blocks > 0) taken(buffer);
            } else {
                float v[4][32];
#pragma unroll
                for (int b = 0; b < 4; ++b)
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[b][j] = 0.0f;
                for (int64_t k = 0; k < blocks; k += (k == 0 ? kFirst : kPart) / kK) {
                    const uint32_t buffer = tile & 1;
                    ok = ok && wait(&s.ready[buffer], tile >> 1 & 1, s);
                    ++tile;
                    fence_after();
                    if (!ok) break;
                    const uint32_t from = columns_of(buffer);
                    if (k == 0) {
#pragma unroll
                        for (int b = 0; b < 4; ++b)
                            if (b * 64 + odd * 32 < count) load_columns(from + b * 64, v[b]);
                        wait_columns();
                    } else {
#pragma unroll
                        for (int b = 0; b < 8; ++b)
                            if (b / 2 * 64 + odd * 32 < count) {
                                float more_of[16];
                                load_half(from + b / 2 * 64 + b % 2 * 16, more_of);
                                wait_columns();
#pragma unroll
                                for (int j = 0; j < 16; ++j) v[b / 2][b % 2 * 16 + j] += more_of[j];
                            }
                    }
                    taken(buffer);
                }
                if (!ok)
#pragma unroll
                    for (int b = 0; b < 4; ++b)
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[b][j] = NAN;
                // The registers' 32 columns after the other, in a loop that moves them down (for the same reason).
                float top = -INFINITY, sum = 0.0f;
#pragma unroll 1
                for (int c = odd * 32; c < count; c += 64) {
                    if constexpr (ENDING != kStatistics) {
                        end_columns(c, v[0]);
                    } else {
                        if (count - c < 32)
#pragma unroll
                            for (int j = 0; j < 32; ++j) v[0][j] = j < count - c ? v[0][j] : -INFINITY;
                        float most[4] = {top, v[0][1], v[0][2], v[0][3]};
#pragma unroll
                        for (int j = 0; j < 32; ++j) most[j & 3] = fmaxf(most[j & 3], v[0][j]);
                        const float next = fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3]));
                        if (__any_sync(0xffffffffu, mine && at >> 5 == c >> 5)) {
#pragma unroll
                            for (int j = 0; j < 32; ++j)
                                if (mine && at == c + j) p.at_label[m] = v[0][j];
                        }
                        const float shift = fabsf(next) == INFINITY ? 0.0f : next;      // (of an infinite one the sum is)
                        float part[4] = {sum * exp2_fast((top - shift) * kLog2E), 0.0f, 0.0f, 0.0f};
#pragma unroll
                        for (int j = 0; j < 32; ++j) part[j & 3] += exp2_fast((v[0][j] - shift) * kLog2E);
                        sum = (part[0] + part[1]) + (part[2] + part[3]);
                        top = next;
                    }
#pragma unroll
                    for (int b = 0; b < 3; ++b)
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[b][j] = v[b + 1][j];
                }
                if constexpr (ENDING == kStatistics) {
                    float2* const other = &s.halves[turn][quarter * 32 + lane];
                    if (odd) *other = make_float2(top, sum);
                    asm volatile("bar.sync %0, 64;" ::"r"(quarter + 1) : "memory");
                    if (!odd && live) {
                        const float2 o = *other;
                        const float most = fmaxf(top, o.x), zero = fabsf(most) == INFINITY ? 0.0f : most;
                        sum = sum * exp2_fast((top - zero) * kLog2E) + o.y * exp2_fast((o.x - zero) * kLog2E);
                        p.parts[w.n_tile * p.m + m] = make_float2(most, sum);
                    }
                }
            }
        }
    }
    fence_before();
    __syncthreads();
    if (threadIdx.x == 0 && s.late != 0) waits_ran_out = 1;
    if (PAIR == 2) {      // no block leaves while its pair may still reach its memory
        asm volatile("barrier.cluster.arrive.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
    }
    if (warp == 1) {
        fence_after();
        if (PAIR == 2) {
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
            asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(kColumns));
        } else {
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
            asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(kColumns));
        }
    }
}

// One thread's and a warp's wait for a barrier that nobody arrives at.
__global__ void __launch_bounds__(64) expiry_kernel(uint64_t limit) {
    __shared__ Shared s;
    if (threadIdx.x == 0) {
        mbar_init(&s.full[0], 1);
        s.late = 0;
        s.rounds = 0;
        s.limit = limit;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    if (threadIdx.x == 0) wait_thread(&s.full[0], 0, s);
    if (threadIdx.x >= 32) wait(&s.full[0], 0, s);
    __syncthreads();
    if (threadIdx.x == 0 && s.late != 0) waits_ran_out = 1;
}

// ---- host -------------------------------------------------------------------------------
std::atomic<uint64_t> wait_limit{kWaitLimitNs};

using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                            const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                            CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
Encode encoder() {
    static const Encode f = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult found = cudaDriverEntryPointSymbolNotFound;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess)
            cudaGetLastError();
        return found == cudaDriverEntryPointSuccess ? reinterpret_cast<Encode>(p) : nullptr;
    }();
    return f;
}
// How a side lies: `size` values of its index (all groups' rows, where it is ragged), k of the sums.
// box: how many of the index a box has; wide (a side that is across): as chunks of 64, which
// have to be whole ones.
bool encode(CUtensorMap* map, const Side& s, const Product& p, int64_t size, int64_t groups, int box, bool wide) {
    const int64_t k = p.k;
    const auto u = [](int64_t n) { return (cuuint64_t)n; };
    const cuuint64_t ld = u(s.ld) * 2, step = groups > 1 ? u(s.step) * 2 : ld;
    const cuuint64_t dims[5] = {u(wide ? 64 : s.across ? size : k), u(s.across ? k : size), u(wide ? size / 64 : 1), u(groups),
                                p.planes ? (cuuint64_t)s.planes : 1u};
    const cuuint64_t strides[4] = {ld, wide ? 128 : ld, step, p.planes ? u(s.plane) * 2 : ld};
    const cuuint32_t boxes[5] = {64, (cuuint32_t)(s.across ? kK : box), wide ? (cuuint32_t)box / 64 : 1, 1, 1},
                     one[5] = {1, 1, 1, 1, 1};
    const Encode f = encoder();
    return f != nullptr &&
           f(map, p.dtype == FASGD_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 5,
             const_cast<void*>(s.p), dims, strides, boxes, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int PAIR, int ENDING, int SUMS, bool PLANES = false>
cudaError_t launch(const TileArgs& t, int64_t most, int device, int sms, cudaStream_t stream) {
    static SharedLimit limit;
    const int bytes = Shape<PAIR>::kBytes;
    const int error = limit.ensure(device, bytes, bytes, [](int64_t n) {
        return (int)cudaFuncSetAttribute(tile_kernel<PAIR, ENDING, SUMS, PLANES>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)n);
    });
    if (error != 0) return (cudaError_t)error;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)std::min<int64_t>(most, sms / PAIR) * PAIR);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = PAIR;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, tile_kernel<PAIR, ENDING, SUMS, PLANES>, t);
}
template <int PAIR>
cudaError_t launch(TileArgs& t, int device, int sms, cudaStream_t stream) {
    const Product& p = t.p;
    t.m_tiles = (p.m + kBlockM * PAIR - 1) / (kBlockM * PAIR);
    t.tile_n = p.ending == kStatistics ? statistics_tile(p.m, p.n) : kTileN;
    const int64_t n_tiles = (p.n + t.tile_n - 1) / t.tile_n + (p.ragged == kRaggedN ? p.groups : 0);
    t.items = t.m_tiles * n_tiles * t.splits * (p.ragged == kRaggedK ? p.groups : 1);
    if (t.items == 0) return cudaSuccess;
    t.planes_a = p.planes ? planes_a(p.a.planes) : 0;
    t.planes_b = p.planes ? planes_b(p.b.planes) : 0;
    t.wide_a = p.a.across && p.m % 64 == 0;
    t.wide_b = p.b.across && p.n % 64 == 0 && t.tile_n == kTileN;
    if (!encode(&t.a, p.a, p, p.m, p.ragged == kRaggedN ? p.groups : 1, kBlockM, t.wide_a) ||
        !encode(&t.b, p.b, p, p.n, 1, t.tile_n / PAIR, t.wide_b) ||
        (p.ragged == kRaggedN && !encode(&t.few, p.b, p, p.n, 1, kFew, false)))
        return cudaErrorInvalidValue;
    switch (p.ending) {
        case kStore: {
            const bool exact = p.exact && p.out_dtype == FASGD_F32;
            // (of ragged k one group may have all)
            return exact                                 ? launch<PAIR, kStore, kExactParts>(t, t.items, device, sms, stream)
                   : p.k > (int64_t)kLongFrom * t.splits ? launch<PAIR, kStore, kLongParts>(t, t.items, device, sms, stream)
                                                         : launch<PAIR, kStore, kOne>(t, t.items, device, sms, stream);
        }
        case kStatistics: return launch<PAIR, kStatistics, kExactParts>(t, t.items, device, sms, stream);
        default:
            // What one accumulator cuts of s (kLong: 6e-5 of it at most, 1.4e-5 as a rule) is a relative error of exp(s - lse)
            // as large as s times that: below rounding to 16 bits for |s| of some 30 (bf16: 100).  Longer rows' sums go on
            // in exact parts, so that they lose no more.
            return p.planes      ? launch<PAIR, kResidual, kExactParts, true>(t, t.items, device, sms, stream)
                   : p.k > kLong ? launch<PAIR, kResidual, kExactParts>(t, t.items, device, sms, stream)
                                 : launch<PAIR, kResidual, kOne>(t, t.items, device, sms, stream);
    }
}

}  // namespace

bool tile_side(const Side& s, int64_t groups) {
    constexpr int64_t kFar = (int64_t)1 << 38;      // values that a copy's steps can be apart, and more
    return (reinterpret_cast<uintptr_t>(s.p) & 15) == 0 && s.ld % 8 == 0 && s.ld < kFar &&
           (groups < 2 || (s.step % s.ld == 0 && s.step < kFar));
}

// The plan that should take the least time, by what was measured on a GB300: 64 k of a tile take a
// block or a pair 0.27 us times the n of the tile over 256 (a block alone a quarter more), and no less
// than 50 GB/s and SM copy its sides in; a group's last rows take a pair 1.2 us a tile (a release that its other block sees),
// a block alone 0.4; parts of k cost their sums' way through memory and a launch.
TilePlan plan_tiles(const Product& p) {
    constexpr int kSms = 152;
    const bool rows = p.ragged == kRaggedN;
    const int64_t groups = rows ? std::min<int64_t>(p.groups, p.n) : p.ragged == kRaggedK ? p.groups : 1;
    const int64_t k = p.ragged == kRaggedK ? (p.k + p.groups - 1) / p.groups : p.k;
    const int64_t blocks = std::max<int64_t>(1, (k + kK - 1) / kK * (p.planes ? kPairs : 1));
    const int64_t per = rows ? std::max<int64_t>(1, p.n / std::max<int64_t>(1, groups)) : p.n;
    const int64_t n_tiles = rows ? std::max<int64_t>(groups, (p.n + kTileN - 1) / kTileN) : (p.n + kTileN - 1) / kTileN;
    const double width = (double)std::min<int64_t>(per, kTileN);
    TilePlan best = {p.m > kBlockM ? 2 : 1, 1};
    double least = 1e300;
    for (int pair = p.m > kBlockM ? 2 : 1; pair >= 1; --pair) {
        const int64_t tiles = (p.m + kBlockM * pair - 1) / (kBlockM * pair) * n_tiles * (p.ragged == kRaggedK ? groups : 1);
        const int teams = kSms / pair;
        const double each = std::max(0.27 * width / 256.0 * (pair == 1 ? 1.25 : 1.0),
                                     (kSideA + std::max(width / pair, 32.0) * kK * 2) / 50e3);
        for (int splits = 1; splits <= 16 && (splits == 1 || (p.ending == kStore && blocks >= 8 * splits)); ++splits) {
            const double waves = (double)((tiles * splits + teams - 1) / teams);
            const double cut = p.ragged != kRaggedK ? 0.0 : pair == 2 ? 1.2 : 0.4;
            double time = waves * ((double)((blocks + splits - 1) / splits) * each + cut);
            if (splits > 1) time += 4.0 + (double)p.m * (double)p.n * (double)groups * splits * (p.add ? 16.0 : 8.0) / 5e6 / (rows ? (double)groups : 1.0);
            if (time < least * 0.97) {
                least = time;
                best = {pair, splits};
            }
        }
    }
    return best;
}

void set_wait_limit(uint64_t ns) { wait_limit.store(ns, std::memory_order_relaxed); }

cudaError_t launch_expiry(cudaStream_t stream) {
    expiry_kernel<<<1, 64, 0, stream>>>(wait_limit.load(std::memory_order_relaxed));
    return cudaGetLastError();
}

cudaError_t read_late(int32_t* late, cudaStream_t stream) {
    int32_t is = 0;
    const int32_t none = 0;
    cudaError_t st = cudaMemcpyFromSymbolAsync(&is, waits_ran_out, sizeof is, 0, cudaMemcpyDeviceToHost, stream);
    if (st == cudaSuccess) st = cudaStreamSynchronize(stream);
    if (st == cudaSuccess && is != 0) {
        st = cudaMemcpyToSymbolAsync(waits_ran_out, &none, sizeof none, 0, cudaMemcpyHostToDevice, stream);
        if (st == cudaSuccess) st = cudaStreamSynchronize(stream);
    }
    if (st == cudaSuccess) *late = is;
    return st;
}

cudaError_t launch_tiles(const Product& p, const TilePlan& plan, cudaStream_t stream) {
    int device = 0, sms = 0;
    cudaError_t st = cudaGetDevice(&device);
    if (st == cudaSuccess) st = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device);
    if (st != cudaSuccess) return st;
    TileArgs t = {};
    t.p = p;
    t.splits = plan.splits;
    t.limit = wait_limit.load(std::memory_order_relaxed);
    return plan.pair == 2 ? launch<2>(t, device, sms, stream) : launch<1>(t, device, sms, stream);
}

}  // namespace fasgd
