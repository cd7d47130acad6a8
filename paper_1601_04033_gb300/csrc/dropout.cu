// fasgd_dropout: out = residual + m x scale, the mask drawn where it is used.

#include "octet.cuh"
#include "pdl.cuh"

namespace fasgd {
namespace {

constexpr int kThreads = 256;

template <class T>
__device__ __forceinline__ T drop_one(T x, bool keep, float scale, bool residual, T res) {
    const float v = keep ? to_f32(x) * scale : 0.f;
    return from_f32<T>(residual ? v + to_f32(res) : v);
}

// Any strides and alignments, from octet `from` on: a thread takes an octet of the
// matrix's elements, which may end in a later row than it began in.
template <class T>
__global__ void __launch_bounds__(kThreads) dropout_any_kernel(const __grid_constant__ DropoutArgs a, int64_t from) {
    pdl_wait();
    pdl_trigger();
    const T* x = static_cast<const T*>(a.x);
    const T* res = static_cast<const T*>(a.residual);
    T* out = static_cast<T*>(a.out);
    const int64_t count = a.rows * a.cols, octets = (count + 7) >> 3;
    const int64_t stride = (int64_t)gridDim.x * kThreads;
    for (int64_t q = from + (int64_t)blockIdx.x * kThreads + threadIdx.x; q < octets; q += stride) {
        const Philox4 r = draw_octet(a.drop, q);
        int64_t row = (q << 3) / a.cols, col = (q << 3) - row * a.cols;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (row >= a.rows) break;
            out[row * a.ld_out + col] =
                drop_one<T>(x[row * a.ld_x + col], kept(r, i, a.drop.cut), a.drop.scale,
                            res != nullptr, res != nullptr ? res[row * a.ld_residual + col] : T());
            if (++col == a.cols) {
                col = 0;
                ++row;
            }
        }
    }
}

// Whole octets of rows that begin with one (a matrix without gaps is one row): a
// block takes kThreads * U of them and each thread U, all asked for before the
// first is used.  Bound by memory: 65536 x 4096 bf16 with a residual, 1.6 GB, and
// its gradient, 1.1 GB: 387 us, 6.94 TB/s; six thousand strided rows of 1,000 in
// 12 us for both, out of L2.
struct DropoutRows {
    int64_t octets, row_octets;      // of the matrix, of a row
    int64_t turn_rows, turn_octets;  // kThreads octets on: rows, and octets of a row
};
template <class T, bool RES, int U>
__global__ void __launch_bounds__(kThreads)
    dropout_octets_kernel(const __grid_constant__ DropoutArgs a, const __grid_constant__ DropoutRows m) {
    pdl_wait();
    pdl_trigger();
    const int64_t q0 = (int64_t)blockIdx.x * (kThreads * U) + threadIdx.x;
    int64_t row = 0, col = q0;       // in octets
    if (m.octets > m.row_octets) {
        row = m.octets >> 32 == 0 ? (int64_t)((uint32_t)q0 / (uint32_t)m.row_octets) : q0 / m.row_octets;
        col = q0 - row * m.row_octets;
    }
    uint4 x[U][kPieces<T>], res[RES ? U : 1][kPieces<T>];
    int64_t at[U];                   // of the output
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (q0 + u * kThreads < m.octets) {
            load_pieces(static_cast<const T*>(a.x) + row * a.ld_x + col * kOctet, x[u]);
            if (RES) load_pieces(static_cast<const T*>(a.residual) + row * a.ld_residual + col * kOctet, res[u]);
        }
        at[u] = row * a.ld_out + col * kOctet;
        row += m.turn_rows;
        col += m.turn_octets;
        if (col >= m.row_octets) {
            col -= m.row_octets;
            ++row;
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t q = q0 + u * kThreads;
        if (q >= m.octets) break;
        const Philox4 r = draw_octet(a.drop, q);
        Oct o = unpack<T>(x[u]), s;
        if (RES) s = unpack<T>(res[u]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            o.v[i] = keep2(r, i, a.drop.last, mul2(o.v[i], f2(a.drop.scale)));
            if (RES) o.v[i] = add2(o.v[i], s.v[i]);
        }
        uint4 raw[kPieces<T>];
        pack<T>(o, raw);
        store_pieces(static_cast<T*>(a.out) + at[u], raw);
    }
}

template <class T, bool RES, int U>
cudaError_t launch_octets(const DropoutArgs& a, const DropoutRows& m, cudaStream_t stream) {
    const int64_t grid = (m.octets + kThreads * U - 1) / (kThreads * U);
    return launch_pdl(dropout_octets_kernel<T, RES, U>, (unsigned)grid, kThreads, 0, stream, a, m);
}

template <class T>
cudaError_t launch(const DropoutArgs& a, int num_sms, cudaStream_t stream) {
    const int64_t count = a.rows * a.cols;
    const bool gapless = a.rows < 2 || (a.ld_x == a.cols && a.ld_out == a.cols &&
                                        (a.residual == nullptr || a.ld_residual == a.cols));
    const auto fits = [&](const void* p, int64_t ld) {
        return p == nullptr || (reinterpret_cast<uintptr_t>(p) % (kOctet * sizeof(T)) == 0 &&
                                (gapless || (a.cols % kOctet == 0 && ld % kOctet == 0)));
    };
    // (At cut 0 keep2 would drop draws of 0; the kernel of any layout takes it, 16384 x 4096
    // bf16 both directions in 354 us, 100 with draws.)
    if (a.drop.cut != 0 && fits(a.x, a.ld_x) && fits(a.residual, a.ld_residual) && fits(a.out, a.ld_out)) {
        DropoutRows m;
        m.octets = count / kOctet;
        m.row_octets = gapless ? m.octets : a.cols / kOctet;
        if (m.octets > 0 && m.octets < ((int64_t)1 << 38)) {
            m.turn_rows = kThreads / m.row_octets;
            m.turn_octets = kThreads % m.row_octets;
            // Four a thread where that leaves every SM eight blocks.
            const bool four = m.octets >= (int64_t)num_sms * 8 * 4 * kThreads;
            cudaError_t st;
            if (a.residual != nullptr)
                st = four ? launch_octets<T, true, 4>(a, m, stream) : launch_octets<T, true, 1>(a, m, stream);
            else
                st = four ? launch_octets<T, false, 4>(a, m, stream) : launch_octets<T, false, 1>(a, m, stream);
            if (st != cudaSuccess || m.octets * kOctet == count) return st;
            // The last, begun octet of a gapless matrix.
            return launch_pdl(dropout_any_kernel<T>, 1, kThreads, 0, stream, a, m.octets);
        }
    }
    int64_t grid = ((count + 7) / 8 + kThreads - 1) / kThreads;
    if (grid > (int64_t)num_sms * 16) grid = (int64_t)num_sms * 16;
    return launch_pdl(dropout_any_kernel<T>, (unsigned)grid, kThreads, 0, stream, a, (int64_t)0);
}

}  // namespace

cudaError_t launch_dropout(const DropoutArgs& a, int dtype, int num_sms, cudaStream_t stream) {
    if (a.rows == 0) return cudaSuccess;
    if (dtype == FASGD_F32) return launch<float>(a, num_sms, stream);
    if (dtype == FASGD_BF16) return launch<__nv_bfloat16>(a, num_sms, stream);
    return launch<__half>(a, num_sms, stream);
}

}  // namespace fasgd
