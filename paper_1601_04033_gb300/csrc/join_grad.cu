// The plan of a gradient call, and its launch by type (join_grad.cuh has the
// kernels; each type is a translation unit of its own, for the time it takes).

#include "join_grad.cuh"

namespace fasgd {

cudaError_t launch_join_grad_f32(const JoinArgs& a, int num_sms, cudaStream_t stream);
cudaError_t launch_join_grad_bf16(const JoinArgs& a, int num_sms, cudaStream_t stream);
cudaError_t launch_join_grad_f16(const JoinArgs& a, int num_sms, cudaStream_t stream);

// Splits of each group's rows for `most` subs: fewest row turns of the busiest
// sub, a unit costing about four more to begin and to leave its sums.
static int64_t best_splits(int64_t groups, int64_t rows, int64_t most, int64_t step) {
    int64_t best = step, least = INT64_MAX;
    for (int64_t rounds = 0; rounds <= 16; ++rounds) {        // the most splits of so many units a sub
        int64_t s = rounds * most / groups / step * step;
        s = s < step ? step : s > rows ? rows / step * step : s;
        const int64_t cost = (groups * s + most - 1) / most * ((rows + s - 1) / s + 4);
        if (cost < least) {
            least = cost;
            best = s;
        }
    }
    return best;
}

JoinPlan join_grad_plan(const JoinArgs& a, int dtype, int num_sms) {
    JoinPlan p;
    p.parts = p.splits = p.row_means = 0;
    if (a.rows == 0) return p;
    const RowForm form = form_of(a, dtype == FASGD_F32 ? 4 : 2);
    if (form != kValues) {
        const RowShape s(row_octets(a.cols), kGradThreads, form == kLoose);
        const int64_t block_subs = s.rows, per_sm = kGradThreads / s.threads;
        const int64_t most = (int64_t)num_sms * per_sm / s.blocks / 8 * 8 * block_subs;
        if (a.groups == 1) {
            p.splits = at_most(a.rows, most);
        } else {
            p.splits = best_splits(a.groups, a.group_rows, most, a.cols % 8 != 0 ? 8 : 1);
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
    if (dtype == FASGD_F32) return launch_join_grad_f32(a, num_sms, stream);
    if (dtype == FASGD_BF16) return launch_join_grad_bf16(a, num_sms, stream);
    return launch_join_grad_f16(a, num_sms, stream);
}

}  // namespace fasgd
