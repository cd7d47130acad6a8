#include "join_grad.cuh"

namespace fasgd {
cudaError_t launch_join_grad_f32(const JoinArgs& a, int num_sms, cudaStream_t stream) {
    return launch<float>(a, num_sms, stream);
}
}  // namespace fasgd
