#include "join_grad.cuh"

namespace fasgd {
cudaError_t launch_join_grad_bf16(const JoinArgs& a, int num_sms, cudaStream_t stream) {
    return launch<__nv_bfloat16>(a, num_sms, stream);
}
}  // namespace fasgd
