// Gradients of block_norm for bf16 blocks on an fp32 residual stream, without a norm before the next block.
#include "block_norm_backward.cuh"

namespace mpm {

cudaError_t launch_block_norm_backward_mixed_no_pre(const NormBackward& a, bool vec, int num_sms, cudaStream_t stream) {
  return launch_vec<__nv_bfloat16, float, false>(a, vec, num_sms, stream);
}

}  // namespace mpm
