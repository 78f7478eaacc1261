// Gradients of block_norm for fp32 blocks, without a norm before the next block.
#include "block_norm_backward.cuh"

namespace mpm {

cudaError_t launch_block_norm_backward_f32_no_pre(const NormBackward& a, bool vec, int num_sms, cudaStream_t stream) {
  return launch_vec<float, float, false>(a, vec, num_sms, stream);
}

}  // namespace mpm
