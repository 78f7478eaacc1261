// Gradients of block_norm for bf16 blocks on an fp32 residual stream.
#include "block_norm_backward.cuh"

namespace mpm {

cudaError_t launch_block_norm_backward_mixed(const NormBackward& a, bool vec, int num_sms, cudaStream_t stream) {
  return launch_vec<__nv_bfloat16, float, true>(a, vec, num_sms, stream);
}

}  // namespace mpm
