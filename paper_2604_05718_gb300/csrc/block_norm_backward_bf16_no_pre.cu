// Gradients of block_norm for bf16 blocks, without a norm before the next block.
#include "block_norm_backward.cuh"

namespace mpm {

cudaError_t launch_block_norm_backward_bf16_no_pre(const NormBackward& a, bool vec, int num_sms, cudaStream_t stream) {
  return launch_vec<__nv_bfloat16, __nv_bfloat16, false>(a, vec, num_sms, stream);
}

}  // namespace mpm
