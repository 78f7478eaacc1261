// Gradients of block_norm for bf16 blocks.
#include "block_norm_backward.cuh"

namespace mpm {

cudaError_t launch_block_norm_backward_bf16(const NormBackward& a, bool vec, int num_sms, cudaStream_t stream) {
  return launch_vec<__nv_bfloat16, __nv_bfloat16, true>(a, vec, num_sms, stream);
}

size_t block_norm_workspace_floats(int dim) {
  return static_cast<size_t>(dim) * kMaxBlocks * (kSums + 4 * static_cast<size_t>(max_groups(dim)));
}

cudaError_t launch_block_norm_backward(const NormBackward& a, NormTypes types, bool vec, int num_sms,
                                       cudaStream_t stream) {
  const bool pre = a.pre_weight != nullptr;
  switch (types) {
    case NormTypes::kF32:
      return pre ? launch_block_norm_backward_f32(a, vec, num_sms, stream)
                 : launch_block_norm_backward_f32_no_pre(a, vec, num_sms, stream);
    case NormTypes::kBf16:
      return pre ? launch_block_norm_backward_bf16(a, vec, num_sms, stream)
                 : launch_block_norm_backward_bf16_no_pre(a, vec, num_sms, stream);
    case NormTypes::kBf16StreamF32:
      return pre ? launch_block_norm_backward_mixed(a, vec, num_sms, stream)
                 : launch_block_norm_backward_mixed_no_pre(a, vec, num_sms, stream);
  }
  return cudaErrorInvalidValue;
}

}  // namespace mpm
