// Internal launchers of the encoder-block operators (not part of the public ABI).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

namespace mpm {

// Token types of one block_norm call: the branch (y, h and their gradients)
// and the residual stream.
enum class NormTypes : int { kF32 = 0, kBf16 = 1, kBf16StreamF32 = 2 };

struct NormForward {
  const void* y;            // [rows] rows of dim, y_stride elements apart
  const void* residual;     // [rows] rows of dim, residual_stride elements apart
  int64_t y_stride, residual_stride;
  const int64_t* offsets;   // int64[batch + 1], or null: one image of `rows` rows
  int64_t rows;
  int32_t batch, dim;
  const float* post_weight; // null: no norm after the block
  const float* post_bias;
  const float* gate;        // null, [dim], or [batch, dim] (gate_rows == batch)
  int32_t gate_per_image;
  const float* pre_weight;  // null: no norm before the next block (h is not written)
  const float* pre_bias;
  float alpha, eps;
  int32_t layer;            // 1: layer norm, 0: root mean square
  void* residual_out;       // [rows, dim]
  void* h;                  // [rows, dim]
  float4* stats;            // (mean, 1 / deviation) of both norms, or null
  int32_t* status;
};

struct NormBackward {
  const void* d_residual_out;  // null: zero
  const void* d_h;             // null: zero
  int64_t d_residual_out_stride, d_h_stride;
  const void* y;
  const void* residual;
  int64_t y_stride, residual_stride;
  const float4* stats;
  const int64_t* offsets;
  int64_t rows;
  int32_t batch, dim;
  const float* post_weight;
  const float* post_bias;
  const float* gate;
  int32_t gate_per_image;
  const float* pre_weight;
  float alpha;
  int32_t layer;
  void* d_y;
  void* d_residual;
  // Gradients of the parameters, each null when it is not wanted.
  float* d_gate;
  float* d_post_weight;
  float* d_post_bias;
  float* d_pre_weight;
  float* d_pre_bias;
  float* partial;  // workspace of block_norm_workspace_floats(...)
  int32_t* status;
};

// Columns that one warp takes at a time: eight a lane.
constexpr int kNormWarpCols = 256;

cudaError_t launch_block_norm(const NormForward& a, NormTypes types, bool vec, int num_sms, cudaStream_t stream);
cudaError_t launch_block_norm_backward(const NormBackward& a, NormTypes types, bool vec, int num_sms,
                                       cudaStream_t stream);
// Its parts, a file each.
cudaError_t launch_block_norm_backward_f32(const NormBackward& a, bool vec, int num_sms, cudaStream_t stream);
cudaError_t launch_block_norm_backward_bf16(const NormBackward& a, bool vec, int num_sms, cudaStream_t stream);
cudaError_t launch_block_norm_backward_mixed(const NormBackward& a, bool vec, int num_sms, cudaStream_t stream);
// And without pre_weight.
cudaError_t launch_block_norm_backward_f32_no_pre(const NormBackward& a, bool vec, int num_sms, cudaStream_t stream);
cudaError_t launch_block_norm_backward_bf16_no_pre(const NormBackward& a, bool vec, int num_sms, cudaStream_t stream);
cudaError_t launch_block_norm_backward_mixed_no_pre(const NormBackward& a, bool vec, int num_sms, cudaStream_t stream);
// Floats of workspace that the backward pass's partial sums take.
size_t block_norm_workspace_floats(int dim);

}  // namespace mpm
