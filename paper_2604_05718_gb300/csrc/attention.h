// Internal arguments and launchers of attention between packed sequences and of
// rotary positions (not part of the public ABI).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

namespace mpm {

constexpr int kAttentionMaxDim = 128;
// Most parts that a row's keys (or a key's queries) are split into.
constexpr int kAttentionMaxSplits = 64;

// [rows, heads, dim] values: row r, head h begins row * r + head * h elements on.
struct Heads {
  const void* p;
  int64_t row, head;
};

struct AttentionArgs {
  Heads q, k, v;
  const int64_t* q_offsets;  // int64[batch + 1], or null: one sequence of all rows
  const int64_t* k_offsets;
  int64_t q_rows, k_rows;
  int32_t batch, q_heads, kv_heads, dim;
  float scale;
  const uint8_t* mask;       // [k_rows], 0: key left out; or null
  void* out;                 // [q_rows, q_heads, dim]
  void* rest;                // bf16 [q_rows, q_heads, dim], what the rounding of out left; or null
  float* lse;                // [q_rows, q_heads], or null (forward)
  // Backward.
  Heads d_out;
  const float* stats;        // the forward pass's lse
  float* delta;              // workspace: sum over a head's features of d_out * out
  void* d_q;                 // [q_rows, q_heads, dim]
  void* d_k;                 // [k_rows, kv_heads, dim]
  void* d_v;
  // Parts, where the streamed side is split: fp32 [splits, rows * heads, dim] and,
  // forward, log2 of the parts' sums [splits, rows * heads].
  float* partial;
  float* partial_lse;
  int32_t splits;            // of the keys (forward, d_q)
  int32_t key_splits;        // of the queries (d_k, d_v)
  int32_t* status;
  bool vec;                  // four elements of any row can be loaded at once
};

cudaError_t launch_attention_f32(const AttentionArgs& a, bool bf16, cudaStream_t stream);
cudaError_t launch_attention_backward_f32(const AttentionArgs& a, bool bf16, int num_sms, cudaStream_t stream);
// bf16 whose rows and heads are 16-byte aligned, on the tensor cores.
cudaError_t launch_attention_tc(const AttentionArgs& a, cudaStream_t stream);
// bf16, 16-byte aligned, head_dim a multiple of 8: blocks of `queries` queries, `cluster` blocks a sequence.
cudaError_t launch_attention_few(const AttentionArgs& a, int queries, int cluster, cudaStream_t stream);
cudaError_t launch_attention_backward_tc(const AttentionArgs& a, int num_sms, cudaStream_t stream);
// out (and lse) from the parts.
cudaError_t launch_attention_join(const AttentionArgs& a, bool bf16, int num_sms, cudaStream_t stream);
// delta from out and d_out.
cudaError_t launch_attention_delta(const AttentionArgs& a, bool bf16, int num_sms, cudaStream_t stream);
// What parts are parts of: sequences in tiles of `tile` rows, `times` over.
struct Streamed {
  const int64_t* offsets;
  int64_t rows;
  int tile, times;
};
// Sums of the parts that a row's sequence has, rounded once to out.
cudaError_t launch_attention_sum(const float* parts, int splits, int64_t rows, const int64_t* offsets, int batch, int heads,
                                 int dim, const Streamed& streamed, void* out, bool bf16, int num_sms, cudaStream_t stream);

struct RotaryArgs {
  Heads x;
  void* out;
  int64_t out_row, out_head;
  const float* positions;      // [rows, axes]
  const double* frequencies;   // [pairs], radians per unit of position
  const int64_t* offsets;      // rows from offsets[batch] on are left alone; or null
  int64_t rows;
  int32_t batch, heads, dim, pairs, axes;
  int32_t first_pair[8];       // first pair of each axis
  bool halves, inverse, vec;
  int32_t* status;
};
constexpr int kRotaryMaxAxes = 8;
constexpr int kRotaryMaxDim = 1024;
cudaError_t launch_rotary(const RotaryArgs& a, bool bf16, int num_sms, cudaStream_t stream);

}  // namespace mpm
