// The MXFP4 layout (OCP Microscaling Formats 1.0): E2M1 elements in blocks of
// 32 along a row that share a power-of-two scale, 2^(c - 127).
//
// Codes: rows of code_pitch(dim) bytes, two elements a byte, the even one in
// the low half, zeros after the row's own; a multiple of 32 bytes, which is
// the 64 elements that one tensor-core product takes.
// Scales: tiles of 128 rows x 4 blocks, 512 bytes each, the tiles of a row
// tile next to one another.  Within a tile row r, block j is byte
// 16 (r % 32) + 4 (r / 32) + j: four 8 x 16-byte matrices, the form in which
// tcgen05.cp spreads scales over tensor memory without any shuffling.
#pragma once

#include <stdint.h>

namespace mpm {
namespace mx {

constexpr int kBlock = 32;
constexpr int kTileRows = 128;
constexpr int kTileBlocks = 4;
constexpr int kTileBytes = 512;
constexpr int kNanScale = 255;

__host__ __device__ constexpr int code_pitch(int dim) { return (dim + 63) / 64 * 32; }
__host__ __device__ constexpr int scale_tiles(int dim) { return (dim + kBlock * kTileBlocks - 1) / (kBlock * kTileBlocks); }
__host__ __device__ constexpr int64_t row_tiles(int64_t rows) { return (rows + kTileRows - 1) / kTileRows; }

}  // namespace mx

struct QuantizeArgs {
  const void* x;      // rows of dim values, `stride` elements apart
  int64_t stride, rows;
  int dim;
  uint8_t* codes;     // [rows, code_pitch(dim)]
  uint8_t* scales;    // [row_tiles(rows), scale_tiles(dim), 512]
};
struct DequantizeArgs {
  const uint8_t* codes;
  const uint8_t* scales;
  int64_t rows;
  int dim;
  void* out;          // rows of dim values, `stride` elements apart
  int64_t stride;
};
struct MxMatmulArgs {
  const uint8_t* a_codes;
  const uint8_t* a_scales;
  int64_t m;
  const uint8_t* b_codes;
  const uint8_t* b_scales;
  int n, k;
  const float* bias;  // [n] or null
  void* out;          // rows of n values, `stride` elements apart
  int64_t stride;
  int32_t* status;
};

cudaError_t launch_mxfp4_quantize(const QuantizeArgs& a, bool bf16, bool vec, int num_sms, cudaStream_t stream);
cudaError_t launch_mxfp4_dequantize(const DequantizeArgs& a, bool bf16, bool vec, int num_sms, cudaStream_t stream);
cudaError_t launch_mxfp4_matmul(const MxMatmulArgs& a, bool bf16, int num_sms, cudaStream_t stream);

}  // namespace mpm
