// Host side of the encoder-block entry points (fused norms, MXFP4): argument
// validation and launches.  Nothing is allocated here.
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <nvtx3/nvToolsExt.h>

#include <initializer_list>

#include "block_launch.h"
#include "launch.h"
#include "mpm.h"
#include "mxfp4.cuh"

namespace {

struct Range {
  explicit Range(const char* name) { nvtxRangePushA(name); }
  ~Range() { nvtxRangePop(); }
  Range(const Range&) = delete;
  Range& operator=(const Range&) = delete;
};

constexpr int64_t kMaxMatmulRows = int64_t{1} << 30;  // tile coordinates are 32-bit
constexpr size_t kStatusBytes = 2 * sizeof(int32_t);

int elem(mpm_dtype t) { return t == MPM_BF16 ? 2 : 4; }
bool valid_dtype(mpm_dtype t) { return t == MPM_F32 || t == MPM_BF16; }
bool aligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }
mpm_status status_of(cudaError_t e) { return e == cudaSuccess ? MPM_OK : MPM_ERR_CUDA; }

// A buffer in memory: what an output must not share with an input or another output.
struct Extent {
  uintptr_t begin, end;
};
Extent extent(const void* p, size_t bytes) {
  const uintptr_t b = reinterpret_cast<uintptr_t>(p);
  return {b, p == nullptr ? b : b + bytes};
}
Extent extent(const void* p, int64_t rows, int64_t dim, int64_t stride, int size) {
  return extent(p, rows > 0 ? static_cast<size_t>((rows - 1) * stride + dim) * size : 0);
}
bool overlap(const Extent& a, const Extent& b) { return a.begin < a.end && b.begin < b.end && a.begin < b.end && b.begin < a.end; }
// Whether an output overlaps an input or an earlier output.
bool any_overlap(std::initializer_list<Extent> outs, std::initializer_list<Extent> ins) {
  for (const Extent* o = outs.begin(); o != outs.end(); ++o) {
    for (const Extent& i : ins)
      if (overlap(*o, i)) return true;
    for (const Extent* p = outs.begin(); p != o; ++p)
      if (overlap(*o, *p)) return true;
  }
  return false;
}

bool stride_ok(int64_t stride, int64_t rows, int64_t dim) { return rows <= 1 || stride >= dim; }
bool vector_rows(const void* p, int64_t stride, int size) { return aligned(p, 16) && stride * size % 16 == 0; }

// The current device's SMs.  (The kernels are built for compute capability 10.3: elsewhere launches fail.)
mpm_status device_sms(int* sms) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return MPM_ERR_CUDA;
  if (cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || *sms <= 0) return MPM_ERR_CUDA;
  return MPM_OK;
}

// The arguments that forward and backward share.
struct NormShape {
  int64_t rows;
  int32_t batch, dim;
  mpm_dtype dtype, stream_dtype;
  const int64_t* offsets;
  mpm_norm_kind norm;
  float residual_scale;
  const float *post_weight, *post_bias, *gate, *pre_weight;
  int32_t gate_per_image;
};
size_t gate_bytes(const NormShape& s) {
  return sizeof(float) * static_cast<size_t>(s.dim) * (s.gate_per_image ? static_cast<size_t>(s.batch) : 1);
}
Extent gate_extent(const NormShape& s) { return extent(s.gate, gate_bytes(s)); }
Extent offsets_extent(const NormShape& s) { return extent(s.offsets, sizeof(int64_t) * (static_cast<size_t>(s.batch) + 1)); }

mpm_status check_norm(const NormShape& s, mpm::NormTypes* types) {
  if (!valid_dtype(s.dtype) || !valid_dtype(s.stream_dtype) || s.dim < 1 || s.batch < 1 || s.rows < 0 ||
      s.rows > INT32_MAX || (s.norm != MPM_NORM_RMS && s.norm != MPM_NORM_LAYER) || !isfinite(s.residual_scale))
    return MPM_ERR_INVALID_ARG;
  if (s.dim > MPM_MAX_DIM) return MPM_ERR_UNSUPPORTED;
  if (s.dtype == MPM_F32 && s.stream_dtype == MPM_BF16) return MPM_ERR_UNSUPPORTED;
  if (s.post_bias != nullptr && s.post_weight == nullptr) return MPM_ERR_INVALID_ARG;
  if (s.gate_per_image && (s.gate == nullptr || s.offsets == nullptr)) return MPM_ERR_INVALID_ARG;
  if (!aligned(s.offsets, 8)) return MPM_ERR_ALIGNMENT;
  for (const float* p : {s.post_weight, s.post_bias, s.gate, s.pre_weight})
    if (!aligned(p, 4)) return MPM_ERR_ALIGNMENT;
  *types = s.dtype == MPM_F32 ? mpm::NormTypes::kF32
           : s.stream_dtype == MPM_F32 ? mpm::NormTypes::kBf16StreamF32 : mpm::NormTypes::kBf16;
  return MPM_OK;
}

bool mx_dims_ok(int64_t rows, int32_t dim) {
  return rows >= 0 && rows <= INT32_MAX && dim >= 1 && dim <= MPM_MXFP4_MAX_DIM;
}
size_t mx_code_bytes(int64_t rows, int32_t dim) { return static_cast<size_t>(rows) * mpm::mx::code_pitch(dim); }
size_t mx_scale_bytes(int64_t rows, int32_t dim) {
  return static_cast<size_t>(mpm::mx::row_tiles(rows)) * mpm::mx::scale_tiles(dim) * mpm::mx::kTileBytes;
}

}  // namespace

extern "C" {

mpm_status mpm_block_norm(const void* y, int64_t y_stride, const void* residual, int64_t residual_stride,
                          const int64_t* offsets, int32_t batch, int64_t rows, int32_t dim, mpm_dtype dtype,
                          mpm_dtype stream_dtype, mpm_norm_kind norm, float eps, float residual_scale,
                          const float* post_weight, const float* post_bias, const float* gate,
                          int32_t gate_per_image, const float* pre_weight, const float* pre_bias, void* residual_out,
                          void* h, float* stats, int32_t* device_status, void* stream) {
  const Range range("mpm_block_norm");
  mpm::NormTypes types;
  const NormShape shape{rows, batch, dim, dtype, stream_dtype, offsets, norm, residual_scale,
                        post_weight, post_bias, gate, pre_weight, gate_per_image};
  const mpm_status st = check_norm(shape, &types);
  if (st != MPM_OK) return st;
  if (!(eps >= 0.f) || !isfinite(eps)) return MPM_ERR_INVALID_ARG;
  if ((pre_weight == nullptr) != (h == nullptr) && rows > 0) return MPM_ERR_INVALID_ARG;
  if (pre_bias != nullptr && pre_weight == nullptr) return MPM_ERR_INVALID_ARG;
  if (rows == 0) return MPM_OK;
  if (y == nullptr || residual == nullptr || residual_out == nullptr) return MPM_ERR_INVALID_ARG;
  if (!stride_ok(y_stride, rows, dim) || !stride_ok(residual_stride, rows, dim)) return MPM_ERR_INVALID_ARG;
  const int e = elem(dtype), es = elem(stream_dtype);
  if (!aligned(y, e) || !aligned(h, e) || !aligned(residual, es) || !aligned(residual_out, es) || !aligned(stats, 16) ||
      !aligned(pre_bias, 4) || !aligned(device_status, 4))
    return MPM_ERR_ALIGNMENT;
  const Extent in_y = extent(y, rows, dim, y_stride, e), in_x = extent(residual, rows, dim, residual_stride, es);
  const Extent out_x = extent(residual_out, rows, dim, dim, es), out_h = extent(h, rows, dim, dim, e);
  const Extent out_s = extent(stats, static_cast<size_t>(rows) * 16);
  // In place on the stream: each thread reads its own columns of a row before it writes them.
  const bool in_place = residual_out == residual && (residual_stride == dim || rows == 1);
  const Extent out_status = extent(device_status, kStatusBytes);
  const size_t vector = sizeof(float) * static_cast<size_t>(dim);
  if (any_overlap({out_x, out_h, out_s, out_status},
                  {in_y, extent(post_weight, vector), extent(post_bias, vector), gate_extent(shape),
                   extent(pre_weight, vector), extent(pre_bias, vector), offsets_extent(shape)}) ||
      any_overlap({out_h, out_s, out_status}, {in_x}) || (!in_place && overlap(out_x, in_x)))
    return MPM_ERR_ALIASING;
  const bool vec = dim % 8 == 0 && vector_rows(y, y_stride, e) && vector_rows(residual, residual_stride, es) &&
                   aligned(residual_out, 16) && aligned(h, 16) && aligned(post_weight, 16) && aligned(post_bias, 16) &&
                   aligned(gate, 16) && aligned(pre_weight, 16) && aligned(pre_bias, 16);
  int sms = 0;
  const mpm_status ds = device_sms(&sms);
  if (ds != MPM_OK) return ds;
  mpm::NormForward a{};
  a.y = y;
  a.residual = residual;
  a.y_stride = y_stride;
  a.residual_stride = residual_stride;
  a.offsets = offsets;
  a.rows = rows;
  a.batch = batch;
  a.dim = dim;
  a.post_weight = post_weight;
  a.post_bias = post_bias;
  a.gate = gate;
  a.gate_per_image = gate_per_image;
  a.pre_weight = pre_weight;
  a.pre_bias = pre_bias;
  a.alpha = residual_scale;
  a.eps = eps;
  a.layer = norm == MPM_NORM_LAYER;
  a.residual_out = residual_out;
  a.h = h;
  a.stats = reinterpret_cast<float4*>(stats);
  a.status = device_status;
  return status_of(mpm::launch_block_norm(a, types, vec, sms, static_cast<cudaStream_t>(stream)));
}

size_t mpm_block_norm_workspace_size(int32_t dim) {
  return dim < 1 || dim > MPM_MAX_DIM ? 0 : mpm::block_norm_workspace_floats(dim) * sizeof(float);
}

mpm_status mpm_block_norm_backward(const void* d_residual_out, int64_t d_residual_out_stride, const void* d_h,
                                   int64_t d_h_stride, const void* y, int64_t y_stride, const void* residual,
                                   int64_t residual_stride, const float* stats, const int64_t* offsets, int32_t batch,
                                   int64_t rows, int32_t dim, mpm_dtype dtype, mpm_dtype stream_dtype,
                                   mpm_norm_kind norm, float residual_scale, const float* post_weight,
                                   const float* post_bias, const float* gate, int32_t gate_per_image,
                                   const float* pre_weight, void* d_y, void* d_residual, float* d_post_weight,
                                   float* d_post_bias, float* d_gate, float* d_pre_weight, float* d_pre_bias,
                                   void* workspace, size_t workspace_bytes, int32_t* device_status, void* stream) {
  const Range range("mpm_block_norm_backward");
  mpm::NormTypes types;
  const NormShape shape{rows, batch, dim, dtype, stream_dtype, offsets, norm, residual_scale,
                        post_weight, post_bias, gate, pre_weight, gate_per_image};
  const mpm_status st = check_norm(shape, &types);
  if (st != MPM_OK) return st;
  if ((d_h != nullptr || d_pre_weight != nullptr || d_pre_bias != nullptr) && pre_weight == nullptr)
    return MPM_ERR_INVALID_ARG;
  if ((d_post_weight != nullptr || d_post_bias != nullptr) && post_weight == nullptr) return MPM_ERR_INVALID_ARG;
  if (d_gate != nullptr && gate == nullptr) return MPM_ERR_INVALID_ARG;
  if (rows > 0 && (y == nullptr || residual == nullptr || stats == nullptr || d_y == nullptr || d_residual == nullptr))
    return MPM_ERR_INVALID_ARG;
  if (!stride_ok(y_stride, rows, dim) || !stride_ok(residual_stride, rows, dim) ||
      (d_h != nullptr && !stride_ok(d_h_stride, rows, dim)) ||
      (d_residual_out != nullptr && !stride_ok(d_residual_out_stride, rows, dim)))
    return MPM_ERR_INVALID_ARG;
  const int e = elem(dtype), es = elem(stream_dtype);
  if (!aligned(y, e) || !aligned(d_h, e) || !aligned(d_y, e) || !aligned(residual, es) || !aligned(d_residual_out, es) ||
      !aligned(d_residual, es) || !aligned(stats, 16) || !aligned(device_status, 4))
    return MPM_ERR_ALIGNMENT;
  const float* const grads[] = {d_post_weight, d_post_bias, d_gate, d_pre_weight, d_pre_bias};
  bool grads16 = true;
  for (const float* g : grads) {
    if (!aligned(g, 4)) return MPM_ERR_ALIGNMENT;
    grads16 = grads16 && aligned(g, 16);
  }
  const size_t need = mpm_block_norm_workspace_size(dim);
  if (workspace == nullptr || !aligned(workspace, 256) || workspace_bytes < need) return MPM_ERR_WORKSPACE;
  const size_t vector = sizeof(float) * static_cast<size_t>(dim);
  if (any_overlap({extent(d_y, rows, dim, dim, e), extent(d_residual, rows, dim, dim, es), extent(d_post_weight, vector),
                   extent(d_post_bias, vector), extent(d_gate, gate_bytes(shape)), extent(d_pre_weight, vector),
                   extent(d_pre_bias, vector), extent(workspace, need), extent(device_status, kStatusBytes)},
                  {extent(y, rows, dim, y_stride, e), extent(residual, rows, dim, residual_stride, es),
                   extent(d_h, rows, dim, d_h_stride, e),
                   extent(d_residual_out, rows, dim, d_residual_out_stride, es),
                   extent(stats, static_cast<size_t>(rows) * 16), extent(post_weight, vector), extent(post_bias, vector),
                   gate_extent(shape), extent(pre_weight, vector), offsets_extent(shape)}))
    return MPM_ERR_ALIASING;
  const bool vec = dim % 8 == 0 && vector_rows(y, y_stride, e) && vector_rows(residual, residual_stride, es) &&
                   (d_h == nullptr || vector_rows(d_h, d_h_stride, e)) &&
                   (d_residual_out == nullptr || vector_rows(d_residual_out, d_residual_out_stride, es)) &&
                   aligned(d_y, 16) && aligned(d_residual, 16) && aligned(post_weight, 16) && aligned(post_bias, 16) &&
                   aligned(gate, 16) && aligned(pre_weight, 16) && grads16;
  int sms = 0;
  const mpm_status ds = device_sms(&sms);
  if (ds != MPM_OK) return ds;
  mpm::NormBackward a{};
  a.d_residual_out = d_residual_out;
  a.d_h = d_h;
  a.d_residual_out_stride = d_residual_out_stride;
  a.d_h_stride = d_h_stride;
  a.y = y;
  a.residual = residual;
  a.y_stride = y_stride;
  a.residual_stride = residual_stride;
  a.stats = reinterpret_cast<const float4*>(stats);
  a.offsets = offsets;
  a.rows = rows;
  a.batch = batch;
  a.dim = dim;
  a.post_weight = post_weight;
  a.post_bias = post_bias;
  a.gate = gate;
  a.gate_per_image = gate_per_image;
  a.pre_weight = pre_weight;
  a.alpha = residual_scale;
  a.layer = norm == MPM_NORM_LAYER;
  a.d_y = d_y;
  a.d_residual = d_residual;
  a.d_gate = d_gate;
  a.d_post_weight = d_post_weight;
  a.d_post_bias = d_post_bias;
  a.d_pre_weight = d_pre_weight;
  a.d_pre_bias = d_pre_bias;
  a.partial = static_cast<float*>(workspace);
  a.status = device_status;
  return status_of(mpm::launch_block_norm_backward(a, types, vec, sms, static_cast<cudaStream_t>(stream)));
}

size_t mpm_mxfp4_code_bytes(int64_t rows, int32_t dim) { return mx_dims_ok(rows, dim) ? mx_code_bytes(rows, dim) : 0; }

size_t mpm_mxfp4_scale_bytes(int64_t rows, int32_t dim) { return mx_dims_ok(rows, dim) ? mx_scale_bytes(rows, dim) : 0; }

mpm_status mpm_mxfp4_quantize(const void* tokens, int64_t stride, int64_t rows, int32_t dim, mpm_dtype dtype,
                              uint8_t* codes, uint8_t* scales, void* stream) {
  const Range range("mpm_mxfp4_quantize");
  if (!valid_dtype(dtype) || rows < 0 || rows > INT32_MAX || dim < 1) return MPM_ERR_INVALID_ARG;
  if (dim > MPM_MXFP4_MAX_DIM) return MPM_ERR_UNSUPPORTED;
  if (rows == 0) return MPM_OK;
  if (tokens == nullptr || codes == nullptr || scales == nullptr || !stride_ok(stride, rows, dim)) return MPM_ERR_INVALID_ARG;
  const int e = elem(dtype);
  if (!aligned(tokens, e) || !aligned(codes, 16) || !aligned(scales, 16)) return MPM_ERR_ALIGNMENT;
  if (any_overlap({extent(codes, mx_code_bytes(rows, dim)), extent(scales, mx_scale_bytes(rows, dim))},
                  {extent(tokens, rows, dim, stride, e)}))
    return MPM_ERR_ALIASING;
  int sms = 0;
  const mpm_status ds = device_sms(&sms);
  if (ds != MPM_OK) return ds;
  const mpm::QuantizeArgs a{tokens, stride, rows, dim, codes, scales};
  return status_of(mpm::launch_mxfp4_quantize(a, dtype == MPM_BF16, vector_rows(tokens, stride, e), sms,
                                              static_cast<cudaStream_t>(stream)));
}

mpm_status mpm_mxfp4_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t rows, int32_t dim, mpm_dtype dtype,
                                void* out, int64_t out_stride, void* stream) {
  const Range range("mpm_mxfp4_dequantize");
  if (!valid_dtype(dtype) || rows < 0 || rows > INT32_MAX || dim < 1) return MPM_ERR_INVALID_ARG;
  if (dim > MPM_MXFP4_MAX_DIM) return MPM_ERR_UNSUPPORTED;
  if (rows == 0) return MPM_OK;
  if (codes == nullptr || scales == nullptr || out == nullptr || !stride_ok(out_stride, rows, dim))
    return MPM_ERR_INVALID_ARG;
  const int e = elem(dtype);
  if (!aligned(out, e) || !aligned(codes, 16) || !aligned(scales, 16)) return MPM_ERR_ALIGNMENT;
  if (any_overlap({extent(out, rows, dim, out_stride, e)},
                  {extent(codes, mx_code_bytes(rows, dim)), extent(scales, mx_scale_bytes(rows, dim))}))
    return MPM_ERR_ALIASING;
  int sms = 0;
  const mpm_status ds = device_sms(&sms);
  if (ds != MPM_OK) return ds;
  const mpm::DequantizeArgs a{codes, scales, rows, dim, out, out_stride};
  return status_of(mpm::launch_mxfp4_dequantize(a, dtype == MPM_BF16, vector_rows(out, out_stride, e), sms,
                                                static_cast<cudaStream_t>(stream)));
}

mpm_status mpm_mxfp4_matmul(const uint8_t* a_codes, const uint8_t* a_scales, int64_t m, const uint8_t* b_codes,
                            const uint8_t* b_scales, int32_t n, int32_t k, const float* bias, mpm_dtype dtype, void* out,
                            int64_t out_stride, int32_t* device_status, void* stream) {
  const Range range("mpm_mxfp4_matmul");
  if (!valid_dtype(dtype) || m < 0 || n < 1 || k < 1) return MPM_ERR_INVALID_ARG;
  if (m > kMaxMatmulRows || n > kMaxMatmulRows || k > MPM_MXFP4_MAX_DIM ||
      mpm::mx::row_tiles(m > n ? m : n) * mpm::mx::scale_tiles(k) > kMaxMatmulRows)
    return MPM_ERR_UNSUPPORTED;
  if (m == 0) return MPM_OK;
  if (a_codes == nullptr || a_scales == nullptr || b_codes == nullptr || b_scales == nullptr || out == nullptr ||
      !stride_ok(out_stride, m, n))
    return MPM_ERR_INVALID_ARG;
  const int e = elem(dtype);
  for (const uint8_t* p : {a_codes, a_scales, b_codes, b_scales})
    if (!aligned(p, 16)) return MPM_ERR_ALIGNMENT;
  if (!aligned(out, e) || !aligned(bias, 4) || !aligned(device_status, 4)) return MPM_ERR_ALIGNMENT;
  if (any_overlap({extent(out, m, n, out_stride, e), extent(device_status, kStatusBytes)},
                  {extent(a_codes, mx_code_bytes(m, k)), extent(a_scales, mx_scale_bytes(m, k)),
                   extent(b_codes, mx_code_bytes(n, k)), extent(b_scales, mx_scale_bytes(n, k)),
                   extent(bias, sizeof(float) * static_cast<size_t>(n))}))
    return MPM_ERR_ALIASING;
  if (!mpm::tc_available()) return MPM_ERR_UNSUPPORTED;
  int sms = 0;
  const mpm_status ds = device_sms(&sms);
  if (ds != MPM_OK) return ds;
  const mpm::MxMatmulArgs a{a_codes, a_scales, m, b_codes, b_scales, n, k, bias, out, out_stride, device_status};
  return status_of(mpm::launch_mxfp4_matmul(a, dtype == MPM_BF16, sms, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
