// Host side of attention between packed sequences and of rotary positions:
// argument validation, the choice of kernels and the split of long sequences.
// Nothing is allocated here.
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <nvtx3/nvToolsExt.h>

#include <algorithm>
#include <initializer_list>

#include "attention.h"
#include "mpm.h"

namespace {

struct Range {
  explicit Range(const char* name) { nvtxRangePushA(name); }
  ~Range() { nvtxRangePop(); }
  Range(const Range&) = delete;
  Range& operator=(const Range&) = delete;
};

using mpm::Heads;

constexpr size_t kStatusBytes = 2 * sizeof(int32_t);
constexpr int64_t kSms = 152;  // of a GB300: the workspace's size is a function of the shape alone

int elem(mpm_dtype t) { return t == MPM_BF16 ? 2 : 4; }
bool valid_dtype(mpm_dtype t) { return t == MPM_F32 || t == MPM_BF16; }
bool aligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }
mpm_status status_of(cudaError_t e) { return e == cudaSuccess ? MPM_OK : MPM_ERR_CUDA; }

mpm_status device_sms(int* sms) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return MPM_ERR_CUDA;
  if (cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || *sms <= 0) return MPM_ERR_CUDA;
  return MPM_OK;
}

// A buffer in memory, from its first to behind its last byte.
struct Extent {
  uintptr_t begin, end;
};
Extent extent(const void* p, size_t bytes) {
  const uintptr_t b = reinterpret_cast<uintptr_t>(p);
  return {b, p == nullptr ? b : b + bytes};
}
Extent extent(const Heads& x, int64_t rows, int64_t heads, int64_t dim, int size) {
  return extent(x.p, rows == 0 ? 0 : static_cast<size_t>((rows - 1) * x.row + (heads - 1) * x.head + dim) * size);
}
bool overlap(const Extent& a, const Extent& b) { return a.begin < a.end && b.begin < b.end && a.begin < b.end && b.begin < a.end; }
bool any_overlap(std::initializer_list<Extent> outs, std::initializer_list<Extent> ins) {
  for (const Extent* o = outs.begin(); o != outs.end(); ++o) {
    for (const Extent& i : ins)
      if (overlap(*o, i)) return true;
    for (const Extent* p = outs.begin(); p != o; ++p)
      if (overlap(*o, *p)) return true;
  }
  return false;
}

// Strides of [rows, heads, dim] whose rows and heads do not overlap; strides that
// nothing goes by are set to ones that suit every kernel.
bool strides_ok(Heads* x, int64_t rows, int64_t heads, int64_t dim) {
  if (heads <= 1) x->head = (dim + 7) / 8 * 8;
  if (rows <= 1) x->row = heads * x->head;
  if (x->row < dim || x->head < dim) return false;
  return x->row >= (heads - 1) * x->head + dim || x->head >= (rows - 1) * x->row + dim;
}
// `count` elements of any row can be loaded at once.
bool vector_heads(const Heads& x, int size, int count) {
  return aligned(x.p, size * count) && x.row % count == 0 && x.head % count == 0;
}

struct Shape {
  int32_t batch;
  int64_t q_rows, k_rows;
  int32_t q_heads, kv_heads, dim;
  mpm_dtype dtype;
};
mpm_status check_shape(const Shape& s) {
  if (!valid_dtype(s.dtype) || s.batch < 1 || s.q_rows < 0 || s.k_rows < 0 || s.q_rows > INT32_MAX || s.k_rows > INT32_MAX ||
      s.q_heads < 1 || s.kv_heads < 1 || s.q_heads % s.kv_heads != 0 || s.dim < 1)
    return MPM_ERR_INVALID_ARG;
  if (s.dim > MPM_ATTENTION_MAX_HEAD_DIM || s.q_heads > MPM_ATTENTION_MAX_HEADS) return MPM_ERR_UNSUPPORTED;
  return MPM_OK;
}

// How many parts the fp32 kernels' streamed side of length `stream` (all sequences)
// is split into, where `rows` rows of the other side, in tiles of `tile`, times `heads`
// are the work: as many as fill `ways` blocks an SM, a tile of 64 each in a sequence of
// four times the mean length, which is all that is known.  A shorter sequence's last
// parts are not there and cost next to nothing (4 sequences of 1 to 785 keys, 6 heads:
// forward and gradients 70 us, with as many parts as the mean has tiles 114).
int splits_for(int64_t rows, int64_t tile, int64_t heads, int64_t stream, int64_t batch, int64_t ways) {
  const int64_t items = std::max((rows + tile - 1) / tile, std::min(batch, rows)) * heads;
  if (items == 0) return 1;
  const int64_t mean = (stream / std::max<int64_t>(1, std::min(batch, stream)) + 63) / 64;
  const int64_t most = mean <= 1 ? mean : std::min((stream + 63) / 64, 4 * mean);
  return static_cast<int>(std::max<int64_t>(1, std::min({kSms * ways / items, most, int64_t{mpm::kAttentionMaxSplits}})));
}
struct Plan {
  int splits, key_splits;
};
// The fp32 kernels' tiles: streamed ones of 64 rows, their own of 64 too, but for gradients of wide heads.
Plan plan_f32(const Shape& s) { return {splits_for(s.q_rows, 64, s.q_heads, s.k_rows, s.batch, 4), 1}; }
Plan plan_f32_backward(const Shape& s) {
  const int64_t group = s.q_heads / s.kv_heads, tile = s.dim <= 64 ? 64 : 128, ways = s.dim <= 64 ? 4 : 2;
  return {splits_for(s.q_rows, tile, s.q_heads, s.k_rows, s.batch, ways),
          splits_for(s.k_rows, tile, s.kv_heads, s.q_rows * group, s.batch, ways)};
}

// Parts of the tensor-core kernels' streamed side: the rounds of items over the SMs
// times an item's length, and what writing and joining the parts costs, `launches` of
// 4 us and every part's fp32 rows there and back at 4 TB/s.  A part has eight tiles
// or more.  us of a tile: what the kernels take at head widths of 64 to 128.  (Against
// as many parts as fill two blocks an SM: 4096 tokens, 8 heads of 128 forward whole 56
// us, in two 72; 2 x 5000 and 1999 tokens, 8 heads of 128 on 2, gradients with keys in
// three parts 782 us, whole 901; 24 x 100 queries, 1024 to 4096 keys, 8 heads of 32
// whole 29 us, in two 38.)
int parts_for(int64_t rows, int64_t tile, int64_t heads, int64_t stream, int64_t batch, double tile_us, int launches,
              int64_t values) {
  const int64_t items = std::max((rows + tile - 1) / tile, std::min(batch, rows)) * heads;
  const int64_t tiles = (stream / std::max<int64_t>(1, std::min(batch, stream)) + 127) / 128;
  int best = 1;
  double least = 0;
  for (int parts = 1; parts == 1 || (parts <= mpm::kAttentionMaxSplits && parts * 8 <= tiles); ++parts) {
    const int64_t rounds = (items * parts + kSms - 1) / kSms;
    double us = static_cast<double>(rounds) * (static_cast<double>((tiles + parts - 1) / parts) * tile_us + 2);
    if (parts > 1) us += 4 * launches + 2e-6 * static_cast<double>(values) * parts;
    if (parts > 1 && us >= least) continue;
    least = us;
    best = parts;
  }
  return best;
}
Plan plan_tc(const Shape& s) {
  // Of a lone tile of queries the even and the odd tiles of keys run side by side.
  const double tile_us = s.q_rows <= int64_t{128} * s.batch ? 0.7 : 1.4;
  return {parts_for(s.q_rows, 256, s.q_heads, s.k_rows, s.batch, tile_us, 1, s.q_rows * s.q_heads * s.dim), 1};
}
Plan plan_tc_backward(const Shape& s) {
  const int64_t group = s.q_heads / s.kv_heads;
  return {parts_for(s.q_rows, 128, s.q_heads, s.k_rows, s.batch, 1.6, 1, s.q_rows * s.q_heads * s.dim),
          parts_for(s.k_rows, 128, s.kv_heads, s.q_rows * group, s.batch, 1.6, 2, 2 * s.k_rows * s.kv_heads * s.dim)};
}
// Few queries: blocks of 16 rows, of the heads that share a kv head.  Taken where
// the sequences' queries are so few on the mean (a longer sequence takes several
// blocks, which read its keys again).
struct FewPlan {
  int queries, cluster, splits;  // queries 0: not taken
};
FewPlan plan_few(const Shape& s) {
  const int64_t group = s.q_heads / s.kv_heads, sequences = std::min<int64_t>(s.batch, s.q_rows);
  if (s.dtype != MPM_BF16 || s.dim % 8 != 0 || group > 16 || s.q_rows * group > 16 * sequences) return {0, 1, 1};
  const int queries = static_cast<int>(16 / group);
  const int64_t items = std::max((s.q_rows + queries - 1) / queries, sequences) * s.kv_heads;
  const int64_t passes = (s.k_rows / std::max<int64_t>(1, std::min<int64_t>(s.batch, s.k_rows)) + 63) / 64;
  // Of the blocks, of which an SM holds three (head_dim <= 64) or two, the rounds times
  // their length in passes, where starting and joining takes about five: 192 items of 256
  // passes alone leave the second round of SMs a third full (347 us; by threes 303, by
  // fours 292), 768 items of 14 passes are best left whole (43 us; in twos 55, in eights
  // 130).  Clusters of five and seven do not fill the GPCs (128 items: by sevens 227, by
  // fours 202, by twos 208).
  const int64_t resident = kSms * (s.dim <= 64 ? 3 : 2);
  int cluster = 1;
  int64_t least = INT64_MAX;
  for (const int c : {1, 2, 3, 4, 6, 8}) {
    const int64_t cost = (items * c + resident - 1) / resident * ((passes + c - 1) / c + 5);
    if (c > std::max<int64_t>(1, passes) || cost >= least) continue;
    least = cost;
    cluster = c;
  }
  int64_t splits = 1;
  if (cluster == 8 && items * 8 < kSms) splits = std::max<int64_t>(1, std::min({2 * kSms / (items * 8), passes / 16, int64_t{mpm::kAttentionMaxSplits}}));
  if ((s.q_rows / queries + s.batch) * s.kv_heads * splits * cluster > INT32_MAX) return {0, 1, 1};
  return {queries, cluster, static_cast<int>(splits)};
}
// Whether the tensor-core kernels can load a tensor: TMA's addresses and strides are multiples of 16 bytes.
bool tc_heads(const Heads& x) { return vector_heads(x, 2, 8); }

size_t round256(size_t n) { return (n + 255) / 256 * 256; }
size_t part_bytes(int splits, int64_t rows, int heads, int dim) {
  return splits <= 1 ? 0 : round256(sizeof(float) * static_cast<size_t>(splits) * rows * heads * dim);
}
size_t part_lse_bytes(int splits, int64_t rows, int heads) { return part_bytes(splits, rows, heads, 1); }
size_t delta_bytes(const Shape& s) { return round256(sizeof(float) * static_cast<size_t>(s.q_rows) * s.q_heads); }

size_t forward_bytes(const Shape& s, const Plan& p) {
  return part_bytes(p.splits, s.q_rows, s.q_heads, s.dim) + part_lse_bytes(p.splits, s.q_rows, s.q_heads);
}
size_t backward_bytes(const Shape& s, const Plan& p) {
  return delta_bytes(s) + std::max(part_bytes(p.splits, s.q_rows, s.q_heads, s.dim),
                                   part_bytes(p.key_splits, s.k_rows, s.kv_heads, 2 * s.dim));
}

// What a caller provides: enough for either kind of kernels, since the shape alone does not tell which runs.
size_t forward_need(const Shape& s) {
  const FewPlan few = plan_few(s);
  return std::max({forward_bytes(s, plan_f32(s)), forward_bytes(s, plan_tc(s)), forward_bytes(s, {few.splits, 1})});
}
size_t backward_need(const Shape& s) { return std::max(backward_bytes(s, plan_f32_backward(s)), backward_bytes(s, plan_tc_backward(s))); }

mpm::AttentionArgs common_args(const Shape& s, const Heads& q, const Heads& k, const Heads& v, const int64_t* q_offsets,
                               const int64_t* k_offsets, float scale, const uint8_t* mask, int32_t* status) {
  mpm::AttentionArgs a{};
  a.q = q;
  a.k = k;
  a.v = v;
  a.q_offsets = q_offsets;
  a.k_offsets = k_offsets;
  a.q_rows = s.q_rows;
  a.k_rows = s.k_rows;
  a.batch = s.batch;
  a.q_heads = s.q_heads;
  a.kv_heads = s.kv_heads;
  a.dim = s.dim;
  a.scale = scale;
  a.mask = mask;
  a.splits = a.key_splits = 1;
  a.status = status;
  return a;
}

// What both directions ask of their inputs.
mpm_status check_inputs(const Shape& s, std::initializer_list<Heads*> of_q, std::initializer_list<Heads*> of_k,
                        const int64_t* q_offsets, const int64_t* k_offsets, float scale, const int32_t* status) {
  if (!(scale > 0.f) || !isfinite(scale)) return MPM_ERR_INVALID_ARG;
  if ((q_offsets == nullptr) != (k_offsets == nullptr) || (q_offsets == nullptr && s.batch != 1)) return MPM_ERR_INVALID_ARG;
  const int e = elem(s.dtype);
  for (Heads* x : of_q)
    if ((x->p == nullptr && s.q_rows > 0) || !strides_ok(x, s.q_rows, s.q_heads, s.dim)) return MPM_ERR_INVALID_ARG;
  for (Heads* x : of_k)
    if ((x->p == nullptr && s.k_rows > 0) || !strides_ok(x, s.k_rows, s.kv_heads, s.dim)) return MPM_ERR_INVALID_ARG;
  for (auto list : {of_q, of_k})
    for (Heads* x : list)
      if (!aligned(x->p, e)) return MPM_ERR_ALIGNMENT;
  if (!aligned(q_offsets, 8) || !aligned(k_offsets, 8) || !aligned(status, 4)) return MPM_ERR_ALIGNMENT;
  return MPM_OK;
}
Extent offsets_extent(const int64_t* p, int32_t batch) { return extent(p, sizeof(int64_t) * (static_cast<size_t>(batch) + 1)); }

}  // namespace

extern "C" {

size_t mpm_cross_attention_workspace_size(int32_t batch, int64_t q_rows, int64_t k_rows, int32_t q_heads, int32_t kv_heads,
                                          int32_t head_dim, mpm_dtype dtype) {
  const Shape s{batch, q_rows, k_rows, q_heads, kv_heads, head_dim, dtype};
  return check_shape(s) != MPM_OK ? 0 : forward_need(s);
}

size_t mpm_cross_attention_backward_workspace_size(int32_t batch, int64_t q_rows, int64_t k_rows, int32_t q_heads,
                                                   int32_t kv_heads, int32_t head_dim, mpm_dtype dtype) {
  const Shape s{batch, q_rows, k_rows, q_heads, kv_heads, head_dim, dtype};
  return check_shape(s) != MPM_OK ? 0 : backward_need(s);
}

mpm_status mpm_cross_attention(const void* q, int64_t q_row_stride, int64_t q_head_stride, const void* k,
                               int64_t k_row_stride, int64_t k_head_stride, const void* v, int64_t v_row_stride,
                               int64_t v_head_stride, const int64_t* q_offsets, const int64_t* k_offsets, int32_t batch,
                               int64_t q_rows, int64_t k_rows, int32_t q_heads, int32_t kv_heads, int32_t head_dim,
                               mpm_dtype dtype, float scale, const uint8_t* key_mask, void* out,
                               void* out_rest, float* lse, void* workspace, size_t workspace_bytes,
                               int32_t* device_status, void* stream) {
  const Range range("mpm_cross_attention");
  const Shape s{batch, q_rows, k_rows, q_heads, kv_heads, head_dim, dtype};
  mpm_status st = check_shape(s);
  if (st != MPM_OK) return st;
  Heads hq{q, q_row_stride, q_head_stride}, hk{k, k_row_stride, k_head_stride}, hv{v, v_row_stride, v_head_stride};
  st = check_inputs(s, {&hq}, {&hk, &hv}, q_offsets, k_offsets, scale, device_status);
  if (st != MPM_OK) return st;
  if (q_rows == 0) return MPM_OK;
  if (out == nullptr) return MPM_ERR_INVALID_ARG;
  const int e = elem(dtype);
  if (dtype == MPM_F32 && out_rest != nullptr) return MPM_ERR_UNSUPPORTED;
  if (!aligned(out, e) || !aligned(out_rest, e) || !aligned(lse, 4)) return MPM_ERR_ALIGNMENT;
  const bool tc = dtype == MPM_BF16 && tc_heads(hq) && tc_heads(hk) && tc_heads(hv);
  const FewPlan few = tc ? plan_few(s) : FewPlan{0, 1, 1};
  const Plan plan = few.queries > 0 ? Plan{few.splits, 1} : tc ? plan_tc(s) : plan_f32(s);
  const size_t need = forward_need(s);
  if (need > 0 && (workspace == nullptr || !aligned(workspace, 256) || workspace_bytes < need)) return MPM_ERR_WORKSPACE;
  const size_t q_values = static_cast<size_t>(q_rows) * q_heads;
  if (any_overlap({extent(out, q_values * head_dim * e), extent(out_rest, q_values * head_dim * e), extent(lse, q_values * 4),
                   extent(workspace, need),
                   extent(device_status, kStatusBytes)},
                  {extent(hq, q_rows, q_heads, head_dim, e), extent(hk, k_rows, kv_heads, head_dim, e),
                   extent(hv, k_rows, kv_heads, head_dim, e), offsets_extent(q_offsets, batch),
                   offsets_extent(k_offsets, batch), extent(key_mask, static_cast<size_t>(k_rows))}))
    return MPM_ERR_ALIASING;
  int sms = 0;
  st = device_sms(&sms);
  if (st != MPM_OK) return st;
  mpm::AttentionArgs a = common_args(s, hq, hk, hv, q_offsets, k_offsets, scale, key_mask, device_status);
  a.out = out;
  a.rest = out_rest;
  a.lse = lse;
  a.splits = plan.splits;
  a.partial = static_cast<float*>(workspace);
  a.partial_lse = a.partial + part_bytes(plan.splits, q_rows, q_heads, head_dim) / sizeof(float);
  a.vec = head_dim % 4 == 0 && vector_heads(hq, e, 4) && vector_heads(hk, e, 4) && vector_heads(hv, e, 4);
  const cudaStream_t on = static_cast<cudaStream_t>(stream);
  cudaError_t err = few.queries > 0 ? mpm::launch_attention_few(a, few.queries, few.cluster, on)
                    : tc            ? mpm::launch_attention_tc(a, on)
                                    : mpm::launch_attention_f32(a, dtype == MPM_BF16, on);
  if (err == cudaSuccess && a.splits > 1) err = mpm::launch_attention_join(a, dtype == MPM_BF16, sms, on);
  return status_of(err);
}

mpm_status mpm_cross_attention_backward(const void* d_out, int64_t d_out_row_stride, int64_t d_out_head_stride,
                                        const void* q, int64_t q_row_stride, int64_t q_head_stride, const void* k,
                                        int64_t k_row_stride, int64_t k_head_stride, const void* v, int64_t v_row_stride,
                                        int64_t v_head_stride, const void* out, const void* out_rest,
                                        const float* lse, const int64_t* q_offsets,
                                        const int64_t* k_offsets, int32_t batch, int64_t q_rows, int64_t k_rows,
                                        int32_t q_heads, int32_t kv_heads, int32_t head_dim, mpm_dtype dtype, float scale,
                                        const uint8_t* key_mask, void* d_q, void* d_k, void* d_v, void* workspace,
                                        size_t workspace_bytes, int32_t* device_status, void* stream) {
  const Range range("mpm_cross_attention_backward");
  const Shape s{batch, q_rows, k_rows, q_heads, kv_heads, head_dim, dtype};
  mpm_status st = check_shape(s);
  if (st != MPM_OK) return st;
  Heads hg{d_out, d_out_row_stride, d_out_head_stride};
  Heads hq{q, q_row_stride, q_head_stride}, hk{k, k_row_stride, k_head_stride}, hv{v, v_row_stride, v_head_stride};
  st = check_inputs(s, {&hq, &hg}, {&hk, &hv}, q_offsets, k_offsets, scale, device_status);
  if (st != MPM_OK) return st;
  if (q_rows == 0 && k_rows == 0) return MPM_OK;
  if ((q_rows > 0 && (out == nullptr || lse == nullptr || d_q == nullptr)) ||
      (k_rows > 0 && (d_k == nullptr || d_v == nullptr)))
    return MPM_ERR_INVALID_ARG;
  const int e = elem(dtype);
  if (dtype == MPM_F32 && out_rest != nullptr) return MPM_ERR_UNSUPPORTED;
  for (const void* p : {out, out_rest, static_cast<const void*>(d_q), static_cast<const void*>(d_k), static_cast<const void*>(d_v)})
    if (!aligned(p, e)) return MPM_ERR_ALIGNMENT;
  if (!aligned(lse, 4)) return MPM_ERR_ALIGNMENT;
  const bool tc = dtype == MPM_BF16 && tc_heads(hq) && tc_heads(hk) && tc_heads(hv) && tc_heads(hg);
  const Plan plan = tc ? plan_tc_backward(s) : plan_f32_backward(s);
  const size_t need = backward_need(s);
  if (need > 0 && (workspace == nullptr || !aligned(workspace, 256) || workspace_bytes < need)) return MPM_ERR_WORKSPACE;
  const size_t q_values = static_cast<size_t>(q_rows) * q_heads, k_bytes = static_cast<size_t>(k_rows) * kv_heads * head_dim * e;
  if (any_overlap({extent(d_q, q_values * head_dim * e), extent(d_k, k_bytes), extent(d_v, k_bytes), extent(workspace, need),
                   extent(device_status, kStatusBytes)},
                  {extent(hq, q_rows, q_heads, head_dim, e), extent(hg, q_rows, q_heads, head_dim, e),
                   extent(hk, k_rows, kv_heads, head_dim, e), extent(hv, k_rows, kv_heads, head_dim, e),
                   extent(out, q_values * head_dim * e), extent(out_rest, q_values * head_dim * e), extent(lse, q_values * 4),
                   offsets_extent(q_offsets, batch),
                   offsets_extent(k_offsets, batch), extent(key_mask, static_cast<size_t>(k_rows))}))
    return MPM_ERR_ALIASING;
  int sms = 0;
  st = device_sms(&sms);
  if (st != MPM_OK) return st;
  mpm::AttentionArgs a = common_args(s, hq, hk, hv, q_offsets, k_offsets, scale, key_mask, device_status);
  a.d_out = hg;
  a.out = const_cast<void*>(out);
  a.rest = const_cast<void*>(out_rest);
  a.stats = lse;
  a.d_q = d_q;
  a.d_k = d_k;
  a.d_v = d_v;
  a.splits = plan.splits;
  a.key_splits = plan.key_splits;
  a.delta = static_cast<float*>(workspace);
  a.partial = a.delta + delta_bytes(s) / sizeof(float);
  a.vec = head_dim % 4 == 0 && vector_heads(hq, e, 4) && vector_heads(hk, e, 4) && vector_heads(hv, e, 4) &&
          vector_heads(hg, e, 4);
  const cudaStream_t on = static_cast<cudaStream_t>(stream);
  const cudaError_t err =
      tc ? mpm::launch_attention_backward_tc(a, sms, on) : mpm::launch_attention_backward_f32(a, dtype == MPM_BF16, sms, on);
  return status_of(err);
}

mpm_status mpm_rotary(const void* x, int64_t x_row_stride, int64_t x_head_stride, const float* positions,
                      const double* frequencies, const int32_t* sections, int32_t axes, mpm_rotary_layout layout,
                      int32_t inverse, const int64_t* offsets, int32_t batch, int64_t rows, int32_t heads,
                      int32_t head_dim, mpm_dtype dtype, void* out, int64_t out_row_stride, int64_t out_head_stride,
                      int32_t* device_status, void* stream) {
  const Range range("mpm_rotary");
  if (!valid_dtype(dtype) || rows < 0 || rows > INT32_MAX || heads < 1 || head_dim < 2 || batch < 1 || axes < 1 ||
      sections == nullptr || (layout != MPM_ROTARY_HALVES && layout != MPM_ROTARY_INTERLEAVED))
    return MPM_ERR_INVALID_ARG;
  if (axes > MPM_ROTARY_MAX_AXES || head_dim > MPM_ROTARY_MAX_HEAD_DIM || heads > MPM_ATTENTION_MAX_HEADS)
    return MPM_ERR_UNSUPPORTED;
  mpm::RotaryArgs a{};
  for (int i = 0; i < axes; ++i) {
    if (sections[i] < 1 || sections[i] > head_dim / 2 - a.pairs) return MPM_ERR_INVALID_ARG;
    a.first_pair[i] = a.pairs;
    a.pairs += sections[i];
  }
  if (rows == 0) return MPM_OK;
  if (x == nullptr || out == nullptr || positions == nullptr || frequencies == nullptr) return MPM_ERR_INVALID_ARG;
  Heads in{x, x_row_stride, x_head_stride}, to{out, out_row_stride, out_head_stride};
  if (!strides_ok(&in, rows, heads, head_dim) || !strides_ok(&to, rows, heads, head_dim)) return MPM_ERR_INVALID_ARG;
  const int e = elem(dtype);
  if (!aligned(x, e) || !aligned(out, e) || !aligned(positions, 4) || !aligned(frequencies, 8) || !aligned(offsets, 8) ||
      !aligned(device_status, 4))
    return MPM_ERR_ALIGNMENT;
  const bool in_place = out == x && to.row == in.row && to.head == in.head;
  const Extent written = extent(to, rows, heads, head_dim, e), status = extent(device_status, kStatusBytes);
  const Extent read = extent(in, rows, heads, head_dim, e);
  if (any_overlap({written, status}, {extent(positions, sizeof(float) * static_cast<size_t>(rows) * axes),
                                      extent(frequencies, sizeof(double) * a.pairs), extent(offsets, offsets == nullptr ? 0 : sizeof(int64_t) * (static_cast<size_t>(batch) + 1))}) ||
      overlap(status, read) || (!in_place && overlap(written, read)))
    return MPM_ERR_ALIASING;
  int sms = 0;
  const mpm_status st = device_sms(&sms);
  if (st != MPM_OK) return st;
  a.x = in;
  a.out = out;
  a.out_row = to.row;
  a.out_head = to.head;
  a.positions = positions;
  a.frequencies = frequencies;
  a.offsets = offsets;
  a.rows = rows;
  a.batch = batch;
  a.heads = heads;
  a.dim = head_dim;
  a.axes = axes;
  a.halves = layout == MPM_ROTARY_HALVES;
  a.inverse = inverse != 0;
  a.status = device_status;
  const int s = 16 / e;
  a.vec = head_dim % s == 0 && (a.halves ? a.pairs : 2 * a.pairs) % s == 0 && vector_heads(in, e, s) && vector_heads(to, e, s);
  return status_of(mpm::launch_rotary(a, dtype == MPM_BF16, sms, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
