// Attention between packed sequences on the CUDA cores, in fp32 throughout: for
// fp32 tokens, and for bf16 tokens whose rows the tensor-core kernels cannot load
// (strides or addresses that are not 16-byte multiples).
//
//   s = scale q.k;  p = exp(s - lse);  o = sum p v
//   ds = p (do.v - delta), delta = do.o;  dq = scale sum ds k;  dk = scale sum ds q;  dv = sum p do
//
// One scheme serves the three passes.  A block of 256 threads keeps a tile of 64
// rows (queries, or keys for dk and dv) in shared memory and streams tiles of 64
// columns past it.  Thread (y, x) of 16 x 16 computes rows 4 y .. + 3 and columns
// x, x + 16, .. of the scores, so that neighbours read rows whose 16-byte pieces
// lie in different banks; a row's statistics are joined by shuffles within a
// half-warp.  The probabilities go to shared memory and multiply a streamed tile,
// 4 rows by 4 (dim <= 64) or 8 features a thread.  The running maximum and sum
// make it one pass over the keys.
//
// Bound: the latency of shared loads with two blocks an SM: the FMA pipe is half
// busy (8 x 1024 tokens, 12 heads of 64: 827 us forward, 31 TFLOP/s; backward 2503,
// 36 with the scores formed twice).  Eight rows a thread (794 and 2459, but 3146
// instead of 2622 for heads of 128), tiles loaded ahead into registers (854, 2651),
// FMAs in pairs (833, 2635) and three blocks (857, 3196) were no faster on the whole.
//
// Nothing outside a sequence enters a sum: rows past its end and masked keys are
// loaded as zeros (a NaN there would survive a product with 0) and their scores
// count as minus infinity.
#include "attention_common.cuh"

namespace mpm {
namespace {

using namespace attn;

constexpr int kTile = 64;
constexpr int kR = 4;              // rows of a thread
constexpr int kThreads = 16 * kTile / kR;
constexpr int kRowThreads = 256;   // of the kernels that work row by row

template <int DP>
struct Shape {
  static constexpr int kPitch = DP + 4;        // floats of a row in shared memory
  static constexpr int kCols = DP / 16;        // features that a thread sums
  static constexpr int kMatrix = kTile * kPitch;
  // Forward, wide heads: probabilities in the keys' place, so that an SM holds two blocks.
  static constexpr bool kOverKeys = DP == 128;
};
constexpr int kScorePitch = kTile + 4;
constexpr int kScores = kTile * kScorePitch;

// Rows first .. first + 63 of one head on their way to shared memory, all of a
// thread's pieces of four features under way at once.  Zeros past the
// sequence, past the head's width and for masked rows.
template <typename T, int DP>
struct Rows {
  static constexpr int kPieces = kTile * DP / 4 / kThreads;
  float4 v[kPieces];

  __device__ __forceinline__ void load(const Heads& x, int head, const Span& s, int first, int dim, int d4, bool vec,
                                       const uint8_t* __restrict__ mask) {
    const T* base = static_cast<const T*>(x.p) + x.head * head;
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int u = threadIdx.x + kThreads * i, c = u % (DP / 4) * 4, row = first + u / (DP / 4);
      v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (c < d4 && row < s.n && (mask == nullptr || __ldg(mask + s.lo + row) != 0)) {
        const T* p = base + x.row * (s.lo + row) + c;
        if (vec) {
          if constexpr (sizeof(T) == 4) {
            v[i] = __ldg(reinterpret_cast<const float4*>(p));
          } else {
            const uint2 w = __ldg(reinterpret_cast<const uint2*>(p));
            v[i] = make_float4(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xFFFF0000u), __uint_as_float(w.y << 16),
                               __uint_as_float(w.y & 0xFFFF0000u));
          }
        } else {
          v[i].x = to_f32(p[0]);
          if (c + 1 < dim) v[i].y = to_f32(p[1]);
          if (c + 2 < dim) v[i].z = to_f32(p[2]);
          if (c + 3 < dim) v[i].w = to_f32(p[3]);
        }
      }
    }
  }
  // All columns are written, so that sums over them find zeros past the width.
  __device__ __forceinline__ void store(float* sm) const {
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int u = threadIdx.x + kThreads * i;
      *reinterpret_cast<float4*>(sm + u / (DP / 4) * Shape<DP>::kPitch + u % (DP / 4) * 4) = v[i];
    }
  }
};
// acc[i][j] = rows[kR y + i] . cols[x + 16 j]
template <int DP>
__device__ __forceinline__ void dot_tile(const float* rows, const float* cols, int d4, float (&acc)[kR][4]) {
  const int x = threadIdx.x & 15, y = threadIdx.x >> 4;
#pragma unroll
  for (int i = 0; i < kR; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = 0.f;
#pragma unroll 4
  for (int d = 0; d < d4; d += 4) {
    float4 r[kR], c[4];
#pragma unroll
    for (int i = 0; i < kR; ++i) r[i] = *reinterpret_cast<const float4*>(rows + (kR * y + i) * Shape<DP>::kPitch + d);
#pragma unroll
    for (int j = 0; j < 4; ++j) c[j] = *reinterpret_cast<const float4*>(cols + (x + 16 * j) * Shape<DP>::kPitch + d);
#pragma unroll
    for (int i = 0; i < kR; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        acc[i][j] = fmaf(r[i].x, c[j].x, acc[i][j]);
        acc[i][j] = fmaf(r[i].y, c[j].y, acc[i][j]);
        acc[i][j] = fmaf(r[i].z, c[j].z, acc[i][j]);
        acc[i][j] = fmaf(r[i].w, c[j].w, acc[i][j]);
      }
  }
}

// Features 4 x + 64 g + {0 .. 3} of acc[i], in pairs, += sum over columns c of scores[kR y + i][c] * tile[c]
template <int DP>
__device__ __forceinline__ void sum_tile(const float* scores, const float* tile, float2 (&acc)[kR][Shape<DP>::kCols / 2]) {
  const int x = threadIdx.x & 15, y = threadIdx.x >> 4;
#pragma unroll 4
  for (int c = 0; c < kTile; c += 4) {
    float4 s[kR];
#pragma unroll
    for (int i = 0; i < kR; ++i) s[i] = *reinterpret_cast<const float4*>(scores + (kR * y + i) * kScorePitch + c);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
#pragma unroll
      for (int g = 0; g < DP / 64; ++g) {
        const float4 t = *reinterpret_cast<const float4*>(tile + (c + k) * Shape<DP>::kPitch + 4 * x + 64 * g);
#pragma unroll
        for (int i = 0; i < kR; ++i) {
          const float w = k == 0 ? s[i].x : k == 1 ? s[i].y : k == 2 ? s[i].z : s[i].w;
          acc[i][2 * g] = norm::fma(make_float2(w, w), make_float2(t.x, t.y), acc[i][2 * g]);
          acc[i][2 * g + 1] = norm::fma(make_float2(w, w), make_float2(t.z, t.w), acc[i][2 * g + 1]);
        }
      }
    }
  }
}

// The thread's scores to shared memory.
__device__ __forceinline__ void put_scores(float* scores, const float (&v)[kR][4]) {
  const int x = threadIdx.x & 15, y = threadIdx.x >> 4;
#pragma unroll
  for (int i = 0; i < kR; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) scores[(kR * y + i) * kScorePitch + x + 16 * j] = v[i][j];
}

// The thread's sums, times a factor a row, to rows of `dim` contiguous values, and
// what their rounding left to rows of `rest`, if that is wanted.
template <typename T, int DP>
__device__ __forceinline__ void store_rows(T* out, int64_t row0, int rows, int heads, int head, int dim,
                                           const float2 (&acc)[kR][Shape<DP>::kCols / 2], const float (&factor)[kR], T* rest = nullptr) {
  const int x = threadIdx.x & 15, y = threadIdx.x >> 4;
#pragma unroll
  for (int i = 0; i < kR; ++i) {
    if (kR * y + i >= rows) continue;
    const int64_t at = ((row0 + kR * y + i) * heads + head) * dim;
#pragma unroll
    for (int e = 0; e < Shape<DP>::kCols; ++e) {
      const int c = 4 * x + 64 * (e / 4) + e % 4;
      if (c >= dim) continue;
      const float v = (e % 2 == 0 ? acc[i][e / 2].x : acc[i][e / 2].y) * factor[i];
      out[at + c] = from_f32<T>(v);
      if (rest != nullptr) rest[at + c] = rest_of<T>(v);
    }
  }
}

__device__ __forceinline__ float half_warp_max(float v) {
#pragma unroll
  for (int d = 8; d > 0; d >>= 1) v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, d));
  return v;
}
__device__ __forceinline__ float half_warp_sum(float v) {
#pragma unroll
  for (int d = 8; d > 0; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
  return v;
}

struct Item {
  Tile tile;
  int head, split;
};
// Items are numbered with the tile fastest: neighbours read the same head's rows.
template <int T>
__device__ __forceinline__ Item item_of(int64_t item, const int64_t* off, int batch, int64_t rows, int heads) {
  const int64_t slots = tile_slots<T>(off, batch, rows), rest = item / slots;
  return {tile_of<T>(off, batch, rows, item % slots), static_cast<int>(rest % heads), static_cast<int>(rest / heads)};
}

template <typename T, int DP>
__global__ void __launch_bounds__(kThreads, DP == 64 ? 2 : 1) attention_simt_kernel(const AttentionArgs a) {
  extern __shared__ float sm[];
  float* sq = sm;
  float* sk = sq + Shape<DP>::kMatrix;
  float* sv = sk + Shape<DP>::kMatrix;
  float* sp = Shape<DP>::kOverKeys ? sk : sv + Shape<DP>::kMatrix;
  wait_for_previous_grid();
  allow_next_grid();
  if (blockIdx.x == 0) {
    check_offsets(a.q_offsets, a.batch, a.q_rows, a.status);
    check_offsets(a.k_offsets, a.batch, a.k_rows, a.status);
  }
  const int x = threadIdx.x & 15, y = threadIdx.x >> 4;
  const int d4 = (a.dim + 3) / 4 * 4;
  const float c = a.scale * kLog2e;
  const int64_t items = tile_slots<kTile>(a.q_offsets, a.batch, a.q_rows) * a.q_heads * a.splits;
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const Item w = item_of<kTile>(it, a.q_offsets, a.batch, a.q_rows, a.q_heads);
    if (w.tile.image < 0) continue;
    const Span ks = span_of(a.k_offsets, w.tile.image, a.k_rows);
    const int kv = w.head / (a.q_heads / a.kv_heads);
    const Part part = part_of((ks.n + kTile - 1) / kTile, w.split, a.splits);
    float2 acc[kR][Shape<DP>::kCols / 2] = {};
    float top[kR], sum[kR];
#pragma unroll
    for (int i = 0; i < kR; ++i) {
      top[i] = -INFINITY;
      sum[i] = 0.f;
    }
    Rows<T, DP> next, values;
    values.load(a.q, w.head, w.tile.rows, w.tile.first, a.dim, d4, a.vec, nullptr);
    __syncthreads();  // the last item's tiles have been read
    values.store(sq);
    for (int t = part.begin; t < part.end; ++t) {
      if (Shape<DP>::kOverKeys && t > part.begin) __syncthreads();
      next.load(a.k, kv, ks, t * kTile, a.dim, d4, a.vec, a.mask);
      next.store(sk);
      __syncthreads();
      float s[kR][4];
      dot_tile<DP>(sq, sk, d4, s);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int key = t * kTile + x + 16 * j;
        const bool there = key < ks.n && (a.mask == nullptr || __ldg(a.mask + ks.lo + key) != 0);
#pragma unroll
        for (int i = 0; i < kR; ++i)
          if (!there) s[i][j] = -INFINITY;
      }
#pragma unroll
      for (int i = 0; i < kR; ++i) {
        // In units of log2: c is positive, so the largest score is the largest product.
        const float m = fmaxf(top[i], half_warp_max(fmaxf(fmaxf(s[i][0], s[i][1]), fmaxf(s[i][2], s[i][3]))) * c);
        const float base = m == -INFINITY ? 0.f : m;
        const float shrink = exp2f(top[i] - base);
        top[i] = m;
        float part_sum = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          s[i][j] = exp2f(fmaf(s[i][j], c, -base));
          part_sum += s[i][j];
        }
        sum[i] = fmaf(sum[i], shrink, half_warp_sum(part_sum));
#pragma unroll
        for (int e = 0; e < Shape<DP>::kCols / 2; ++e) acc[i][e] = norm::mul(acc[i][e], make_float2(shrink, shrink));
      }
      if (Shape<DP>::kOverKeys) __syncthreads();
      put_scores(sp, s);
      values.load(a.v, kv, ks, t * kTile, a.dim, d4, a.vec, a.mask);
      values.store(sv);
      __syncthreads();
      sum_tile<DP>(sp, sv, acc);
    }
    const int64_t row0 = w.tile.rows.lo + w.tile.first;
    const int rows = w.tile.rows.n - w.tile.first;
    float factor[kR];
#pragma unroll
    for (int i = 0; i < kR; ++i) factor[i] = sum[i] == 0.f ? 0.f : 1.f / sum[i];
    const int64_t part0 = a.splits == 1 ? 0 : static_cast<int64_t>(w.split) * a.q_rows * a.q_heads;
    if (a.splits == 1)
      store_rows<T, DP>(static_cast<T*>(a.out), row0, rows, a.q_heads, w.head, a.dim, acc, factor, static_cast<T*>(a.rest));
    else
      store_rows<float, DP>(a.partial + part0 * a.dim, row0, rows, a.q_heads, w.head, a.dim, acc, factor);
    float* lse = a.splits == 1 ? a.lse : a.partial_lse + part0;
    if (lse != nullptr && x == 0) {
#pragma unroll
      for (int i = 0; i < kR; ++i)
        if (kR * y + i < rows)
          lse[(row0 + kR * y + i) * a.q_heads + w.head] = (top[i] + log2f(sum[i])) * (a.splits == 1 ? kLn2 : 1.f);
    }
  }
}

// p and ds of the thread's 4 x 4 scores; `there` holds for the column.
__device__ __forceinline__ void back_scores(float s, float dp, float c, float lse2, float delta, bool there, float& p, float& ds) {
  p = there ? exp2f(fmaf(s, c, -lse2)) : 0.f;
  ds = there ? p * (dp - delta) : 0.f;
}
// The row's statistic in log2 units; a row without keys has no probabilities.
__device__ __forceinline__ float log2_stat(float lse) { return lse == -INFINITY ? INFINITY : lse * kLog2e; }

template <typename T, int DP>
__global__ void __launch_bounds__(kThreads, DP == 64 ? 2 : 1) attention_simt_dq_kernel(const AttentionArgs a) {
  extern __shared__ float sm[];
  float* sq = sm;
  float* sg = sq + Shape<DP>::kMatrix;
  float* sk = sg + Shape<DP>::kMatrix;
  float* sv = sk + Shape<DP>::kMatrix;
  float* sp = sv + Shape<DP>::kMatrix;
  wait_for_previous_grid();
  allow_next_grid();
  const int x = threadIdx.x & 15, y = threadIdx.x >> 4;
  const int d4 = (a.dim + 3) / 4 * 4;
  const float c = a.scale * kLog2e;
  const int64_t items = tile_slots<kTile>(a.q_offsets, a.batch, a.q_rows) * a.q_heads * a.splits;
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const Item w = item_of<kTile>(it, a.q_offsets, a.batch, a.q_rows, a.q_heads);
    if (w.tile.image < 0) continue;
    const Span ks = span_of(a.k_offsets, w.tile.image, a.k_rows);
    const int kv = w.head / (a.q_heads / a.kv_heads);
    const Part part = part_of((ks.n + kTile - 1) / kTile, w.split, a.splits);
    const int64_t row0 = w.tile.rows.lo + w.tile.first;
    const int rows = w.tile.rows.n - w.tile.first;
    float2 acc[kR][Shape<DP>::kCols / 2] = {};
    float lse2[kR], delta[kR];
#pragma unroll
    for (int i = 0; i < kR; ++i) {
      const bool live = kR * y + i < rows;
      lse2[i] = live ? log2_stat(__ldg(a.stats + (row0 + kR * y + i) * a.q_heads + w.head)) : INFINITY;
      delta[i] = live ? a.delta[(row0 + kR * y + i) * a.q_heads + w.head] : 0.f;
    }
    Rows<T, DP> one, two;
    one.load(a.q, w.head, w.tile.rows, w.tile.first, a.dim, d4, a.vec, nullptr);
    two.load(a.d_out, w.head, w.tile.rows, w.tile.first, a.dim, d4, a.vec, nullptr);
    __syncthreads();  // the last item's tiles have been read
    one.store(sq);
    two.store(sg);
    for (int t = part.begin; t < part.end; ++t) {
      if (t > part.begin) __syncthreads();
      one.load(a.k, kv, ks, t * kTile, a.dim, d4, a.vec, a.mask);
      two.load(a.v, kv, ks, t * kTile, a.dim, d4, a.vec, a.mask);
      one.store(sk);
      two.store(sv);
      __syncthreads();
      float s[kR][4], dp[kR][4];
      dot_tile<DP>(sq, sk, d4, s);
      dot_tile<DP>(sg, sv, d4, dp);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int key = t * kTile + x + 16 * j;
        const bool there = key < ks.n && (a.mask == nullptr || __ldg(a.mask + ks.lo + key) != 0);
#pragma unroll
        for (int i = 0; i < kR; ++i) {
          float p;
          back_scores(s[i][j], dp[i][j], c, lse2[i], delta[i], there && lse2[i] != INFINITY, p, s[i][j]);
        }
      }
      put_scores(sp, s);
      __syncwarp();
      sum_tile<DP>(sp, sk, acc);
    }
    float factor[kR];
#pragma unroll
    for (int i = 0; i < kR; ++i) factor[i] = a.scale;
    if (a.splits == 1)
      store_rows<T, DP>(static_cast<T*>(a.d_q), row0, rows, a.q_heads, w.head, a.dim, acc, factor);
    else
      store_rows<float, DP>(a.partial + static_cast<int64_t>(w.split) * a.q_rows * a.q_heads * a.dim, row0, rows, a.q_heads,
                            w.head, a.dim, acc, factor);
  }
}

template <typename T, int DP>
__global__ void __launch_bounds__(kThreads, DP == 64 ? 2 : 1) attention_simt_dkv_kernel(const AttentionArgs a) {
  extern __shared__ float sm[];
  float* sk = sm;
  float* sv = sk + Shape<DP>::kMatrix;
  float* sq = sv + Shape<DP>::kMatrix;
  float* sg = sq + Shape<DP>::kMatrix;
  float* sp = sg + Shape<DP>::kMatrix;
  __shared__ float stat[kTile], dot[kTile];
  wait_for_previous_grid();
  allow_next_grid();
  const int x = threadIdx.x & 15, y = threadIdx.x >> 4;
  const int d4 = (a.dim + 3) / 4 * 4;
  const float c = a.scale * kLog2e;
  const int group = a.q_heads / a.kv_heads;
  const int64_t items = tile_slots<kTile>(a.k_offsets, a.batch, a.k_rows) * a.kv_heads * a.key_splits;
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const Item w = item_of<kTile>(it, a.k_offsets, a.batch, a.k_rows, a.kv_heads);
    if (w.tile.image < 0) continue;
    const Span qs = span_of(a.q_offsets, w.tile.image, a.q_rows);
    const int tiles = (qs.n + kTile - 1) / kTile;
    const Part part = part_of(tiles * group, w.split, a.key_splits);
    const int64_t row0 = w.tile.rows.lo + w.tile.first;
    const int rows = w.tile.rows.n - w.tile.first;
    float2 dk[kR][Shape<DP>::kCols / 2] = {}, dv[kR][Shape<DP>::kCols / 2] = {};
    bool there[kR];
#pragma unroll
    for (int i = 0; i < kR; ++i)
      there[i] = kR * y + i < rows && (a.mask == nullptr || __ldg(a.mask + row0 + kR * y + i) != 0);
    Rows<T, DP> one, two;
    one.load(a.k, w.head, w.tile.rows, w.tile.first, a.dim, d4, a.vec, a.mask);
    two.load(a.v, w.head, w.tile.rows, w.tile.first, a.dim, d4, a.vec, a.mask);
    __syncthreads();  // the last item's tiles have been read
    one.store(sk);
    two.store(sv);
    for (int t = part.begin; t < part.end; ++t) {
      if (t > part.begin) __syncthreads();
      const int head = w.head * group + t / tiles, first = t % tiles * kTile;
      one.load(a.q, head, qs, first, a.dim, d4, a.vec, nullptr);
      two.load(a.d_out, head, qs, first, a.dim, d4, a.vec, nullptr);
      one.store(sq);
      two.store(sg);
      if (threadIdx.x < kTile) {
        const int r = first + threadIdx.x;
        const int64_t at = (qs.lo + r) * a.q_heads + head;
        stat[threadIdx.x] = r < qs.n ? log2_stat(__ldg(a.stats + at)) : INFINITY;
        dot[threadIdx.x] = r < qs.n ? a.delta[at] : 0.f;
      }
      __syncthreads();
      float s[kR][4], dp[kR][4];
      dot_tile<DP>(sk, sq, d4, s);
      dot_tile<DP>(sv, sg, d4, dp);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float l = stat[x + 16 * j], e = dot[x + 16 * j];
#pragma unroll
        for (int i = 0; i < kR; ++i)
          back_scores(s[i][j], dp[i][j], c, l, e, there[i] && l != INFINITY, s[i][j], dp[i][j]);
      }
      put_scores(sp, s);
      __syncwarp();
      sum_tile<DP>(sp, sg, dv);
      __syncwarp();
      put_scores(sp, dp);
      __syncwarp();
      sum_tile<DP>(sp, sq, dk);
    }
    float scales[kR], ones[kR];
#pragma unroll
    for (int i = 0; i < kR; ++i) {
      scales[i] = a.scale;
      ones[i] = 1.f;
    }
    if (a.key_splits == 1) {
      store_rows<T, DP>(static_cast<T*>(a.d_k), row0, rows, a.kv_heads, w.head, a.dim, dk, scales);
      store_rows<T, DP>(static_cast<T*>(a.d_v), row0, rows, a.kv_heads, w.head, a.dim, dv, ones);
    } else {
      const int64_t each = a.k_rows * a.kv_heads * a.dim;
      float* p = a.partial + w.split * each;
      store_rows<float, DP>(p, row0, rows, a.kv_heads, w.head, a.dim, dk, scales);
      store_rows<float, DP>(p + a.key_splits * each, row0, rows, a.kv_heads, w.head, a.dim, dv, ones);
    }
  }
}

// out = sum over parts of 2^(l_s - l) o_s, l = log2 sum 2^l_s: a warp a row and head.
template <typename T>
__global__ void __launch_bounds__(kRowThreads) attention_join_kernel(const AttentionArgs a) {
  wait_for_previous_grid();
  allow_next_grid();
  const int lane = threadIdx.x & 31;
  const int64_t all = a.q_rows * a.q_heads, live = live_rows(a.q_offsets, a.batch, a.q_rows) * a.q_heads;
  for (int64_t r = blockIdx.x * int64_t{kRowThreads / 32} + threadIdx.x / 32; r < live; r += gridDim.x * int64_t{kRowThreads / 32}) {
    // Two parts a lane.
    float l[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) l[i] = lane + 32 * i < a.splits ? a.partial_lse[(lane + 32 * i) * all + r] : -INFINITY;
    float top = fmaxf(l[0], l[1]);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
    const float base = top == -INFINITY ? 0.f : top;
    float w[2] = {exp2f(l[0] - base), exp2f(l[1] - base)};
    float sum = w[0] + w[1];
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    w[0] *= inv;
    w[1] *= inv;
    float v[kAttentionMaxDim / 32] = {};
#pragma unroll 4
    for (int s = 0; s < a.splits; ++s) {
      const float f = __shfl_sync(0xFFFFFFFFu, s < 32 ? w[0] : w[1], s & 31);
      const float* p = a.partial + (s * all + r) * a.dim;
#pragma unroll
      for (int i = 0; i < kAttentionMaxDim / 32; ++i)
        if (lane + 32 * i < a.dim) v[i] = fmaf(f, p[lane + 32 * i], v[i]);
    }
    T* out = static_cast<T*>(a.out) + r * a.dim;
#pragma unroll
    for (int i = 0; i < kAttentionMaxDim / 32; ++i)
      if (lane + 32 * i < a.dim) {
        out[lane + 32 * i] = from_f32<T>(v[i]);
        if (a.rest != nullptr) static_cast<T*>(a.rest)[r * a.dim + lane + 32 * i] = rest_of<T>(v[i]);
      }
    if (a.lse != nullptr && lane == 0) a.lse[r] = (top + log2f(sum)) * kLn2;
  }
}

template <typename T>
__global__ void __launch_bounds__(kRowThreads) attention_delta_kernel(const AttentionArgs a, bool wide) {
  wait_for_previous_grid();
  allow_next_grid();
  if (blockIdx.x == 0) {
    check_offsets(a.q_offsets, a.batch, a.q_rows, a.status);
    check_offsets(a.k_offsets, a.batch, a.k_rows, a.status);
  }
  const int lane = threadIdx.x & 31;
  const int64_t live = live_rows(a.q_offsets, a.batch, a.q_rows) * a.q_heads;
  if constexpr (sizeof(T) == 2) {
    if (wide) {
      // Eight features a lane, eight or sixteen lanes a row and head.
      const int lanes = a.dim <= 64 ? 8 : 16, d = lane % lanes * 8, each = 32 / lanes;
      const bool there = d < a.dim;
      const int64_t step = gridDim.x * int64_t{kRowThreads} / lanes;
      for (int64_t first = (blockIdx.x * int64_t{kRowThreads} + threadIdx.x) / 32 * each; first < live; first += step) {
        const int64_t r = first + lane / lanes;
        float v = 0.f;
        if (there && r < live) {
          const int64_t row = r <= UINT32_MAX ? static_cast<uint32_t>(r) / static_cast<uint32_t>(a.q_heads) : r / a.q_heads;
          const uint4 o = ld_stream(reinterpret_cast<const uint4*>(static_cast<const T*>(a.out) + r * a.dim + d));
          uint4 e = make_uint4(0, 0, 0, 0);
          if (a.rest != nullptr) e = ld_stream(reinterpret_cast<const uint4*>(static_cast<const T*>(a.rest) + r * a.dim + d));
          const uint4 g = __ldg(reinterpret_cast<const uint4*>(static_cast<const T*>(a.d_out.p) + a.d_out.row * row +
                                                               a.d_out.head * (r - row * a.q_heads) + d));
          const norm::F8 fo = norm::widen(o), fe = norm::widen(e), fg = norm::widen(g);
          float2 s = make_float2(0.f, 0.f);
#pragma unroll
          for (int k = 0; k < 4; ++k) s = norm::fma(norm::add(fo.p[k], fe.p[k]), fg.p[k], s);
          v = s.x + s.y;
        }
#pragma unroll
        for (int x = 8; x > 0; x >>= 1)
          if (x < lanes) v += __shfl_xor_sync(0xFFFFFFFFu, v, x);
        if (d == 0 && r < live) a.delta[r] = v;
      }
      return;
    }
  }
  for (int64_t r = blockIdx.x * int64_t{kRowThreads / 32} + threadIdx.x / 32; r < live; r += gridDim.x * int64_t{kRowThreads / 32}) {
    const T* o = static_cast<const T*>(a.out) + r * a.dim;
    const T* rest = a.rest == nullptr ? nullptr : static_cast<const T*>(a.rest) + r * a.dim;
    const T* g = static_cast<const T*>(a.d_out.p) + a.d_out.row * (r / a.q_heads) + a.d_out.head * (r % a.q_heads);
    float s = 0.f;
    for (int d = lane; d < a.dim; d += 32) s = fmaf(to_f32(o[d]) + (rest == nullptr ? 0.f : to_f32(rest[d])), to_f32(g[d]), s);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
    if (lane == 0) a.delta[r] = s;
  }
}

template <typename T>
__global__ void __launch_bounds__(kRowThreads) attention_sum_kernel(const float* __restrict__ parts, int splits, int64_t rows,
                                                                 const int64_t* __restrict__ offsets, int batch, int width,
                                                                 T* __restrict__ out) {
  wait_for_previous_grid();
  allow_next_grid();
  const int64_t each = rows * width, live = live_rows(offsets, batch, rows) * width;
  for (int64_t i = blockIdx.x * int64_t{kRowThreads} + threadIdx.x; i < live; i += gridDim.x * int64_t{kRowThreads}) {
    float s = 0.f;
#pragma unroll 4
    for (int p = 0; p < splits; ++p) s += parts[p * each + i];
    out[i] = from_f32<T>(s);
  }
}

int blocks_for(int64_t work, int64_t most) { return static_cast<int>(work < 1 ? 1 : work < most ? work : most); }

// Launches with dynamic shared memory on as many blocks as are resident at once.
template <typename K>
cudaError_t launch_tiles(K kernel, size_t smem, int64_t items, const AttentionArgs& a, int num_sms, cudaStream_t stream) {
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
  if (e != cudaSuccess) return e;
  int each = 0;
  e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&each, kernel, kThreads, smem);
  if (e != cudaSuccess) return e;
  return launch_dependent(kernel, dim3(blocks_for(items, int64_t{num_sms} * (each < 1 ? 1 : each))), dim3(kThreads), smem, stream, a);
}

template <typename T, int DP>
cudaError_t forward(const AttentionArgs& a, int num_sms, cudaStream_t stream) {
  const int64_t items = tile_slots<kTile>(a.q_offsets, a.batch, a.q_rows) * a.q_heads * a.splits;
  return launch_tiles(attention_simt_kernel<T, DP>, sizeof(float) * (3 * Shape<DP>::kMatrix + (Shape<DP>::kOverKeys ? 0 : kScores)), items, a, num_sms, stream);
}
template <typename T, int DP>
cudaError_t backward(const AttentionArgs& a, int num_sms, cudaStream_t stream) {
  constexpr size_t smem = sizeof(float) * (4 * Shape<DP>::kMatrix + kScores);
  const int64_t q_items = tile_slots<kTile>(a.q_offsets, a.batch, a.q_rows) * a.q_heads * a.splits;
  const int64_t k_items = tile_slots<kTile>(a.k_offsets, a.batch, a.k_rows) * a.kv_heads * a.key_splits;
  constexpr bool bf16 = sizeof(T) == 2;
  cudaError_t e = launch_attention_delta(a, bf16, num_sms, stream);
  if (e == cudaSuccess && a.q_rows > 0) {
    e = launch_tiles(attention_simt_dq_kernel<T, DP>, smem, q_items, a, num_sms, stream);
    if (e == cudaSuccess && a.splits > 1)
      e = launch_attention_sum(a.partial, a.splits, a.q_rows, a.q_offsets, a.batch, a.q_heads, a.dim, a.d_q, bf16, num_sms, stream);
  }
  if (e == cudaSuccess && a.k_rows > 0) {
    e = launch_tiles(attention_simt_dkv_kernel<T, DP>, smem, k_items, a, num_sms, stream);
    const int64_t each = a.k_rows * a.kv_heads * a.dim;
    if (e == cudaSuccess && a.key_splits > 1)
      e = launch_attention_sum(a.partial, a.key_splits, a.k_rows, a.k_offsets, a.batch, a.kv_heads, a.dim, a.d_k, bf16, num_sms, stream);
    if (e == cudaSuccess && a.key_splits > 1)
      e = launch_attention_sum(a.partial + a.key_splits * each, a.key_splits, a.k_rows, a.k_offsets, a.batch, a.kv_heads, a.dim,
                               a.d_v, bf16, num_sms, stream);
  }
  return e;
}

}  // namespace

cudaError_t launch_attention_simt(const AttentionArgs& a, bool bf16, int num_sms, cudaStream_t stream) {
  if (bf16) return a.dim <= 64 ? forward<__nv_bfloat16, 64>(a, num_sms, stream) : forward<__nv_bfloat16, 128>(a, num_sms, stream);
  return a.dim <= 64 ? forward<float, 64>(a, num_sms, stream) : forward<float, 128>(a, num_sms, stream);
}

cudaError_t launch_attention_backward_simt(const AttentionArgs& a, bool bf16, int num_sms, cudaStream_t stream) {
  if (bf16) return a.dim <= 64 ? backward<__nv_bfloat16, 64>(a, num_sms, stream) : backward<__nv_bfloat16, 128>(a, num_sms, stream);
  return a.dim <= 64 ? backward<float, 64>(a, num_sms, stream) : backward<float, 128>(a, num_sms, stream);
}

cudaError_t launch_attention_join(const AttentionArgs& a, bool bf16, int num_sms, cudaStream_t stream) {
  const int blocks = blocks_for((a.q_rows * a.q_heads + 7) / 8, int64_t{num_sms} * 8);
  return bf16 ? launch_dependent(attention_join_kernel<__nv_bfloat16>, dim3(blocks), dim3(kRowThreads), 0, stream, a)
              : launch_dependent(attention_join_kernel<float>, dim3(blocks), dim3(kRowThreads), 0, stream, a);
}

cudaError_t launch_attention_delta(const AttentionArgs& a, bool bf16, int num_sms, cudaStream_t stream) {
  const int blocks = blocks_for((a.q_rows * a.q_heads + 7) / 8, int64_t{num_sms} * 8);
  const uintptr_t all = reinterpret_cast<uintptr_t>(a.out) | reinterpret_cast<uintptr_t>(a.rest) | reinterpret_cast<uintptr_t>(a.d_out.p);
  const bool wide = bf16 && a.dim % 8 == 0 && all % 16 == 0 && a.d_out.row % 8 == 0 && a.d_out.head % 8 == 0;
  return bf16 ? launch_dependent(attention_delta_kernel<__nv_bfloat16>, dim3(blocks), dim3(kRowThreads), 0, stream, a, wide)
              : launch_dependent(attention_delta_kernel<float>, dim3(blocks), dim3(kRowThreads), 0, stream, a, wide);
}

cudaError_t launch_attention_sum(const float* parts, int splits, int64_t rows, const int64_t* offsets, int batch, int heads,
                                 int dim, void* out, bool bf16, int num_sms, cudaStream_t stream) {
  const int width = heads * dim;
  const int blocks = blocks_for((rows * width + kRowThreads - 1) / kRowThreads, int64_t{num_sms} * 8);
  return bf16 ? launch_dependent(attention_sum_kernel<__nv_bfloat16>, dim3(blocks), dim3(kRowThreads), 0, stream, parts, splits, rows,
                                 offsets, batch, width, static_cast<__nv_bfloat16*>(out))
              : launch_dependent(attention_sum_kernel<float>, dim3(blocks), dim3(kRowThreads), 0, stream, parts, splits, rows, offsets,
                                 batch, width, static_cast<float*>(out));
}

}  // namespace mpm
