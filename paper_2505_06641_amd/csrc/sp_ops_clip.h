// The norm over all gradients of a model, and the gradients scaled to at most a given norm.
//   norm = sqrt(sum g^2),  g' = g min(1, max_norm / (norm + 1e-6))
// Squares are summed in 64 bits (no overflow, and sums over 10^8 values keep their last bits; the adds hide behind the loads).  The
// tensors come as a table in the kernels' arguments, cut into pieces, one workgroup each.  One pass leaves every piece's sum in a slot of
// its own; in the next every workgroup adds up all slots, in the same order, and scales its piece: two launches for up to 128
// tensors, and a norm that does not depend on the order in which workgroups run.  (A counter of ended workgroups instead of the kernel
// boundary makes every workgroup write its die's L2 back: the sums over 1.2e8 elements took 391 us, now 131.)  Bound by memory.
#pragma once
#include "sp_ops_common.h"

namespace sp {

constexpr int kClipTensors = 128;          // to a launch: the table has to fit the kernel's arguments
constexpr int kClipThreads = 1024;          // few pieces fill the device: 65536 elements each at 1.2e8
constexpr int kClipPieceMin = 8192, kClipPieceMax = 65536;       // elements; see clip_piece

struct ClipTable {
  const void* src[kClipTensors];
  void* dst[kClipTensors];
  int64_t size[kClipTensors];
  int32_t first[kClipTensors + 1];         // each tensor's first piece within the launch
  int32_t count, piece;                    // tensors, elements of a piece
};

__device__ __forceinline__ int clip_tensor(const ClipTable& tb, int piece) {
  int lo = 0, hi = tb.count;               // first[lo] <= piece < first[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (tb.first[mid] <= piece) lo = mid; else hi = mid;
  }
  return lo;
}

__device__ __forceinline__ double wave_sum_f64(double v) {
#pragma unroll
  for (int s = 1; s < 64; s *= 2) v += __shfl_xor(v, s);
  return v;
}

// Sum of a value over the workgroup's wavefronts, on every thread.
__device__ __forceinline__ double block_sum_f64(double v, double* waves) {
  v = wave_sum_f64(v);
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = v;
  __syncthreads();
  double all = 0.0;
#pragma unroll
  for (int w = 0; w < kClipThreads / 64; ++w) all += waves[w];
  return all;
}

// What a gradient is multiplied by.  A norm that is no number leaves none behind either.
__device__ __forceinline__ float clip_coefficient(double norm, float max_norm) {
  const double ratio = (double)max_norm / (norm + 1e-6);
  return ratio > 1.0 ? 1.f : (float)ratio;
}

// Few elements: one workgroup does both passes with everything in registers between them, and the call is one launch (the second one
// costs the host 3 us and the device a start: 28000 elements in 14 tensors take the device 8 us either way, the host 3 us instead of 6).  Pieces are of 16 bytes;
// a thread takes every 1024th, and has all of its loads under way together.
constexpr int kClipFewEach = 8;

template <typename T>
__global__ __launch_bounds__(kClipThreads) void k_clip_few(ClipTable tb, float max_norm, float* __restrict__ norm_out) {
  constexpr int V = kPiece<T>;
  __shared__ double waves[kClipThreads / 64];
  __shared__ const T* src[kClipTensors];
  __shared__ T* dst[kClipTensors];
  __shared__ int32_t size[kClipTensors], first[kClipTensors + 1];
  if (threadIdx.x < kClipTensors) {
    const int k = threadIdx.x;
    src[k] = (const T*)tb.src[k];
    dst[k] = (T*)tb.dst[k];
    size[k] = (int32_t)tb.size[k];
    first[k] = tb.first[k];
    if (k == 0) first[tb.count] = tb.first[tb.count];
  }
  __syncthreads();
  const int pieces = first[tb.count];
  float v[kClipFewEach][V];
  int tensor[kClipFewEach] = {};
  double s = 0.0;
#pragma unroll
  for (int step = kClipTensors / 2; step > 0; step /= 2)   // the last tensor whose first piece is not behind this one
#pragma unroll
    for (int u = 0; u < kClipFewEach; ++u) {
      const int k = tensor[u] + step;
      if (k < tb.count && first[k] <= (int)threadIdx.x + u * kClipThreads) tensor[u] = k;
    }
#pragma unroll
  for (int u = 0; u < kClipFewEach; ++u) {
    const int piece = threadIdx.x + u * kClipThreads, k = tensor[u], at = (piece - first[k]) * V;
    load_some(src[k] + at, piece < pieces ? size[k] - at : 0, 0.f, v[u]);
  }
#pragma unroll
  for (int u = 0; u < kClipFewEach; ++u)
#pragma unroll
    for (int j = 0; j < V; ++j) s += (double)v[u][j] * (double)v[u][j];
  const double norm = sqrt(block_sum_f64(s, waves));
  if (threadIdx.x == 0) *norm_out = (float)norm;
  const float c = clip_coefficient(norm, max_norm);
#pragma unroll
  for (int u = 0; u < kClipFewEach; ++u) {
    const int piece = threadIdx.x + u * kClipThreads, k = tensor[u], at = (piece - first[k]) * V;
    if (piece >= pieces || (c == 1.f && src[k] == dst[k])) continue;
#pragma unroll
    for (int j = 0; j < V; ++j) v[u][j] *= c;
    store_some(dst[k] + at, size[k] - at, v[u]);
  }
}

// The elements of a workgroup's piece.
template <typename T>
__device__ __forceinline__ int clip_piece_of(const ClipTable& tb, int block, const T** src, T** dst) {
  const int k = clip_tensor(tb, block);
  const int64_t at = (int64_t)(block - tb.first[k]) * tb.piece;
  *src = (const T*)tb.src[k] + at;
  *dst = (T*)tb.dst[k] + at;
  return (int)min((int64_t)tb.piece, tb.size[k] - at);
}


template <typename T>
__global__ __launch_bounds__(kClipThreads) void k_clip_sum(ClipTable tb, double* __restrict__ part) {
  constexpr int V = kPiece<T>;
  __shared__ double waves[kClipThreads / 64];
  const T* src;
  T* dst;
  const int count = clip_piece_of(tb, (int)blockIdx.x, &src, &dst);
  double s = 0.0;
  int i = threadIdx.x * V;
  for (; i + 3 * kClipThreads * V + V <= count; i += 4 * kClipThreads * V) {           // four loads under way
    float v[4][V];
#pragma unroll
    for (int u = 0; u < 4; ++u) load_piece(src + i + u * kClipThreads * V, v[u]);
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int j = 0; j < V; ++j) s += (double)v[u][j] * (double)v[u][j];
  }
  for (; i < count; i += kClipThreads * V) {
    float v[V];
    load_some(src + i, count - i, 0.f, v);
#pragma unroll
    for (int j = 0; j < V; ++j) s += (double)v[j] * (double)v[j];
  }
  s = block_sum_f64(s, waves);
  if (threadIdx.x == 0) part[blockIdx.x] = s;
}

template <typename T>
__global__ __launch_bounds__(kClipThreads) void k_clip_scale(ClipTable tb, int pieces, const double* __restrict__ part, float max_norm,
                                                    float* __restrict__ norm_out) {
  constexpr int V = kPiece<T>;
  __shared__ double waves[kClipThreads / 64];
  double all = 0.0;
  for (int i = threadIdx.x; i < pieces; i += kClipThreads) all += part[i];
  const double norm = sqrt(block_sum_f64(all, waves));
  if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = (float)norm;
  const float c = clip_coefficient(norm, max_norm);
  const T* src;
  T* dst;
  const int count = clip_piece_of(tb, (int)(gridDim.x - 1 - blockIdx.x), &src, &dst);       // the last ones read are still in the cache
  if (c == 1.f && src == dst) return;                      // stays as it is
  int i = threadIdx.x * V;
  for (; i + 3 * kClipThreads * V + V <= count; i += 4 * kClipThreads * V) {
    float v[4][V];
#pragma unroll
    for (int u = 0; u < 4; ++u) load_piece(src + i + u * kClipThreads * V, v[u]);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
#pragma unroll
      for (int j = 0; j < V; ++j) v[u][j] *= c;
      store_piece(dst + i + u * kClipThreads * V, v[u]);
    }
  }
  for (; i < count; i += kClipThreads * V) {
    float v[V];
    load_some(src + i, count - i, 0.f, v);
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] *= c;
    store_some(dst + i, count - i, v);
  }
}

}  // namespace sp
