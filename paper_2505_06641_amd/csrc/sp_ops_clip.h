// The norm over all gradients of a model, and the gradients scaled to at most a given norm.
//   norm = sqrt(sum g^2),  g' = g min(1, max_norm / (norm + 1e-6))
// Squares are summed in 64 bits (no overflow, and sums over 10^8 values keep their last bits; the adds hide behind the loads).  The
// tensors come as a table in the kernel's arguments, cut into pieces of kClipPiece elements, one workgroup each; every piece's
// sum goes to a slot of its own, and the workgroup that ends last adds the slots up in their order: the norm does not depend on the
// order in which workgroups run.  Bound by memory.
#pragma once
#include "sp_ops_common.h"

namespace sp {

constexpr int kClipTensors = 128;          // to a launch: the table has to fit the kernel's arguments
constexpr int kClipPiece = 16384;

struct ClipTable {
  const void* src[kClipTensors];
  void* dst[kClipTensors];
  int64_t size[kClipTensors];
  int32_t first[kClipTensors + 1];         // each tensor's first piece within the launch
  int32_t count;
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

// What the launches of a call share in the operators' workspace.
struct ClipSum {
  unsigned int ended;                      // pieces that have been summed: 0 between calls
  float coefficient;
};

template <typename T>
__global__ __launch_bounds__(256) void k_clip_sum(ClipTable tb, int piece0, int pieces, double* __restrict__ part, ClipSum* sum,
                                                  float max_norm, float* __restrict__ norm_out) {
  constexpr int V = kPiece<T>;
  __shared__ double waves[4];
  __shared__ bool last;
  const int k = clip_tensor(tb, (int)blockIdx.x);
  const int64_t at = (int64_t)((int)blockIdx.x - tb.first[k]) * kClipPiece;
  const T* src = (const T*)tb.src[k] + at;
  const int count = (int)min((int64_t)kClipPiece, tb.size[k] - at);
  double s = 0.0;
  for (int i = threadIdx.x * V; i < count; i += 256 * V) {
    float v[V];
    load_some(src + i, count - i, 0.f, v);
#pragma unroll
    for (int j = 0; j < V; ++j) s += (double)v[j] * (double)v[j];
  }
  s = wave_sum_f64(s);
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    s = (waves[0] + waves[1]) + (waves[2] + waves[3]);
    __hip_atomic_store(part + piece0 + blockIdx.x, s, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    last = __hip_atomic_fetch_add(&sum->ended, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == (unsigned)pieces - 1u;
  }
  __syncthreads();
  if (!last) return;
  double all = 0.0;
  for (int i = threadIdx.x; i < pieces; i += 256)
    all += __hip_atomic_load(part + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  all = wave_sum_f64(all);
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = all;
  __syncthreads();
  if (threadIdx.x == 0) {
    const double norm = sqrt((waves[0] + waves[1]) + (waves[2] + waves[3]));
    *norm_out = (float)norm;
    const double c = (double)max_norm / (norm + 1e-6);
    sum->coefficient = c > 1.0 ? 1.f : (float)c;         // (a norm that is no number leaves none behind either)
    sum->ended = 0u;
  }
}

template <typename T>
__global__ __launch_bounds__(256) void k_clip_scale(ClipTable tb, const ClipSum* __restrict__ sum) {
  constexpr int V = kPiece<T>;
  const int k = clip_tensor(tb, (int)blockIdx.x);
  const int64_t at = (int64_t)((int)blockIdx.x - tb.first[k]) * kClipPiece;
  const T* src = (const T*)tb.src[k] + at;
  T* dst = (T*)tb.dst[k] + at;
  const int count = (int)min((int64_t)kClipPiece, tb.size[k] - at);
  const float c = sum->coefficient;
  for (int i = threadIdx.x * V; i < count; i += 256 * V) {
    float v[V];
    load_some(src + i, count - i, 0.f, v);
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] *= c;
    store_some(dst + i, count - i, v);
  }
}

}  // namespace sp
