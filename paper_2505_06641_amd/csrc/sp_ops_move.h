// Rows on their way to the experts and back.
//   dispatch       xs[place_ij] = x_i
//   combine        y_i = sum over j of w_ij ys[place_ij] + r_i
//   its gradients  dys[place_ij] = w_ij dy_i        dw_ij = dy_i . ys[place_ij]
// A team of lanes takes a row of x, y or dy; the rows at the places are whole rows somewhere else, so that every access is a run of
// 16-byte pieces.  Bound by memory.
#pragma once
#include "sp_ops_common.h"

namespace sp {

constexpr int kMoveBlocks = 8192;

// A pair's place, or -1: none, or one that is no row.
__device__ __forceinline__ int place_of(const int32_t* __restrict__ place, int64_t pair, int rows, uint32_t* err, bool report) {
  const int p = place[pair];
  if (p >= -1 && p < rows) return p;
  if (report) atomicOr(err, kErrPlace);
  return -1;
}

template <typename T, int TEAM>
__global__ __launch_bounds__(256) void k_dispatch(int n, int d, int top, const T* __restrict__ x, int64_t x_stride,
                                                  const int32_t* __restrict__ place, int rows, T* __restrict__ xs, int64_t xs_stride,
                                                  uint32_t* err) {
  constexpr int V = kPiece<T>, ROWS = 256 / TEAM;
  const int t = threadIdx.x % TEAM, team = threadIdx.x / TEAM;
  for (int64_t row = (int64_t)blockIdx.x * ROWS + team; row < n; row += (int64_t)gridDim.x * ROWS) {
    for (int64_t col = t * V; col < d; col += TEAM * V) {
      float v[V];
      load_some(x + row * x_stride + col, (int)(d - col), 0.f, v);
      for (int j = 0; j < top; ++j) {
        const int p = place_of(place, row * top + j, rows, err, t == 0);
        if (p >= 0) store_some(xs + p * xs_stride + col, (int)(d - col), v);
      }
    }
  }
}

template <typename T, int TEAM>
__global__ __launch_bounds__(256) void k_combine(int n, int d, int top, int rows, const T* __restrict__ ys, int64_t ys_stride,
                                                 const int32_t* __restrict__ place, const float* __restrict__ weight, const T* residual,
                                                 int64_t residual_stride, T* y, int64_t y_stride, uint32_t* err) {
  constexpr int V = kPiece<T>, ROWS = 256 / TEAM;
  const int t = threadIdx.x % TEAM, team = threadIdx.x / TEAM;
  for (int64_t row = (int64_t)blockIdx.x * ROWS + team; row < n; row += (int64_t)gridDim.x * ROWS) {
    for (int64_t col = t * V; col < d; col += TEAM * V) {
      const int count = (int)min((int64_t)V, d - col);
      float sum[V] = {};
      for (int j = 0; j < top; ++j) {
        const int p = place_of(place, row * top + j, rows, err, t == 0);
        if (p < 0) continue;
        const float w = weight ? weight[row * top + j] : 1.f;
        float v[V];
        load_some(ys + p * ys_stride + col, count, 0.f, v);
#pragma unroll
        for (int i = 0; i < V; ++i) sum[i] += w * v[i];
      }
      if (residual) {
        float r[V];
        load_some(residual + row * residual_stride + col, count, 0.f, r);
#pragma unroll
        for (int i = 0; i < V; ++i) sum[i] += r[i];
      }
      store_some(y + row * y_stride + col, count, sum);
    }
  }
}

template <typename T, int TEAM>
__global__ __launch_bounds__(256) void k_combine_back(int n, int d, int top, const T* __restrict__ dy, int64_t dy_stride, int rows,
                                                      const T* ys, int64_t ys_stride, const int32_t* __restrict__ place,
                                                      const float* __restrict__ weight, T* dys, int64_t dys_stride,
                                                      float* __restrict__ dweight, uint32_t* err) {
  constexpr int V = kPiece<T>, ROWS = 256 / TEAM;
  const int t = threadIdx.x % TEAM, team = threadIdx.x / TEAM;
  for (int64_t row = (int64_t)blockIdx.x * ROWS + team; row < n; row += (int64_t)gridDim.x * ROWS) {
    for (int j = 0; j < top; ++j) {
      const int p = place_of(place, row * top + j, rows, err, t == 0);
      const float w = weight ? weight[row * top + j] : 1.f;
      float dot = 0.f;
      if (p >= 0)
        for (int64_t col = t * V; col < d; col += TEAM * V) {
          const int count = (int)min((int64_t)V, d - col);
          float g[V], v[V];
          load_some(dy + row * dy_stride + col, count, 0.f, g);
          if (dweight) {
            load_some(ys + p * ys_stride + col, count, 0.f, v);
#pragma unroll
            for (int i = 0; i < V; ++i) dot += g[i] * v[i];
          }
          if (dys) {
#pragma unroll
            for (int i = 0; i < V; ++i) g[i] *= w;
            store_some(dys + p * dys_stride + col, count, g);
          }
        }
      if (dweight) {
        dot = team_sum<TEAM>(dot, nullptr);
        if (t == 0) dweight[row * top + j] = dot;
      }
    }
  }
}

}  // namespace sp
