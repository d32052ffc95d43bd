// Rows on their way to the experts and back.
//   dispatch       xs[place_ij] = x_i
//   combine        y_i = sum over j of w_ij ys[place_ij] + r_i
//   its gradients  dys[place_ij] = w_ij dy_i        dw_ij = dy_i . ys[place_ij]
// A team of lanes takes a row of x, y or dy; the rows at the places are whole rows somewhere else, so that every access is a run of
// 16-byte pieces.  Bound by memory: 65536 x 512 bfloat16 to 4 places each 68 us (5.0 TB/s), 65536 x 256 float32 of 2 places and a residual 51
// (5.3), the gradients of 32768 x 768 bfloat16 with 8 places each 169 (4.9).
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

// Up to AT of a row's pairs: their places and weights, and the pieces at the places, which are on their way together.  (As many as the row has up to 8: 32768
// rows of 768 bfloat16 with 8 pairs 97 us, with each read behind the one before 127.)
template <int AT>
struct Pairs {
  int p[AT];
  float w[AT];
  __device__ __forceinline__ Pairs(const int32_t* __restrict__ place, const float* __restrict__ weight, int64_t row, int first, int top, int rows,
                                   uint32_t* err, bool report) {
#pragma unroll
    for (int u = 0; u < AT; ++u) {
      const int64_t pair = row * top + min(first + u, top - 1);
      p[u] = place_of(place, pair, rows, err, report);
      w[u] = weight ? weight[pair] : 1.f;
      if (first + u >= top) p[u] = -1;
    }
  }
  // (a pair without a place reads the first row, and does not count)
  template <typename T>
  __device__ __forceinline__ void load(const T* ys, int64_t stride, int col, int d, raw_piece (&v)[AT]) const {
#pragma unroll
    for (int u = 0; u < AT; ++u) v[u] = load_raw_piece(ys + max(p[u], 0) * stride, col, d);
  }
};

template <typename T, int TEAM, int AT>
__global__ __launch_bounds__(256) void k_dispatch(int n, int d, int top, const T* __restrict__ x, int64_t x_stride,
                                                  const int32_t* __restrict__ place, int rows, T* __restrict__ xs, int64_t xs_stride,
                                                  uint32_t* err) {
  constexpr int V = kPiece<T>, ROWS = 256 / TEAM;
  const int t = threadIdx.x % TEAM, team = threadIdx.x / TEAM;
  for (int64_t row = (int64_t)blockIdx.x * ROWS + team; row < n; row += (int64_t)gridDim.x * ROWS) {
    for (int j = 0; j < top; j += AT) {
      const Pairs<AT> q(place, nullptr, row, j, top, rows, err, t == 0);
      for (int col = t * V; col < d; col += TEAM * V) {
        float v[V];
        load_some(x + row * x_stride + col, d - col, 0.f, v);
#pragma unroll
        for (int u = 0; u < AT; ++u)
          if (q.p[u] >= 0) store_some(xs + q.p[u] * xs_stride + col, d - col, v);
      }
    }
  }
}

template <typename T, int TEAM, int AT>
__global__ __launch_bounds__(256) void k_combine(int n, int d, int top, int rows, const T* __restrict__ ys, int64_t ys_stride,
                                                 const int32_t* __restrict__ place, const float* __restrict__ weight, const T* residual,
                                                 int64_t residual_stride, T* y, int64_t y_stride, uint32_t* err) {
  constexpr int V = kPiece<T>, ROWS = 256 / TEAM;
  const int t = threadIdx.x % TEAM, team = threadIdx.x / TEAM;
  for (int64_t row = (int64_t)blockIdx.x * ROWS + team; row < n; row += (int64_t)gridDim.x * ROWS) {
    const Pairs<AT> first(place, weight, row, 0, top, rows, err, t == 0);
    for (int col = t * V; col < d; col += TEAM * V) {
      float sum[V] = {};
      raw_piece r;
      if (residual) r = load_raw_piece(residual + row * residual_stride, col, d);
      auto add = [&](const Pairs<AT>& q) {
        raw_piece v[AT];
        q.load(ys, ys_stride, col, d, v);
#pragma unroll
        for (int u = 0; u < AT; ++u)
#pragma unroll
          for (int i = 0; i < V; ++i) sum[i] += q.p[u] >= 0 ? q.w[u] * of_raw((const T*)nullptr, v[u], i) : 0.f;
      };
      if (rows > 0) add(first);                                       // (no rows: no pair has a place)
      for (int j = AT; j < top && rows > 0; j += AT) add(Pairs<AT>(place, weight, row, j, top, rows, err, t == 0));
      if (residual) {
#pragma unroll
        for (int i = 0; i < V; ++i) sum[i] += of_raw((const T*)nullptr, r, i);
      }
      store_some(y + row * y_stride + col, d - col, sum);
    }
  }
}

// dys may lie where ys does: a lane reads its piece of a row before it writes it, and nobody else reads that (a pair without a place reads what it
// does not use).
template <typename T, int TEAM, int AT>
__global__ __launch_bounds__(256) void k_combine_back(int n, int d, int top, const T* __restrict__ dy, int64_t dy_stride, int rows,
                                                      const T* ys, int64_t ys_stride, const int32_t* __restrict__ place,
                                                      const float* __restrict__ weight, T* dys, int64_t dys_stride,
                                                      float* __restrict__ dweight, uint32_t* err) {
  constexpr int V = kPiece<T>, ROWS = 256 / TEAM;
  const int t = threadIdx.x % TEAM, team = threadIdx.x / TEAM;
  for (int64_t row = (int64_t)blockIdx.x * ROWS + team; row < n; row += (int64_t)gridDim.x * ROWS) {
    for (int j = 0; j < top; j += AT) {
      const Pairs<AT> q(place, weight, row, j, top, rows, err, t == 0);
      float dot[AT] = {};
      for (int col = t * V; col < d; col += TEAM * V) {
        const raw_piece raw = load_raw_piece(dy + row * dy_stride, col, d);
        raw_piece v[AT];
        if (dweight && rows > 0) {
          q.load(ys, ys_stride, col, d, v);
        } else {
#pragma unroll
          for (int u = 0; u < AT; ++u) v[u] = raw_piece{0, 0, 0, 0};
        }
        float g[V];
#pragma unroll
        for (int i = 0; i < V; ++i) g[i] = of_raw((const T*)nullptr, raw, i);
        if (dweight) {
#pragma unroll
          for (int u = 0; u < AT; ++u)
#pragma unroll
            for (int i = 0; i < V; ++i) dot[u] += g[i] * of_raw((const T*)nullptr, v[u], i);
        }
        if (dys) {
#pragma unroll
          for (int u = 0; u < AT; ++u)
            if (q.p[u] >= 0) {
              float o[V];
#pragma unroll
              for (int i = 0; i < V; ++i) o[i] = g[i] * q.w[u];
              store_some(dys + q.p[u] * dys_stride + col, d - col, o);
            }
        }
      }
      if (dweight) {
#pragma unroll
        for (int u = 0; u < AT; ++u) {
          const float s = team_sum<TEAM>(dot[u], nullptr);
          if (t == 0 && j + u < top) dweight[row * top + j + u] = q.p[u] >= 0 ? s : 0.f;
        }
      }
    }
  }
}

}  // namespace sp
