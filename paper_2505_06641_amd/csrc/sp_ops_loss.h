// Softmax cross entropy over each application's own classes, and the gradient of the logits.
//   lse = log sum_{c < C} exp z_c,  loss = w (lse - z_label),  dz_c = scale w (exp(z_c - lse) - [c = label]),  0 for c >= C
// One pass: a row's team of lanes keeps it in registers, subtracts the row's maximum, and writes loss and gradient.  Rows wider
// than a workgroup's registers are read twice, with a running maximum and sum.  Bound by memory.
#pragma once
#include "sp_ops_common.h"

namespace sp {

struct LossRow {
  int classes, label;       // classes 0: the row is not counted (no label, or bad data)
  float w;
};
__device__ __forceinline__ LossRow loss_row(int64_t row, int c_max, int n_apps, const int32_t* app, const int32_t* n_classes,
                                            const int32_t* label, const float* weight, uint32_t* err, bool report) {
  LossRow r;
  r.classes = c_max;
  uint32_t bad = 0;
  if (app) {
    const int a = app[row];
    if (a < 0 || a >= n_apps) {
      bad = kErrAppId;
    } else {
      r.classes = n_classes[a];
      if (r.classes < 1 || r.classes > c_max) bad = kErrClassCount;
    }
  }
  r.label = label[row];
  if (!bad && (r.label < -1 || r.label >= r.classes)) bad = kErrLabel;
  if (bad && report) atomicOr(err, bad);
  if (bad || r.label < 0) r.classes = 0;
  r.w = weight ? weight[row] : 1.f;
  return r;
}

// A value's load has ended here.
__device__ __forceinline__ void here(const float& v) { asm volatile("" : : "v"(v)); }

constexpr int kLossBlocks = 4096;

template <typename T, typename TO, int TEAM, int C>
__global__ __launch_bounds__(kTeamThreads<TEAM>) void k_loss(int n, int c_max, const T* z, int64_t z_stride, int n_apps,
                                                             const int32_t* __restrict__ app, const int32_t* __restrict__ n_classes,
                                                             const int32_t* __restrict__ label, const float* __restrict__ weight,
                                                             float scale, float* __restrict__ loss, TO* dz, int64_t dz_stride,
                                                             uint32_t* err) {
  constexpr int V = kPiece<T>, ROWS = kTeamThreads<TEAM> / TEAM;
  __shared__ float red[2][TEAM > 64 ? TEAM / 64 : 1];
  const int t = threadIdx.x % TEAM, team = threadIdx.x / TEAM;
  for (int64_t row = (int64_t)blockIdx.x * ROWS + team; row < n; row += (int64_t)gridDim.x * ROWS) {
    const LossRow r = loss_row(row, c_max, n_apps, app, n_classes, label, weight, err, t == 0);
    const float at_label = r.classes ? to_float(z[row * z_stride + r.label]) : 0.f;
    here(at_label);                               // before any lane writes a gradient into the logits' place
    float v[C][V];
    float top = -INFINITY;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int col = (c * TEAM + t) * V;
      load_some(z + row * z_stride + col, r.classes - col, -INFINITY, v[c]);
#pragma unroll
      for (int i = 0; i < V; ++i) top = fmaxf(top, v[c][i]);
    }
    top = team_max<TEAM>(top, red[0]);
    const float from = top == -INFINITY ? 0.f : top;
    float s = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        v[c][i] = expf(v[c][i] - from);
        s += v[c][i];
      }
    s = team_sum<TEAM>(s, red[1]);
    const bool none = s == 0.f;                   // not counted, or all logits are -inf: nothing to learn from the row
    if (t == 0) loss[row] = none ? 0.f : r.w * (logf(s) + (from - at_label));
    if (dz) {
      const float per = none ? 0.f : 1.f / s, by = none ? 0.f : r.w * scale;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int col = (c * TEAM + t) * V;
#pragma unroll
        for (int i = 0; i < V; ++i) v[c][i] = (v[c][i] * per - (col + i == r.label ? 1.f : 0.f)) * by;
        store_some(dz + row * dz_stride + col, c_max - col, v[c]);
      }
    }
  }
}

// Rows of any width: one workgroup to a row.
template <typename T, typename TO>
__global__ __launch_bounds__(1024) void k_loss_wide(int n, int c_max, const T* z, int64_t z_stride, int n_apps,
                                                    const int32_t* __restrict__ app, const int32_t* __restrict__ n_classes,
                                                    const int32_t* __restrict__ label, const float* __restrict__ weight, float scale,
                                                    float* __restrict__ loss, TO* dz, int64_t dz_stride, uint32_t* err) {
  constexpr int V = kPiece<T>, TEAM = 1024;
  __shared__ float red[2][TEAM / 64];
  const int t = threadIdx.x;
  for (int64_t row = blockIdx.x; row < n; row += gridDim.x) {
    const LossRow r = loss_row(row, c_max, n_apps, app, n_classes, label, weight, err, t == 0);
    const float at_label = r.classes ? to_float(z[row * z_stride + r.label]) : 0.f;
    here(at_label);                               // before any lane writes a gradient into the logits' place
    float top = -INFINITY, s = 0.f;
    for (int col = t * V; col < r.classes; col += TEAM * V) {
      float v[V];
      load_some(z + row * z_stride + col, r.classes - col, -INFINITY, v);
      float m = top;
#pragma unroll
      for (int i = 0; i < V; ++i) m = fmaxf(m, v[i]);
      if (m > top) s *= expf(top - m);
      top = m;
#pragma unroll
      for (int i = 0; i < V; ++i) s += expf(v[i] - (m == -INFINITY ? 0.f : m));
    }
    const float all = team_max<TEAM>(top, red[0]);
    const float from = all == -INFINITY ? 0.f : all;
    s = team_sum<TEAM>(all == -INFINITY ? s : s * expf(top - all), red[1]);
    const bool none = s == 0.f;
    if (t == 0) loss[row] = none ? 0.f : r.w * (logf(s) + (from - at_label));
    if (dz) {
      const float per = none ? 0.f : 1.f / s, by = none ? 0.f : r.w * scale;
      for (int col = t * V; col < c_max; col += TEAM * V) {
        float v[V];
        load_some(z + row * z_stride + col, r.classes - col, -INFINITY, v);
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = none ? 0.f : (expf(v[i] - from) * per - (col + i == r.label ? 1.f : 0.f)) * by;
        store_some(dz + row * dz_stride + col, c_max - col, v);
      }
    }
    __syncthreads();                              // red is free for the next row
  }
}

}  // namespace sp
