// Softmax cross entropy over each application's own classes, and the gradient of the logits.
//   lse = log sum_{c < C} exp z_c,  loss = w (lse - z_label),  dz_c = scale w (exp(z_c - lse) - [c = label]),  0 for c >= C
// One pass: a row's team of lanes keeps it in registers, subtracts the row's maximum, and writes loss and gradient.  Rows wider
// than a workgroup's registers are read twice, with a running maximum and sum.  Bound by memory.
#pragma once
#include "sp_ops_common.h"

namespace sp {

// What there is to know about a row.  Loaded in two steps, since the second hangs on the first: a team asks for its next row's while it
// works on the one before (three trips to memory one after the other for every row otherwise: 60000 bfloat16 rows of 4000 classes
// 261 us, so 208 us).
struct LossRow {
  const int32_t *app, *n_classes, *label;
  const float* weight;
  int n, c_max, n_apps;

  int a, classes, y;                              // classes 0: the row is not counted (no label, bad data, or no row)
  float w;
  __device__ __forceinline__ void ask(int64_t row) {
    const bool in = row < n;
    a = in && app ? app[row] : 0;
    y = in ? label[row] : -1;
    w = in && weight ? weight[row] : 1.f;
  }
  __device__ __forceinline__ void ask_classes() {
    classes = c_max;
    if (app) classes = a >= 0 && a < n_apps ? n_classes[a] : -1;
  }
  __device__ __forceinline__ void settle(uint32_t* err, bool report) {
    uint32_t bad = 0;
    if (a < 0 || (app && a >= n_apps)) bad = kErrAppId;
    else if (classes < 1 || classes > c_max) bad = kErrClassCount;
    else if (y < -1 || y >= classes) bad = kErrLabel;
    if (bad && report) atomicOr(err, bad);
    if (bad || y < 0) classes = 0;
  }
};

// A value's load has ended here.
__device__ __forceinline__ void here(const float& v) { asm volatile("" : : "v"(v)); }

// exp(d) for d <= 0, as 2 to the power of d log2(e).  The product's rounding makes the result's relative error |d| half steps larger, which
// the rounding of the difference d has done already; what an error of that size leaves of a class far below the top does not count
// against the sum.  (The library's expf is exact to a step and takes five times the instructions, which is what bounds bfloat16 rows.)
// NaN stays NaN, -inf gives 0.
__device__ __forceinline__ float exp_of(float d) { return __builtin_amdgcn_exp2f(d * 1.44269504f); }

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
  const int64_t step = (int64_t)gridDim.x * ROWS;
  LossRow next{app, n_classes, label, weight, n, c_max, n_apps};
  next.ask((int64_t)blockIdx.x * ROWS + team);
  next.ask_classes();
  for (int64_t row = (int64_t)blockIdx.x * ROWS + team; row < n; row += step) {
    LossRow r = next;
    r.settle(err, t == 0);
    const float at_label = r.classes ? to_float(z[row * z_stride + r.y]) : 0.f;
    float v[C][V];
    float top = -INFINITY;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int col = (c * TEAM + t) * V;
      load_some(z + row * z_stride + col, r.classes - col, -INFINITY, v[c]);
    }
    next.ask(row + step);
    here(at_label);                               // before any lane writes a gradient into the logits' place
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < V; ++i) top = fmaxf(top, v[c][i]);
    top = team_max<TEAM>(top, red[0]);
    next.ask_classes();
    const float from = top == -INFINITY ? 0.f : top;
    float s = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        v[c][i] = exp_of(v[c][i] - from);
        s += v[c][i];
      }
    s = team_sum<TEAM>(s, red[1]);
    const bool none = s == 0.f;                   // not counted, or all logits are -inf: nothing to learn from the row
    if (t == 0) loss[row] = none ? 0.f : r.w * (logf(s) + (from - at_label));
    if (dz) {
      const float by = none ? 0.f : r.w * scale, per = none ? 0.f : by / s;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int col = (c * TEAM + t) * V;
#pragma unroll
        for (int i = 0; i < V; ++i) v[c][i] *= per;
        if ((unsigned)(r.y - col) < (unsigned)V) {
#pragma unroll
          for (int i = 0; i < V; ++i) v[c][i] -= col + i == r.y ? by : 0.f;
        }
        store_some(dz + row * dz_stride + col, c_max - col, v[c]);
      }
    }
  }
}

// Rows of any width: one workgroup to a row.  Columns are counted without a sign: the last step of a row of close to 2^31 classes ends
// behind 2^31 - 1.
template <typename T, typename TO>
__global__ __launch_bounds__(1024) void k_loss_wide(int n, int c_max, const T* z, int64_t z_stride, int n_apps,
                                                    const int32_t* __restrict__ app, const int32_t* __restrict__ n_classes,
                                                    const int32_t* __restrict__ label, const float* __restrict__ weight, float scale,
                                                    float* __restrict__ loss, TO* dz, int64_t dz_stride, uint32_t* err) {
  constexpr int V = kPiece<T>, TEAM = 1024;
  __shared__ float red[2][TEAM / 64];
  const int t = threadIdx.x;
  for (int64_t row = blockIdx.x; row < n; row += gridDim.x) {
    LossRow r{app, n_classes, label, weight, n, c_max, n_apps};
    r.ask(row);
    r.ask_classes();
    r.settle(err, t == 0);
    const float at_label = r.classes ? to_float(z[row * z_stride + r.y]) : 0.f;
    here(at_label);                               // before any lane writes a gradient into the logits' place
    float top = -INFINITY, s = 0.f;
    for (uint32_t col = t * V; col < (uint32_t)r.classes; col += TEAM * V) {
      float v[V];
      load_some(z + row * z_stride + col, (int)(r.classes - col), -INFINITY, v);
      float m = top;
#pragma unroll
      for (int i = 0; i < V; ++i) m = fmaxf(m, v[i]);
      if (m > top) s *= exp_of(top - m);
      top = m;
#pragma unroll
      for (int i = 0; i < V; ++i) s += exp_of(v[i] - (m == -INFINITY ? 0.f : m));
    }
    const float all = team_max<TEAM>(top, red[0]);
    const float from = all == -INFINITY ? 0.f : all;
    s = team_sum<TEAM>(all == -INFINITY ? s : s * exp_of(top - all), red[1]);
    const bool none = s == 0.f;
    if (t == 0) loss[row] = none ? 0.f : r.w * (logf(s) + (from - at_label));
    if (dz) {
      const float by = none ? 0.f : r.w * scale, per = none ? 0.f : by / s;
      for (uint32_t col = t * V; col < (uint32_t)c_max; col += TEAM * V) {
        float v[V];
        load_some(z + row * z_stride + col, (int)(r.classes - col), -INFINITY, v);
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = none ? 0.f : exp_of(v[i] - from) * per - (col + i == (uint32_t)r.y ? by : 0.f);
        store_some(dz + row * dz_stride + col, (int)(c_max - col), v);
      }
    }
    __syncthreads();                              // red is free for the next row
  }
}

}  // namespace sp
