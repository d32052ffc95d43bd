// Linear layers of rows that are grouped by application, and their gradients.
//   y_i = act(x_i W_g + b_g) + r_i      dx_i = dz_i W_g^T      dW_g = sum over the group's rows x_i^T dz_i      db_g = sum dz_i
// with dz = dy where the activation passed something, 0 elsewhere.
#pragma once
#include "sp_ops_common.h"

namespace sp {

struct LinearArgs {
  int n, k, m, groups;
  const void* x;  int64_t x_stride;      // [n, k]
  const int32_t* offsets;                // [groups + 1]
  const void* w;                         // [groups, k, m]
  const float* bias;                     // [groups, m] or null
  int relu;
  const void* residual;  int64_t residual_stride;   // [n, m] or null
  void* y;  int64_t y_stride;            // [n, m]
  void* act;  int64_t act_stride;        // [n, m] or null: forward writes act(..), backward reads where it is positive
  const void* dy;  int64_t dy_stride;    // [n, m]
  void* dx;  int64_t dx_stride;          // [n, k] or null
  float* dw;                             // [groups, k, m] or null
  float* db;                             // [groups, m] or null
  uint32_t* err;
};

constexpr int kSimpleTile = 64, kSimpleDepth = 16;

// Where NaN has to stay NaN: only what is below 0 becomes 0.
__device__ __forceinline__ float relu_of(float z) { return z < 0.f ? 0.f : z; }

template <typename T>
__device__ __forceinline__ float dz_at(const LinearArgs& a, int64_t row, int col) {
  const float g = to_float(((const T*)a.dy)[row * a.dy_stride + col]);
  if (!a.act) return g;
  return to_float(((const T*)a.act)[row * a.act_stride + col]) <= 0.f ? 0.f : g;
}

// One 64 x 64 tile of a product a workgroup, operands staged through LDS, float32 multiply-adds.
// FORM 0: y, 1: dx, 2: dW.
template <typename T, typename TO, int FORM>
__global__ __launch_bounds__(256) void k_linear_simple(LinearArgs a) {
  __shared__ float A[kSimpleDepth][kSimpleTile + 1], B[kSimpleDepth][kSimpleTile + 1];
  RowTile rt;
  int depth, r0, c0, rows, cols;
  const int width = FORM == 1 ? a.k : a.m;
  if (blockIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0 && threadIdx.x < 64) check_offsets(a.offsets, a.groups, a.n, a.err);
  if (FORM == 2) {
    rt.g = blockIdx.z;
    group_rows(a.offsets, a.n, rt.g, &rt.lo, &rt.hi);
    depth = rt.hi - rt.lo;
    r0 = blockIdx.x * kSimpleTile;
    rows = min(kSimpleTile, a.k - r0);
  } else {
    if (!find_row_tile<kSimpleTile>(a.offsets, a.groups, a.n, blockIdx.x, &rt)) return;
    depth = rt.g < a.groups ? (FORM == 0 ? a.k : a.m) : 0;
    r0 = rt.lo;
    rows = rt.hi - rt.lo;
  }
  c0 = blockIdx.y * kSimpleTile;
  cols = min(kSimpleTile, width - c0);
  const T* w = (const T*)a.w + (int64_t)rt.g * a.k * a.m;
  const T* x = (const T*)a.x;
  float acc[4][4] = {};
  const int tr = threadIdx.x / 16, tc = threadIdx.x % 16;
  for (int t0 = 0; t0 < depth; t0 += kSimpleDepth) {
    for (int i = threadIdx.x; i < kSimpleTile * kSimpleDepth; i += 256) {
      if (FORM == 2) {
        const int t = i / kSimpleTile, r = i % kSimpleTile;
        const bool in = t0 + t < depth;
        const int64_t row = rt.lo + t0 + t;
        A[t][r] = in && r < rows ? to_float(x[row * a.x_stride + r0 + r]) : 0.f;
        B[t][r] = in && r < cols ? dz_at<T>(a, row, c0 + r) : 0.f;
      } else {
        const int r = i / kSimpleDepth, t = i % kSimpleDepth;
        const int64_t row = r0 + r;
        const bool in = t0 + t < depth;
        A[t][r] = in && r < rows ? (FORM == 0 ? to_float(x[row * a.x_stride + t0 + t]) : dz_at<T>(a, row, t0 + t)) : 0.f;
        if (FORM == 0) {
          const int t2 = i / kSimpleTile, c = i % kSimpleTile;
          B[t2][c] = t0 + t2 < depth && c < cols ? to_float(w[(int64_t)(t0 + t2) * a.m + c0 + c]) : 0.f;
        } else {
          B[t][r] = in && r < cols ? to_float(w[(int64_t)(c0 + r) * a.m + t0 + t]) : 0.f;
        }
      }
    }
    __syncthreads();
    for (int t = 0; t < kSimpleDepth; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] += A[t][tr * 4 + i] * B[t][tc + 16 * j];
    __syncthreads();
  }
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) {
      const int r = tr * 4 + i, c = tc + 16 * j;
      if (r >= rows || c >= cols) continue;
      float v = acc[i][j];
      const int64_t row = r0 + r;
      if (FORM == 2) {
        a.dw[((int64_t)rt.g * a.k + row) * a.m + c0 + c] = v;
      } else if (FORM == 1) {
        ((TO*)a.dx)[row * a.dx_stride + c0 + c] = from_float<TO>(v);
      } else {
        const bool in = rt.g < a.groups;
        if (in && a.bias) v += a.bias[(int64_t)rt.g * a.m + c0 + c];
        if (a.relu) v = relu_of(v);
        if (a.act) ((TO*)a.act)[row * a.act_stride + c0 + c] = from_float<TO>(v);
        if (in && a.residual) v += to_float(((const TO*)a.residual)[row * a.residual_stride + c0 + c]);
        ((TO*)a.y)[row * a.y_stride + c0 + c] = from_float<TO>(v);
      }
    }
}

// db: 64 columns of one group to a workgroup, four rows at a time.
template <typename T>
__global__ __launch_bounds__(256) void k_bias_grad(LinearArgs a) {
  __shared__ float sums[4][64];
  int lo, hi;
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x < 64) check_offsets(a.offsets, a.groups, a.n, a.err);
  group_rows(a.offsets, a.n, blockIdx.y, &lo, &hi);
  const int lane = threadIdx.x % 64, slice = threadIdx.x / 64, col = blockIdx.x * 64 + lane;
  float s = 0.f;
  if (col < a.m)
    for (int row = lo + slice; row < hi; row += 4) s += dz_at<T>(a, row, col);
  sums[slice][lane] = s;
  __syncthreads();
  if (slice == 0 && col < a.m)
    a.db[(int64_t)blockIdx.y * a.m + col] = (sums[0][lane] + sums[1][lane]) + (sums[2][lane] + sums[3][lane]);
}

}  // namespace sp
