// Grouped linear layers for few rows: a request, a window of them, a small batch, where a call's time is that of a few trips to memory
// and tiles of 128 rows would leave most of the device idle.  A workgroup takes 16 rows of one group and 32 (dx: 16) columns, and its
// wavefronts share out the depth, 32 at a time: each has its own reads under way, none waits for another, and their sums meet in LDS
// at the end.  Bound by the trips: offsets, weights and rows, the result.
#pragma once
#include "sp_ops_linear.h"

namespace sp {

constexpr int kFewRows = 16, kFewCols = 32, kFewThreads = 512;
constexpr int kFewDxCols = 16, kFewDxThreads = 256;

// Eight elements of the depth of one row, in memory's form and as the matrix cores take them.
template <typename T>
struct DepthPiece {
  float v[8];
  __device__ __forceinline__ void load(const T* p, int count) {
    constexpr int V = kPiece<T>;
#pragma unroll
    for (int h = 0; h < 8; h += V) {
      float e[V];
      load_some(p + h, count - h, 0.f, e);
#pragma unroll
      for (int i = 0; i < V; ++i) v[h + i] = e[i];
    }
  }
  __device__ __forceinline__ void fragment(bf16x8 (&out)[kPlanes<T>]) {
#pragma unroll
    for (int pl = 0; pl < kPlanes<T>; ++pl)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        out[pl][i] = (bf16)v[i];
        v[i] -= (float)out[pl][i];
      }
  }
};

template <int P>
__device__ __forceinline__ void multiply_16(f32x4& acc, const bf16x8 (&cols)[P], const bf16x8 (&rows)[P]) {
#pragma unroll
  for (int p = P - 1; p >= 0; --p)
#pragma unroll
    for (int q = P - 1 - p; q >= 0; --q) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(cols[q], rows[p], acc, 0, 0, 0);
}

// y.  A wavefront's 32 x 32 weights go through its own part of LDS, since a lane needs eight of one column: [plane][32 depth][32 columns].
template <typename T, typename TO>
__global__ __launch_bounds__(kFewThreads) void k_linear_few(LinearArgs a) {
  constexpr int V = kPiece<T>, P = kPlanes<T>, WAVES = kFewThreads / 64, BN = kFewCols;
  constexpr int kAcross = BN / V, kStep = 64 / kAcross, kPieces = 32 / kStep;         // a lane's pieces of the weights
  __shared__ __align__(16) uint16_t lds[WAVES][P * 32 * BN];
  __shared__ float part[WAVES][kFewRows * (BN + 1)];
  if (blockIdx.x == 0 && threadIdx.x < 64) check_offsets(a.offsets, a.groups, a.n, a.err);
  const int tile = xcd_tile(blockIdx.x, a.row_tiles * a.col_tiles);
  if (tile < 0) return;
  const int rt = tile / a.col_tiles, c0 = (tile % a.col_tiles) * BN;
  RowTile rows;
  if (!find_row_tile(a.offsets, a.groups, a.n, kFewRows, rt, &rows)) return;
  const int n_rows = rows.hi - rows.lo, depth = rows.g < a.groups ? a.k : 0;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, mine = lane & 15, quarter = lane >> 4;
  const int major = lane / kAcross, minor = (lane % kAcross) * V, left = a.m - c0 - minor;
  const T* w = (const T*)a.w + ((int64_t)min(rows.g, a.groups - 1) * a.k + major) * a.m + c0 + minor;
  const T* x = (const T*)a.x + ((int64_t)rows.lo + mine) * a.x_stride + 8 * quarter;
  const bool has_row = mine < n_rows;
  uint16_t* own = lds[wave];

  float wv[kPieces][V];
  DepthPiece<T> xv;
  auto load = [&](int t0) {
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int t = t0 + i * kStep;
      load_some(w + (int64_t)t * a.m, t + major < depth ? left : 0, 0.f, wv[i]);
    }
    xv.load(x + t0, has_row ? depth - t0 - 8 * quarter : 0);
  };
  f32x4 acc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
  int t0 = wave * 32;
  if (t0 < depth) load(t0);
  for (; t0 < depth; t0 += WAVES * 32) {
#pragma unroll
    for (int i = 0; i < kPieces; ++i)
#pragma unroll
      for (int p = 0; p < P; ++p) {
        uint16_t* at = own + (p * 32 + major + i * kStep) * BN + minor;
        uint32_t h[V / 2];
#pragma unroll
        for (int j = 0; j < V / 2; ++j) {
          h[j] = pack_bf16(wv[i][2 * j], wv[i][2 * j + 1]);
          wv[i][2 * j] -= low_bf16(h[j]);
          wv[i][2 * j + 1] -= high_bf16(h[j]);
        }
        if constexpr (V == 8) *reinterpret_cast<u32x4*>(at) = u32x4{h[0], h[1], h[2], h[3]};
        else *reinterpret_cast<u32x2*>(at) = u32x2{h[0], h[1]};
      }
    bf16x8 fr[P];
    xv.fragment(fr);
    if (t0 + WAVES * 32 < depth) load(t0 + WAVES * 32);
    wave_sync();
    typedef __attribute__((address_space(3))) s16x4* lds_ptr;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      bf16x8 fc[P];
#pragma unroll
      for (int p = 0; p < P; ++p) {
        uint16_t* at = own + (p * 32 + 8 * quarter + mine / 4) * BN + j * 16 + 4 * (mine & 3);
        union { s16x4 h[2]; bf16x8 v; } u;
        u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)at);
        u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(at + 4 * BN));
        fc[p] = u.v;
      }
      multiply_16<P>(acc[j], fc, fr);
    }
    wave_sync();
  }
  // lane l has row l % 16, columns 4 (l / 16) .. + 3 of each half
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) part[wave][mine * (BN + 1) + j * 16 + 4 * quarter + e] = acc[j][e];
  __syncthreads();
  const int r = threadIdx.x / BN, col = c0 + threadIdx.x % BN;
  static_assert(kFewThreads == kFewRows * BN, "a result to a thread");
  if (r >= n_rows || col >= a.m) return;
  float v = 0.f;
#pragma unroll
  for (int q = 0; q < WAVES; ++q) v += part[q][r * (BN + 1) + threadIdx.x % BN];
  const int64_t row = rows.lo + r;
  const bool in = rows.g < a.groups;
  if (in && a.bias) v += a.bias[(int64_t)rows.g * a.m + col];
  if (a.relu) v = relu_of(v);
  if (a.act) ((TO*)a.act)[row * a.act_stride + col] = from_float<TO>(v);
  if (in && a.residual) v += to_float(((const TO*)a.residual)[row * a.residual_stride + col]);
  ((TO*)a.y)[row * a.y_stride + col] = from_float<TO>(v);
}

// dx: rows of weights are contiguous along the depth, so that both sides' fragments come straight from memory.
template <typename T>
__device__ __forceinline__ void linear_few_dx(const LinearArgs& a, int block) {
  constexpr int P = kPlanes<T>, WAVES = kFewDxThreads / 64;
  __shared__ float part[WAVES][16 * 17];
  if (block == 0 && threadIdx.x < 64) check_offsets(a.offsets, a.groups, a.n, a.err);
  const int tile = xcd_tile(block, a.row_tiles * a.col_tiles);
  if (tile < 0) return;
  const int rt = tile / a.col_tiles, c0 = (tile % a.col_tiles) * kFewDxCols;
  RowTile rows;
  if (!find_row_tile(a.offsets, a.groups, a.n, kFewRows, rt, &rows)) return;
  const int n_rows = rows.hi - rows.lo, depth = rows.g < a.groups ? a.m : 0;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, mine = lane & 15, t_own = 8 * (lane >> 4);
  const T* w = (const T*)a.w + ((int64_t)min(rows.g, a.groups - 1) * a.k + c0 + mine) * a.m;
  const T* dy = (const T*)a.dy + ((int64_t)rows.lo + mine) * a.dy_stride;
  const T* act = a.act ? (const T*)a.act + ((int64_t)rows.lo + mine) * a.act_stride : nullptr;
  const bool has_col = c0 + mine < a.k, has_row = mine < n_rows;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int t0 = wave * 32; t0 < depth; t0 += WAVES * 32) {
    const int t = t0 + t_own, count = depth - t;
    DepthPiece<T> pc, pr, pa;
    pc.load(w + t, has_col ? count : 0);
    pr.load(dy + t, has_row ? count : 0);
    if (act) {
      pa.load(act + t, has_row ? count : 0);
#pragma unroll
      for (int i = 0; i < 8; ++i) pr.v[i] = pa.v[i] > 0.f ? pr.v[i] : 0.f;
    }
    bf16x8 fc[P], fr[P];
    pc.fragment(fc);
    pr.fragment(fr);
    multiply_16<P>(acc, fc, fr);
  }
  // lane l has row l % 16, columns 4 (l / 16) .. + 3
#pragma unroll
  for (int e = 0; e < 4; ++e) part[wave][mine * 17 + 4 * (lane >> 4) + e] = acc[e];
  __syncthreads();
  const int r = threadIdx.x / 16, col = threadIdx.x % 16;
  if (r >= n_rows || c0 + col >= a.k) return;
  float v = 0.f;
#pragma unroll
  for (int q = 0; q < WAVES; ++q) v += part[q][r * 17 + col];
  ((T*)a.dx)[((int64_t)rows.lo + r) * a.dx_stride + c0 + col] = from_float<T>(v);
}

template <typename T>
__global__ __launch_bounds__(kFewDxThreads) void k_linear_few_dx(LinearArgs a) {
  linear_few_dx<T>(a, blockIdx.x);
}

// A small layer's dx and dW in one launch, where the device holds about all of dW's workgroups at once: the first dw_blocks are dW's, whose way
// through the rows is the longer one, and dx's run beside and behind them.
// (12 rows of 7 applications, 479 x 113 float32: 11.2 -> 7.9 us a call, of which the second launch costs the host 2;
// 3000 rows of 3, 64 x 64 bfloat16: 11.3 -> 8.6; 2048 rows of 8, 256 x 256 float32 with a mask: 34 -> 30.)
template <typename T, int BM, int BN, bool MASK>
__global__ __launch_bounds__(kFewDxThreads, 2) void k_linear_few_back(LinearArgs dx, LinearArgs dw, int dw_blocks) {
  if ((int)blockIdx.x < dw_blocks) linear_tile<T, float, kFormDw, BM, BN, MASK, kFewDxThreads>(dw, blockIdx.x);
  else linear_few_dx<T>(dx, (int)blockIdx.x - dw_blocks);
}

}  // namespace sp
