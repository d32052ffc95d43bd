// Grouped linear layers in 8 bits, for serving.
//   rows     scale_i = max_c |x_ic| / 127        q_ic = x_ic (127 / max_c |x_ic|), rounded to the nearest whole number, ties to even
//   layer    y_i = act(scale_i w_scale_go sum_c q_ic w_goc + b_go) + r_i, the sum in 32-bit integers: exact
// Weights lie with an output's inputs next to each other, [groups, m, k], so that both sides' 16 consecutive inputs are what a lane of the matrix
// cores takes.
#pragma once
#include "sp_common.h"
#include "sp_ops_common.h"

namespace sp {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t bytes16 __attribute__((ext_vector_type(4)));
typedef uint32_t bytes16_any __attribute__((ext_vector_type(4), aligned(1)));

// What turns a row into whole numbers.  Rows with an infinity or NaN become zeros with scale NaN, so that what is made of them is NaN.  Where
// 127 / high would overflow, the row is multiplied by 2^64 first, which is exact.
struct RowScale {
  float lift, by, scale;
  __device__ __forceinline__ explicit RowScale(float high, bool finite) {
    lift = high < 0x1p-60f ? 0x1p64f : 1.f;
    by = high > 0.f && finite ? 127.f / (high * lift) : 0.f;
    scale = finite ? high / 127.f : __builtin_nanf("");
  }
  __device__ __forceinline__ int of(float v) const { return by == 0.f ? 0 : (int)rintf(v * lift * by); }
};

template <int V>
__device__ __forceinline__ void store_bytes(int8_t* p, int count, const int (&q)[V]) {
  if (count >= V) {
    uint32_t w[V / 4];
#pragma unroll
    for (int i = 0; i < V / 4; ++i)
      w[i] = (q[4 * i] & 0xff) | (q[4 * i + 1] & 0xff) << 8 | (q[4 * i + 2] & 0xff) << 16 | (uint32_t)q[4 * i + 3] << 24;
    __builtin_memcpy(p, w, V);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i < count) p[i] = (int8_t)q[i];
  }
}

template <typename T, int TEAM, int C>
__global__ __launch_bounds__(kTeamThreads<TEAM>) void k_quantize(int n, int d, const T* __restrict__ x, int64_t x_stride, int8_t* __restrict__ q,
                                                                 int64_t q_stride, float* __restrict__ scale) {
  constexpr int V = kPiece<T>, ROWS = kTeamThreads<TEAM> / TEAM;
  __shared__ float red[2][TEAM > 64 ? TEAM / 64 : 1];
  const int t = threadIdx.x % TEAM, team = threadIdx.x / TEAM;
  int turn = 0;
  for (int64_t row = (int64_t)blockIdx.x * ROWS + team; row < n; row += (int64_t)gridDim.x * ROWS, turn ^= 1) {
    float v[C][V], high = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int col = (c * TEAM + t) * V;
      load_some(x + row * x_stride + col, d - col, 0.f, v[c]);
#pragma unroll
      for (int i = 0; i < V; ++i) high = !(fabsf(v[c][i]) < INFINITY) ? INFINITY : fmaxf(high, fabsf(v[c][i]));
    }
    high = team_max<TEAM>(high, red[turn]);
    const RowScale s(high, high < INFINITY);
    if (t == 0) scale[row] = s.scale;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int col = (c * TEAM + t) * V;
      int b[V];
#pragma unroll
      for (int i = 0; i < V; ++i) b[i] = s.of(v[c][i]);
      if (col < d) store_bytes(q + row * q_stride + col, d - col, b);
    }
  }
}

// Rows of any width: one workgroup to a row, which is read twice.
template <typename T>
__global__ __launch_bounds__(1024) void k_quantize_wide(int n, int d, const T* __restrict__ x, int64_t x_stride, int8_t* __restrict__ q,
                                                        int64_t q_stride, float* __restrict__ scale) {
  constexpr int V = kPiece<T>;
  __shared__ float red[2][16];
  int turn = 0;
  for (int64_t row = blockIdx.x; row < n; row += gridDim.x, turn ^= 1) {
    float high = 0.f;
    for (int col = threadIdx.x * V; col < d; col += 1024 * V) {
      float v[V];
      load_some(x + row * x_stride + col, d - col, 0.f, v);
#pragma unroll
      for (int i = 0; i < V; ++i) high = !(fabsf(v[i]) < INFINITY) ? INFINITY : fmaxf(high, fabsf(v[i]));
    }
    high = team_max<1024>(high, red[turn]);
    const RowScale s(high, high < INFINITY);
    if (threadIdx.x == 0) scale[row] = s.scale;
    for (int col = threadIdx.x * V; col < d; col += 1024 * V) {
      float v[V];
      int b[V];
      load_some(x + row * x_stride + col, d - col, 0.f, v);
#pragma unroll
      for (int i = 0; i < V; ++i) b[i] = s.of(v[i]);
      store_bytes(q + row * q_stride + col, d - col, b);
    }
  }
}

struct QuantizedArgs {
  int n, k, m, groups;
  const int8_t* x;  int64_t x_stride;            // [n, k]
  const float* x_scale;                          // [n]
  const int32_t* offsets;                        // [groups + 1]
  const int8_t* w;                               // [groups, m, k]
  const float* w_scale;                          // [groups, m]
  const float* bias;                             // [groups, m] or null
  int relu;
  const void* residual;  int64_t residual_stride;   // [n, m] or null
  void* y;  int64_t y_stride;                    // [n, m]
  uint32_t* err;
  int row_tiles, col_tiles;
};

// Sixteen bytes of a row of `depth` from `t` on; what lies behind the row is 0 (CUT), or whatever is there.  left: bytes from p to the
// array's end.
template <bool CUT>
__device__ __forceinline__ bytes16 load_bytes(const int8_t* p, int t, int depth, int64_t left) {
  if (t >= depth) return bytes16{0, 0, 0, 0};
  const int count = depth - t;
  if (count >= 16) return *reinterpret_cast<const bytes16_any*>(p);
  bytes16 q = {0, 0, 0, 0};
  if (left >= 16) {
    q = *reinterpret_cast<const bytes16_any*>(p);
    if (CUT) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int keep = count - 4 * i;
        q[i] = keep >= 4 ? q[i] : keep > 0 ? q[i] & ((1u << 8 * keep) - 1u) : 0u;
      }
    }
  } else {
#pragma unroll 1
    for (int i = count - 1; i >= 0; --i)
      q = bytes16{q[0] << 8 | (uint8_t)p[i], q[1] << 8 | q[0] >> 24, q[2] << 8 | q[1] >> 24, q[3] << 8 | q[2] >> 24};
  }
  return q;
}

// A tile of 128 rows of one group by 128 columns, four wavefronts of 64 by 64, 128 bytes of the depth at a time through LDS.  Rows and columns
// beyond the tile's last are that one again, and not written.
template <typename TO>
__global__ __launch_bounds__(256) void k_quantized(QuantizedArgs a) {
  constexpr int BM = 128, BN = 128, D = 128;
  __shared__ __align__(16) uint8_t lds[(BM + BN) * D];
  if (blockIdx.x == 0 && threadIdx.x < 64) check_offsets(a.offsets, a.groups, a.n, a.err);
  const int tile = xcd_tile(blockIdx.x, a.row_tiles * a.col_tiles);
  if (tile < 0) return;
  RowTile rows;
  const int rt = tile / a.col_tiles, c0 = (tile % a.col_tiles) * BN;
  if (!find_row_tile(a.offsets, a.groups, a.n, BM, rt, &rows)) return;
  const bool in = rows.g < a.groups;
  const int depth = in ? a.k : 0, g = min(rows.g, a.groups - 1), last_row = rows.hi - 1, last_col = a.m - 1;
  const int8_t* w = a.w + (int64_t)g * a.m * a.k;
  const int64_t x_end = (int64_t)(a.n - 1) * a.x_stride + a.k, w_end = (int64_t)(a.groups - g) * a.m * a.k;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wr = wave / 2 * 64, wc = wave % 2 * 64;
  i32x16 acc[2][2] = {};
  bytes16 raw[2][4];
  auto load = [&](int t0) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int p = threadIdx.x + i * 256, major = p / 8, t = t0 + p % 8 * 16;
      const int64_t xo = (int64_t)min(rows.lo + major, last_row) * a.x_stride + t, wo = (int64_t)min(c0 + major, last_col) * a.k + t;
      raw[0][i] = load_bytes<true>(a.x + xo, t, depth, x_end - xo);
      raw[1][i] = load_bytes<false>(w + wo, t, depth, w_end - wo);
    }
  };
  auto place = [](int major, int piece) { return major * D + ((piece ^ (major & 7)) * 16); };
  if (depth > 0) load(0);
  for (int t0 = 0; t0 < depth; t0 += D) {
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int p = threadIdx.x + i * 256;
        *reinterpret_cast<bytes16*>(lds + s * BM * D + place(p / 8, p % 8)) = raw[s][i];
      }
    __syncthreads();
    if (t0 + D < depth) load(t0 + D);
#pragma unroll
    for (int step = 0; step < D / 32; ++step) {
      i32x4 fr[2], fc[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        fr[i] = *reinterpret_cast<const i32x4*>(lds + place(wr + i * 32 + (lane & 31), step * 2 + (lane >> 5)));
        fc[i] = *reinterpret_cast<const i32x4*>(lds + BM * D + place(wc + i * 32 + (lane & 31), step * 2 + (lane >> 5)));
      }
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fc[j], fr[i], acc[i][j], 0, 0, 0);
    }
    __syncthreads();
  }
  // lane l has row l % 32, columns 8 q + 4 (l / 32) .. + 3 in registers 4 q .. 4 q + 3
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int row = rows.lo + wr + i * 32 + (lane & 31);
    if (row > last_row) continue;
    const float xs = in ? a.x_scale[row] : 0.f;
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int col = c0 + wc + j * 32 + 8 * (e / 4) + 4 * (lane >> 5) + e % 4;
        if (col > last_col) continue;
        float v = 0.f;
        if (in) {
          v = (float)acc[i][j][e] * xs * a.w_scale[(int64_t)g * a.m + col];
          if (a.bias) v += a.bias[(int64_t)g * a.m + col];
          if (a.relu) v = v < 0.f ? 0.f : v;
          if (a.residual) v += to_float(((const TO*)a.residual)[row * a.residual_stride + col]);
        }
        ((TO*)a.y)[row * a.y_stride + col] = from_float<TO>(v);
      }
  }
}

}  // namespace sp
