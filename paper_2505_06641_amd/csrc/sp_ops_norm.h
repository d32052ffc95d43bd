// Layer norm of rows and its gradients.
//   mu = mean x, rstd = 1 / sqrt(mean (x - mu)^2 + eps), xh = (x - mu) rstd, y = xh gamma + beta
//   q = dy gamma;  dx = rstd (q - mean q - xh mean(q xh));  dgamma = sum over rows dy xh;  dbeta = sum over rows dy
// A row belongs to a team of lanes that keeps it in registers: one pass over memory, the variance from the differences to the
// mean (no sum of squares less a square: that loses everything where the mean is far from 0).  Bound by memory.
#pragma once
#include "sp_ops_common.h"

namespace sp {

constexpr int kNormBlocks = 2048;           // workgroups that share out the rows of a forward pass
constexpr int kNormBackBlocks = 1024;       // and of a backward pass, each with a row of sums of its own to be added up

// Elements from one row of partial sums to the next: whole 16-byte pieces.
__host__ __device__ __forceinline__ int64_t norm_part_stride(int d) { return (2 * (int64_t)d + 3) / 4 * 4; }

// A team's columns: piece c of lane t holds columns (c * TEAM + t) * V on.  Where a row is no whole number of pieces (not WHOLE), its
// last piece starts V columns before the row's end instead and holds `skip` columns that are another lane's as well: read whole like any
// other, counted from `skip` on, and written with the values that the other lane writes there too.  (Element by element that piece
// costs more than all others of the row: 665558 bfloat16 rows of 111 columns 145 us, so 72 us, of 112 columns 67 us.)  Rows shorter than
// a piece are read and written element by element.
template <typename T, int TEAM, bool WHOLE>
struct NormPiece {
  static constexpr int V = kPiece<T>;
  int col, skip;                              // skip >= V: nothing of the row
  __device__ __forceinline__ NormPiece(int d, int c, int t) {
    const int at = (c * TEAM + t) * V;
    col = WHOLE || d < V ? at : min(at, d - V);
    skip = WHOLE || d < V ? (at < d ? 0 : V) : at - col;
  }
  __device__ __forceinline__ bool any() const { return skip < V; }
  __device__ __forceinline__ bool own(int i, int d) const { return WHOLE ? true : i >= skip && col + i < d; }
  template <typename E>
  __device__ __forceinline__ void load(const E* row, int d, float fill, float (&v)[V]) const {
    if (any()) {
      if (WHOLE || d >= V) load_piece(row + col, v);
      else load_some(row + col, d - col, fill, v);
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = fill;
    }
  }
  __device__ __forceinline__ void store(T* row, int d, const float (&v)[V]) const {
    if (!any()) return;
    if (WHOLE || d >= V) store_piece(row + col, v);
    else store_some(row + col, d - col, v);
  }
};

template <typename T, int TEAM, int C, bool WHOLE>
__global__ __launch_bounds__(kTeamThreads<TEAM>) void k_norm(int n, int d, const T* x, int64_t x_stride, const float* __restrict__ gamma,
                                                             const float* __restrict__ beta, float eps, T* y, int64_t y_stride,
                                                             float* __restrict__ mean_out, float* __restrict__ rstd_out) {
  constexpr int V = kPiece<T>, ROWS = kTeamThreads<TEAM> / TEAM;
  typedef NormPiece<T, TEAM, WHOLE> Piece;
  __shared__ float red[2][TEAM > 64 ? TEAM / 64 : 1];
  const int t = threadIdx.x % TEAM, team = threadIdx.x / TEAM;
  float ga[C][V], be[C][V];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const Piece p(d, c, t);
#pragma unroll
    for (int i = 0; i < V; ++i) ga[c][i] = 1.f, be[c][i] = 0.f;
    if (gamma) p.load(gamma, d, 1.f, ga[c]);
    if (beta) p.load(beta, d, 0.f, be[c]);
  }
  const float fd = (float)d;
  for (int64_t row = (int64_t)blockIdx.x * ROWS + team; row < n; row += (int64_t)gridDim.x * ROWS) {
    float v[C][V];
    float s = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const Piece p(d, c, t);
      p.load(x + row * x_stride, d, 0.f, v[c]);
#pragma unroll
      for (int i = 0; i < V; ++i) s += p.own(i, d) ? v[c][i] : 0.f;
    }
    const float mu = team_sum<TEAM>(s, red[0]) / fd;
    float q = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const Piece p(d, c, t);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        v[c][i] -= mu;
        q += p.any() && p.own(i, d) ? v[c][i] * v[c][i] : 0.f;
      }
    }
    const float rstd = 1.f / sqrtf(team_sum<TEAM>(q, red[1]) / fd + eps);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const Piece p(d, c, t);
#pragma unroll
      for (int i = 0; i < V; ++i) v[c][i] = v[c][i] * rstd * ga[c][i] + be[c][i];
      p.store(y + row * y_stride, d, v[c]);
    }
    if (t == 0) {
      if (mean_out) mean_out[row] = mu;
      if (rstd_out) rstd_out[row] = rstd;
    }
  }
}

// Every team walks its rows with dgamma's and dbeta's sums of its columns in registers; the workgroup's teams add theirs up,
// those of a wavefront across lanes and the wavefronts one after the other in LDS, and write one row of partial sums:
// part[workgroup][2][d], each row of them at a 16-byte piece.  A single workgroup writes dgamma and dbeta.
template <typename T, int TEAM, int C, bool WHOLE>
__global__ __launch_bounds__(kTeamThreads<TEAM>) void k_norm_back(int n, int d, const T* dy, int64_t dy_stride, const T* x,
                                                                  int64_t x_stride, const float* __restrict__ gamma,
                                                                  const float* __restrict__ mean, const float* __restrict__ rstd, T* dx,
                                                                  int64_t dx_stride, float* __restrict__ part,
                                                                  float* __restrict__ dgamma, float* __restrict__ dbeta) {
  constexpr int V = kPiece<T>, ROWS = kTeamThreads<TEAM> / TEAM;
  typedef NormPiece<T, TEAM, WHOLE> Piece;
  __shared__ float red[2][TEAM > 64 ? TEAM / 64 : 1];
  __shared__ float sums[TEAM <= 64 ? TEAM * C * V : 1][2];
  const int t = threadIdx.x % TEAM, team = threadIdx.x / TEAM;
  float ga[C][V], dg[C][V], db[C][V];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const Piece p(d, c, t);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      ga[c][i] = 1.f;
      dg[c][i] = db[c][i] = 0.f;
    }
    if (gamma) p.load(gamma, d, 1.f, ga[c]);
  }
  const float fd = (float)d;
  for (int64_t row = (int64_t)blockIdx.x * ROWS + team; row < n; row += (int64_t)gridDim.x * ROWS) {
    float g[C][V], xh[C][V];
    const float mu = mean[row], rs = rstd[row];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const Piece p(d, c, t);
      p.load(dy + row * dy_stride, d, 0.f, g[c]);          // (columns beyond the row: dy = 0, xh = 0)
      p.load(x + row * x_stride, d, mu, xh[c]);
    }
    float sq = 0.f, sqx = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const Piece p(d, c, t);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float own = p.own(i, d) ? g[c][i] : 0.f;
        xh[c][i] = (xh[c][i] - mu) * rs;
        db[c][i] += own;
        dg[c][i] += own * xh[c][i];
        sq += own * ga[c][i];
        sqx += own * ga[c][i] * xh[c][i];
        g[c][i] *= ga[c][i];
      }
    }
    if (!dx) continue;
    const float mq = team_sum<TEAM>(sq, red[0]) / fd, mqx = team_sum<TEAM>(sqx, red[1]) / fd;
#pragma unroll
    for (int c = 0; c < C; ++c) {
#pragma unroll
      for (int i = 0; i < V; ++i) g[c][i] = rs * (g[c][i] - mq - xh[c][i] * mqx);
      Piece(d, c, t).store(dx + row * dx_stride, d, g[c]);
    }
  }
  if (!part && !dgamma && !dbeta) return;
  if (TEAM <= 64) {
    constexpr int WAVES = kTeamThreads<TEAM> / 64;
    const int wave = threadIdx.x >> 6;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < V; ++i)
#pragma unroll
        for (int s = TEAM; s < 64; s *= 2) {
          dg[c][i] += __shfl_xor(dg[c][i], s);
          db[c][i] += __shfl_xor(db[c][i], s);
        }
    for (int turn = 0; turn < WAVES; ++turn) {
      if (turn == wave && (threadIdx.x & 63) < TEAM) {
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int i = 0; i < V; ++i) {
            float* at = sums[(c * V + i) * TEAM + t];
            if (turn > 0) { dg[c][i] += at[0]; db[c][i] += at[1]; }
            if (turn < WAVES - 1) { at[0] = dg[c][i]; at[1] = db[c][i]; }
          }
      }
      __syncthreads();
    }
    if (wave != WAVES - 1 || (threadIdx.x & 63) >= TEAM) return;
  }
  float* to_gamma = part ? part + blockIdx.x * norm_part_stride(d) : dgamma;
  float* to_beta = part ? to_gamma + d : dbeta;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const Piece p(d, c, t);
    if (!p.any()) continue;
    if (WHOLE) {
      if (to_gamma) store_piece(to_gamma + p.col, dg[c]);
      if (to_beta) store_piece(to_beta + p.col, db[c]);
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (p.own(i, d)) {
          if (to_gamma) to_gamma[p.col + i] = dg[c][i];
          if (to_beta) to_beta[p.col + i] = db[c][i];
        }
    }
  }
}

// Sums of the workgroups' rows of partial sums: 32 columns to a workgroup of 256, 32 threads to 4 columns, their loads under way
// together (one thread that adds 128 rows one after the other takes 30 us).
__global__ __launch_bounds__(256) void k_norm_join(int parts, int d, const float* __restrict__ part, float* __restrict__ dgamma,
                                                   float* __restrict__ dbeta) {
  __shared__ f32x4 sums[32][8];
  const int lane = threadIdx.x % 8, slice = threadIdx.x / 8;
  const int64_t cols = 2 * (int64_t)d, stride = norm_part_stride(d), col = (int64_t)blockIdx.x * 32 + lane * 4;
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
  if (col < cols) {
#pragma unroll 8
    for (int p = slice; p < parts; p += 32) s += *reinterpret_cast<const f32x4*>(part + p * stride + col);
  }
  sums[slice][lane] = s;
  __syncthreads();
  if (slice > 0) return;
  for (int j = 1; j < 32; ++j) s += sums[j][lane];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int64_t c = col + e;
    float* out = c < d ? dgamma : dbeta;
    if (c < cols && out) out[c < d ? c : c - d] = s[e];
  }
}

}  // namespace sp
