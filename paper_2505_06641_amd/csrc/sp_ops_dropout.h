// Dropout without a stored mask.
//   y = r + (number(row, column) >= drop ? x 65536 / (65536 - drop) : 0)
// The numbers are the 16-bit halves of the words of Philox 4x32 with ten rounds (J. Salmon, M. Moraes, R. Dror, D. Shaw, "Parallel random
// numbers: as easy as 1, 2, 3", 2011), so that one computation serves the eight columns of a piece: counter (piece of the row, row, offset low,
// offset high), key the seed, column 8 piece + 2 word + half with the low half first.  They hang on nothing else: not on type, stride or
// launch, and the backward pass is the same call on dy.  Bound by memory: 65536 x 768 bfloat16 with a residual 52 us (5.8 TB/s, the residual partly from
// the last-level cache), 262144 x 256 float32 91 us (5.9 TB/s); one computation to four columns would take as long as the memory does.
#pragma once
#include "sp_ops_common.h"

namespace sp {

struct DropoutArgs {
  int n, d, pieces;                              // pieces of eight columns of a row
  uint32_t drop;                                 // of 65536
  float scale;
  uint32_t key0, key1;
  uint64_t offset;
  const int64_t* step;                           // [1] or null: added to the offset
  const void* x;  int64_t x_stride;
  const void* residual;  int64_t residual_stride;
  void* y;  int64_t y_stride;
};

__device__ __forceinline__ void philox(uint32_t (&c)[4], uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t a = (uint64_t)c[0] * 0xD2511F53u, b = (uint64_t)c[2] * 0xCD9E8D57u;
    const uint32_t c1 = c[1], c3 = c[3];
    c[0] = (uint32_t)(b >> 32) ^ c1 ^ k0;
    c[1] = (uint32_t)b;
    c[2] = (uint32_t)(a >> 32) ^ c3 ^ k1;
    c[3] = (uint32_t)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
}

// Eight columns of a row as they are in memory.
template <typename T>
struct RawColumns {
  static constexpr int V = kPiece<T>;
  raw_piece q[8 / V];
  __device__ __forceinline__ void load(const T* row, int col, int d) {
#pragma unroll
    for (int h = 0; h < 8 / V; ++h) q[h] = load_raw_piece(row, col + h * V, d);
  }
  __device__ __forceinline__ float operator[](int i) const { return of_raw((const T*)nullptr, q[i / V], i % V); }
};

// A piece to a thread, in launches of one or two dimensions of workgroups.  (Four bfloat16 or two float32 pieces to a thread, on their way together: 65536 x 768
// bfloat16 with a residual 56 us against 53, 262144 x 256 float32 98 against 91.)
template <typename T>
__global__ __launch_bounds__(256) void k_dropout(DropoutArgs a) {
  const uint64_t offset = a.offset + (a.step ? (uint64_t)*a.step : 0u);
  const int64_t at = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 256 + threadIdx.x;
  const int64_t row = at >> 32 ? at / a.pieces : (int64_t)((uint32_t)at / (uint32_t)a.pieces);
  if (row >= a.n) return;
  const int col = (int)(at - row * a.pieces) * 8;
  RawColumns<T> x, r;
  x.load((const T*)a.x + row * a.x_stride, col, a.d);
  if (a.residual) r.load((const T*)a.residual + row * a.residual_stride, col, a.d);
  uint32_t c[4] = {(uint32_t)col / 8, (uint32_t)row, (uint32_t)offset, (uint32_t)(offset >> 32)};
  philox(c, a.key0, a.key1);
  float v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t number = i % 2 ? c[i / 2] >> 16 : c[i / 2] & 0xffffu;
    v[i] = number >= a.drop ? x[i] * a.scale : 0.f;
    if (a.residual) v[i] += r[i];
  }
  store_some((T*)a.y + row * a.y_stride + col, a.d - col, v);
}

}  // namespace sp
