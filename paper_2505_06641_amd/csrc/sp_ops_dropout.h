// Dropout without a stored mask.
//   y = r + (number(row, column) >= drop ? x 65536 / (65536 - drop) : 0)
// The numbers are the 16-bit halves of the words of Philox 4x32 with ten rounds (J. Salmon, M. Moraes, R. Dror, D. Shaw, "Parallel random
// numbers: as easy as 1, 2, 3", 2011), so that one computation serves the eight columns of a piece: counter (piece of the row, row, offset low,
// offset high), key the seed, column 8 piece + 2 word + half with the low half first.  They hang on nothing else: not on type, stride or
// launch, and the backward pass is the same call on dy.
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

constexpr int kDropoutEach = 4;                  // pieces of a thread

template <typename T>
__global__ __launch_bounds__(256) void k_dropout(DropoutArgs a) {
  const uint64_t offset = a.offset + (a.step ? (uint64_t)*a.step : 0u);
  const int64_t all = (int64_t)a.n * a.pieces, base = (int64_t)blockIdx.x * (256 * kDropoutEach);
#pragma unroll
  for (int u = 0; u < kDropoutEach; ++u) {
    const int64_t at = base + u * 256 + threadIdx.x;
    if (at >= all) return;
    const int64_t row = at / a.pieces;
    const int piece = (int)(at % a.pieces), col = piece * 8, count = a.d - col;
    float v[8], r[8];
    load_some((const T*)a.x + row * a.x_stride + col, count, 0.f, v);
    if (a.residual) load_some((const T*)a.residual + row * a.residual_stride + col, count, 0.f, r);
    uint32_t c[4] = {(uint32_t)piece, (uint32_t)row, (uint32_t)offset, (uint32_t)(offset >> 32)};
    philox(c, a.key0, a.key1);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t number = i % 2 ? c[i / 2] >> 16 : c[i / 2] & 0xffffu;
      v[i] = number >= a.drop ? v[i] * a.scale : 0.f;
      if (a.residual) v[i] += r[i];
    }
    store_some((T*)a.y + row * a.y_stride + col, count, v);
  }
}

}  // namespace sp
