// What the kernels of the head-training operators (sp_ops_*.h) share: element types, 16-byte pieces of rows, sums over
// teams of lanes, the rows of a group.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "sp_wave.h"

namespace sp {

typedef __bf16 bf16;

// error bits raised by kernels on bad data (reported by sp_ops_check)
constexpr uint32_t kErrOffsets = 1u;
constexpr uint32_t kErrLabel = 2u;
constexpr uint32_t kErrClassCount = 4u;
constexpr uint32_t kErrAppId = 8u;
constexpr uint32_t kErrRouterLogit = 16u;   // a router's logit that is NaN or +inf
constexpr uint32_t kErrExpert = 32u;
constexpr uint32_t kErrPlace = 64u;

// Elements of a 16-byte piece.
template <typename T> constexpr int kPiece = 16 / (int)sizeof(T);

// Pieces are read and written whole wherever a row starts: global memory takes 16-byte accesses at any element's address,
// and the rows of an odd width start at all of them.
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef uint16_t u16x8_any __attribute__((ext_vector_type(8), aligned(2)));
typedef uint16_t u16x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(bf16 v) { return (float)v; }
// The one rounding of an output: float32 to bfloat16, to the nearest, ties to even.
template <typename T> __device__ __forceinline__ T from_float(float v) { return (T)v; }

__device__ __forceinline__ void load_piece(const float* p, float (&v)[4]) {
  const f32x4_any q = *reinterpret_cast<const f32x4_any*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = q[i];
}
__device__ __forceinline__ void load_piece(const bf16* p, float (&v)[8]) {
  const u16x8_any q = *reinterpret_cast<const u16x8_any*>(p);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = __uint_as_float((uint32_t)q[i] << 16);
}
__device__ __forceinline__ void load_piece(const float* p, float (&v)[8]) {
  const f32x4_any a = *reinterpret_cast<const f32x4_any*>(p), b = *reinterpret_cast<const f32x4_any*>(p + 4);
#pragma unroll
  for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
}
__device__ __forceinline__ void store_piece(float* p, const float (&v)[4]) {
  f32x4_any q;
#pragma unroll
  for (int i = 0; i < 4; ++i) q[i] = v[i];
  *reinterpret_cast<f32x4_any*>(p) = q;
}
__device__ __forceinline__ void store_piece(bf16* p, const float (&v)[8]) {
  u16x8_any q;
#pragma unroll
  for (int i = 0; i < 8; ++i) q[i] = __builtin_bit_cast(uint16_t, (bf16)v[i]);
  *reinterpret_cast<u16x8_any*>(p) = q;
}
__device__ __forceinline__ void store_piece(bf16* p, const float (&v)[4]) {
  u16x4_any q;
#pragma unroll
  for (int i = 0; i < 4; ++i) q[i] = __builtin_bit_cast(uint16_t, (bf16)v[i]);
  *reinterpret_cast<u16x4_any*>(p) = q;
}

__device__ __forceinline__ void store_piece(float* p, const float (&v)[8]) {
  const float a[4] = {v[0], v[1], v[2], v[3]}, b[4] = {v[4], v[5], v[6], v[7]};
  store_piece(p, a);
  store_piece(p + 4, b);
}

// The first `count` elements of a piece (all of them, some, or none); the others are `fill`.
template <typename T, int V>
__device__ __forceinline__ void load_some(const T* p, int count, float fill, float (&v)[V]) {
  if (count >= V) {
    load_piece(p, v);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = i < count ? to_float(p[i]) : fill;
  }
}
template <typename T, int V>
__device__ __forceinline__ void store_some(T* p, int count, const float (&v)[V]) {
  if (count >= V) {
    store_piece(p, v);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i < count) p[i] = from_float<T>(v[i]);
  }
}

// A 16-byte piece of a row of d columns as it is in memory, from column `col` on: what makes numbers of it would wait for it.  What lies behind the
// row is 0; a piece that the row ends in is the row's last 16 bytes, moved down.
typedef uint32_t raw_piece __attribute__((ext_vector_type(4)));
typedef uint32_t raw_piece_any __attribute__((ext_vector_type(4), aligned(2)));
template <typename T>
__device__ __forceinline__ raw_piece load_raw_piece(const T* row, int col, int d) {
  constexpr int V = kPiece<T>;
  if (col + V <= d) return *reinterpret_cast<const raw_piece_any*>(row + col);
  raw_piece q = {0, 0, 0, 0};
  if (col >= d) return q;
  if (d >= V) {
    q = *reinterpret_cast<const raw_piece_any*>(row + d - V);
    const uint64_t low = (uint64_t)q[1] << 32 | q[0], high = (uint64_t)q[3] << 32 | q[2];
    const int by = (col + V - d) * (int)sizeof(T) * 8, rest = by & 63;
    const uint64_t a = by >= 64 ? high : low, b = by >= 64 ? 0 : high;
    const uint64_t lo = rest ? a >> rest | b << (64 - rest) : a, hi = b >> rest;
    return raw_piece{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
  }
#pragma unroll
  for (int i = 0; i < V - 1; ++i)                                     // (col is 0: a row of less than a piece)
    if (i < d) {
      if constexpr (V == 4) q[i] = __float_as_uint(row[i]);
      else q[i / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(row)[i] << (i % 2 * 16);
    }
  return q;
}
__device__ __forceinline__ float of_raw(const float*, raw_piece q, int i) { return __uint_as_float(q[i]); }
__device__ __forceinline__ float of_raw(const bf16*, raw_piece q, int i) {
  return __uint_as_float(i % 2 ? q[i / 2] & 0xffff0000u : q[i / 2] << 16);
}

// Sum and maximum over a team: TEAM consecutive lanes of a wavefront (2 to 64), or the TEAM > 64 threads of a
// workgroup.  Every lane of the team has the result, and every lane adds in the same order.  `lds`: one float per
// wavefront; two reductions that follow each other take different arrays.
template <int TEAM>
__device__ __forceinline__ float team_sum(float v, float* lds) {
  static_assert(TEAM == 2 || TEAM == 4 || TEAM == 8 || TEAM == 16 || TEAM == 32 || TEAM % 64 == 0, "parts of a wavefront or whole ones");
  if (TEAM == 2) v += __shfl_xor(v, 1);
  else if (TEAM == 4) v = sum4(v);
  else if (TEAM == 8) v = sum8(v);
  else v = sum16(v);
  if (TEAM >= 32) v += __shfl_xor(v, 16);
  if (TEAM >= 64) v += __shfl_xor(v, 32);
  if (TEAM > 64) {
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int w = 0; w < TEAM / 64; ++w) v += lds[w];
  }
  return v;
}
template <int TEAM>
__device__ __forceinline__ float team_max(float v, float* lds) {
#pragma unroll
  for (int s = 1; s < (TEAM < 64 ? TEAM : 64); s *= 2) v = fmaxf(v, __shfl_xor(v, s));
  if (TEAM > 64) {
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = lds[0];
#pragma unroll
    for (int w = 1; w < TEAM / 64; ++w) v = fmaxf(v, lds[w]);
  }
  return v;
}

// The threads of a workgroup whose teams take one row each at a time.
template <int TEAM> constexpr int kTeamThreads = TEAM > 256 ? TEAM : 256;

// Inclusive prefix maximum across a wavefront of values that are not negative, as wave_scan_incl adds them up: a lane that a step does
// not write sees 0.
__device__ __forceinline__ int wave_scan_max(int x) {
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false));   // row_shr:1
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false));   // row_shr:2
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false));   // row_shr:4
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false));   // row_shr:8
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false));   // row_bcast:15 into rows 1 and 3
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false));   // row_bcast:31 into rows 2 and 3
  return x;
}

// The rows of group g.  Offsets that are not 0 <= ... <= n in order are reported by whoever walks them all; here they are
// only kept inside the arrays.
__device__ __forceinline__ void group_rows(const int32_t* offsets, int n, int g, int* lo, int* hi) {
  const int a = min(max(offsets[g], 0), n);
  *lo = a;
  *hi = min(max(offsets[g + 1], a), n);
}

// Which rows a workgroup's tile of at most tile_rows rows holds.  The tiles of group 0 come first, then those of group 1, ...; a group
// without rows has none.  Rows behind the last group form one more group (g == n_groups).  Every wavefront looks for itself:
// 64 groups at a time, each lane one of them.  Returns false where there are fewer tiles than `tile` + 1.
struct RowTile {
  int g, lo, hi;      // rows lo .. hi of group g
  int start;          // the group's first row
  bool whole;         // they are all of the group's rows
};
__device__ __forceinline__ bool find_row_tile(const int32_t* offsets, int n_groups, int n, int tile_rows, int tile, RowTile* out) {
  const int lane = threadIdx.x & 63;
  int before = 0, end = 0;                       // tiles and rows of the groups before this turn's
  for (int base = 0; base <= n_groups; base += 64) {
    const int g = base + lane;
    int e = g < n_groups ? min(max(offsets[g + 1], 0), n) : n;
    e = max(e, end);
    e = wave_scan_max(e);                        // ends in order, whatever the offsets say
    int s0 = __shfl_up(e, 1);
    if (lane == 0) s0 = end;
    const int tiles = g <= n_groups ? (int)(((uint32_t)(e - s0) + (uint32_t)tile_rows - 1u) / (uint32_t)tile_rows) : 0;
    const int upto = before + (int)wave_scan_incl((uint32_t)tiles);
    const unsigned long long has = __ballot(upto > tile);
    if (has) {
      const int l = __ffsll(has) - 1;            // (scalars from here on: the same on every lane, and known to be)
      const int first = __builtin_amdgcn_readlane(s0 + (tile - (upto - tiles)) * tile_rows, l), last = __builtin_amdgcn_readlane(e, l);
      out->g = base + l;
      out->lo = first;
      out->start = __builtin_amdgcn_readlane(s0, l);
      out->hi = last - first < tile_rows ? last : first + tile_rows;
      out->whole = __builtin_amdgcn_readlane(tiles, l) == 1;
      return true;
    }
    before = __builtin_amdgcn_readlane(upto, 63);
    end = __builtin_amdgcn_readlane(e, 63);
  }
  return false;
}

// Offsets have to start at 0, not to decrease, and not to pass n.  By one wavefront of a launch.
__device__ __forceinline__ void check_offsets(const int32_t* offsets, int n_groups, int n, uint32_t* err) {
  bool bad = false;
  for (int g = threadIdx.x & 63; g <= n_groups; g += 64) {
    const int o = offsets[g];
    bad |= o < 0 || o > n || (g == 0 ? o != 0 : o < offsets[g - 1]);
  }
  if (__ballot(bad) && (threadIdx.x & 63) == 0) atomicOr(err, kErrOffsets);
}

}  // namespace sp
