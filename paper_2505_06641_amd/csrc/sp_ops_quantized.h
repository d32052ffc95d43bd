// Grouped linear layers in 8 bits, for serving.
//   rows     scale_i = max_c |x_ic| / 127        q_ic = x_ic (127 / max_c |x_ic|), rounded to the nearest whole number, ties to even
//   layer    y_i = act(scale_i w_scale_go sum_c q_ic w_goc + b_go) + r_i, the sum in 32-bit integers: exact
// Weights lie with an output's inputs next to each other, [groups, m, k], so that both sides' 16 consecutive inputs are what a lane of the matrix
// cores takes.
#pragma once
#include <type_traits>

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

// A team of lanes keeps a row between its largest value and the rounding.  Bound by memory: 262144 x 1024 bfloat16 150 us (5.4 TB/s).
template <typename T, int TEAM, int C>
__global__ __launch_bounds__(kTeamThreads<TEAM>) void k_quantize(int n, int d, const T* __restrict__ x, int64_t x_stride, int8_t* __restrict__ q,
                                                                 int64_t q_stride, float* __restrict__ scale) {
  constexpr int V = kPiece<T>, ROWS = kTeamThreads<TEAM> / TEAM;
  __shared__ float red[2][TEAM > 64 ? TEAM / 64 : 1];
  const int t = threadIdx.x % TEAM, team = threadIdx.x / TEAM;
  int turn = 0;
  for (int64_t row = (int64_t)blockIdx.x * ROWS + team; row < n; row += (int64_t)gridDim.x * ROWS, turn ^= 1) {
    raw_piece v[C];
    float high = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) v[c] = load_raw_piece(x + row * x_stride, (c * TEAM + t) * V, d);
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < V; ++i) high = __builtin_elementwise_maximum(high, fabsf(of_raw((const T*)nullptr, v[c], i)));     // (NaN stays)
    high = team_max<TEAM>(high < INFINITY ? high : INFINITY, red[turn]);
    const RowScale s(high, high < INFINITY);
    if (t == 0) scale[row] = s.scale;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int col = (c * TEAM + t) * V;
      int b[V];
#pragma unroll
      for (int i = 0; i < V; ++i) b[i] = s.of(of_raw((const T*)nullptr, v[c], i));
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
  bool past_caches;                              // y is too long for the last-level cache: written past it
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

// A workgroup computes BM rows of one group by BN columns, wavefronts of 64 by BN / 2, D bytes of the depth at a time by way of LDS.  Rows and
// columns beyond the tile's last are that one again, and not written.  LDS: [rows of both sides][D bytes], the 16-byte pieces of a row permuted
// by the row, so that the eight rows that are read together lie in different banks.  Two stages of the depth lie there, one of them being multiplied.
//   DIRECT: memory to LDS without registers.  For depths, strides and addresses that are multiples of 16.
//   else by way of registers, which takes any address and cuts what lies behind the depth.
// Tiles of 128 by 128 have four workgroups to a compute unit, which hide each other's trips to memory (two stages of 64 bytes: 65536 rows,
// 1024 -> 1024 97 us; three stages and three workgroups 101; tiles of 128 by 256, whose wavefronts read a quarter less from LDS, and two workgroups
// 103).  Many tiles of long depths (256 by 256, one workgroup to a compute unit): 262144 rows of rounded normal numbers, 1024 -> 1024 360 us and 2048 -> 1024 616,
// so that the sums are made at 2140 TOP/s, near the library's rate on such numbers (8192 x 8192 x 8192 2150, with one side transposed 2520), and some 100 us go
// to what nothing of a workgroup's own overlaps: its first loads and its results, 512 MB in all.  The cycles are those of zeros, matrix cores and vector instructions
// busy a third of them each and wavefronts waiting for a third; the clock is not: 2.1 GHz, on zeros 2.4 (316 us).
template <int BM, int BN, int D>
struct QuantizedTile {
  static constexpr int WAVES = BM / 32, FR = 2, FC = BN / 64, kRows = BM + BN;
  static constexpr int kAcross = D / 16, kRun = 64 / kAcross;         // pieces of a row, rows of a run
  static constexpr int kChunks = kRows / kRun / WAVES, kOfX = BM / kRun / WAVES;   // a wavefront's runs, the first of them rows of x
  static constexpr int kSums = WAVES * 32 * (BN / 2) * 4;             // 32 rows of every wavefront's
  static constexpr int kBytes = 2 * kRows * D > kSums ? 2 * kRows * D : kSums;
  static __device__ __forceinline__ int swap(int row) { return D == 128 ? row & 7 : row >> 1 & 3; }
  static __device__ __forceinline__ int place(int row, int piece) { return row * D + ((piece ^ swap(row)) * 16); }
};

// Sixteen bytes for every lane from base + off to LDS: the wavefront's lanes one after the other from `to` on.  (In asm, since the compiler would wait
// for all such loads before every read of LDS; there is no output that it could take for written.)  The load takes `to` from M0, one wait state behind
// a scalar write of it at the earliest, which the compiler does not see to in front of asm.
__device__ __forceinline__ void load_to_lds(uint32_t to, const int8_t* base, uint32_t off) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "{m0}"(to), "v"(off), "s"(base) : "memory");
}
// Eight results, which nobody reads before much else has gone through the caches.
typedef uint32_t u32x4_at4 __attribute__((ext_vector_type(4), aligned(4)));
__device__ __forceinline__ void store_past_caches(float* p, const float (&v)[8]) {
#pragma unroll
  for (int h = 0; h < 8; h += 4) {
    const u32x4_at4 q = {__float_as_uint(v[h]), __float_as_uint(v[h + 1]), __float_as_uint(v[h + 2]), __float_as_uint(v[h + 3])};
    __builtin_nontemporal_store(q, reinterpret_cast<u32x4_at4*>(p + h));
  }
}
__device__ __forceinline__ void store_past_caches(bf16* p, const float (&v)[8]) {
  u16x8_any q;
#pragma unroll
  for (int i = 0; i < 8; ++i) q[i] = __builtin_bit_cast(uint16_t, (bf16)v[i]);
  __builtin_nontemporal_store(q, reinterpret_cast<u16x8_any*>(p));
}
// A sum, of less than 2^31, is multiplied by its row's scale and then by its output's.  The scale of a row of large numbers comes last: the sum times it might
// pass float32 where the result does not.
constexpr float kLateScale = 0x1p64f;
__device__ __forceinline__ float early_scale(float s) { return s > kLateScale ? 1.f : s; }
__device__ __forceinline__ float late_scale(float s) { return s > kLateScale ? s : 1.f; }
// Until the wavefront's loads have arrived.
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(0)" : : : "memory"); }
// All wavefronts have come here, and what they read from LDS before has arrived.
__device__ __forceinline__ void meet() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory"); }

template <typename TO, int BM, int BN, int D, bool DIRECT>
__global__ __launch_bounds__(BM * 2, BM == 256 ? 2 : DIRECT ? 4 : 3) void k_quantized(QuantizedArgs a) {
  typedef QuantizedTile<BM, BN, D> Tile;
  constexpr int FR = Tile::FR, FC = Tile::FC, CH = Tile::kChunks, CX = Tile::kOfX, WAVES = Tile::WAVES, kStageBytes = Tile::kRows * D;
  constexpr int WN = BN / 2;                                          // columns of a wavefront
  __shared__ __align__(16) uint8_t lds[Tile::kBytes];
  if (blockIdx.x == 0 && threadIdx.x < 64) check_offsets(a.offsets, a.groups, a.n, a.err);
  const int tile = xcd_tile(blockIdx.x, a.row_tiles * a.col_tiles);
  if (tile < 0) return;
  RowTile rows;
  const int rt = tile / a.col_tiles, c0 = (tile % a.col_tiles) * BN;
  if (!find_row_tile(a.offsets, a.groups, a.n, BM, rt, &rows)) return;
  const int depth = a.k, g = min(rows.g, a.groups - 1), n_rows = rows.hi - rows.lo, n_cols = min(BN, a.m - c0);
  const int stages = (depth + D - 1) / D;
  const int8_t* x = a.x + (int64_t)rows.lo * a.x_stride;
  const int8_t* w = a.w + ((int64_t)g * a.m + c0) * a.k;
  if (rows.g == a.groups) {                                           // rows of no group
    for (int i = threadIdx.x; i < n_rows * n_cols; i += BM * 2) ((TO*)a.y)[(int64_t)(rows.lo + i / n_cols) * a.y_stride + c0 + i % n_cols] = from_float<TO>(0.f);
    return;
  }
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wr = wave / 2 * 64, wc = wave % 2 * WN;
  // what the sums are multiplied by, on its way while they are made: a lane's rows' scales, and those of the columns that it will write
  constexpr int VO = 8, kAcross = WN / VO, kAtOnce = 64 / kAcross;    // columns of a lane, lanes of a row, rows at once
  const int mine = (lane % kAcross) * VO, col = c0 + wc + mine, left = a.m - col;
  float xs[FR], ws[VO], bias[VO] = {};
#pragma unroll
  for (int i = 0; i < FR; ++i) xs[i] = a.x_scale[rows.lo + min(wr + i * 32 + (lane & 31), n_rows - 1)];
  load_some(a.w_scale + (int64_t)g * a.m + col, left, 0.f, ws);
  if (a.bias) load_some(a.bias + (int64_t)g * a.m + col, left, 0.f, bias);

  // a lane's piece of chunk i: which one of its row, and where from
  int row_of[CH];
  uint32_t off[CH];
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int r = (wave + i * WAVES) * Tile::kRun + lane / Tile::kAcross;                     // rows of x, then columns
    row_of[i] = r;
    off[i] = i < CX ? (uint32_t)min(r, n_rows - 1) * (uint32_t)a.x_stride : (uint32_t)min(r - BM, n_cols - 1) * (uint32_t)a.k;
  }
  auto piece_of = [&](int i) { return (lane % Tile::kAcross) ^ Tile::swap(row_of[i]); };

  i32x16 acc[FR][FC] = {};
  auto multiply = [&](const uint8_t* at) {
#pragma unroll
    for (int step = 0; step < D / 32; ++step) {
      i32x4 fr[FR], fc[FC];
#pragma unroll
      for (int i = 0; i < FR; ++i) fr[i] = *reinterpret_cast<const i32x4*>(at + Tile::place(wr + i * 32 + (lane & 31), step * 2 + (lane >> 5)));
#pragma unroll
      for (int j = 0; j < FC; ++j) fc[j] = *reinterpret_cast<const i32x4*>(at + Tile::place(BM + wc + j * 32 + (lane & 31), step * 2 + (lane >> 5)));
#pragma unroll
      for (int i = 0; i < FR; ++i)
#pragma unroll
        for (int j = 0; j < FC; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fc[j], fr[i], acc[i][j], 0, 0, 0);
    }
  };

  if constexpr (DIRECT) {
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds;
    auto load = [&](int s) {                                          // stage s of the depth; pieces behind the depth read the last one
      const int t0 = s * D, most = (depth - t0) / 16 - 1;
      const uint32_t to = lds0 + s % 2 * kStageBytes + wave * 1024;
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        const uint32_t from = off[i] + min(piece_of(i), most) * 16;
        load_to_lds(to + i * WAVES * 1024, (i < CX ? x : w) + t0, from);
      }
    };
    load(0);
    for (int s = 0; s < stages; ++s) {
      wait_loads();                                                   // (this stage's)
      uint8_t* at = lds + s % 2 * kStageBytes;
      const int most = (depth - s * D) / 16;
      if (most < Tile::kAcross) {                                                 // x behind the depth is 0
#pragma unroll
        for (int i = 0; i < CX; ++i)
          if (piece_of(i) >= most) *reinterpret_cast<bytes16*>(at + Tile::place(row_of[i], piece_of(i))) = bytes16{0, 0, 0, 0};
      }
      meet();                                                         // (nobody reads the stage before any more)
      if (s + 1 < stages) load(s + 1);
      multiply(at);
    }
  } else {
    bytes16 raw[CH];
    const int64_t x_end = (int64_t)(a.n - 1 - rows.lo) * a.x_stride + a.k, w_end = ((int64_t)(a.groups - g) * a.m - c0) * a.k;
    auto load = [&](int s) {
      if ((s + 1) * D <= depth) {
#pragma unroll
        for (int i = 0; i < CH; ++i) raw[i] = *reinterpret_cast<const bytes16_any*>((i < CX ? x : w) + s * D + (off[i] + piece_of(i) * 16));
        return;
      }
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        const int t = s * D + piece_of(i) * 16;
        raw[i] = i < CX ? load_bytes<true>(x + off[i] + t, t, depth, x_end - off[i] - t) : load_bytes<false>(w + off[i] + t, t, depth, w_end - off[i] - t);
      }
    };
    auto store = [&](int s) {
#pragma unroll
      for (int i = 0; i < CH; ++i) *reinterpret_cast<bytes16*>(lds + s % 2 * kStageBytes + Tile::place(row_of[i], piece_of(i))) = raw[i];
    };
    load(0);
    for (int s = 0; s < stages; ++s) {
      store(s);
      if (s + 1 < stages) load(s + 1);
      __syncthreads();
      multiply(lds + s % 2 * kStageBytes);
    }
  }

  // Sums to memory by way of each wavefront's own part of LDS, 32 rows at a time, so that whole lines are written: lane l has row l % 32, of a block's
  // columns 8 q + 4 (l / 32) .. + 3 in registers 4 q .. 4 q + 3.  The 16-byte pieces of a row are permuted by the row.
  float* stage = reinterpret_cast<float*>(lds) + wave * 32 * WN;
  __syncthreads();
  // all: all of the tile's rows and columns are there, and none of the wavefront's rows has a scale that comes last (to ask for each row costs 262144 rows,
  // 1024 -> 1024 30 us)
  bool late = false;
#pragma unroll
  for (int i = 0; i < FR; ++i) late |= xs[i] > kLateScale;
  const bool whole = n_rows == BM && n_cols == BN && !__any(late);
  auto finish = [&](auto all, auto past_caches) {
#pragma unroll
    for (int i = 0; i < FR; ++i) {
      const int r = lane & 31;
      const float by = all ? xs[i] : early_scale(xs[i]);
#pragma unroll
      for (int j = 0; j < FC; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *reinterpret_cast<f32x4*>(stage + r * WN + (((j * 8 + 2 * q + (lane >> 5)) ^ (r % (WN / 4))) * 4)) =
              f32x4{(float)acc[i][j][4 * q] * by, (float)acc[i][j][4 * q + 1] * by, (float)acc[i][j][4 * q + 2] * by,
                    (float)acc[i][j][4 * q + 3] * by};
      wave_sync();
#pragma unroll
      for (int u = 0; u < 32 / kAtOnce; ++u) {
        const int sr = u * kAtOnce + lane / kAcross, tr = wr + i * 32 + sr;
        const float then = all ? 1.f : late_scale(__shfl(xs[i], sr));
        if (!all && (tr >= n_rows || left <= 0)) continue;
        const int64_t row = rows.lo + tr;
        const int count = all ? VO : left;
        float v[VO], res[VO];
        if (a.residual) load_some((const TO*)a.residual + row * a.residual_stride + col, count, 0.f, res);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const f32x4 f = *reinterpret_cast<const f32x4*>(stage + sr * WN + (((mine / 4 + h) ^ (sr % (WN / 4))) * 4));
#pragma unroll
          for (int e = 0; e < 4; ++e) v[4 * h + e] = f[e];
        }
#pragma unroll
        for (int e = 0; e < VO; ++e) {
          v[e] = (all ? v[e] * ws[e] : v[e] * ws[e] * then) + bias[e];
          if (a.relu) v[e] = v[e] < 0.f ? 0.f : v[e];
          if (a.residual) v[e] += res[e];
        }
        TO* out = (TO*)a.y + row * a.y_stride + col;
        if constexpr (past_caches) store_past_caches(out, v);
        else store_some(out, count, v);
      }
      wave_sync();
    }
  };
  if (whole && a.past_caches) finish(std::true_type{}, std::true_type{});
  else if (whole) finish(std::true_type{}, std::false_type{});
  else finish(std::false_type{}, std::false_type{});
}

// Few rows: a request, a window of them, a small batch.  A workgroup takes 16 rows of one group and 16 columns, its wavefronts share out the
// depth, 64 bytes at a time, straight from memory, and their sums meet in LDS.  Bound by trips to memory: offsets, weights and rows, the result
// (a request, 512 -> 256: 3.5 us in a row of calls, which is a launch; 256 rows, 1024 -> 1024 7.2 us).
constexpr int kFewQuantizedRows = 16, kFewQuantizedCols = 16, kFewQuantizedThreads = 256;

template <typename TO>
__global__ __launch_bounds__(kFewQuantizedThreads) void k_quantized_few(QuantizedArgs a) {
  constexpr int WAVES = kFewQuantizedThreads / 64;
  __shared__ int32_t part[WAVES][16 * 17];
  if (blockIdx.x == 0 && threadIdx.x < 64) check_offsets(a.offsets, a.groups, a.n, a.err);
  const int tile = xcd_tile(blockIdx.x, a.row_tiles * a.col_tiles);
  if (tile < 0) return;
  const int rt = tile / a.col_tiles, c0 = (tile % a.col_tiles) * kFewQuantizedCols;
  RowTile rows;
  if (!find_row_tile(a.offsets, a.groups, a.n, kFewQuantizedRows, rt, &rows)) return;
  const bool in = rows.g < a.groups;
  const int n_rows = rows.hi - rows.lo, depth = in ? a.k : 0, g = min(rows.g, a.groups - 1);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, mine = lane & 15, own = 16 * (lane >> 4);
  const int64_t row_at = (int64_t)(rows.lo + min(mine, n_rows - 1)) * a.x_stride, x_end = (int64_t)(a.n - 1) * a.x_stride + a.k;
  const int64_t col_at = ((int64_t)g * a.m + min(c0 + mine, a.m - 1)) * a.k, w_end = (int64_t)a.groups * a.m * a.k;
  // what the sum is multiplied by
  const int r = threadIdx.x / 16, col = c0 + threadIdx.x % 16;
  const bool writes = r < n_rows && col < a.m;
  const int64_t row = rows.lo + r, at = (int64_t)g * a.m + col;
  float xs = 0.f, ws = 0.f, bias = 0.f, res = 0.f;
  if (writes && in) {
    xs = a.x_scale[row];
    ws = a.w_scale[at];
    if (a.bias) bias = a.bias[at];
    if (a.residual) res = to_float(((const TO*)a.residual)[row * a.residual_stride + col]);
  }
  i32x4 acc = {0, 0, 0, 0};
  for (int t0 = wave * 64; t0 < depth; t0 += WAVES * 64) {
    const int t = t0 + own;
    const bytes16 fr = load_bytes<true>(a.x + row_at + t, t, depth, x_end - row_at - t), fc = load_bytes<false>(a.w + col_at + t, t, depth, w_end - col_at - t);
    acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, fc), __builtin_bit_cast(i32x4, fr), acc, 0, 0, 0);
  }
  // lane l has row l % 16, columns 4 (l / 16) .. + 3
#pragma unroll
  for (int e = 0; e < 4; ++e) part[wave][mine * 17 + 4 * (lane >> 4) + e] = acc[e];
  __syncthreads();
  if (!writes) return;
  int sum = 0;
#pragma unroll
  for (int q = 0; q < WAVES; ++q) sum += part[q][r * 17 + threadIdx.x % 16];
  float v = in ? (float)sum * early_scale(xs) * ws * late_scale(xs) + bias : 0.f;
  if (a.relu) v = v < 0.f ? 0.f : v;
  ((TO*)a.y)[row * a.y_stride + col] = from_float<TO>(v + res);
}

}  // namespace sp
