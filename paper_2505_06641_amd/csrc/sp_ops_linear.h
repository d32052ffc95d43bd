// Linear layers of rows that are grouped by application, and their gradients.
//   y_i = act(x_i W_g + b_g) + r_i      dx_i = dz_i W_g^T      dW_g = sum over the group's rows x_i^T dz_i      db_g = sum dz_i
// with dz = dy where the activation passed something, 0 elsewhere.
//
// All three are products of a "row side" and a "column side" over a common depth:
//   y   rows x [n, k]         columns w [k, m]           depth k
//   dx  rows dz [n, m]        columns w^T                depth m
//   dW  rows x^T              columns dz                 depth: the group's rows
// A workgroup computes a tile of 128 rows by BN columns with the matrix cores (v_mfma_f32_32x32x16_bf16, sums in float32).  Both
// sides of a piece of the depth go from memory through registers into LDS, while the matrix cores work on the piece before: on the
// way the mask of the activation is applied, what lies beyond the tile, the group or the depth becomes 0, and float32 is split.
// A side whose depth is the contiguous one in memory lies in LDS as it came and is read 8 elements of the depth at a time; one
// whose depth is strided is read by the LDS's transposing loads.
//
// Float32: a value is the sum of three bfloat16 numbers, each the rounded rest of the ones before it.  bfloat16 has 8 significant bits, so the
// second number is at most 2^-8 of the value and the third 2^-17, which leaves nothing over: 8 + 8 + 8 bits are float32's 24.  Where
// the last of them would be below bfloat16's smallest subnormal, 2^-133 (values below 2^-110), up to 2^-134 is left over; the matrix cores
// take subnormals as they are.  Of the nine products of two such sums the six largest are taken, each exact in the float32 sum; the
// three others are at most 2 x 2^-25 + 2^-34 of the product together.  Six instructions of the bfloat16 rate are 2.6 times the float32
// instruction's rate.  An infinite factor (or one that rounds to one in bfloat16, from 3.39e38 on) makes its results NaN: its rest is
// one.
#pragma once
#include "sp_common.h"
#include "sp_ops_common.h"

namespace sp {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));

// A piece's elements from `first` on, as far as there are any.
template <typename T, int V>
__device__ __forceinline__ void store_part(T* p, int first, int count, const float (&v)[V]) {
  if (first == 0) {
    store_some(p, count, v);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i >= first && i < count) p[i] = from_float<T>(v[i]);
  }
}

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
  int row_tiles, col_tiles;              // of the launch (dW: tiles of k and of m)
  int chunk;                             // dW: rows of a group that a workgroup adds up, 0: all of them
  float* part;                           // dW: sums of the chunks, [chunks][k * m + m]
};

// Elements from one chunk's sums (dW, then db) to the next: whole 16-byte pieces.
__host__ __device__ __forceinline__ int64_t chunk_stride(const LinearArgs& a) { return ((int64_t)a.k * a.m + a.m + 3) / 4 * 4; }

enum LinearForm { kFormY = 0, kFormDx = 1, kFormDw = 2 };

template <typename T> constexpr int kPlanes = sizeof(T) == 4 ? 3 : 1; // bfloat16 numbers that make up a value
template <typename T> constexpr int kDepth = sizeof(T) == 4 ? 32 : 64; // depth of a piece: 48 KB of LDS with 128 columns, 32 KB

// Where NaN has to stay NaN: only what is below 0 becomes 0.
__device__ __forceinline__ float relu_of(float z) { return z < 0.f ? 0.f : z; }

// The first `count` elements of a piece, one by one (at the very end of an array; few registers matter more here than time).
__device__ __forceinline__ u32x4 load_raw_some(const float* p, int count) {
  u32x4 q = {0, 0, 0, 0};
#pragma unroll 1
  for (int i = count - 1; i >= 0; --i) q = u32x4{__float_as_uint(p[i]), q[0], q[1], q[2]};
  return q;
}
__device__ __forceinline__ u32x4 load_raw_some(const bf16* p, int count) {
  const uint16_t* h = reinterpret_cast<const uint16_t*>(p);
  u32x4 q = {0, 0, 0, 0};
#pragma unroll 1
  for (int i = count - 1; i >= 0; --i)
    q = u32x4{q[0] << 16 | h[i], q[1] << 16 | q[0] >> 16, q[2] << 16 | q[1] >> 16, q[3] << 16 | q[2] >> 16};
  return q;
}
// dz: dy where act > 0, 0 elsewhere (also where act is NaN).
__device__ __forceinline__ u32x4 masked(const float*, u32x4 dy, u32x4 act) {
#pragma unroll
  for (int i = 0; i < 4; ++i) dy[i] = __uint_as_float(act[i]) > 0.f ? dy[i] : 0u;
  return dy;
}
__device__ __forceinline__ u32x4 masked(const bf16*, u32x4 dy, u32x4 act) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t lo = __uint_as_float(act[i] << 16) > 0.f ? 0xffffu : 0u;
    const uint32_t hi = __uint_as_float(act[i] & 0xffff0000u) > 0.f ? 0xffff0000u : 0u;
    dy[i] &= lo | hi;
  }
  return dy;
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  const f32x2 v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}
__device__ __forceinline__ float low_bf16(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float high_bf16(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }

// One side of a tile: W rows (or columns) by kDepth<T> of the depth.
// LDS, per plane: contiguous depth [W][depth], the 16-byte pieces of a row permuted by the row, so that the eight rows that are
// read together lie in different banks; strided depth [depth][W], the 64-byte pieces permuted likewise by the depth.
template <typename T, int W, bool STRIDED, bool MASK, int THREADS>
struct Side {
  static constexpr int V = kPiece<T>, D = kDepth<T>, P = kPlanes<T>;
  static constexpr int kPieces = W * D / V / THREADS;        // of 16 bytes, each thread's
  static constexpr int kAcross = (STRIDED ? W : D) / V;             // pieces of a contiguous run in memory
  static constexpr int kElems = W * D;
  u32x4 raw[kPieces];
  u32x4 act[MASK ? kPieces : 1];

  uint32_t off, act_off;                                            // bytes from the piece of the depth's first element
  int64_t step, act_step;                                           // elements from one of a thread's pieces to the next
  static constexpr int kStep = THREADS / kAcross;            // the same in rows

  __device__ __forceinline__ void init(int64_t stride, int64_t act_stride) {
    const uint32_t major = threadIdx.x / kAcross, minor = (threadIdx.x % kAcross) * V;
    off = (major * (uint32_t)stride + minor) * (uint32_t)sizeof(T);
    act_off = (major * (uint32_t)act_stride + minor) * (uint32_t)sizeof(T);
    step = kStep * stride;
    act_step = kStep * act_stride;
  }
  // at: that element.  Where everything lies inside the tile and the depth:
  __device__ __forceinline__ void load(const T* at, const T* act_at) {
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      raw[i] = load_raw(at + i * step, off);
      if (MASK) act[i] = load_raw(act_at + i * act_step, act_off);
    }
  }
  // ... and where it does not.  limit: elements from `at` to the array's end (where its last row ends); valid rows (columns) and depth
  // are what is left of them.  A piece that reaches beyond what is left is read as far as the array goes, and cut later.
  __device__ __forceinline__ void load_edge(const T* at, int64_t limit, const T* act_at, int64_t act_limit, int valid, int depth) {
    const int major = threadIdx.x / kAcross, minor = (threadIdx.x % kAcross) * V;
    const int rows = STRIDED ? depth : valid, cols = STRIDED ? valid : depth;
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int count = major + i * kStep < rows ? cols - minor : 0;
      raw[i] = load_cut(at + i * step, off, limit - i * step, count);
      if (MASK) act[i] = load_cut(act_at + i * act_step, act_off, act_limit - i * act_step, count);
    }
  }
  __device__ __forceinline__ static u32x4 load_raw(const T* base, uint32_t off) {
    const u32x4_any q = *reinterpret_cast<const u32x4_any*>(reinterpret_cast<const char*>(base) + off);
    return u32x4{q[0], q[1], q[2], q[3]};
  }
  __device__ __forceinline__ static u32x4 load_cut(const T* base, uint32_t off, int64_t limit, int count) {
    if (count <= 0) return u32x4{0, 0, 0, 0};
    if (count < V && (int64_t)off + 16 > limit * (int64_t)sizeof(T))
      return load_raw_some(reinterpret_cast<const T*>(reinterpret_cast<const char*>(base) + off), count);
    return load_raw(base, off);
  }
  // (Apart from the load, so that no piece's load is waited for before the next one's is under way.)
  __device__ __forceinline__ void cut(int valid, int depth) {
    const int minor = (threadIdx.x % kAcross) * V, cols = STRIDED ? valid : depth;
    if (valid >= W && depth >= D) return;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int left = cols - minor - j * (V / 4);                  // (pieces of rows beyond the last are 0 already)
      const uint32_t keep = V == 4 ? (left > 0 ? 0xffffffffu : 0u) : left >= 2 ? 0xffffffffu : left == 1 ? 0xffffu : 0u;
#pragma unroll
      for (int i = 0; i < kPieces; ++i) raw[i][j] &= keep;
    }
  }

  __device__ __forceinline__ static int place(int major, int minor) {     // element of a plane, minor a multiple of 4
    if (STRIDED) {
      const int swap = W == 128 ? major & 3 : (major >> 1) & 1;
      return major * W + (((minor / 32) ^ swap) * 32) + minor % 32;
    }
    const int swap = D == 64 ? major & 7 : (major >> 1) & 3;
    return major * D + (((minor / 8) ^ swap) * 8) + minor % 8;
  }

  __device__ __forceinline__ void store(uint16_t* lds) {
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int p = threadIdx.x + i * THREADS, major = p / kAcross, minor = (p % kAcross) * V;
      if (MASK) raw[i] = masked((const T*)nullptr, raw[i], act[i]);
      uint16_t* at = lds + place(major, minor);
      if constexpr (P == 1) {
        *reinterpret_cast<u32x4*>(at) = raw[i];
      } else {
        float v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = __uint_as_float(raw[i][j]);
#pragma unroll
        for (int pl = 0; pl < 3; ++pl) {
          const u32x2 h = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
          *reinterpret_cast<u32x2*>(at + pl * kElems) = h;
          v[0] -= low_bf16(h[0]);
          v[1] -= high_bf16(h[0]);
          v[2] -= low_bf16(h[1]);
          v[3] -= high_bf16(h[1]);
        }
      }
    }
  }

  // Columns' sums of what the thread has loaded (strided sides: a thread's pieces share their columns).
  __device__ __forceinline__ void add_columns(float (&sum)[V]) const {
#pragma unroll
    for (int i = 0; i < kPieces; ++i)
#pragma unroll
      for (int j = 0; j < V; ++j) {
        if constexpr (P == 3) sum[j] += __uint_as_float(raw[i][j]);
        else sum[j] += j % 2 ? high_bf16(raw[i][j / 2]) : low_bf16(raw[i][j / 2]);
      }
  }

  // The fragment of 32 rows (columns) from w0 on and 16 of the depth: lane l holds w0 + l % 32, 8 (l / 32) .. + 7 of the depth.
  __device__ __forceinline__ static bf16x8 fragment(const uint16_t* lds, int w0, int step) {
    const int l = threadIdx.x & 63;
    if (!STRIDED) return *reinterpret_cast<const bf16x8*>(lds + place(w0 + (l & 31), step * 16 + 8 * (l >> 5)));
    // transposing load: of every 16 lanes, lane s gives 4 columns from 4 (s % 4) on at depth s / 4, and gets column s at 4 depths
    typedef __attribute__((address_space(3))) s16x4* lds_ptr;
    const int t = step * 16 + 8 * (l >> 5) + (l & 15) / 4, c = w0 + 16 * ((l >> 4) & 1) + 4 * (l & 3);
    union { s16x4 h[2]; bf16x8 v; } u;
    u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(lds + place(t, c)));
    u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(lds + place(t + 4, c)));
    return u.v;
  }
};

// The last tile of a group's rows, and the last one of the columns, starts early enough to be a whole one where there is enough before it:
// it computes again what the tile before it has, and leaves the writing to that one (float32 256 -> 1000: 921 -> 861 us; pieces that are cut take
// twice as long).  Columns of the tile: 128, or 64 for narrow outputs; rows: 128, or 64 for dW of few
// inputs (90070 rows, 5 -> 544 float32: dW 92 us with 128, 66 with 64).  Four wavefronts, 64 rows and BN / 2 columns each, or eight of 64 by 32: a wavefront
// of 64 by 64 reads a third less from LDS for its products (65536 x 1024 -> 512 bfloat16 99 us against 109, the LDS being what is busiest),
// eight are quicker through a tile where the device is not full (6170 x 256 -> 862 21 us against 24) and where the mask's registers leave
// room for two workgroups of four only.
template <typename T, typename TO, int FORM, int BM, int BN, bool MASK, int THREADS>
__device__ __forceinline__ void linear_tile(const LinearArgs& a, int block) {
  constexpr int D = kDepth<T>, P = kPlanes<T>, FR = BM / 64, FC = BN * 2 / (THREADS / 2), V = kPiece<T>;
  constexpr int WM = FR * 32, WN = FC * 32, WAVE_COLS = BN / WN;     // rows and columns of a wavefront, wavefronts side by side
  typedef Side<T, BM, FORM == kFormDw, FORM == kFormDx && MASK, THREADS> Rows;
  typedef Side<T, BN, FORM != kFormDx, FORM == kFormDw && MASK, THREADS> Cols;
  constexpr int kBoth = P * (Rows::kElems + Cols::kElems), kSums = 64 * BN * 2;      // two sides; 64 rows of sums
  __shared__ __align__(16) uint16_t lds[kBoth > kSums ? kBoth : kSums];
  uint16_t* lds_rows = lds;
  uint16_t* lds_cols = lds + P * Rows::kElems;
  if (block == 0 && threadIdx.x < 64) check_offsets(a.offsets, a.groups, a.n, a.err);

  // the tile: consecutive ones share rows, and go to one die as far as that is possible
  const int tile = xcd_tile(block, a.row_tiles * a.col_tiles);
  if (tile < 0) return;
  RowTile rows;
  const int rt = tile / a.col_tiles, ct = tile % a.col_tiles;
  int r0, n_rows, depth;
  int skip_r = 0;                                          // rows (columns) of the tile that are another one's to write
  int64_t slot = -1;                                       // dW: where a chunk's sums go
  const int width = FORM == kFormDx ? a.k : a.m;
  const int c0 = max(min(ct * BN, width - BN), 0), skip_c = ct * BN - c0;
  if (FORM == kFormDw) {
    const int k_tiles = (a.k + BM - 1) / BM, kt = rt % k_tiles, item = rt / k_tiles;
    if (a.chunk == 0) {
      rows.g = item;
      group_rows(a.offsets, a.n, item, &rows.lo, &rows.hi);
    } else {
      if (!find_row_tile(a.offsets, a.groups, a.n, a.chunk, item, &rows) || rows.g >= a.groups) return;
      if (!rows.whole) slot = item;
    }
    r0 = max(min(kt * BM, a.k - BM), 0);
    skip_r = kt * BM - r0;
    n_rows = a.k - r0;
    depth = rows.hi - rows.lo;
  } else {
    if (!find_row_tile(a.offsets, a.groups, a.n, BM, rt, &rows)) return;
    r0 = max(min(rows.lo, rows.hi - BM), rows.start);
    skip_r = rows.lo - r0;
    n_rows = rows.hi - r0;
    depth = rows.g < a.groups ? (FORM == kFormY ? a.k : a.m) : 0;
  }
  const T* x = (const T*)a.x;
  const T* w = (const T*)a.w + (int64_t)(FORM != kFormDw ? min(rows.g, a.groups - 1) : 0) * a.k * a.m;
  const int64_t w_left = (int64_t)(a.groups - min(rows.g, a.groups - 1)) * a.k * a.m;       // elements from there on
  const T* dy = (const T*)a.dy;
  const T* act = (const T*)a.act;

  Rows sr;
  Cols sc;
  if (FORM == kFormY) {
    sr.init(a.x_stride, 0);
    sc.init(a.m, 0);
  } else if (FORM == kFormDx) {
    sr.init(a.dy_stride, a.act_stride);
    sc.init(a.m, 0);
  } else {
    sr.init(a.x_stride, 0);
    sc.init(a.dy_stride, a.act_stride);
  }
  const bool inside = n_rows >= BM && width - c0 >= BN;
  auto load = [&](int t0, bool edge) {
    const T *pr, *pc, *qr = nullptr, *qc = nullptr;
    int64_t end_r, end_c, qend_r = 0, qend_c = 0;
    if (FORM == kFormY) {
      pr = x + (int64_t)r0 * a.x_stride + t0;
      end_r = (int64_t)(a.n - 1 - r0) * a.x_stride + a.k - t0;
      const int64_t skip = (int64_t)t0 * a.m + c0;
      pc = w + skip;
      end_c = w_left - skip;
    } else if (FORM == kFormDx) {
      const int64_t below = a.n - 1 - r0;
      pr = dy + (int64_t)r0 * a.dy_stride + t0;
      end_r = below * a.dy_stride + a.m - t0;
      qr = act + (int64_t)r0 * a.act_stride + t0;
      qend_r = below * a.act_stride + a.m - t0;
      const int64_t skip = (int64_t)c0 * a.m + t0;
      pc = w + skip;
      end_c = w_left - skip;
    } else {
      const int64_t row = rows.lo + t0, below = a.n - 1 - row;
      pr = x + row * a.x_stride + r0;
      end_r = below * a.x_stride + a.k - r0;
      pc = dy + row * a.dy_stride + c0;
      end_c = below * a.dy_stride + a.m - c0;
      qc = act + row * a.act_stride + c0;
      qend_c = below * a.act_stride + a.m - c0;
    }
    if (edge) {
      sr.load_edge(pr, end_r, qr, qend_r, n_rows, depth - t0);
      sc.load_edge(pc, end_c, qc, qend_c, width - c0, depth - t0);
    } else {
      sr.load(pr, qr);
      sc.load(pc, qc);
    }
  };

  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int wr = wave / WAVE_COLS * WM, wc = wave % WAVE_COLS * WN;
  f32x16 acc[FR][FC];
#pragma unroll
  for (int i = 0; i < FR; ++i)
#pragma unroll
    for (int j = 0; j < FC; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
  const bool sum_columns = FORM == kFormDw && a.db && r0 == 0 && skip_r == 0;
  float sums[V] = {};

  auto store = [&]() {
    sr.store(lds_rows);
    sc.store(lds_cols);
    if (FORM == kFormDw && sum_columns) sc.add_columns(sums);
    __syncthreads();
  };
  auto multiply = [&]() {
#pragma unroll
    for (int step = 0; step < D / 16; ++step) {
      bf16x8 fr[FR][P], fc[FC][P];
#pragma unroll
      for (int p = 0; p < P; ++p) {
#pragma unroll
        for (int i = 0; i < FR; ++i) fr[i][p] = Rows::fragment(lds_rows + p * Rows::kElems, wr + i * 32, step);
#pragma unroll
        for (int j = 0; j < FC; ++j) fc[j][p] = Cols::fragment(lds_cols + p * Cols::kElems, wc + j * 32, step);
      }
#pragma unroll
      for (int p = P - 1; p >= 0; --p)
#pragma unroll
        for (int q = P - 1 - p; q >= 0; --q)
#pragma unroll
          for (int i = 0; i < FR; ++i)
#pragma unroll
            for (int j = 0; j < FC; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fc[j][q], fr[i][p], acc[i][j], 0, 0, 0);
    }
    __syncthreads();
  };
  // Inside the tile and the depth no piece is cut; the loop for the others has branches and registers that would slow this one down.
  int t0 = 0;
  if (inside && depth >= D) {
    load(0, false);
    for (; t0 + 2 * D <= depth; t0 += D) {
      store();
      load(t0 + D, false);
      __builtin_amdgcn_sched_barrier(0);                   // the loads go out before the products, not between the last of them
      multiply();
    }
  } else if (depth > 0) {
    load(0, true);
  }
  for (; t0 < depth; t0 += D) {
    sr.cut(n_rows, depth - t0);
    sc.cut(width - c0, depth - t0);
    store();
    if (t0 + D < depth) load(t0 + D, true);
    __builtin_amdgcn_sched_barrier(0);
    multiply();
  }

  // Sums to memory by way of LDS, 64 rows at a time, so that whole lines are read and written: lane l has row l % 32 of a 32 x 32
  // block, and of its columns 8 q + 4 (l / 32) .. + 3 in registers 4 q .. 4 q + 3.  In LDS the 16-byte pieces of a row are permuted
  // by the row, so that neither side meets in a bank.
  float* stage = reinterpret_cast<float*>(lds);            // [64][BN]
  constexpr int VO = kPiece<TO>, kAcross = BN / VO;        // 16 bytes of output a time
#pragma unroll
  for (int i = 0; i < FR; ++i) {
    const int mine = wave / WAVE_COLS * 32 + (lane & 31);
    // the residual is on its way while the sums go through LDS
    constexpr int kEach = 64 * kAcross / THREADS;
    u32x4 res[FORM == kFormY ? kEach : 1];                 // (as it is in memory: what turns it into floats would wait for it)
    if (FORM == kFormY && a.residual && rows.g < a.groups) {
#pragma unroll
      for (int u = 0; u < kEach; ++u) {
        const int p = threadIdx.x + u * THREADS, sr_ = p / kAcross, sc_ = (p % kAcross) * VO;
        const int r = (sr_ >> 5) * WM + i * 32 + (sr_ & 31), c = c0 + sc_;
        const TO* from = (const TO*)a.residual + (int64_t)(r0 + r) * a.residual_stride + c;
        const int count = r >= skip_r && r < n_rows ? width - c : 0;
        if (count >= VO) res[u] = __builtin_bit_cast(u32x4, *reinterpret_cast<const u32x4_any*>(from));
        else res[u] = load_raw_some(from, count);
      }
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < FC; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int piece = (wc + j * 32 + 8 * q) / 4 + (lane >> 5);
        *reinterpret_cast<f32x4*>(stage + mine * BN + ((piece ^ (mine % (BN / 4))) * 4)) =
            f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
      }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kEach; ++u) {
      const int p = threadIdx.x + u * THREADS, sr_ = p / kAcross, sc_ = (p % kAcross) * VO;
      const int r = (sr_ >> 5) * WM + i * 32 + (sr_ & 31), c = c0 + sc_, left = width - c;
      if (r < skip_r || r >= n_rows || left <= 0 || sc_ + VO <= skip_c) continue;
      const int64_t row = r0 + r;
      const int first = max(skip_c - sc_, 0);              // of the piece's elements
      float v[VO];
#pragma unroll
      for (int h = 0; h < VO / 4; ++h) {
        const f32x4 f = *reinterpret_cast<const f32x4*>(stage + sr_ * BN + (((sc_ / 4 + h) ^ (sr_ % (BN / 4))) * 4));
#pragma unroll
        for (int e = 0; e < 4; ++e) v[4 * h + e] = f[e];
      }
      if (FORM == kFormDw) {
        float* out = slot < 0 ? a.dw + (int64_t)rows.g * a.k * a.m : a.part + slot * chunk_stride(a);
        store_part(out + row * a.m + c, first, left, v);
      } else if (FORM == kFormDx) {
        store_part((TO*)a.dx + row * a.dx_stride + c, first, left, v);
      } else {
        const bool in = rows.g < a.groups;
        if (in && a.bias) {
          float b[VO];
          load_some(a.bias + (int64_t)rows.g * a.m + c, left, 0.f, b);
#pragma unroll
          for (int e = 0; e < VO; ++e) v[e] += b[e];
        }
        if (a.relu) {
#pragma unroll
          for (int e = 0; e < VO; ++e) v[e] = relu_of(v[e]);
        }
        if (a.act) store_part((TO*)a.act + row * a.act_stride + c, first, left, v);
        if (in && a.residual) {
#pragma unroll
          for (int e = 0; e < VO; ++e) {
            if constexpr (VO == 4) v[e] += __uint_as_float(res[u][e]);
            else v[e] += e % 2 ? high_bf16(res[u][e / 2]) : low_bf16(res[u][e / 2]);
          }
        }
        store_part((TO*)a.y + row * a.y_stride + c, first, left, v);
      }
    }
  }
  if (FORM == kFormDw && sum_columns) {                    // the threads that have loaded the same columns: their sums through LDS
    constexpr int across = Cols::kAcross, same = THREADS / across;
    float* s = stage;                                      // [same][BN]
    static_assert(same <= 64, "sums of columns fit");
    __syncthreads();
#pragma unroll
    for (int j = 0; j < V; ++j) s[(threadIdx.x / across) * BN + (threadIdx.x % across) * V + j] = sums[j];
    __syncthreads();
    const int c = c0 + threadIdx.x;
    if (threadIdx.x < BN && threadIdx.x >= skip_c && c < a.m) {
      float v = 0.f;
      for (int u = 0; u < same; ++u) v += s[u * BN + threadIdx.x];
      float* out = slot < 0 ? a.db + (int64_t)rows.g * a.m : a.part + slot * chunk_stride(a) + (int64_t)a.k * a.m;
      out[c] = v;
    }
  }
}

template <typename T, typename TO, int FORM, int BM, int BN, bool MASK, int THREADS>
__global__ __launch_bounds__(THREADS, THREADS == 512 ? 2 : MASK ? 2 : 3) void k_linear(LinearArgs a) {
  linear_tile<T, TO, FORM, BM, BN, MASK, THREADS>(a, blockIdx.x);
}

// Adds up the chunks of the groups that have several, and clears the gradients of the empty groups.  A workgroup takes 4 elements of
// the gradient for each of its 256 / SLICES columns of threads; SLICES threads share out an element's chunks (many where there are many
// chunks, so that their loads are under way together), and their sums meet in LDS, in a fixed order.
template <int SLICES>
__global__ __launch_bounds__(256) void k_join_chunks(LinearArgs a) {
  constexpr int kAcross = 256 / SLICES;
  __shared__ f32x4 sums[SLICES][kAcross];
  const int g = blockIdx.y;
  const int64_t km = (int64_t)a.k * a.m, stride = chunk_stride(a), all = km + (a.db ? a.m : 0);
  // the chunks of the groups before this one, and its own
  int lo = 0, hi = 0, end = 0, before = 0;
  const int lane = threadIdx.x & 63;
  for (int base = 0; base <= g; base += 64) {
    const int q = base + lane;
    int e = q <= g ? min(max(a.offsets[q + 1], 0), a.n) : 0;
    e = max(e, end);
    e = wave_scan_max(e);
    int s0 = __shfl_up(e, 1);
    if (lane == 0) s0 = end;
    const int chunks = q <= g ? (int)(((uint32_t)(e - s0) + (uint32_t)a.chunk - 1u) / (uint32_t)a.chunk) : 0;
    const int upto = before + (int)wave_scan_incl((uint32_t)chunks);
    if (g - base < 64) {
      lo = __shfl(upto - chunks, g - base);
      hi = __shfl(upto, g - base);
    }
    before = __shfl(upto, 63);
    end = __shfl(e, 63);
  }
  if (hi - lo == 1) return;                                // written by the one chunk's workgroups
  const int col = threadIdx.x % kAcross, slice = threadIdx.x / kAcross;
  const int64_t at = ((int64_t)blockIdx.x * kAcross + col) * 4;
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  if (at < all) {                                          // (what lies behind the sums is never looked at)
#pragma unroll 4
    for (int s = lo + slice; s < hi; s += SLICES) v += *reinterpret_cast<const f32x4*>(a.part + s * stride + at);
  }
  sums[slice][col] = v;
  __syncthreads();
  if (slice > 0) return;
  for (int s = 1; s < SLICES; ++s) v += sums[s][col];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int64_t i = at + e;
    if (i >= all) break;
    if (i < km) a.dw[g * km + i] = v[e]; else a.db[(int64_t)g * a.m + i - km] = v[e];
  }
}

// db alone: 64 columns of one group to a workgroup, four rows at a time.  A thread adds up 256 rows and then that sum to the others', so that a
// group of n rows is off by (256 + n / 1024 + 4) half steps of the terms' magnitudes at most, not n / 4: 262144 rows of 0.1 came out
// 10359 half steps off in one sequence.  Bound by a thread's loads, one row after the other: for short groups (262144 rows of one group, 64
// outputs float32 take 18.5 ms).
constexpr int kBiasRows = 256;

template <typename T>
__global__ __launch_bounds__(256) void k_bias_grad(LinearArgs a) {
  __shared__ float sums[4][64];
  int lo, hi;
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x < 64) check_offsets(a.offsets, a.groups, a.n, a.err);
  group_rows(a.offsets, a.n, blockIdx.y, &lo, &hi);
  const int lane = threadIdx.x % 64, slice = threadIdx.x / 64, col = blockIdx.x * 64 + lane;
  float s = 0.f;
  if (col < a.m)
    for (int64_t first = lo + slice; first < hi; first += 4 * kBiasRows) {
      const int64_t end = min(first + 4 * kBiasRows, (int64_t)hi);
      float part = 0.f;
      for (int64_t row = first; row < end; row += 4) {
        const float g = to_float(((const T*)a.dy)[row * a.dy_stride + col]);
        part += !a.act || to_float(((const T*)a.act)[row * a.act_stride + col]) > 0.f ? g : 0.f;
      }
      s += part;
    }
  sums[slice][lane] = s;
  __syncthreads();
  if (slice == 0 && col < a.m)
    a.db[(int64_t)blockIdx.y * a.m + col] = (sums[0][lane] + sums[1][lane]) + (sums[2][lane] + sums[3][lane]);
}

}  // namespace sp
