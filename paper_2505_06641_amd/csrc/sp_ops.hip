// C entry points of the operators that train the heads: argument checks, workspace, launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>
#include <cmath>
#include <new>
#include <string>

#include "sneakpeek.h"
#include "sp_host.h"
#include "sp_ops_clip.h"
#include "sp_ops_common.h"
#include "sp_ops_linear.h"
#include "sp_ops_linear_few.h"
#include "sp_ops_loss.h"
#include "sp_ops_norm.h"

using namespace sp;

struct sp_ops {
  int device = 0;
  char* ws = nullptr;              // partial sums
  int64_t ws_bytes = 0;
  uint32_t* err = nullptr;         // behind them: kErr* bits since the last sp_ops_check; those of the last one
  std::string hip_err;
};

namespace {

__global__ void k_ops_report(uint32_t* err) { err[1] = atomicExch(err, 0u); }
__global__ void k_clip_none(float* norm_out) { *norm_out = 0.f; }

bool dtype_ok(int32_t t) { return t == SP_F32 || t == SP_BF16; }
int64_t elem_bytes(int32_t t) { return t == SP_F32 ? 4 : 2; }
// Elements at their own size's multiples; null passes.
bool aligned(const void* p, int32_t t) { return ((uintptr_t)p & (uintptr_t)(elem_bytes(t) - 1)) == 0; }
bool aligned4(const void* p) { return ((uintptr_t)p & 3u) == 0; }

sp_status launched(sp_ops* o) {
  SP_HIP(o, hipGetLastError());
  return SP_OK;
}

// Calls f<TEAM, C>() with the smallest team that holds rows of `pieces` 16-byte pieces: parts of a wavefront for narrow rows, so
// that no lane idles, one wavefront with up to four pieces a lane (a sum over lanes costs a wavefront nothing but its own
// instructions, one over a workgroup two barriers), then workgroups.  False where no team does.
template <typename F>
bool with_team(int64_t pieces, F&& f) {
  if (pieces <= 2) f.template operator()<2, 1>();
  else if (pieces <= 4) f.template operator()<4, 1>();
  else if (pieces <= 8) f.template operator()<8, 1>();
  else if (pieces <= 16) f.template operator()<16, 1>();
  else if (pieces <= 32) f.template operator()<32, 1>();
  else if (pieces <= 64) f.template operator()<64, 1>();
  else if (pieces <= 128) f.template operator()<64, 2>();
  else if (pieces <= 256) f.template operator()<64, 4>();
  else if (pieces <= 512) f.template operator()<256, 2>();
  else if (pieces <= 1024) f.template operator()<256, 4>();
  else if (pieces <= 2048) f.template operator()<1024, 2>();
  else if (pieces <= 4096) f.template operator()<1024, 4>();
  else return false;
  return true;
}

}  // namespace

extern "C" {

sp_status sp_ops_create(int device_id, int64_t workspace_bytes, sp_ops** out) {
  if (!out) return SP_EINVAL;
  *out = nullptr;
  if (workspace_bytes < SP_OPS_MIN_WORKSPACE) return SP_EINVAL;
  int ndev = 0;
  if (hipGetDeviceCount(&ndev) != hipSuccess || device_id < 0 || device_id >= ndev) return SP_EDEVICE;
  sp_ops* o = new (std::nothrow) sp_ops;
  if (!o) return SP_ENOMEM;
  o->device = device_id;
  DeviceGuard g(device_id);
  sp_status rc = g.ok ? SP_OK : SP_EDEVICE;
  auto need = [&](hipError_t e) { if (rc == SP_OK && e != hipSuccess) rc = e == hipErrorOutOfMemory ? SP_ENOMEM : SP_EDEVICE; };
  const int64_t bytes = (workspace_bytes + 255) / 256 * 256;
  const uint32_t none[2] = {0u, 0u};
  if (rc == SP_OK) need(hipMalloc((void**)&o->ws, (size_t)bytes + sizeof(none)));
  if (rc == SP_OK) {
    o->ws_bytes = workspace_bytes;
    o->err = reinterpret_cast<uint32_t*>(o->ws + bytes);
    need(hipMemcpy(o->err, none, sizeof(none), hipMemcpyHostToDevice));
  }
  if (rc != SP_OK) {
    sp_ops_destroy(o);
    return rc;
  }
  *out = o;
  return SP_OK;
}

void sp_ops_destroy(sp_ops* o) {
  if (!o) return;
  DeviceGuard g(o->device);
  (void)hipDeviceSynchronize();
  if (o->ws) (void)hipFree(o->ws);
  delete o;
}

const char* sp_ops_last_hip_error(const sp_ops* o) { return o ? o->hip_err.c_str() : ""; }

sp_status sp_ops_check(sp_ops* o, void* stream) {
  if (!o) return SP_EINVAL;
  DeviceGuard g(o->device);
  if (!g.ok) return SP_EDEVICE;
  hipStream_t s = (hipStream_t)stream;
  uint32_t seen = 0u;
  hipLaunchKernelGGL(k_ops_report, dim3(1), dim3(1), 0, s, o->err);
  SP_HIP(o, hipGetLastError());
  SP_HIP(o, hipMemcpyAsync(&seen, o->err + 1, sizeof(seen), hipMemcpyDeviceToHost, s));
  SP_HIP(o, hipStreamSynchronize(s));
  return seen ? SP_EINVAL : SP_OK;
}

sp_status sp_layer_norm(sp_ops* o, int32_t n, int32_t d, int32_t dtype, const void* x, int64_t x_stride, const float* gamma,
                        const float* beta, float eps, void* y, int64_t y_stride, float* mean_out, float* rstd_out, void* stream) {
  if (!o || n < 0 || d < 1 || !dtype_ok(dtype) || x_stride < d || y_stride < d || !(eps >= 0.f) || !std::isfinite(eps)) return SP_EINVAL;
  if (n > 0 && (!x || !y)) return SP_EINVAL;
  if (!aligned(x, dtype) || !aligned(y, dtype) || !aligned4(gamma) || !aligned4(beta) || !aligned4(mean_out) || !aligned4(rstd_out))
    return SP_EINVAL;
  if (d > SP_MAX_NORM_DIM) return SP_ECAPACITY;
  if (n == 0) return SP_OK;
  DeviceGuard g(o->device);
  if (!g.ok) return SP_EDEVICE;
  auto run = [&]<typename T>() {
    with_team((d + kPiece<T> - 1) / kPiece<T>, [&]<int TEAM, int C>() {
      if constexpr (TEAM * C * kPiece<T> <= SP_MAX_NORM_DIM) {
        constexpr int threads = kTeamThreads<TEAM>, rows = threads / TEAM;
        const int blocks = (int)std::min<int64_t>(((int64_t)n + rows - 1) / rows, kNormBlocks);
        hipLaunchKernelGGL((d % kPiece<T> ? k_norm<T, TEAM, C, false> : k_norm<T, TEAM, C, true>), dim3(blocks), dim3(threads), 0, (hipStream_t)stream, n, d, (const T*)x, x_stride, gamma,
                           beta, eps, (T*)y, y_stride, mean_out, rstd_out);
      }
    });
  };
  if (dtype == SP_F32) run.template operator()<float>(); else run.template operator()<bf16>();
  return launched(o);
}

sp_status sp_layer_norm_backward(sp_ops* o, int32_t n, int32_t d, int32_t dtype, const void* dy, int64_t dy_stride, const void* x,
                                 int64_t x_stride, const float* gamma, const float* mean, const float* rstd, void* dx, int64_t dx_stride,
                                 float* dgamma, float* dbeta, void* stream) {
  if (!o || n < 0 || d < 1 || !dtype_ok(dtype) || dy_stride < d || x_stride < d || (dx && dx_stride < d)) return SP_EINVAL;
  if (n > 0 && (!dy || !x || !mean || !rstd)) return SP_EINVAL;
  if (!aligned(x, dtype) || !aligned(dy, dtype) || !aligned(dx, dtype) || !aligned4(gamma) || !aligned4(mean) || !aligned4(rstd) ||
      !aligned4(dgamma) || !aligned4(dbeta))
    return SP_EINVAL;
  if (d > SP_MAX_NORM_DIM) return SP_ECAPACITY;
  const bool sums = dgamma || dbeta;
  if ((n == 0 || !dx) && !sums) return SP_OK;
  DeviceGuard g(o->device);
  if (!g.ok) return SP_EDEVICE;
  const int64_t most = o->ws_bytes / (norm_part_stride(d) * (int64_t)sizeof(float));
  int parts = 0;
  if (n > 0) {
    auto run = [&]<typename T>() {
      with_team((d + kPiece<T> - 1) / kPiece<T>, [&]<int TEAM, int C>() {
        if constexpr (TEAM * C * kPiece<T> <= SP_MAX_NORM_DIM) {
          constexpr int threads = kTeamThreads<TEAM>, rows = threads / TEAM;
          parts = (int)std::min<int64_t>({((int64_t)n + rows - 1) / rows, kNormBackBlocks, sums ? most : kNormBackBlocks});
          if (parts <= 4) parts = 1;           // one workgroup in up to four turns: no sums to be joined by a second launch
          hipLaunchKernelGGL((d % kPiece<T> ? k_norm_back<T, TEAM, C, false> : k_norm_back<T, TEAM, C, true>), dim3(parts), dim3(threads), 0, (hipStream_t)stream, n, d, (const T*)dy, dy_stride,
                             (const T*)x, x_stride, gamma, mean, rstd, (T*)dx, dx_stride, sums && parts > 1 ? (float*)o->ws : nullptr,
                             parts > 1 ? nullptr : dgamma, parts > 1 ? nullptr : dbeta);
        }
      });
    };
    if (dtype == SP_F32) run.template operator()<float>(); else run.template operator()<bf16>();
  }
  if (sums && parts != 1)                      // (without rows: zeros)
    hipLaunchKernelGGL(k_norm_join, dim3((2 * d + 31) / 32), dim3(256), 0, (hipStream_t)stream, parts, d, (const float*)o->ws, dgamma,
                       dbeta);
  return launched(o);
}

sp_status sp_cross_entropy(sp_ops* o, int32_t n, int32_t c_max, int32_t dtype, const void* logits, int64_t logits_stride, int32_t n_apps,
                           const int32_t* app, const int32_t* n_classes, const int32_t* label, const float* weight, float scale,
                           float* loss, int32_t grad_dtype, void* dlogits, int64_t dlogits_stride, void* stream) {
  if (!o || n < 0 || c_max < 1 || !dtype_ok(dtype) || logits_stride < c_max || !std::isfinite(scale)) return SP_EINVAL;
  if (dlogits && (!dtype_ok(grad_dtype) || dlogits_stride < c_max || (dtype == SP_BF16 && grad_dtype == SP_F32))) return SP_EINVAL;
  if (app ? !n_classes || n_apps < 1 : n_classes && n > 0) return SP_EINVAL;       // (an array of no rows may have no address)
  if (n > 0 && (!logits || !label || !loss)) return SP_EINVAL;
  if (!aligned(logits, dtype) || (dlogits && !aligned(dlogits, grad_dtype)) || !aligned4(app) || !aligned4(n_classes) || !aligned4(label) ||
      !aligned4(weight) || !aligned4(loss))
    return SP_EINVAL;
  if (n == 0) return SP_OK;
  DeviceGuard g(o->device);
  if (!g.ok) return SP_EDEVICE;
  auto run = [&]<typename T, typename TO>() {
    const bool fits = with_team(((int64_t)c_max + kPiece<T> - 1) / kPiece<T>, [&]<int TEAM, int C>() {
      constexpr int threads = kTeamThreads<TEAM>, rows = threads / TEAM;
      const int blocks = (int)std::min<int64_t>(((int64_t)n + rows - 1) / rows, kLossBlocks);
      hipLaunchKernelGGL((k_loss<T, TO, TEAM, C>), dim3(blocks), dim3(threads), 0, (hipStream_t)stream, n, c_max, (const T*)logits,
                         logits_stride, n_apps, app, n_classes, label, weight, scale, loss, (TO*)dlogits, dlogits_stride, o->err);
    });
    if (!fits)
      hipLaunchKernelGGL((k_loss_wide<T, TO>), dim3(std::min(n, kLossBlocks)), dim3(1024), 0, (hipStream_t)stream, n, c_max,
                         (const T*)logits, logits_stride, n_apps, app, n_classes, label, weight, scale, loss, (TO*)dlogits,
                         dlogits_stride, o->err);
  };
  if (dtype == SP_BF16) run.template operator()<bf16, bf16>();
  else if (dlogits && grad_dtype == SP_BF16) run.template operator()<float, bf16>();
  else run.template operator()<float, float>();
  return launched(o);
}

sp_status sp_clip_grad_norm(sp_ops* o, int32_t n_tensors, int32_t dtype, const void* const* grads, const int64_t* sizes, float max_norm,
                            void* const* out, float* norm_out, void* stream) {
  if (!o || n_tensors < 0 || !dtype_ok(dtype) || !norm_out || !aligned4(norm_out) || !(max_norm >= 0.f) || !std::isfinite(max_norm))
    return SP_EINVAL;
  if (n_tensors > 0 && (!grads || !sizes)) return SP_EINVAL;
  int64_t total = 0, pieces = 0;
  for (int i = 0; i < n_tensors; ++i) {
    if (sizes[i] < 0 || (sizes[i] > 0 && (!grads[i] || (out && !out[i])))) return SP_EINVAL;
    if (!aligned(grads[i], dtype) || (out && !aligned(out[i], dtype))) return SP_EINVAL;
  }
  for (int i = 0; i < n_tensors; ++i) {
    if (sizes[i] > ((int64_t)1 << 44)) return SP_ECAPACITY;
    total += sizes[i];
    if (total > ((int64_t)1 << 46)) return SP_ECAPACITY;
  }
  // some 2,000 workgroups share the elements, but none gets less than is worth a workgroup
  int piece = (int)std::clamp<int64_t>((total / 2048 + 4095) / 4096 * 4096, kClipPieceMin, kClipPieceMax);
  for (int i = 0; i < n_tensors; ++i) pieces += (sizes[i] + piece - 1) / piece;
  if (pieces > INT_MAX || pieces * (int64_t)sizeof(double) > o->ws_bytes) return SP_ECAPACITY;
  const int vec = (int)(16 / elem_bytes(dtype));
  const bool few = n_tensors <= kClipTensors && total / vec + n_tensors <= kClipThreads * kClipFewEach;
  if (few) piece = vec;
  DeviceGuard g(o->device);
  if (!g.ok) return SP_EDEVICE;
  hipStream_t s = (hipStream_t)stream;
  double* part = (double*)o->ws;
  if (pieces == 0) {
    hipLaunchKernelGGL(k_clip_none, dim3(1), dim3(1), 0, s, norm_out);
    return launched(o);
  }
  // Tables from the first tensor on for the sums; back again for the scaling, whose first reads the last-level cache then still holds.
  auto fill = [&](ClipTable* tb, int* from, int dir) {
    int64_t k = 0;
    tb->count = 0;
    tb->piece = piece;
    for (; *from >= 0 && *from < n_tensors && tb->count < kClipTensors; *from += dir) {
      const int i = *from;
      if (sizes[i] == 0) continue;
      tb->src[tb->count] = grads[i];
      tb->dst[tb->count] = out ? out[i] : const_cast<void*>(grads[i]);
      tb->size[tb->count] = sizes[i];
      tb->first[tb->count++] = (int32_t)k;
      k += (sizes[i] + piece - 1) / piece;
    }
    tb->first[tb->count] = (int32_t)k;
    return (unsigned)k;
  };
  int64_t done = 0;
  ClipTable tb;
  for (int at = 0; at < n_tensors && !few;) {
    const unsigned k = fill(&tb, &at, 1);
    if (k == 0) continue;
    if (dtype == SP_F32) hipLaunchKernelGGL(k_clip_sum<float>, dim3(k), dim3(kClipThreads), 0, s, tb, part + done);
    else hipLaunchKernelGGL(k_clip_sum<bf16>, dim3(k), dim3(kClipThreads), 0, s, tb, part + done);
    SP_HIP(o, hipGetLastError());
    done += k;
  }
  float* norm = norm_out;                // written by the first of the launches
  for (int at = n_tensors - 1; at >= 0;) {
    const unsigned k = fill(&tb, &at, -1);
    if (k == 0) continue;
    if (few && dtype == SP_F32) hipLaunchKernelGGL(k_clip_few<float>, dim3(1), dim3(kClipThreads), 0, s, tb, max_norm, norm);
    else if (few) hipLaunchKernelGGL(k_clip_few<bf16>, dim3(1), dim3(kClipThreads), 0, s, tb, max_norm, norm);
    else if (dtype == SP_F32) hipLaunchKernelGGL(k_clip_scale<float>, dim3(k), dim3(kClipThreads), 0, s, tb, (int)pieces, part, max_norm, norm);
    else hipLaunchKernelGGL(k_clip_scale<bf16>, dim3(k), dim3(kClipThreads), 0, s, tb, (int)pieces, part, max_norm, norm);
    SP_HIP(o, hipGetLastError());
    norm = nullptr;
  }
  return SP_OK;
}

}  // extern "C"

namespace {

// Whether a layer is better off in pieces of 16 rows than in tiles of 128: as long as the device holds about all of the small pieces'
// workgroups at once, their shorter way through the depth wins (bfloat16 1024 -> 1024: 512 rows 15 us against 17, 1024 rows 24 against 17;
// float32: 1024 rows 52 against 66, 2048 rows 93 against 67; 512 -> 256 of one request: 5 against 14).  bfloat16's smaller bound is that of
// float32 where one turn of dx's wavefronts covers the depth (gradients of 4096 rows, 128 -> 64 with a mask 12.9 us against 15.9, 2048 rows,
// 256 -> 64 11.8 against 14.8; but of 600 rows, 1024 -> 256 25 against 23).
bool few_rows(int64_t n, int64_t width, int cols, int64_t groups, int32_t dtype, int64_t depth) {
  const int64_t workgroups = ((n + kFewRows - 1) / kFewRows + std::min(n, groups)) * ((width + cols - 1) / cols);
  return workgroups <= (dtype == SP_F32 || (cols == kFewDxCols && depth <= kFewDxThreads / 64 * 32) ? 2560 : 1280);
}

// Rows of a group that one workgroup adds up for dW (0: all).  A workgroup takes about 19 ns a row (float32 55 ns), and every chunk's
// sums are written and read again at about 4 TB/s: the number of rows at which both cost the same, but not so many that the device runs
// empty, nor so few that the workgroups wait in line.
int dw_chunk(const sp_ops* o, const LinearArgs& a, int64_t tiles, int32_t dtype) {
  const double n = a.n, sums = 8.0 * (double)chunk_stride(a) / 4e12, row = dtype == SP_F32 ? 55e-9 : 19e-9;
  int64_t chunk = (int64_t)std::sqrt(n * sums / row);
  chunk = std::clamp<int64_t>(chunk, a.n * tiles / 2048, std::max<int64_t>(a.n * tiles / 2048, a.n * tiles / 256));
  chunk = (std::max<int64_t>(chunk, 64) + 63) / 64 * 64;
  const int64_t most = o->ws_bytes / (chunk_stride(a) * (int64_t)sizeof(float)) - a.groups;    // chunks: at most n / chunk + groups
  if (most <= 0 || chunk_stride(a) > INT_MAX) return 0;          // (the join has a thread to each of a chunk's sums)
  chunk = std::max(chunk, ((int64_t)a.n + most - 1) / most);
  return chunk < a.n ? (int)chunk : 0;
}

// Tiles of at most `rows` rows that n rows can make: a tile holds rows of one group or of none, and no more groups have any than there
// are rows.  Up to eight more where there are groups without rows: with them the tiles that share rows stay on one die (a request of one
// of eight groups, 512 -> 256 bfloat16: 4.2 us, on eight dies 4.45).
int64_t most_row_tiles(int64_t n, int64_t groups, int64_t rows) {
  return std::min((n + rows - 1) / rows + groups, (n + std::min(n, groups + 1) * (rows - 1)) / rows + kXcds);
}

// The launch's tiles; false where there are more than a launch holds, whose threads are counted in 32 bits.
bool linear_grid(LinearArgs* a, int64_t row_tiles, int64_t col_tiles, int threads) {
  if ((row_tiles * col_tiles + kXcds) * threads > UINT32_MAX) return false;
  a->row_tiles = (int)row_tiles;
  a->col_tiles = (int)col_tiles;
  return true;
}
int linear_blocks(const LinearArgs& a) { return (a.row_tiles * a.col_tiles + kXcds - 1) / kXcds * kXcds; }
void launch_linear(void (*kernel)(LinearArgs), int threads, const LinearArgs& a, void* stream) {
  hipLaunchKernelGGL(kernel, dim3((unsigned)linear_blocks(a)), dim3(threads), 0, (hipStream_t)stream, a);
}

// Rows and columns of the tiles of an output: 64 where it is no wider.
int tile_rows(int64_t k) { return k <= 64 ? 64 : 128; }           // dW's rows are inputs; the other forms' rows are requests: 128
int tile_cols(int64_t width) { return width <= 64 ? 64 : 128; }

// Tiles of 128 by 128 have eight wavefronts where the device holds all of them at once, or where there is a mask, else four.
int many_tiles_threads(int bm, int bn, bool mask) { return mask && bm == 128 && bn == 128 ? 512 : 256; }
template <typename T, typename TO, int FORM, bool MASK>
void launch_tiles(int bm, int bn, const LinearArgs& a, void* stream) {
  if constexpr (FORM == kFormDw) {
    if (bm == 64) {
      if (bn == 64) launch_linear(k_linear<T, TO, FORM, 64, 64, MASK, 256>, 256, a, stream);
      else launch_linear(k_linear<T, TO, FORM, 64, 128, MASK, 256>, 256, a, stream);
      return;
    }
  }
  if (bn == 64) {
    launch_linear(k_linear<T, TO, FORM, 128, 64, MASK, 256>, 256, a, stream);
  } else if constexpr (MASK) {
    launch_linear(k_linear<T, TO, FORM, 128, 128, MASK, 512>, 512, a, stream);
  } else if ((int64_t)a.row_tiles * a.col_tiles <= 768) {
    launch_linear(k_linear<T, TO, FORM, 128, 128, MASK, 512>, 512, a, stream);
  } else {
    launch_linear(k_linear<T, TO, FORM, 128, 128, MASK, 256>, 256, a, stream);
  }
}

// Shared checks of the grouped linear layers.
sp_status linear_sizes(const sp_ops* o, int32_t n, int32_t k, int32_t m, int32_t groups, int32_t dtype) {
  if (!o || n < 0 || k < 1 || m < 1 || groups < 1 || !dtype_ok(dtype)) return SP_EINVAL;
  if (groups > SP_MAX_APPS || k > SP_MAX_LINEAR_DIM || m > SP_MAX_LINEAR_DIM) return SP_ECAPACITY;
  return SP_OK;
}

}  // namespace

extern "C" {

sp_status sp_grouped_linear(sp_ops* o, int32_t n, int32_t k, int32_t m, int32_t groups, int32_t dtype, const void* x, int64_t x_stride,
                            const int32_t* offsets, const void* w, const float* bias, int32_t activation, int32_t out_dtype,
                            const void* residual, int64_t residual_stride, void* y, int64_t y_stride, void* act_out,
                            int64_t act_stride, void* stream) {
  const sp_status bad = linear_sizes(o, n, k, m, groups, dtype);
  if (bad != SP_OK) return bad;
  if (x_stride < k || y_stride < m || (residual && residual_stride < m) || (act_out && act_stride < m)) return SP_EINVAL;
  if (activation != SP_ACT_NONE && activation != SP_ACT_RELU) return SP_EINVAL;
  if (!dtype_ok(out_dtype) || (dtype == SP_F32 && out_dtype == SP_BF16)) return SP_EINVAL;
  if (n > 0 && (!x || !offsets || !w || !y)) return SP_EINVAL;
  if (!aligned(x, dtype) || !aligned(w, dtype) || !aligned(y, out_dtype) || !aligned(residual, out_dtype) || !aligned(act_out, out_dtype) ||
      !aligned4(offsets) || !aligned4(bias))
    return SP_EINVAL;
  if (x_stride > SP_MAX_LINEAR_STRIDE) return SP_ECAPACITY;
  if (n == 0) return SP_OK;
  LinearArgs a{};
  a.n = n; a.k = k; a.m = m; a.groups = groups; a.x = x; a.x_stride = x_stride; a.offsets = offsets; a.w = w; a.bias = bias;
  a.relu = activation == SP_ACT_RELU; a.residual = residual; a.residual_stride = residual_stride; a.y = y; a.y_stride = y_stride;
  a.act = act_out; a.act_stride = act_stride; a.err = o->err;
  const bool few = few_rows(n, m, kFewCols, groups, dtype, k);
  const int bn = tile_cols(m);
  if (few ? !linear_grid(&a, most_row_tiles(n, groups, kFewRows), (m + kFewCols - 1) / kFewCols, kFewThreads)
          : !linear_grid(&a, most_row_tiles(n, groups, 128), (m + bn - 1) / bn, many_tiles_threads(128, bn, false)))
    return SP_ECAPACITY;
  DeviceGuard g(o->device);
  if (!g.ok) return SP_EDEVICE;
  if (few) {
    if (dtype == SP_F32) launch_linear(k_linear_few<float, float>, kFewThreads, a, stream);
    else if (out_dtype == SP_F32) launch_linear(k_linear_few<bf16, float>, kFewThreads, a, stream);
    else launch_linear(k_linear_few<bf16, bf16>, kFewThreads, a, stream);
    return launched(o);
  }
  auto run = [&]<typename T, typename TO>() {
    launch_tiles<T, TO, kFormY, false>(128, bn, a, stream);
  };
  if (dtype == SP_F32) run.template operator()<float, float>();
  else if (out_dtype == SP_F32) run.template operator()<bf16, float>();
  else run.template operator()<bf16, bf16>();
  return launched(o);
}

sp_status sp_grouped_linear_backward(sp_ops* o, int32_t n, int32_t k, int32_t m, int32_t groups, int32_t dtype, const void* dy,
                                     int64_t dy_stride, const void* act, int64_t act_stride, const void* x, int64_t x_stride,
                                     const int32_t* offsets, const void* w, void* dx, int64_t dx_stride, float* dw, float* db,
                                     void* stream) {
  const sp_status bad = linear_sizes(o, n, k, m, groups, dtype);
  if (bad != SP_OK) return bad;
  if (dy_stride < m || (act && act_stride < m) || (dw && x_stride < k) || (dx && dx_stride < k)) return SP_EINVAL;
  if (!offsets || (n > 0 && (!dy || (dx && !w) || (dw && !x)))) return SP_EINVAL;
  if (!aligned(dy, dtype) || !aligned(act, dtype) || !aligned(x, dtype) || !aligned(w, dtype) || !aligned(dx, dtype) || !aligned4(offsets) ||
      !aligned4(dw) || !aligned4(db))
    return SP_EINVAL;
  if (dy_stride > SP_MAX_LINEAR_STRIDE || (act && act_stride > SP_MAX_LINEAR_STRIDE) || (dw && x_stride > SP_MAX_LINEAR_STRIDE))
    return SP_ECAPACITY;
  if ((n == 0 || !dx) && !dw && !db) return SP_OK;
  LinearArgs a{};
  a.n = n; a.k = k; a.m = m; a.groups = groups; a.x = x; a.x_stride = x_stride; a.offsets = offsets; a.w = w;
  a.act = const_cast<void*>(act); a.act_stride = act_stride; a.dy = dy; a.dy_stride = dy_stride; a.dx = dx; a.dx_stride = dx_stride;
  a.dw = dw; a.db = db; a.err = o->err;
  hipStream_t s = (hipStream_t)stream;
  // both products' launches, before either is made
  const bool want_dx = dx && n > 0, few = want_dx && few_rows(n, k, kFewDxCols, groups, dtype, m);
  const int dx_cols = tile_cols(k), dw_rows = tile_rows(k), dw_cols = tile_cols(m);
  LinearArgs ax = a, aw = a;
  if (few && !linear_grid(&ax, most_row_tiles(n, groups, kFewRows), (k + kFewDxCols - 1) / kFewDxCols, kFewDxThreads)) return SP_ECAPACITY;
  if (want_dx && !few &&
      !linear_grid(&ax, most_row_tiles(n, groups, 128), (k + dx_cols - 1) / dx_cols, many_tiles_threads(128, dx_cols, act != nullptr)))
    return SP_ECAPACITY;
  if (dw) {
    const int64_t k_tiles = (k + dw_rows - 1) / dw_rows, m_tiles = (m + dw_cols - 1) / dw_cols;
    aw.chunk = dw_chunk(o, a, k_tiles * m_tiles, dtype);
    aw.part = (float*)o->ws;
    if (!linear_grid(&aw, (aw.chunk ? ((int64_t)n + aw.chunk - 1) / aw.chunk + groups : groups) * k_tiles, m_tiles,
                     many_tiles_threads(dw_rows, dw_cols, act != nullptr)))
      return SP_ECAPACITY;
  }
  DeviceGuard g(o->device);
  if (!g.ok) return SP_EDEVICE;
  const int dx_blocks = few ? linear_blocks(ax) : 0, dw_blocks = dw ? linear_blocks(aw) : 0;
  // (two or three workgroups to a compute unit: all of dW's run at once, or nearly)
  const bool together = few && dw && dw_blocks <= 768;
  auto run = [&]<typename T, bool MASK>() {
    if (together) {
      const dim3 grid((unsigned)(dx_blocks + dw_blocks));
      auto both = dw_rows == 64 ? (dw_cols == 64 ? k_linear_few_back<T, 64, 64, MASK> : k_linear_few_back<T, 64, 128, MASK>)
                                : (dw_cols == 64 ? k_linear_few_back<T, 128, 64, MASK> : k_linear_few_back<T, 128, 128, MASK>);
      hipLaunchKernelGGL(both, grid, dim3(kFewDxThreads), 0, s, ax, aw, dw_blocks);
    } else {
      if (few) launch_linear(k_linear_few_dx<T>, kFewDxThreads, ax, stream);
      else if (want_dx) launch_tiles<T, T, kFormDx, MASK>(128, dx_cols, ax, stream);
      if (dw) launch_tiles<T, float, kFormDw, MASK>(dw_rows, dw_cols, aw, stream);
    }
    if (dw && aw.chunk) {
      const int64_t elems = (int64_t)k * m + (db ? m : 0);
      // few elements: what fills the device is that many threads share an element's chunks
      if (elems * groups < 512 * 256 && (n + aw.chunk - 1) / aw.chunk >= 8 * (int64_t)groups)
        hipLaunchKernelGGL(k_join_chunks<32>, dim3((unsigned)((elems + 31) / 32), groups), dim3(256), 0, s, aw);
      else
        hipLaunchKernelGGL(k_join_chunks<4>, dim3((unsigned)((elems + 255) / 256), groups), dim3(256), 0, s, aw);
    }
    if (db && !dw) hipLaunchKernelGGL((k_bias_grad<T>), dim3((m + 63) / 64, groups), dim3(256), 0, s, a);
  };
  if (dtype == SP_F32 && act) run.template operator()<float, true>();
  else if (dtype == SP_F32) run.template operator()<float, false>();
  else if (act) run.template operator()<bf16, true>();
  else run.template operator()<bf16, false>();
  return launched(o);
}

}  // extern "C"
