// C entry points of the operators for heads that are made of experts: argument checks, workspace, launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>
#include <cmath>

#include "sneakpeek.h"
#include "sp_host.h"
#include "sp_ops_common.h"
#include "sp_ops_dropout.h"
#include "sp_ops_host.h"
#include "sp_ops_move.h"
#include "sp_ops_quantized.h"
#include "sp_ops_route.h"

using namespace sp;

static_assert(kMaxExperts == SP_MAX_EXPERTS, "a launch's counters hold all experts");
static_assert(SP_MAX_EXPERTS <= 64 * 16, "a wavefront's lanes hold a row of logits");
static_assert(SP_MAX_EXPERTS <= 64 * 2 * kPiece<bf16> && SP_MAX_EXPERTS <= 64 * 4 * kPiece<float>, "the router's gradient holds a row in a wavefront");

namespace {

bool score_ok(int32_t s) { return s == SP_SCORE_SOFTMAX || s == SP_SCORE_SIGMOID; }

int power_from(int v) {                // the power of two from v on
  int p = 1;
  while (p < v) p *= 2;
  return p;
}

// Calls f<T>() with the element type.
template <typename F>
void with_type(int32_t dtype, F&& f) {
  if (dtype == SP_F32) f.template operator()<float>();
  else f.template operator()<bf16>();
}

}  // namespace

extern "C" {

sp_status sp_route(sp_ops* o, int32_t n, int32_t experts, int32_t top, int32_t dtype, const void* logits, int64_t logits_stride, int32_t score,
                   const float* bias, int32_t groups, int32_t top_groups, int32_t renormalize, float scale, int32_t* expert, float* weight,
                   void* stream) {
  if (!o || n < 0 || experts < 1 || top < 1 || top > experts || !dtype_ok(dtype) || logits_stride < experts || !score_ok(score)) return SP_EINVAL;
  if (groups < 1 || experts % groups != 0 || top_groups < 1 || top_groups > groups || (int64_t)top_groups * (experts / groups) < top) return SP_EINVAL;
  if (!std::isfinite(scale) || (n > 0 && (!logits || !expert || !weight))) return SP_EINVAL;
  if (!aligned(logits, dtype) || !aligned4(bias) || !aligned4(expert) || !aligned4(weight)) return SP_EINVAL;
  if (experts > SP_MAX_EXPERTS || top > SP_MAX_TOP || groups > SP_MAX_EXPERT_GROUPS) return SP_ECAPACITY;
  if (n == 0) return SP_OK;
  RouteArgs a{};
  a.n = n; a.experts = experts; a.top = top; a.groups = groups; a.top_groups = top_groups; a.width = experts / groups;
  a.group_lanes = 64 / power_from(groups);
  a.sigmoid = score == SP_SCORE_SIGMOID; a.renormalize = renormalize != 0; a.scale = scale;
  a.z = logits; a.z_stride = logits_stride; a.bias = bias; a.expert = expert; a.weight = weight; a.err = o->err;
  DeviceGuard g(o->device);
  if (!g.ok) return SP_EDEVICE;
  const int power = power_from(groups);
  auto per_lane = [&](int team) { return (a.width + team / power - 1) / (team / power); };
  // a wavefront to a row while the device holds about all of them at once: 2048 rows of 64 bfloat16 experts 4.0 us either way, 16384 rows 4.3 us in
  // teams of 8 and 11.7 in wavefronts; 256 rows of 256 experts in groups 8.0 us and 5.8
  const bool narrow = experts <= 256 && top <= 8 && groups <= 8 && per_lane(8) <= 32 && n > 2048;
  const int team = narrow ? 8 : 64, per = per_lane(team), rows = 4 * 64 / team;
  const dim3 grid((unsigned)std::min<int64_t>(((int64_t)n + rows - 1) / rows, 2048));
  with_type(dtype, [&]<typename T>() {
    auto kernel = [&]<bool BY_LOGIT>() {
      return narrow ? (per <= 1    ? k_route<T, 8, 1, BY_LOGIT>
                       : per <= 2  ? k_route<T, 8, 2, BY_LOGIT>
                       : per <= 4  ? k_route<T, 8, 4, BY_LOGIT>
                       : per <= 8  ? k_route<T, 8, 8, BY_LOGIT>
                       : per <= 16 ? k_route<T, 8, 16, BY_LOGIT>
                                   : k_route<T, 8, 32, BY_LOGIT>)
                    : (per <= 1    ? k_route<T, 64, 1, BY_LOGIT>
                       : per <= 2  ? k_route<T, 64, 2, BY_LOGIT>
                       : per <= 4  ? k_route<T, 64, 4, BY_LOGIT>
                       : per <= 8  ? k_route<T, 64, 8, BY_LOGIT>
                       : BY_LOGIT || per <= 16 ? k_route<T, 64, 16, BY_LOGIT>                        // (without groups a lane has at most 16)
                                               : k_route<T, 64, BY_LOGIT ? 16 : 32, BY_LOGIT>);
    };
    hipLaunchKernelGGL((bias || groups > 1 ? kernel.template operator()<false>() : kernel.template operator()<true>()), grid, dim3(256), 0,
                       (hipStream_t)stream, a);
  });
  return launched(o);
}

sp_status sp_route_backward(sp_ops* o, int32_t n, int32_t experts, int32_t top, int32_t dtype, const void* logits, int64_t logits_stride,
                            int32_t score, int32_t renormalize, float scale, const int32_t* expert, const float* dweight, void* dlogits,
                            int64_t dlogits_stride, void* stream) {
  if (!o || n < 0 || experts < 1 || top < 1 || top > experts || !dtype_ok(dtype) || logits_stride < experts || dlogits_stride < experts ||
      !score_ok(score))
    return SP_EINVAL;
  if (!std::isfinite(scale) || (n > 0 && (!logits || !expert || !dweight || !dlogits))) return SP_EINVAL;
  if (!aligned(logits, dtype) || !aligned(dlogits, dtype) || !aligned4(expert) || !aligned4(dweight)) return SP_EINVAL;
  if (experts > SP_MAX_EXPERTS || top > SP_MAX_TOP) return SP_ECAPACITY;
  if (n == 0) return SP_OK;
  DeviceGuard g(o->device);
  if (!g.ok) return SP_EDEVICE;
  with_type(dtype, [&]<typename T>() {
    auto run = [&]<int TEAM, int C>() {
      constexpr int rows = 256 / TEAM;
      const dim3 grid((unsigned)std::min<int64_t>(((int64_t)n + rows - 1) / rows, 8192));
      hipLaunchKernelGGL((k_route_back<T, TEAM, C>), grid, dim3(256), 0, (hipStream_t)stream, n, experts, top, (const T*)logits, logits_stride,
                         score == SP_SCORE_SIGMOID, renormalize != 0, scale, expert, dweight, (T*)dlogits, dlogits_stride, o->err);
    };
    const int lanes = std::max((experts + kPiece<T> - 1) / kPiece<T>, top);        // (a lane for every chosen expert)
    if (lanes <= 8) run.template operator()<8, 1>();
    else if (lanes <= 16) run.template operator()<16, 1>();
    else if (lanes <= 32) run.template operator()<32, 1>();
    else if (lanes <= 64) run.template operator()<64, 1>();
    else if (sizeof(T) == 2 || lanes <= 128) run.template operator()<64, 2>();          // (SP_MAX_EXPERTS bfloat16 are 128 pieces)
    else if constexpr (sizeof(T) == 4) run.template operator()<64, 4>();
  });
  return launched(o);
}

sp_status sp_route_order(sp_ops* o, int32_t n, int32_t top, int32_t experts, const int32_t* expert, int32_t* offsets, int32_t* place, void* stream) {
  if (!o || n < 0 || top < 1 || experts < 1 || !offsets || (n > 0 && (!expert || !place))) return SP_EINVAL;
  if (!aligned4(expert) || !aligned4(offsets) || !aligned4(place)) return SP_EINVAL;
  const int64_t pairs = (int64_t)n * top;
  if (experts > SP_MAX_EXPERTS || top > SP_MAX_TOP || pairs > INT32_MAX) return SP_ECAPACITY;
  int bits = 0;
  while ((1 << bits) < experts) ++bits;
  // One launch whose workgroups each look through all pairs, up to 8192 of them (5.0 us against 6.1; 16388 pairs 6.5 against 6.4, 32768 9.7 against 7.0);
  // else as many tiles as have 65536 counts together, up to one to every half of a compute unit (2097152 pairs of 256 experts: 64 tiles 41.6 us, 256
  // 20.3, 512 29.3; 524288 of 1000: 64 tiles 20.4, 256 27.5; 8000000 of 128: 256 tiles 57.5, 512 46.9).
  const int64_t most = std::clamp(65536 / experts, 64, 512);
  const bool few = pairs <= 8192;
  const int64_t tile = few ? 1024 : std::max<int64_t>(((pairs + most - 1) / most + 1023) / 1024 * 1024, 1024);
  const int tiles = (int)std::max<int64_t>(1, (pairs + tile - 1) / tile);
  if (!few && (int64_t)tiles * experts * 4 > o->ws_bytes) return SP_ECAPACITY;
  int32_t* counts = few ? nullptr : (int32_t*)o->ws;
  DeviceGuard g(o->device);
  if (!g.ok) return SP_EDEVICE;
  hipStream_t s = (hipStream_t)stream;
  if (!few) hipLaunchKernelGGL(k_order_count, dim3(tiles), dim3(kOrderThreads), 0, s, pairs, (int)tile, experts, expert, counts, o->err);
  hipLaunchKernelGGL(k_order_place, dim3(tiles), dim3(kOrderThreads), 0, s, pairs, (int)tile, tiles, experts, bits, expert, counts, offsets, place,
                     o->err);
  return launched(o);
}

}  // extern "C"

namespace {

sp_status move_sizes(const sp_ops* o, int32_t n, int32_t d, int32_t top, int32_t dtype, int32_t rows, const int32_t* place) {
  if (!o || n < 0 || d < 1 || top < 1 || !dtype_ok(dtype) || rows < 0 || (n > 0 && !place) || !aligned4(place)) return SP_EINVAL;
  if (top > SP_MAX_TOP || d > SP_MAX_LINEAR_DIM) return SP_ECAPACITY;
  return SP_OK;
}

// Calls f<T, TEAM, AT>(workgroups) with a team for rows of d columns and the pairs of a row that are on their way together.
template <typename F>
void with_rows(int32_t n, int32_t d, int32_t top, int32_t dtype, F&& f) {
  with_type(dtype, [&]<typename T>() {
    const int pieces = (d + kPiece<T> - 1) / kPiece<T>;
    auto team = [&]<int TEAM>() {
      constexpr int rows = 256 / TEAM;
      const dim3 grid((unsigned)std::min<int64_t>(((int64_t)n + rows - 1) / rows, kMoveBlocks));
      if (top == 1) f.template operator()<T, TEAM, 1>(grid);
      else if (top == 2) f.template operator()<T, TEAM, 2>(grid);
      else if (top <= 4) f.template operator()<T, TEAM, 4>(grid);
      else f.template operator()<T, TEAM, 8>(grid);
    };
    // The largest team that leaves the fewest lanes without a piece in the last turn, in at most four turns.  96 pieces (32768 x 768 bfloat16, 8 pairs): 32 lanes
    // in three turns combine in 96 us, 64 in two in 107; 16 pieces (262144 x 64 float32, 2 pairs) 16 lanes 44 us, 64 lanes 88; 65 pieces (65536 x 520 bfloat16,
    // 4 pairs) 32 lanes 75 us, 16 lanes in five turns 82, 64 lanes 81.
    auto idle = [&](int lanes) { return (pieces + lanes - 1) / lanes * lanes - pieces; };
    int best = 64;
    for (int lanes = 32; lanes >= 4; lanes /= 2)
      if (idle(lanes) < idle(best) && (pieces + lanes - 1) / lanes <= 4) best = lanes;
    if (best == 4) team.template operator()<4>();
    else if (best == 8) team.template operator()<8>();
    else if (best == 16) team.template operator()<16>();
    else if (best == 32) team.template operator()<32>();
    else team.template operator()<64>();
  });
}

}  // namespace

extern "C" {

sp_status sp_dispatch(sp_ops* o, int32_t n, int32_t d, int32_t top, int32_t dtype, const void* x, int64_t x_stride, const int32_t* place,
                      int32_t rows, void* xs, int64_t xs_stride, void* stream) {
  const sp_status bad = move_sizes(o, n, d, top, dtype, rows, place);
  if (bad != SP_OK) return bad;
  if (x_stride < d || xs_stride < d || (n > 0 && !x) || (n > 0 && rows > 0 && !xs) || !aligned(x, dtype) || !aligned(xs, dtype)) return SP_EINVAL;
  if (n == 0) return SP_OK;
  DeviceGuard g(o->device);
  if (!g.ok) return SP_EDEVICE;
  with_rows(n, d, top, dtype, [&]<typename T, int TEAM, int AT>(dim3 grid) {
    hipLaunchKernelGGL((k_dispatch<T, TEAM, AT>), grid, dim3(256), 0, (hipStream_t)stream, n, d, top, (const T*)x, x_stride, place, rows, (T*)xs,
                       xs_stride, o->err);
  });
  return launched(o);
}

sp_status sp_combine(sp_ops* o, int32_t n, int32_t d, int32_t top, int32_t dtype, int32_t rows, const void* ys, int64_t ys_stride,
                     const int32_t* place, const float* weight, const void* residual, int64_t residual_stride, void* y, int64_t y_stride,
                     void* stream) {
  const sp_status bad = move_sizes(o, n, d, top, dtype, rows, place);
  if (bad != SP_OK) return bad;
  if (ys_stride < d || y_stride < d || (residual && residual_stride < d) || (n > 0 && !y) || (n > 0 && rows > 0 && !ys)) return SP_EINVAL;
  if (!aligned(ys, dtype) || !aligned(y, dtype) || !aligned(residual, dtype) || !aligned4(weight)) return SP_EINVAL;
  if (n == 0) return SP_OK;
  DeviceGuard g(o->device);
  if (!g.ok) return SP_EDEVICE;
  with_rows(n, d, top, dtype, [&]<typename T, int TEAM, int AT>(dim3 grid) {
    hipLaunchKernelGGL((k_combine<T, TEAM, AT>), grid, dim3(256), 0, (hipStream_t)stream, n, d, top, rows, (const T*)ys, ys_stride, place, weight,
                       (const T*)residual, residual_stride, (T*)y, y_stride, o->err);
  });
  return launched(o);
}

sp_status sp_combine_backward(sp_ops* o, int32_t n, int32_t d, int32_t top, int32_t dtype, const void* dy, int64_t dy_stride, int32_t rows,
                              const void* ys, int64_t ys_stride, const int32_t* place, const float* weight, void* dys, int64_t dys_stride,
                              float* dweight, void* stream) {
  const sp_status bad = move_sizes(o, n, d, top, dtype, rows, place);
  if (bad != SP_OK) return bad;
  if (dy_stride < d || (dweight && ys_stride < d) || (dys && dys_stride < d) || (n > 0 && !dy) || (n > 0 && rows > 0 && dweight && !ys))
    return SP_EINVAL;
  if (!aligned(dy, dtype) || !aligned(ys, dtype) || !aligned(dys, dtype) || !aligned4(weight) || !aligned4(dweight)) return SP_EINVAL;
  if (n == 0 || (!dys && !dweight)) return SP_OK;
  DeviceGuard g(o->device);
  if (!g.ok) return SP_EDEVICE;
  with_rows(n, d, top, dtype, [&]<typename T, int TEAM, int AT>(dim3 grid) {
    hipLaunchKernelGGL((k_combine_back<T, TEAM, AT>), grid, dim3(256), 0, (hipStream_t)stream, n, d, top, (const T*)dy, dy_stride, rows,
                       (const T*)ys, ys_stride, place, weight, (T*)dys, dys_stride, dweight, o->err);
  });
  return launched(o);
}

sp_status sp_dropout(sp_ops* o, int32_t n, int32_t d, int32_t dtype, const void* x, int64_t x_stride, float p, uint64_t seed, uint64_t offset,
                     const int64_t* step, const void* residual, int64_t residual_stride, void* y, int64_t y_stride, void* stream) {
  if (!o || n < 0 || d < 1 || !dtype_ok(dtype) || x_stride < d || y_stride < d || (residual && residual_stride < d)) return SP_EINVAL;
  if (!(p >= 0.f && p <= 1.f) || (n > 0 && (!x || !y))) return SP_EINVAL;
  if (!aligned(x, dtype) || !aligned(y, dtype) || !aligned(residual, dtype) || ((uintptr_t)step & 7u)) return SP_EINVAL;
  if (d > SP_MAX_LINEAR_DIM) return SP_ECAPACITY;
  DropoutArgs a{};
  a.n = n; a.d = d; a.pieces = (d + 7) / 8;
  a.drop = (uint32_t)std::lround((double)p * 65536.0);
  if (p > 0.f && a.drop == 0) a.drop = 1;
  if (p < 1.f && a.drop == 65536) a.drop = 65535;
  a.scale = a.drop == 65536 ? 0.f : 65536.f / (float)(65536 - a.drop);
  a.key0 = (uint32_t)seed; a.key1 = (uint32_t)(seed >> 32); a.offset = offset; a.step = step;
  a.x = x; a.x_stride = x_stride; a.residual = residual; a.residual_stride = residual_stride; a.y = y; a.y_stride = y_stride;
  const int64_t pieces = (int64_t)n * a.pieces;
  if (pieces / 2 > UINT32_MAX - 512) return SP_ECAPACITY;
  if (n == 0) return SP_OK;
  DeviceGuard g(o->device);
  if (!g.ok) return SP_EDEVICE;
  const int64_t blocks = (pieces + 255) / 256, turns = (blocks + (1 << 23) - 1) >> 23;      // (a launch has less than 2^32 threads in a dimension)
  with_type(dtype, [&]<typename T>() {
    hipLaunchKernelGGL(k_dropout<T>, dim3((unsigned)((blocks + turns - 1) / turns), (unsigned)turns), dim3(256), 0, (hipStream_t)stream, a);
  });
  return launched(o);
}

sp_status sp_quantize_rows(sp_ops* o, int32_t n, int32_t d, int32_t dtype, const void* x, int64_t x_stride, int8_t* q, int64_t q_stride,
                           float* scale, void* stream) {
  if (!o || n < 0 || d < 1 || !dtype_ok(dtype) || x_stride < d || q_stride < d || (n > 0 && (!x || !q || !scale))) return SP_EINVAL;
  if (!aligned(x, dtype) || !aligned4(scale)) return SP_EINVAL;
  if (d > SP_MAX_LINEAR_DIM) return SP_ECAPACITY;
  if (n == 0) return SP_OK;
  DeviceGuard g(o->device);
  if (!g.ok) return SP_EDEVICE;
  with_type(dtype, [&]<typename T>() {
    const bool fits = with_team((d + kPiece<T> - 1) / kPiece<T>, [&]<int TEAM, int C>() {
      constexpr int threads = kTeamThreads<TEAM>, rows = threads / TEAM;
      const int blocks = (int)std::min<int64_t>(((int64_t)n + rows - 1) / rows, 8192);
      hipLaunchKernelGGL((k_quantize<T, TEAM, C>), dim3(blocks), dim3(threads), 0, (hipStream_t)stream, n, d, (const T*)x, x_stride, q, q_stride,
                         scale);
    });
    if (!fits)
      hipLaunchKernelGGL((k_quantize_wide<T>), dim3(std::min(n, 4096)), dim3(1024), 0, (hipStream_t)stream, n, d, (const T*)x, x_stride, q,
                         q_stride, scale);
  });
  return launched(o);
}

sp_status sp_grouped_linear_quantized(sp_ops* o, int32_t n, int32_t k, int32_t m, int32_t groups, const int8_t* x, int64_t x_stride,
                                      const float* x_scale, const int32_t* offsets, const int8_t* w, const float* w_scale, const float* bias,
                                      int32_t activation, int32_t out_dtype, const void* residual, int64_t residual_stride, void* y,
                                      int64_t y_stride, void* stream) {
  if (!o || n < 0 || k < 1 || m < 1 || groups < 1 || x_stride < k || y_stride < m || (residual && residual_stride < m)) return SP_EINVAL;
  if ((activation != SP_ACT_NONE && activation != SP_ACT_RELU) || !dtype_ok(out_dtype)) return SP_EINVAL;
  if (n > 0 && (!x || !x_scale || !offsets || !w || !w_scale || !y)) return SP_EINVAL;
  if (!aligned(y, out_dtype) || !aligned(residual, out_dtype) || !aligned4(x_scale) || !aligned4(offsets) || !aligned4(w_scale) || !aligned4(bias))
    return SP_EINVAL;
  if (groups > SP_MAX_APPS || k > SP_MAX_QUANTIZED_INPUTS || m > SP_MAX_LINEAR_DIM || x_stride > SP_MAX_LINEAR_STRIDE) return SP_ECAPACITY;
  if (n == 0) return SP_OK;
  QuantizedArgs a{};
  a.n = n; a.k = k; a.m = m; a.groups = groups; a.x = x; a.x_stride = x_stride; a.x_scale = x_scale; a.offsets = offsets; a.w = w;
  a.w_scale = w_scale; a.bias = bias; a.relu = activation == SP_ACT_RELU; a.residual = residual; a.residual_stride = residual_stride;
  a.y = y; a.y_stride = y_stride; a.err = o->err;
  // Pieces of 16 rows while the device holds about all of their workgroups and each is through its depth soon (256 rows, 1024 -> 1024: 7.2 us
  // against 11.4 in tiles; 1024 rows, 1024 -> 512 11.1 against 10.5, 256 rows, 2048 -> 2048 20.9 against 16.0; addresses that are no multiples of 16 cost
  // them more: 256 rows of 32 groups, 1023 -> 515 21.4 against 16.6).  Tiles of 256 by 256, one to a compute unit, where there are many long ones
  // (262144 rows, 2048 -> 2048: 1220 us against 1510 in tiles of 128 by 128, 1024 -> 1024 362 against 412; 512 -> 512 127 against 122).  y past the
  // caches where it is longer than 128 MB, half of the last-level cache (256 -> 1024, bfloat16, past them and through them: 256 MB 83 us and 107, 512 MB 161
  // and 213; 96 MB 31.5 and 33.3, but 65 and 62 with the next reader of y).
  const bool direct = (((uintptr_t)x | (uintptr_t)w | (uintptr_t)k | (uintptr_t)x_stride) & 15u) == 0;
  auto grid = [&](int64_t bm, int64_t bn, int64_t threads) {         // false: more workgroups than a launch holds
    const int64_t row_tiles = std::min<int64_t>((n + bm - 1) / bm + groups, n), col_tiles = (m + bn - 1) / bn;
    if ((row_tiles * col_tiles + kXcds) * threads > UINT32_MAX) return false;
    a.row_tiles = (int)row_tiles;
    a.col_tiles = (int)col_tiles;
    return true;
  };
  const int64_t few_tiles = (((int64_t)n + kFewQuantizedRows - 1) / kFewQuantizedRows + std::min(n, groups)) * ((m + kFewQuantizedCols - 1) / kFewQuantizedCols);
  const bool few = few_tiles <= 2048 && few_tiles * k <= (direct ? 1 << 21 : 1 << 20);
  const bool large = direct && k >= 1024 && ((int64_t)n + 255) / 256 * ((m + 255) / 256) >= 2048;
  if (!(few ? grid(kFewQuantizedRows, kFewQuantizedCols, kFewQuantizedThreads) : large ? grid(256, 256, 512) : grid(128, 128, 256))) return SP_ECAPACITY;
  const unsigned blocks = (unsigned)(((int64_t)a.row_tiles * a.col_tiles + kXcds - 1) / kXcds * kXcds);
  a.past_caches = (int64_t)n * m * elem_bytes(out_dtype) > (int64_t)128 << 20;
  DeviceGuard g(o->device);
  if (!g.ok) return SP_EDEVICE;
  with_type(out_dtype, [&]<typename T>() {
    auto kernel = few ? k_quantized_few<T> : large ? k_quantized<T, 256, 256, 128, true>
                  : direct ? k_quantized<T, 128, 128, 64, true> : k_quantized<T, 128, 128, 64, false>;
    hipLaunchKernelGGL(kernel, dim3(blocks), dim3(few ? kFewQuantizedThreads : large ? 512 : 256), 0, (hipStream_t)stream, a);
  });
  return launched(o);
}

}  // extern "C"
