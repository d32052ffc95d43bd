// Routing: which few of its experts a row goes through, with what weights, and the gradient of that.
//   s = softmax(z) or sigmoid(z) over a row's experts       c = s + b, by which experts are chosen (b: a bias that balances them)
//   groups of consecutive experts: a group's value is the sum of its two largest c (one, where it has one); the top_groups groups of
//   the largest values stay.  Of what stays the `top` largest c are chosen, in descending order.  Ties go to the lowest number.
//   w_j = scale s_j, or scale s_j / (sum of the chosen s)
// An expert whose logit is -inf is not there: never chosen, s = 0.  Where fewer than `top` are left, the rest of the row is -1 with weight 0.
// c are compared in 64 bits (without a bias and groups: the logits themselves, which s rises with), so that what is chosen does not hang on the
// rounding of s.
#pragma once
#include "sp_ops_common.h"

namespace sp {

struct RouteArgs {
  int n, experts, top, groups, top_groups, width;    // width: experts of a group
  int group_lanes;                                   // lanes of a wavefront that share a group, a power of two
  bool sigmoid, renormalize;
  float scale;
  const void* z;  int64_t z_stride;                  // [n, experts]
  const float* bias;                                 // [experts] or null
  int32_t* expert;                                   // [n, top]
  float* weight;                                     // [n, top]
  uint32_t* err;
};

__device__ __forceinline__ float exp_below(float d) { return __builtin_amdgcn_exp2f(d * 1.44269504f); }     // d <= 0; NaN stays NaN

// What a lane that holds one chosen expert's logit (-inf for none) makes of it.  The sum over the chosen ones is taken of values relative to the
// largest, so that it is not 0 where all scores are.
struct ChosenScore {
  float s;        // score: sigmoid(z), or exp(z - from)
  float share;    // s over the sum of the chosen ones' s
};
template <int TEAM>
__device__ __forceinline__ ChosenScore chosen_score(float z, bool sigmoid, float from) {
  ChosenScore r;
  const float a = sigmoid ? fminf(z, 0.f) : z, high = team_max<TEAM>(a, nullptr), base = high == -INFINITY ? 0.f : high;
  float t = expf(a - base);
  if (sigmoid) {
    const float over = 1.f + expf(-fabsf(z));
    t /= over;
    r.s = expf(a) / over;
  } else {
    r.s = expf(z - from);
  }
  const float total = team_sum<TEAM>(t, nullptr);
  r.share = total > 0.f ? t / total : 0.f;
  return r;
}

// One row by one wavefront, in 64 bits.  Group g belongs to lanes g * group_lanes .. + group_lanes - 1, which deal its experts out among them.
template <typename T, int PER>
__device__ __forceinline__ void route_row(const RouteArgs& a, int64_t row) {
  const int lane = threadIdx.x & 63, g = lane / a.group_lanes, sub = lane % a.group_lanes, first = g * a.width + sub;
  const T* z = (const T*)a.z + row * a.z_stride;
  const bool by_logit = !a.bias && a.groups == 1;
  float v[PER];
  bool bad = false;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int at = i * a.group_lanes;
    v[i] = g < a.groups && at + sub < a.width ? to_float(z[first + at]) : -INFINITY;
    bad |= !(v[i] < INFINITY);
  }
  if (__any(bad)) {
    if (lane == 0) atomicOr(a.err, kErrRouterLogit);
    if (lane < a.top) {
      a.expert[row * a.top + lane] = -1;
      a.weight[row * a.top + lane] = 0.f;
    }
    return;
  }
  float high = -INFINITY;
#pragma unroll
  for (int i = 0; i < PER; ++i) high = fmaxf(high, v[i]);
  high = team_max<64>(high, nullptr);
  const float from = high == -INFINITY ? 0.f : high;
  float total = 0.f;
  if (!a.sigmoid && !a.renormalize) {
#pragma unroll
    for (int i = 0; i < PER; ++i) total += exp_below(v[i] - from);
    total = team_sum<64>(total, nullptr);
  }
  double c[PER];
  if (by_logit) {
#pragma unroll
    for (int i = 0; i < PER; ++i) c[i] = v[i];
  } else {
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      c[i] = a.sigmoid ? 1.0 / (1.0 + exp(-(double)v[i])) : exp((double)v[i] - from);
      sum += c[i];
    }
#pragma unroll
    for (int s = 1; s < 64; s *= 2) sum += __shfl_xor(sum, s);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (!a.sigmoid) c[i] /= sum;
      if (v[i] == -INFINITY) c[i] = -INFINITY;
      else if (a.bias) c[i] += (double)a.bias[first + i * a.group_lanes];
    }
  }
  if (a.groups > 1) {
    double m1 = -INFINITY, m2 = -INFINITY;                 // the group's two largest
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      m2 = fmax(m2, fmin(m1, c[i]));
      m1 = fmax(m1, c[i]);
    }
    for (int s = 1; s < a.group_lanes; s *= 2) {
      const double o1 = __shfl_xor(m1, s), o2 = __shfl_xor(m2, s);
      m2 = fmax(fmin(m1, o1), fmax(m2, o2));
      m1 = fmax(m1, o1);
    }
    const double value = m2 == -INFINITY ? m1 : m1 + m2;
    int before = 0;
    for (int h = 0; h < a.groups; ++h) {
      const double o = __shfl(value, h * a.group_lanes);
      before += o > value || (o == value && h < g);
    }
    if (before >= a.top_groups) {
#pragma unroll
      for (int i = 0; i < PER; ++i) c[i] = -INFINITY;
    }
  }
  int mine = -1;
  for (int j = 0; j < a.top; ++j) {
    double b = -INFINITY;
    int e = INT32_MAX;
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (c[i] > b) {
        b = c[i];
        e = first + i * a.group_lanes;
      }
#pragma unroll
    for (int s = 1; s < 64; s *= 2) {
      const double ob = __shfl_xor(b, s);
      const int oe = __shfl_xor(e, s);
      if (ob > b || (ob == b && oe < e)) {
        b = ob;
        e = oe;
      }
    }
    if (e == INT32_MAX) break;                             // (the same on every lane)
    if (lane == j) mine = e;
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (first + i * a.group_lanes == e) c[i] = -INFINITY;
  }
  const float zc = mine >= 0 ? to_float(z[mine]) : -INFINITY;
  const ChosenScore r = chosen_score<64>(zc, a.sigmoid, from);
  if (lane < a.top) {
    a.expert[row * a.top + lane] = mine;
    a.weight[row * a.top + lane] = mine < 0 ? 0.f : a.scale * (a.renormalize ? r.share : a.sigmoid ? r.s : r.s / total);
  }
}

template <typename T, int PER>
__global__ __launch_bounds__(256) void k_route(RouteArgs a) {
  for (int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); row < a.n; row += (int64_t)gridDim.x * 4) route_row<T, PER>(a, row);
}

// The gradient of the logits from that of the weights.  With D = sum over the chosen of dw_l w_l / scale:
//   renormalised   dz_j = scale w'_j (dw_j - D)   (times 1 - s_j for sigmoid), w' the shares; 0 for experts not chosen
//   sigmoid        dz_j = scale dw_j s_j (1 - s_j)
//   softmax        dz_e = s_e (scale dw_e - sum_l scale dw_l s_l), every expert
// A team holds a row.  Lane j has the j-th chosen expert; what the others need of it goes through LDS.  A row without an expert has gradient 0.
template <typename T, int TEAM, int C>
__global__ __launch_bounds__(256) void k_route_back(int n, int experts, int top, const T* z, int64_t z_stride, bool sigmoid, bool renormalize,
                                                    float scale, const int32_t* __restrict__ expert, const float* __restrict__ dweight, T* dz,
                                                    int64_t dz_stride, uint32_t* err) {
  constexpr int V = kPiece<T>, ROWS = 256 / TEAM, WIDE = TEAM * C * V;
  __shared__ __align__(16) float up[ROWS][WIDE];
  const int t = threadIdx.x % TEAM, team = threadIdx.x / TEAM;
  const bool all = !sigmoid && !renormalize;
  for (int64_t base = (int64_t)blockIdx.x * ROWS; base < n; base += (int64_t)gridDim.x * ROWS) {
    const int64_t row = base + team;
    const bool in = row < n;
    int e = in && t < top ? expert[row * top + t] : -1;
    if (e < -1 || e >= experts) {
      atomicOr(err, kErrExpert);
      e = -1;
    }
    const float dw = e >= 0 ? scale * dweight[row * top + t] : 0.f;
    const float zc = e >= 0 ? to_float(z[row * z_stride + e]) : -INFINITY;
    float v[C][V];
    float from = 0.f, total = 1.f;
    if (all) {
      float high = -INFINITY;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int col = (c * TEAM + t) * V;
        load_some(z + (in ? row : 0) * z_stride + col, in ? experts - col : 0, -INFINITY, v[c]);
#pragma unroll
        for (int i = 0; i < V; ++i) high = fmaxf(high, v[c][i]);
      }
      high = team_max<TEAM>(high, nullptr);
      from = high == -INFINITY ? 0.f : high;
      total = 0.f;
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < V; ++i) {
          v[c][i] = exp_below(v[c][i] - from);
          total += v[c][i];
        }
      total = team_sum<TEAM>(total, nullptr);
    }
    const ChosenScore r = chosen_score<TEAM>(zc, sigmoid, from);
    float mine;                                            // what the chosen expert's logit gets (softmax: what its score gets)
    const float share = all ? r.s / total : r.share, dot = team_sum<TEAM>(e >= 0 ? dw * share : 0.f, nullptr);
    if (all) {
      mine = dw;
    } else {
      const float rest = zc == -INFINITY ? 1.f : 1.f / (1.f + expf(zc));              // 1 - s
      mine = renormalize ? share * (dw - dot) : dw * r.s;
      if (sigmoid) mine *= rest;
    }
    // an expert that is named twice gets both parts, in order
    bool first = e >= 0;
    float sum = 0.f;
    int named = 0;
    for (int j = 0; j < top; ++j) {
      const int o = __shfl(e, j, TEAM);
      const float om = __shfl(mine, j, TEAM);
      named += o >= 0;
      if (o == e) sum += om;
      first &= o != e || j >= t;
    }
    __syncthreads();                                       // the row before has been read
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int h = 0; h < V; h += 4) *reinterpret_cast<f32x4*>(&up[team][(c * TEAM + t) * V + h]) = f32x4{0.f, 0.f, 0.f, 0.f};
    __syncthreads();
    if (first) up[team][e] = sum;
    __syncthreads();
    if (!in) continue;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int col = (c * TEAM + t) * V;
      float u[V];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        u[i] = up[team][col + i];
        if (all) u[i] = named ? v[c][i] / total * (u[i] - dot) : 0.f;
      }
      store_some(dz + row * dz_stride + col, experts - col, u);
    }
  }
}

// Places: (row, expert) pairs in the order of their experts, pairs of one expert in their own order.
//   offsets_e = pairs of experts before e        place = offsets_e + pairs of e before this one; -1 for pairs without an expert
// Tiles of pairs are counted by one launch and placed by a second, whose workgroups add up the counts of the tiles before theirs; few pairs
// are one tile and one launch.  Inside a tile each wavefront has a run of pairs and looks for equal experts 64 pairs at a time, by ballots over
// the bits of their numbers.
constexpr int kOrderThreads = 1024;
constexpr int kMaxExperts = 1024;

__device__ __forceinline__ int expert_of(const int32_t* expert, int64_t pair, int64_t end, int experts, uint32_t* err) {
  if (pair >= end) return -1;
  const int e = expert[pair];
  if (e >= -1 && e < experts) return e;
  atomicOr(err, kErrExpert);
  return -1;
}

__global__ __launch_bounds__(kOrderThreads) void k_order_count(int64_t pairs, int tile, int experts, const int32_t* __restrict__ expert,
                                                               int32_t* counts, uint32_t* err) {
  __shared__ int32_t count[kMaxExperts];
  for (int e = threadIdx.x; e < experts; e += kOrderThreads) count[e] = 0;
  __syncthreads();
  const int64_t lo = (int64_t)blockIdx.x * tile, hi = min(lo + tile, pairs);
  for (int64_t p = lo + threadIdx.x; p < hi; p += kOrderThreads) {
    const int e = expert_of(expert, p, hi, experts, err);
    if (e >= 0) atomicAdd(&count[e], 1);
  }
  __syncthreads();
  for (int e = threadIdx.x; e < experts; e += kOrderThreads) counts[(int64_t)blockIdx.x * experts + e] = count[e];
}

// counts null: this tile is the only one.
__global__ __launch_bounds__(kOrderThreads) void k_order_place(int64_t pairs, int tile, int tiles, int experts, int bits,
                                                               const int32_t* __restrict__ expert, const int32_t* __restrict__ counts,
                                                               int32_t* offsets, int32_t* place, uint32_t* err) {
  constexpr int WAVES = kOrderThreads / 64;
  __shared__ int32_t count[WAVES][kMaxExperts];            // first the wavefronts' counts, then where their next pair of an expert goes
  __shared__ int32_t sums[WAVES];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int i = threadIdx.x; i < WAVES * experts; i += kOrderThreads) count[i / experts][i % experts] = 0;
  __syncthreads();
  const int64_t lo = (int64_t)blockIdx.x * tile, hi = min(lo + tile, pairs);
  const int run = (int)((hi - lo + WAVES * 64 - 1) / (WAVES * 64)) * 64;
  const int64_t from = lo + (int64_t)wave * run, to = min(from + run, hi);
  for (int64_t p = from + lane; p < to; p += 64) {
    const int e = expert_of(expert, p, to, experts, err);
    if (e >= 0) atomicAdd(&count[wave][e], 1);
  }
  __syncthreads();
  const int e = threadIdx.x;
  int before = 0, all = 0;
  if (e < experts) {
    if (counts) {
#pragma unroll 8
      for (int q = 0; q < tiles; ++q) {
        const int c = counts[(int64_t)q * experts + e];
        all += c;
        before += q < (int)blockIdx.x ? c : 0;
      }
    } else {
      for (int w = 0; w < WAVES; ++w) all += count[w][e];
    }
  }
  int upto = (int)wave_scan_incl((uint32_t)all);
  if (lane == 63) sums[wave] = upto;
  __syncthreads();
  for (int w = 0; w < wave; ++w) upto += sums[w];
  if (e < experts) {
    if (blockIdx.x == 0) {
      offsets[e] = upto - all;
      if (e == experts - 1) offsets[experts] = upto;
    }
    int at = upto - all + before;
    for (int w = 0; w < WAVES; ++w) {
      const int c = count[w][e];
      count[w][e] = at;
      at += c;
    }
  }
  __syncthreads();
  for (int64_t p = from + lane; p - lane < to; p += 64) {
    const int own = expert_of(expert, p, to, experts, err);
    unsigned long long same = __ballot(own >= 0);
    for (int b = 0; b < bits; ++b) {
      const unsigned long long set = __ballot((own >> b) & 1);
      same &= (own >> b) & 1 ? set : ~set;
    }
    int at = -1;
    if (own >= 0) {
      const int rank = __popcll(same & ((1ull << lane) - 1));
      at = count[wave][own] + rank;
    }
    wave_sync();
    if (own >= 0 && (same >> lane) == 1ull) count[wave][own] = at + 1;      // the last of them
    wave_sync();
    if (p < to) place[p] = at;
  }
}

}  // namespace sp
