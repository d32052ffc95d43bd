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

// Lane l ^ S of every eight lanes.
template <int S>
__device__ __forceinline__ float lane_xor(float v) {
  static_assert(S > 0 && S < 8, "of eight lanes");
  constexpr int q = S < 4 ? S : S ^ 7, perm = (0 ^ q) | (1 ^ q) << 2 | (2 ^ q) << 4 | (3 ^ q) << 6;
  int x = __float_as_int(v);
  if (S >= 4) x = __builtin_amdgcn_update_dpp(0, x, 0x141, 0xf, 0xf, false);          // row_half_mirror: lane ^ 7
  if (q) x = __builtin_amdgcn_update_dpp(0, x, perm, 0xf, 0xf, false);
  return __int_as_float(x);
}
// A team's fold of an operation that is the same in any order, on every lane.
template <int TEAM, typename F>
__device__ __forceinline__ float team_fold(float v, F f) {
  v = f(v, lane_xor<1>(v));
  v = f(v, lane_xor<2>(v));
  v = f(v, lane_xor<7>(v));
#pragma unroll
  for (int s = 8; s < TEAM; s *= 2) v = f(v, __shfl_xor(v, s));
  return v;
}
template <int TEAM>
__device__ __forceinline__ uint32_t team_max_u32(uint32_t v) {
  if (TEAM == 64) return wave_max_u32(v);
  v = wave_max_step32<0xB1, 0xf>(v);
  v = wave_max_step32<0x4E, 0xf>(v);
  return wave_max_step32<0x141, 0xf>(v);
}
__device__ __forceinline__ float larger(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ float smaller(float a, float b) { return fminf(a, b); }
// NaN if either is.
__device__ __forceinline__ float maximum(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// exp(d) for d <= 0, to 3 u: the product with log2(e) in two parts, the second of which exp2 does not get.
__device__ __forceinline__ float exp_near(float d) {
  const float p = d * 1.44269502f;
  float r = fmaf(d, 1.44269502f, -p);
  r = fmaf(d, 1.92596299e-8f, r);
  const float e = __builtin_amdgcn_exp2f(p);
  return p == -INFINITY ? 0.f : fmaf(e, r * 0.693147181f, e);
}

// The weight of a lane's chosen expert from its logit (-inf for none): s over `total`, or over the sum of the chosen ones' s, which is taken of values
// relative to the largest, so that it is not 0 where all scores are.  from: the row's largest logit.
template <int TEAM>
__device__ __forceinline__ float chosen_weight(float z, bool sigmoid, bool renormalize, float from, float total) {
  const float a = sigmoid ? fminf(z, 0.f) : z;
  const float high = renormalize ? team_fold<TEAM>(a, larger) : sigmoid ? 0.f : from;
  float t = exp_near(a - (high == -INFINITY ? 0.f : high));
  if (sigmoid) t *= __builtin_amdgcn_rcpf(1.f + exp_near(-fabsf(z)));
  if (renormalize) total = team_sum<TEAM>(t, nullptr);
  else if (sigmoid) total = 1.f;
  return total > 0.f ? t * __builtin_amdgcn_rcpf(total) : 0.f;
}

// One row by one wavefront, in 64 bits.  Group g belongs to lanes g * group_lanes .. + group_lanes - 1, which deal its experts out among them.
// c: the wavefront's part of LDS, a number for every expert; loops are not unrolled, so that this rare way does not take the registers of the other.
template <typename T>
__device__ __forceinline__ void route_row(const RouteArgs& a, int64_t row, double* c) {
  const int lane = threadIdx.x & 63, step = a.group_lanes, g = lane / step, sub = lane % step;
  const T* z = (const T*)a.z + row * a.z_stride;
  const int begin = g < a.groups ? g * a.width + sub : a.experts, end = g < a.groups ? (g + 1) * a.width : a.experts;      // the lane's experts
  const bool by_logit = !a.bias && a.groups == 1;
  bool bad = false;
  float high = -INFINITY;
#pragma unroll 4
  for (int e = begin; e < end; e += step) {
    const float v = to_float(z[e]);
    bad |= !(v < INFINITY);
    high = fmaxf(high, v);
    c[e] = v;
  }
  if (__any(bad)) {
    if (lane == 0) atomicOr(a.err, kErrRouterLogit);
    if (lane < a.top) {
      a.expert[row * a.top + lane] = -1;
      a.weight[row * a.top + lane] = 0.f;
    }
    return;
  }
  high = team_fold<64>(high, larger);
  const float from = high == -INFINITY ? 0.f : high;
  double sum = 0.0;
#pragma unroll 1
  for (int e = begin; e < end && !(by_logit && a.sigmoid); e += step) {
    const double v = c[e], x = exp(a.sigmoid ? -v : v - from);
    sum += x;
    if (!by_logit) c[e] = v == -INFINITY ? v : a.sigmoid ? 1.0 / (1.0 + x) : x;
  }
  if (!a.sigmoid) {
#pragma unroll
    for (int s = 1; s < 64; s *= 2) sum += __shfl_xor(sum, s);
  }
  double m1 = -INFINITY, m2 = -INFINITY;                   // the lane's, then the group's two largest
#pragma unroll 4
  for (int e = begin; e < end && !by_logit; e += step) {
    double s = a.sigmoid ? c[e] : c[e] / sum;
    if (a.bias) s += (double)a.bias[e];
    if (s != s) s = -INFINITY;                             // (a bias that is no number)
    c[e] = s;
    m2 = fmax(m2, fmin(m1, s));
    m1 = fmax(m1, s);
  }
  if (a.groups > 1) {
    for (int s = 1; s < step; s *= 2) {
      const double o1 = __shfl_xor(m1, s), o2 = __shfl_xor(m2, s);
      m2 = fmax(fmin(m1, o1), fmax(m2, o2));
      m1 = fmax(m1, o1);
    }
    const double value = m2 == -INFINITY ? m1 : m1 + m2;
    int before = 0;
    for (int h = 0; h < a.groups; ++h) {
      const double o = __shfl(value, h * step);
      before += o > value || (o == value && h < g);
    }
    if (before >= a.top_groups)
      for (int e = begin; e < end; e += step) c[e] = -INFINITY;
  }
  int mine = -1;
  for (int j = 0; j < a.top; ++j) {
    double b = -INFINITY;
    int e = INT32_MAX;
#pragma unroll 4
    for (int q = begin; q < end; q += step) {
      const double v = c[q];
      if (v > b) {
        b = v;
        e = q;
      }
    }
    // the bits of a double in the order of the numbers (adding 0 makes -0 a 0), 0 for a lane that has none
    const long long bits = __double_as_longlong(b + 0.0);
    const unsigned long long rank = e == INT32_MAX ? 0ull : (unsigned long long)(bits ^ (bits >> 63 | INT64_MIN));
    const unsigned long long best = wave_max_u64(rank);
    if (best == 0ull) break;                               // (the same on every lane)
    e = (int)~wave_max_u32(rank == best ? ~(uint32_t)e : 0u);
    if (lane == j) mine = e;
    if (e >= begin && e < end && (e - begin) % step == 0) c[e] = -INFINITY;      // (every lane reads and writes its own experts only)
  }
  const float zc = mine >= 0 ? to_float(z[mine]) : -INFINITY;
  const float w = chosen_weight<64>(zc, a.sigmoid, a.renormalize, from, (float)sum);
  if (lane < a.top) {
    a.expert[row * a.top + lane] = mine;
    a.weight[row * a.top + lane] = a.scale * w;
  }
}

// V neighbours of a row of `all` from `at` on, of which the first `count` count; the others become -inf.
template <typename T, int V>
__device__ __forceinline__ void load_run(const T* row, int at, int all, int count, float (&v)[V]) {
  if constexpr (V == 1) {
    v[0] = count > 0 ? to_float(row[at]) : -INFINITY;
  } else if constexpr (V == 4) {
    load_some(row + at, count > 0 ? all - at : 0, -INFINITY, v);      // (a piece that ends inside the row is read whole)
#pragma unroll
    for (int h = 0; h < V; ++h) v[h] = h < count ? v[h] : -INFINITY;
  } else {
    const raw_piece q = load_raw_piece(row, count > 0 ? at : all, all);
#pragma unroll
    for (int h = 0; h < V; ++h) v[h] = h < count ? of_raw((const T*)nullptr, q, h) : -INFINITY;
  }
}

// The N (a power of two up to 32) keys of a lane in descending order, the nine largest of them.
__device__ __forceinline__ void order(uint32_t& a, uint32_t& b) {
  const uint32_t high = max(a, b);
  b = min(a, b);
  a = high;
}
__device__ __forceinline__ void sort_8(uint32_t (&k)[8]) {            // Batcher's merge exchange, nineteen comparators
  order(k[0], k[1]); order(k[2], k[3]); order(k[4], k[5]); order(k[6], k[7]);
  order(k[0], k[2]); order(k[1], k[3]); order(k[4], k[6]); order(k[5], k[7]);
  order(k[1], k[2]); order(k[5], k[6]);
  order(k[0], k[4]); order(k[1], k[5]); order(k[2], k[6]); order(k[3], k[7]);
  order(k[2], k[4]); order(k[3], k[5]);
  order(k[1], k[2]); order(k[3], k[4]); order(k[5], k[6]);
}
template <int N>
__device__ __forceinline__ void sort_keys(const uint32_t (&key)[N], uint32_t (&list)[10]) {
  if constexpr (N == 32) {
    uint32_t half[16], other[10] = {};
#pragma unroll
    for (int i = 0; i < 16; ++i) half[i] = key[i];
    sort_keys<16>(half, list);
#pragma unroll
    for (int i = 0; i < 16; ++i) half[i] = key[16 + i];
    sort_keys<16>(half, other);
    uint32_t ninth = max(list[8], other[8]);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t a = list[i], b = list[7 - i];
      ninth = max(ninth, max(min(a, other[7 - i]), min(b, other[i])));
      list[i] = max(a, other[7 - i]);
      list[7 - i] = max(b, other[i]);
    }
#pragma unroll
    for (int s = 4; s > 0; s /= 2)
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (!(i & s)) order(list[i], list[i + s]);
    list[8] = ninth;
  } else if constexpr (N == 16) {
    uint32_t a[8], b[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      a[i] = key[i];
      b[i] = key[8 + i];
    }
    sort_8(a);
    sort_8(b);
    // the larger of each pair from both ends are the eight largest, rising and falling; the ninth is the largest of the others
    uint32_t ninth = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      list[i] = max(a[i], b[7 - i]);
      ninth = max(ninth, min(a[i], b[7 - i]));
    }
#pragma unroll
    for (int s = 4; s > 0; s /= 2)
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (!(i & s)) order(list[i], list[i + s]);
    list[8] = ninth;
  } else if constexpr (N == 8) {
    uint32_t a[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] = key[i];
    sort_8(a);
#pragma unroll
    for (int i = 0; i < 8; ++i) list[i] = a[i];
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) list[i] = key[i];
    if constexpr (N == 4) {
      order(list[0], list[1]); order(list[2], list[3]);
      order(list[0], list[2]); order(list[1], list[3]);
      order(list[1], list[2]);
    }
    if constexpr (N == 2) order(list[0], list[1]);
  }
}

// Rows by teams of 8 lanes (up to 256 experts, 8 of a row, 8 groups) or of 64, in 32 bits where that decides, else by route_row.
//   c is computed in float32, with a bound `off` of its error.  Every expert gets a key of 31 bits, its c as a whole number of 23 (21) bits between a
//   bound that the `top` largest c are above and the largest c, and 2^8 (2^10) less its number, so that keys are different and the larger one of equal
//   c is that of the lower number.
//   Each lane sorts its keys, and a round pops the largest of the lanes' first ones; where a lane may have more than nine to give
//   (teams of 64), a round takes the largest key below the one before, of differences in 32 bits the largest.  A row is settled where all of its
//   chosen keys and the next one are further apart than the errors can be, or where those that are not prove to be in order when they are compared in
//   64 bits; groups that are close leave it open.  Rows left open, rows that end early and rows with logits that are no numbers go to 64 bits: each wavefront
//   takes its own when it is through, some 6 us a row.  Of drawn scores of 256 experts some 3 rows in 10000 do, but all rows that have fewer experts than
//   `top`, and all whose float32 logits tie at the cut: 262144 rows of 256 that are equal 650 us, 262144 of 8 experts of which 8 are asked for 21 us, and 197
//   where 5% of the logits are -inf.
// Bound by vector instructions in teams of 8 (262144 rows of 256, 8 chosen, float32 and bfloat16: by logits 62 us and 61, 4.6 and 2.4 TB/s; sigmoid and bias 100
// and 100, with 4 of 8 groups 120 and 108; a wavefront to a row in 64 bits 640), whose lanes share what a row costs besides its experts: teams of 16 took 73, 108
// and 137 of float32.
template <typename T, int TEAM, int PER, bool BY_LOGIT>
__global__ __launch_bounds__(256, TEAM == 64 ? 2 : PER == 32 && !BY_LOGIT ? 3 : 4) void k_route(RouteArgs a) {
  constexpr int ROWS = 64 / TEAM, BITS = TEAM < 64 ? 8 : 10, LAST = (1 << BITS) - 1, FIELD = 31 - BITS;
  constexpr int V = PER < kPiece<T> ? 1 : kPiece<T>;                  // experts that lie next to each other
  constexpr float U = 0x1p-24f, kTop = (float)(1 << FIELD);
  constexpr int kKept = 64;                                           // rows that a wavefront puts off
  __shared__ double row_c[4][1 << BITS];
  __shared__ int32_t later[4][kKept];
  __shared__ __align__(16) float biases[BY_LOGIT ? 1 : PER / V][TEAM][V];             // as the lanes hold their experts
  const int lane = threadIdx.x & 63, t = lane % TEAM, team = lane / TEAM;
  const int lanes = a.group_lanes * TEAM / 64, g = t / lanes, sub = t % lanes;       // lanes of a group
  int first = (g < a.groups ? g : 0) * a.width + sub * V;             // element i of the lane: expert first + (i / V) lanes V + i % V
  int left = g < a.groups ? a.width - sub * V : 0;
  const bool whole = a.width == lanes * PER && a.groups * lanes == TEAM;      // every element of every lane is an expert
  auto number = [&](int i) { return first + i / V * lanes * V + i % V; };
  auto low_bits = [&](int i) { return (uint32_t)(LAST - number(i)) & (TEAM < 64 ? ~0u : (uint32_t)LAST); };
  auto count = [&](int i) { return left - i / V * lanes * V; };       // of the piece that holds element i, as far as there are any
  float bias_low = 0.f, bias_high = 0.f, bias_size = 0.f;
  if (!BY_LOGIT && a.bias) {
    bias_low = INFINITY;
    bias_high = -INFINITY;
#pragma unroll 1
    for (int p = 0; p < PER / V; ++p)
#pragma unroll 1
      for (int h = 0; h < V; ++h) {
        const bool is = h < count(p * V);
        float b = is ? a.bias[number(p * V) + h] : 0.f;
        if (b != b) b = -INFINITY;                                    // (no number in a maximum or a median)
        if (threadIdx.x < TEAM) biases[p][t][h] = b;
        if (is && b > -INFINITY) {                                    // (-inf: so is c, whatever the score)
          bias_low = fminf(bias_low, b);
          bias_high = fmaxf(bias_high, b);
        }
      }
    bias_low = team_fold<TEAM>(bias_low, smaller);
    bias_high = team_fold<TEAM>(bias_high, larger);
    bias_size = bias_low <= bias_high ? fmaxf(fabsf(bias_low), fabsf(bias_high)) : 0.f;
    __syncthreads();
  }
  int64_t base = ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 6)) * ROWS;
  while (base < a.n) {
    int kept = 0;
    for (; base < a.n && kept <= kKept - ROWS; base += (int64_t)gridDim.x * 4 * ROWS) {
      const int64_t row = base + team;
      const bool in = row < a.n;
      const T* z = (const T*)a.z + (in ? row : base) * a.z_stride;
      const unsigned long long mates = TEAM == 64 ? ~0ull : ((1ull << (TEAM & 63)) - 1) << (team * TEAM);
      asm volatile("" : "+v"(first), "+v"(left));                       // (else what follows from them is kept for all rows, in registers that are not there)
      float c[PER];
      float high = -INFINITY, low = INFINITY;
      if (whole) {
  #pragma unroll
        for (int i = 0; i < PER; i += V) {
          if constexpr (V == 1) {
            c[i] = to_float(z[number(i)]);
          } else {
            float v[V];
            load_piece(z + number(i), v);
  #pragma unroll
            for (int h = 0; h < V; ++h) c[i + h] = v[h];
          }
        }
      } else {
  #pragma unroll
        for (int i = 0; i < PER; i += V) {
          float v[V];
          load_run(z, number(i), a.experts, count(i), v);
  #pragma unroll
          for (int h = 0; h < V; ++h) c[i + h] = v[h];
        }
      }
  #pragma unroll
      for (int i = 0; i < PER; ++i) {
        high = maximum(high, c[i]);
        low = fminf(low, c[i]);
      }
      float m1 = high, m2 = -INFINITY;                                  // the lane's two largest c
      high = team_fold<TEAM>(high, maximum);
      const float from = high == -INFINITY ? 0.f : high;
      const bool empty = high == -INFINITY;
      bool settled = high < INFINITY;                                   // (NaN and inf: no)
      float total = 1.f;
      if (!a.sigmoid && (!a.renormalize || !BY_LOGIT)) {
        total = 0.f;
  #pragma unroll
        for (int i = 0; i < PER; ++i) {
          const float e = exp_below(c[i] - from);
          total += e;
          if (!BY_LOGIT) c[i] = c[i] == -INFINITY ? -INFINITY : e;
        }
        total = team_sum<TEAM>(total, nullptr);
      }
      float off = 0.f;
      if constexpr (!BY_LOGIT) {
        if (a.sigmoid) {
          // with e = exp(-z) s is off by s (1 - s) (0.85 |z log2(e)| + 2) u for the rounded product and exp2, 3 s u for 1 + e and its reciprocal
          off = 4.f * U;
          auto score = [](float v) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(v * -1.44269504f)); };
          if (__any(low == -INFINITY)) {                                // experts that are not there, for some lane of the wavefront
  #pragma unroll
            for (int i = 0; i < PER; ++i) c[i] = c[i] == -INFINITY ? -INFINITY : score(c[i]);
          } else {
  #pragma unroll
            for (int i = 0; i < PER; ++i) c[i] = score(c[i]);
          }
        } else {
          // a term is off by (2.3 d + 3) e^-d u, the sum by less than (2.3 ln experts + 3 + 40) u of itself
          const float by = __builtin_amdgcn_rcpf(total);
          off = 72.f * U * by;
  #pragma unroll
          for (int i = 0; i < PER; ++i) c[i] *= by;
        }
        if (a.bias) {
  #pragma unroll
          for (int i = 0; i < PER; ++i) c[i] += biases[i / V][t][i % V];
        }
        off += U * (1.f + bias_size);
        m1 = -INFINITY;
        if (a.groups > 1) {
  #pragma unroll
          for (int i = 0; i < PER; ++i) {
            m2 = __builtin_amdgcn_fmed3f(m1, m2, c[i]);
            m1 = fmaxf(m1, c[i]);
          }
          float g1 = m1, g2 = m2;                                       // the group's
          auto join = [&](float o1, float o2) {
            g2 = fmaxf(fminf(g1, o1), fmaxf(g2, o2));
            g1 = fmaxf(g1, o1);
          };
          if (lanes > 1) join(lane_xor<1>(g1), lane_xor<1>(g2));
          if (lanes > 2) join(lane_xor<2>(g1), lane_xor<2>(g2));
          if (lanes > 4) join(lane_xor<7>(g1), lane_xor<7>(g2));
          for (int s = 8; s < lanes; s *= 2) {
            const float o1 = __shfl_xor(g1, s), o2 = __shfl_xor(g2, s);
            join(o1, o2);
          }
          const float value = g2 == -INFINITY ? g1 : g1 + g2;
          int before = 0;                                               // groups of a larger value
          if constexpr (TEAM < 64) {
            auto against = [&]<int S>() { before += lane_xor<S>(value) > value; };
            if (lanes == 1) {
              against.template operator()<1>(); against.template operator()<3>(); against.template operator()<5>(); against.template operator()<7>();
            }
            if (lanes <= 2) {
              against.template operator()<2>(); against.template operator()<6>();
            }
            if (lanes <= 4) against.template operator()<4>();
          } else {
            for (int h = 0; h < a.groups; ++h) before += __shfl(value, h * lanes) > value;
          }
          const bool stays = before < a.top_groups && value > -INFINITY;
          const float least = team_fold<TEAM>(stays ? value : INFINITY, smaller), most = team_fold<TEAM>(stays ? -INFINITY : value, larger);
          settled &= most == -INFINITY || least - most > 4.f * off + 8.f * U * (1.f + bias_size);
          settled &= __popcll(__ballot(stays && sub == 0) & mates) <= a.top_groups;          // (more where values are equal)
          if (!stays) {
            m1 = m2 = -INFINITY;
  #pragma unroll
            for (int i = 0; i < PER; ++i) c[i] = -INFINITY;
          }
        } else {
  #pragma unroll
          for (int i = 0; i < PER; ++i) m1 = fmaxf(m1, c[i]);
        }
        high = team_fold<TEAM>(m1, larger);
      }
      uint32_t key[PER];
      int apart = -1;                                                   // keys that are no further apart settle nothing
      if constexpr (sizeof(T) == 2 && BY_LOGIT) {
        // bfloat16 logits: all 16 bits, in the order of the numbers (adding 0 makes -0 a 0)
  #pragma unroll
        for (int i = 0; i < PER; ++i) {
          const int x = __float_as_int(c[i] + 0.f);
          const uint32_t rank = (uint32_t)(x ^ (x >> 31 | INT32_MIN)) >> 16;
          key[i] = (c[i] == -INFINITY ? 0u : rank << BITS) + low_bits(i);
        }
      } else {
        // a bound that `top` experts reach: each lane's largest c, or its two largest ones, where enough lanes have them
        const int ones = __popcll(__ballot(m1 > -INFINITY) & mates), twos = __popcll(__ballot(m2 > -INFINITY) & mates);
        const bool by_two = ones < a.top;
        float bound = team_fold<TEAM>(by_two ? (m2 > -INFINITY ? m2 : INFINITY) : (m1 > -INFINITY ? m1 : INFINITY), smaller);
        if (by_two && 2 * twos < a.top) bound = high - (BY_LOGIT ? 64.f : 1.f + (bias_high - bias_low));
        const float range = fmaxf(high - bound + 4.f * off, 1e-30f), scale = (kTop - 32.f) * __builtin_amdgcn_rcpf(range);
        const float shift = fmaf(-high, scale, 0x1p24f - 16.f);         // (its rounding moves all keys alike)
        apart = 4 + (int)fminf(2.f * off * scale, kTop);
  #pragma unroll
        for (int i = 0; i < PER; ++i) {
          // below 2^24 a float32's steps are 1: the whole number stands in the low bits
          const float f = __builtin_amdgcn_fmed3f(fmaf(c[i], scale, shift), 0x1p24f - kTop, 0x1p24f - 1.f);
          key[i] = (__float_as_uint(f) << BITS) + low_bits(i);
          if (TEAM == 64) key[i] &= 0x7fffffffu;
        }
      }
      // lane j has the j-th key; `next` is the one behind the chosen ones, `last` the one behind that
      uint32_t last = 0x80000000u, mine = 0, next = 0;
      if constexpr (TEAM < 64) {
        // the lane's keys in order, as far as they can be among the `top` and the two behind: a round pops the largest of the lanes' first
        uint32_t list[10] = {};
        sort_keys<PER>(key, list);
        for (int j = 0; j <= a.top + 1; ++j) {
          last = team_max_u32<TEAM>(list[0]);
          if (t == j) mine = last;
          if (j == a.top) next = last;
          const bool mine_was = list[0] == last;
  #pragma unroll
          for (int i = 0; i < (PER < 9 ? PER : 9); ++i) list[i] = mine_was ? list[i + 1] : list[i];
          if (j < a.top) settled &= last >> BITS != 0;
        }
        settled &= PER < 10 || list[0] != 0;                            // (nine from one lane: it may have had more)
      } else {
        for (int j = 0; j <= a.top + 1; ++j) {
          uint32_t below = 0;
  #pragma unroll
          for (int i = 0; i < PER; ++i) below = max(below, key[i] - last);
          below = team_max_u32<TEAM>(below);
          last = below & 0x80000000u ? below + last : 0;                // 0: there is none
          if (t == j) mine = last;
          if (j == a.top) next = last;
          if (j < a.top) settled &= last >> BITS != 0;
        }
      }
      const uint32_t none = (1u << BITS) - 1;                           // keys up to there are of no expert
      uint32_t after = (uint32_t)__shfl_down((int)mine, 1, TEAM);
      if (t == a.top - 1) after = next;
      const bool chosen = t < a.top && mine > none;
      const int e = LAST - (int)(mine & LAST), ea = LAST - (int)(after & LAST);
      const float zc = chosen ? to_float(z[e]) : -INFINITY;
      const bool close = chosen && after > none && (int)(mine >> BITS) - (int)(after >> BITS) <= apart;
      if (__any(close)) {
        // neighbours that are close are compared in 64 bits; the last chosen one has to be apart from the key behind the next one as well
        bool right = t < a.top - 1 || last <= none || (int)(mine >> BITS) - (int)(last >> BITS) > apart;
        if (close) {
          const float za = to_float(z[ea]);
          if constexpr (BY_LOGIT) {
            right &= zc > za || (zc == za && e < ea);
          } else {
            const double bc = a.bias ? (double)a.bias[e] : 0.0, ba = a.bias ? (double)a.bias[ea] : 0.0;
            const double xc = exp(a.sigmoid ? -(double)zc : (double)zc - from), xa = exp(a.sigmoid ? -(double)za : (double)za - from);
            if (a.sigmoid) {
              const double cc = 1.0 / (1.0 + xc) + bc, ca = 1.0 / (1.0 + xa) + ba;
              right &= cc > ca || (cc == ca && e < ea);
            } else {
              // the sum of all is one of 32 bits: twice its error, of the difference
              const double d = (xc - xa) / total, sure = d + (bc - ba) - 256.0 * 0x1p-24 * fabs(d);
              right &= sure > 0.0 || (zc == za && bc == ba && e < ea);
            }
          }
          settled &= right;
        }
      }
      const float w = chosen_weight<TEAM>(zc, a.sigmoid, a.renormalize, from, total);
      // (a row without any expert is settled too: there may be many where a batch is padded)
      const unsigned long long open = __ballot(!settled);
      const bool mine_open = !empty && (open & mates) != 0;
      if (in && t < a.top && !mine_open) {
        a.expert[row * a.top + t] = empty ? -1 : e;
        a.weight[row * a.top + t] = empty ? 0.f : a.scale * w;
      }
      const unsigned long long heads = __ballot(in && t == 0 && mine_open);
      if (heads) {
        if (heads >> lane & 1) later[threadIdx.x >> 6][kept + __popcll(heads & ((1ull << lane) - 1))] = (int32_t)row;
        kept += __popcll(heads);
      }
    }
    wave_sync();
    for (int q = 0; q < kept; ++q) route_row<T>(a, later[threadIdx.x >> 6][q], row_c[threadIdx.x >> 6]);
    wave_sync();
  }
}

// The gradient of the logits from that of the weights.  With D = sum over the chosen of dw_l w_l / scale:
//   renormalised   dz_j = scale w'_j (dw_j - D)   (times 1 - s_j for sigmoid), w' the shares; 0 for experts not chosen
//   sigmoid        dz_j = scale dw_j s_j (1 - s_j)
//   softmax        dz_e = s_e (scale dw_e - sum_l scale dw_l s_l), every expert
// Bound by memory: 65536 rows of 128 bfloat16 10 us (3.7 TB/s), of 256 float32 27 us (5.2).
// A team of lanes of one wavefront holds a row.  Lane j has the j-th chosen expert.  A row without an expert has gradient 0.
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
    const float share = chosen_weight<TEAM>(zc, sigmoid, renormalize, from, total);         // of the scale
    const float dot = renormalize || all ? team_sum<TEAM>(e >= 0 ? dw * share : 0.f, nullptr) : 0.f;
    const float by = total > 0.f ? __builtin_amdgcn_rcpf(total) : 0.f;
    float mine = dw;                                       // what the chosen expert's logit gets (softmax: what its score gets)
    if (!all) {
      mine = share * (dw - dot);
      if (sigmoid) {                                       // 1 - s
        const float x = exp_near(-fabsf(zc));
        mine *= (zc > 0.f ? x : 1.f) * __builtin_amdgcn_rcpf(1.f + x);
      }
    }
    // What the others need of it goes through the team's own part of LDS: a wavefront's, which nobody else waits for.
    const unsigned long long mates = TEAM == 64 ? ~0ull : ((1ull << (TEAM & 63)) - 1) << (threadIdx.x % 64 / TEAM * TEAM);
    const bool named = (__ballot(e >= 0) & mates) != 0;
    wave_sync();                                           // the row before has been read
    if (e >= 0) up[team][e] = __int_as_float(t);
    wave_sync();
    bool first = e >= 0;
    if (__any(first && __float_as_int(up[team][max(e, 0)]) != t)) {
      // an expert that is named twice gets both parts, in order, from the first lane
      float sum = 0.f;
      for (int j = 0; j < top; ++j) {
        const int o = __shfl(e, j, TEAM);
        const float om = __shfl(mine, j, TEAM);
        if (o == e) sum += om;
        first &= o != e || j >= t;
      }
      mine = sum;
    }
    wave_sync();
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int h = 0; h < V; h += 4) *reinterpret_cast<f32x4*>(&up[team][(c * TEAM + t) * V + h]) = f32x4{0.f, 0.f, 0.f, 0.f};
    wave_sync();
    if (first) up[team][e] = mine;
    wave_sync();
    if (!in) continue;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int col = (c * TEAM + t) * V;
      float u[V];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        u[i] = up[team][col + i];
        if (all) u[i] = named ? v[c][i] * by * (u[i] - dot) : 0.f;
      }
      store_some(dz + row * dz_stride + col, experts - col, u);
    }
  }
}

// Places: (row, expert) pairs in the order of their experts, pairs of one expert in their own order.
//   offsets_e = pairs of experts before e        place = offsets_e + pairs of e before this one; -1 for pairs without an expert
// A workgroup places a tile of pairs; its wavefronts have a run each and look for equal experts 64 pairs at a time, by ballots over the bits of their
// numbers.  How many pairs of each expert lie before the tile it counts for itself, where there are few pairs in all (one launch), or adds up from
// the counts of the tiles, which a launch before it has made.  Bound by trips to memory and LDS: 2048 pairs 3.6 us, 2097152 of 256 experts 20 us.
constexpr int kOrderThreads = 1024, kOrderWaves = kOrderThreads / 64;
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
  if (threadIdx.x < experts) count[threadIdx.x] = 0;
  __syncthreads();
  const int64_t lo = (int64_t)blockIdx.x * tile, hi = min(lo + tile, pairs);
#pragma unroll 4
  for (int64_t p = lo + threadIdx.x; p < hi; p += kOrderThreads) {
    const int e = expert_of(expert, p, hi, experts, err);
    if (e >= 0) atomicAdd(&count[e], 1);
  }
  __syncthreads();
  if (threadIdx.x < experts) counts[(int64_t)blockIdx.x * experts + threadIdx.x] = count[threadIdx.x];
}

// counts null: few pairs.
__global__ __launch_bounds__(kOrderThreads) void k_order_place(int64_t pairs, int tile, int tiles, int experts, int bits,
                                                               const int32_t* __restrict__ expert, const int32_t* __restrict__ counts,
                                                               int32_t* offsets, int32_t* place, uint32_t* err) {
  __shared__ int32_t count[kOrderWaves][kMaxExperts];      // first the wavefronts' counts, then where their next pair of an expert goes
  __shared__ int32_t before[kMaxExperts], all[kMaxExperts];           // pairs of an expert in the tiles before this one, and in all
  __shared__ int32_t sums[kOrderWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, e = threadIdx.x;
#pragma unroll
  for (int w = 0; w < kOrderWaves; ++w)
    if (e < experts) count[w][e] = 0;
  if (e < experts) before[e] = all[e] = 0;
  __syncthreads();
  const int64_t lo = (int64_t)blockIdx.x * tile, hi = min(lo + tile, pairs);
  const int run = tile / kOrderWaves;
  const int64_t from = lo + (int64_t)wave * run, to = min(from + run, hi);
  if (counts) {
    // a row of counts to as many threads as there are experts, several rows at a time
    const int each = kOrderThreads / experts, slice = threadIdx.x / experts, mine = threadIdx.x % experts;
    int b = 0, s = 0;
    if (slice < each) {
#pragma unroll 8
      for (int q = slice; q < tiles; q += each) {
        const int c = counts[(int64_t)q * experts + mine];
        s += c;
        b += q < (int)blockIdx.x ? c : 0;
      }
      atomicAdd(&all[mine], s);
      atomicAdd(&before[mine], b);
    }
  } else {
#pragma unroll 4
    for (int64_t p = threadIdx.x; p < pairs; p += kOrderThreads) {
      const int q = expert_of(expert, p, pairs, experts, err);
      if (q >= 0) {
        atomicAdd(&all[q], 1);
        if (p < lo) atomicAdd(&before[q], 1);
      }
    }
  }
  for (int64_t p = from + lane; p < to; p += 64) {
    const int q = expert_of(expert, p, to, experts, err);
    if (q >= 0) atomicAdd(&count[wave][q], 1);
  }
  __syncthreads();
  const int whole = e < experts ? all[e] : 0;
  int upto = (int)wave_scan_incl((uint32_t)whole);
  if (lane == 63) sums[wave] = upto;
  __syncthreads();
  for (int w = 0; w < wave; ++w) upto += sums[w];
  if (e < experts) {
    if (blockIdx.x == 0) {
      offsets[e] = upto - whole;
      if (e == experts - 1) offsets[experts] = upto;
    }
    int at = upto - whole + before[e];
#pragma unroll
    for (int w = 0; w < kOrderWaves; ++w) {
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
    if (own >= 0) at = count[wave][own] + __popcll(same & ((1ull << lane) - 1));
    wave_sync();
    if (own >= 0 && (same >> lane) == 1ull) count[wave][own] = at + 1;      // the last of them
    wave_sync();
    if (p < to) place[p] = at;
  }
}

}  // namespace sp
