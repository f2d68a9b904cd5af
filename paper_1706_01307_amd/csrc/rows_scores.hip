// Routing by scores: sigmoid or softmax of the logits, a bias a expert for the choice alone,
// experts in groups of which the best stay, the weights renormalised and scaled.
//
// The experts of a row are those of its largest biased scores as 64-bit arithmetic has them,
// ties to the lowest expert.  Two different fp32 evaluations of a score differ in its last
// bits, and so would the choice wherever two scores lie that close, so k_scores looks at the
// gaps: it chooses by fp32 scores, and where a gap that decides something (between one
// choice and the next, between the last group that stays and the best that goes) is within
// the errors of both sides, that row is chosen again from 64-bit scores.
//
// 348,208 fp32 rows to 8 of 64 experts from 4 of 8 groups: 100 us, and 17 + 5 for the pairs'
// order, where the bytes alone would take 27; k_scores is bound by the vector ALU (75 % of the
// cycles it has work): nine searches of 16 scores a lane, then the groups, the scores and the
// rows' weights.  The gradient takes 43 us.
#include <cmath>

#include "rows_route.h"

namespace spc {
namespace {

constexpr int kMaxG = SPCONV_ROUTE_MAX_GROUPS;

// The order of 64-bit scores as unsigned numbers, as order_of: NaN largest, -0 equal to +0.
constexpr uint64_t kNone64 = 0x000fffffffffffffull;        // the order of -infinity
__device__ __forceinline__ uint64_t order_of(double v) {
  if (v != v) return ~0ull;
  const uint64_t u = __builtin_bit_cast(uint64_t, v + 0.0);
  return u >> 63 ? ~u : u | 1ull << 63;
}
__device__ __forceinline__ double value_of(uint64_t o) {
  return __builtin_bit_cast(double, o == ~0ull ? 0x7ff8000000000000ull
                                               : o >> 63 ? o & ~(1ull << 63) : ~o);
}

// The value of the lane at the other end of a butterfly step among LPR lanes.
template <int STEP> __device__ __forceinline__ uint32_t other32(uint32_t v) {
  if constexpr (STEP <= 8) return lane_other<STEP>(v);
  if constexpr (STEP == 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return threadIdx.x & 16 ? r[0] : r[1];
  }
  const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return threadIdx.x & 32 ? r[0] : r[1];
}
template <int STEP, typename V> __device__ __forceinline__ V other(V v) {
  if constexpr (sizeof(V) == 4) {
    return __builtin_bit_cast(V, other32<STEP>(__builtin_bit_cast(uint32_t, v)));
  } else {
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    const uint64_t lo = other32<STEP>(static_cast<uint32_t>(u));
    const uint64_t hi = other32<STEP>(static_cast<uint32_t>(u >> 32));
    return __builtin_bit_cast(V, hi << 32 | lo);
  }
}
// (op is commutative: it does not matter which of the two a lane's own is)
template <int STEP, typename V, typename Op> __device__ __forceinline__ V swap_step(V v, Op op) {
  if constexpr (sizeof(V) == 4) {
    const uint32_t u = __builtin_bit_cast(uint32_t, v);
    if constexpr (STEP == 16) {
      const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
      return op(__builtin_bit_cast(V, static_cast<uint32_t>(r[0])),
                __builtin_bit_cast(V, static_cast<uint32_t>(r[1])));
    } else {
      const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
      return op(__builtin_bit_cast(V, static_cast<uint32_t>(r[0])),
                __builtin_bit_cast(V, static_cast<uint32_t>(r[1])));
    }
  } else {
    return op(v, other<STEP>(v));
  }
}
template <int LPR, typename V, typename Op> __device__ __forceinline__ V over_row(V v, Op op) {
  if constexpr (LPR > 1) v = op(v, other<1>(v));
  if constexpr (LPR > 2) v = op(v, other<2>(v));
  if constexpr (LPR > 4) v = op(v, other<4>(v));
  if constexpr (LPR > 8) v = op(v, other<8>(v));
  if constexpr (LPR > 16) v = swap_step<16>(v, op);
  if constexpr (LPR > 32) v = swap_step<32>(v, op);
  return v;
}
// The largest (order, lowest column) of the row's lanes.
template <int STEP, typename U> __device__ __forceinline__ void better(U& o, uint32_t& c) {
  const U o2 = other<STEP>(o);
  const uint32_t c2 = other<STEP>(c);
  const bool take = o2 > o || (o2 == o && c2 < c);
  o = take ? o2 : o;
  c = take ? c2 : c;
}
template <int LPR, typename U> __device__ __forceinline__ void best_of_row(U& o, uint32_t& c) {
  if constexpr (LPR > 1) better<1>(o, c);
  if constexpr (LPR > 2) better<2>(o, c);
  if constexpr (LPR > 4) better<4>(o, c);
  if constexpr (LPR > 8) better<8>(o, c);
  if constexpr (LPR > 16) better<16>(o, c);
  if constexpr (LPR > 32) better<32>(o, c);
}
// LDS that the lanes of one row share: written before, read after (they are in one wave).
__device__ __forceinline__ void row_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

struct ScoreArgs {
  const void* logits;
  const float* bias;
  int64_t n;
  int E, k, softmax, groups, top_groups, normalize;
  float scale;
  int rows_blk;
  int32_t* experts;
  float* weights;
  int32_t *offsets, *rows, *pos, *counts;
  hipStream_t st;
};

constexpr float kLog2e = 1.44269504f;
constexpr float kUnit = 0x1p-22f;                  // 4 units: of a biased score, twice

// The two largest of two pairs (first >= second).
__device__ __forceinline__ void merge_two(uint32_t& a1, uint32_t& a2, uint32_t b1, uint32_t b2) {
  const uint32_t low = a1 < b1 ? a1 : b1, rest = a2 > b2 ? a2 : b2;
  a1 = a1 > b1 ? a1 : b1;
  a2 = low > rest ? low : rest;
}
// Half of what a group is worth (so that a sum of two numbers never leaves fp32), and of what its
// roundings go with: the magnitudes of its terms, which may cancel in the sum.
__device__ __forceinline__ float worth_of(uint32_t o1, uint32_t o2) {
  const float w = 0.5f * value_of(o1 > kNone ? o1 : kNone);
  return o2 > kNone ? fmaf(0.5f, value_of(o2), w) : w;
}
__device__ __forceinline__ float size_of(uint32_t o1, uint32_t o2) {
  const float w = o1 > kNone ? 0.5f * fabsf(value_of(o1)) : 0.0f;
  return o2 > kNone ? fmaf(0.5f, fabsf(value_of(o2)), w) : w;
}

// The groups of a row that stay, by fp32 scores: o, the orders of a lane's NV * VEC biased scores,
// become 0 where their group goes.  Returns whether the gap between the last group that stays and
// the best that goes is within `near` and the roundings of the worths (half a unit of each biased
// score and of their sum: kUnit of their magnitudes is twice that).  s_v: E words.
// Where a group is of whole pieces of 2^i lanes, its two best are found in registers, piece by
// piece and then over those lanes; else by reading its scores from s_v.
template <int LPR, int NV, int VEC>
__device__ __forceinline__ bool keep_groups(uint32_t (&o)[NV * VEC], int lane, const ScoreArgs& a,
                                            float near, float* s_v) {
  const int per = a.E / a.groups, span = per / VEC;          // (pieces of a group)
  const auto col = [&](int i) { return (lane + LPR * (i / VEC)) * VEC + i % VEC; };
  const auto either = [](uint32_t p, uint32_t q) { return p | q; };
  float low = INFINITY, high = -INFINITY;
  bool odd = false;                                // (NaN among them)
  // (the least that a group that stays can be worth, the most that one that goes can)
  auto note = [&](float worth, float size, bool in) {
    odd |= worth != worth;
    const float off = size < INFINITY ? kUnit * size : 0.0f;
    const float least = worth - off, most = worth + off;
    if (in) low = least < low ? least : low;
    else high = most > high ? most : high;
  };
  if (per % VEC == 0 && (span & (span - 1)) == 0 && span <= LPR) {
    uint32_t o1[NV], o2[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      o1[j] = o2[j] = 0u;
#pragma unroll
      for (int i = 0; i < VEC; ++i) merge_two(o1[j], o2[j], o[j * VEC + i], 0u);
    }
    auto step = [&](auto d) {
      if (decltype(d)::value >= span) return;
#pragma unroll
      for (int j = 0; j < NV; ++j)
        merge_two(o1[j], o2[j], other<decltype(d)::value>(o1[j]), other<decltype(d)::value>(o2[j]));
    };
    if constexpr (LPR > 1) step(std::integral_constant<int, 1>());
    if constexpr (LPR > 2) step(std::integral_constant<int, 2>());
    if constexpr (LPR > 4) step(std::integral_constant<int, 4>());
    if constexpr (LPR > 8) step(std::integral_constant<int, 8>());
    if constexpr (LPR > 16) step(std::integral_constant<int, 16>());
    if constexpr (LPR > 32) step(std::integral_constant<int, 32>());
    float worth[NV];
    uint32_t ow[NV];
    int g[NV], rank[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      worth[j] = worth_of(o1[j], o2[j]);
      ow[j] = order_of(worth[j]);
      g[j] = static_cast<int>((lane + LPR * j + 0.5f) * (1.0f / span));
      rank[j] = 0;
      if ((lane + LPR * j) % span == 0 && g[j] < a.groups) s_v[g[j]] = __uint_as_float(ow[j]);
    }
    row_fence();
    for (int q = 0; q < a.groups; ++q) {
      const uint32_t oq = __float_as_uint(s_v[q]);
#pragma unroll
      for (int j = 0; j < NV; ++j) rank[j] += oq > ow[j] || (oq == ow[j] && q < g[j]);
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const bool in = rank[j] < a.top_groups && ow[j] > kNone;
      if (g[j] < a.groups) note(worth[j], size_of(o1[j], o2[j]), in);
#pragma unroll
      for (int i = 0; i < VEC; ++i) o[j * VEC + i] = in ? o[j * VEC + i] : 0u;
    }
  } else {
#pragma unroll
    for (int i = 0; i < NV * VEC; ++i)
      if (col(i) < a.E) s_v[col(i)] = __uint_as_float(o[i]);
    row_fence();
#pragma unroll 1
    for (int g = lane; g < a.groups; g += LPR) {
      uint32_t o1 = 0, o2 = 0;
      for (int i = 0; i < per; ++i) merge_two(o1, o2, __float_as_uint(s_v[g * per + i]), 0u);
      // (in the places of its first scores; the size of one score alone is its magnitude)
      s_v[g * per] = worth_of(o1, o2);
      if (per > 1) s_v[g * per + 1] = size_of(o1, o2);
    }
    row_fence();
    uint32_t stay = 0;                             // (of this lane's groups)
    int t = 0;
#pragma unroll 1
    for (int g = lane; g < a.groups; g += LPR, ++t) {
      const float worth = s_v[g * per];
      const uint32_t ow = order_of(worth);
      int rank = 0;
      for (int q = 0; q < a.groups; ++q) {
        const uint32_t oq = order_of(s_v[q * per]);
        rank += oq > ow || (oq == ow && q < g);
      }
      const bool in = rank < a.top_groups && ow > kNone;
      note(worth, per > 1 ? s_v[g * per + 1] : ow > kNone ? fabsf(worth) : 0.0f, in);
      stay |= in ? 1u << t : 0u;
    }
    row_fence();
    t = 0;
#pragma unroll 1
    for (int g = lane; g < a.groups; g += LPR, ++t) s_v[g * per] = stay >> t & 1 ? 1.0f : 0.0f;
    row_fence();
    const float inv = 1.0f / per;
#pragma unroll
    for (int i = 0; i < NV * VEC; ++i) {
      // (exact: columns are below 2^10, and half a step from the border)
      const int g = static_cast<int>((col(i) + 0.5f) * inv);
      if (col(i) < a.E && s_v[g * per] == 0.0f) o[i] = 0u;
    }
  }
  low = over_row<LPR>(low, [](float p, float q) { return q < p ? q : p; });
  high = over_row<LPR>(high, [](float p, float q) { return q > p ? q : p; });
  if (over_row<LPR>(odd ? 1u : 0u, either)) return true;
  return a.top_groups < a.groups && high > -INFINITY && low < INFINITY && !(low - high > near);
}

// The k largest of a row's fp32 scores, of orders o, and whether a gap that decides is within
// `near` and the bias' rounding.  For the search the column, from the last one down, takes the
// place of an order's lowest bits (as many as columns have), so that one search finds both, of equal
// scores the lowest column, and no two are equal; scores that those bits would tell apart
// are computed again, two at a time (score(column), as they were).  (Value and column searched for
// apart: 116 us for 348,208 x 64 to 8, and 100 so.)
template <typename T, int LPR, int NV, int VEC, typename Score>
__device__ __forceinline__ bool choose_fast(const ScoreArgs& a, const T* logits,
                                            uint32_t (&o)[NV * VEC], int lane, float near,
                                            uint32_t mask, Score score, int16_t* s_expert) {
  constexpr int N = NV * VEC;
  const uint32_t first = mask - lane * VEC;
#pragma unroll
  for (int i = 0; i < N; ++i)
    o[i] = o[i] ? (o[i] & ~mask) | (first - (LPR * VEC * (i / VEC) + i % VEC)) : 0u;
  // of a score: kUnit, and mask + 1 units of order
  const float unit = kUnit + (mask + 1) * 0x1p-23f;
  bool close = false;
  uint32_t before = 0;
  // (on behind the last choice while those bits could tell one from it, but where many scores of
  // a long row are the same, choose_slow is the faster: all of 64 logits equal, 348,208 rows,
  // 354 us, and 697 by it; of 256, 80,000 rows, beyond 1,000 and 653)
  const int enough = a.E <= 64 ? a.E : a.k + 4;
  for (int s = 0; s < a.E; ++s) {
    if (s > enough) return true;
    uint32_t best = 0u;
#pragma unroll
    for (int i = 0; i < N; ++i) best = o[i] > best ? o[i] : best;
    best = over_row<LPR>(best, [](uint32_t p, uint32_t q) { return q > p ? q : p; });
    if (best <= kNone) {
      // none is left: nor for the slots behind
      for (int t = s + lane; t < a.k; t += LPR) s_expert[t] = -1;
      break;
    }
    const uint32_t c = mask - (best & mask);
    if (s > 0) {
      const float p = value_of(before & ~mask), q = value_of(best & ~mask);
      if (!(p - q > near + unit * (fabsf(p) + fabsf(q)))) {
        // equal logits with equal biases have equal scores in any arithmetic
        const uint32_t d = mask - (before & mask);
        if (Row<T>::get(logits[d]) != Row<T>::get(logits[c]) || (a.bias && a.bias[d] != a.bias[c])) {
          const float u = score(d), v = score(c);
          close = !(u - v > near + kUnit * (fabsf(u) + fabsf(v)));
          if (close) break;                        // (choose_slow writes the row)
        }
      } else if (s >= a.k) {
        break;
      }
    }
    if (s < a.k) before = best;
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] = o[i] == best ? 0u : o[i];
    if (lane == 0 && s < a.k) s_expert[s] = static_cast<int16_t>(c);
  }
  return close;
}

// A row again, by a whole wave in 64 bits, out of LDS: s_v has room for E scores, s_w for a
// value a group.
template <typename T>
__device__ __forceinline__ void choose_slow(const ScoreArgs& a, const T* logits, double* s_v,
                                            double* s_w, int16_t* s_expert) {
  const int lane = threadIdx.x & 63, E = a.E;
  double top = 0.0, sum = 1.0;
  if (a.softmax) {
    float t = -INFINITY;
#pragma unroll 1
    for (int c = lane; c < E; c += 64) {
      const float x = Row<T>::get(logits[c]);
      t = x > t || x != x ? x : t;
    }
    t = over_row<64>(t, [](float p, float q) { return q > p || q != q ? q : p; });
    top = t == -INFINITY ? 0.0f : t;
    sum = 0.0;
#pragma unroll 1
    for (int c = lane; c < E; c += 64) sum += exp(Row<T>::get(logits[c]) - top);
    sum = over_row<64>(sum, [](double p, double q) { return p + q; });
    if (sum == 0.0) sum = 1.0;
  }
#pragma unroll 1
  for (int c = lane; c < E; c += 64) {
    const double x = Row<T>::get(logits[c]), e = exp(a.softmax ? x - top : -x);
    const double v = (a.softmax ? e / sum : 1.0 / (1.0 + e)) + (a.bias ? a.bias[c] : 0.0f);
    s_v[c] = x == -INFINITY ? x : v;
  }
  row_fence();
  if (a.groups > 1) {                              // (a lane a group)
    const int per = E / a.groups;
    uint64_t ow = 0;
    if (lane < a.groups) {
      uint64_t o1 = 0, o2 = 0;
#pragma unroll 1
      for (int i = 0; i < per; ++i) {
        const uint64_t o = order_of(s_v[lane * per + i]);
        if (o > o1) o2 = o1, o1 = o; else if (o > o2) o2 = o;
      }
      double w = value_of(o1 > kNone64 ? o1 : kNone64);
      if (o2 > kNone64) w += value_of(o2);
      s_w[lane] = w;
      ow = order_of(w);
    }
    row_fence();
    if (lane < a.groups) {
      int rank = 0;
#pragma unroll 1
      for (int q = 0; q < a.groups; ++q) {
        const uint64_t oq = order_of(s_w[q]);
        rank += oq > ow || (oq == ow && q < lane);
      }
      if (rank >= a.top_groups)
#pragma unroll 1
        for (int i = 0; i < per; ++i) s_v[lane * per + i] = -INFINITY;
    }
    row_fence();
  }
  for (int s = 0; s < a.k; ++s) {
    uint64_t best = 0;
    uint32_t c = 0xffffffffu;
#pragma unroll 1
    for (int i = lane; i < E; i += 64) {
      const uint64_t o = order_of(s_v[i]);
      if (o > best) best = o, c = i;
    }
    best_of_row<64>(best, c);
    const bool some = best > kNone64;
    if (lane == 0) {
      s_expert[s] = static_cast<int16_t>(some ? static_cast<int32_t>(c) : -1);
      if (some) s_v[c] = -INFINITY;
    }
    row_fence();
  }
}

// Sigmoid scores below exp(kFar) are on their way out of fp32, their ratios, which renormalised
// weights are, are not: a row with a chosen one (or with fewer experts than k) has its scores
// without the factor exp(m), m the largest chosen logit or 0.  sigmoid(x) = exp(x) / (1 + exp(x));
// what x - m loses when it is rounded, up to hundreds of units of exp's value, is put back.  What 64
// bits have as 0, as they do where exp(-x) is past them, is 0: logits of a type's lowest value
// close a row too.
constexpr float kFar = -64.0f, kNothing = -709.7827f;
__device__ __forceinline__ float far_score(float x, float top) {
  if (x <= kNothing) return 0.0f;
  if (x >= 0.0f) return 1.0f / (1.0f + expf(-x));
  const float m = top < 0.0f ? top : 0.0f, d = x - m, lost = (x - d) - m, e = expf(d);
  return fmaf(e, lost, e) / (1.0f + expf(x));
}

// LPR lanes hold a row of at most LPR * NV * VEC logits, 16 a lane.
template <typename T, int LPR, int NV, bool TAIL>
__global__ __launch_bounds__(kThreads, 4) void k_scores(ScoreArgs a) {
  constexpr int VEC = Row<T>::VEC, G = kThreads / LPR, N = NV * VEC;
  static_assert(N <= 16, "the row's LDS is sized for it");
  // Rows' scores while their groups are chosen (a word apart from the next row's, for other
  // banks), then a wave's in 64 bits, then the waves' counts.
  constexpr int kWords = kThreads * 16 + G;
  __shared__ __attribute__((aligned(8))) float s_room[kWords];
  static_assert(kWords >= kWaves * kMaxE, "the counts fit");
  __shared__ int16_t s_expert[kPairs], s_slow[kThreads];
  __shared__ float s_weight[kPairs];
  __shared__ int32_t s_start[kMaxE], s_wave[kWaves], s_nslow;
  __shared__ double s_worth[kWaves][kMaxG];
  // (the whole row's softmax, where the weights ask for it: in s_start, free until then)
  float* const s_top = reinterpret_cast<float*>(s_start);
  float* const s_sum = s_top + kThreads;
  const int lane = threadIdx.x % LPR, group = threadIdx.x / LPR, E = a.E;
  const int64_t row0 = static_cast<int64_t>(blockIdx.x) * a.rows_blk;
  const int nrow = static_cast<int>(a.n - row0 < a.rows_blk ? a.n - row0 : a.rows_blk);
  const T* const logits = static_cast<const T*>(a.logits) + row0 * E;
  if (threadIdx.x == 0) s_nslow = 0;
  __syncthreads();
  float bias[NV][VEC], next[NV][VEC];
  auto request = [&](int q) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (lane + LPR * j) * VEC;
#pragma unroll
      for (int i = 0; i < VEC; ++i) next[j][i] = -INFINITY;
      if (q < nrow && c < E) {
        load_row<T, TAIL>(logits + static_cast<int64_t>(q) * E, c, E, next[j]);
        if constexpr (TAIL) {
#pragma unroll
          for (int i = 0; i < VEC; ++i)
            if (c + i >= E) next[j][i] = -INFINITY;
        }
      }
    }
  };
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = (lane + LPR * j) * VEC;
#pragma unroll
    for (int i = 0; i < VEC; ++i) bias[j][i] = 0.0f;
    if (a.bias && c < E) load_f32<VEC, TAIL>(a.bias, c, E, bias[j]);
  }
  uint32_t mask = 1;
  while (mask < static_cast<uint32_t>(E)) mask *= 2;
  --mask;                                          // (columns are at most this)
  request(group);
  for (int q = group; q < nrow; q += G) {          // (a group's lanes stay together)
    float x[N], v[N];
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = next[i / VEC][i % VEC];
    request(q + G);
    // fp32 scores: within 4 units of 1 of the sigmoid (exp2 and the reciprocal a unit each, the
    // exponent's rounding times s (1 - s) |x| < 0.28), or 32 of the softmax's largest (those,
    // times p |x| < 0.37 p's largest, and the sum of 16 terms and 6 steps); twice as
    // much for both sides of a gap
    float near = 0x1p-21f, top = -INFINITY, inv = 0.0f;
    if (a.softmax) {
      float sum = 0.0f;
#pragma unroll
      for (int i = 0; i < N; ++i) top = x[i] > top || x[i] != x[i] ? x[i] : top;
      top = over_row<LPR>(top, [](float p, float r) { return r > p || r != r ? r : p; });
      if (top == -INFINITY) top = 0.0f;
#pragma unroll
      for (int i = 0; i < N; ++i) sum += v[i] = __builtin_amdgcn_exp2f((x[i] - top) * kLog2e);
      sum = over_row<LPR>(sum, [](float p, float r) { return p + r; });
      inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] *= inv;
      near = 0x1p-18f * inv;                       // (the largest is exp(0) / sum)
      if (lane == 0) s_top[q] = top, s_sum[q] = inv;
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i)
        v[i] = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x[i] * -kLog2e));
    }
    uint32_t o[N];
#pragma unroll
    for (int i = 0; i < N; ++i)
      o[i] = x[i] == -INFINITY ? 0u : order_of(v[i] + bias[i / VEC][i % VEC]);
    bool close = false;
    if (a.groups > 1)
      close = keep_groups<LPR, NV, VEC>(o, lane, a, near, s_room + group * (LPR * N + 1));
    const T* const row = logits + static_cast<int64_t>(q) * E;
    if (!close)
      close = choose_fast<T, LPR, NV, VEC>(
          a, row, o, lane, near, mask,
          [&](uint32_t c) {
            const float xc = Row<T>::get(row[c]);
            const float vc = a.softmax ? __builtin_amdgcn_exp2f((xc - top) * kLog2e) * inv
                                       : __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(xc * -kLog2e));
            return vc + (a.bias ? a.bias[c] : 0.0f);
          },
          s_expert + q * a.k);
    if (close && lane == 0) s_slow[atomicAdd(&s_nslow, 1)] = static_cast<int16_t>(q);
  }
  __syncthreads();
  const int nslow = s_nslow, wave = threadIdx.x >> 6;
  // as many waves as the room has rows of E doubles for
  const int most = kWords / (2 * E), takes = most < kWaves ? most : kWaves;
  if (wave < takes)
    for (int i = wave; i < nslow; i += takes) {
      const int q = s_slow[i];
      choose_slow(a, logits + static_cast<int64_t>(q) * E,
                  reinterpret_cast<double*>(s_room) + wave * E, s_worth[wave], s_expert + q * a.k);
    }
  __syncthreads();
  // The weights, a row a lane, from the chosen logits.
  for (int q = threadIdx.x; q < nrow; q += kThreads) {
    const int16_t* const ex = s_expert + q * a.k;
    float* const wt = s_weight + q * a.k;
    const T* const row = logits + static_cast<int64_t>(q) * E;
    float top = a.softmax ? s_top[q] : 0.0f, sum = 0.0f;
    bool far = false;
#pragma unroll 8
    for (int t = 0; t < a.k; ++t) {
      const float x = ex[t] < 0 ? -INFINITY : Row<T>::get(row[ex[t]]);
      far |= x < kFar;
      wt[t] = x;
    }
    far &= a.normalize && !a.softmax;
    if (far || (a.softmax && a.normalize)) {
      top = -INFINITY;
      for (int t = 0; t < a.k; ++t) top = wt[t] > top || wt[t] != wt[t] ? wt[t] : top;
    }
    for (int t = 0; t < a.k; ++t) {
      const float x = wt[t];
      float w = 0.0f;
      if (ex[t] >= 0)
        w = a.softmax ? expf(x - top) : far ? far_score(x, top) : 1.0f / (1.0f + expf(-x));
      wt[t] = w;
      sum += w;
    }
    const float f = a.normalize ? 1.0f : a.softmax ? s_sum[q] : 1.0f;
    for (int t = 0; t < a.k; ++t) {
      float w = wt[t] * f;
      if (a.normalize) w = sum == 0.0f ? 0.0f : w / sum;
      wt[t] = w * a.scale;
    }
  }
  __syncthreads();
  auto& s_count = *reinterpret_cast<int32_t(*)[kWaves][kMaxE]>(s_room);
  for (int e = threadIdx.x; e < E; e += kThreads)
#pragma unroll
    for (int q = 0; q < kWaves; ++q) s_count[q][e] = 0;
  rank_pairs(a.n, E, a.k, row0, nrow, s_expert, s_weight, s_count, s_start, s_wave, a.experts,
             a.weights, a.offsets, a.rows, a.pos, a.counts);
}

struct ScoreGrad {
  const float* dweights;
  const void* logits;
  const int32_t* experts;
  const float* weights;
  int64_t n;
  int E, k, softmax, normalize;
  float scale;
  void* dlogits;
  hipStream_t st;
};

// The gradient: a row's lanes share its slots, and leave each slot's gradient at its expert's
// column in LDS, from where every lane takes its columns'.
template <typename T, int LPR, int NV, bool TAIL>
__global__ __launch_bounds__(kThreads) void k_scores_bwd(ScoreGrad a) {
  constexpr int VEC = Row<T>::VEC, G = kThreads / LPR, W = LPR * NV * VEC;
  __shared__ __attribute__((aligned(16))) float s_grad[G * W];
  const int lane = threadIdx.x % LPR, E = a.E, k = a.k;
  const int64_t r = static_cast<int64_t>(blockIdx.x) * G + threadIdx.x / LPR;
  if (r >= a.n) return;                            // (a row's lanes together; no barriers)
  const T* const logits = a.logits ? static_cast<const T*>(a.logits) + r * E : nullptr;
  float* const row = s_grad + threadIdx.x / LPR * W;
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int i = 0; i < VEC; i += 4)
      *reinterpret_cast<float4*>(row + (lane + LPR * j) * VEC + i) = make_float4(0, 0, 0, 0);
  // this lane's slots (the whole row's dot product)
  constexpr int S = (kMaxK + LPR - 1) / LPR;
  int32_t e[S];
  float w[S], dw[S], p[S], q[S];                   // (p, q: a sigmoid and 1 - it, to its own last bit)
  float dot = 0.0f;
#pragma unroll
  for (int t = 0; t < S; ++t) {
    const int s = lane + LPR * t;
    e[t] = -1, w[t] = dw[t] = p[t] = q[t] = 0.0f;
    if (LPR * t >= k) continue;                    // (uniform)
    e[t] = s < k ? a.experts[r * k + s] : -1;
    if (e[t] >= E) e[t] = -1;
    w[t] = e[t] < 0 ? 0.0f : a.weights[r * k + s];
    dw[t] = e[t] < 0 ? 0.0f : a.dweights[r * k + s];
    if (!a.softmax && e[t] >= 0) {
      const float x = Row<T>::get(logits[e[t]]), u = expf(-fabsf(x)), r = 1.0f / (1.0f + u);
      p[t] = x < 0.0f ? u * r : r;
      q[t] = x < 0.0f ? r : u * r;
    }
  }
#pragma unroll
  for (int t = 0; t < S; ++t)
    if (e[t] >= 0) dot += w[t] * dw[t];
  const auto add = [](float u, float v) { return u + v; };
  dot = over_row<LPR>(dot, add);
  float g[NV][VEC];
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int i = 0; i < VEC; ++i) g[j][i] = 0.0f;
  if (a.softmax && !a.normalize) {
    // the whole row's softmax
    float top = -INFINITY, all = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (lane + LPR * j) * VEC;
#pragma unroll
      for (int i = 0; i < VEC; ++i) g[j][i] = -INFINITY;
      if (c < E) load_row<T, TAIL>(logits, c, E, g[j]);
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        if (c + i >= E) g[j][i] = -INFINITY;
        top = g[j][i] > top || g[j][i] != g[j][i] ? g[j][i] : top;
      }
    }
    top = over_row<LPR>(top, [](float u, float v) { return v > u || v != v ? v : u; });
    if (top == -INFINITY) top = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < VEC; ++i) all += g[j][i] = expf(g[j][i] - top);
    all = over_row<LPR>(all, add);
    const float f = all == 0.0f ? 0.0f : -dot / all;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < VEC; ++i) g[j][i] *= f;
  }
  row_fence();
#pragma unroll
  for (int t = 0; t < S; ++t) {
    if (LPR * t >= k || e[t] < 0) continue;
    // (of renormalised weights alike: a weight is scale * score / sum, which fp32 can hold where
    // the scores and their sum are too small for it)
    float d;
    if (a.normalize) d = w[t] * (dw[t] - dot / a.scale);
    else d = a.softmax ? w[t] * dw[t] : dw[t] * a.scale * p[t];
    if (!a.softmax) d *= q[t];
    atomicAdd(row + e[t], d);                      // (an expert is chosen once: no order in it)
  }
  row_fence();
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = (lane + LPR * j) * VEC;
    if (c >= E) continue;
#pragma unroll
    for (int i = 0; i < VEC; ++i) g[j][i] += row[c + i];
    store_row<T, TAIL>(static_cast<T*>(a.dlogits) + r * E, c, E, g[j]);
  }
}

template <typename T, int LPR, int NV> int run(ScoreArgs a) {
  a.rows_blk = rows_per_block(a.n, a.E, a.k);
  const int nblk = a.n ? static_cast<int>((a.n + a.rows_blk - 1) / a.rows_blk) : 1;
  if (a.E % Row<T>::VEC) k_scores<T, LPR, NV, true><<<nblk, kThreads, 0, a.st>>>(a);
  else k_scores<T, LPR, NV, false><<<nblk, kThreads, 0, a.st>>>(a);
  if (nblk > 1)
    place_pairs(a.experts, a.counts, nblk, a.n, a.E, a.k, a.rows_blk, a.offsets, a.rows, a.pos,
                a.st);
  return launched();
}
template <typename T, int LPR, int NV> int run(const ScoreGrad& a) {
  const int64_t want = (a.n + kThreads / LPR - 1) / (kThreads / LPR);
  if (!grid_fits(want, kThreads)) return SPCONV_EINVAL;
  const uint32_t blocks = static_cast<uint32_t>(want);
  if (a.E % Row<T>::VEC) k_scores_bwd<T, LPR, NV, true><<<blocks, kThreads, 0, a.st>>>(a);
  else k_scores_bwd<T, LPR, NV, false><<<blocks, kThreads, 0, a.st>>>(a);
  return launched();
}
// Up to 16 logits a lane, then more lanes (k_route's reason: a step of the exchange between
// lanes costs a wave the same for 4 rows as for 16).
template <typename T, typename A> int by_width(const A& a) {
  constexpr int NV = 16 / Row<T>::VEC;
  const int pieces = (a.E + Row<T>::VEC - 1) / Row<T>::VEC;
  if (pieces <= 1) return run<T, 1, 1>(a);
  if (pieces <= 2) return run<T, 1, 2>(a);
  if (pieces <= NV) return run<T, 1, NV>(a);
  if (pieces <= 2 * NV) return run<T, 2, NV>(a);
  if (pieces <= 4 * NV) return run<T, 4, NV>(a);
  if (pieces <= 8 * NV) return run<T, 8, NV>(a);
  if (pieces <= 16 * NV) return run<T, 16, NV>(a);
  if (pieces <= 32 * NV) return run<T, 32, NV>(a);
  return run<T, 64, NV>(a);
}

bool scale_ok(float s) { return s > 0.0f && std::isfinite(s); }
bool flag_ok(int f) { return f == 0 || f == 1; }

}  // namespace
}  // namespace spc

using namespace spc;

extern "C" int spconv_route_scores_forward(int dt, const void* logits, const float* bias,
                                           int64_t n, int E, int k, int score, int groups,
                                           int top_groups, int normalize, float scale,
                                           int32_t* experts, float* weights, int32_t* offsets,
                                           int32_t* rows, int32_t* pos, void* workspace,
                                           size_t workspace_bytes, void* stream) {
  if (!dtype_ok(dt) || !flag_ok(normalize) || !flag_ok(score) || !scale_ok(scale) ||
      !sizes_ok(n, E, k) || groups < 1 || groups > kMaxG || E % groups || top_groups < 1 ||
      top_groups > groups || k > top_groups * (E / groups))
    return SPCONV_EINVAL;
  const size_t need = counts_bytes(n, E, k);
  if (!ptr_ok(logits, n, elem_bytes(dt)) || !aligned_to(bias, 4) || !ptr_ok(experts, n, 4) ||
      !ptr_ok(weights, n, 4) || !ptr_ok(offsets, 1, 4) || !ptr_ok(rows, n, 4) ||
      !ptr_ok(pos, n, 4) ||
      (need && (!workspace || !aligned_to(workspace, 16) || workspace_bytes < need)))
    return SPCONV_EINVAL;
  // (no rows: one workgroup without rows writes the offsets)
  const ScoreArgs a{logits, bias, n, E, k, score, groups, top_groups, normalize, scale, 0,
                    experts, weights, offsets, rows, pos, static_cast<int32_t*>(workspace),
                    static_cast<hipStream_t>(stream)};
  return dt == SPCONV_BF16 ? by_width<bf16_t>(a) : by_width<float>(a);
}

extern "C" int spconv_route_scores_backward(int dt, const float* dweights, const void* logits,
                                            const int32_t* experts, const float* weights,
                                            int64_t n, int E, int k, int score, int normalize,
                                            float scale, void* dlogits, void* stream) {
  if (!dtype_ok(dt) || !flag_ok(normalize) || !flag_ok(score) || !scale_ok(scale) ||
      !sizes_ok(n, E, k))
    return SPCONV_EINVAL;
  const bool reads = score == SPCONV_SCORE_SIGMOID || !normalize;
  if (!ptr_ok(dweights, n, 4) || !ptr_ok(logits, reads ? n : 0, elem_bytes(dt)) ||
      !ptr_ok(experts, n, 4) || !ptr_ok(weights, n, 4) || !ptr_ok(dlogits, n, elem_bytes(dt)))
    return SPCONV_EINVAL;
  if (n == 0) return SPCONV_OK;
  const ScoreGrad a{dweights, logits, experts, weights, n, E, k, score, normalize, scale, dlogits,
                    static_cast<hipStream_t>(stream)};
  return dt == SPCONV_BF16 ? by_width<bf16_t>(a) : by_width<float>(a);
}
