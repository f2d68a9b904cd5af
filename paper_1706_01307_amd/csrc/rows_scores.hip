// Routing by scores: sigmoid or softmax of the logits, a bias a expert for the choice alone,
// experts in groups of which the best stay, the weights renormalised and scaled.
//
// The experts of a row are those of its largest biased scores as 64-bit arithmetic has them,
// ties to the lowest expert.  Two different fp32 evaluations of a score differ in its last
// bits, and so would the choice wherever two scores lie that close, so k_scores looks at the
// gaps: it chooses by fp32 scores, and where a gap that decides something (between one
// choice and the next, between the last group that stays and the best that goes) is within
// the errors of both sides, that row is chosen again from 64-bit scores.
#include <cmath>

#include "rows_route.h"

namespace spc {
namespace {

constexpr int kMaxG = SPCONV_ROUTE_MAX_GROUPS;

// The order of scores as unsigned numbers, as order_of: NaN largest, -0 equal to +0.
template <typename F> struct Order;
template <> struct Order<float> {
  typedef uint32_t U;
  static constexpr U kClosed = kNone;              // -infinity
  __device__ static U of(float v) { return order_of(v); }
  __device__ static float value(U o) { return value_of(o); }
};
template <> struct Order<double> {
  typedef uint64_t U;
  static constexpr U kClosed = 0x000fffffffffffffull;
  __device__ static U of(double v) {
    if (v != v) return ~0ull;
    const U u = __builtin_bit_cast(U, v + 0.0);
    return u >> 63 ? ~u : u | 1ull << 63;
  }
  __device__ static double value(U o) {
    return __builtin_bit_cast(double, o == ~0ull ? 0x7ff8000000000000ull
                                                 : o >> 63 ? o & ~(1ull << 63) : ~o);
  }
};

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
template <int LPR, typename V, typename Op> __device__ __forceinline__ V over_row(V v, Op op) {
  if constexpr (LPR > 1) v = op(v, other<1>(v));
  if constexpr (LPR > 2) v = op(v, other<2>(v));
  if constexpr (LPR > 4) v = op(v, other<4>(v));
  if constexpr (LPR > 8) v = op(v, other<8>(v));
  if constexpr (LPR > 16) v = op(v, other<16>(v));
  if constexpr (LPR > 32) v = op(v, other<32>(v));
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

// What a wave or a part of it shares of a row in LDS: the groups' choice.  v: a lane's biased
// scores, N of them, of columns col(i) (those of E and beyond, and closed ones, -infinity); on
// return those of groups that go are -infinity too.  s_v: E words; a group's worth takes the
// place of its first score.  The gap between the last group that stays and the best that goes is
// returned as whether it is within `near` and the roundings of a sum.
template <typename F, int LPR, int N, typename Col>
__device__ __forceinline__ bool keep_groups(F (&v)[N], Col col, int lane, const ScoreArgs& a,
                                            F near, F unit, F* s_v) {
  typedef Order<F> O;
  typedef typename O::U U;
  const int per = a.E / a.groups;
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (col(i) < a.E) s_v[col(i)] = v[i];
  row_fence();
  for (int g = lane; g < a.groups; g += LPR) {
    U o1 = 0, o2 = 0;
    for (int i = 0; i < per; ++i) {
      const U o = O::of(s_v[g * per + i]);
      if (o > o1) o2 = o1, o1 = o; else if (o > o2) o2 = o;
    }
    F worth = O::value(o1 > O::kClosed ? o1 : O::kClosed);
    if (o2 > O::kClosed) worth += O::value(o2);
    s_v[g * per] = worth;
  }
  row_fence();
  uint32_t stay[2] = {0u, 0u};
  F low = INFINITY, high = -INFINITY;              // the last that stays, the best that goes
  bool odd = false;                                // (NaN among them)
  for (int g = lane; g < a.groups; g += LPR) {
    const F worth = s_v[g * per];
    const U o = O::of(worth);
    int rank = 0;
    for (int q = 0; q < a.groups; ++q) {
      const U oq = O::of(s_v[q * per]);
      rank += oq > o || (oq == o && q < g);
    }
    const bool in = rank < a.top_groups && o > O::kClosed;
    if (in) stay[g >> 5] |= 1u << (g & 31);
    odd |= worth != worth;
    if (in) low = worth < low ? worth : low;
    else high = worth > high ? worth : high;
  }
  const auto either = [](uint32_t p, uint32_t q) { return p | q; };
  stay[0] = over_row<LPR>(stay[0], either);
  if (a.groups > 32) stay[1] = over_row<LPR>(stay[1], either);
  bool close = false;
  if (unit > 0) {
    low = over_row<LPR>(low, [](F p, F q) { return q < p ? q : p; });
    high = over_row<LPR>(high, [](F p, F q) { return q > p ? q : p; });
    close = over_row<LPR>(odd ? 1u : 0u, either) != 0;
    if (a.top_groups < a.groups && high > -INFINITY && low < INFINITY)
      close |= !(low - high > 2 * near + 2 * unit * (fabsf(low) + fabsf(high)));
  }
  const float inv = 1.0f / per;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    // (exact: columns are below 2^10, and half a step from the border)
    const int g = static_cast<int>((col(i) + 0.5f) * inv);
    if (!((stay[(g >> 5) & 1] >> (g & 31)) & 1u)) v[i] = -INFINITY;
  }
  return close;
}

// The k largest of a row's fp32 scores, and whether a gap that decides is within `near` and the
// bias' rounding.  The largest value of the row is found first and its lowest column then: fewer
// operations than with both at once, and the score itself need not be carried (rows_weights
// takes the chosen logits again).
template <typename T, int LPR, int N, typename Col>
__device__ __forceinline__ bool choose_fast(const ScoreArgs& a, const T* logits,
                                            const float (&v)[N], Col col, int lane, float near,
                                            float unit, int16_t* s_expert) {
  uint32_t o[N];
#pragma unroll
  for (int i = 0; i < N; ++i) o[i] = col(i) < a.E ? order_of(v[i]) : 0u;
  bool close = false;
  uint32_t before = 0, before_c = 0;
  // (one more than is chosen)
  const int last = a.k < a.E ? a.k : a.k - 1;
  for (int s = 0; s <= last; ++s) {
    uint32_t best = 0u;
#pragma unroll
    for (int i = 0; i < N; ++i) best = o[i] > best ? o[i] : best;
    best = over_row<LPR>(best, [](uint32_t p, uint32_t q) { return q > p ? q : p; });
    if (best <= kNone) {
      // none is left: nor for the slots behind
      for (int t = s + lane; t < a.k; t += LPR) s_expert[t] = -1;
      break;
    }
    int mine = N;
#pragma unroll
    for (int i = N - 1; i >= 0; --i) mine = o[i] == best ? i : mine;
    uint32_t c = 0xffffffffu;
    if (mine < N) c = col(mine);
    const uint32_t own = c;
    c = over_row<LPR>(c, [](uint32_t p, uint32_t q) { return q < p ? q : p; });
    if (s > 0) {
      const float p = value_of(before), q = value_of(best);
      if (!(p - q > near + unit * (fabsf(p) + fabsf(q)))) {
        // equal logits with equal biases have equal scores in any arithmetic (but past
        // the last choice a tie hides what comes behind it)
        close |= s >= a.k || Row<T>::get(logits[before_c]) != Row<T>::get(logits[c]) ||
                 (a.bias && a.bias[before_c] != a.bias[c]);
      }
    }
    before = best;
    before_c = c;
    if (s >= a.k) break;
    mine = own == c ? mine : N;
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] = i == mine ? 0u : o[i];
    if (lane == 0) s_expert[s] = static_cast<int16_t>(c);
  }
  return close;
}

// A row again, by a whole wave in 64 bits.
template <typename T>
__device__ void choose_slow(const ScoreArgs& a, const T* logits, double* s_v, int16_t* s_expert) {
  constexpr int N = kMaxE / 64;
  typedef Order<double> O;
  const int lane = threadIdx.x & 63;
  const auto col = [&](int i) { return lane + 64 * i; };
  double v[N];
  float top = -INFINITY;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float x = col(i) < a.E ? Row<T>::get(logits[col(i)]) : -INFINITY;
    v[i] = x;
    top = x > top || x != x ? x : top;
  }
  if (a.softmax) {
    top = over_row<64>(top, [](float p, float q) { return q > p || q != q ? q : p; });
    if (top == -INFINITY) top = 0.0f;
  }
  double sum = 0.0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if (64 * i >= a.E) break;
    const double x = v[i];
    const double e = exp(a.softmax ? x - static_cast<double>(top) : -x);
    sum += e;
    v[i] = x == -INFINITY ? -INFINITY : a.softmax ? e : 1.0 / (1.0 + e);
  }
  if (a.softmax) {
    sum = over_row<64>(sum, [](double p, double q) { return p + q; });
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = v[i] == -INFINITY ? v[i] : v[i] / (sum == 0.0 ? 1.0 : sum);
  }
  if (a.bias) {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (col(i) < a.E && v[i] != -INFINITY) v[i] += a.bias[col(i)];
  }
  if (a.groups > 1) keep_groups<double, 64>(v, col, lane, a, 0.0, 0.0, s_v);
  uint64_t o[N];
#pragma unroll
  for (int i = 0; i < N; ++i) o[i] = col(i) < a.E ? O::of(v[i]) : 0u;
  for (int s = 0; s < a.k; ++s) {
    uint64_t best = 0;
    uint32_t c = 0xffffffffu;
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (o[i] > best) best = o[i], c = col(i);
    best_of_row<64>(best, c);
    const bool some = best > O::kClosed;
    if (lane == 0) s_expert[s] = static_cast<int16_t>(some ? static_cast<int32_t>(c) : -1);
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (static_cast<uint32_t>(col(i)) == c) o[i] = 0;
  }
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
  // (the whole row's softmax, where the weights ask for it: in s_start, free until then)
  float* const s_top = reinterpret_cast<float*>(s_start);
  float* const s_sum = s_top + kThreads;
  const int lane = threadIdx.x % LPR, group = threadIdx.x / LPR, E = a.E;
  const int64_t row0 = static_cast<int64_t>(blockIdx.x) * a.rows_blk;
  const int nrow = static_cast<int>(a.n - row0 < a.rows_blk ? a.n - row0 : a.rows_blk);
  const T* const logits = static_cast<const T*>(a.logits) + row0 * E;
  const auto col = [&](int i) { return (lane + LPR * (i / VEC)) * VEC + i % VEC; };
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
  request(group);
  for (int q = group; q < nrow; q += G) {          // (a group's lanes stay together)
    float x[N], v[N];
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = next[i / VEC][i % VEC];
    request(q + G);
    // fp32 scores: within 4 units of the sigmoid, or 32 of the softmax's largest (exp, the
    // sum of 16 terms and 6 steps, a division); twice as much for both sides of a gap
    float near = 0x1p-21f;
    if (a.softmax) {
      float top = -INFINITY, sum = 0.0f;
#pragma unroll
      for (int i = 0; i < N; ++i) top = x[i] > top || x[i] != x[i] ? x[i] : top;
      top = over_row<LPR>(top, [](float p, float r) { return r > p || r != r ? r : p; });
      if (top == -INFINITY) top = 0.0f;
#pragma unroll
      for (int i = 0; i < N; ++i) sum += v[i] = expf(x[i] - top);
      sum = over_row<LPR>(sum, [](float p, float r) { return p + r; });
      const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] *= inv;
      near = 0x1p-18f * inv;                       // (the largest is exp(0) / sum)
      if (lane == 0) s_top[q] = top, s_sum[q] = inv;
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = __builtin_amdgcn_rcpf(1.0f + expf(-x[i]));
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
      v[i] = x[i] == -INFINITY ? -INFINITY : v[i] + bias[i / VEC][i % VEC];
    constexpr float kUnit = 0x1p-22f;              // 4 units: of the biased score, twice
    bool close = false;
    if (a.groups > 1)
      close = keep_groups<float, LPR>(v, col, lane, a, near, kUnit,
                                      s_room + group * (LPR * N + 1));
    close |= choose_fast<T, LPR>(a, logits + static_cast<int64_t>(q) * E, v, col, lane, near, kUnit,
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
                  reinterpret_cast<double*>(s_room) + wave * E, s_expert + q * a.k);
    }
  __syncthreads();
  // The weights, a row a lane, from the chosen logits.
  for (int q = threadIdx.x; q < nrow; q += kThreads) {
    const int16_t* const ex = s_expert + q * a.k;
    float* const wt = s_weight + q * a.k;
    const T* const row = logits + static_cast<int64_t>(q) * E;
    float top = a.softmax ? s_top[q] : 0.0f, sum = 0.0f;
#pragma unroll 8
    for (int t = 0; t < a.k; ++t) wt[t] = ex[t] < 0 ? -INFINITY : Row<T>::get(row[ex[t]]);
    if (a.softmax && a.normalize) {
      top = -INFINITY;
      for (int t = 0; t < a.k; ++t) top = wt[t] > top || wt[t] != wt[t] ? wt[t] : top;
    }
    for (int t = 0; t < a.k; ++t) {
      const float x = wt[t];
      float w = 0.0f;
      if (ex[t] >= 0) w = a.softmax ? expf(x - top) : 1.0f / (1.0f + expf(-x));
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

// The gradient: every lane sums the row's slots itself (they are the same addresses for the
// whole row), then finds its columns among them.
template <typename T, int LPR, int NV, bool TAIL>
__global__ __launch_bounds__(kThreads) void k_scores_bwd(ScoreGrad a) {
  constexpr int VEC = Row<T>::VEC, G = kThreads / LPR;
  const int lane = threadIdx.x % LPR, E = a.E, k = a.k;
  const int64_t r = static_cast<int64_t>(blockIdx.x) * G + threadIdx.x / LPR;
  if (r >= a.n) return;
  const T* const logits = a.logits ? static_cast<const T*>(a.logits) + r * E : nullptr;
  float g[NV][VEC];
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int i = 0; i < VEC; ++i) g[j][i] = 0.0f;
  float dot = 0.0f, sum = 0.0f;
  auto expert = [&](int s) {
    const int32_t e = a.experts[r * k + s];
    return e < E ? e : -1;
  };
  auto score = [&](int32_t e) { return 1.0f / (1.0f + expf(-Row<T>::get(logits[e]))); };
  for (int s = 0; s < k; ++s) {
    const int32_t e = expert(s);
    if (e < 0) continue;
    dot += a.weights[r * k + s] * a.dweights[r * k + s];
    if (!a.softmax && a.normalize) sum += score(e);
  }
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
    top = over_row<LPR>(top, [](float p, float q) { return q > p || q != q ? q : p; });
    if (top == -INFINITY) top = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < VEC; ++i) all += g[j][i] = expf(g[j][i] - top);
    all = over_row<LPR>(all, [](float p, float q) { return p + q; });
    const float f = all == 0.0f ? 0.0f : -dot / all;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < VEC; ++i) g[j][i] *= f;
  }
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
  for (int s = 0; s < k; ++s) {
    const int32_t e = expert(s);
    if (e < 0) continue;
    const float w = a.weights[r * k + s], dw = a.dweights[r * k + s];
    float d;
    if (a.softmax) {
      d = w * (a.normalize ? dw - dot / a.scale : dw);
    } else {
      const float p = score(e);
      d = a.normalize ? (dw * a.scale - dot) * inv : dw * a.scale;
      d = d * p * (1.0f - p);
    }
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < VEC; ++i)
        if ((lane + LPR * j) * VEC + i == e) g[j][i] += d;
  }
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = (lane + LPR * j) * VEC;
    if (c < E) store_row<T, TAIL>(static_cast<T*>(a.dlogits) + r * E, c, E, g[j]);
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
