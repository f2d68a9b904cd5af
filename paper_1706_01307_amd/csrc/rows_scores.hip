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

// The scores of a lane's NV * VEC columns of a row, x: sigmoid, or softmax with the row's
// maximum `top` (0 if all are closed).  fp32 ones are within 4 units of the sigmoid's or 32
// of the softmax's last place (expf, the sum of 16 terms and 6 steps, a division).
template <typename F, int LPR, int NV, int VEC>
__device__ __forceinline__ void scores_of(const float (&x)[NV][VEC], bool softmax, float top,
                                          F (&s)[NV][VEC]) {
  F sum = 0;
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      const F a = softmax ? static_cast<F>(x[j][i]) - static_cast<F>(top) : -static_cast<F>(x[j][i]);
      F e;
      if constexpr (sizeof(F) == 4) e = expf(a); else e = exp(a);
      s[j][i] = softmax ? e : F(1) / (F(1) + e);
      sum += e;
    }
  if (softmax) {
    sum = over_row<LPR>(sum, [](F a, F b) { return a + b; });
    const F inv = sum == 0 ? F(0) : F(1) / sum;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < VEC; ++i) s[j][i] = sizeof(F) == 4 ? s[j][i] * inv : s[j][i] / (sum == 0 ? F(1) : sum);
  }
}

// The choice of one row from its biased scores v (-infinity: closed), of which `keep` is what
// is kept of a chosen one.  near: twice the error of an fp32 score; the function returns
// whether a gap that decides is within it (F double: never).  s_v, s_worth: the row's own LDS.
template <typename T, typename F, int LPR, int NV, int VEC>
__device__ __forceinline__ bool choose(const ScoreArgs& a, const T* logits, F (&v)[NV][VEC],
                                       const float (&keep)[NV][VEC], F near, F* s_v, F* s_worth,
                                       int16_t* s_expert, float* s_weight) {
  typedef Order<F> O;
  typedef typename O::U U;
  constexpr bool kFast = sizeof(F) == 4;
  constexpr F kUnit = F(0x1p-22);                  // 4 units: of the biased score, twice
  const int lane = threadIdx.x % LPR, E = a.E;
  bool close = false;
  if (a.groups > 1) {
    const int per = E / a.groups;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const int c = (lane + LPR * j) * VEC + i;
        if (c < E) s_v[c] = v[j][i];
      }
    row_fence();
    // a group is worth its two best
    for (int g = lane; g < a.groups; g += LPR) {
      U o1 = 0, o2 = 0;
      for (int i = 0; i < per; ++i) {
        const U o = O::of(s_v[g * per + i]);
        if (o > o1) o2 = o1, o1 = o; else if (o > o2) o2 = o;
      }
      F worth = O::value(o1 > O::kClosed ? o1 : O::kClosed);
      if (o2 > O::kClosed) worth += O::value(o2);
      s_worth[g] = worth;
    }
    row_fence();
    uint32_t stay[2] = {0u, 0u};
    F low = INFINITY, high = -INFINITY;            // the last that stays, the best that goes
    bool odd = false;                              // (NaN among them)
    for (int g = lane; g < a.groups; g += LPR) {
      const F worth = s_worth[g];
      const U o = O::of(worth);
      int rank = 0;
      for (int q = 0; q < a.groups; ++q) {
        const U oq = O::of(s_worth[q]);
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
    stay[1] = over_row<LPR>(stay[1], either);
    if constexpr (kFast) {
      low = over_row<LPR>(low, [](F p, F q) { return q < p ? q : p; });
      high = over_row<LPR>(high, [](F p, F q) { return q > p ? q : p; });
      close |= over_row<LPR>(odd ? 1u : 0u, either) != 0;
      if (a.top_groups < a.groups && high > -INFINITY && low < INFINITY)
        close |= !(low - high > 2 * near + 2 * kUnit * (fabsf(low) + fabsf(high)));
    }
    const float inv = 1.0f / per;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        // (exact: columns are below 2^10, and half a step from the border)
        const int g = static_cast<int>(((lane + LPR * j) * VEC + i + 0.5f) * inv);
        if (!((stay[(g >> 5) & 1] >> (g & 31)) & 1u)) v[j][i] = -INFINITY;
      }
  }
  U o[NV][VEC];
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int i = 0; i < VEC; ++i) o[j][i] = (lane + LPR * j) * VEC + i < E ? O::of(v[j][i]) : 0u;
  U before = 0;
  uint32_t before_c = 0;
  // (fp32: one more than is chosen, and on while it ties with the last)
  for (int s = 0; s < E; ++s) {
    if (s >= a.k && (!kFast || s > a.k)) break;
    U bo = 0;
    uint32_t bc = 0xffffffffu;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < VEC; ++i)
        if (o[j][i] > bo) {                        // ascending columns: the lowest of equals
          bo = o[j][i];
          bc = (lane + LPR * j) * VEC + i;
        }
    best_of_row<LPR>(bo, bc);
    const bool some = bo > O::kClosed;
    if constexpr (kFast) {
      if (s > 0 && some) {
        const F p = O::value(before), q = O::value(bo);
        if (!(p - q > near + kUnit * (fabsf(p) + fabsf(q)))) {
          // equal logits with equal biases have equal scores in any arithmetic
          bool same = Row<T>::get(logits[before_c]) == Row<T>::get(logits[bc]) &&
                      (!a.bias || a.bias[before_c] == a.bias[bc]);
          // (past the last choice a tie hides what comes behind it)
          close |= !same || s >= a.k;
        }
      }
      before = bo;
      before_c = bc;
      if (s >= a.k) break;
    }
    float mine = 0.0f;
    bool owner = false;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < VEC; ++i)
        if (static_cast<uint32_t>((lane + LPR * j) * VEC + i) == bc) {
          o[j][i] = 0u;                            // take it out
          mine = keep[j][i];
          owner = true;
        }
    if (some ? owner : lane == 0) {
      s_expert[s] = static_cast<int16_t>(some ? static_cast<int32_t>(bc) : -1);
      s_weight[s] = mine;
    }
    if (!some && s + 1 < a.k) {
      // none is left: nor for the slots behind
      for (int t = s + 1 + lane; t < a.k; t += LPR) s_expert[t] = -1, s_weight[t] = 0.0f;
      break;
    }
  }
  return close;
}

// LPR lanes hold a row of at most LPR * NV * VEC logits, 16 a lane.
template <typename T, int LPR, int NV, bool TAIL>
__global__ __launch_bounds__(kThreads) void k_scores(ScoreArgs a) {
  constexpr int VEC = Row<T>::VEC, G = kThreads / LPR;
  static_assert(NV * VEC <= 16, "the row's LDS is sized for it");
  __shared__ int16_t s_expert[kPairs];
  __shared__ float s_weight[kPairs];
  // a row's scores (a word apart from the next row's, for other banks), its groups' worth;
  // then the waves' counts
  constexpr int kWords = kThreads * 16 + G, kWorth = G * (LPR < 16 ? LPR * 16 < kMaxG ? LPR * 16 : kMaxG : kMaxG);
  __shared__ double s_room[kWords];
  __shared__ double s_worth[kWorth];
  __shared__ int32_t s_start[kMaxE], s_wave[kWaves];
  static_assert(sizeof(s_room) >= sizeof(int32_t) * kWaves * kMaxE, "the counts fit");
  const int lane = threadIdx.x % LPR, group = threadIdx.x / LPR, E = a.E;
  const int64_t row0 = static_cast<int64_t>(blockIdx.x) * a.rows_blk;
  const int nrow = static_cast<int>(a.n - row0 < a.rows_blk ? a.n - row0 : a.rows_blk);
  const T* const logits = static_cast<const T*>(a.logits);
  constexpr int kRowWorth = kWorth / G;
  float bias[NV][VEC], x[NV][VEC], next[NV][VEC];
  auto request = [&](int q) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (lane + LPR * j) * VEC;
#pragma unroll
      for (int i = 0; i < VEC; ++i) next[j][i] = -INFINITY;
      if (q < nrow && c < E) {
        load_row<T, TAIL>(logits + (row0 + q) * E, c, E, next[j]);
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
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < VEC; ++i) x[j][i] = next[j][i];
    request(q + G);
    float top = -INFINITY;
    if (a.softmax) {
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < VEC; ++i) top = x[j][i] > top || x[j][i] != x[j][i] ? x[j][i] : top;
      top = over_row<LPR>(top, [](float p, float r) { return r > p || r != r ? r : p; });
      if (top == -INFINITY) top = 0.0f;
    }
    // what is kept of a chosen score: the score, or, for weights by a softmax over the
    // chosen, the logit
    float s[NV][VEC], v[NV][VEC];
    scores_of<float, LPR>(x, a.softmax, top, s);
    float most = 1.0f;
    if (a.softmax) {
      most = 0.0f;
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < VEC; ++i) most = s[j][i] > most ? s[j][i] : most;
      most = 8.0f * over_row<LPR>(most, [](float p, float r) { return r > p ? r : p; });
    }
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        v[j][i] = x[j][i] == -INFINITY ? -INFINITY : s[j][i] + bias[j][i];
        if (a.softmax && a.normalize) s[j][i] = x[j][i];
      }
    int16_t* const ex = s_expert + q * a.k;
    float* const wt = s_weight + q * a.k;
    const int at = group * (LPR * NV * VEC + 1);
    const T* const row = logits + (row0 + q) * E;
    // 8 units of the largest score (softmax: 64)
    const bool close = choose<T, float, LPR, NV, VEC>(
        a, row, v, s, 0x1p-21f * most, reinterpret_cast<float*>(s_room + at),
        reinterpret_cast<float*>(s_worth + group * kRowWorth), ex, wt);
    if (close) {                                   // (the same for all of the row's lanes)
      double d[NV][VEC];
      scores_of<double, LPR>(x, a.softmax, top, d);
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < VEC; ++i)
          d[j][i] = x[j][i] == -INFINITY ? -INFINITY : d[j][i] + bias[j][i];
      row_fence();
      choose<T, double, LPR, NV, VEC>(a, row, d, s, 0.0, s_room + at, s_worth + group * kRowWorth,
                                      ex, wt);
    }
    row_fence();
    // The weights, every lane those of its slots.
    float peak = -INFINITY, sum = 0.0f;
    if (a.normalize) {
      if (a.softmax) {
        for (int t = 0; t < a.k; ++t)
          if (ex[t] >= 0) peak = wt[t] > peak || wt[t] != wt[t] ? wt[t] : peak;
      }
      for (int t = 0; t < a.k; ++t)
        if (ex[t] >= 0) sum += a.softmax ? expf(wt[t] - peak) : wt[t];
    }
    row_fence();
    for (int t = lane; t < a.k; t += LPR) {
      float w = ex[t] < 0 ? 0.0f : wt[t];
      if (a.normalize) {
        if (a.softmax && ex[t] >= 0) w = expf(w - peak);
        w = sum == 0.0f ? 0.0f : w / sum;
      }
      wt[t] = w * a.scale;
    }
    row_fence();
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
