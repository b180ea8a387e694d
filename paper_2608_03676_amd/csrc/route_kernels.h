// Routing of tokens to experts: scores, an optional balance bias, groups,
// top-k and weights; and the gradient by the logits.
//
//   score  s = softmax(x) or sigmoid(x);   key = s + bias, or x without a bias
//   groups: the best `top_groups` of `groups` equal runs of experts stay, by
//           their largest key, or by the sum of their two largest s + bias
//           (without a bias s, of the softmax without its common divisor: x has
//           the order of s, but a sum of two x not that of two s)
//   chosen: the k largest keys, the lower expert first among equals
//   weight: c s;  renormalised: c softmax over the chosen x, or c s / (sum s + 1e-20)
//
// An expert whose logit or key is NaN or -inf is not chosen; places that are
// left over hold expert -1 and weight 0.
//
// A token's experts lie in the registers of L lanes as ordered integer keys, V
// a lane; a round takes the maximum over them and removes it.  Keys are
// computed with single roundings (no approximations), so that choices are
// those of the formulas in 32 bits, ties included.
#pragma once

#include <type_traits>

#include "route.h"
#include "rowio.h"

namespace taot {
namespace {

constexpr int kNone = INT32_MIN;     // key of an expert that cannot be chosen
constexpr float kTiny = 1e-20f;
constexpr float kBig = 3.402823466e38f;

// Integers in the order of the floats (-0 is 0).
__device__ __forceinline__ int ordered(float x) {
  const int b = __float_as_int(x + 0.f);
  return b ^ ((b >> 31) & 0x7fffffff);
}
__device__ __forceinline__ float unordered(int b) { return __int_as_float(b ^ ((b >> 31) & 0x7fffffff)); }

// Key of a float that may not be chosen when it is NaN or -inf.
__device__ __forceinline__ int key_of(float x) { return x > -INFINITY ? ordered(x) : kNone; }

__device__ __forceinline__ float sigmoid(float x) { return 1.f / (1.f + expf(-x)); }

// Without a bias: value of a group by two, from its two largest logits (-infinity: none); m: the token's largest.
__device__ __forceinline__ int two_scores(const RouteArgs& a, float x1, float x2, float m) {
  if (!(x1 > -INFINITY)) return kNone;
  return ordered(a.flags & TAOT_ROUTE_SIGMOID ? sigmoid(x1) + sigmoid(x2) : expf(x1 - m) + expf(x2 - m));
}

// Value of a group from its two largest keys.
__device__ __forceinline__ int group_value(const RouteArgs& a, int b1, int b2, float m) {
  if (!(a.flags & TAOT_ROUTE_GROUP_TWO) || b1 == kNone) return b1;
  const float x2 = b2 == kNone ? -INFINITY : unordered(b2);
  if (!a.bias) return two_scores(a, unordered(b1), x2, m);
  return b2 == kNone ? b1 : ordered(unordered(b1) + x2);
}

// Whether the largest logit and the sum of exponentials are needed: of every softmax score that is more than a weight
// among the chosen.
__device__ __forceinline__ bool needs_sum(const RouteArgs& a) {
  if (a.flags & TAOT_ROUTE_SIGMOID) return false;
  return a.bias || !(a.flags & TAOT_ROUTE_RENORM) || (a.groups > 1 && (a.flags & TAOT_ROUTE_GROUP_TWO));
}

// Weights of the chosen experts; lane j of a block of L has the j-th (id -1: none).
// m, sum: the largest logit and the sum of exp(x - m), where the plain softmax needs them.
template <int L>
__device__ __forceinline__ void finish_with(const RouteArgs& a, int64_t t, bool mine, int j, int id, float x, float m,
                                            float sum) {
  const bool has = mine && id >= 0 && id < a.E;
  float w;
  if (a.flags & TAOT_ROUTE_SIGMOID) {
    w = has ? sigmoid(x) : 0.f;
    if (a.flags & TAOT_ROUTE_RENORM) w = w / (block_reduce<L>(w, SumOp()) + kTiny);
  } else if (a.flags & TAOT_ROUTE_RENORM) {
    const float top = block_reduce<L>(x, MaxOp());
    w = has ? expf(x - top) : 0.f;
    const float total = block_reduce<L>(w, SumOp());
    w = has ? w / total : 0.f;
  } else {
    w = has ? expf(x - m) / sum : 0.f;
  }
  if (mine) {
    a.ids[t * a.k + j] = has ? id : -1;
    a.weights[t * a.k + j] = w * a.scale;
  }
}
template <int L, typename T>
__device__ __forceinline__ void finish(const RouteArgs& a, int64_t t, bool mine, int j, int id, float m, float sum) {
  const bool has = mine && id >= 0 && id < a.E;
  const float x = has ? fminf((float)static_cast<const T*>(a.logits)[t * a.E + id], kBig) : -INFINITY;
  finish_with<L>(a, t, mine, j, id, x, m, sum);
}

// Where a token's experts lie when L lanes hold it, V a lane.  One group: runs
// of a 16-byte load per lane, interleaved.  More: a group is `lpg` lanes; a whole
// wave's lanes interleave such runs over their group, fewer lanes have `per`
// experts in a row (places then differ by the same everywhere).  `whole`: every
// such load is inside its lane's part or outside it altogether; `full`: all are
// inside.
struct Layout {
  int32_t lpg, per;
  bool whole, full;
};

template <typename T, int L, int V, bool GROUPED>
struct Lanes {
  static constexpr int W = 16 / (int)sizeof(T), kWords = 4;
  static constexpr bool kSpread = GROUPED && L == kWave;
  typedef T vec __attribute__((ext_vector_type(W)));
  typedef __attribute__((aligned(sizeof(T)))) vec at;
  typedef uint32_t words __attribute__((ext_vector_type(kWords)));
  int32_t E, first, mine, sl, step;
  int g;
  bool whole, full;
  __device__ __forceinline__ Lanes(const RouteArgs& a, const Layout& lay)
      : E(a.E), whole(lay.whole), full(lay.full) {
    sl = (threadIdx.x & (kWave - 1)) % L;
    const int32_t gs = GROUPED ? E / a.groups : E;
    g = GROUPED ? sl / lay.lpg : 0;
    const bool in = !GROUPED || g < a.groups;
    step = lay.lpg * W;
    first = GROUPED ? (in ? g * gs + (sl % lay.lpg) * (kSpread ? W : lay.per) : 0) : sl * W;
    // experts of its run, or from its first one to its group's end
    mine = kSpread ? (in ? gs - (sl % lay.lpg) * W : 0)
                   : GROUPED ? (in ? min(lay.per, gs - (sl % lay.lpg) * lay.per) : 0) : E;
  }
  // Expert of place v, if the lane has it: its first one and a distance that all lanes share.
  static constexpr int away(int v) { return GROUPED ? v : (v / W) * L * W + v % W; }
  __device__ __forceinline__ int32_t index(int v) const { return first + (kSpread ? (v / W) * step + v % W : away(v)); }
  // Experts from place v0 on (a multiple of W) in its run: less than W at the end, 0 or less behind it.
  __device__ __forceinline__ int32_t left(int v0) const {
    return kSpread ? mine - (v0 / W) * step : GROUPED ? mine - v0 : E - index(v0);
  }

  // The row's logits by place, -infinity where the lane has none.
  __device__ __forceinline__ void load(const T* row, vec* d) const {
    constexpr bool k32 = sizeof(T) == 4;
    constexpr uint32_t kLow = k32 ? 0xFF800000u : std::is_same<T, __bf16>::value ? 0xFF80FF80u : 0xFC00FC00u;
    if (E < W) {  // no load of 16 bytes fits
      typedef typename std::conditional<k32, uint32_t, uint16_t>::type raw;
      const raw* p = reinterpret_cast<const raw*>(row);
#pragma unroll
      for (int v0 = 0; v0 < V; v0 += W) {
        words r = kLow;
#pragma unroll
        for (int u = 0; u < W; ++u) {
          if (u >= left(v0)) continue;
          const uint32_t x = p[index(v0 + u)];
          if (k32) r[u % kWords] = x;
          else r[u / 2] = u % 2 ? (r[u / 2] & 0xFFFFu) | x << 16 : (r[u / 2] & 0xFFFF0000u) | x;
        }
        d[v0 / W] = __builtin_bit_cast(vec, r);
      }
      return;
    }
#pragma unroll
    for (int v0 = 0; v0 < V; v0 += W) d[v0 / W] = *reinterpret_cast<const at*>(row + max(0, min(index(v0), E - W)));
    if (full) return;
    if (whole) {
#pragma unroll
      for (int v0 = 0; v0 < V; v0 += W) {
        const bool in = left(v0) > 0;
        words r = __builtin_bit_cast(words, d[v0 / W]);
#pragma unroll
        for (int u = 0; u < kWords; ++u) r[u] = in ? r[u] : kLow;
        d[v0 / W] = __builtin_bit_cast(vec, r);
      }
      return;
    }
#pragma unroll
    for (int v0 = 0; v0 < V; v0 += W) {
      const int32_t n = left(v0);
      words r = __builtin_bit_cast(words, d[v0 / W]);
      const int32_t off = index(v0) - min(index(v0), E - W);  // the load was moved back by this
      constexpr int kPer = k32 ? 1 : 2;                       // values of a word
#pragma unroll
      for (int s = W / 2; s >= kPer; s /= 2)
#pragma unroll
        for (int u = 0; u < kWords; ++u) r[u] = off & s ? (u + s / kPer < kWords ? r[u + s / kPer] : 0u) : r[u];
      if (!k32) {
#pragma unroll
        for (int u = 0; u < kWords; ++u)
          r[u] = off & 1 ? (r[u] >> 16) | (u + 1 < kWords ? r[u + 1] << 16 : 0u) : r[u];
      }
#pragma unroll
      for (int u = 0; u < kWords; ++u) {
        const uint32_t keep = n >= (u + 1) * kPer ? ~0u : !k32 && n == 2 * u + 1 ? 0xFFFFu : 0u;
        r[u] = (r[u] & keep) | (kLow & ~keep);
      }
      d[v0 / W] = __builtin_bit_cast(vec, r);
    }
  }
};

// Rank of a lane's group by an ordered value.
__device__ __forceinline__ int group_rank(const RouteArgs& a, int value, int g, int base, int32_t lpg) {
  int rank = 0;
  for (int o = 0; o < a.groups; ++o) {
    const int other = __shfl(value, base + o * lpg, kWave);
    rank += other > value || (other == value && o < g) ? 1 : 0;
  }
  return rank;
}

// The two largest of a group's lanes, from the two largest (b1 >= b2) of each.
template <typename V>
__device__ __forceinline__ void join_two(V& b1, V& b2, int32_t lpg) {
  auto join = [&](V o1, V o2) {
    b2 = max(min(b1, o1), max(b2, o2));
    b1 = max(b1, o1);
  };
  if (lpg >= 2) join(lane_step<0>(b1), lane_step<0>(b2));
  if (lpg >= 4) join(lane_step<1>(b1), lane_step<1>(b2));
  if (lpg >= 8) join(lane_step<2>(b1), lane_step<2>(b2));
  if (lpg >= 16) join(lane_step<3>(b1), lane_step<3>(b2));
  if (lpg >= 32) join(__shfl_xor(b1, 16, kWave), __shfl_xor(b2, 16, kWave));
}

// Tokens by keys of 32 bits, rounded as the formulas say: a round takes the
// maximum over the registers and removes it.  Any number of choices; bound by
// k passes over the registers (65536 x 256 bfloat16, 12 choices: 43 us for 40 MB,
// 1600 vector instructions a wave that issue all the time).
template <typename T, int L, int V, bool GROUPED>
__device__ __forceinline__ void route_exact(const RouteArgs& a, int64_t t, const Layout& lay) {
  const Lanes<T, L, V, GROUPED> at(a, lay);
  constexpr int W = Lanes<T, L, V, GROUPED>::W;
  const int lane = threadIdx.x & (kWave - 1), sl = lane % L, base = lane - sl;
  const bool live = t < a.T;
  typename Lanes<T, L, V, GROUPED>::vec d[V / W];
  at.load(static_cast<const T*>(a.logits) + (live ? t : a.T - 1) * a.E, d);
  auto logit = [&](int v) {
    const float x = (float)d[v / W][v % W];
    return x > -INFINITY ? fminf(x, kBig) : -INFINITY;
  };
  const bool sigm = a.flags & TAOT_ROUTE_SIGMOID;
  float m = 0.f, sum = 1.f;
  if (needs_sum(a)) {
    m = logit(0);
#pragma unroll
    for (int v = 1; v < V; ++v) m = fmaxf(m, logit(v));
    m = block_reduce<L>(m, MaxOp());
    const float base_m = m > -INFINITY ? m : 0.f;
    sum = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v) sum += expf(logit(v) - base_m);
    sum = block_reduce<L>(sum, SumOp());
  }
  int key[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const float x = logit(v);
    key[v] = key_of(x);
    if (a.bias) {
      const float s = sigm ? sigmoid(x) : expf(x - m) / sum;
      if (key[v] != kNone) key[v] = key_of(s + a.bias[at.index(v)]);
    }
  }

  if constexpr (GROUPED) {
    int b1 = kNone, b2 = kNone;  // the two best of the lane, then of the group
#pragma unroll
    for (int v = 0; v < V; ++v) {
      b2 = max(b2, min(b1, key[v]));
      b1 = max(b1, key[v]);
    }
    join_two(b1, b2, lay.lpg);
    if (group_rank(a, group_value(a, b1, b2, m), at.g, base, lay.lpg) >= a.top_groups) {
#pragma unroll
      for (int v = 0; v < V; ++v) key[v] = kNone;
    }
  }

  int id = -1;
  for (int j = 0; j < a.k; ++j) {
    int best = key[0];
#pragma unroll
    for (int v = 1; v < V; ++v) best = max(best, key[v]);
    const int top = block_reduce<L>(best, MaxOp());
    int e = INT32_MAX;  // the lane's first expert of that key
#pragma unroll
    for (int v = V - 1; v >= 0; --v) e = key[v] == top ? at.index(v) : e;
    const int win = block_reduce<L>(e, MinOp());
#pragma unroll
    for (int v = 0; v < V; ++v) key[v] = at.index(v) == win ? kNone : key[v];
    if (sl == j) id = top == kNone ? -1 : win;
  }
  finish<L, T>(a, t, live && sl < a.k, sl, id, m, sum);
}

template <typename T, int L, int V, bool GROUPED>
__global__ void __launch_bounds__(256)
route_kernel(RouteArgs a, Layout lay) {
  route_exact<T, L, V, GROUPED>(a, ((int64_t)blockIdx.x * 256 + threadIdx.x) / L, lay);
}

// A token by a block of 256 threads, any number of experts: the keys of
// route_exact in LDS.  Bound by its passes over the row and its barriers, one a
// round (8192 x 4096 bfloat16, softmax and bias, 8 choices: 131 us; without the bias
// route_wide_kernel takes 18).
template <typename T>
__device__ void route_block(const RouteArgs& a, int64_t t, int* keys) {
  __shared__ int value[TAOT_MAX_ROUTE_GROUPS];
  __shared__ int found[2][2][4];
  __shared__ float part[2][4];
  __shared__ int chosen[kWave];
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wid = tid / kWave;
  const T* row = static_cast<const T*>(a.logits) + t * a.E;
  auto logit = [&](int e) {
    const float x = (float)row[e];
    return x > -INFINITY ? fminf(x, kBig) : -INFINITY;
  };
  const bool sigm = a.flags & TAOT_ROUTE_SIGMOID;
  float m = 0.f, sum = 1.f;
  if (needs_sum(a)) {
    m = -INFINITY;
    for (int e = tid; e < a.E; e += 256) m = fmaxf(m, logit(e));
    m = block_reduce<kWave>(m, MaxOp());
    if (lane == 0) part[0][wid] = m;
    __syncthreads();
    m = fmaxf(fmaxf(part[0][0], part[0][1]), fmaxf(part[0][2], part[0][3]));
    const float base_m = m > -INFINITY ? m : 0.f;
    sum = 0.f;
    for (int e = tid; e < a.E; e += 256) sum += expf(logit(e) - base_m);
    sum = block_reduce<kWave>(sum, SumOp());
    if (lane == 0) part[1][wid] = sum;
    __syncthreads();
    sum = part[1][0] + part[1][1] + part[1][2] + part[1][3];
  }
#pragma unroll 4
  for (int e = tid; e < a.E; e += 256) {
    const float x = logit(e);
    if (!a.bias) keys[e] = key_of(x);
    else keys[e] = x > -INFINITY ? key_of((sigm ? sigmoid(x) : expf(x - m) / sum) + a.bias[e]) : kNone;
  }
  __syncthreads();
  if (a.groups > 1) {
    const int32_t gs = a.E / a.groups;
    for (int g = wid; g < a.groups; g += 4) {
      int b1 = kNone, b2 = kNone;
      for (int i = lane; i < gs; i += kWave) {
        const int x = keys[g * gs + i];
        b2 = max(b2, min(b1, x));
        b1 = max(b1, x);
      }
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) {
        const int o1 = __shfl_xor(b1, o, kWave), o2 = __shfl_xor(b2, o, kWave);
        b2 = max(min(b1, o1), max(b2, o2));
        b1 = max(b1, o1);
      }
      if (lane == 0) value[g] = group_value(a, b1, b2, m);
    }
    __syncthreads();
    for (int g = wid; g < a.groups; g += 4) {
      int rank = 0;
      for (int o = 0; o < a.groups; ++o) rank += value[o] > value[g] || (value[o] == value[g] && o < g) ? 1 : 0;
      if (rank >= a.top_groups)
        for (int i = lane; i < gs; i += kWave) keys[g * gs + i] = kNone;
    }
    __syncthreads();
  }
  // each thread's best key; after a round only the winner's thread looks again
  int best, at;
  auto look = [&] {
    best = kNone;
    at = INT32_MAX;
#pragma unroll 4
    for (int e = tid; e < a.E; e += 256) {
      const int x = keys[e];
      at = x > best ? e : at;
      best = max(best, x);
    }
  };
  look();
  for (int j = 0; j < a.k; ++j) {
    const int most = block_reduce<kWave>(best, MaxOp()), first = block_reduce<kWave>(best == most ? at : INT32_MAX, MinOp());
    int(*turn)[4] = found[j & 1];  // two sets of words take turns: one barrier a round
    if (lane == 0) {
      turn[0][wid] = most;
      turn[1][wid] = first;
    }
    __syncthreads();
    int top = turn[0][0], win = turn[1][0];
#pragma unroll
    for (int w = 1; w < 4; ++w) {
      const int x = turn[0][w], e = turn[1][w];
      win = x > top ? e : x == top ? min(win, e) : win;
      top = max(top, x);
    }
    if (tid == 0) chosen[j] = top == kNone ? -1 : win;
    if (top != kNone && tid == win % 256) {
      keys[win] = kNone;
      look();
    }
  }
  __syncthreads();
  if (wid == 0) finish<kWave, T>(a, t, lane < a.k, lane, lane < a.k ? chosen[lane] : -1, m, sum);
}

template <typename T>
__global__ void __launch_bounds__(256)
route_block_kernel(RouteArgs a) {
  extern __shared__ __attribute__((aligned(16))) int keys[];
  route_block<T>(a, blockIdx.x, keys);
}

// ---- up to eight choices -----------------------------------------------------------
// Key and expert share one word, the key above, the expert's complement below:
// words differ, and a larger word is the better choice.  A lane keeps its DEPTH
// largest words in order, one median per place and expert; a round is then a
// maximum over the lanes' first words, and the lane that had it moves up.
//
// kExact16  16-bit logits without a bias: the logit itself is the key.
// kLogit    32-bit logits without a bias: the distance to the row's maximum in
//           fixed point.  It does not rise as the logit falls, so different keys
//           are in the logits' order; equal ones are undecided.
// kSigmoid  sigmoid plus bias, from the hardware's exponential and reciprocal,
//           in fixed point: keys nearer than their error are undecided.
// A token whose first k + 1 words or whose groups are undecided, one with a lane
// that ran out of words, and one with keys that the fixed point does not hold
// (0: masked, or too low) is done again by exact keys, with the whole wave.
// Bound by the eight medians of every expert: 65536 x 256 float32, bias, 8 groups:
// 30 us (71 MB, 2.4 TB/s; 1056 vector instructions a wave, 15 us of issue); 65536 x
// 256 bfloat16: 13 us (806 and 11).  Equal float32 logits among a token's first k + 1
// are undecided too: rounded to bfloat16 first, 65536 x 256 take 66 us, 20 else.
constexpr int kExact16 = 0, kLogit = 1, kSigmoid = 2;
constexpr float kLogitRange = 32.f;

__device__ __forceinline__ int median(int a, int b, int c) {
  int r;
  asm("v_med3_i32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

// Its error at -d is at most 0.8 d + 2 units of 2^-24 (the product's rounding, the constant's, the instruction's).
// Good enough for keys that are looked at again where it could decide, and for the sum of a softmax: mass at a distance
// d takes e^d experts, so that of 4096 the sum is off by 9 units at most, 1 for normally distributed logits, where
// its own 70 additions are worth as much.  With the remainder (exp_near): 8192 x 4096 bfloat16 19.6 us instead of 17.4,
// 65536 x 256 14.2 instead of 12.8.
__device__ __forceinline__ float exp_fast(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504f); }

// The same for x <= 0 with what the product rounds away: within 1.5 units in the last place (the fast one's error grows
// with the distance from 0: 31 units of 2^-24 at -40), 0 below the smallest normal number.  -infinity gives 0, NaN too.
__device__ __forceinline__ float exp_near(float x) {
  const float c = fmaxf(x, -128.f), t = c * 1.44269504f, e = __builtin_amdgcn_exp2f(t);
  const float d = fmaf(t, 1.90465429e-9f, fmaf(t, -0.693147182f, c));  // c - t ln 2, ln 2 in two parts
  return fmaf(e, d, e);
}

constexpr int log2_of(int n) { return n <= 1 ? 0 : 1 + log2_of(n / 2); }

template <typename T, int L, int V, int MODE, bool GROUPED>
__global__ void __launch_bounds__(256, sizeof(T) == 4 || MODE == kSigmoid ? 4 : 5)
route_few_kernel(RouteArgs a, Layout lay) {
  using Place = Lanes<T, L, V, GROUPED>;
  constexpr int DEPTH = 8;
  static_assert(L < kWave && V >= DEPTH, "a lane's list holds every choice");
  constexpr int W = Place::W;
  constexpr int kInf16 = std::is_same<T, __bf16>::value ? 0x7F80 : 0x7C00;
  constexpr int kShift = MODE == kExact16 ? 16 : log2_of(L * V), kLow = (1 << kShift) - 1;
  constexpr float kMost = (float)((1 << (31 - kShift < 24 ? 31 - kShift : 24)) - 1);  // largest key in fixed point
  constexpr int kRanOut = INT32_MIN + 1;  // behind a lane's last word
  auto low = [](int v) { return (uint32_t)(kLow - Place::away(v)); };
  const int lane = threadIdx.x & (kWave - 1), sl = lane % L, base = lane - sl;
  const int64_t t = ((int64_t)blockIdx.x * 256 + threadIdx.x) / L;
  const bool live = t < a.T;
  const Place at(a, lay);
  typename Place::vec d[V / W];
  at.load(static_cast<const T*>(a.logits) + (live ? t : a.T - 1) * a.E, d);
  auto logit = [&](int v) { return (float)d[v / W][v % W]; };
  bool open = false;  // this lane has seen something undecided

  float m = 0.f, sum = 1.f;
  const bool plain = !(a.flags & (TAOT_ROUTE_SIGMOID | TAOT_ROUTE_RENORM));
  const bool two = GROUPED && (a.flags & TAOT_ROUTE_GROUP_TWO);
  if (MODE == kLogit || (MODE == kExact16 && (plain || (two && !(a.flags & TAOT_ROUTE_SIGMOID))))) {
    m = logit(0);
#pragma unroll
    for (int v = 1; v < V; ++v) m = fmaxf(m, logit(v));
    m = block_reduce<L>(m, MaxOp());
    open |= m == INFINITY;
    m = m > -INFINITY ? m : 0.f;
    if (plain) {
      sum = 0.f;
#pragma unroll
      for (int v = 0; v < V; ++v) sum += exp_fast(logit(v) - m);
      sum = block_reduce<L>(sum, SumOp());
      open |= sum != sum;
    }
  }

  // by two without a bias: the lane's best logits themselves, so that the sums of scores decide as exact keys' would
  float x1 = -INFINITY, x2 = -INFINITY;
  if (MODE == kLogit && two) {
    float all = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const float x = logit(v);
      x2 = __builtin_amdgcn_fmed3f(x1, x2, x);
      x1 = fmaxf(x1, x);
      all += x;
    }
    open |= all != all;  // NaN: the second largest is not to be relied on
  }

  int best[DEPTH];
#pragma unroll
  for (int i = 0; i < DEPTH; ++i) best[i] = INT32_MIN;
  auto insert = [&](int word) {
#pragma unroll
    for (int i = DEPTH - 1; i > 0; --i) best[i] = median(best[i - 1], best[i], word);
    best[0] = max(best[0], word);
  };
  int apart = 1;      // keys that differ by this are decided
  int apart_two = 1;  // groups
  if constexpr (MODE == kExact16) {
    typedef short pair __attribute__((ext_vector_type(2)));
    pair big = 0;
#pragma unroll
    for (int v = 0; v < V; v += 2) {
      const typename Place::words r = __builtin_bit_cast(typename Place::words, d[v / W]);
      const uint32_t word = r[v % W / 2];
      const pair x = __builtin_bit_cast(pair, word);
      const pair size = x & (short)0x7fff, sign = x >> (short)15;
      big = __builtin_elementwise_max(big, size);
      const uint32_t o = __builtin_bit_cast(uint32_t, (pair)((size ^ sign) - sign));
      insert((int)((o << 16) | low(v)));
      insert((int)((o & 0xFFFF0000u) | low(v + 1)));
    }
    open |= max((int)big[0], (int)big[1]) > kInf16;  // NaN
  } else if constexpr (MODE == kLogit) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const uint32_t q = (uint32_t)fmaf(logit(v) - m, kMost / kLogitRange, kMost);  // negative and NaN: 0
      insert((int)((q << kShift) | low(v)));
    }
    apart_two = 8;  // each key is cut by less than one unit
  } else {
    // fixed point over the range of the keys, by the largest bias of all experts (infinite or NaN: exact keys)
    float most = 0.f, least = INFINITY;
    float bias[V];
    if (at.whole) {
      typedef float four __attribute__((ext_vector_type(4)));
      typedef __attribute__((aligned(4))) four at4;
#pragma unroll
      for (int v = 0; v < V; v += 4) {
        const four b = *reinterpret_cast<const at4*>(a.bias + max(0, min(at.index(v), a.E - 4)));
#pragma unroll
        for (int u = 0; u < 4; ++u) bias[v + u] = b[u];
      }
    } else {
#pragma unroll
      for (int v = 0; v < V; ++v) bias[v] = a.bias[min(at.index(v), a.E - 1)];
    }
#pragma unroll
    for (int v = 0; v < V; ++v) most = fmaxf(most, fabsf(bias[v]));
    most = block_reduce<L>(most, MaxOp());
    const float unit = (kMost - 16.f) / (1.f + 2.f * most), zero = most * unit + 4.f;
#pragma unroll
    for (int v = 0; v < V; ++v) least = fminf(least, logit(v));
    auto fill = [&](auto masked) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const float x = logit(v), b = fmaf(bias[v], unit, zero);
        const uint32_t k = (uint32_t)fmaf(__builtin_amdgcn_rcpf(1.f + exp_fast(-x)), unit, b);  // NaN: 0
        const uint32_t q = !masked.value || x > -INFINITY ? k : 0u;
        insert((int)((q << kShift) | low(v)));
      }
    };
    if (__ballot(least == -INFINITY) != 0) fill(std::true_type());
    else fill(std::false_type());
    // The sigmoid's product, exponential, sum and reciprocal stay within 8 units of 2^-24, the exact key within 4
    // of the formula's value and 1 + |bias| of it for the sum; the fixed point adds less than 4 of its units.
    const float slack = 14.f * 0x1p-24f * (1.f + most) * unit;
    open |= !(slack < 1e6f && most < 1e30f);
    apart = 8 + (int)(2.f * fminf(slack, 1e6f));
    apart_two = 2 * apart;
  }
#pragma unroll
  for (int i = 0; i < DEPTH; ++i) best[i] -= at.first;  // the place's complement becomes the expert's

  if constexpr (GROUPED) {
    const bool in = at.g < a.groups;
    bool stays;
    if (MODE == kLogit && two) {
      join_two(x1, x2, lay.lpg);
      stays = in && group_rank(a, two_scores(a, x1, x2, m), at.g, base, lay.lpg) < a.top_groups;
    } else {
      int b1 = best[0] >> kShift, b2 = best[1] >> kShift, value;
      join_two(b1, b2, lay.lpg);
      if constexpr (MODE == kExact16) {
        auto float_of = [&](int o) {
          return o > -kInf16 ? fminf((float)__builtin_bit_cast(T, (short)(o < 0 ? 0x8000 | -o : o)), kBig) : -INFINITY;
        };
        const float x = float_of(b1);
        value = two ? two_scores(a, x, float_of(b2), m) : key_of(x);
      } else {
        value = b1 + (two ? b2 : 0);
        open |= in && (b1 <= 0 || (two && b2 <= 0));
      }
      stays = in && group_rank(a, value, at.g, base, lay.lpg) < a.top_groups;
      if constexpr (MODE != kExact16) {
        const int last = -block_reduce<L>(stays ? -value : INT32_MIN, MaxOp());
        const int next = block_reduce<L>(!stays && in ? value : 0, MaxOp());
        open |= next > 0 && last - next < apart_two;
      }
    }
#pragma unroll
    for (int i = 0; i < DEPTH; ++i) best[i] = stays ? best[i] : INT32_MIN;
  }

  int mine = 0, top = 0;
  const int rounds = MODE == kExact16 ? a.k : a.k + 1;
  for (int j = 0; j < rounds; ++j) {
    open |= best[0] == kRanOut;
    top = block_reduce<L>(best[0], MaxOp());
    const bool won = best[0] == top && top > kRanOut;
#pragma unroll
    for (int i = 0; i + 1 < DEPTH; ++i) best[i] = won ? best[i + 1] : best[i];
    best[DEPTH - 1] = won ? kRanOut : best[DEPTH - 1];
    mine = sl == j ? top : mine;
  }
  const bool chooses = live && sl < a.k;
  int id = kLow - (mine & kLow);
  if constexpr (MODE == kExact16) {
    id = mine >> kShift > -kInf16 ? id : -1;
  } else {
    const int up = __builtin_amdgcn_mov_dpp(mine, 0x101, 0xF, 0xF, true);  // of the lane above
    const int key = mine >> kShift, after = max(0, (sl + 1 < a.k ? up : top) >> kShift);
    open |= sl < a.k && (key <= 0 || key - after < apart);
  }
  uint64_t again = __ballot(open && live);
  // a token is done again if one of its lanes says so
  const uint64_t seg = ((1ull << L) - 1) << base;
  const bool redo = (again & seg) != 0;
  finish<L, T>(a, t, chooses && !redo, sl, id, m, sum);
  Layout wide = lay;  // the same experts over 64 lanes
  if constexpr (GROUPED) {
    wide.lpg = lay.lpg * (kWave / L);
    wide.whole = false;
  }
  wide.full = false;
  while (again != 0) {
    const int s = __ffsll((unsigned long long)again) - 1;
    again &= ~(((1ull << L) - 1) << (s / L * L));
    route_exact<T, kWave, 8, GROUPED>(a, ((int64_t)blockIdx.x * 256 + (threadIdx.x & ~(kWave - 1)) + s) / L, wide);
  }
}

// ---- wide rows, up to sixteen choices ------------------------------------------------
// A wave per token, 64 lanes with V experts each.  The k-th largest of the lanes'
// own maxima is a bound that the k best reach: few others do.  Those that reach it go to LDS, one a lane,
// where exact keys are compared with one another: one comparison an expert, where
// lists would take a median for each of their places.  Without a bias the logits
// themselves are the keys; with one, keys from the hardware's exponential and
// reciprocal set the bound, lowered by twice their error.  A token with groups
// nearer than that error, with infinite or NaN values, or with more than 64
// experts that reach the bound is done again by the block.
// 8192 x 4096 bfloat16, plain softmax: 18 us (68 MB, 3.8 TB/s; 22 with a lane's
// four largest in a list), bound by the softmax's sum (15 us without it); float32:
// 25 us (134 MB, 5.4 TB/s); sigmoid and bias, bfloat16: 35 us, bound by the sigmoid.
constexpr int kWideMost = 16;

template <typename T, int V, bool BIAS, bool GROUPED>
__global__ void __launch_bounds__(256, sizeof(T) == 4 && BIAS ? 2 : sizeof(T) == 4 || BIAS ? 3 : 6)
route_wide_kernel(RouteArgs a, Layout lay) {
  using Place = Lanes<T, kWave, V, GROUPED>;
  constexpr int W = Place::W;
  extern __shared__ __attribute__((aligned(16))) int keys[];  // the wide rows' biases are read 16 bytes at a time
  __shared__ int2 found[4][kWave + 1];  // an expert and its logit; behind the 64th all in one place
  __shared__ int32_t undecided[4];
  __shared__ float part[4];
  const int lane = threadIdx.x & (kWave - 1), wid = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int64_t t = (int64_t)blockIdx.x * 4 + wid;
  const bool live = t < a.T;
  const T* row = static_cast<const T*>(a.logits) + (live ? t : a.T - 1) * a.E;
  const Place at(a, lay);
  typename Place::vec d[V / W];
  at.load(row, d);
  auto logit = [&](int v) { return (float)d[v / W][v % W]; };
  // From here on the logits are widened anew: V of them would take more registers than leave room for enough waves.
  auto narrow = [&] {
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int v = 0; v < V; v += W) {
        typename Place::words r = __builtin_bit_cast(typename Place::words, d[v / W]);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          uint32_t w = r[u];
          asm("" : "+v"(w));
          r[u] = w;
        }
        d[v / W] = __builtin_bit_cast(typename Place::vec, r);
      }
    }
  };
  bool open = false;

  // the lane's largest key, and the second where groups need it
  float b1 = -INFINITY, b2 = -INFINITY, m = 0.f, sum = 1.f, slack = 0.f;
  float key[BIAS ? V : 1];
  if constexpr (!BIAS) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if (GROUPED) b2 = __builtin_amdgcn_fmed3f(b1, b2, logit(v));
      b1 = fmaxf(b1, logit(v));
      // keeps the compiler from widening all V first, which spills
      if (GROUPED && v % W == W - 1) asm volatile("" : "+v"(b1), "+v"(b2));
    }
    m = block_reduce<kWave>(b1, MaxOp());
    open |= m == INFINITY;
    m = m > -INFINITY ? m : 0.f;
    narrow();
    if (!(a.flags & (TAOT_ROUTE_SIGMOID | TAOT_ROUTE_RENORM))) {
      sum = 0.f;
#pragma unroll
      for (int v = 0; v < V; ++v) sum += exp_fast(logit(v) - m);
      sum = block_reduce<kWave>(sum, SumOp());
      open |= sum != sum;
    } else if (GROUPED) {  // NaN: the second largest is not to be relied on
      float all = 0.f;
#pragma unroll
      for (int v = 0; v < V; ++v) all += logit(v);
      open |= all != all;
    }
  } else {
    float most = 0.f, least = INFINITY;
    float* bias = reinterpret_cast<float*>(keys);  // the biases in LDS: by the block once, not by each wave
    for (int e = threadIdx.x; e < a.E; e += 256) {
      bias[e] = a.bias[e];
      most = fmaxf(most, fabsf(bias[e]));
    }
    most = block_reduce<kWave>(most, MaxOp());
    if (lane == 0) part[wid] = most;
    __syncthreads();
    most = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
    open |= !(most < 1e30f);
    // The sigmoid's product, exponential, sum and reciprocal stay within 8 units of 2^-24, the exact key within 4
    // of the formula's value, and each sum's rounding within 1 + |bias| of them.
    slack = 16.f * 0x1p-24f * (1.f + most);
#pragma unroll
    for (int v = 0; v < V; ++v) least = fminf(least, logit(v));
    narrow();
    typedef float four __attribute__((ext_vector_type(4)));
    auto fill = [&](auto masked, auto whole) {
#pragma unroll
      for (int v0 = 0; v0 < V; v0 += 4) {
        four b;
        if constexpr (whole.value) {
          b = *reinterpret_cast<const four*>(bias + max(0, min(at.index(v0), a.E - 4)));
        } else {
#pragma unroll
          for (int u = 0; u < 4; ++u) b[u] = bias[min(at.index(v0 + u), a.E - 1)];
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const float x = logit(v0 + u), y = __builtin_amdgcn_rcpf(1.f + exp_fast(-x)) + b[u];
          key[v0 + u] = !masked.value || x > -INFINITY ? y : -INFINITY;
        }
        if (v0 % 8 == 4) asm volatile("" : "+v"(key[v0]), "+v"(key[v0 + 1]), "+v"(key[v0 + 2]), "+v"(key[v0 + 3]));
      }
    };
    const bool masked = __ballot(least == -INFINITY) != 0;
    if (!at.whole) fill(std::true_type(), std::false_type());
    else if (masked) fill(std::true_type(), std::true_type());
    else fill(std::false_type(), std::true_type());
    float all = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if (GROUPED) {
        b2 = __builtin_amdgcn_fmed3f(b1, b2, key[v]);
        all += key[v];
      }
      b1 = fmaxf(b1, key[v]);
    }
    open |= all != all;
  }
  auto value_of = [&](int v) {
    if constexpr (BIAS) return key[v];
    else return logit(v);
  };

  bool stays = true;
  if constexpr (GROUPED) {
    float g1 = b1, g2 = b2;
    join_two(g1, g2, lay.lpg);
    const bool two = a.flags & TAOT_ROUTE_GROUP_TWO, in = at.g < a.groups;
    const float value = two && g2 > -INFINITY ? g1 + g2 : g1;
    const int rank_by = !BIAS && two ? two_scores(a, g1, g2, m) : g1 > -INFINITY ? ordered(value) : kNone;
    stays = in && group_rank(a, rank_by, at.g, 0, lay.lpg) < a.top_groups;
    if constexpr (BIAS) {
      const float last = -block_reduce<kWave>(stays ? -value : -INFINITY, MaxOp());
      const float next = block_reduce<kWave>(!stays && in ? value : -INFINITY, MaxOp());
      open |= next > -INFINITY && !(last - next > 4.f * slack);
    }
  }

  // the largest number that k lanes' maxima reach, of a float's upper bits in order: all of bfloat16's; else 26, so
  // that keys close to one another (sigmoids near 1, logits far from 0) do not all reach it
  constexpr int kLastBit = std::is_same<T, __bf16>::value && !BIAS ? 16 : 6;
  const uint32_t mine = (uint32_t)key_of(stays ? b1 : -INFINITY) ^ 0x80000000u;
  uint32_t bound = 0;
#pragma unroll
  for (int bit = 31; bit >= kLastBit; --bit) {
    const uint32_t trial = bound | 1u << bit;
    bound = __popcll(__ballot(mine >= trial)) >= a.k ? trial : bound;
  }
  const float reach = unordered(max((int)(bound ^ 0x80000000u), ordered(-kBig))) - 2.f * slack;
  const float limit = stays ? reach : INFINITY;

  if constexpr (!BIAS) narrow();
  int n = 0;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const float x = value_of(v);
    const bool in = x >= limit;
    const uint64_t who = __ballot(in);
    if (who == 0) continue;
    const int below = __builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0));
    if (in) found[wid][min(n + below, kWave)] = int2{at.index(v), __float_as_int(x)};
    n += __popcll(who);
  }
  open |= n > kWave;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();

  const int count = min(n, kWave);
  int2 f = found[wid][lane];
  bool has = lane < count;
  const int e = has ? f.x : 0;
  float x = __int_as_float(f.y);
  if constexpr (BIAS) x = (float)row[e];
  x = fminf(x, kBig);
  int exact = key_of(x);
  if constexpr (BIAS) exact = key_of(sigmoid(x) + a.bias[e]);
  exact = has ? exact : kNone;
  has = exact != kNone;
  int rank = 0;
  for (int c = 0; c < count; ++c) {
    const int other = lane_value(exact, c), oe = lane_value(e, c);
    rank += other > exact || (other == exact && oe < e) ? 1 : 0;
  }
  __builtin_amdgcn_wave_barrier();
  if (has && rank < a.k) found[wid][rank] = int2{e, __float_as_int(x)};
  const int chosen = min((int)__popcll(__ballot(has)), a.k);
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  f = found[wid][lane];
  const bool redo = __ballot(open && live) != 0;
  finish_with<kWave>(a, t, live && lane < a.k && !redo, lane, lane < chosen ? f.x : -1,
                     lane < chosen ? __int_as_float(f.y) : -INFINITY, m, sum);
  if (lane == 0) undecided[wid] = redo;
  __syncthreads();
  for (int w = 0; w < 4; ++w)
    if (undecided[w]) route_block<T>(a, (int64_t)blockIdx.x * 4 + w, keys);
}

// ---- gradient ------------------------------------------------------------------
// A wave per token.  CPL chunks of eight experts a lane hold the row in
// registers; CPL = 0: any number of experts, the row is read three times.  The k
// chosen experts' gradients go to the wave's row of LDS (zero elsewhere), which is
// read back as the row to write, or, where that row would leave room for few
// waves, to their places in registers one after the other (4096 x 4096: 23 us, 29
// by LDS; 32768 x 384: 26 us, 17 by LDS).  The plain softmax adds
// -p_e sum_j dw_j w_j to every expert.  dlogits may lie in the logits' memory: the
// chosen experts' are read before the wave writes, the others by the lane that
// writes them, before it does.
template <typename T, int CPL>
__global__ void __launch_bounds__(256)
route_backward_kernel(const float* __restrict__ dweights, const T* logits, const int32_t* __restrict__ ids,
                      int64_t tokens, int32_t E, int32_t k, float scale, uint32_t flags, T* dlogits, int32_t pitch) {
  extern __shared__ float lds[];
  const int lane = threadIdx.x & (kWave - 1), wid = threadIdx.x / kWave;
  const int waves = blockDim.x / kWave;
  float* at = lds + (size_t)wid * pitch;
  if constexpr (CPL <= 2) {
    for (int e = lane; e < pitch; e += kWave) at[e] = 0.f;
  }
  // The fast exponential's error is less than a hundredth of what rounding to 16 bits costs, but not of 32.
  auto exponential = [](float x) { return sizeof(T) == 4 ? exp_near(x) : exp_fast(x); };
  const bool sigm = flags & TAOT_ROUTE_SIGMOID, renorm = flags & TAOT_ROUTE_RENORM, dense = !sigm && !renorm;
  for (int64_t t = (int64_t)blockIdx.x * waves + wid; t < tokens; t += (int64_t)gridDim.x * waves) {
    const T* row = logits + t * E;
    T* out = dlogits + t * E;
    auto chunk = [&](int e) {  // logits e .. e + 7, -inf where there is none
      const int n = E - e;
      f32x8 r = load_row(row + e, n);
#pragma unroll
      for (int u = 0; u < 8; ++u) r[u] = u < n && r[u] > -INFINITY ? fminf(r[u], kBig) : -INFINITY;
      return r;
    };
    f32x8 p[CPL > 0 ? CPL : 1];
    if (dense) {
#pragma unroll
      for (int i = 0; i < CPL; ++i) p[i] = chunk(8 * (i * kWave + lane));
    }
    int id = -1;
    float dw = 0.f, x = -INFINITY;
    if (lane < k) {
      id = ids[t * k + lane];
      dw = dweights[t * k + lane] * scale;
      x = id >= 0 && id < E ? (float)row[id] : -INFINITY;
      x = x > -INFINITY ? fminf(x, kBig) : -INFINITY;
      if (!(x > -INFINITY)) id = -1;
    }
    const bool has = id >= 0;
    dw = has ? dw : 0.f;
    float d = dw, m = 0.f, inv = 0.f, q = 0.f;
    if (sigm) {
      const float s = has ? sigmoid(x) : 0.f;
      if (renorm) {
        const float total = block_reduce<kWave>(s, SumOp()) + kTiny;
        dw = (dw - block_reduce<kWave>(dw * s, SumOp()) / total) / total;
      }
      d = dw * s * (1.f - s);
    } else if (renorm) {
      const float top = block_reduce<kWave>(x, MaxOp());
      float v = has ? expf(x - top) : 0.f;
      const float total = block_reduce<kWave>(v, SumOp());
      v = has ? v / total : 0.f;
      d = v * (dw - block_reduce<kWave>(dw * v, SumOp()));
    } else {
      float sum = 0.f;
      auto most = [&](const f32x8& r) {
#pragma unroll
        for (int u = 0; u < 8; ++u) m = fmaxf(m, r[u]);
      };
      auto add = [&](f32x8& r) {
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          r[u] = exponential(r[u] - m);
          sum += r[u];
        }
      };
      m = -INFINITY;
      if constexpr (CPL > 0) {
#pragma unroll
        for (int i = 0; i < CPL; ++i) most(p[i]);
      } else {
        for (int e = 8 * lane; e < E; e += 8 * kWave) most(chunk(e));
      }
      m = block_reduce<kWave>(m, MaxOp());
      m = m > -INFINITY ? m : 0.f;
      if constexpr (CPL > 0) {
#pragma unroll
        for (int i = 0; i < CPL; ++i) add(p[i]);
      } else {
        for (int e = 8 * lane; e < E; e += 8 * kWave) {
          f32x8 r = chunk(e);
          add(r);
        }
      }
      sum = block_reduce<kWave>(sum, SumOp());
      inv = sum > 0.f ? 1.f / sum : 0.f;
      q = block_reduce<kWave>(has ? dw * (exponential(x - m) * inv) : 0.f, SumOp());
    }
    if constexpr (CPL > 2) {
      f32x8 r[CPL];
#pragma unroll
      for (int i = 0; i < CPL; ++i) r[i] = 0.f;
      for (int j = 0; j < k; ++j) {  // the same expert for all lanes: one of them has it, at one place
        const int e = lane_value(id, j);
        const float v = lane_value(d, j);
        if (e < 0) continue;
#pragma unroll
        for (int i = 0; i < CPL; ++i) {
          if (e / (8 * kWave) != i) continue;
          const bool here = (e / 8) % kWave == lane;
#pragma unroll
          for (int u = 0; u < 8; ++u) r[i][u] = here && e % 8 == u ? v : r[i][u];
        }
      }
#pragma unroll
      for (int i = 0; i < CPL; ++i) {
        const int e = 8 * (i * kWave + lane);
        if (dense) {
#pragma unroll
          for (int u = 0; u < 8; ++u) r[i][u] = p[i][u] * inv * (r[i][u] - q);
        }
        store_row(out + e, r[i], E - e);
      }
    } else {
      if (has) at[id] = d;
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      auto write = [&](int e, const f32x8& p) {
        f32x8 r;
#pragma unroll
        for (int u = 0; u < 8; ++u) r[u] = at[e + u];
        if (dense) r = p * inv * (r - q);
        store_row(out + e, r, E - e);
      };
      if constexpr (CPL > 0) {
#pragma unroll
        for (int i = 0; i < CPL; ++i) {
          const int e = 8 * (i * kWave + lane);
          if (e < E) write(e, p[i]);
        }
      } else {
        for (int e = 8 * lane; e < E; e += 8 * kWave) {
          f32x8 z = 0.f;
          if (dense) {
            z = chunk(e);
#pragma unroll
            for (int u = 0; u < 8; ++u) z[u] = exponential(z[u] - m);
          }
          write(e, z);
        }
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      if (has) at[id] = 0.f;
    }
  }
}

template <typename T, int L, int V, bool GROUPED>
taot_status go(const RouteArgs& a, Layout lay, hipStream_t stream) {
  constexpr int kPlain = std::is_same<T, float>::value ? kLogit : kExact16;
  constexpr int W = 16 / (int)sizeof(T);
  const unsigned blocks = (unsigned)((a.T * L + 255) / 256);
  const size_t lds = (size_t)a.E * sizeof(int);
  const int32_t gs = a.E / a.groups;
  if (GROUPED && round_up(lay.per, W) <= V) lay.per = (int32_t)round_up(lay.per, W);
  lay.whole = !GROUPED ? a.E % W == 0 : gs % W == 0 && (L == kWave || lay.per % W == 0);
  lay.full = GROUPED ? a.groups * lay.lpg == L && (L == kWave || lay.per == V) && gs == lay.lpg * V : a.E == L * V;
  const bool sigm = a.flags & TAOT_ROUTE_SIGMOID;
  if constexpr (L == kWave) {
    if (a.k <= kWideMost && !a.bias) route_wide_kernel<T, V, false, GROUPED><<<blocks, 256, lds, stream>>>(a, lay);
    else if (a.k <= kWideMost && sigm) route_wide_kernel<T, V, true, GROUPED><<<blocks, 256, lds, stream>>>(a, lay);
    else if constexpr (V <= 16) route_kernel<T, L, V, GROUPED><<<blocks, 256, 0, stream>>>(a, lay);
  } else {
    // by route_of's rules eight lanes have few choices only, and 16 of 16 experts without groups many only
    constexpr bool kFew = L != 16 || V != 16 || GROUPED, kMany = L != 8;
    const bool plain = a.k <= 8 && !a.bias, sigmoids = a.k <= 8 && a.bias && sigm;
    if constexpr (kFew) {
      if (plain) route_few_kernel<T, L, V, kPlain, GROUPED><<<blocks, 256, 0, stream>>>(a, lay);
      else if (sigmoids) route_few_kernel<T, L, V, kSigmoid, GROUPED><<<blocks, 256, 0, stream>>>(a, lay);
    }
    if constexpr (kMany) {
      if (!kFew || !(plain || sigmoids)) route_kernel<T, L, V, GROUPED><<<blocks, 256, 0, stream>>>(a, lay);
    }
  }
  return hipGetLastError() == hipSuccess ? TAOT_OK : TAOT_ERR_LAUNCH;
}

template <typename T, int L, int V>
taot_status go(const RouteArgs& a, const Layout& lay, hipStream_t stream) {
  return a.groups > 1 ? go<T, L, V, true>(a, lay, stream) : go<T, L, V, false>(a, lay, stream);
}

template <typename T>
taot_status route_of(const RouteArgs& a, hipStream_t stream) {
  // lanes of a group, and experts of a lane, when L lanes hold a token
  auto layout = [&](int L) {
    Layout lay{1, 0, false, false};
    while (2 * lay.lpg * a.groups <= L) lay.lpg *= 2;
    lay.per = (a.E / a.groups + lay.lpg - 1) / lay.lpg;
    return lay;
  };
  // As few lanes a token as hold it: a round's reduction serves more tokens (65536 tokens, bfloat16, 8 choices; us by
  // 8, 16 and 64 lanes: 128 experts 9, 14 and 48; 256 experts 13, 14 and 46; 384 experts by 16 and 64: 21 and 46;
  // 16384 tokens of 1000 experts by 64 lanes and by a block: 15 and 78).
  const Layout by8 = layout(8), by16 = layout(16), by64 = layout(kWave);
  const bool known = !a.bias || (a.flags & TAOT_ROUTE_SIGMOID), few = a.k <= 8 && known;
  if (few && a.groups <= 8 && by8.per <= 16) return go<T, 8, 16>(a, by8, stream);
  if (few && a.groups <= 8 && by8.per <= 32) return go<T, 8, 32>(a, by8, stream);
  if (a.k <= 16 && a.groups <= 16 && by16.per <= 16) return go<T, 16, 16>(a, by16, stream);
  if (a.k <= 16 && a.groups <= 16 && by16.per <= 32) return go<T, 16, 32>(a, by16, stream);
  if (a.groups <= kWave && by64.per <= 16) return go<T, 64, 16>(a, by64, stream);
  if (a.k <= kWideMost && known && a.groups <= kWave && by64.per <= 64) return go<T, 64, 64>(a, by64, stream);
  const size_t lds = (size_t)a.E * sizeof(int);
  auto* kernel = route_block_kernel<T>;
  if (!allow_lds(reinterpret_cast<const void*>(kernel), lds)) return TAOT_ERR_LAUNCH;
  kernel<<<(unsigned)a.T, 256, lds, stream>>>(a);
  return hipGetLastError() == hipSuccess ? TAOT_OK : TAOT_ERR_LAUNCH;
}

template <typename T>
taot_status backward_of(const float* dweights, const void* logits, const int32_t* ids, int64_t tokens, int32_t E,
                        int32_t k, float scale, uint32_t flags, void* dlogits, hipStream_t stream) {
  const int32_t pitch = (E + 7) / 8 * 8;
  auto* kernel = E <= 512 ? route_backward_kernel<T, 1> : E <= 1024 ? route_backward_kernel<T, 2>
               : E <= 4096 ? route_backward_kernel<T, 8> : route_backward_kernel<T, 0>;
  const int waves = E <= 4096 ? 4 : 1;
  const size_t lds = E > 1024 && E <= 4096 ? 0 : (size_t)pitch * waves * sizeof(float);
  if (!allow_lds(reinterpret_cast<const void*>(kernel), lds)) return TAOT_ERR_LAUNCH;
  const int64_t blocks = (tokens + waves - 1) / waves;
  kernel<<<(unsigned)(blocks < 4096 ? blocks : 4096), kWave * waves, lds, stream>>>(
      dweights, static_cast<const T*>(logits), ids, tokens, E, k, scale, flags, static_cast<T*>(dlogits), pitch);
  return hipGetLastError() == hipSuccess ? TAOT_OK : TAOT_ERR_LAUNCH;
}

}  // namespace
}  // namespace taot
