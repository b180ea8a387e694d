// Routing of tokens to experts: scores, an optional balance bias, groups,
// top-k and weights; and the gradient by the logits.
//
//   score  s = softmax(x) or sigmoid(x);   key = s + bias, or x without a bias
//   groups: the best `top_groups` of `groups` equal runs of experts stay, by
//           their largest key or the sum of their two largest
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
#include "rowio.h"

namespace taot {
namespace {

constexpr int kNone = INT32_MIN;     // key of an expert that cannot be chosen
constexpr float kTiny = 1e-20f;
constexpr float kBig = 3.402823466e38f;

struct RouteArgs {
  const void* logits;
  const float* bias;
  int64_t T;
  int32_t E, k, groups, top_groups;
  float scale;
  uint32_t flags;
  int32_t* ids;
  float* weights;
};

// Integers in the order of the floats (-0 is 0).
__device__ __forceinline__ int ordered(float x) {
  const int b = __float_as_int(x + 0.f);
  return b ^ ((b >> 31) & 0x7fffffff);
}
__device__ __forceinline__ float unordered(int b) { return __int_as_float(b ^ ((b >> 31) & 0x7fffffff)); }

// Key of a float that may not be chosen when it is NaN or -inf.
__device__ __forceinline__ int key_of(float x) { return x > -INFINITY ? ordered(x) : kNone; }

__device__ __forceinline__ float sigmoid(float x) { return 1.f / (1.f + expf(-x)); }

// Weights of the chosen experts; lane j of a block of L has the j-th (id -1: none).
// m, sum: the largest logit and the sum of exp(x - m), where the plain softmax needs them.
template <int L, typename T>
__device__ __forceinline__ void finish(const RouteArgs& a, int64_t t, bool mine, int j, int id, float m, float sum) {
  const bool has = mine && id >= 0;
  const float x = has ? fminf((float)static_cast<const T*>(a.logits)[t * a.E + id], kBig) : -INFINITY;
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

// L lanes a token, V experts a lane.  One group: runs of a 16-byte load per
// lane, interleaved.  More: a group is `lpg` lanes, a lane has `per` experts in
// a row.
template <typename T, int L, int V, bool GROUPED>
__global__ void __launch_bounds__(256)
route_kernel(RouteArgs a, int32_t lpg, int32_t per) {
  constexpr int W = 16 / (int)sizeof(T);
  const int lane = threadIdx.x & (kWave - 1), sl = lane % L, base = lane - sl;
  const int64_t t = ((int64_t)blockIdx.x * 256 + threadIdx.x) / L;
  const bool live = t < a.T;
  const T* row = static_cast<const T*>(a.logits) + (live ? t : 0) * a.E;
  const int32_t gs = GROUPED ? a.E / a.groups : a.E;
  const int g = GROUPED ? sl / lpg : 0;
  const int32_t first = GROUPED ? g * gs + (sl % lpg) * per : 0;
  const int32_t mine = GROUPED ? (g < a.groups ? min(per, gs - (sl % lpg) * per) : 0) : a.E;
  auto index = [&](int v) { return GROUPED ? first + v : ((v / W) * L + sl) * W + v % W; };
  auto there = [&](int v) { return live && (GROUPED ? v < mine : index(v) < mine); };

  int key[V];
  float m = 0.f, sum = 1.f;
  {
    float x[V];
#pragma unroll
    for (int v0 = 0; v0 < V; v0 += W) {
      if (there(v0 + W - 1)) {
        typedef T vec __attribute__((ext_vector_type(W)));
        typedef __attribute__((aligned(sizeof(T)))) vec at;
        const vec d = *reinterpret_cast<const at*>(row + index(v0));
#pragma unroll
        for (int u = 0; u < W; ++u) x[v0 + u] = (float)d[u];
      } else {
#pragma unroll
        for (int u = 0; u < W; ++u) x[v0 + u] = there(v0 + u) ? (float)row[index(v0 + u)] : -INFINITY;
      }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) x[v] = x[v] > -INFINITY ? fminf(x[v], kBig) : -INFINITY;
    const bool sigm = a.flags & TAOT_ROUTE_SIGMOID;
    if (!sigm && (a.bias || !(a.flags & TAOT_ROUTE_RENORM))) {
      m = x[0];
#pragma unroll
      for (int v = 1; v < V; ++v) m = fmaxf(m, x[v]);
      m = block_reduce<L>(m, MaxOp());
      const float base_m = m > -INFINITY ? m : 0.f;
      sum = 0.f;
#pragma unroll
      for (int v = 0; v < V; ++v) sum += expf(x[v] - base_m);
      sum = block_reduce<L>(sum, SumOp());
    }
    if (!a.bias) {
#pragma unroll
      for (int v = 0; v < V; ++v) key[v] = key_of(x[v]);
    } else {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const float s = sigm ? sigmoid(x[v]) : expf(x[v] - m) / sum;
        key[v] = x[v] > -INFINITY ? key_of(s + (there(v) ? a.bias[index(v)] : 0.f)) : kNone;
      }
    }
  }

  if constexpr (GROUPED) {
    int b1 = kNone, b2 = kNone;  // the two best of the lane, then of the group
#pragma unroll
    for (int v = 0; v < V; ++v) {
      b2 = max(b2, min(b1, key[v]));
      b1 = max(b1, key[v]);
    }
    auto join = [&](int o1, int o2) {
      b2 = max(min(b1, o1), max(b2, o2));
      b1 = max(b1, o1);
    };
    if (lpg >= 2) join(lane_step<0>(b1), lane_step<0>(b2));
    if (lpg >= 4) join(lane_step<1>(b1), lane_step<1>(b2));
    if (lpg >= 8) join(lane_step<2>(b1), lane_step<2>(b2));
    if (lpg >= 16) join(lane_step<3>(b1), lane_step<3>(b2));
    if (lpg >= 32) join(__shfl_xor(b1, 16, kWave), __shfl_xor(b2, 16, kWave));
    int value = b1;
    if ((a.flags & TAOT_ROUTE_GROUP_TWO) && b2 != kNone) value = ordered(unordered(b1) + unordered(b2));
    int rank = 0;
    for (int o = 0; o < a.groups; ++o) {
      const int other = __shfl(value, base + o * lpg, kWave);
      rank += other > value || (other == value && o < g) ? 1 : 0;
    }
    if (rank >= a.top_groups) {
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
    int at = 0;
#pragma unroll
    for (int v = V - 1; v > 0; --v) at = key[v] == top ? v : at;
    at = key[0] == top ? 0 : at;
    const int e = best == top ? index(at) : INT32_MAX;
    const int win = block_reduce<L>(e, MinOp());
#pragma unroll
    for (int v = 0; v < V; ++v) key[v] = e == win && v == at ? kNone : key[v];
    if (sl == j) id = top == kNone ? -1 : win;
  }
  finish<L, T>(a, t, live && sl < a.k, sl, id, m, sum);
}

// Any number of experts: a block per token, the keys in LDS.
template <typename T>
__global__ void __launch_bounds__(256)
route_block_kernel(RouteArgs a) {
  extern __shared__ int keys[];
  __shared__ int value[TAOT_MAX_ROUTE_GROUPS];
  __shared__ unsigned long long found[4];
  __shared__ float part[2][4];
  __shared__ int chosen[kWave];
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wid = tid / kWave;
  const int64_t t = blockIdx.x;
  const T* row = static_cast<const T*>(a.logits) + t * a.E;
  auto logit = [&](int e) {
    const float x = (float)row[e];
    return x > -INFINITY ? fminf(x, kBig) : -INFINITY;
  };
  const bool sigm = a.flags & TAOT_ROUTE_SIGMOID;
  float m = 0.f, sum = 1.f;
  if (!sigm && (a.bias || !(a.flags & TAOT_ROUTE_RENORM))) {
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
      if (lane == 0) {
        const bool two = (a.flags & TAOT_ROUTE_GROUP_TWO) && b2 != kNone;
        value[g] = two ? ordered(unordered(b1) + unordered(b2)) : b1;
      }
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
  for (int j = 0; j < a.k; ++j) {
    int best = kNone, at = INT32_MAX;
    for (int e = tid; e < a.E; e += 256) {
      const int x = keys[e];
      at = x > best ? e : at;
      best = max(best, x);
    }
    // larger key first, then the lower expert
    unsigned long long p = ((unsigned long long)((uint32_t)best ^ 0x80000000u) << 32) | (0x7fffffffu - (uint32_t)at);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      const unsigned long long q = __shfl_xor(p, o, kWave);
      p = q > p ? q : p;
    }
    if (lane == 0) found[wid] = p;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 4; ++w) p = found[w] > p ? found[w] : p;
    const bool none = (p >> 32) == 0;
    const int win = (int)(0x7fffffffu - (uint32_t)p);
    if (tid == 0) {
      chosen[j] = none ? -1 : win;
      if (!none) keys[win] = kNone;
    }
    __syncthreads();
  }
  if (wid == 0) finish<kWave, T>(a, t, lane < a.k, lane, lane < a.k ? chosen[lane] : -1, m, sum);
}

// ---- gradient ------------------------------------------------------------------
// A wave per token.  The k chosen experts' gradients go to the wave's row of
// LDS (zero elsewhere), which is read back as the row to write; the plain
// softmax adds -p_e sum_j dw_j w_j to every expert.
template <typename T>
__global__ void __launch_bounds__(256)
route_backward_kernel(const float* __restrict__ dweights, const T* __restrict__ logits,
                      const int32_t* __restrict__ ids, int64_t tokens, int32_t E, int32_t k, float scale,
                      uint32_t flags, T* __restrict__ dlogits, int32_t pitch) {
  extern __shared__ float lds[];
  const int lane = threadIdx.x & (kWave - 1), wid = threadIdx.x / kWave;
  const int waves = blockDim.x / kWave;
  float* at = lds + (size_t)wid * pitch;
  for (int e = lane; e < pitch; e += kWave) at[e] = 0.f;
  const bool sigm = flags & TAOT_ROUTE_SIGMOID, renorm = flags & TAOT_ROUTE_RENORM;
  for (int64_t t = (int64_t)blockIdx.x * waves + wid; t < tokens; t += (int64_t)gridDim.x * waves) {
    const T* row = logits + t * E;
    int id = -1;
    float dw = 0.f, x = -INFINITY;
    if (lane < k) {
      id = ids[t * k + lane];
      x = id >= 0 && id < E ? (float)row[id] : -INFINITY;
      x = x > -INFINITY ? fminf(x, kBig) : -INFINITY;
      if (x > -INFINITY) dw = dweights[t * k + lane] * scale;
      else id = -1;
    }
    const bool has = id >= 0;
    float d = 0.f, m = 0.f, inv = 0.f, q = 0.f;
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
      m = -INFINITY;
      for (int e = 8 * lane; e < E; e += 8 * kWave) {
        const f32x8 r = load_row(row + e, E - e);
#pragma unroll
        for (int u = 0; u < 8; ++u)
          if (e + u < E && r[u] > -INFINITY) m = fmaxf(m, fminf(r[u], kBig));
      }
      m = block_reduce<kWave>(m, MaxOp());
      m = m > -INFINITY ? m : 0.f;
      float sum = 0.f;
      for (int e = 8 * lane; e < E; e += 8 * kWave) {
        const f32x8 r = load_row(row + e, E - e);
#pragma unroll
        for (int u = 0; u < 8; ++u) sum += e + u < E && r[u] > -INFINITY ? expf(fminf(r[u], kBig) - m) : 0.f;
      }
      sum = block_reduce<kWave>(sum, SumOp());
      inv = sum > 0.f ? 1.f / sum : 0.f;
      d = has ? dw : 0.f;
      q = block_reduce<kWave>(has ? dw * (expf(x - m) * inv) : 0.f, SumOp());
    }
    if (has) at[id] = d;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    for (int e = 8 * lane; e < E; e += 8 * kWave) {
      f32x8 r;
#pragma unroll
      for (int u = 0; u < 8; ++u) r[u] = at[e + u];
      if (!sigm && !renorm) {
        const f32x8 z = load_row(row + e, E - e);
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const float p = z[u] > -INFINITY ? expf(fminf(z[u], kBig) - m) * inv : 0.f;
          r[u] = p * (r[u] - q);
        }
      }
      store_row(dlogits + t * E + e, r, E - e);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    if (has) at[id] = 0.f;
  }
}

template <typename T, int L, int V, bool GROUPED>
void go(const RouteArgs& a, int32_t lpg, int32_t per, hipStream_t stream) {
  const int64_t blocks = (a.T * L + 255) / 256;
  route_kernel<T, L, V, GROUPED><<<(unsigned)blocks, 256, 0, stream>>>(a, lpg, per);
}

template <typename T>
taot_status route_of(const RouteArgs& a, hipStream_t stream) {
  // lanes of a group, and experts of a lane, when L lanes hold a token
  auto lanes = [&](int L) {
    int32_t n = 1;
    while (2 * n * a.groups <= L) n *= 2;
    return n;
  };
  auto per = [&](int L) { return (a.E / a.groups + lanes(L) - 1) / lanes(L); };
  const bool grouped = a.groups > 1;
  if (a.k <= 16 && a.groups <= 16 && per(16) <= 32) {
    const int32_t n = per(16), lpg = lanes(16);
    if (grouped) {
      if (n <= 8) go<T, 16, 8, true>(a, lpg, n, stream);
      else if (n <= 16) go<T, 16, 16, true>(a, lpg, n, stream);
      else go<T, 16, 32, true>(a, lpg, n, stream);
    } else {
      if (a.E <= 128) go<T, 16, 8, false>(a, lpg, n, stream);
      else if (a.E <= 256) go<T, 16, 16, false>(a, lpg, n, stream);
      else go<T, 16, 32, false>(a, lpg, n, stream);
    }
  } else if (a.groups <= kWave && per(kWave) <= 64) {
    const int32_t n = per(kWave), lpg = lanes(kWave);
    if (grouped) {
      if (n <= 16) go<T, 64, 16, true>(a, lpg, n, stream);
      else go<T, 64, 64, true>(a, lpg, n, stream);
    } else {
      if (a.E <= 1024) go<T, 64, 16, false>(a, lpg, n, stream);
      else go<T, 64, 64, false>(a, lpg, n, stream);
    }
  } else {
    const size_t lds = (size_t)a.E * sizeof(int);
    auto* kernel = route_block_kernel<T>;
    if (!allow_lds(reinterpret_cast<const void*>(kernel), lds)) return TAOT_ERR_LAUNCH;
    kernel<<<(unsigned)a.T, 256, lds, stream>>>(a);
  }
  return hipGetLastError() == hipSuccess ? TAOT_OK : TAOT_ERR_LAUNCH;
}

template <typename T>
taot_status backward_of(const float* dweights, const void* logits, const int32_t* ids, int64_t tokens, int32_t E,
                        int32_t k, float scale, uint32_t flags, void* dlogits, hipStream_t stream) {
  const int32_t pitch = (E + 7) / 8 * 8;
  const int waves = pitch <= 4096 ? 4 : 1;  // a row of LDS per wave, 64 KiB a block
  const size_t lds = (size_t)pitch * waves * sizeof(float);
  auto* kernel = route_backward_kernel<T>;
  if (!allow_lds(reinterpret_cast<const void*>(kernel), lds)) return TAOT_ERR_LAUNCH;
  const int64_t blocks = (tokens + waves - 1) / waves;
  kernel<<<(unsigned)(blocks < 4096 ? blocks : 4096), kWave * waves, lds, stream>>>(
      dweights, static_cast<const T*>(logits), ids, tokens, E, k, scale, flags, static_cast<T*>(dlogits), pitch);
  return hipGetLastError() == hipSuccess ? TAOT_OK : TAOT_ERR_LAUNCH;
}

}  // namespace

taot_status launch_route(const void* logits, const float* bias, int64_t T, int32_t E, int32_t k, int32_t groups,
                         int32_t top_groups, float scale, uint32_t flags, int32_t dtype, int32_t* ids,
                         float* weights, hipStream_t stream) {
  const RouteArgs a{logits, bias, T, E, k, groups, top_groups, scale, flags, ids, weights};
  if (dtype == TAOT_BF16) return route_of<__bf16>(a, stream);
  if (dtype == TAOT_F16) return route_of<_Float16>(a, stream);
  return route_of<float>(a, stream);
}

taot_status launch_route_backward(const float* dweights, const void* logits, const int32_t* ids, int64_t T,
                                  int32_t E, int32_t k, float scale, uint32_t flags, int32_t dtype, void* dlogits,
                                  hipStream_t stream) {
  if (dtype == TAOT_BF16) return backward_of<__bf16>(dweights, logits, ids, T, E, k, scale, flags, dlogits, stream);
  if (dtype == TAOT_F16) return backward_of<_Float16>(dweights, logits, ids, T, E, k, scale, flags, dlogits, stream);
  return backward_of<float>(dweights, logits, ids, T, E, k, scale, flags, dlogits, stream);
}

}  // namespace taot
