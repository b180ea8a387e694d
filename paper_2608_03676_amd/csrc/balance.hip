// The router's balance loss, what it is made of, and its gradient.
//
//   p_t = softmax(x_t), or sigmoid(x_t) / (sum + tiny);  n tokens count (mask);
//   c_e choices of e among them, P_e = (1 / n) sum_t p_te,
//   loss = E sum_e (c_e / sum c) P_e,   z = (1 / n) sum_t (log sum exp x_t)^2.
//   With a_e = dloss E c_e / (n sum c):
//   softmax:  dx = p (a - <a, p> + 2 dz / n lse);  sigmoid s with sum V:  dx = (a - <a, p>) / V s (1 - s).
//
// A token's logits are read once and held in registers, by 16 lanes, a wave or a
// block.  Sums over tokens are taken by lane, then over a block's waves, then over
// the blocks, always in the same order; choices are whole numbers, counted in LDS.
// A logit of -infinity or NaN is an expert with p = 0, +infinity counts as the
// largest float; a token of such experts alone has p = 0 everywhere and lse = 0.
#include <float.h>

#include "rowio.h"

namespace taot {
namespace {

constexpr float kTiny = 1e-20f;  // added to a sum of sigmoids before it divides
constexpr int kWhole = 0;        // lanes of a token: all of the block

// A token's scores.  L lanes hold it (kWhole: the block's waves), lane l columns
// 8 (i L + l) .. + 7.  v: p;  total: the sum that p was divided by.
template <int L>
struct Group {
  int lanes, lane, waves, slot;
  float (*part)[16];
  template <typename Op>
  __device__ __forceinline__ float reduce(float v, Op op) {
    if constexpr (L == kWhole) {
      v = row_reduce(v, op, part, slot, waves);
      slot ^= 1;
      return v;
    } else {
      return block_reduce<L>(v, op);
    }
  }
};

template <bool SIGMOID, int L, int CPL>
__device__ __forceinline__ void scores(Group<L>& g, int32_t E, f32x8 (&v)[CPL], float& total, float& lse, float& inv) {
  lse = 0.f;
  total = 0.f;
  float top = -INFINITY;
#pragma unroll
  for (int i = 0; i < CPL; ++i)
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int col = 8 * (i * g.lanes + g.lane) + u;
      const float x = v[i][u];
      v[i][u] = col < E && x == x ? fminf(x, FLT_MAX) : -INFINITY;
      if (!SIGMOID) top = fmaxf(top, v[i][u]);
    }
  if (SIGMOID) {
#pragma unroll
    for (int i = 0; i < CPL; ++i)
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        v[i][u] = 1.f / (1.f + expf(-v[i][u]));
        total += v[i][u];
      }
    total = g.reduce(total, SumOp()) + kTiny;
    inv = 1.f / total;
  } else {
    top = fmaxf(g.reduce(top, MaxOp()), -FLT_MAX);
#pragma unroll
    for (int i = 0; i < CPL; ++i)
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        v[i][u] = expf(v[i][u] - top);
        total += v[i][u];
      }
    total = g.reduce(total, SumOp());
    inv = total > 0.f ? 1.f / total : 0.f;
    if (total > 0.f) lse = top + logf(total);
  }
}

struct Tokens {
  int64_t rows, tokens;
  int32_t E, k, blocks;  // blocks of a row
};

// Block (row, b) has tokens b * each .. of its row and writes its share of the sums.
template <typename T, bool SIGMOID, int L, int CPL>
__global__ void __launch_bounds__(1024)
balance_kernel(const T* __restrict__ logits, const int32_t* __restrict__ ids, const uint8_t* __restrict__ mask, Tokens s,
               int64_t each, float* __restrict__ part_p, int32_t* __restrict__ part_c, float* __restrict__ part_z,
               int32_t* __restrict__ part_n) {
  extern __shared__ int32_t room[];
  __shared__ float part[2][16], zs[16];
  __shared__ int32_t ns;
  const int waves = blockDim.x / kWave, tid = threadIdx.x, wid = tid / kWave;
  constexpr int kPer = L == kWhole ? 1 : kWave / (L == kWhole ? kWave : L);  // tokens of a wave
  const int64_t row = blockIdx.x / (uint32_t)s.blocks, block = blockIdx.x % (uint32_t)s.blocks;
  const int64_t lo = block * each, hi = min(lo + each, s.tokens);
  int32_t* hits = room;                                  // [E]
  float* sums = reinterpret_cast<float*>(room + s.E);    // [waves][E], not where the block holds a token
  for (int32_t e = tid; e < s.E; e += blockDim.x) hits[e] = 0;
  if (tid == 0) ns = 0;
  __syncthreads();
  Group<L> g;
  g.lanes = L == kWhole ? blockDim.x : L;
  g.lane = L == kWhole ? tid : tid % (L == kWhole ? kWave : L);
  g.waves = waves;
  g.slot = 0;
  g.part = part;
  const int64_t first = L == kWhole ? lo : lo + tid / (L == kWhole ? kWave : L), step = L == kWhole ? 1 : waves * kPer;
  f32x8 acc[CPL];
  float z = 0.f;
#pragma unroll
  for (int i = 0; i < CPL; ++i) acc[i] = 0.f;
  const int64_t turns = (hi - lo + step - 1) / step;  // the same for all lanes: they work together
  for (int64_t j = 0; j < turns; ++j) {
    const int64_t t = first + j * step, at = row * s.tokens + t;
    const bool in = t < hi && (!mask || mask[at]);
    f32x8 v[CPL];
#pragma unroll
    for (int i = 0; i < CPL; ++i) {
      const int col = 8 * (i * g.lanes + g.lane);
      v[i] = load_row(logits + at * s.E + col, in ? s.E - col : 0);
    }
    float total, lse, inv;
    scores<SIGMOID>(g, s.E, v, total, lse, inv);
    if (!in) inv = lse = 0.f;
#pragma unroll
    for (int i = 0; i < CPL; ++i) acc[i] += v[i] * inv;
    z = fmaf(lse, lse, z);
  }
  int32_t counted = 0;
  for (int64_t i = lo + tid; i < hi; i += blockDim.x) counted += !mask || mask[row * s.tokens + i];
  for (int64_t i = tid; i < (hi - lo) * s.k; i += blockDim.x) {
    const int64_t at = row * s.tokens + lo;
    const int32_t e = ids[at * s.k + i];
    if ((uint32_t)e < (uint32_t)s.E && (!mask || mask[at + i / s.k])) atomicAdd(&hits[e], 1);
  }
  if (counted) atomicAdd(&ns, counted);
  if (L != kWhole && L < kWave) {  // a wave's tokens
#pragma unroll
    for (int o = L; o < kWave; o *= 2) {
      z += __shfl_xor(z, o, kWave);
#pragma unroll
      for (int i = 0; i < CPL; ++i)
#pragma unroll
        for (int u = 0; u < 8; ++u) acc[i][u] += __shfl_xor(acc[i][u], o, kWave);
    }
  }
  if (L == kWhole) {
#pragma unroll
    for (int i = 0; i < CPL; ++i) {
      const int col = 8 * (i * g.lanes + g.lane);
      store_row(part_p + (int64_t)blockIdx.x * s.E + col, acc[i], s.E - col);
    }
  } else {
    if (tid % kWave < L)
#pragma unroll
      for (int i = 0; i < CPL; ++i) {
        const int col = 8 * (i * g.lanes + g.lane);
        store_row(sums + wid * s.E + col, acc[i], s.E - col);
      }
    if (tid % kWave == 0) zs[wid] = z;
  }
  __syncthreads();
  for (int32_t e = tid; e < s.E; e += blockDim.x) {
    part_c[(int64_t)blockIdx.x * s.E + e] = hits[e];
    if (L != kWhole) {
      float p = 0.f;
      for (int w = 0; w < waves; ++w) p += sums[w * s.E + e];
      part_p[(int64_t)blockIdx.x * s.E + e] = p;
    }
  }
  if (tid == 0) {
    if (L != kWhole) {
      z = 0.f;
      for (int w = 0; w < waves; ++w) z += zs[w];
    }
    part_z[blockIdx.x] = z;
    part_n[blockIdx.x] = ns;
  }
}

// prob and counts of 32 experts of a row, 32 threads each.
__global__ void __launch_bounds__(1024)
balance_sums_kernel(const float* __restrict__ part_p, const int32_t* __restrict__ part_c, const int32_t* __restrict__ part_n,
                    int32_t blocks, int32_t E, float* __restrict__ prob, int32_t* __restrict__ counts) {
  __shared__ float sum[32][33];
  __shared__ int32_t cnt[32][33];
  __shared__ int32_t ns;
  const int c = threadIdx.x % 32, r = threadIdx.x / 32;
  const int32_t tiles = (E + 31) / 32, e = (int32_t)(blockIdx.x % (uint32_t)tiles) * 32 + c;
  const int64_t row = blockIdx.x / (uint32_t)tiles, at = row * blocks;
  if (threadIdx.x == 0) ns = 0;
  __syncthreads();
  int32_t n = 0;
  for (int32_t b = threadIdx.x; b < blocks; b += 1024) n += part_n[at + b];
  if (n) atomicAdd(&ns, n);
  float p = 0.f;
  int32_t k = 0;
  if (e < E)
#pragma unroll 4
    for (int32_t b = r; b < blocks; b += 32) {
      p += part_p[(at + b) * E + e];
      k += part_c[(at + b) * E + e];
    }
  sum[r][c] = p;
  cnt[r][c] = k;
  __syncthreads();
  if (r == 0 && e < E) {
#pragma unroll
    for (int w = 1; w < 32; ++w) {
      p += sum[w][c];
      k += cnt[w][c];
    }
    prob[row * E + e] = p / (float)max(ns, 1);
    counts[row * E + e] = k;
  }
}

// loss, z and the number of tokens of a row, a block each.
__global__ void __launch_bounds__(256)
balance_loss_kernel(const float* __restrict__ prob, const int32_t* __restrict__ counts, const float* __restrict__ part_z,
                    const int32_t* __restrict__ part_n, int32_t blocks, int32_t E, float* __restrict__ loss,
                    float* __restrict__ z, int32_t* __restrict__ counted) {
  __shared__ float part[4][4];
  const int64_t row = blockIdx.x;
  float s = 0.f, zz = 0.f;
  int32_t n = 0, all = 0;
  for (int32_t e = threadIdx.x; e < E; e += 256) {
    const int32_t k = counts[row * E + e];
    s = fmaf((float)k, prob[row * E + e], s);
    all += k;
  }
  for (int32_t b = threadIdx.x; b < blocks; b += 256) {
    zz += part_z[row * blocks + b];
    n += part_n[row * blocks + b];
  }
  s = wave_sum(s);
  zz = wave_sum(zz);
  for (int o = 32; o > 0; o >>= 1) {
    n += __shfl_xor(n, o, kWave);
    all += __shfl_xor(all, o, kWave);
  }
  const int w = threadIdx.x / kWave;
  if (threadIdx.x % kWave == 0) {
    part[0][w] = s;
    part[1][w] = zz;
    part[2][w] = __int_as_float(n);
    part[3][w] = __int_as_float(all);
  }
  __syncthreads();
  if (threadIdx.x != 0) return;
  s = zz = 0.f;
  n = all = 0;
  for (int i = 0; i < 4; ++i) {
    s += part[0][i];
    zz += part[1][i];
    n += __float_as_int(part[2][i]);
    all += __float_as_int(part[3][i]);
  }
  loss[row] = (float)E * (s / (float)max(all, 1));
  if (z) z[row] = zz / (float)max(n, 1);
  if (counted) counted[row] = n;
}

// Block (row, b) as in balance_kernel; a lane holds its experts' a throughout.
// dlogits may lie in the logits' or add's memory: a lane reads a token's columns
// before it writes them.
template <typename T, bool SIGMOID, int L, int CPL>
__global__ void __launch_bounds__(1024)
balance_backward_kernel(const float* __restrict__ dloss, const float* __restrict__ dz, const T* logits,
                        const int32_t* __restrict__ counts, const int32_t* __restrict__ counted,
                        const uint8_t* __restrict__ mask, const T* add, Tokens s, int64_t each, T* dlogits) {
  __shared__ float part[2][16];
  constexpr int kLanes = L == kWhole ? kWave : L;
  const int waves = blockDim.x / kWave, tid = threadIdx.x;
  const int64_t row = blockIdx.x / (uint32_t)s.blocks, block = blockIdx.x % (uint32_t)s.blocks;
  const int64_t lo = block * each, hi = min(lo + each, s.tokens);
  Group<L> g;
  g.lanes = L == kWhole ? blockDim.x : L;
  g.lane = L == kWhole ? tid : tid % kLanes;
  g.waves = waves;
  g.slot = 0;
  g.part = part;
  const float n = (float)max(counted[row], 1);
  f32x8 a[CPL];
  float all = 0.f;
#pragma unroll
  for (int i = 0; i < CPL; ++i) {
    const int col = 8 * (i * g.lanes + g.lane);
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      a[i][u] = col + u < s.E ? (float)counts[row * s.E + col + u] : 0.f;
      all += a[i][u];
    }
  }
  all = g.reduce(all, SumOp());
  const float f = dloss[row] * (float)s.E / (fmaxf(all, 1.f) * n), fz = dz ? 2.f * dz[row] / n : 0.f;
#pragma unroll
  for (int i = 0; i < CPL; ++i) a[i] = a[i] * f;
  const int64_t first = L == kWhole ? lo : lo + tid / kLanes, step = L == kWhole ? 1 : waves * (kWave / kLanes);
  const int64_t turns = (hi - lo + step - 1) / step;
  for (int64_t j = 0; j < turns; ++j) {
    const int64_t t = first + j * step, at = row * s.tokens + t;
    const bool is = t < hi, in = is && (!mask || mask[at]);
    f32x8 v[CPL];
#pragma unroll
    for (int i = 0; i < CPL; ++i) {
      const int col = 8 * (i * g.lanes + g.lane);
      v[i] = load_row(logits + at * s.E + col, in ? s.E - col : 0);
    }
    float total, lse, inv, dot = 0.f;
    scores<SIGMOID>(g, s.E, v, total, lse, inv);
#pragma unroll
    for (int i = 0; i < CPL; ++i)
#pragma unroll
      for (int u = 0; u < 8; ++u) dot = fmaf(a[i][u], v[i][u], dot);
    dot = g.reduce(dot, SumOp()) * inv;
    const float up = SIGMOID ? 0.f : fz * lse;
#pragma unroll
    for (int i = 0; i < CPL; ++i) {
      const int col = 8 * (i * g.lanes + g.lane), m = is ? s.E - col : 0;
      f32x8 d = 0.f;
      if (add) d = load_row(add + at * s.E + col, m);
      if (in) {
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const float p = v[i][u];
          d[u] += SIGMOID ? (a[i][u] - dot) * inv * p * (1.f - p) : p * inv * ((a[i][u] - dot) + up);
        }
      }
      store_row(dlogits + at * s.E + col, d, m);
    }
  }
}

// Lanes and chunks that hold a token, and the blocks that share a row.
struct Layout {
  int lanes, cpl, threads;  // lanes kWhole: all threads
  int32_t blocks;
  int64_t each;
};
Layout layout_of(int64_t rows, int64_t tokens, int32_t E) {
  Layout l;
  if (E <= 512) {
    l = {16, E <= 128 ? 1 : E <= 256 ? 2 : 4, 256, 0, 0};
  } else if (E <= 2048) {
    l = {64, E <= 1024 ? 2 : 4, 256, 0, 0};
  } else {
    const int chunks = (E + 7) / 8;
    int cpl = 1;
    while (cpl * 1024 < chunks) cpl *= 2;
    l = {kWhole, cpl, (chunks + cpl * kWave - 1) / (cpl * kWave) * kWave, 0, 0};
  }
  const int64_t at_once = l.lanes == kWhole ? 1 : l.threads / l.lanes, most = (tokens + at_once - 1) / at_once;
  int64_t blocks = (1024 + rows - 1) / rows;
  if (blocks > most) blocks = most;
  if (blocks < 1) blocks = 1;
  l.each = ((tokens + blocks - 1) / blocks + at_once - 1) / at_once * at_once;
  if (l.each < 1) l.each = 1;
  l.blocks = (int32_t)((tokens + l.each - 1) / l.each);
  if (l.blocks < 1) l.blocks = 1;
  return l;
}

struct Partial {
  float* p;
  int32_t* c;
  float* z;
  int32_t* n;
  size_t bytes;
};
Partial carve(void* ws, int64_t rows, int32_t E, int32_t blocks) {
  Carver c{static_cast<char*>(ws)};
  Partial p;
  p.p = c.take<float>((size_t)rows * blocks * E);
  p.c = c.take<int32_t>((size_t)rows * blocks * E);
  p.z = c.take<float>((size_t)rows * blocks);
  p.n = c.take<int32_t>((size_t)rows * blocks);
  p.bytes = c.off;
  return p;
}

// f(lanes, chunks) as constants.
template <typename F>
void with_layout(const Layout& l, F f) {
  using std::integral_constant;
  if (l.lanes == 16) {
    if (l.cpl == 1) f(integral_constant<int, 16>(), integral_constant<int, 1>());
    else if (l.cpl == 2) f(integral_constant<int, 16>(), integral_constant<int, 2>());
    else f(integral_constant<int, 16>(), integral_constant<int, 4>());
  } else if (l.lanes == 64) {
    if (l.cpl == 2) f(integral_constant<int, 64>(), integral_constant<int, 2>());
    else f(integral_constant<int, 64>(), integral_constant<int, 4>());
  } else {
    if (l.cpl == 1) f(integral_constant<int, kWhole>(), integral_constant<int, 1>());
    else if (l.cpl == 2) f(integral_constant<int, kWhole>(), integral_constant<int, 2>());
    else f(integral_constant<int, kWhole>(), integral_constant<int, 4>());
  }
}

template <typename F>
bool by_type(int32_t dtype, F f) {
  if (dtype == TAOT_BF16) return f(__bf16());
  if (dtype == TAOT_F16) return f(_Float16());
  return f(float());
}

constexpr int64_t kRowsAtOnce = kMaxBlocks / (TAOT_MAX_EXPERTS / 32);  // of a launch: up to a block for each 32 experts of a row

}  // namespace

size_t balance_loss_ws(int64_t rows, int64_t tokens, int32_t E) {
  const int64_t n = rows < kRowsAtOnce ? rows : kRowsAtOnce;
  return carve(nullptr, n, E, layout_of(n, tokens, E).blocks).bytes;
}

taot_status launch_balance_loss(const void* logits, const int32_t* ids, const uint8_t* mask, int64_t rows,
                                int64_t tokens, int32_t E, int32_t k, uint32_t flags, int32_t dtype, float* loss,
                                float* z, int32_t* counts, float* prob, int32_t* counted, void* ws, hipStream_t stream) {
  const Layout l = layout_of(rows < kRowsAtOnce ? rows : kRowsAtOnce, tokens, E);
  const Partial p = carve(ws, rows < kRowsAtOnce ? rows : kRowsAtOnce, E, l.blocks);
  const size_t lds = (size_t)E * 4 * (1 + (l.lanes == kWhole ? 0 : l.threads / kWave));
  for (int64_t r = 0; r < rows; r += kRowsAtOnce) {  // one after the other in the same workspace
    const int64_t n = rows - r < kRowsAtOnce ? rows - r : kRowsAtOnce, at = r * tokens;
    const Tokens s{n, tokens, E, k, l.blocks};
    const bool ok = by_type(dtype, [&](auto type) {
      using T = decltype(type);
      bool fine = true;
      with_layout(l, [&](auto lanes, auto cpl) {
        auto* kernel = flags & TAOT_ROUTE_SIGMOID ? balance_kernel<T, true, lanes.value, cpl.value>
                                                  : balance_kernel<T, false, lanes.value, cpl.value>;
        fine = allow_lds(reinterpret_cast<const void*>(kernel), lds);
        if (fine)
          kernel<<<(unsigned)(n * l.blocks), l.threads, lds, stream>>>(
              static_cast<const T*>(logits) + at * E, ids + at * k, mask ? mask + at : nullptr, s, l.each, p.p, p.c, p.z,
              p.n);
      });
      return fine;
    });
    if (!ok) return TAOT_ERR_LAUNCH;
    balance_sums_kernel<<<(unsigned)(n * ((E + 31) / 32)), 1024, 0, stream>>>(p.p, p.c, p.n, l.blocks, E, prob + r * E,
                                                                              counts + r * E);
    balance_loss_kernel<<<(unsigned)n, 256, 0, stream>>>(prob + r * E, counts + r * E, p.z, p.n, l.blocks, E, loss + r,
                                                         z ? z + r : nullptr, counted ? counted + r : nullptr);
  }
  return hipGetLastError() == hipSuccess ? TAOT_OK : TAOT_ERR_LAUNCH;
}

taot_status launch_balance_loss_backward(const float* dloss, const float* dz, const void* logits, const int32_t* counts,
                                         const int32_t* counted, const uint8_t* mask, const void* add, int64_t rows,
                                         int64_t tokens, int32_t E, uint32_t flags, int32_t dtype, void* dlogits,
                                         hipStream_t stream) {
  const Layout l = layout_of(rows < kRowsAtOnce ? rows : kRowsAtOnce, tokens, E);
  for (int64_t r = 0; r < rows; r += kRowsAtOnce) {
    const int64_t n = rows - r < kRowsAtOnce ? rows - r : kRowsAtOnce, at = r * tokens;
    const Tokens s{n, tokens, E, 0, l.blocks};
    by_type(dtype, [&](auto type) {
      using T = decltype(type);
      with_layout(l, [&](auto lanes, auto cpl) {
        auto* kernel = flags & TAOT_ROUTE_SIGMOID ? balance_backward_kernel<T, true, lanes.value, cpl.value>
                                                  : balance_backward_kernel<T, false, lanes.value, cpl.value>;
        kernel<<<(unsigned)(n * l.blocks), l.threads, 0, stream>>>(
            dloss + r, dz ? dz + r : nullptr, static_cast<const T*>(logits) + at * E, counts + r * E, counted + r,
            mask ? mask + at : nullptr, add ? static_cast<const T*>(add) + at * E : nullptr, s, l.each,
            static_cast<T*>(dlogits) + at * E);
      });
      return true;
    });
  }
  return hipGetLastError() == hipSuccess ? TAOT_OK : TAOT_ERR_LAUNCH;
}

}  // namespace taot
