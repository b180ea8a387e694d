// The router's balance loss, what it is made of, and its gradient.
//
//   p_t = softmax(x_t), or sigmoid(x_t) / (sum + tiny);  n tokens count (mask);
//   c_e choices of e among them, P_e = (1 / n) sum_t p_te,
//   loss = E sum_e (c_e / sum c) P_e,   z = (1 / n) sum_t (log sum exp x_t)^2.
//   With a_e = dloss E c_e / (n sum c):
//   softmax:  dx = p (a - <a, p> + 2 dz / n lse);  sigmoid s with sum V:  dx = (a - <a, p>) / V s (1 - s).
//
// A token's logits are read once and held in registers, by 2, 8 or 16 lanes (E to 16,
// 64 and 512), a wave (to 2048) or a block.  Sums over tokens are taken by lane, then over a block's waves,
// then over the blocks, always in the same order; choices are whole numbers, counted in LDS.
// A logit of -infinity or NaN is an expert with p = 0, +infinity counts as the
// largest float; a token of such experts alone has p = 0 everywhere and lse = 0.
#include <float.h>

#include "rowio.h"

namespace taot {
namespace {

constexpr float kTiny = 1e-20f;  // added to a sum of sigmoids before it divides
constexpr int kWhole = 0;        // lanes of a token: all of the block
// Counters of rows lie in cache lines of their own: atomics on one line wait for one
// another (32 rows of 128 tokens of 4096 experts, the sums' kernel: 49 us in a line, 10 so).
constexpr int kLine = 32;

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

// FULL: all columns of the lanes are experts.
template <bool SIGMOID, bool FULL, int L, int CPL>
__device__ __forceinline__ void scores(Group<L>& g, int32_t E, f32x8 (&v)[CPL], float& total, float& lse, float& inv) {
  lse = 0.f;
  total = 0.f;
  if (!FULL) {
#pragma unroll
    for (int i = 0; i < CPL; ++i)
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (8 * (i * g.lanes + g.lane) + u >= E) v[i][u] = -INFINITY;
  }
  if (SIGMOID) {
#pragma unroll
    for (int i = 0; i < CPL; ++i)
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        // below -87 the sigmoid is not a normal number, and 0 here; so is that of NaN.  The hardware's reciprocal is
        // off by a unit in the last place, as the exponential is
        const float x = v[i][u], s = __builtin_amdgcn_rcpf(1.f + exponential(within(-x, -150.f, 88.f)));
        v[i][u] = x >= -87.f ? s : 0.f;
        total += v[i][u];
      }
    total = g.reduce(total, SumOp()) + kTiny;
    inv = 1.f / total;
  } else {
    float top = -FLT_MAX;
#pragma unroll
    for (int i = 0; i < CPL; ++i)
#pragma unroll
      for (int u = 0; u < 8; ++u) top = fmaxf(top, v[i][u]);  // the number where one of the two is NaN
    top = fminf(g.reduce(top, MaxOp()), FLT_MAX);
#pragma unroll
    for (int i = 0; i < CPL; ++i)
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        v[i][u] = exponential(within(v[i][u] - top, -150.f, 0.f));  // 0 at -150, where -infinity and NaN are
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
// 65536 tokens of 256 experts, 8 choices, in 32 bits: 14 us for 69 MB, 4.8 TB/s; 8 of them
// the vector units issue.  The sums behind take 5, a chain of loads and one of writes.
template <typename T, bool SIGMOID, bool FULL, int L, int CPL>
__global__ void __launch_bounds__(1024)
balance_kernel(const T* __restrict__ logits, const int32_t* __restrict__ ids, const uint8_t* __restrict__ mask, Tokens s,
               int64_t each, float* __restrict__ part_p, int32_t* __restrict__ part_c, float* __restrict__ part_z,
               int32_t* __restrict__ part_n, int32_t* __restrict__ done) {
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
  if (tid == 0) {
    ns = 0;
    if (block == 0) done[row * kLine] = 0;
  }
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
  typename Row8<T>::vec raw[CPL];
  bool in = false;
  auto fetch = [&](int64_t t) {
    const int64_t at = row * s.tokens + t;
    in = t < hi && (!mask || mask[at]);
#pragma unroll
    for (int i = 0; i < CPL; ++i) {
      const int col = 8 * (i * g.lanes + g.lane);
      raw[i] = load_raw(logits + at * s.E + col, t >= hi ? 0 : FULL ? 8 : s.E - col);
    }
  };
  fetch(first);
  int32_t counted = 0;
  for (int64_t i = lo + tid; i < hi; i += blockDim.x) counted += !mask || mask[row * s.tokens + i];
  for (int64_t i = tid; i < (hi - lo) * s.k; i += blockDim.x) {
    const int64_t at = row * s.tokens + lo;
    const int32_t e = ids[at * s.k + i];
    if ((uint32_t)e < (uint32_t)s.E && (!mask || mask[at + i / s.k])) atomicAdd(&hits[e], 1);
  }
  if (counted) atomicAdd(&ns, counted);
  for (int64_t j = 0; j < turns; ++j) {
    f32x8 v[CPL];
#pragma unroll
    for (int i = 0; i < CPL; ++i) v[i] = widen(raw[i]);
    const bool now = in;
    if (j + 1 < turns) fetch(first + (j + 1) * step);
    float total, lse, inv;
    scores<SIGMOID, FULL>(g, s.E, v, total, lse, inv);
    if (!now) inv = lse = 0.f;
#pragma unroll
    for (int i = 0; i < CPL; ++i)
#pragma unroll
      for (int u = 0; u < 8; ++u) acc[i][u] = fmaf(v[i][u], inv, acc[i][u]);
    z = fmaf(lse, lse, z);
  }
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

// prob and counts of kTile experts of a row, up to 32 threads each, and these experts'
// part of the loss.  The last block of a row adds the parts up, in order.
constexpr int kTile = 32;
struct Part {
  float loss;
  int32_t choices;
};
template <int THREADS>
__global__ void __launch_bounds__(THREADS)
balance_sums_kernel(const float* __restrict__ part_p, const int32_t* __restrict__ part_c, const float* __restrict__ part_z,
                    const int32_t* __restrict__ part_n, int32_t blocks, int32_t E, float* __restrict__ prob,
                    int32_t* __restrict__ counts, uint64_t* parts, int32_t* done, float* __restrict__ loss,
                    float* __restrict__ z, int32_t* __restrict__ counted) {
  constexpr int kWaves = THREADS / kWave;
  __shared__ float sum[kWaves][kTile], zs[kWaves];
  __shared__ int32_t cnt[kWaves][kTile], ns[kWaves], all[kWaves];
  __shared__ int32_t last;
  const int c = threadIdx.x % kTile, r = threadIdx.x / kTile, wid = threadIdx.x / kWave;
  const int32_t tiles = (E + kTile - 1) / kTile, e = (int32_t)(blockIdx.x % (uint32_t)tiles) * kTile + c;
  const int64_t row = blockIdx.x / (uint32_t)tiles, at = row * blocks;
  float p = 0.f, zz = 0.f;  // z is the last block's to write, but here its way is short
  int32_t k = 0, n = 0;
  for (int32_t b = threadIdx.x; b < blocks; b += THREADS) {
    n += part_n[at + b];
    zz += part_z[at + b];
  }
  if (e < E)
#pragma unroll 8
    for (int32_t b = r; b < blocks; b += THREADS / kTile) {
      p += part_p[(at + b) * E + e];
      k += part_c[(at + b) * E + e];
    }
  zz = wave_sum(zz);
  for (int o = 32; o > 0; o >>= 1) n += __shfl_xor(n, o, kWave);
  if (threadIdx.x % kWave == 0) {
    ns[wid] = n;
    zs[wid] = zz;
  }
#pragma unroll
  for (int o = kTile; o < kWave; o *= 2) {
    p += __shfl_xor(p, o, kWave);
    k += __shfl_xor(k, o, kWave);
  }
  if (threadIdx.x % kWave < kTile) {
    sum[wid][c] = p;
    cnt[wid][c] = k;
  }
  __syncthreads();
  n = 0;
  zz = 0.f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    n += ns[w];
    zz += zs[w];
  }
  if (threadIdx.x < kTile) {
    p = 0.f;
    k = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      p += sum[w][c];
      k += cnt[w][c];
    }
    p /= (float)max(n, 1);
    if (e < E) {
      prob[row * E + e] = p;
      counts[row * E + e] = k;
    }
    float mine = block_reduce<kTile>((float)k * p, SumOp());  // the others have neither
    for (int o = 1; o < kTile; o *= 2) k += __shfl_xor(k, o, kTile);
    if (threadIdx.x == 0) {
      // The part is written past the die's own cache, and is there when the wait is over; no other write has to be seen
      // by the last block.
      __hip_atomic_store(parts + blockIdx.x, __builtin_bit_cast(uint64_t, Part{mine, k}), __ATOMIC_RELAXED,
                         __HIP_MEMORY_SCOPE_AGENT);
      __atomic_signal_fence(__ATOMIC_SEQ_CST);
      __builtin_amdgcn_s_waitcnt(0);
      __atomic_signal_fence(__ATOMIC_SEQ_CST);
      last = __hip_atomic_fetch_add(done + row * kLine, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == tiles - 1;
    }
  }
  __syncthreads();
  if (!last) return;
  float l = 0.f;
  k = 0;
  for (int32_t i = threadIdx.x; i < tiles; i += THREADS) {
    const Part q = __builtin_bit_cast(
        Part, __hip_atomic_load(parts + row * tiles + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
    l += q.loss;
    k += q.choices;
  }
  l = wave_sum(l);
  for (int o = 32; o > 0; o >>= 1) k += __shfl_xor(k, o, kWave);
  if (threadIdx.x % kWave == 0) {
    sum[wid][0] = l;
    all[wid] = k;
  }
  __syncthreads();
  if (threadIdx.x != 0) return;
  l = 0.f;
  k = 0;
  for (int w = 0; w < kWaves; ++w) {
    l += sum[w][0];
    k += all[w];
  }
  loss[row] = (float)E * (l / (float)max(k, 1));
  if (z) z[row] = zz / (float)max(n, 1);
  if (counted) counted[row] = n;
}

// Block (row, b) as in balance_kernel; a lane finds its experts' counts in LDS.  32768
// tokens of 384 experts in bfloat16, sigmoid, with another gradient: 17 us for 75 MB,
// 4.5 TB/s; 9 of them the vector units issue.
// dlogits may lie in the logits' or add's memory: a lane reads a token's columns
// before it writes them.
template <typename T, bool SIGMOID, bool FULL, int L, int CPL>
__global__ void __launch_bounds__(L == kWhole ? 1024 : 256)
balance_backward_kernel(const float* __restrict__ dloss, const float* __restrict__ dz, const T* logits,
                        const int32_t* __restrict__ counts, const int32_t* __restrict__ counted,
                        const uint8_t* __restrict__ mask, const T* add, Tokens s, int64_t each, T* dlogits) {
  extern __shared__ f32x8 table[];  // count of each expert, 0 behind the last
  __shared__ float part[2][16], alls[16];
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
  const int64_t first = L == kWhole ? lo : lo + tid / kLanes, step = L == kWhole ? 1 : waves * (kWave / kLanes);
  const int64_t turns = (hi - lo + step - 1) / step;
  typename Row8<T>::vec raw[CPL], more[CPL];
  bool in = false;
  auto fetch = [&](int64_t t) {
    const int64_t at = row * s.tokens + t;
    in = t < hi && (!mask || mask[at]);
#pragma unroll
    for (int i = 0; i < CPL; ++i) {
      const int col = 8 * (i * g.lanes + g.lane), m = t >= hi ? 0 : FULL ? 8 : s.E - col;
      raw[i] = load_raw(logits + at * s.E + col, m);
      if (add) more[i] = load_raw(add + at * s.E + col, m);
    }
  };
  fetch(first);
  float* const words = reinterpret_cast<float*>(table);
  float all = 0.f;
  for (int32_t e = tid; e < (s.E + 7) / 8 * 8; e += blockDim.x) {
    const float c = e < s.E ? (float)counts[row * s.E + e] : 0.f;
    words[e] = c;
    all += c;
  }
  all = block_reduce<kWave>(all, SumOp());
  if (tid % kWave == 0) alls[tid / kWave] = all;
  const float n = (float)max(counted[row], 1), fz = dz ? 2.f * (dz[row] / n) : 0.f, fl = dloss[row];
  __syncthreads();
  all = 0.f;
  for (int w = 0; w < waves; ++w) all += alls[w];
  const float f = fl * ((float)s.E / (fmaxf(all, 1.f) * n));  // fl E may be no float where f is one
  for (int64_t j = 0; j < turns; ++j) {
    const int64_t t = first + j * step, at = row * s.tokens + t;
    f32x8 v[CPL];
    typename Row8<T>::vec also[CPL];
#pragma unroll
    for (int i = 0; i < CPL; ++i) {
      v[i] = widen(raw[i]);
      also[i] = more[i];
    }
    const bool now = in;
    if (j + 1 < turns) fetch(t + step);
    float total, lse, inv, dot = 0.f;
    scores<SIGMOID, FULL>(g, s.E, v, total, lse, inv);
    const f32x8* const a = table + g.lane;
#pragma unroll
    for (int i = 0; i < CPL; ++i) {
      const f32x8 c = FULL || 8 * (i * g.lanes + g.lane) < s.E ? a[i * g.lanes] : f32x8(0.f);
#pragma unroll
      for (int u = 0; u < 8; ++u) dot = fmaf(c[u], v[i][u], dot);
    }
    dot = g.reduce(dot, SumOp()) * inv * f;
    // A finite dz has a finite term, also where lse is the largest float: experts of p = 0 get 0.  A dz that is not
    // finite has none, so that who looks for it in the gradient finds it.
    const float zl = fz * lse, term = fabsf(fz) <= FLT_MAX ? within(zl, -FLT_MAX, FLT_MAX) : zl;
    const float up = SIGMOID ? dot : dot - term, each_p = now ? inv : 0.f;
#pragma unroll
    for (int i = 0; i < CPL; ++i) {
      const int col = 8 * (i * g.lanes + g.lane), m = t >= hi ? 0 : FULL ? 8 : s.E - col;
      const f32x8 c = FULL || col < s.E ? a[i * g.lanes] : f32x8(0.f);
      f32x8 d = 0.f;
      if (add) d = widen(also[i]);
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const float p = v[i][u] * each_p;
        const float w = SIGMOID ? p - p * v[i][u] : p;
        if (now) d[u] = fmaf(fmaf(c[u], f, -up), w, d[u]);
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
// Forward: blocks of 16 waves, one on each of the 256 compute units: more of them cost
// more in the sums than they bring (65536 tokens of 256 in 32 bits, us by blocks of 16,
// 8 and 8 waves: 256 22.5, 768 25.4, 1024 26.9).  Backward: what is resident at once
// (32768 of 384 in 16 bits, 1280 blocks of four waves 18.2, 2048 21.0, 4096 21.0).
Layout layout_of(int64_t rows, int64_t tokens, int32_t E, bool backward) {
  Layout l;
  if (E <= 16) {
    l = {2, 1, backward ? 256 : 1024, 0, 0};
  } else if (E <= 64) {
    l = {8, 1, backward ? 256 : 1024, 0, 0};
  } else if (E <= 512) {
    l = {16, (E + 127) / 128, backward ? 256 : 1024, 0, 0};
  } else if (E <= 2048) {
    l = {64, E <= 1024 ? 2 : 4, backward ? 256 : 1024, 0, 0};
  } else {
    const int chunks = (E + 7) / 8;
    int cpl = 1;
    while (cpl * 1024 < chunks) cpl *= 2;
    l = {kWhole, cpl, (chunks + cpl * kWave - 1) / (cpl * kWave) * kWave, 0, 0};
  }
  const int64_t at_once = l.lanes == kWhole ? 1 : l.threads / l.lanes, most = (tokens + at_once - 1) / at_once;
  const int64_t wanted = 256 * (backward && l.lanes != kWhole ? 5 : 1024 / l.threads);
  int64_t blocks = (wanted + rows - 1) / rows;
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
  int32_t *n, *done;
  uint64_t* parts;
  size_t bytes;
};
Partial carve(void* ws, int64_t rows, int32_t E, int32_t blocks) {
  Carver c{static_cast<char*>(ws)};
  Partial p;
  p.p = c.take<float>((size_t)rows * blocks * E);
  p.c = c.take<int32_t>((size_t)rows * blocks * E);
  p.z = c.take<float>((size_t)rows * blocks);
  p.n = c.take<int32_t>((size_t)rows * blocks);
  p.done = c.take<int32_t>((size_t)rows * kLine);
  p.parts = c.take<uint64_t>((size_t)rows * ((E + kTile - 1) / kTile));
  p.bytes = c.off;
  return p;
}

// f(lanes, chunks, whether they hold experts alone) as constants.
template <int L, int CPL, typename F>
void with_full(int32_t E, F f) {
  using std::integral_constant;
  if constexpr (L >= 2 && L <= 16) {
    if (E == 8 * L * CPL) return f(integral_constant<int, L>(), integral_constant<int, CPL>(), std::true_type());
  }
  f(integral_constant<int, L>(), integral_constant<int, CPL>(), std::false_type());
}
template <typename F>
void with_layout(const Layout& l, int32_t E, F f) {
  if (l.lanes == 2) with_full<2, 1>(E, f);
  else if (l.lanes == 8) with_full<8, 1>(E, f);
  else if (l.lanes == 16) {
    if (l.cpl == 1) with_full<16, 1>(E, f);
    else if (l.cpl == 2) with_full<16, 2>(E, f);
    else if (l.cpl == 3) with_full<16, 3>(E, f);
    else with_full<16, 4>(E, f);
  } else if (l.lanes == 64) {
    if (l.cpl == 2) with_full<64, 2>(E, f);
    else with_full<64, 4>(E, f);
  } else {
    if (l.cpl == 1) with_full<kWhole, 1>(E, f);
    else if (l.cpl == 2) with_full<kWhole, 2>(E, f);
    else with_full<kWhole, 4>(E, f);
  }
}

template <typename F>
bool by_type(int32_t dtype, F f) {
  if (dtype == TAOT_BF16) return f(__bf16());
  if (dtype == TAOT_F16) return f(_Float16());
  return f(float());
}

constexpr int64_t kRowsAtOnce = kMaxBlocks / (TAOT_MAX_EXPERTS / kTile);  // of a launch: up to a block for each tile of a row

}  // namespace

size_t balance_loss_ws(int64_t rows, int64_t tokens, int32_t E) {
  const int64_t n = rows < kRowsAtOnce ? rows : kRowsAtOnce;
  return carve(nullptr, n, E, layout_of(n, tokens, E, false).blocks).bytes;
}

taot_status launch_balance_loss(const void* logits, const int32_t* ids, const uint8_t* mask, int64_t rows,
                                int64_t tokens, int32_t E, int32_t k, uint32_t flags, int32_t dtype, float* loss,
                                float* z, int32_t* counts, float* prob, int32_t* counted, void* ws, hipStream_t stream) {
  const Layout l = layout_of(rows < kRowsAtOnce ? rows : kRowsAtOnce, tokens, E, false);
  const Partial p = carve(ws, rows < kRowsAtOnce ? rows : kRowsAtOnce, E, l.blocks);
  const size_t lds = (size_t)E * 4 * (1 + (l.lanes == kWhole ? 0 : l.threads / kWave));
  for (int64_t r = 0; r < rows; r += kRowsAtOnce) {  // one after the other in the same workspace
    const int64_t n = rows - r < kRowsAtOnce ? rows - r : kRowsAtOnce, at = r * tokens;
    const Tokens s{n, tokens, E, k, l.blocks};
    const bool ok = by_type(dtype, [&](auto type) {
      using T = decltype(type);
      bool fine = true;
      with_layout(l, E, [&](auto lanes, auto cpl, auto full) {
        auto* kernel = flags & TAOT_ROUTE_SIGMOID ? balance_kernel<T, true, full.value, lanes.value, cpl.value>
                                                  : balance_kernel<T, false, full.value, lanes.value, cpl.value>;
        fine = allow_lds(reinterpret_cast<const void*>(kernel), lds);
        if (fine)
          kernel<<<(unsigned)(n * l.blocks), l.threads, lds, stream>>>(
              static_cast<const T*>(logits) + at * E, ids + at * k, mask ? mask + at : nullptr, s, l.each, p.p, p.c, p.z,
              p.n, p.done);
      });
      return fine;
    });
    if (!ok) return TAOT_ERR_LAUNCH;
    const bool few = l.blocks <= 2 * 256 / kTile;
    auto* const sums = few ? balance_sums_kernel<256> : balance_sums_kernel<1024>;
    sums<<<(unsigned)(n * ((E + kTile - 1) / kTile)), few ? 256 : 1024, 0, stream>>>(
        p.p, p.c, p.z, p.n, l.blocks, E, prob + r * E, counts + r * E, p.parts, p.done, loss + r, z ? z + r : nullptr,
        counted ? counted + r : nullptr);
  }
  return hipGetLastError() == hipSuccess ? TAOT_OK : TAOT_ERR_LAUNCH;
}

taot_status launch_balance_loss_backward(const float* dloss, const float* dz, const void* logits, const int32_t* counts,
                                         const int32_t* counted, const uint8_t* mask, const void* add, int64_t rows,
                                         int64_t tokens, int32_t E, uint32_t flags, int32_t dtype, void* dlogits,
                                         hipStream_t stream) {
  const Layout l = layout_of(rows < kRowsAtOnce ? rows : kRowsAtOnce, tokens, E, true);
  const size_t lds = (size_t)((E + 7) / 8) * sizeof(f32x8);
  for (int64_t r = 0; r < rows; r += kRowsAtOnce) {
    const int64_t n = rows - r < kRowsAtOnce ? rows - r : kRowsAtOnce, at = r * tokens;
    const Tokens s{n, tokens, E, 0, l.blocks};
    const bool ok = by_type(dtype, [&](auto type) {
      using T = decltype(type);
      bool fine = true;
      with_layout(l, E, [&](auto lanes, auto cpl, auto full) {
        auto* kernel = flags & TAOT_ROUTE_SIGMOID ? balance_backward_kernel<T, true, full.value, lanes.value, cpl.value>
                                                  : balance_backward_kernel<T, false, full.value, lanes.value, cpl.value>;
        fine = allow_lds(reinterpret_cast<const void*>(kernel), lds);
        if (!fine) return;
        kernel<<<(unsigned)(n * l.blocks), l.threads, lds, stream>>>(
            dloss + r, dz ? dz + r : nullptr, static_cast<const T*>(logits) + at * E, counts + r * E, counted + r,
            mask ? mask + at : nullptr, add ? static_cast<const T*>(add) + at * E : nullptr, s, l.each,
            static_cast<T*>(dlogits) + at * E);
      });
      return fine;
    });
    if (!ok) return TAOT_ERR_LAUNCH;
  }
  return hipGetLastError() == hipSuccess ? TAOT_OK : TAOT_ERR_LAUNCH;
}

}  // namespace taot
