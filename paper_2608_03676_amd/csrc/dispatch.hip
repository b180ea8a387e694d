// Carrying out a plan on the tokens: where each routed copy goes in its source
// rank's send buffer, moving rows there, and the weighted way back with its
// gradient.
//
// Copy i of a row (problem, source rank) is occurrence j of its expert e in the
// row, in the order of i.  The guest slots of e, in ascending slot order, take
// X[rank][slot] occurrences each, the home rank takes the rest.  The instances
// (an expert at home, or a guest slot) are ordered by rank, a rank's own
// experts before its guest slots; the send buffer holds them in that order and
// the copies of an instance in the order of i.  All of it is a stable counting
// sort: integers, and the same on every run.
//
// Kernels
//   lists_kernel  (B + 1 blocks)  slots of each expert; experts of each rank
//   count_kernel  (a wave per chunk of a row)  copies of each expert in the chunk
//   bases_kernel  (a thread per row and expert)  running sums over the chunks
//   tables_kernel (a block per row)  slots' shares, instance offsets, sends
//   place_kernel  (a wave per chunk)  occurrence by occurrence to a position
//   rows_kernel, combine_kernel, combine_backward_kernel  (one or four waves a token)
#include "rowio.h"

namespace taot {
namespace {

constexpr int kListThreads = 1024;
constexpr int kUnroll = 4;
constexpr int32_t kChunkMin = 1024, kChunkMax = 32768;
constexpr int64_t kWavesWanted = 16384;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((aligned(1))) u32x4 u32x4_at;

// Lanes of the wave (among `valid`) that hold the same key, of `bits` bits.
__device__ __forceinline__ uint64_t same_key(uint32_t key, int bits, uint64_t valid) {
  uint64_t m = valid;
  for (int b = 0; b < bits; ++b) {
    const bool s = (key >> b) & 1u;
    const uint64_t v = __ballot(s);
    m &= s ? v : ~v;
  }
  return m;
}

// Number of bits that hold 0 .. n.
__host__ __device__ inline int bits_for(uint32_t n) {
  int b = 0;
  while (n >> b) ++b;
  return b;
}

// Exclusive sum over a block of kListThreads threads; *total gets the block's.
template <typename V>
__device__ __forceinline__ V block_exclusive(V v, V* part, V* total) {
  const int lane = threadIdx.x & (kWave - 1), wid = threadIdx.x / kWave;
  V incl = v;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const V y = __shfl_up(incl, o, kWave);
    incl += lane >= o ? y : (V)0;
  }
  __syncthreads();  // part may still be read from the call before
  if (lane == kWave - 1) part[wid] = incl;
  __syncthreads();
  V off = incl - v, all = 0;
  for (int w = 0; w < kListThreads / kWave; ++w) {
    off += w < wid ? part[w] : (V)0;
    all += part[w];
  }
  *total = all;
  return off;
}

// Stable order of n keys in [0, nkeys]: first[q] = keys below q (q <= nkeys),
// place(i, position).  cnt: nkeys + 1 words of LDS.
template <typename Key, typename Place>
__device__ void stable_order(int32_t n, int32_t nkeys, Key key, Place place, int32_t* __restrict__ first, int32_t* cnt) {
  __shared__ int32_t part[kListThreads / kWave];
  const int tid = threadIdx.x, lane = tid & (kWave - 1);
  for (int32_t q = tid; q <= nkeys; q += kListThreads) cnt[q] = 0;
  __syncthreads();
  for (int32_t i = tid; i < n; i += kListThreads) atomicAdd(&cnt[key(i)], 1);
  __syncthreads();
  int32_t run = 0;
  for (int32_t q0 = 0; q0 <= nkeys; q0 += kListThreads) {
    const int32_t q = q0 + tid;
    int32_t total;
    const int32_t mine = q <= nkeys ? cnt[q] : 0;
    const int32_t at = run + block_exclusive(mine, part, &total);
    if (q <= nkeys) {
      cnt[q] = at;
      first[q] = at;
    }
    run += total;
  }
  __syncthreads();
  if (tid >= kWave) return;
  const int bits = bits_for((uint32_t)nkeys);
  for (int32_t i0 = 0; i0 < n; i0 += kWave) {
    const int32_t i = i0 + lane;
    const bool in = i < n;
    const int32_t q = in ? key(i) : nkeys;
    const uint64_t m = same_key((uint32_t)q, bits, __ballot(in));
    const int before = __popcll(m & ((1ull << lane) - 1));
    if (in) {
      const int32_t at = cnt[q] + before;
      place(i, at);
    }
    __builtin_amdgcn_wave_barrier();
    if (in && (m >> lane) == 1) cnt[q] += before + 1;  // the last lane of the key
    __builtin_amdgcn_wave_barrier();
  }
}

// Block b < B: slots of problem b by expert.  Block B: experts by home rank.
__global__ void __launch_bounds__(kListThreads)
lists_kernel(const int32_t* __restrict__ home, const int32_t* __restrict__ slot_expert, int32_t B, int32_t R,
             int32_t E, int32_t K, int32_t* __restrict__ own_at, int32_t* __restrict__ rank_first,
             int32_t* __restrict__ slot_first, int32_t* __restrict__ slot_of, uint32_t* __restrict__ status) {
  extern __shared__ int32_t cnt[];
  __shared__ int32_t bad;
  const int32_t S = R * K, b = blockIdx.x;
  if (b == B) {
    auto key = [&](int32_t e) {
      const int32_t h = home[e];
      return h >= 0 && h < R ? h : R;
    };
    stable_order(E, R, key, [&](int32_t e, int32_t at) { own_at[e] = at + K * key(e); }, rank_first, cnt);
    return;
  }
  const int32_t* slots = slot_expert + (int64_t)b * S;
  if (threadIdx.x == 0) bad = 0;
  __syncthreads();
  for (int32_t e = threadIdx.x; e < E; e += kListThreads)
    if (home[e] < 0 || home[e] >= R) bad = 1;
  __syncthreads();
  if (threadIdx.x == 0 && status) status[b] = bad ? TAOT_ST_BAD_INPUT : 0u;
  auto key = [&](int32_t s) {
    const int32_t e = slots[s];
    return e >= 0 && e < E ? e : E;
  };
  stable_order(S, E, key, [&](int32_t s, int32_t at) { slot_of[(int64_t)b * S + at] = s; },
               slot_first + (int64_t)b * (E + 1), cnt);
}

// hist[row][chunk][e]: copies of expert e in the chunk; e = E: ids that are no expert.
__global__ void __launch_bounds__(256)
count_kernel(const int32_t* __restrict__ ids, int64_t N, int32_t E, int32_t chunk, int32_t chunks, int64_t jobs,
             int32_t* __restrict__ hist) {
  extern __shared__ int32_t cnt[];
  const int lane = threadIdx.x & (kWave - 1);
  const int64_t job = (int64_t)blockIdx.x * (blockDim.x / kWave) + threadIdx.x / kWave;
  if (job >= jobs) return;
  int32_t* mine = cnt + (threadIdx.x / kWave) * (E + 1);
  const int64_t row = job / chunks, lo = (job % chunks) * (int64_t)chunk;
  const int32_t n = (int32_t)min((int64_t)chunk, N - lo);
  const int32_t* src = ids + row * N + lo;
  for (int32_t e = lane; e <= E; e += kWave) mine[e] = 0;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
#pragma unroll 8
  for (int32_t i = lane; i < n; i += kWave) {
    const int32_t e = src[i];
    atomicAdd(&mine[(uint32_t)e < (uint32_t)E ? e : E], 1);
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  int32_t* dst = hist + job * (E + 1);
  for (int32_t e = lane; e <= E; e += kWave) dst[e] = mine[e];
}

// hist becomes the copies of e before the chunk; total[row][e] those of the row.
__global__ void __launch_bounds__(256)
bases_kernel(int32_t* __restrict__ hist, int32_t E, int32_t chunks, int64_t entries, int32_t* __restrict__ total) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= entries) return;
  const int64_t row = i / (E + 1), e = i % (E + 1);
  int32_t* h = hist + row * chunks * (E + 1) + e;
  int32_t run = 0, c = 0;
  for (; c + 8 <= chunks; c += 8) {
    int32_t v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = h[(int64_t)(c + u) * (E + 1)];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      h[(int64_t)(c + u) * (E + 1)] = run;
      run += v[u];
    }
  }
  for (; c < chunks; ++c) {
    const int32_t v = h[(int64_t)c * (E + 1)];
    h[(int64_t)c * (E + 1)] = run;
    run += v;
  }
  total[i] = run;
}

struct Tables {
  const int32_t* own_at;      // [E]          instance of an expert at home
  const int32_t* rank_first;  // [R + 1]      experts at ranks below
  const int32_t* slot_first;  // [B][E + 1]   filled slots of experts below
  const int32_t* slot_of;     // [B][S]       slots by expert
  const int32_t* total;       // [rows][E + 1]
  int64_t* upto;              // [rows][S + 1]  running sum of X over the slots by expert
  int32_t* slot_before;       // [rows][S]    copies of the expert that slots before take
  int32_t* slot_base;         // [rows][S]    position of occurrence 0, were it the slot's
  int2* own;                  // [rows][E]    copies at guests; position of occurrence 0, were it at home
  int32_t* placed;            // [rows]       copies that go somewhere
};

__global__ void __launch_bounds__(kListThreads)
tables_kernel(Tables t, const int32_t* __restrict__ X, int64_t N, int32_t rows, int32_t rank0, int32_t R, int32_t E,
              int32_t K, int32_t* __restrict__ offsets, int32_t* __restrict__ sends, uint32_t* __restrict__ status) {
  __shared__ int64_t part64[kListThreads / kWave];
  __shared__ int32_t part[kListThreads / kWave];
  const int tid = threadIdx.x;
  const int64_t row = blockIdx.x, b = row / rows;
  const int32_t S = R * K, I = E + S, r = rank0 + (int32_t)(row % rows);
  const int32_t* first = t.slot_first + b * (E + 1);
  const int32_t* slot_of = t.slot_of + b * S;
  const int32_t* total = t.total + row * (E + 1);
  const int32_t* share = X + (b * R + r) * (int64_t)S;
  int64_t* upto = t.upto + row * (S + 1);
  int32_t* before = t.slot_before + row * S;
  int32_t* base = t.slot_base + row * S;
  int2* own = t.own + row * E;
  int32_t* off = offsets + row * (I + 1);
  const int32_t filled = S > 0 ? first[E] : 0;
  auto guest_at = [&](int32_t s) { return s + t.rank_first[s / K + 1]; };

  int64_t run = 0;
  for (int32_t i0 = 0; i0 < filled; i0 += kListThreads) {
    const int32_t i = i0 + tid;
    const int64_t x = i < filled ? (int64_t)max(share[slot_of[i]], 0) : 0;
    int64_t all;
    const int64_t at = run + block_exclusive(x, part64, &all);
    if (i < filled) upto[i] = at;
    run += all;
  }
  if (tid == 0) upto[filled] = run;
  for (int32_t s = tid; s < I; s += kListThreads) off[s] = 0;  // slots that hold no expert
  __syncthreads();
  for (int32_t e = tid; e < E; e += kListThreads) {
    const int32_t lo = S > 0 ? first[e] : 0, hi = S > 0 ? first[e + 1] : 0;
    const int64_t guests = upto[hi] - upto[lo];
    const int32_t taken = (int32_t)min(guests, (int64_t)total[e]);
    off[t.own_at[e]] = total[e] - taken;
    own[e].x = taken;
  }
  // the expert of a sorted slot by its place in `first`
  for (int32_t i = tid; i < filled; i += kListThreads) {
    int32_t lo = 0, hi = E;  // first[lo] <= i < first[hi]
    while (lo + 1 < hi) {
      const int32_t mid = (lo + hi) / 2;
      if (first[mid] <= i) lo = mid;
      else hi = mid;
    }
    const int32_t n = total[lo];
    const int32_t c = (int32_t)min(upto[i] - upto[first[lo]], (int64_t)n);
    before[i] = c;
    off[guest_at(slot_of[i])] = (int32_t)min((int64_t)(n - c), upto[i + 1] - upto[i]);
  }
  __syncthreads();
  int32_t sum = 0;
  for (int32_t i0 = 0; i0 < I; i0 += kListThreads) {
    const int32_t i = i0 + tid;
    const int32_t v = i < I ? off[i] : 0;
    int32_t all;
    const int32_t at = sum + block_exclusive(v, part, &all);
    if (i < I) off[i] = at;
    sum += all;
  }
  if (tid == 0) off[I] = sum;
  __syncthreads();
  // experts without a home rank lie behind all instances
  const int32_t valid = t.rank_first[R] + S;
  const int32_t placed = off[valid];
  for (int32_t e = tid; e < E; e += kListThreads) own[e].y = off[t.own_at[e]] - own[e].x;
  for (int32_t i = tid; i < filled; i += kListThreads) base[i] = off[guest_at(slot_of[i])] - before[i];
  for (int32_t j = tid; j < R; j += kListThreads)
    sends[row * R + j] = off[t.rank_first[j + 1] + K * (j + 1)] - off[t.rank_first[j] + K * j];
  if (tid == 0) {
    t.placed[row] = placed;
    if (status && total[E] > 0) atomicOr(&status[b], TAOT_ST_BAD_ID);
  }
  __syncthreads();
  for (int32_t i = valid + 1 + tid; i <= I; i += kListThreads) off[i] = placed;
}

__global__ void __launch_bounds__(256)
place_kernel(const int32_t* __restrict__ ids, Tables t, const int32_t* __restrict__ hist, int64_t N, int32_t rows,
             int32_t E, int32_t S, int32_t chunk, int32_t chunks, int64_t jobs, int bits, int32_t* __restrict__ pos) {
  extern __shared__ int32_t cnt[];
  const int lane = threadIdx.x & (kWave - 1);
  const int64_t job = (int64_t)blockIdx.x * (blockDim.x / kWave) + threadIdx.x / kWave;
  if (job >= jobs) return;
  int32_t* mine = cnt + (threadIdx.x / kWave) * (E + 1);
  const int64_t row = job / chunks, lo = (job % chunks) * (int64_t)chunk, b = row / rows;
  const int32_t n = (int32_t)min((int64_t)chunk, N - lo);
  const int32_t* src = ids + row * N + lo;
  int32_t* dst = pos + row * N + lo;
  const int32_t* first = t.slot_first + b * (E + 1);
  const int32_t* before = t.slot_before + row * S;
  const int32_t* base = t.slot_base + row * S;
  const int2* own = t.own + row * E;
  const int32_t placed = t.placed[row];
  const int32_t dropped = (int32_t)(N - t.total[row * (E + 1) + E]);  // where ids that are no expert begin
  for (int32_t e = lane; e <= E; e += kWave) mine[e] = hist[job * (E + 1) + e];
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  for (int32_t i0 = 0; i0 < n; i0 += kUnroll * kWave) {
    int32_t e[kUnroll], j[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int32_t i = i0 + u * kWave + lane;
      const int32_t q = i < n ? src[i] : E;
      e[u] = (uint32_t)q < (uint32_t)E ? q : E;
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const bool in = i0 + u * kWave + lane < n;
      const uint64_t m = same_key((uint32_t)e[u], bits, __ballot(in));
      const int at = __popcll(m & ((1ull << lane) - 1));
      j[u] = mine[e[u]] + at;
      __builtin_amdgcn_wave_barrier();
      if (in && (m >> lane) == 1) mine[e[u]] = j[u] + 1;
      __builtin_amdgcn_wave_barrier();
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int32_t i = i0 + u * kWave + lane;
      if (i >= n) continue;
      int32_t p;
      if (e[u] == E) {
        p = dropped + j[u];
      } else {
        const int2 o = own[e[u]];
        if (j[u] >= o.x) {
          p = o.y + j[u];
        } else {
          int32_t a = first[e[u]], z = first[e[u] + 1];  // before[a] <= j < before[z]
          while (a + 1 < z) {
            const int32_t mid = (a + z) / 2;
            if (before[mid] <= j[u]) a = mid;
            else z = mid;
          }
          p = base[a] + j[u];
        }
      }
      dst[i] = p < placed ? p : ~p;
    }
  }
}

// ---- rows ------------------------------------------------------------------------
// A row of `bytes` bytes, 16 a lane and step; `lanes` lanes hold one token.
struct Payload {
  const char* in;
  char* out;
  int64_t bytes;
};

template <int WAVES>
__device__ __forceinline__ void spread(const Payload& p, int64_t t, int64_t row0, int64_t N, int32_t k,
                                       const int32_t* __restrict__ pos, int lane) {
  constexpr int kLanes = WAVES * kWave;
  const char* src = p.in + t * p.bytes;
  for (int64_t c = (int64_t)lane * 16; c < p.bytes; c += kLanes * 16) {
    const int n = (int)min((int64_t)16, p.bytes - c);
    u32x4 v = 0;
    if (n == 16) {
      v = *reinterpret_cast<const u32x4_at*>(src + c);
    } else {
#pragma unroll
      for (int u = 0; u < 16; ++u)
        if (u < n) v[u / 4] |= (uint32_t)(uint8_t)src[c + u] << (8 * (u % 4));
    }
    for (int32_t j = 0; j < k; ++j) {
      const int32_t q = pos[j];
      const int64_t to = q >= 0 ? q : ~q;  // a dropped copy leaves its row empty
      if (to >= N) continue;
      const u32x4 w = q >= 0 ? v : u32x4(0);
      char* dst = p.out + (row0 + to) * p.bytes + c;
      if (n == 16) {
        *reinterpret_cast<u32x4_at*>(dst) = w;
      } else {
#pragma unroll
        for (int u = 0; u < 16; ++u)
          if (u < n) dst[u] = (char)(w[u / 4] >> (8 * (u % 4)));
      }
    }
  }
}

template <int WAVES>
__global__ void __launch_bounds__(256)
rows_kernel(Payload a, Payload b, int64_t all, int64_t tokens, int32_t k, const int32_t* __restrict__ pos) {
  constexpr int kLanes = WAVES * kWave;
  const int64_t t = (int64_t)blockIdx.x * (256 / kLanes) + threadIdx.x / kLanes;
  if (t >= all) return;
  const int lane = threadIdx.x % kLanes;
  const int64_t N = tokens * k, row0 = t / tokens * N;
  spread<WAVES>(a, t, row0, N, k, pos + t * k, lane);
  if (b.in) spread<WAVES>(b, t, row0, N, k, pos + t * k, lane);
}

template <typename T, int WAVES>
__global__ void __launch_bounds__(256)
combine_kernel(const T* __restrict__ y, const int32_t* __restrict__ pos, const float* __restrict__ weights,
               int64_t all, int64_t tokens, int32_t k, int32_t H, T* __restrict__ out) {
  constexpr int kLanes = WAVES * kWave;
  constexpr int kAhead = 4;
  const int64_t t = (int64_t)blockIdx.x * (256 / kLanes) + threadIdx.x / kLanes;
  if (t >= all) return;
  const int lane = threadIdx.x % kLanes;
  const int64_t N = tokens * k;
  const T* base = y + t / tokens * N * H;
  for (int32_t c = 8 * lane; c < H; c += 8 * kLanes) {
    f32x8 acc = 0.f;
    for (int32_t j0 = 0; j0 < k; j0 += kAhead) {
      f32x8 v[kAhead];
      float w[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int32_t q = j0 + u < k ? pos[t * k + j0 + u] : -1;
        const bool in = q >= 0 && q < N;
        w[u] = in ? (weights ? weights[t * k + j0 + u] : 1.f) : 0.f;
        v[u] = load_row(base + (in ? q : 0) * (int64_t)H + c, in ? H - c : 0);
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] = fmaf(w[u], v[u][i], acc[i]);
    }
    store_row(out + t * H + c, acc, H - c);
  }
}

// dy[pos] = w dout, dw = <dout, y[pos]>; kAhead copies at a time.  The rows of dy
// are written once, anywhere: past the caches (8192 tokens of 2048 in 16 bits, 8
// copies: 114 us, 119 through them; 16384 of 512, 4 copies: 26 and 44 us).
template <typename T, int WAVES>
__global__ void __launch_bounds__(256)
combine_backward_kernel(const T* __restrict__ dout, const T* __restrict__ y, const int32_t* __restrict__ pos,
                        const float* __restrict__ weights, int64_t all, int64_t tokens, int32_t k, int32_t H,
                        T* __restrict__ dy, float* __restrict__ dweights) {
  using Raw = typename Row8<T>::vec;
  constexpr int kLanes = WAVES * kWave, kAhead = 4;
  __shared__ float part[2][kAhead][4];
  const int64_t t = (int64_t)blockIdx.x * (256 / kLanes) + threadIdx.x / kLanes;
  if (t >= all) return;  // whole waves, and whole blocks where waves share a token
  const int lane = threadIdx.x % kLanes;
  const int64_t N = tokens * k, row0 = t / tokens * N;
  int slot = 0;
  for (int32_t j0 = 0; j0 < k; j0 += kAhead, slot ^= 1) {
    float dot[kAhead], w[kAhead];
    int32_t to[kAhead];  // the copy's row, ~row of a dropped one, or none
    bool any[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      to[u] = j0 + u < k ? pos[t * k + j0 + u] : 0;
      any[u] = j0 + u < k && (to[u] >= 0 ? to[u] : ~to[u]) < N;
      w[u] = any[u] && to[u] >= 0 ? weights[t * k + j0 + u] : 0.f;
      dot[u] = 0.f;
    }
    for (int32_t c = 8 * lane; c < H; c += 8 * kLanes) {
      const int n = H - c;
      Raw v[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const bool in = any[u] && to[u] >= 0;
        v[u] = load_raw(y + (row0 + (in ? to[u] : 0)) * H + c, in ? n : 0);
      }
      const f32x8 d = load_row(dout + t * H + c, n);
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const f32x8 r = widen(v[u]);
#pragma unroll
        for (int i = 0; i < 8; ++i) dot[u] = fmaf(d[i], r[i], dot[u]);
        if (any[u]) {
          T* p = dy + (row0 + (to[u] >= 0 ? to[u] : ~to[u])) * H + c;
          const f32x8 o = to[u] >= 0 ? d * w[u] : f32x8(0.f);
          if (n >= 8) __builtin_nontemporal_store(__builtin_convertvector(o, Raw), reinterpret_cast<typename Row8<T>::at*>(p));
          else store_row(p, o, n);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) dot[u] = block_reduce<kWave>(dot[u], SumOp());
    if constexpr (WAVES > 1) {
      if ((lane & (kWave - 1)) == 0)
#pragma unroll
        for (int u = 0; u < kAhead; ++u) part[slot][u][lane / kWave] = dot[u];
      __syncthreads();  // the two sets of words take turns: one barrier is enough
      if (lane < kAhead && j0 + lane < k) {
        const int32_t q = pos[t * k + j0 + lane];
        const float* s = part[slot][lane];
        dweights[t * k + j0 + lane] = q >= 0 && q < N ? s[0] + s[1] + s[2] + s[3] : 0.f;
      }
    } else {
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        if (lane == 0 && j0 + u < k) dweights[t * k + j0 + u] = any[u] && to[u] >= 0 ? dot[u] : 0.f;
    }
  }
}

// Ids of a wave: enough waves to fill the chip, and no more counters than ids.
int32_t chunk_of(int64_t rows, int64_t N, int32_t E) {
  int64_t c = kChunkMin;
  while (c < kChunkMax && (c < E || rows * ((N + c - 1) / c) > kWavesWanted)) c *= 2;
  return (int32_t)c;
}

struct Plan {
  Tables t;
  int32_t* own_at;
  int32_t* rank_first;
  int32_t* slot_first;
  int32_t* slot_of;
  int32_t* total;
  int32_t* hist;
  size_t bytes;
};

Plan carve(void* ws, int32_t B, int32_t rows, int64_t N, int32_t R, int32_t E, int32_t K) {
  Carver c{static_cast<char*>(ws)};
  const size_t n = (size_t)B * rows, S = (size_t)R * K;
  const int32_t chunk = chunk_of((int64_t)n, N, E);
  const size_t chunks = (size_t)((N + chunk - 1) / chunk);
  Plan p{};
  p.own_at = c.take<int32_t>(E);
  p.rank_first = c.take<int32_t>((size_t)R + 1);
  p.slot_first = c.take<int32_t>((size_t)B * (E + 1));
  p.slot_of = c.take<int32_t>((size_t)B * S);
  p.total = c.take<int32_t>(n * (E + 1));
  p.t.upto = c.take<int64_t>(n * (S + 1));
  p.t.slot_before = c.take<int32_t>(n * S);
  p.t.slot_base = c.take<int32_t>(n * S);
  p.t.own = c.take<int2>(n * E);
  p.t.placed = c.take<int32_t>(n);
  p.hist = c.take<int32_t>(n * chunks * (E + 1));
  p.t.own_at = p.own_at;
  p.t.rank_first = p.rank_first;
  p.t.slot_first = p.slot_first;
  p.t.slot_of = p.slot_of;
  p.t.total = p.total;
  p.bytes = c.off;
  return p;
}

template <typename F>
taot_status by_type(int32_t dtype, F f) {
  if (dtype == TAOT_BF16) f(__bf16());
  else if (dtype == TAOT_F16) f(_Float16());
  else f(float());
  return hipGetLastError() == hipSuccess ? TAOT_OK : TAOT_ERR_LAUNCH;
}

}  // namespace

size_t dispatch_map_ws(int32_t B, int32_t rows, int64_t N, int32_t R, int32_t E, int32_t K) {
  return carve(nullptr, B, rows, N, R, E, K).bytes;
}

taot_status launch_dispatch_map(const int32_t* ids, int32_t B, int32_t rows, int32_t rank0, int64_t N,
                                const int32_t* home, int32_t R, int32_t E, int32_t K, const int32_t* slot_expert,
                                const int32_t* X, int32_t* pos, int32_t* offsets, int32_t* sends, uint32_t* status,
                                void* ws, hipStream_t stream) {
  const Plan p = carve(ws, B, rows, N, R, E, K);
  const int64_t n = (int64_t)B * rows;
  const int32_t chunk = chunk_of(n, N, E), chunks = (int32_t)((N + chunk - 1) / chunk);
  const int64_t jobs = n * chunks;
  const int32_t most = E > R ? E : R;
  const size_t list_lds = (size_t)(most + 1) * sizeof(int32_t);
  if (!allow_lds(reinterpret_cast<const void*>(lists_kernel), list_lds)) return TAOT_ERR_LAUNCH;
  lists_kernel<<<(unsigned)B + 1, kListThreads, list_lds, stream>>>(home, slot_expert, B, R, E, K, p.own_at,
                                                                    p.rank_first, p.slot_first, p.slot_of, status);
  const size_t row_lds = (size_t)(E + 1) * sizeof(int32_t);
  const int waves = 4 * row_lds <= 65536 ? 4 : 2 * row_lds <= 65536 ? 2 : 1;
  const unsigned blocks = (unsigned)((jobs + waves - 1) / waves);
  if (jobs > 0) {
    if (!allow_lds(reinterpret_cast<const void*>(count_kernel), waves * row_lds)) return TAOT_ERR_LAUNCH;
    count_kernel<<<blocks, kWave * waves, waves * row_lds, stream>>>(ids, N, E, chunk, chunks, jobs, p.hist);
  }
  const int64_t entries = n * (E + 1);
  bases_kernel<<<(unsigned)((entries + 255) / 256), 256, 0, stream>>>(p.hist, E, chunks, entries, p.total);
  tables_kernel<<<(unsigned)n, kListThreads, 0, stream>>>(p.t, X, N, rows, rank0, R, E, K, offsets, sends, status);
  if (jobs > 0) {
    if (!allow_lds(reinterpret_cast<const void*>(place_kernel), waves * row_lds)) return TAOT_ERR_LAUNCH;
    place_kernel<<<blocks, kWave * waves, waves * row_lds, stream>>>(ids, p.t, p.hist, N, rows, E, R * K, chunk, chunks,
                                                                     jobs, bits_for((uint32_t)E), pos);
  }
  return hipGetLastError() == hipSuccess ? TAOT_OK : TAOT_ERR_LAUNCH;
}

taot_status launch_dispatch_rows(const void* x, int64_t row_bytes, const void* x_more, int64_t more_bytes,
                                 int64_t rows, int64_t tokens, int32_t k, const int32_t* pos, void* out,
                                 void* out_more, hipStream_t stream) {
  const Payload a{static_cast<const char*>(x), static_cast<char*>(out), row_bytes};
  const Payload b{static_cast<const char*>(x_more), static_cast<char*>(out_more), more_bytes};
  const int64_t all = rows * tokens;
  if (row_bytes > 2048) rows_kernel<4><<<(unsigned)all, 256, 0, stream>>>(a, b, all, tokens, k, pos);
  else rows_kernel<1><<<(unsigned)((all + 3) / 4), 256, 0, stream>>>(a, b, all, tokens, k, pos);
  return hipGetLastError() == hipSuccess ? TAOT_OK : TAOT_ERR_LAUNCH;
}

taot_status launch_combine_rows(const void* y, const int32_t* pos, const float* weights, int64_t rows, int64_t tokens,
                                int32_t k, int32_t H, int32_t dtype, void* out, hipStream_t stream) {
  const int64_t all = rows * tokens;
  return by_type(dtype, [&](auto z) {
    using T = decltype(z);
    const T* in = static_cast<const T*>(y);
    if (H > 1024)
      combine_kernel<T, 4><<<(unsigned)all, 256, 0, stream>>>(in, pos, weights, all, tokens, k, H, static_cast<T*>(out));
    else
      combine_kernel<T, 1><<<(unsigned)((all + 3) / 4), 256, 0, stream>>>(in, pos, weights, all, tokens, k, H,
                                                                         static_cast<T*>(out));
  });
}

taot_status launch_combine_rows_backward(const void* dout, const void* y, const int32_t* pos, const float* weights,
                                         int64_t rows, int64_t tokens, int32_t k, int32_t H, int32_t dtype, void* dy,
                                         float* dweights, hipStream_t stream) {
  const int64_t all = rows * tokens;
  return by_type(dtype, [&](auto z) {
    using T = decltype(z);
    const T *d = static_cast<const T*>(dout), *in = static_cast<const T*>(y);
    T* o = static_cast<T*>(dy);
    if (H > 1024)
      combine_backward_kernel<T, 4><<<(unsigned)all, 256, 0, stream>>>(d, in, pos, weights, all, tokens, k, H, o, dweights);
    else
      combine_backward_kernel<T, 1><<<(unsigned)((all + 3) / 4), 256, 0, stream>>>(d, in, pos, weights, all, tokens, k, H,
                                                                                  o, dweights);
  });
}

}  // namespace taot
