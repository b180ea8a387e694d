// Products of 8-bit integers with a scale for each row and each channel, over runs
// of rows that have a weight each: the experts of a mixture on the rows sent to them.
//
//   out[t][n] = scale[t] weight_scale[e][n] sum_k x[t][k] weight[e][n][k]
//
// The sum is of whole numbers and exact in 32 bits (K up to TAOT_MAX_INNER); it is
// rounded to a float, multiplied by the two scales in 32 bits and rounded to the output's
// type.  The order of the sum does not matter, so waves and blocks may share it.
//
// runs_kernel lists the tiles of rows: a tile lies within one run.  The weights are
// the matrix unit's first operand, so a lane's results are neighbouring channels.
//   product_few_kernel     16 rows, 16 channels   few rows a run: the weights' way from memory
//   product_some_kernel    64 rows, 32 channels   few tiles in all: waves share the inner dimension
//   product_kernel         64 rows, 128 channels  middling runs (and 256 by 256 where rows do not
//                                                 begin at multiples of 16 bytes)
//   product_half_kernel    128 rows, 128 channels  runs that are too few for the next
//   product_wide_kernel    256 rows, 256 channels  long runs: the matrix units
// The rule is at kind_of, with both sides of each bound.
#include "rowio.h"

namespace taot {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));
typedef __attribute__((aligned(1))) i32x4 i32x4_at;
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((aligned(4))) f32x4 f32x4_at;

// Rows of one run, or (expert < 0) rows that no expert has and that become zero.
struct Tile {
  int32_t row, rows, expert, pad;
};

// Runs as they are worked on: [0, o_0), the given ones, [o_runs, M).  Offsets are
// taken in [0, M], and each as at least the one before it.
template <int kRunThreads>
__global__ void __launch_bounds__(kRunThreads)
runs_kernel(const int32_t* __restrict__ offsets, const int32_t* __restrict__ experts, int32_t runs, int32_t G, int64_t M,
            int32_t rows_of_tile, Tile* __restrict__ tiles, int32_t* __restrict__ total) {
  __shared__ int32_t starts[kRunThreads + 1], firsts[kRunThreads + 1], part[kRunThreads / kWave], whose[kRunThreads];
  const int tid = threadIdx.x, lane = tid % kWave, wid = tid / kWave;
  const int32_t V = runs + 2;
  int32_t start = 0, done = 0;  // of the next run, and tiles so far
  for (int32_t v0 = 0; v0 < V; v0 += kRunThreads) {
    const int32_t v = v0 + tid;
    // the end of run v: the largest offset up to it
    int32_t end = (int32_t)M;
    if (v <= runs) end = max(0, min(offsets[v], (int32_t)M));
    whose[tid] = v >= 1 && v <= runs ? (experts ? experts[v - 1] : v - 1) : -1;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
      const int32_t y = __shfl_up(end, o, kWave);
      if (lane >= o) end = max(end, y);
    }
    if (lane == kWave - 1) part[wid] = end;
    __syncthreads();
    end = max(end, start);
    for (int w = 0; w < wid; ++w) end = max(end, part[w]);
    starts[tid + 1] = end;
    if (tid == 0) starts[0] = start;
    __syncthreads();
    const int32_t n = v < V ? (end - starts[tid] + rows_of_tile - 1) / rows_of_tile : 0;
    int32_t upto = n;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
      const int32_t y = __shfl_up(upto, o, kWave);
      upto += lane >= o ? y : 0;
    }
    if (lane == kWave - 1) part[wid] = upto;
    __syncthreads();
    for (int w = 0; w < wid; ++w) upto += part[w];
    firsts[tid + 1] = upto;
    if (tid == 0) firsts[0] = 0;
    __syncthreads();
    const int32_t here = firsts[kRunThreads];
    for (int32_t t = tid; t < here; t += kRunThreads) {
      int32_t a = 0, z = kRunThreads;
      while (a + 1 < z) {  // firsts[a] <= t < firsts[z]
        const int32_t mid = (a + z) / 2;
        if (firsts[mid] <= t) a = mid;
        else z = mid;
      }
      const int32_t row = starts[a] + (t - firsts[a]) * rows_of_tile, e = whose[a];
      tiles[done + t] = Tile{row, min(rows_of_tile, starts[a + 1] - row), (uint32_t)e < (uint32_t)G ? e : -1, 0};
    }
    done += here;
    start = starts[kRunThreads];
    __syncthreads();
  }
  if (tid == 0) *total = done;
}

// 16 P bytes of a row as the words that hold them.  SHIFT: they begin `shift` bytes
// behind a word, and there is a word more (16 rows by 8192 channels of 8191: 69 us with
// reads at the bytes' own addresses, 24 for 8192).  What is loaded is not touched before
// it is needed, so that it may be on its way.
template <bool SHIFT, int P>
struct Words {
  i32x4 w[P];
  int last;
  __device__ __forceinline__ void load(const int8_t* __restrict__ from, uint32_t shift) {
    const int8_t* const at = from - (SHIFT ? shift : 0);
#pragma unroll
    for (int s = 0; s < P; ++s) w[s] = *reinterpret_cast<const i32x4_at*>(at + 16 * s);
    if (SHIFT) last = *reinterpret_cast<const int*>(at + 16 * P);
  }
  // The words that hold one of the next n bytes of the row, zeros for others.
  __device__ __forceinline__ void load_end(const int8_t* __restrict__ from, uint32_t shift, int n) {
    const int* const at = reinterpret_cast<const int*>(from - (SHIFT ? shift : 0));
    const int m = n > 0 ? n + (SHIFT ? (int)shift : 0) : 0;
#pragma unroll
    for (int u = 0; u < 4 * P; ++u) {
      w[u / 4][u % 4] = 0;
      if (4 * u < m) w[u / 4][u % 4] = at[u];
    }
    last = 0;
    if (SHIFT && 16 * P < m) last = at[4 * P];
  }
  __device__ __forceinline__ i32x4 bytes(int s, uint32_t shift) const {
    if constexpr (!SHIFT) return w[s];
    i32x4 v;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int next = u < 3 ? w[s][u + 1] : s < P - 1 ? w[s + 1 < P ? s + 1 : s][0] : last;
      v[u] = (int)__builtin_amdgcn_alignbyte((uint32_t)next, (uint32_t)w[s][u], shift);
    }
    return v;
  }
  // As many as n of them, zeros behind.
  __device__ __forceinline__ i32x4 bytes_end(int s, uint32_t shift, int n) const {
    i32x4 v = bytes(s, shift);
    if constexpr (SHIFT) {
#pragma unroll
      for (int u = 0; u < 4; ++u) v[u] &= (int)((1ull << (8 * min(max(n - 16 * s - 4 * u, 0), 4))) - 1);
    }
    return v;
  }
};
__device__ __forceinline__ uint32_t within_word(const int8_t* p) { return (uint32_t)reinterpret_cast<uintptr_t>(p) & 3; }

// A sum with its scales, rounded to a float: without the empty statement the last
// product and the rounding to 16 bits become one instruction in some kernels and not in
// others, and the same call has other bits where its operands begin elsewhere.
__device__ __forceinline__ float scaled(int sum, float row, float channel) {
  float v = (float)sum * row * channel;
  asm("" : "+v"(v));
  return v;
}

// Four neighbouring channels of a row.
template <typename T>
__device__ __forceinline__ void store4(T* p, const float (&v)[4], int n) {
  typedef T vec __attribute__((ext_vector_type(4)));
  typedef __attribute__((aligned(sizeof(T)))) vec at;
  if (n >= 4) {
    vec r;
#pragma unroll
    for (int u = 0; u < 4; ++u) r[u] = (T)v[u];
    *reinterpret_cast<at*>(p) = r;
  } else {
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (u < n) p[u] = (T)v[u];
  }
}

struct Work {
  const Tile* tiles;     // null: one run of all rows
  const int32_t* total;
};
__device__ __forceinline__ Tile tile_of(const Work& w, int32_t i, int64_t M, int32_t rows_of_tile) {
  if (w.tiles) {
    const Tile t = w.tiles[i];  // the same for all lanes
    return Tile{__builtin_amdgcn_readfirstlane(t.row), __builtin_amdgcn_readfirstlane(t.rows),
                __builtin_amdgcn_readfirstlane(t.expert), 0};
  }
  const int64_t row = (int64_t)i * rows_of_tile;
  return Tile{(int32_t)row, (int32_t)min((int64_t)rows_of_tile, M - row), 0, 0};
}

// Which tiles a block works on, and in which order.  Blocks go to the eight dies in
// turn; a die gets a contiguous part of the tiles, in groups of kGroup tiles of rows
// by all channels, so that what its blocks read at a time is near a square and is
// found in its L2 cache; in groups of one where each weight is read by one block, which
// goes through memory in order (64 rows of 64 runs, 4096 x 4096: 172 us, 178 in groups of
// four; 64 of 128, 2048 x 2048: 30 and 35).
constexpr int kStep = 128;  // bytes of the inner dimension that a step has
constexpr int kDies = 8, kGroup = 4, kUnits = 256;  // compute units
struct Walk {
  int64_t at, end, step;  // the block's part of the tiles by channels
  int32_t across, tiles, group;
  __device__ __forceinline__ Walk(const Work& w, int32_t most, int32_t N, int bn, int32_t of_group = kGroup)
      : group(of_group) {
    across = (N + bn - 1) / bn;
    tiles = w.tiles ? __builtin_amdgcn_readfirstlane(min(*w.total, most)) : most;
    const int64_t all = (int64_t)tiles * across, per = (all + kDies - 1) / kDies, die = blockIdx.x % kDies;
    at = die * per + blockIdx.x / kDies;
    end = min(die * per + per, all);
    step = gridDim.x / kDies;
  }
  __device__ __forceinline__ bool more() const { return at < end; }
  // The tile of rows and the tile of channels.
  __device__ __forceinline__ int32_t place(int32_t& channels) const {
    const int64_t which = at / (group * (int64_t)across);
    const int32_t in = (int32_t)(at - which * group * across), first = (int32_t)which * group;
    const int32_t rows = min(group, tiles - first);
    channels = in / rows;
    return first + in % rows;
  }
};

// 16 neighbouring channels of a row, of which the lane has 4 half .. + 3 and 8 + 4 half
// .. + 3 and the lane 32 further the others.  16-bit values change lanes first, so
// that a lane writes 16 bytes.
template <typename T>
__device__ __forceinline__ void store16(T* p, const float (&v)[2][4], int half, bool in) {
  if constexpr (sizeof(T) == 4) {
    if (!in) return;
    store4(p + 4 * half, v[0], 4);
    store4(p + 8 + 4 * half, v[1], 4);
  } else {
    typedef T two __attribute__((ext_vector_type(2)));
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((aligned(2))) u32x4 u32x4_at;
    u32x4 r;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const uint32_t x = __builtin_bit_cast(uint32_t, two{(T)v[0][2 * u], (T)v[0][2 * u + 1]});
      const uint32_t y = __builtin_bit_cast(uint32_t, two{(T)v[1][2 * u], (T)v[1][2 * u + 1]});
      const auto s = __builtin_amdgcn_permlane32_swap(x, y, false, false);
      r[u] = s[0];
      r[2 + u] = s[1];
    }
    if (in) *reinterpret_cast<u32x4_at*>(p + 8 * half) = r;
  }
}

// The scales of a lane's channels and rows, and its results with them: TN x TM blocks of
// 32 channels by 32 rows from channel n0 and row m0 of the tile.
template <typename T, int TN, int TM>
struct Results {
  f32x4 sn[TN][4];
  float sm[TM];
  bool whole;
  __device__ __forceinline__ void scales(const ProductArgs& p, const Tile& t, int32_t n0, int m0) {
    const int lane = threadIdx.x % kWave;
    const float* const sw = p.weight_scale + (int64_t)max(t.expert, 0) * p.N;
    whole = n0 + 32 * TN <= p.N;
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int32_t n = n0 + 32 * i + 8 * q + 4 * (lane / 32);
        if (t.expert < 0) {
          sn[i][q] = 0.f;
        } else if (whole) {
          sn[i][q] = *reinterpret_cast<const f32x4_at*>(sw + n);
        } else {
#pragma unroll
          for (int u = 0; u < 4; ++u) sn[i][q][u] = sw[min(n + u, p.N - 1)];
        }
      }
#pragma unroll
    for (int j = 0; j < TM; ++j)
      sm[j] = t.expert < 0 ? 0.f : p.scale[t.row + min(m0 + 32 * j + lane % 32, t.rows - 1)];
  }
  // Blocks of rows FROM .. TO - 1.
  template <int FROM = 0, int TO = TM>
  __device__ __forceinline__ void store(const ProductArgs& p, const Tile& t, int32_t n0, int m0,
                                        const i32x16 (&acc)[TN][TM]) const {
    const int lane = threadIdx.x % kWave;
#pragma unroll
    for (int j = FROM; j < TO; ++j) {
      const int m = m0 + 32 * j + lane % 32;
      T* const to = static_cast<T*>(p.out) + (int64_t)(t.row + m) * p.N;
#pragma unroll
      for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int q = 0; q < 4; q += 2) {
          float v[2][4];
#pragma unroll
          for (int u = 0; u < 8; ++u) v[u / 4][u % 4] = scaled(acc[i][j][4 * q + u], sm[j], sn[i][q + u / 4][u % 4]);
          const int32_t n = n0 + 32 * i + 8 * q;
          if (whole) {
            store16(to + n, v, lane / 32, m < t.rows);
          } else if (m < t.rows) {
            const int32_t at = n + 4 * (lane / 32);
            if (at < p.N) store4(to + at, v[0], p.N - at);
            if (at + 8 < p.N) store4(to + at + 8, v[1], p.N - at - 8);
          }
        }
    }
  }
};

// 16-byte pieces of a row of LDS change places by half the row's number: 16 lanes are
// served at a time out of 64 banks, which two rows of a step fill (by the row's own
// number half of all cycles of the reads are conflicts: 32768 x 4096 x 1024 178 us, 165
// so).
__device__ __forceinline__ int turn_of(int row) { return row / 2 % (kStep / 16); }

// BN channels by BM rows of a tile, by WN x WM waves; kStep bytes of the inner
// dimension at a time, those of the next AHEAD steps on their way in registers while
// the present ones are worked on out of LDS.
template <typename T, int BN, int BM, int WN, int WM, int AHEAD, bool SHIFT>
__global__ void __launch_bounds__(kWave * WN * WM) __attribute__((amdgpu_waves_per_eu(AHEAD > 1 ? 3 : 2)))
product_kernel(ProductArgs p, Work work, int32_t most) {
  constexpr int kThreads = kWave * WN * WM, TN = BN / WN / 32, TM = BM / WM / 32, kPieces = kStep / 16;
  constexpr int LN = BN * kPieces / kThreads, LM = BM * kPieces / kThreads;
  extern __shared__ i32x4 room[];
  const int tid = threadIdx.x, lane = tid % kWave, wid = tid / kWave;
  const int wn = wid % WN * (BN / WN), wm = wid / WN * (BM / WM);
  for (Walk walk(work, most, p.N, BN); walk.more(); walk.at += walk.step) {
    int32_t channels;
    const Tile t = tile_of(work, walk.place(channels), p.M, BM);
    const int32_t n0 = channels * BN, K = t.expert < 0 ? 0 : p.K;
    const int8_t* const W = p.weight + (int64_t)max(t.expert, 0) * p.N * p.K;
    const int8_t *from_n[LN], *from_m[LM];
    int to_n[LN], to_m[LM];
    const int piece = tid % kPieces;
#pragma unroll
    for (int i = 0; i < LN; ++i) {
      const int r = tid / kPieces + i * (kThreads / kPieces);
      from_n[i] = W + (int64_t)min(n0 + r, p.N - 1) * p.K;
      to_n[i] = r * kPieces + (piece ^ turn_of(r));
    }
#pragma unroll
    for (int i = 0; i < LM; ++i) {
      const int r = tid / kPieces + i * (kThreads / kPieces);
      from_m[i] = p.x + (int64_t)(t.row + min(r, t.rows - 1)) * p.K;
      to_m[i] = BN * kPieces + r * kPieces + (piece ^ turn_of(r));
    }
    Words<SHIFT, 1> next_n[AHEAD][LN], next_m[AHEAD][LM];
    auto fetch = [&](int32_t k, int s) {
      const int n = K - k - 16 * piece;
      if (n >= (SHIFT ? 20 : 16)) {
#pragma unroll
        for (int i = 0; i < LN; ++i) next_n[s][i].load(from_n[i] + k + 16 * piece, within_word(from_n[i]));
#pragma unroll
        for (int i = 0; i < LM; ++i) next_m[s][i].load(from_m[i] + k + 16 * piece, within_word(from_m[i]));
      } else {
#pragma unroll
        for (int i = 0; i < LN; ++i) next_n[s][i].load_end(from_n[i] + k + 16 * piece, within_word(from_n[i]), n);
#pragma unroll
        for (int i = 0; i < LM; ++i) next_m[s][i].load_end(from_m[i] + k + 16 * piece, within_word(from_m[i]), n);
      }
    };
    auto put = [&](int32_t k, i32x4* to, int s) {
      if (k + kStep <= K) {
#pragma unroll
        for (int i = 0; i < LN; ++i) to[to_n[i]] = next_n[s][i].bytes(0, within_word(from_n[i]));
#pragma unroll
        for (int i = 0; i < LM; ++i) to[to_m[i]] = next_m[s][i].bytes(0, within_word(from_m[i]));
      } else {
        const int n = K - k - 16 * piece;
#pragma unroll
        for (int i = 0; i < LN; ++i) to[to_n[i]] = next_n[s][i].bytes_end(0, within_word(from_n[i]), n);
#pragma unroll
        for (int i = 0; i < LM; ++i) to[to_m[i]] = next_m[s][i].bytes_end(0, within_word(from_m[i]), n);
      }
    };
#pragma unroll
    for (int s = 0; s < AHEAD; ++s) fetch(s * kStep, s);
    Results<T, TN, TM> results;
    if (AHEAD > 1) results.scales(p, t, n0 + wn, wm);
    i32x16 acc[TN][TM];
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
      for (int j = 0; j < TM; ++j) acc[i][j] = 0;
    put(0, room, 0);
    fetch(AHEAD * kStep, 0);
    __syncthreads();
    int buf = 0;
    for (int32_t k0 = 0; k0 < K; k0 += AHEAD * kStep) {
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const int32_t k = k0 + u * kStep;
        if (k >= K) break;
        const i32x4* const lds = room + buf * (BN + BM) * kPieces;
#pragma unroll
        for (int s = 0; s < kStep / 32; ++s) {
          i32x4 a[TN], b[TM];
          const int c = 2 * s + lane / 32;
#pragma unroll
          for (int i = 0; i < TN; ++i) {
            const int r = wn + 32 * i + lane % 32;
            a[i] = lds[r * kPieces + (c ^ turn_of(r))];
          }
#pragma unroll
          for (int j = 0; j < TM; ++j) {
            const int r = wm + 32 * j + lane % 32;
            b[j] = lds[BN * kPieces + r * kPieces + (c ^ turn_of(r))];
          }
#pragma unroll
          for (int i = 0; i < TN; ++i)
#pragma unroll
            for (int j = 0; j < TM; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(a[i], b[j], acc[i][j], 0, 0, 0);
        }
        buf ^= 1;
        if (k + kStep < K) {
          put(k + kStep, room + buf * (BN + BM) * kPieces, (u + 1) % AHEAD);
          fetch(k + (AHEAD + 1) * kStep, (u + 1) % AHEAD);
        }
        __syncthreads();
      }
    }
    if (AHEAD == 1) results.scales(p, t, n0 + wn, wm);  // many results: no registers for them before
    results.store(p, t, n0 + wn, wm, acc);
    __syncthreads();  // a run of no expert waits nowhere else
  }
}

// Many rows, whole 16-byte pieces: a wave on each SIMD holds 128 x 128 results (of
// smaller ones the reads of LDS would take as long as the products), and pieces go from
// memory to LDS without passing through registers.  The operands of the next 32 bytes
// are read out of LDS while the present ones are multiplied, and those of the next
// step's first 32 before the present step's last are.  A step's 16 loads and 32 reads
// lie between its 64 products, one or two at a time: a wave has its SIMD for itself, and
// what it issues in a row the matrix unit waits for (8192 x 4096 and 8192, zeros: 2.6 to
// 2.8 POP/s with all of them in a row, 3.6 to 4.1 so).
// 65536 rows of 32 runs, 4096 x 4096: 1060 to 1110 us by the card, 2.0 POP/s; 8192^3 2.3 to 2.5.  Bound by
// power: 8192^3 of zeros reaches 3.5, the clock falls from 2.4 to 1.75 GHz, and products
// alone, no loads and no reads, reach 3.0 to 3.3 of random values and 4.1 to 4.7 of zeros.
constexpr int kWideN = 256, kWideM = 256, kWideThreads = 256;
constexpr int kRawBuffer = 0x00027000;  // a buffer's description: untyped, checked by bytes
constexpr int kAllLoads = 0x0F70;       // waits for memory alone

typedef __attribute__((address_space(3))) void LdsPlace;
typedef __amdgpu_buffer_rsrc_t Buffer;

template <typename T>
__global__ void __launch_bounds__(kWideThreads) __attribute__((amdgpu_waves_per_eu(1, 1)))
product_wide_kernel(ProductArgs p, Work work, int32_t most) {
  constexpr int kPieces = kStep / 16, kWaves = kWideThreads / kWave, kLoads = (kWideN + kWideM) * kPieces / kWideThreads;
  __shared__ i32x4 even[(kWideN + kWideM) * kPieces], odd[(kWideN + kWideM) * kPieces];
  const int tid = threadIdx.x, lane = tid % kWave, wid = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int wn = wid % 2 * 128, wm = wid / 2 * 128;
  // where this lane's operands lie in a step's room
  int at_n[4], at_m[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    at_n[i] = (wn + 32 * i + lane % 32) * kPieces;
    at_m[i] = (kWideN + wm + 32 * i + lane % 32) * kPieces;
  }
  const int turn = turn_of(lane % 32);  // of the row's pieces
  auto bring = [&](Buffer rows_n, Buffer rows_m, uint32_t from, i32x4* to, int i) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(i < kLoads / 2 ? rows_n : rows_m,
                                             (LdsPlace*)(to + (i * kWaves + wid) * kWave), 16,
                                             from + (uint32_t)(i % (kLoads / 2) * kWaves * 8 * p.K), 0, 0, 0);
  };
  // A wave brings eight rows at a time, a lane the piece whose place is its own.  Rows and pieces behind the ends are
  // out of the buffers' ranges, and come as zeros.
  const int own = 16 * ((lane % kPieces) ^ turn_of(wid * 8 + lane / kPieces));
  const uint32_t first = (uint32_t)((wid * 8 + lane / kPieces) * p.K + own);
  auto offset = [&](int32_t k) { return k + own < p.K ? first + (uint32_t)k : 0x80000000u; };
  Walk walk(work, most, p.N, kWideN);
  if (!walk.more()) return;
  auto look = [&](int32_t& n0) {
    int32_t channels;
    const Tile t = tile_of(work, walk.place(channels), p.M, kWideM);
    n0 = channels * kWideN;
    return t;
  };
  auto buffer_n = [&](const Tile& t, int32_t n0) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t*>(p.weight) + ((int64_t)max(t.expert, 0) * p.N + n0) * p.K, 0,
                                             min(kWideN, p.N - n0) * p.K, kRawBuffer);
  };
  auto buffer_m = [&](const Tile& t) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t*>(p.x) + (int64_t)t.row * p.K, 0, t.rows * p.K, kRawBuffer);
  };
  auto begin = [&](Buffer rows_n, Buffer rows_m) {  // the first step's pieces, and half of the second's
#pragma unroll
    for (int i = 0; i < kLoads; ++i) bring(rows_n, rows_m, offset(0), even, i);
#pragma unroll
    for (int i = 0; i < kLoads / 2; ++i) bring(rows_n, rows_m, offset(kStep), odd, i);
  };
  int32_t n0;
  Tile t = look(n0);
  auto rows_n = buffer_n(t, n0), rows_m = buffer_m(t);
  begin(rows_n, rows_m);
  __builtin_amdgcn_s_waitcnt(kAllLoads);
  for (bool more = true; more;) {
    walk.at += walk.step;
    more = walk.more();
    int32_t next_n0 = n0;
    Tile next = t;
    if (more) next = look(next_n0);
    const int32_t K = t.expert < 0 ? 0 : p.K;
    i32x4 a[2][4], b[2][4];
    auto take = [&](const i32x4* lds, int s, int into, int i) {
      const int c = (2 * s + lane / 32) ^ turn;
      if (i % 2 == 0) b[into][i / 2] = lds[at_m[i / 2] + c];
      else a[into][i / 2] = lds[at_n[i / 2] + c];
    };
    i32x16 acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][j] = 0;
    // 16 products; `also` comes before each, so that what it starts runs beside them
    auto multiply = [&](int from, auto also) {
#pragma unroll
      for (int n = 0; n < 16; ++n) {
        also(n);
        acc[n / 4][n % 4] =
            __builtin_amdgcn_mfma_i32_32x32x32_i8(a[from][n / 4], b[from][n % 4], acc[n / 4][n % 4], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    auto step = [&](int32_t k, i32x4* here, i32x4* there) {
#pragma unroll
      for (int s = 0; s < 3; ++s)
        multiply(s % 2, [&](int n) {
          if (n < 8) take(here, s + 1, (s + 1) % 2, n);
          if (s == 0 && n % 2 == 1) bring(rows_n, rows_m, offset(k + kStep), there, kLoads / 2 + n / 2);
        });
      __builtin_amdgcn_s_waitcnt(kAllLoads);
      __syncthreads();  // the next step's pieces are there, and nothing reads this one's any more
      multiply(1, [&](int n) {
        if (n < 8) take(there, 0, 0, n);
        if (n % 2 == 1) bring(rows_n, rows_m, offset(k + 2 * kStep), here, n / 2);
      });
    };
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) take(even, 0, 0, i);
    int32_t k = 0;
    for (; k + kStep < K; k += 2 * kStep) {
      step(k, even, odd);
      step(k + kStep, odd, even);
    }
    if (k < K) step(k, even, odd);
    // What was brought last is of no use, but on its way.  No wave reads LDS any more (but for operands that it does
    // not use), so the next tile's first pieces come while this one's results go.
    Results<T, 4, 4> results;
    results.scales(p, t, n0 + wn, wm);
    __builtin_amdgcn_s_waitcnt(kAllLoads);
    const auto next_rows_n = buffer_n(next, next_n0), next_rows_m = buffer_m(next);
    if (more) begin(next_rows_n, next_rows_m);
    results.template store<0, 3>(p, t, n0 + wn, wm, acc);
    __builtin_amdgcn_s_waitcnt(kAllLoads);  // the pieces are there, and the last results are not waited for
    results.template store<3, 4>(p, t, n0 + wn, wm, acc);
    t = next;
    n0 = next_n0;
    rows_n = next_rows_n;
    rows_m = next_rows_m;
  }
}

// The same for tiles of 128 by 128, where those of 256 are too few for the chip: a wave
// holds 64 x 64 results, and as a step is over in a quarter of the time, four of them are
// on their way.  The barrier waits for the step that is next alone.  512 rows, 8192 x 8192:
// 37 us, 1.85 POP/s (58 by tiles of 64 by 128 through registers, 76 by those of 256); 128
// rows, 4096 x 4096: 14.  A step's 16 reads of 1 KB by each of four waves, and its pieces,
// keep LDS busy for longer than the matrix units (768 and 512 cycles), and 64 steps of
// 8192 take 23 us however few the rows.
constexpr int kHalfTile = 128, kHalfThreads = 256;
constexpr int kAllButTwo = 0x4070;  // waits for LDS, and for memory but for the last 16 loads

template <typename T>
__global__ void __launch_bounds__(kHalfThreads) __attribute__((amdgpu_waves_per_eu(1, 1)))
product_half_kernel(ProductArgs p, Work work, int32_t most) {
  constexpr int kPieces = kStep / 16, kWaves = kHalfThreads / kWave, kRoom = 2 * kHalfTile * kPieces;
  constexpr int kLoads = kRoom / kHalfThreads;
  static_assert(2 * kLoads == 16, "kAllButTwo counts two steps' loads");
  __shared__ i32x4 room0[kRoom], room1[kRoom], room2[kRoom], room3[kRoom];
  const int tid = threadIdx.x, lane = tid % kWave, wid = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int wn = wid % 2 * 64, wm = wid / 2 * 64, turn = turn_of(lane % 32);
  int at_n[2], at_m[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    at_n[i] = (wn + 32 * i + lane % 32) * kPieces;
    at_m[i] = (kHalfTile + wm + 32 * i + lane % 32) * kPieces;
  }
  const int own = 16 * ((lane % kPieces) ^ turn_of(wid * 8 + lane / kPieces));
  const uint32_t first = (uint32_t)((wid * 8 + lane / kPieces) * p.K + own);
  for (Walk walk(work, most, p.N, kHalfTile); walk.more(); walk.at += walk.step) {
    int32_t channels;
    const Tile t = tile_of(work, walk.place(channels), p.M, kHalfTile);
    const int32_t n0 = channels * kHalfTile, K = t.expert < 0 ? 0 : p.K;
    const Buffer rows_n = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<int8_t*>(p.weight) + ((int64_t)max(t.expert, 0) * p.N + n0) * p.K, 0, min(kHalfTile, p.N - n0) * p.K,
        kRawBuffer);
    const Buffer rows_m =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t*>(p.x) + (int64_t)t.row * p.K, 0, t.rows * p.K, kRawBuffer);
    auto bring = [&](int32_t k, i32x4* to, int i) {
      const uint32_t from = k + own < p.K ? first + (uint32_t)k : 0x80000000u;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(i < kLoads / 2 ? rows_n : rows_m,
                                               (LdsPlace*)(to + (i * kWaves + wid) * kWave), 16,
                                               from + (uint32_t)(i % (kLoads / 2) * kWaves * 8 * p.K), 0, 0, 0);
    };
#pragma unroll
    for (int i = 0; i < kLoads; ++i) bring(0, room0, i);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) bring(kStep, room1, i);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) bring(2 * kStep, room2, i);
    i32x4 a[2][2], b[2][2];
    auto take = [&](const i32x4* lds, int s, int into, int i) {
      const int c = (2 * s + lane / 32) ^ turn;
      if (i % 2 == 0) b[into][i / 2] = lds[at_m[i / 2] + c];
      else a[into][i / 2] = lds[at_n[i / 2] + c];
    };
    i32x16 acc[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) acc[i][j] = 0;
    auto multiply = [&](int from, auto also) {
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        also(n);
        acc[n / 2][n % 2] =
            __builtin_amdgcn_mfma_i32_32x32x32_i8(a[from][n / 2], b[from][n % 2], acc[n / 2][n % 2], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    // The next step's pieces are there for all waves, and nothing reads this one's any more: __syncthreads would
    // wait for all loads.
    auto meet = [] {
      __atomic_signal_fence(__ATOMIC_SEQ_CST);
      __builtin_amdgcn_s_waitcnt(kAllButTwo);
      __builtin_amdgcn_s_barrier();
      __atomic_signal_fence(__ATOMIC_SEQ_CST);
    };
    // `free`: the room of the step before, which all waves have read
    auto step = [&](int32_t k, i32x4* here, i32x4* there, i32x4* free) {
#pragma unroll
      for (int s = 0; s < 3; ++s)
        multiply(s % 2, [&](int n) {
          take(here, s + 1, (s + 1) % 2, n);
          if (s < 2) bring(k + 3 * kStep, free, 4 * s + n);
        });
      meet();
      multiply(1, [&](int n) { take(there, 0, 0, n); });
    };
    meet();
#pragma unroll
    for (int i = 0; i < 4; ++i) take(room0, 0, 0, i);
    int32_t k = 0;
    for (; k + 3 * kStep < K; k += 4 * kStep) {
      step(k, room0, room1, room3);
      step(k + kStep, room1, room2, room0);
      step(k + 2 * kStep, room2, room3, room1);
      step(k + 3 * kStep, room3, room0, room2);
    }
    if (k < K) step(k, room0, room1, room3);
    if (k + kStep < K) step(k + kStep, room1, room2, room0);
    if (k + 2 * kStep < K) step(k + 2 * kStep, room2, room3, room1);
    Results<T, 2, 2> results;
    results.scales(p, t, n0 + wn, wm);
    results.store(p, t, n0 + wn, wm, acc);
    __builtin_amdgcn_s_waitcnt(kAllLoads);  // what was brought last is of no use, but on its way
    __syncthreads();
  }
}

// A few rows of each run: tiles of 16 rows by 16 channels, whose four waves share the
// inner dimension.  A lane reads 32 neighbouring bytes of its row, a wave whole lines.
// Bound by memory where the weights are many (64 rows of 64 runs, 4096 x 4096: 172 us for
// 1.07 GB, 6.2 TB/s), by the blocks' own chains of loads where they are few (64 rows over
// 31 of 128 runs, 2048 x 2048: 26 us for 130 MB, and the list of tiles).
constexpr int kFewRows = 16, kFewN = 16, kFewWaves = 4, kFewAhead = 2;
template <typename T, bool SHIFT>
__global__ void __launch_bounds__(kWave * kFewWaves)
product_few_kernel(ProductArgs p, Work work, int32_t most) {
  __shared__ i32x4 part[2][kFewWaves][kWave];
  const int lane = threadIdx.x % kWave, wid = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  int slot = 0;
  for (Walk walk(work, most, p.N, kFewN, 1); walk.more(); walk.at += walk.step, slot ^= 1) {
    int32_t channels;
    const Tile t = tile_of(work, walk.place(channels), p.M, kFewRows);
    const int32_t n0 = channels * kFewN, n = n0 + lane / 16 * 4, K = t.expert < 0 ? 0 : p.K;
    const int m = min(lane % 16, t.rows - 1);
    const int8_t* const w = p.weight + ((int64_t)max(t.expert, 0) * p.N + min(n0 + lane % 16, p.N - 1)) * p.K;
    const int8_t* const x = p.x + (int64_t)(t.row + m) * p.K;
    const uint32_t shift_w = within_word(w), shift_x = within_word(x);
    constexpr int32_t kAll = kStep * kFewWaves, kNeeds = kStep + (SHIFT ? 4 : 0);
    const int32_t mine = lane / 16 * 32;
    i32x4 acc = 0;
    Words<SHIFT, 2> a[kFewAhead], b[kFewAhead];
    auto fetch = [&](int32_t k, int u) {
      if (k + kNeeds > K) return;
      a[u].load(w + k + mine, shift_w);
      b[u].load(x + k + mine, shift_x);
    };
    int32_t k = wid * kStep;
#pragma unroll
    for (int u = 0; u < kFewAhead; ++u) fetch(k + u * kAll, u);
    float sx = 0.f, sn[4] = {};
    if (wid == 0 && t.expert >= 0) {
      sx = p.scale[t.row + m];
#pragma unroll
      for (int u = 0; u < 4; ++u) sn[u] = p.weight_scale[(int64_t)t.expert * p.N + min(n + u, p.N - 1)];
    }
    while (k + kNeeds <= K) {
#pragma unroll
      for (int u = 0; u < kFewAhead; ++u) {
        if (k + kNeeds > K) break;
#pragma unroll
        for (int s = 0; s < 2; ++s)
          acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[u].bytes(s, shift_w), b[u].bytes(s, shift_x), acc, 0, 0, 0);
        fetch(k + kFewAhead * kAll, u);
        k += kAll;
      }
    }
    if (k < K) {  // the row's end: of one wave, or of two where words are shifted and it is 1 to 3 bytes
      const int left = K - k - mine;
      a[0].load_end(w + k + mine, shift_w, left);
      b[0].load_end(x + k + mine, shift_x, left);
#pragma unroll
      for (int s = 0; s < 2; ++s)
        acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[0].bytes_end(s, shift_w, left), b[0].bytes_end(s, shift_x, left), acc, 0, 0, 0);
    }
    part[slot][wid][lane] = acc;
    __syncthreads();  // the two sets of sums take turns
    if (wid == 0 && lane % 16 < t.rows && n < p.N) {
#pragma unroll
      for (int i = 1; i < kFewWaves; ++i) acc += part[slot][i][lane];
      float v[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) v[u] = scaled(acc[u], sx, sn[u]);
      store4(static_cast<T*>(p.out) + (int64_t)(t.row + m) * p.N + n, v, p.N - n);
    }
  }
}

// Fewer rows than fill the matrix units: all that counts is the weights' way from
// memory.  A block has 32 channels and up to 32 TM rows, and its waves share the inner
// dimension: operands go from memory to registers, the next step's while the present
// one's are multiplied, and meet as sums in LDS, which are whole numbers and have no
// order.  A lane reads 64 neighbouring bytes of its row, a wave whole lines of 128 of
// each; which bytes meet in a product is the same for both operands.  Blocks of 32 rows
// that a tile does not have are left out.  32 rows, 8192 x 8192: 19 us, 3.6 TB/s (39 by tiles
// of 64 by 128 that go through LDS, of which there are too few for the chip).
constexpr int kSomeN = 32, kSomeWaves = 8, kSomeThreads = kSomeWaves * kWave;

template <typename T, int TM, bool SHIFT>
__global__ void __launch_bounds__(kSomeThreads)
product_some_kernel(ProductArgs p, Work work, int32_t most) {
  constexpr int kRows = 32 * TM, kPitch = kRows + 1, kTasks = kRows * kSomeN / 4, kMine = (kTasks + kSomeThreads - 1) / kSomeThreads;
  __shared__ int sum[kSomeN * kPitch];
  const int tid = threadIdx.x, lane = tid % kWave, wid = __builtin_amdgcn_readfirstlane(tid / kWave);
  for (Walk walk(work, most, p.N, kSomeN); walk.more(); walk.at += walk.step) {
    int32_t channels;
    const Tile t = tile_of(work, walk.place(channels), p.M, kRows);
    const int32_t n0 = channels * kSomeN, K = t.expert < 0 ? 0 : p.K;
    const int8_t* const w = p.weight + ((int64_t)max(t.expert, 0) * p.N + min(n0 + lane % 32, p.N - 1)) * p.K;
    const int8_t* x[TM];
#pragma unroll
    for (int j = 0; j < TM; ++j) x[j] = p.x + (int64_t)(t.row + min(32 * j + lane % 32, t.rows - 1)) * p.K;
    const int32_t mine = 64 * (lane / 32);
    const uint32_t shift_w = within_word(w);
    uint32_t shift_x[TM];
#pragma unroll
    for (int j = 0; j < TM; ++j) shift_x[j] = within_word(x[j]);
    Words<SHIFT, 4> a, b[TM], next_a, next_b[TM];
    auto fetch = [&](int32_t k, Words<SHIFT, 4>& to_a, Words<SHIFT, 4>(&to_b)[TM]) {
      to_a.load(w + k + mine, shift_w);
#pragma unroll
      for (int j = 0; j < TM; ++j)
        if (32 * j < t.rows) to_b[j].load(x[j] + k + mine, shift_x[j]);
    };
    constexpr int32_t kAll = kStep * kSomeWaves, kNeeds = kStep + (SHIFT ? 4 : 0);
    int32_t k = wid * kStep;
    if (k + kNeeds <= K) fetch(k, a, b);
    // the results that this thread gives: four channels of a row each
    const int32_t n = n0 + tid % 8 * 4;
    float sx[kMine], sn[4];
#pragma unroll
    for (int u = 0; u < 4; ++u)
      sn[u] = t.expert < 0 ? 0.f : p.weight_scale[(int64_t)t.expert * p.N + min(n + u, p.N - 1)];
#pragma unroll
    for (int i = 0; i < kMine; ++i)
      sx[i] = t.expert < 0 ? 0.f : p.scale[t.row + min((tid + i * kSomeThreads) / 8, t.rows - 1)];
    for (int i = tid; i < kSomeN * kPitch; i += kSomeThreads) sum[i] = 0;
    i32x16 acc[TM];
#pragma unroll
    for (int j = 0; j < TM; ++j) acc[j] = 0;
    __syncthreads();
    for (; k + kNeeds <= K; k += kAll) {
      if (k + kAll + kNeeds <= K) fetch(k + kAll, next_a, next_b);
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const i32x4 ws = a.bytes(s, shift_w);
#pragma unroll
        for (int j = 0; j < TM; ++j)
          if (32 * j < t.rows)
            acc[j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(ws, b[j].bytes(s, shift_x[j]), acc[j], 0, 0, 0);
      }
      a = next_a;
#pragma unroll
      for (int j = 0; j < TM; ++j) b[j] = next_b[j];
    }
    if (k < K) {  // the row's end: of one wave, or of two where words are shifted and it is 1 to 3 bytes
      const int left = K - k - mine;
      a.load_end(w + k + mine, shift_w, left);
#pragma unroll
      for (int j = 0; j < TM; ++j)
        if (32 * j < t.rows) {
          b[j].load_end(x[j] + k + mine, shift_x[j], left);
#pragma unroll
          for (int s = 0; s < 4; ++s)
            acc[j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(a.bytes_end(s, shift_w, left), b[j].bytes_end(s, shift_x[j], left),
                                                           acc[j], 0, 0, 0);
        }
    }
#pragma unroll
    for (int j = 0; j < TM; ++j)
      if (32 * j < t.rows)
#pragma unroll
        for (int q = 0; q < 16; ++q) {
          const int c = 8 * (q / 4) + 4 * (lane / 32) + q % 4;
          __hip_atomic_fetch_add(&sum[c * kPitch + 32 * j + lane % 32], acc[j][q], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
        }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      const int m = (tid + i * kSomeThreads) / 8;
      if (m >= t.rows || n >= p.N) continue;
      float v[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) v[u] = scaled(sum[(tid % 8 * 4 + u) * kPitch + m], sx[i], sn[u]);
      store4(static_cast<T*>(p.out) + (int64_t)(t.row + m) * p.N + n, v, p.N - n);
    }
    __syncthreads();
  }
}

// Which kernel, by how many rows a run has on average and how many tiles there are.  Us by
// few, some, middle, half and wide (rows in all, runs; K = N):
//   16    1 8192  17.0 16.1  38  23  67      32  1 8192    31 18.6  39 23.4  67      64 1 8192   59 25.9  39 23.7  67
//   64    1 4096  17.6 14.4  21 13.9 37     128  1 4096    32 15.1  22 14.2  37     512 1 8192  190 189.7  58 37  76
//   1024  1 8192   -   376  118  73  87    1536  1 8192   1334 562 167 107   98    2048 1 4096   -  213   60 43.9  52
//   3000  1 4096  659  314   83  64  56    4096  1 4096   894  417 113  85   65    256  8 4096   73  55   29 27.5  46
//   512   8 4096  137   86   37  29  47    2048  8 4096    -   248  73  62   58    1024 32 2048  75  63   27  31   35
//   2000 30 4096   -   334  121 120 133    4096 30 2048    -   161  44  46   39    6000 64 2048 365 260   80  84   83
//   8192 64 2048   -   333   99 103  90   16384 64 2048   932  579 163 147  121    25180 8 5120 x 256 - 234  85  69  76
// Rows that do not begin at multiples of 16 bytes have no half, and their 256 by 256 go
// through registers.
// The average is all that the host knows: the runs' own lengths live on the GPU, and rows of
// no run count too.  Where one run has nearly all rows and the average says few, its weight is
// read for each 16 of them (us, even split; one run has all but a row a run; one has all, the
// others none; a product of one weight): 4096 rows of 256 runs, 2048 x 2048 260 449 241 25;
// 1024 of 64, 4096 x 4096 255 443 232 22.  From 48 rows a run on: 4096 of 64, 2048 x 2048
// 61 82 - 26, 8192 of 64 85 - 40 36, 16384 of 64 100 136; and where all but a 32nd of the rows
// are of no run, 16384 of 64 take 130, 32768 191 (even 176).
enum Kind { kFew, kSome, kMiddle, kHalf, kLarge };
Kind kind_of(int64_t M, int32_t N, int32_t runs, bool pieces) {
  const int64_t sets = runs > 0 ? runs : 1, each = M / sets;
  auto tiles = [&](int rows, int channels) { return (M / rows + sets) * ((N + channels - 1) / channels); };
  if (each <= kFewRows) return kFew;
  if (pieces && each >= 48) return each >= 96 && tiles(256, 256) >= 176 ? kLarge : kHalf;
  if (!pieces && each >= 64 && tiles(256, 256) >= 96) return kLarge;
  return tiles(64, 128) <= 128 ? kSome : kMiddle;
}
int32_t rows_of(Kind k) { return k == kFew ? kFewRows : k == kSome ? 64 : k == kMiddle ? 64 : k == kHalf ? kHalfTile : 256; }

// Tiles of all runs, at most.
int64_t most_tiles(int64_t M, int32_t runs, bool listed, int32_t rows) {
  const int64_t full = (M + rows - 1) / rows, also = (int64_t)runs + 2 < M ? (int64_t)runs + 2 : M;
  return listed ? full + also : full;
}

template <typename T>
taot_status product(const ProductArgs& p, void* ws, hipStream_t stream) {
  const bool pieces =
      p.K % 16 == 0 && reinterpret_cast<uintptr_t>(p.x) % 16 == 0 && reinterpret_cast<uintptr_t>(p.weight) % 16 == 0;
  const Kind kind = kind_of(p.M, p.N, p.runs, pieces);
  const int32_t rows = rows_of(kind);
  const int64_t most = most_tiles(p.M, p.runs, p.offsets, rows);
  Work work{nullptr, nullptr};
  if (p.offsets) {
    Carver c{static_cast<char*>(ws)};
    int32_t* total = c.take<int32_t>(1);
    Tile* tiles = c.take<Tile>((size_t)most);
    // a block of 256 starts and ends sooner
    auto* kernel = p.runs + 2 <= 256 ? runs_kernel<256> : runs_kernel<1024>;
    kernel<<<1, p.runs + 2 <= 256 ? 256 : 1024, 0, stream>>>(p.offsets, p.experts, p.runs, p.G, p.M, rows, tiles, total);
    work = Work{tiles, total};
  }
  auto go = [&](auto* kernel, int bn, int threads, size_t lds, int64_t most_blocks = kMaxBlocks) {
    if (!allow_lds(reinterpret_cast<const void*>(kernel), lds)) return false;
    const int64_t blocks = round_up(most * ((p.N + bn - 1) / bn), kDies);
    kernel<<<(unsigned)(blocks < most_blocks ? blocks : most_blocks), threads, lds, stream>>>(p, work, (int32_t)most);
    return true;
  };
  bool ok;
  const bool words = (p.K | (int32_t)reinterpret_cast<uintptr_t>(p.x) | (int32_t)reinterpret_cast<uintptr_t>(p.weight)) % 4 == 0;
  if (kind == kFew)
    ok = go(words ? product_few_kernel<T, false> : product_few_kernel<T, true>, kFewN, kWave * kFewWaves, 0);
  else if (kind == kSome)
    ok = go(words ? product_some_kernel<T, 2, false> : product_some_kernel<T, 2, true>, kSomeN, kSomeThreads, 0);
  else if (kind == kMiddle)
    ok = go(words ? product_kernel<T, 128, 64, 2, 2, 2, false> : product_kernel<T, 128, 64, 2, 2, 2, true>, 128, 256, 2 * (128 + 64) * kStep);
  else if (kind == kHalf) ok = go(product_half_kernel<T>, kHalfTile, kHalfThreads, 0);
  else if (pieces)
    ok = go(product_wide_kernel<T>, kWideN, kWideThreads, 0, kUnits);
  else ok = go(words ? product_kernel<T, 256, 256, 2, 4, 1, false> : product_kernel<T, 256, 256, 2, 4, 1, true>, 256, 512, 2 * (256 + 256) * kStep);
  return ok && hipGetLastError() == hipSuccess ? TAOT_OK : TAOT_ERR_LAUNCH;
}

}  // namespace

size_t matmul_i8_ws(int64_t M, int32_t runs) {
  Carver c{nullptr};
  c.take<int32_t>(1);
  c.take<Tile>((size_t)most_tiles(M, runs, true, rows_of(kFew)));  // the smallest tiles: the number of channels is not known
  return c.off;
}

taot_status launch_matmul_i8(const ProductArgs& p, int32_t dtype, void* ws, hipStream_t stream) {
  return dtype == TAOT_BF16 ? product<__bf16>(p, ws, stream) : dtype == TAOT_F16 ? product<_Float16>(p, ws, stream)
                                                                                : product<float>(p, ws, stream);
}

}  // namespace taot
