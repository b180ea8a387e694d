// Products of 8-bit integers with a scale for each row and each channel, over runs
// of rows that have a weight each: the experts of a mixture on the rows sent to them.
//
//   out[t][n] = scale[t] weight_scale[e][n] sum_k x[t][k] weight[e][n][k]
//
// The sum is of whole numbers and exact in 32 bits (K up to TAOT_MAX_INNER); it is
// rounded to a float, multiplied by the two scales and rounded once to the output's
// type.  The order of the sum does not matter, so waves and blocks may share it.
//
// runs_kernel lists the tiles of rows: a tile lies within one run.  The weights are
// the matrix unit's first operand, so a lane's results are neighbouring channels.
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
constexpr int kRunThreads = 1024;
__global__ void __launch_bounds__(kRunThreads)
runs_kernel(const int32_t* __restrict__ offsets, const int32_t* __restrict__ experts, int32_t runs, int32_t G, int64_t M,
            int32_t rows_of_tile, Tile* __restrict__ tiles, int32_t* __restrict__ total) {
  __shared__ int32_t starts[kRunThreads + 1], firsts[kRunThreads + 1], part[16], whose[kRunThreads];
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

// Bytes k .. k + 15 of a row of K, zeros behind its end.
__device__ __forceinline__ i32x4 bytes16(const int8_t* __restrict__ row, int32_t k, int32_t K) {
  const int n = K - k;
  if (n >= 16) return *reinterpret_cast<const i32x4_at*>(row + k);
  i32x4 v = 0;
#pragma unroll
  for (int u = 0; u < 16; ++u)
    if (u < n) v[u / 4] |= (int)((uint32_t)(uint8_t)row[k + u] << (8 * (u % 4)));
  return v;
}

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
// found in its L2 cache.
constexpr int kDies = 8, kGroup = 4, kUnits = 256;  // compute units
struct Walk {
  int64_t all, at, end, step;  // all tiles by channels, and the block's part of them
  int32_t across, tiles;
  __device__ __forceinline__ Walk(const Work& w, int32_t most, int32_t N, int bn) {
    across = (N + bn - 1) / bn;
    tiles = w.tiles ? __builtin_amdgcn_readfirstlane(min(*w.total, most)) : most;
    all = (int64_t)tiles * across;
    const int64_t per = (all + kDies - 1) / kDies, die = blockIdx.x % kDies;
    at = die * per + blockIdx.x / kDies;
    end = min(die * per + per, all);
    step = gridDim.x / kDies;
  }
  __device__ __forceinline__ bool more() const { return at < end; }
  // The tile of rows and the tile of channels.
  __device__ __forceinline__ int32_t place(int32_t& channels) const {
    const int64_t group = at / (kGroup * (int64_t)across);
    const int32_t in = (int32_t)(at - group * kGroup * across), first = (int32_t)group * kGroup;
    const int32_t rows = min(kGroup, tiles - first);
    channels = in / rows;
    return first + in % rows;
  }
};

// BN channels by BM rows of a tile, by WN x WM waves; kStep bytes of the inner
// dimension at a time, the next ones on their way in registers while the present
// ones are worked on out of LDS.  16-byte pieces of a row of LDS change places by
// the row's number, so that lanes of neighbouring rows read other banks.
constexpr int kStep = 128;
template <typename T, int BN, int BM, int WN, int WM>
__global__ void __launch_bounds__(kWave * WN * WM)
product_kernel(ProductArgs p, Work work, int32_t most) {
  constexpr int kThreads = kWave * WN * WM, TN = BN / WN / 32, TM = BM / WM / 32, kPieces = kStep / 16;
  constexpr int LN = BN * kPieces / kThreads, LM = BM * kPieces / kThreads;
  extern __shared__ i32x4 room[];
  const int tid = threadIdx.x, lane = tid % kWave, wid = tid / kWave;
  const int wn = wid % WN * (BN / WN), wm = wid / WN * (BM / WM);
  T* const out = static_cast<T*>(p.out);
  for (Walk walk(work, most, p.N, BN); walk.more(); walk.at += walk.step) {
    int32_t channels;
    const Tile t = tile_of(work, walk.place(channels), p.M, BM);
    const int32_t n0 = channels * BN;
    if (t.expert < 0) {
      const int32_t wide = min(BN, p.N - n0);
      for (int32_t i = tid; i < t.rows * BN; i += kThreads)
        if (i % BN < wide) out[(int64_t)(t.row + i / BN) * p.N + n0 + i % BN] = (T)0.f;
      continue;
    }
    const int8_t* const W = p.weight + (int64_t)t.expert * p.N * p.K;
    const int8_t *from_n[LN], *from_m[LM];
    int to_n[LN], to_m[LM];
    const int piece = tid % kPieces;
#pragma unroll
    for (int i = 0; i < LN; ++i) {
      const int r = tid / kPieces + i * (kThreads / kPieces);
      from_n[i] = W + (int64_t)min(n0 + r, p.N - 1) * p.K;
      to_n[i] = r * kPieces + (piece ^ (r % kPieces));
    }
#pragma unroll
    for (int i = 0; i < LM; ++i) {
      const int r = tid / kPieces + i * (kThreads / kPieces);
      from_m[i] = p.x + (int64_t)(t.row + min(r, t.rows - 1)) * p.K;
      to_m[i] = BN * kPieces + r * kPieces + (piece ^ (r % kPieces));
    }
    i32x4 next_n[LN], next_m[LM];
    auto fetch = [&](int32_t k) {
#pragma unroll
      for (int i = 0; i < LN; ++i) next_n[i] = bytes16(from_n[i], k + 16 * piece, p.K);
#pragma unroll
      for (int i = 0; i < LM; ++i) next_m[i] = bytes16(from_m[i], k + 16 * piece, p.K);
    };
    auto put = [&](i32x4* to) {
#pragma unroll
      for (int i = 0; i < LN; ++i) to[to_n[i]] = next_n[i];
#pragma unroll
      for (int i = 0; i < LM; ++i) to[to_m[i]] = next_m[i];
    };
    i32x16 acc[TN][TM];
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
      for (int j = 0; j < TM; ++j) acc[i][j] = 0;
    fetch(0);
    put(room);
    __syncthreads();
    int buf = 0;
    for (int32_t k = 0; k < p.K; k += kStep, buf ^= 1) {
      const i32x4* const lds = room + buf * (BN + BM) * kPieces;
      const bool more = k + kStep < p.K;
      if (more) fetch(k + kStep);
#pragma unroll
      for (int s = 0; s < kStep / 32; ++s) {
        i32x4 a[TN], b[TM];
        const int c = 2 * s + lane / 32;
#pragma unroll
        for (int i = 0; i < TN; ++i) {
          const int r = wn + 32 * i + lane % 32;
          a[i] = lds[r * kPieces + (c ^ (r % kPieces))];
        }
#pragma unroll
        for (int j = 0; j < TM; ++j) {
          const int r = wm + 32 * j + lane % 32;
          b[j] = lds[BN * kPieces + r * kPieces + (c ^ (r % kPieces))];
        }
#pragma unroll
        for (int i = 0; i < TN; ++i)
#pragma unroll
          for (int j = 0; j < TM; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(a[i], b[j], acc[i][j], 0, 0, 0);
      }
      if (more) put(room + (buf ^ 1) * (BN + BM) * kPieces);
      __syncthreads();
    }
    const float* const sw = p.weight_scale + (int64_t)t.expert * p.N;
#pragma unroll
    for (int j = 0; j < TM; ++j) {
      const int m = wm + 32 * j + lane % 32;
      if (m >= t.rows) continue;
      const float sx = p.scale[t.row + m];
      T* const to = out + (int64_t)(t.row + m) * p.N;
#pragma unroll
      for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int32_t n = n0 + wn + 32 * i + 8 * q + 4 * (lane / 32);
          if (n >= p.N) continue;
          float v[4];
#pragma unroll
          for (int u = 0; u < 4; ++u) v[u] = scaled(acc[i][j][4 * q + u], sx, sw[min(n + u, p.N - 1)]);
          store4(to + n, v, p.N - n);
        }
    }
  }
}

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

// Many rows, whole 16-byte pieces: a wave on each SIMD holds 128 x 128 results, and
// pieces go from memory to LDS without passing through registers.  The operands of
// the next 32 bytes are read out of LDS while the present ones are multiplied, and
// those of the next step's first 32 before the present step's last are.
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
  T* const out = static_cast<T*>(p.out);
  // where this lane's operands lie in a step's room
  int at_n[4], at_m[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    at_n[i] = (wn + 32 * i + lane % 32) * kPieces;
    at_m[i] = (kWideN + wm + 32 * i + lane % 32) * kPieces;
  }
  const int turn = lane % kPieces;  // of the row's pieces
  auto bring = [&](Buffer rows_n, Buffer rows_m, uint32_t from, i32x4* to, int i) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(i < kLoads / 2 ? rows_n : rows_m,
                                             (LdsPlace*)(to + (i * kWaves + wid) * kWave), 16,
                                             from + (uint32_t)(i % (kLoads / 2) * kWaves * 8 * p.K), 0, 0, 0);
  };
  // A wave brings eight rows at a time, a lane the piece whose place is its own.  Rows and pieces behind the ends are
  // out of the buffers' ranges, and come as zeros.
  const int own = 16 * ((lane % kPieces) ^ (lane / kPieces));
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
    const float* const sw = p.weight_scale + (int64_t)max(t.expert, 0) * p.N;
    const bool whole = n0 + kWideN <= p.N;
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
    __builtin_amdgcn_s_waitcnt(kAllLoads);
    const auto next_rows_n = buffer_n(next, next_n0), next_rows_m = buffer_m(next);
    if (more) begin(next_rows_n, next_rows_m);
    f32x4 sn[4][4];
    float sm[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int32_t n = n0 + wn + 32 * i + 8 * q + 4 * (lane / 32);
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
    for (int j = 0; j < 4; ++j)
      sm[j] = t.expert < 0 ? 0.f : p.scale[t.row + min(wm + 32 * j + lane % 32, t.rows - 1)];
    __builtin_amdgcn_s_waitcnt(kAllLoads);  // the next tile's pieces too, and not for the results that go now
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int m = wm + 32 * j + lane % 32;
      T* const to = out + (int64_t)(t.row + m) * p.N;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int q = 0; q < 4; q += 2) {
          float v[2][4];
#pragma unroll
          for (int u = 0; u < 8; ++u) v[u / 4][u % 4] = scaled(acc[i][j][4 * q + u], sm[j], sn[i][q + u / 4][u % 4]);
          const int32_t n = n0 + wn + 32 * i + 8 * q;
          if (whole) {
            store16(to + n, v, lane / 32, m < t.rows);
          } else if (m < t.rows) {
            const int32_t at = n + 4 * (lane / 32);
            if (at < p.N) store4(to + at, v[0], p.N - at);
            if (at + 8 < p.N) store4(to + at + 8, v[1], p.N - at - 8);
          }
        }
    }
    t = next;
    n0 = next_n0;
    rows_n = next_rows_n;
    rows_m = next_rows_m;
  }
}

// Few rows: all that counts is the weights' way from memory.  A block has 16
// channels and up to 16 rows, its waves share the inner dimension; nothing passes
// through LDS but the waves' sums.  A lane reads 32 neighbouring bytes of its row, a
// wave whole lines of 128; which bytes meet in a step is the same for both operands.
constexpr int kFewRows = 16, kFewWaves = 4, kFewAhead = 4;
template <typename T>
__global__ void __launch_bounds__(kWave * kFewWaves)
product_few_kernel(ProductArgs p, Work work, int32_t most) {
  __shared__ i32x4 part[kFewWaves][kWave];
  const int lane = threadIdx.x % kWave, wid = threadIdx.x / kWave;
  const int32_t across = (p.N + 15) / 16;
  const int64_t all = (int64_t)(work.tiles ? min(*work.total, most) : most) * across;
  T* const out = static_cast<T*>(p.out);
  for (int64_t at = blockIdx.x; at < all; at += gridDim.x) {
    const Tile t = tile_of(work, (int32_t)(at / across), p.M, kFewRows);
    const int32_t n0 = (int32_t)(at % across) * 16;
    i32x4 acc = 0;
    if (t.expert >= 0) {
      const int8_t* const w = p.weight + ((int64_t)t.expert * p.N + min(n0 + lane % 16, p.N - 1)) * p.K;
      const int8_t* const x = p.x + (int64_t)(t.row + min(lane % 16, t.rows - 1)) * p.K;
      int32_t k = wid * kStep;
      constexpr int32_t kAll = kStep * kFewWaves;
      const int32_t mine = lane / 16 * 32;
      for (; k + (kFewAhead - 1) * kAll + kStep <= p.K; k += kFewAhead * kAll) {
        i32x4 a[kFewAhead][2], b[kFewAhead][2];
#pragma unroll
        for (int u = 0; u < kFewAhead; ++u)
#pragma unroll
          for (int s = 0; s < 2; ++s) a[u][s] = *reinterpret_cast<const i32x4_at*>(w + k + u * kAll + mine + 16 * s);
#pragma unroll
        for (int u = 0; u < kFewAhead; ++u)
#pragma unroll
          for (int s = 0; s < 2; ++s) b[u][s] = *reinterpret_cast<const i32x4_at*>(x + k + u * kAll + mine + 16 * s);
#pragma unroll
        for (int u = 0; u < kFewAhead; ++u)
#pragma unroll
          for (int s = 0; s < 2; ++s) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[u][s], b[u][s], acc, 0, 0, 0);
      }
      for (; k < p.K; k += kAll)
#pragma unroll
        for (int s = 0; s < 2; ++s)
          acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(bytes16(w, k + mine + 16 * s, p.K), bytes16(x, k + mine + 16 * s, p.K),
                                                      acc, 0, 0, 0);
    }
    part[wid][lane] = acc;
    __syncthreads();
    const int m = lane % 16;
    if (wid == 0 && m < t.rows) {
#pragma unroll
      for (int w = 1; w < kFewWaves; ++w) acc += part[w][lane];
      const int32_t n = n0 + lane / 16 * 4;
      if (n < p.N) {
        const float sx = t.expert >= 0 ? p.scale[t.row + m] : 0.f;
        float v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u)
          v[u] = t.expert >= 0 ? scaled(acc[u], sx, p.weight_scale[(int64_t)t.expert * p.N + min(n + u, p.N - 1)]) : 0.f;
        store4(out + (int64_t)(t.row + m) * p.N + n, v, p.N - n);
      }
    }
    __syncthreads();
  }
}

// Rows of a tile, by how many a run has on average.
enum Kind { kFew, kMiddle, kLarge };
Kind kind_of(int64_t M, int32_t runs) {
  const int64_t each = M / (runs > 0 ? runs : 1);
  return each <= 16 ? kFew : each < 128 ? kMiddle : kLarge;
}
int32_t rows_of(Kind k) { return k == kFew ? kFewRows : k == kMiddle ? 64 : 256; }

// Tiles of all runs, at most.
int64_t most_tiles(int64_t M, int32_t runs, bool listed, int32_t rows) {
  const int64_t full = (M + rows - 1) / rows, also = (int64_t)runs + 2 < M ? (int64_t)runs + 2 : M;
  return listed ? full + also : full;
}

template <typename T>
taot_status product(const ProductArgs& p, void* ws, hipStream_t stream) {
  const Kind kind = kind_of(p.M, p.runs);
  const int32_t rows = rows_of(kind);
  const int64_t most = most_tiles(p.M, p.runs, p.offsets, rows);
  Work work{nullptr, nullptr};
  if (p.offsets) {
    Carver c{static_cast<char*>(ws)};
    int32_t* total = c.take<int32_t>(1);
    Tile* tiles = c.take<Tile>((size_t)most);
    runs_kernel<<<1, kRunThreads, 0, stream>>>(p.offsets, p.experts, p.runs, p.G, p.M, rows, tiles, total);
    work = Work{tiles, total};
  }
  auto go = [&](auto* kernel, int bn, int threads, size_t lds, int64_t most_blocks = kMaxBlocks) {
    if (!allow_lds(reinterpret_cast<const void*>(kernel), lds)) return false;
    const int64_t blocks = round_up(most * ((p.N + bn - 1) / bn), kDies);
    kernel<<<(unsigned)(blocks < most_blocks ? blocks : most_blocks), threads, lds, stream>>>(p, work, (int32_t)most);
    return true;
  };
  bool ok;
  if (kind == kFew) ok = go(product_few_kernel<T>, 16, kWave * kFewWaves, 0);
  else if (kind == kMiddle) ok = go(product_kernel<T, 128, 64, 2, 2>, 128, 256, 2 * (128 + 64) * kStep);
  else if (p.K % 16 == 0 && reinterpret_cast<uintptr_t>(p.x) % 16 == 0 && reinterpret_cast<uintptr_t>(p.weight) % 16 == 0)
    ok = go(product_wide_kernel<T>, kWideN, kWideThreads, 0, kUnits);
  else ok = go(product_kernel<T, 256, 256, 2, 4>, 256, 512, 2 * (256 + 256) * kStep);
  return ok && hipGetLastError() == hipSuccess ? TAOT_OK : TAOT_ERR_LAUNCH;
}

}  // namespace

size_t matmul_i8_ws(int64_t M, int32_t runs) {
  Carver c{nullptr};
  c.take<int32_t>(1);
  c.take<Tile>((size_t)most_tiles(M, runs, true, rows_of(kind_of(M, runs))));
  return c.off;
}

taot_status launch_matmul_i8(const ProductArgs& p, int32_t dtype, void* ws, hipStream_t stream) {
  return dtype == TAOT_BF16 ? product<__bf16>(p, ws, stream) : dtype == TAOT_F16 ? product<_Float16>(p, ws, stream)
                                                                                : product<float>(p, ws, stream);
}

}  // namespace taot
