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
//   count_kernel  (a wave per chunk of a row)  copies of each expert in the chunk;
//                 its first B + 1 blocks: slots of each expert, experts of each rank
//   bases_kernel  (16 threads per row and expert)  running sums over the chunks
//   tables_kernel (a block per row)  slots' shares, instance offsets, sends
//   place_kernel  (a wave per chunk)  occurrence by occurrence to a position
//   row_kernel    (a block per row)  all of these for a short row, in one launch
//   rows_kernel, combine_kernel, combine_backward_kernel  (one or four waves a token)
#include "rowio.h"

namespace taot {
namespace {

constexpr int kThreads = 256, kTableThreads = 1024;
constexpr int kUnroll = 4;
constexpr int32_t kChunkMin = 256, kChunkMax = 32768;
// 64 rows of 131072 ids, 256 experts: the kernels take 53 us in all; 53 with half as many waves, 58 with twice (more counts)
constexpr int64_t kWavesWanted = 4096;
// A row's tables are made in LDS up to this size, else in memory (1024 ranks: from 3 slots a rank).
constexpr size_t kTableLds = 32768;
// Waves keep their stretches in LDS beside the row's tables, as many waves a block as there is room for (8 rows of
// 131072, 1024 experts: 42 us, 48 with copies that look theirs up), unless a block would bring many words of tables for
// each of its ids (8 rows of 65536, 256 experts, 8192 slots, 16 words an id: 135 us, 117 without; 8 of 131072, 4096
// experts, 512 slots, 3 words: 92 and 137).
constexpr size_t kKeepLds = 163840;
constexpr int64_t kBroughtWords = 8;
// Rows up to this length are done by one block and in one launch (384 experts, 512 slots, calls from end to end: a row
// of 8192 24 us, 30 in four launches; 256 such rows 29 and 59; from there on a block takes 5 us more for 4096 ids more).
constexpr int64_t kRowIds = 8192;
constexpr size_t kRowLds = 65536;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((aligned(1))) u32x4 u32x4_at;

// Lanes of the wave (among `valid`) that hold the same key, of `bits` bits, as two halves.
struct Same {
  uint32_t lo, hi;
  __device__ __forceinline__ int below() const { return (int)__builtin_amdgcn_mbcnt_hi(hi, __builtin_amdgcn_mbcnt_lo(lo, 0)); }
  __device__ __forceinline__ int all() const { return __popc(lo) + __popc(hi); }
};
__device__ __forceinline__ void same_bit(Same& m, uint32_t key, int b) {
  const uint32_t s = (uint32_t)__builtin_amdgcn_sbfe((int32_t)key, b, 1);  // the bit, everywhere
  const uint64_t v = __ballot(s != 0);
  m.lo &= ~((uint32_t)v ^ s);
  m.hi &= ~((uint32_t)(v >> 32) ^ s);
}
template <int BITS>
__device__ __forceinline__ Same same_key(uint32_t key, uint64_t valid) {
  Same m{(uint32_t)valid, (uint32_t)(valid >> 32)};
#pragma unroll
  for (int b = 0; b < BITS; ++b) same_bit(m, key, b);
  return m;
}

// Number of bits that hold 0 .. n.
__host__ __device__ inline int bits_for(uint32_t n) {
  int b = 0;
  while (n >> b) ++b;
  return b;
}

// Exclusive sum over a block of NT threads; *total gets the block's.
template <int NT, typename V>
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
  for (int w = 0; w < NT / kWave; ++w) {
    off += w < wid ? part[w] : (V)0;
    all += part[w];
  }
  *total = all;
  return off;
}

// Stable order of n keys in [0, nkeys], in three steps: their counts, running
// sums of those (first[q] = keys below q, q <= nkeys), and positions, by one wave:
// put(i, its key, position) for keys up to `last`.  cnt: nkeys + 1 words of LDS.
template <int NT, typename Key>
__device__ __forceinline__ void order_counts(int32_t n, Key key, int32_t* cnt) {
  for (int32_t i = threadIdx.x; i < n; i += NT) atomicAdd(&cnt[key(i)], 1);
}

template <int NT>
__device__ __forceinline__ void order_sums(int32_t nkeys, int32_t* first, int32_t* cnt, int32_t* part) {
  int32_t run = 0;
  for (int32_t q0 = 0; q0 <= nkeys; q0 += NT) {
    const int32_t q = q0 + threadIdx.x;
    int32_t total;
    const int32_t mine = q <= nkeys ? cnt[q] : 0;
    const int32_t at = run + block_exclusive<NT>(mine, part, &total);
    if (q <= nkeys) {
      cnt[q] = at;
      first[q] = at;
    }
    run += total;
  }
}

// last < 2^BITS
template <int BITS, typename Key, typename Put>
__device__ __forceinline__ void order_positions(int32_t n, int32_t last, Key key, Put put, int32_t* cnt) {
  const int lane = threadIdx.x & (kWave - 1);
  int32_t next = key(min(lane, n - 1));
  for (int32_t i0 = 0; i0 < n; i0 += kWave) {
    const int32_t i = i0 + lane, q = next;
    const bool in = (i < n) & (q <= last);
    next = key(min(i + kWave, n - 1));
    const Same m = same_key<BITS>((uint32_t)q, __ballot(in));
    const int before = m.below();
    const int32_t at = cnt[min(q, last)] + before;
    if (in) put(i, q, at);
    __builtin_amdgcn_wave_barrier();
    if (in & (before + 1 == m.all())) cnt[q] = at + 1;  // the last lane of the key
    __builtin_amdgcn_wave_barrier();
  }
}

constexpr int kRankBits = 12;  // holds 0 .. TAOT_MAX_RANKS
static_assert(TAOT_MAX_RANKS < 1 << kRankBits, "bits of a rank");
constexpr int kExpertBits = 15;
static_assert(TAOT_MAX_EXPERTS <= 1 << kExpertBits, "bits of an expert");

// Ranks of experts (R: none) and experts of slots (E: none).
struct HomeKey {
  const int32_t* home;
  int32_t R;
  __device__ __forceinline__ int32_t operator()(int32_t e) const { return (uint32_t)home[e] < (uint32_t)R ? home[e] : R; }
};
struct SlotKey {
  const int32_t* slots;
  int32_t E;
  __device__ __forceinline__ int32_t operator()(int32_t s) const { return (uint32_t)slots[s] < (uint32_t)E ? slots[s] : E; }
};

struct Lists {
  const int32_t* home;
  const int32_t* slot_expert;
  int32_t* own_at;
  int32_t* rank_first;
  int32_t* slot_first;
  int32_t* slot_of;
  uint32_t* status;
};

// Block b < B: slots of problem b by expert.  Block B: experts by home rank.
__device__ void lists(const Lists& l, int32_t b, int32_t B, int32_t R, int32_t E, int32_t K, int32_t* cnt) {
  __shared__ int32_t part[kThreads / kWave];
  __shared__ int32_t bad;
  const int32_t S = R * K, n = b == B ? E : S, nkeys = b == B ? R : E;
  const HomeKey home{l.home, R};
  const SlotKey slot{l.slot_expert + (int64_t)b * S, E};
  if (threadIdx.x == 0) bad = 0;
  for (int32_t q = threadIdx.x; q <= nkeys; q += kThreads) cnt[q] = 0;
  __syncthreads();
  if (b == B) {
    order_counts<kThreads>(n, home, cnt);
  } else {
    order_counts<kThreads>(n, slot, cnt);
    for (int32_t e = threadIdx.x; e < E; e += kThreads)
      if (home(e) == R) bad = 1;
  }
  __syncthreads();
  order_sums<kThreads>(nkeys, b == B ? l.rank_first : l.slot_first + (int64_t)b * (E + 1), cnt, part);
  if (b < B && threadIdx.x == 0 && l.status) l.status[b] = bad ? TAOT_ST_BAD_INPUT : 0u;
  __syncthreads();
  if (threadIdx.x >= kWave || n == 0) return;
  if (b == B)
    order_positions<kRankBits>(n, R, home, [&](int32_t e, int32_t h, int32_t at) { l.own_at[e] = at + K * h; }, cnt);
  else
    order_positions<kExpertBits>(n, E - 1, slot, [&](int32_t s, int32_t, int32_t at) { l.slot_of[(int64_t)b * S + at] = s; },
                                 cnt);
}

// hist[row][chunk][e]: copies of expert e in the chunk; e = E: ids that are no
// expert.  The lists do not depend on the counts and take longer to start than to
// finish, so they ride along.
__global__ void __launch_bounds__(kThreads)
count_kernel(Lists l, int32_t B, int32_t R, int32_t K, const int32_t* __restrict__ ids, int64_t N, int32_t E,
             int32_t chunk, int32_t chunks, int32_t blocks_of_row, int waves, int32_t* __restrict__ hist) {
  extern __shared__ int32_t cnt[];
  if ((int32_t)blockIdx.x <= B) {
    lists(l, (int32_t)blockIdx.x, B, R, E, K, cnt);
    return;
  }
  const int lane = threadIdx.x & (kWave - 1), wid = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const uint32_t block = blockIdx.x - (uint32_t)B - 1, in_row = block % (uint32_t)blocks_of_row;
  const int32_t my_chunk = (int32_t)in_row * waves + wid;
  if (wid >= waves || my_chunk >= chunks) return;
  int32_t* mine = cnt + wid * (E + 1);
  const int64_t row = block / (uint32_t)blocks_of_row, job = row * chunks + my_chunk, lo = my_chunk * (int64_t)chunk;
  const int32_t n = (int32_t)min((int64_t)chunk, N - lo);
  const int32_t* src = ids + row * N + lo;
  for (int32_t e = lane; e <= E; e += kWave) mine[e] = 0;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  auto count = [&](int32_t e) { atomicAdd(&mine[(uint32_t)e < (uint32_t)E ? e : E], 1); };
  typedef int32_t four __attribute__((ext_vector_type(4)));
  typedef __attribute__((aligned(4))) four four_at;
  const int32_t n4 = n / 4;  // the order does not matter here: four ids a load
#pragma unroll 4
  for (int32_t i = lane; i < n4; i += kWave) {
    const four v = *reinterpret_cast<const four_at*>(src + 4 * i);
    count(v.x);
    count(v.y);
    count(v.z);
    count(v.w);
  }
  if (4 * n4 + lane < n) count(src[4 * n4 + lane]);
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  int32_t* dst = hist + job * (E + 1);
  for (int32_t e = lane; e <= E; e += kWave) dst[e] = mine[e];
}

// hist becomes the copies of e before the chunk; total[row][e] those of the row.
// A block has 64 experts of a row, 16 threads each, which share the chunks and
// hold up to kHeld counts each.
constexpr int kBaseThreads = 1024, kHeld = 16;
__global__ void __launch_bounds__(kBaseThreads)
bases_kernel(int32_t* __restrict__ hist, int32_t E, int32_t chunks, int32_t* __restrict__ total) {
  constexpr int kGroups = kBaseThreads / kWave;
  __shared__ int32_t part[kGroups][kWave];
  const int32_t tiles = (E + kWave) / kWave;
  const int64_t row = blockIdx.x / (uint32_t)tiles;
  const int32_t c = threadIdx.x % kWave, g = threadIdx.x / kWave, e = (int32_t)(blockIdx.x % (uint32_t)tiles) * kWave + c;
  const int32_t each = (chunks + kGroups - 1) / kGroups, lo = min(g * each, chunks), hi = min(lo + each, chunks);
  int32_t* h = hist + row * chunks * (E + 1) + e;
  int32_t sum = 0, v[kHeld];
  const bool held = each <= kHeld;
  if (e <= E) {
    if (held) {
#pragma unroll
      for (int u = 0; u < kHeld; ++u) v[u] = lo + u < hi ? h[(int64_t)(lo + u) * (E + 1)] : 0;
#pragma unroll
      for (int u = 0; u < kHeld; ++u) sum += v[u];
    } else {
#pragma unroll 8
      for (int32_t k = lo; k < hi; ++k) sum += h[(int64_t)k * (E + 1)];
    }
  }
  part[g][c] = sum;
  __syncthreads();
  if (e > E) return;
  int32_t run = 0;
#pragma unroll
  for (int w = 0; w < kGroups; ++w) run += w < g ? part[w][c] : 0;
  if (held) {
#pragma unroll
    for (int u = 0; u < kHeld; ++u) {
      if (lo + u < hi) h[(int64_t)(lo + u) * (E + 1)] = run;
      run += v[u];
    }
  } else {
#pragma unroll 8
    for (int32_t k = lo; k < hi; ++k) {
      const int32_t x = h[(int64_t)k * (E + 1)];
      h[(int64_t)k * (E + 1)] = run;
      run += x;
    }
  }
  if (g == kGroups - 1) total[row * (E + 1) + e] = run;
}

struct Tables {
  const int32_t* own_at;      // [E]          instance of an expert at home
  const int32_t* rank_first;  // [R + 1]      experts at ranks below
  const int32_t* slot_first;  // [B][E + 1]   filled slots of experts below
  const int32_t* slot_of;     // [B][S]       slots by expert
  const int32_t* total;       // [rows][E + 1]
  int64_t* upto;              // [rows][S + 1]  running sum of X over the slots by expert
  // [rows][E + S], of a row first its experts: copies at guests, and the position of occurrence 0, were it at home;
  // then its slots by expert: copies of the expert that slots before take, and the position of its occurrence 0, were
  // it this slot's
  int2* shares;
  int32_t* placed;            // [rows]       copies that go somewhere
};

// What a row's tables are made from and go to, in LDS or in memory.
struct Row {
  const int32_t* own_at;
  const int32_t* rank_first;
  const int32_t* first;
  const int32_t* slot_of;
  const int32_t* total;
  int64_t* upto;
  int32_t* off;
  int2* guest;
  int2* own;
};

// The whole block; returns the number of copies that go somewhere.  A barrier
// lies behind `off`, none behind `guest` and `own`.
__device__ __forceinline__ int32_t tables(const Row& t, const int32_t* expert, const int32_t* share, int32_t R,
                                          int32_t E, int32_t K, int32_t* sends, int64_t* part64, int32_t* part) {
  const int tid = threadIdx.x;
  const int32_t S = R * K, I = E + S, filled = t.first[E];
  auto guest_at = [&](int32_t s) { return s + t.rank_first[s / K + 1]; };
  auto at_guests = [&](int32_t e) { return min(t.upto[t.first[e + 1]] - t.upto[t.first[e]], (int64_t)t.total[e]); };
  int64_t run = 0;
  for (int32_t i0 = 0; i0 < filled; i0 += kTableThreads) {
    const int32_t i = i0 + tid;
    const int64_t x = i < filled ? (int64_t)max(share[t.slot_of[i]], 0) : 0;
    int64_t all;
    const int64_t at = run + block_exclusive<kTableThreads>(x, part64, &all);
    if (i < filled) t.upto[i] = at;
    run += all;
  }
  if (tid == 0) t.upto[filled] = run;
  for (int32_t s = tid; s < I; s += kTableThreads) t.off[s] = 0;  // slots that hold no expert
  __syncthreads();
  for (int32_t e = tid; e < E; e += kTableThreads) t.off[t.own_at[e]] = t.total[e] - (int32_t)at_guests(e);
  for (int32_t i = tid; i < filled; i += kTableThreads) {
    const int32_t s = t.slot_of[i], e = expert[s], n = t.total[e];
    const int32_t c = (int32_t)min(t.upto[i] - t.upto[t.first[e]], (int64_t)n);
    t.guest[i].x = c;
    t.off[guest_at(s)] = (int32_t)min((int64_t)(n - c), t.upto[i + 1] - t.upto[i]);
  }
  __syncthreads();
  int32_t sum = 0;
  for (int32_t i0 = 0; i0 < I; i0 += kTableThreads) {
    const int32_t i = i0 + tid;
    const int32_t v = i < I ? t.off[i] : 0;
    int32_t all;
    const int32_t at = sum + block_exclusive<kTableThreads>(v, part, &all);
    if (i < I) t.off[i] = at;
    sum += all;
  }
  if (tid == 0) t.off[I] = sum;
  __syncthreads();
  for (int32_t e = tid; e < E; e += kTableThreads) {
    const int32_t taken = (int32_t)at_guests(e);
    t.own[e] = int2{taken, t.off[t.own_at[e]] - taken};
  }
  for (int32_t i = tid; i < filled; i += kTableThreads) t.guest[i].y = t.off[guest_at(t.slot_of[i])] - t.guest[i].x;
  for (int32_t j = tid; j < R; j += kTableThreads)
    sends[j] = t.off[t.rank_first[j + 1] + K * (j + 1)] - t.off[t.rank_first[j] + K * j];
  return t.off[t.rank_first[R] + S];  // experts without a home rank lie behind all instances
}

// LDS: the running sums and instances lie in LDS.
template <bool LDS>
__global__ void __launch_bounds__(kTableThreads)
tables_kernel(Tables t, const int32_t* __restrict__ slot_expert, const int32_t* __restrict__ X, int32_t rows,
              int32_t rank0, int32_t R, int32_t E, int32_t K, int32_t* __restrict__ offsets,
              int32_t* __restrict__ sends, uint32_t* __restrict__ status) {
  extern __shared__ int64_t room[];
  __shared__ int64_t part64[kTableThreads / kWave];
  __shared__ int32_t part[kTableThreads / kWave];
  const int tid = threadIdx.x;
  const int64_t row = blockIdx.x, b = blockIdx.x / (uint32_t)rows;
  const int32_t S = R * K, I = E + S, r = rank0 + (int32_t)(blockIdx.x % (uint32_t)rows);
  int32_t* out = offsets + row * (I + 1);
  Row w{t.own_at, t.rank_first, t.slot_first + b * (E + 1), t.slot_of + b * S, t.total + row * (E + 1),
        LDS ? room : t.upto + row * (S + 1), LDS ? reinterpret_cast<int32_t*>(room + S + 1) : out,
        t.shares + row * (E + S) + E, t.shares + row * (E + S)};
  const int32_t placed = tables(w, slot_expert + b * S, X + (b * R + r) * (int64_t)S, R, E, K, sends + row * R, part64,
                                part);
  if (tid == 0) {
    t.placed[row] = placed;
    if (status && w.total[E] > 0) atomicOr(&status[b], TAOT_ST_BAD_ID);
  }
  const int32_t valid = t.rank_first[R] + S;
  if (LDS) {
    for (int32_t i = tid; i <= I; i += kTableThreads) out[i] = i <= valid ? w.off[i] : placed;
  } else {
    __syncthreads();
    for (int32_t i = valid + 1 + tid; i <= I; i += kTableThreads) out[i] = placed;
  }
}

// What the copies of an expert in a row go to, in LDS or in memory.
struct Shares {
  const int2* own;
  const int32_t* first;
  const int2* guest;
};

// A run of an expert's occurrences that go to one place: position = base + occurrence, below `end`.
struct Stretch {
  int32_t base, end;
};
// The wave's lanes that hold the same expert meet in an LDS word of the expert's:
// lanes in it, among those that are `in`; the word is 0 before and after.
__device__ __forceinline__ Same meet(unsigned long long* word, bool in, int lane) {
  if (in) __hip_atomic_fetch_or(word, 1ull << lane, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
  __builtin_amdgcn_wave_barrier();  // a wave's LDS operations are done in order
  const uint64_t all = __hip_atomic_load(word, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
  __builtin_amdgcn_wave_barrier();
  __hip_atomic_store(word, 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
  __builtin_amdgcn_wave_barrier();
  return Same{(uint32_t)all, (uint32_t)(all >> 32)};
}

__device__ __forceinline__ Stretch stretch(const Shares& s, int32_t e, int32_t j) {
  const int2 o = s.own[e];
  if (j >= o.x) return Stretch{o.y, INT32_MAX};
  int32_t a = s.first[e], z = s.first[e + 1];
  const int32_t last = z;
  while (a + 1 < z) {  // guest[a].x <= j < guest[z].x
    const int32_t mid = (a + z) / 2;
    if (s.guest[mid].x <= j) a = mid;
    else z = mid;
  }
  return Stretch{s.guest[a].y, a + 1 < last ? s.guest[a + 1].x : o.x};
}

// A wave: ids src[0 .. n) of a row, n > 0, in order; mine[e]: occurrences of e
// before them.  kKept: mine[e] holds the stretch of the next occurrence too (j,
// base, end), which most copies fall into, and `words` a word of each expert where
// its lanes meet.  Else E <= 2^BITS, the lanes compare their experts bit by bit and
// every copy looks its stretch up.
constexpr int kKept = 0;
constexpr int kKeptWords = 6;  // 32-bit words an expert and wave
template <int BITS>
__device__ __forceinline__ void place(const int32_t* __restrict__ src, int32_t n, int32_t E, int32_t* mine,
                                      const Shares& shares, int32_t placed, int32_t dropped,
                                      int32_t* __restrict__ dst, unsigned long long* words = nullptr) {
  const int lane = threadIdx.x & (kWave - 1);
  constexpr bool KEEP = BITS == kKept;
  int4* kept = reinterpret_cast<int4*>(mine);
  int32_t next[kUnroll];
  auto fetch = [&](int32_t i0) {  // past the end: the last id again
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) next[u] = src[min(i0 + u * kWave + lane, n - 1)];
  };
  fetch(0);
  for (int32_t i0 = 0; i0 < n; i0 += kUnroll * kWave) {
    int32_t e[kUnroll], j[kUnroll], p[kUnroll];
    Same m[kUnroll];
    bool in[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      in[u] = i0 + u * kWave + lane < n;
      e[u] = (uint32_t)next[u] < (uint32_t)E ? next[u] : E;
    }
    fetch(i0 + kUnroll * kWave);
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {  // ids that are no expert are one key more
      if constexpr (KEEP) {
        m[u] = meet(words + e[u], in[u], lane);
        continue;
      }
      const uint64_t experts = __ballot(in[u] & (e[u] < E)), others = __ballot(in[u] & (e[u] == E));
      m[u] = same_key<BITS>((uint32_t)e[u], experts);
      if (others != 0) {
        m[u].lo = e[u] < E ? m[u].lo : (uint32_t)others;
        m[u].hi = e[u] < E ? m[u].hi : (uint32_t)(others >> 32);
      }
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int below = m[u].below();
      const bool last = in[u] & (below + 1 == m[u].all());
      if constexpr (KEEP) {
        const int4 k = kept[e[u]];
        Stretch s{k.y, k.z};
        j[u] = k.x + below;
        if (j[u] >= s.end) s = stretch(shares, e[u], j[u]);
        p[u] = s.base + j[u];
        __builtin_amdgcn_wave_barrier();
        if (last) kept[e[u]] = int4{j[u] + 1, s.base, s.end, 0};
      } else {
        j[u] = mine[e[u]] + below;
        __builtin_amdgcn_wave_barrier();
        if (last) mine[e[u]] = j[u] + 1;
      }
      __builtin_amdgcn_wave_barrier();
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      if (!KEEP) p[u] = (e[u] < E ? stretch(shares, e[u], j[u]).base : dropped) + j[u];
      if (in[u]) dst[i0 + u * kWave + lane] = p[u] < placed ? p[u] : ~p[u];
    }
  }
}

// n words into LDS by `threads` threads, eight loads at a time.
__device__ __forceinline__ void bring(int32_t* to, const int32_t* __restrict__ from, int32_t n, int i, int threads) {
  for (; i < n; i += 8 * threads) {
    int32_t v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = from[min(i + u * threads, n - 1)];
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (i + u * threads < n) to[i + u * threads] = v[u];
  }
}

// BITS as in place().  kKept: the row's tables are brought into LDS too, which the
// waves' first stretches come from.  A block works on chunks of one row.
// 64 rows of 131072 ids, 256 experts: 28 us for 67 MB, bound by its instructions;
// 30 where the lanes compare experts bit by bit, 65 where every copy looks its
// stretch up as well.
template <int BITS>
__global__ void __launch_bounds__(kThreads)
place_kernel(const int32_t* __restrict__ ids, Tables t, const int32_t* __restrict__ hist, int64_t N, int32_t rows,
             int32_t E, int32_t S, int32_t chunk, int32_t chunks, int32_t blocks_of_row, int waves,
             int32_t* __restrict__ pos) {
  constexpr bool KEEP = BITS == kKept;
  extern __shared__ int4 stretches[];
  const int lane = threadIdx.x & (kWave - 1), wid = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const uint32_t at_row = blockIdx.x / (uint32_t)blocks_of_row;
  const int64_t row = at_row, b = at_row / (uint32_t)rows;
  const int32_t my_chunk = (int32_t)(blockIdx.x % (uint32_t)blocks_of_row) * waves + wid;
  const bool works = wid < waves && my_chunk < chunks;
  const int64_t job = row * chunks + (works ? my_chunk : 0), lo = my_chunk * (int64_t)chunk;
  Shares shares{t.shares + row * (E + S), t.slot_first + b * (E + 1), t.shares + row * (E + S) + E};
  const int32_t dropped = (int32_t)(N - t.total[row * (E + 1) + E]);  // where ids that are no expert begin
  int32_t* mine = reinterpret_cast<int32_t*>(stretches) + (KEEP ? 4 : 1) * wid * (E + 1);
  unsigned long long* words = reinterpret_cast<unsigned long long*>(stretches + waves * (E + 1));
  if constexpr (KEEP) {
    int32_t *own = reinterpret_cast<int32_t*>(words + waves * (E + 1)), *first = own + 2 * (E + S);
    int32_t j[4], f[4];
    const int32_t* base = hist + job * (E + 1);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      j[u] = base[min(lane + u * kWave, E)];
      f[u] = shares.first[min((int)threadIdx.x + u * kThreads, E)];
    }
    bring(own, reinterpret_cast<const int32_t*>(shares.own), 2 * (E + S), threadIdx.x, kThreads);
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if ((int)threadIdx.x + u * kThreads <= E) first[threadIdx.x + u * kThreads] = f[u];
    if (E >= 4 * kThreads) bring(first, shares.first, E + 1, threadIdx.x + 4 * kThreads, kThreads);
    shares = Shares{reinterpret_cast<const int2*>(own), first, reinterpret_cast<const int2*>(own) + E};
    for (int32_t e = threadIdx.x; e < waves * (E + 1); e += kThreads) words[e] = 0;
    __syncthreads();
    if (!works) return;
    int4* kept = reinterpret_cast<int4*>(mine);
    for (int32_t e0 = lane; e0 <= E; e0 += 4 * kWave) {
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int32_t e = e0 + u * kWave;
        if (e > E) continue;
        Stretch s{dropped, INT32_MAX};
        if (e < E) s = stretch(shares, e, j[u]);
        kept[e] = int4{j[u], s.base, s.end, 0};
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) j[u] = base[min(e0 + (u + 4) * kWave, E)];
    }
  } else {
    if (!works) return;
    bring(mine, hist + job * (E + 1), E + 1, lane, kWave);
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  const int32_t n = (int32_t)min((int64_t)chunk, N - lo);
  place<BITS>(ids + row * N + lo, n, E, mine, shares, t.placed[row], dropped, pos + row * N + lo, words + wid * (E + 1));
}

// A short row by one block and in one launch: everything above, in LDS.
struct RowRoom {
  size_t rank_cnt, slot_cnt, own_at, rank_first, first, slot_of, total, upto, off, guest, own, hist, bytes;
};
__host__ __device__ inline RowRoom row_room(int32_t R, int32_t E, int32_t S, int waves) {
  RowRoom r{};
  size_t at = 0;
  auto take = [&](size_t n) {
    const size_t was = at;
    at += (n + 7) / 8 * 8;
    return was;
  };
  r.upto = take((size_t)(S + 1) * 8);
  r.guest = take((size_t)S * 8);
  r.own = take((size_t)E * 8);
  r.rank_cnt = take((size_t)(R + 1) * 4);
  r.slot_cnt = take((size_t)(E + 1) * 4);
  r.own_at = take((size_t)E * 4);
  r.rank_first = take((size_t)(R + 1) * 4);
  r.first = take((size_t)(E + 1) * 4);
  r.slot_of = take((size_t)S * 4);
  r.total = take((size_t)(E + 1) * 4);
  r.off = take((size_t)(E + S + 1) * 4);
  r.hist = take((size_t)waves * (E + 1) * 4);
  r.bytes = at;
  return r;
}

template <int BITS>
__global__ void __launch_bounds__(kTableThreads)
row_kernel(const int32_t* __restrict__ home, const int32_t* __restrict__ slot_expert, const int32_t* __restrict__ X,
           const int32_t* __restrict__ ids, int32_t N, int32_t rows, int32_t rank0, int32_t R, int32_t E, int32_t K,
           int waves, int32_t* __restrict__ pos, int32_t* __restrict__ offsets, int32_t* __restrict__ sends,
           uint32_t* __restrict__ bad) {
  extern __shared__ int64_t room[];
  __shared__ int64_t part64[kTableThreads / kWave];
  __shared__ int32_t part[kTableThreads / kWave];
  __shared__ int32_t bad_home;
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wid = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int64_t row = blockIdx.x, b = blockIdx.x / (uint32_t)rows;
  const int32_t S = R * K, I = E + S, r = rank0 + (int32_t)(blockIdx.x % (uint32_t)rows);
  const RowRoom at = row_room(R, E, S, waves);
  char* base = reinterpret_cast<char*>(room);
  auto words = [&](size_t o) { return reinterpret_cast<int32_t*>(base + o); };
  int32_t *own_at = words(at.own_at), *rank_first = words(at.rank_first), *first = words(at.first),
          *slot_of = words(at.slot_of), *total = words(at.total), *hist = words(at.hist), *rank_cnt = words(at.rank_cnt),
          *slot_cnt = words(at.slot_cnt);
  int2 *guest = reinterpret_cast<int2*>(base + at.guest), *own = reinterpret_cast<int2*>(base + at.own);
  // `waves` runs of the row, in order
  const int32_t run = (N + waves * kWave - 1) / (waves * kWave) * kWave, lo = min(wid * run, N), n = min(run, N - lo);
  const int32_t* src = ids + row * N + lo;
  int32_t* mine = hist + wid * (E + 1);
  if (tid == 0) bad_home = 0;
  for (int32_t q = tid; q <= R; q += kTableThreads) rank_cnt[q] = 0;
  for (int32_t q = tid; q <= E; q += kTableThreads) slot_cnt[q] = 0;
  if (wid < waves)
    for (int32_t e = lane; e <= E; e += kWave) mine[e] = 0;
  const HomeKey home_key{home, R};
  const SlotKey slot_key{slot_expert + b * S, E};
  __syncthreads();
  order_counts<kTableThreads>(E, home_key, rank_cnt);
  order_counts<kTableThreads>(S, slot_key, slot_cnt);
  for (int32_t e = tid; e < E; e += kTableThreads)
    if (home_key(e) == R) bad_home = 1;
  __syncthreads();
  order_sums<kTableThreads>(R, rank_first, rank_cnt, part);
  order_sums<kTableThreads>(E, first, slot_cnt, part);
  __syncthreads();
  // the last two waves order the experts and the slots, the ids' runs begin with the first
  if (wid == kTableThreads / kWave - 1)
    order_positions<kRankBits>(E, R, home_key, [&](int32_t e, int32_t h, int32_t at) { own_at[e] = at + K * h; }, rank_cnt);
  if (wid == kTableThreads / kWave - 2 && S > 0)
    order_positions<BITS>(S, E - 1, slot_key, [&](int32_t s, int32_t, int32_t at) { slot_of[at] = s; }, slot_cnt);
  if (wid < waves) {
    for (int32_t i = lane; i < n; i += kWave) {
      const int32_t e = src[i];
      atomicAdd(&mine[(uint32_t)e < (uint32_t)E ? e : E], 1);
    }
  }
  __syncthreads();
  for (int32_t e = tid; e <= E; e += kTableThreads) {
    int32_t sum = 0;
    for (int w = 0; w < waves; ++w) {
      const int32_t v = hist[w * (E + 1) + e];
      hist[w * (E + 1) + e] = sum;
      sum += v;
    }
    total[e] = sum;
  }
  __syncthreads();
  Row w{own_at, rank_first, first, slot_of, total, reinterpret_cast<int64_t*>(base + at.upto), words(at.off), guest, own};
  const int32_t placed =
      tables(w, slot_expert + b * S, X + (b * R + r) * (int64_t)S, R, E, K, sends + row * R, part64, part);
  int32_t* out = offsets + row * (I + 1);
  const int32_t valid = rank_first[R] + S;
  for (int32_t i = tid; i <= I; i += kTableThreads) out[i] = i <= valid ? w.off[i] : placed;
  if (tid == 0) bad[row] = (bad_home ? TAOT_ST_BAD_INPUT : 0u) | (total[E] > 0 ? TAOT_ST_BAD_ID : 0u);
  __syncthreads();
  if (wid < waves && n > 0)
    place<BITS>(src, n, E, mine, Shares{own, first, guest}, placed, N - total[E], pos + row * N + lo);
}

// status[b] of the rows' bits, a wave a problem.
__global__ void __launch_bounds__(kWave)
status_kernel(const uint32_t* __restrict__ bad, int32_t rows, uint32_t* __restrict__ status) {
  const int64_t b = blockIdx.x;
  uint32_t s = 0;
  for (int32_t r = threadIdx.x; r < rows; r += kWave) s |= bad[b * rows + r];
  const uint64_t input = __ballot((s & TAOT_ST_BAD_INPUT) != 0), ids = __ballot((s & TAOT_ST_BAD_ID) != 0);
  if (threadIdx.x == 0) status[b] = (input ? TAOT_ST_BAD_INPUT : 0u) | (ids ? TAOT_ST_BAD_ID : 0u);
}

// The token of a group of WAVES waves, among `all`, and the first row of its row of copies.
struct Token {
  int64_t t, row0;
};
template <int WAVES>
__device__ __forceinline__ Token token_of(uint32_t first, int64_t tokens, int32_t k) {
  const uint32_t t = first + blockIdx.x * (4 / WAVES) + __builtin_amdgcn_readfirstlane(threadIdx.x / (WAVES * kWave));
  return Token{t, (int64_t)(t / (uint32_t)tokens) * tokens * k};
}

// ---- rows ------------------------------------------------------------------------
// A row of `bytes` bytes, 16 a lane and step; a token's waves read it once and
// write its k copies.  Bound by the writes: 8192 tokens of 4096 bytes and 128 of
// scales, 8 copies: 53 us for 302 MB, 5.7 TB/s.
struct Payload {
  const char* in;
  char* out;
  int64_t bytes;
};

template <int WAVES, bool FAR>
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
        if constexpr (FAR) __builtin_nontemporal_store(w, reinterpret_cast<u32x4_at*>(dst));
        else *reinterpret_cast<u32x4_at*>(dst) = w;
      } else {
#pragma unroll
        for (int u = 0; u < 16; ++u)
          if (u < n) dst[u] = (char)(w[u / 4] >> (8 * (u % 4)));
      }
    }
  }
}

template <int WAVES, bool FAR>
__global__ void __launch_bounds__(256)
rows_kernel(Payload a, Payload b, uint32_t first, int64_t all, int64_t tokens, int32_t k, const int32_t* __restrict__ pos) {
  constexpr int kLanes = WAVES * kWave;
  const auto [t, row0] = token_of<WAVES>(first, tokens, k);
  if (t >= all) return;
  const int lane = threadIdx.x % kLanes;
  const int64_t N = tokens * k;
  spread<WAVES, FAR>(a, t, row0, N, k, pos + t * k, lane);
  if (b.in) spread<WAVES, false>(b, t, row0, N, k, pos + t * k, lane);
}

// out = sum w y[pos], in the order of the choices; kAhead copies at a time, so that
// their loads are in flight together.  8192 tokens of 2048 in 16 bits, 8 copies:
// 58 us for 302 MB, 5.2 TB/s.
template <typename T, int WAVES>
__global__ void __launch_bounds__(256)
combine_kernel(const T* __restrict__ y, const int32_t* __restrict__ pos, const float* __restrict__ weights,
               uint32_t first, int64_t all, int64_t tokens, int32_t k, int32_t H, T* __restrict__ out) {
  constexpr int kLanes = WAVES * kWave;
  constexpr int kAhead = 4;
  const auto [t, row0] = token_of<WAVES>(first, tokens, k);
  if (t >= all) return;
  const int lane = threadIdx.x % kLanes;
  const int64_t N = tokens * k;
  const T* base = y + row0 * H;
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

// dy[pos] = w dout, dw = <dout, y[pos]>; kAhead copies at a time.  8192 tokens of
// 2048 in 16 bits, 8 copies: 112 us for 570 MB, 5.1 TB/s; 119 through the caches.
template <typename T, int WAVES, bool FAR>
__global__ void __launch_bounds__(256)
combine_backward_kernel(const T* __restrict__ dout, const T* __restrict__ y, const int32_t* __restrict__ pos,
                        const float* __restrict__ weights, uint32_t first, int64_t all, int64_t tokens, int32_t k, int32_t H,
                        T* __restrict__ dy, float* __restrict__ dweights) {
  using Raw = typename Row8<T>::vec;
  constexpr int kLanes = WAVES * kWave, kAhead = 4;
  __shared__ float part[2][kAhead][4];
  const auto [t, row0] = token_of<WAVES>(first, tokens, k);
  if (t >= all) return;  // whole waves, and whole blocks where waves share a token
  const int lane = threadIdx.x % kLanes;
  const int64_t N = tokens * k;
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
          store_row<FAR>(p, o, n);
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
  p.t.shares = c.take<int2>(n * (E + S));
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

// f by the number of bits of an expert (MOST at most), as a constant that is large enough.
template <int MOST, typename F>
auto with_bits(int bits, F f) {
  if (bits <= 6) return f(std::integral_constant<int, 6>());
  if (bits <= 8) return f(std::integral_constant<int, 8>());
  if (bits <= 9) return f(std::integral_constant<int, 9>());
  if constexpr (MOST > 12) {
    if (bits > 12) return f(std::integral_constant<int, MOST>());
  }
  return f(std::integral_constant<int, 12>());
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
  const int32_t batch = (int32_t)(kMaxBlocks / rows / ((E + kWave) / kWave)), S = R * K;
  if (B > batch) {  // one after the other in the same workspace; so many rows have the longest chunks
    for (int32_t b = 0; b < B; b += batch) {
      const int64_t row = (int64_t)b * rows;
      if (taot_status s = launch_dispatch_map(ids + row * N, B - b < batch ? B - b : batch, rows, rank0, N, home, R, E, K,
                                              slot_expert + (int64_t)b * S, X + (int64_t)b * R * S, pos + row * N,
                                              offsets + row * (E + S + 1), sends + row * R, status ? status + b : nullptr,
                                              ws, stream))
        return s;
    }
    return TAOT_OK;
  }
  const int64_t n = (int64_t)B * rows;
  const int32_t chunk = chunk_of(n, N, E), chunks = (int32_t)((N + chunk - 1) / chunk);
  const int32_t I = E + S, most = E > R ? E : R;
  const Lists lists{home, slot_expert, p.own_at, p.rank_first, p.slot_first, p.slot_of, status};
  const size_t list_lds = (size_t)(most + 1) * sizeof(int32_t), row_lds = (size_t)(E + 1) * sizeof(int32_t);
  const int waves = 4 * row_lds <= 65536 ? 4 : 2 * row_lds <= 65536 ? 2 : 1;
  const size_t count_lds = waves * row_lds > list_lds ? waves * row_lds : list_lds;
  const int bits = bits_for((uint32_t)E - 1);
  if (N <= kRowIds) {
    const int wanted = (int)((N + kWave - 1) / kWave), row_waves = wanted < 1 ? 1 : wanted < 16 ? wanted : 16;
    const size_t lds = row_room(R, E, S, row_waves).bytes;
    if (lds <= kRowLds) {
      // an expert takes 32 bytes of a row's LDS and more: no 4096 of them fit
      static_assert(kRowLds < 32 << 12, "bits of an expert of a short row");
      auto* kernel = with_bits<12>(bits, [](auto n) { return row_kernel<n.value>; });
      if (!allow_lds(reinterpret_cast<const void*>(kernel), lds)) return TAOT_ERR_LAUNCH;
      // one row a problem: its bits are the problem's status
      uint32_t* bad = status && rows == 1 ? status : reinterpret_cast<uint32_t*>(p.t.placed);
      kernel<<<(unsigned)n, kTableThreads, lds, stream>>>(home, slot_expert, X, ids, (int32_t)N, rows, rank0, R, E, K,
                                                          row_waves, pos, offsets, sends, bad);
      if (status && rows > 1)
        status_kernel<<<(unsigned)B, kWave, 0, stream>>>(bad, rows, status);
      return hipGetLastError() == hipSuccess ? TAOT_OK : TAOT_ERR_LAUNCH;
    }
  }
  if (!allow_lds(reinterpret_cast<const void*>(count_kernel), count_lds)) return TAOT_ERR_LAUNCH;
  const int32_t blocks = chunks > 0 ? (chunks + waves - 1) / waves : 1;  // of a row
  count_kernel<<<(unsigned)(B + 1 + (chunks > 0 ? n * blocks : 0)), kThreads, count_lds, stream>>>(
      lists, B, R, K, ids, N, E, chunk, chunks, blocks, waves, p.hist);
  bases_kernel<<<(unsigned)(n * ((E + kWave) / kWave)), kBaseThreads, 0, stream>>>(p.hist, E, chunks, p.total);
  const size_t table_lds = (size_t)(S + 1) * sizeof(int64_t) + (size_t)(I + 1) * sizeof(int32_t);
  const bool small_tables = table_lds <= kTableLds;
  (small_tables ? tables_kernel<true> : tables_kernel<false>)<<<(unsigned)n, kTableThreads, small_tables ? table_lds : 0,
                                                               stream>>>(p.t, slot_expert, X, rows, rank0, R, E, K,
                                                                         offsets, sends, status);
  if (chunks > 0) {
    auto kept = [&](int w) { return kKeptWords * w * row_lds + (size_t)(E + S) * sizeof(int2) + row_lds; };
    int place_waves = 4;
    while (place_waves > 1 && kept(place_waves) > kKeepLds) place_waves /= 2;
    const int64_t brought = 2 * (int64_t)(E + S) + E + 1, placed = (int64_t)place_waves * chunk;
    const bool keep = kept(place_waves) <= kKeepLds && brought <= kBroughtWords * placed;
    if (!keep) place_waves = waves;
    const int32_t place_blocks = (chunks + place_waves - 1) / place_waves;
    const size_t lds = keep ? kept(place_waves) : waves * row_lds;
    auto* kernel = keep ? place_kernel<kKept> : with_bits<kExpertBits>(bits, [](auto n) { return place_kernel<n.value>; });
    if (!allow_lds(reinterpret_cast<const void*>(kernel), lds)) return TAOT_ERR_LAUNCH;
    kernel<<<(unsigned)(n * place_blocks), kThreads, lds, stream>>>(ids, p.t, p.hist, N, rows, E, S, chunk, chunks,
                                                                  place_blocks, place_waves, pos);
  }
  return hipGetLastError() == hipSuccess ? TAOT_OK : TAOT_ERR_LAUNCH;
}

// f(first token, blocks) for all tokens, `per` of them a block.
template <typename F>
void by_blocks(int64_t all, int per, F f) {
  for (int64_t t = 0; t < all; t += kMaxBlocks * per) {
    const int64_t n = all - t < kMaxBlocks * per ? all - t : kMaxBlocks * per;
    f((uint32_t)t, (unsigned)((n + per - 1) / per));
  }
}

taot_status launch_dispatch_rows(const void* x, int64_t row_bytes, const void* x_more, int64_t more_bytes,
                                 int64_t rows, int64_t tokens, int32_t k, const int32_t* pos, void* out,
                                 void* out_more, hipStream_t stream) {
  const Payload a{static_cast<const char*>(x), static_cast<char*>(out), row_bytes};
  const Payload b{static_cast<const char*>(x_more), static_cast<char*>(out_more), more_bytes};
  const int64_t all = rows * tokens;
  with_far(all * k * (row_bytes + more_bytes), [&](auto far) {
    const bool wide = row_bytes > 2048;
    auto* kernel = wide ? rows_kernel<4, far.value> : rows_kernel<1, far.value>;
    by_blocks(all, wide ? 1 : 4, [&](uint32_t first, unsigned blocks) {
      kernel<<<blocks, 256, 0, stream>>>(a, b, first, all, tokens, k, pos);
    });
  });
  return hipGetLastError() == hipSuccess ? TAOT_OK : TAOT_ERR_LAUNCH;
}

taot_status launch_combine_rows(const void* y, const int32_t* pos, const float* weights, int64_t rows, int64_t tokens,
                                int32_t k, int32_t H, int32_t dtype, void* out, hipStream_t stream) {
  const int64_t all = rows * tokens;
  return by_type(dtype, [&](auto z) {
    using T = decltype(z);
    const T* in = static_cast<const T*>(y);
    auto* kernel = H > 1024 ? combine_kernel<T, 4> : combine_kernel<T, 1>;
    by_blocks(all, H > 1024 ? 1 : 4, [&](uint32_t first, unsigned blocks) {
      kernel<<<blocks, 256, 0, stream>>>(in, pos, weights, first, all, tokens, k, H, static_cast<T*>(out));
    });
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
    with_far(all * k * H * (int64_t)sizeof(T), [&](auto far) {
      auto* kernel = H > 1024 ? combine_backward_kernel<T, 4, far.value> : combine_backward_kernel<T, 1, far.value>;
      by_blocks(all, H > 1024 ? 1 : 4, [&](uint32_t first, unsigned blocks) {
        kernel<<<blocks, 256, 0, stream>>>(d, in, pos, weights, first, all, tokens, k, H, o, dweights);
      });
    });
  });
}

}  // namespace taot
